"""Which kernels the GPU tests of shared rows reach: they make up their sizes for the rules that choose them, which stand in the sources as written here."""
import os

import pytest

from tests.test_gpu_attention import behind_empty

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_19269_amd", "csrc")

RULES = {"attention.hip": ["if (p.Tk <= 64) return 1;", "const int64_t room = p.D > 64 ? 288 : 576;",
                           "return attn_about(p.Tq, p.n_seqs, 32) * p.heads <= room ? 4 : attn_about(p.Tq, p.n_seqs, 64) * p.heads <= 2 * room ? 2 : 1;"],
         "attention_bwd.hip": ["const int64_t room = p.f.D > 64 ? 288 : 576;",
                               "return p.f.D <= 64 && attn_about(p.f.Tq, p.f.n_seqs, 32) * p.f.heads <= room ? 4 : attn_about(p.f.Tq, p.f.n_seqs, 64) * p.f.heads <= 2 * room ? 2 : 1;",
                               "return attn_about(p.f.Tk, p.f.n_seqs, 32) * p.f.kv_heads <= 512 ? 32 : 64;"],
         "attn_launch.hpp": ["return ((int64_t)T - 1) / rows + 1 + (n_seqs - 1) / 2;"],
         "attention_cached.hip": ["return Tq * group > 32 * (int64_t)n_seqs;"]}


@pytest.mark.parametrize("file", sorted(RULES))
def test_the_rules_are_those_that_the_tests_reckon_with(file):
    text = open(os.path.join(CSRC, file)).read()
    for rule in RULES[file]:
        assert text.count(rule) == 1, rule


def about(T, n_seqs, rows):
    return (T + rows - 1) // rows + (n_seqs - 1) // 2 if T else 1 + (n_seqs - 1) // 2


def split(T, n_seqs, heads, D, forward):
    room = 288 if D > 64 else 576
    if (forward or D <= 64) and about(T, n_seqs, 32) * heads <= room:
        return 4
    return 2 if about(T, n_seqs, 64) * heads <= 2 * room else 1


@pytest.mark.parametrize("D", [40, 64, 96, 128])
@pytest.mark.parametrize("streams", [1, 2, 4])
@pytest.mark.parametrize("lens", [[65], [129, 31, 1], [257, 0, 64], [300], [300, 140], [77], [150], [130]])
def test_sizes_of_the_tests_of_shared_rows(lens, streams, D):
    """Four heads over two: as many streams as the test says (dQ has two where there would be four of 128 columns), 64 keys a workgroup for one stream, else 32 in some"""
    n = len(lens) + behind_empty(D, 4, streams)
    T = sum(lens)
    assert split(T, n, 4, D, True) == streams
    assert split(T, n, 4, D, False) == (min(streams, 2) if D > 64 else streams)
    keys = 32 if about(T, n, 32) * 2 <= 512 else 64
    assert keys == {1: 64, 4: 32}.get(streams, keys)
