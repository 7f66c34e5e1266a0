"""Quantising to 8 bits with block scales and back, on the GPU, against the definition in 64 bits: every byte."""
import numpy as np
import pytest
import torch

from paper_2605_19269_amd import coda
from tests import q8_ref as R

pytestmark = pytest.mark.gpu


def guarded(rows, cols, fill=0xA5):
    """A [rows x cols] view at a pitch of whole sixteens, and more, in a buffer of one value; and a check that the rest still has it."""
    pitch = (cols + 15) // 16 * 16 + 32
    full = torch.full((rows + 2, pitch), fill, dtype=torch.uint8, device="cuda")

    def untouched():
        c = full.clone()
        c[1:1 + rows, :cols] = fill
        assert bool((c == fill).all()), "bytes outside the output were written"
    return full[1:1 + rows, :cols], untouched


def inputs(rows, cols, seed, pad=0):
    """bf16 with rows of every size, zero blocks, largest values at the borders of a scale, infinities, NaN and subnormals."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-20, 20, (rows, 1), generator=g).float())
    x = x.to(torch.bfloat16)
    v = x.view(-1)
    n = v.numel()
    pick = lambda k: torch.randint(0, n, (k,), generator=g)
    if rows > 3:
        x[1] = 0
        x[2] = (torch.randn(cols, generator=g) * 1e-39).to(torch.bfloat16)
        x[3, : min(cols, 128)] = float("nan")
    if rows > 6:
        x[4] = (torch.rand(cols, generator=g) * 2 - 1).to(torch.bfloat16)
        x[4, ::64] = 1.75                        # at the border, and the next value behind it
        x[5] = x[4]
        x[5, ::64] = 1.7578125
        x[6] = 3.38e38
        v[pick(2)] = float("inf")
        v[pick(2)] = float("-inf")
        v[pick(2)] = float("nan")
    out = torch.zeros(rows, cols + pad, dtype=torch.bfloat16, device="cuda")[:, :cols]
    out.copy_(x)
    return x.double(), out


def check_codes(codes, byte_per_element, x):
    """Finite elements have the bytes of the nearest code (the sign of a zero is the element's), the others are NaN."""
    v = R.decode(codes.cpu())
    fin = torch.isfinite(x)
    want = R.round_e4m3(torch.where(fin, x, torch.zeros_like(x)) / byte_per_element)
    assert torch.isnan(v[~fin]).all()
    assert torch.equal(v[fin], want[fin])


SIZES = [(1, 8), (1, 128), (3, 16), (7, 136), (16, 128), (17, 392), (33, 4096), (64, 264), (130, 1000), (509, 5632)]


@pytest.mark.parametrize("rows,cols", SIZES + [(4099, 2056)])       # the last in passes of four
def test_rows(rows, cols):
    x, X = inputs(rows, cols, rows + cols, pad=8 * (rows % 3))
    q, q_ok = guarded(rows, cols)
    s, s_ok = guarded(R.blocks(cols), rows)
    coda.coda_quantize(X, q, s)
    torch.cuda.synchronize()
    q_ok(); s_ok()
    byte, per = R.along_rows(x)
    assert torch.equal(s.cpu().long(), byte)
    check_codes(q, per, x)


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("both", [True, False])
def test_square_blocks(rows, cols, both):
    x, X = inputs(rows, cols, rows + cols, pad=8 * (rows % 3))
    q, q_ok = guarded(rows, cols)
    s, s_ok = guarded(R.blocks(cols), rows)
    st, st_ok = guarded(R.blocks(rows), cols)
    coda.coda_quantize(X, q, s, scales_t=st if both else None, square=True)
    torch.cuda.synchronize()
    q_ok(); s_ok(); st_ok()
    along_rows, along_cols, per = R.square(x)
    assert torch.equal(s.cpu().long(), along_rows)
    assert torch.equal(st.cpu().long(), along_cols) if both else bool((st == 0xA5).all())
    check_codes(q, per, x)


@pytest.mark.parametrize("rows,cols", SIZES + [(4099, 2056)])
def test_restore(rows, cols):
    g = torch.Generator().manual_seed(rows * cols)
    q, q_ok = guarded(rows, cols)
    s, s_ok = guarded(R.blocks(cols), rows)
    q.copy_(torch.randint(0, 256, (rows, cols), generator=g, dtype=torch.int64).to(torch.uint8))
    s.copy_(torch.randint(0, 256, (R.blocks(cols), rows), generator=g, dtype=torch.int64).to(torch.uint8))
    full = torch.full((rows + 2, cols + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    out = full[1:1 + rows, :cols]
    coda.coda_dequantize(q, s, out)
    torch.cuda.synchronize()
    want = R.decode(q.cpu()) * R.per_element(s.cpu(), rows, cols)
    got = out.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fine = ~torch.isnan(want)
    # 448 * 2^127 and the like are beyond bf16: infinities; the rest is exact down to 2^-133, below that off by half of it
    want = want.to(torch.bfloat16).double()
    assert torch.equal(got[fine], want[fine])
    guard = full.clone()
    guard[1:1 + rows, :cols] = 7.0
    assert bool((guard == 7.0).all())


def test_restore_undoes_quantising():
    x, X = inputs(200, 640, 5)
    x, X = x[7:], X[7:]
    q, s = torch.empty(193, 640, dtype=torch.uint8, device="cuda"), torch.empty(5, 208, dtype=torch.uint8, device="cuda")
    out = torch.empty(193, 640, dtype=torch.bfloat16, device="cuda")
    coda.coda_quantize(X, q, s)
    coda.coda_dequantize(q, s, out)
    again, s2 = torch.empty_like(q), torch.empty_like(s)
    coda.coda_quantize(out, again, s2)                       # what has been rounded once stays
    back = torch.empty_like(out)
    coda.coda_dequantize(again, s2, back)
    fin = torch.isfinite(x)
    d, (_, per) = out.cpu().double(), R.along_rows(x)
    assert torch.equal(torch.isnan(d), ~fin)
    # half a step: 2^-4 of the value, or of the format's least normal value 2^-6
    assert ((d - x).abs()[fin] <= torch.maximum(x.abs(), per * 2.0 ** -6)[fin] * 2.0 ** -4).all()
    assert torch.equal(torch.nan_to_num(back.float(), 0.0), torch.nan_to_num(out.float(), 0.0))


def test_pitched_scales_of_a_longer_batch_are_left_alone():
    """Rows 48 .. 100 of a buffer of scales for 160: its neighbours belong to other sequences."""
    x, X = inputs(52, 256, 9)
    q = torch.empty(52, 256, dtype=torch.uint8, device="cuda")
    s = torch.full((2, 160), 0x5A, dtype=torch.uint8, device="cuda")
    coda.coda_quantize(X, q, s[:, 48:100])
    assert torch.equal(s[:, 48:100].cpu().long(), R.along_rows(x)[0])
    s[:, 48:100] = 0x5A
    assert bool((s == 0x5A).all())


def test_float8_tensors_are_taken_too():
    x, X = inputs(40, 256, 3)
    q, s = torch.empty(40, 256, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(2, 48, dtype=torch.float8_e8m0fnu, device="cuda")
    coda.coda_quantize(X, q, s)
    out = torch.empty(40, 256, dtype=torch.bfloat16, device="cuda")
    coda.coda_dequantize(q, s, out)
    want = R.decode(q.view(torch.uint8).cpu()) * R.per_element(s.view(torch.uint8).cpu(), 40, 256)
    assert np.array_equal(out.cpu().double().numpy(), want.to(torch.bfloat16).double().numpy(), equal_nan=True)
