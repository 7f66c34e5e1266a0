"""What a barrier of the attention kernels publishes has arrived: the loads that go to LDS directly are not in the compiler's wait counts, so the wait has to be in the
source, whatever the compiler happens to wait for at that place."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_19269_amd", "csrc")


def kernel(file, name):
    text = open(os.path.join(CSRC, file)).read()
    begin = text.index("void %s(" % name)
    return re.sub(r"//[^\n]*", "", text[begin: text.index("\n}\n", begin)])


def test_values_in_lds_have_arrived_ahead_of_every_first_barrier():
    """dK's kernel at 128 columns: all waves load a part of V's tile and all read the whole of it"""
    text = kernel("attention_bwd.hip", "attention_dkv_kernel")
    begin = text.index("key0, k.count, v_tile)")
    rounds = text.index("for (int i = 0; i < rounds")
    inside = text.index("attn_barrier()", rounds)                           # where waves that had none before have their first
    assert "attn_wait()" in text[rounds: inside]
    before = [m.start() for m in re.finditer(r"attn_barrier\(\)", text[begin: rounds])]
    assert before, "no wave has a barrier ahead of the rounds"
    for at in before:
        statement = text[:begin + at].rsplit("{", 1)[-1] if "{" in text[begin + at - 80: begin + at] else ""
        assert "attn_wait()" in statement, text[begin + at - 80: begin + at + 20]


def test_no_shared_tile_is_changed_while_others_read_it():
    """The gradients' kernels: rows of a tile are read for S and dP by waves that a barrier has to hold before anyone clears what is not finite in it"""
    text = kernel("attention_bwd.hip", "attention_dkv_kernel")
    loop = text[text.index("for (int i = 0; i < rounds"):]
    products = loop.rindex("attn_rows<DP>(rows, ROWS")                      # the last that reads rows
    assert products < loop.index("attn_barrier()", products) < loop.index("attn_clean(")
    text = kernel("attention_bwd.hip", "attention_dq_kernel")
    assert text.count("attn_clean(") == 1
    clean = text[text.index("const auto clean"):]
    clean = clean[: clean.index("};")]
    assert clean.index("attn_barrier()") < clean.index("attn_clean(") < clean.index("attn_reads_done()") < clean.rindex("attn_barrier()")
