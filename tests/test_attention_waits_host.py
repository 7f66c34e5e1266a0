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
