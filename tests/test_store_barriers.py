"""The LDS counters of the kernels over the 4-bit store, read from the source (no run
can show a missing barrier dependably)."""
import os
import re

from test_lds_barriers import CSRC, kernel_body


def test_counters_in_lds_go_through_the_wave_barriers():
    """A lane's branch around an LDS counter joined with another one across a loop's
    back edge lets the other lanes run ahead, so the kernels over the store have one
    such branch, between wave barriers."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "attn_store.hip")).read())
    m = re.search(r"void wave_add_one\(int\* counter\) \{(.*?)\n\}", text, re.S)
    assert re.sub(r"\s+", "", m.group(1)) == (
        "__builtin_amdgcn_wave_barrier();if(__lane_id()==0)atomicAdd(counter,1);"
        "__builtin_amdgcn_wave_barrier();")
    rest = text.replace(m.group(1), "")
    assert "atomicAdd" not in rest and "fetch_add" not in rest
    assert "wave_add_one(&merged)" in kernel_body("attn_store.hip", "attn_quant_kernel")
