"""Barriers of the kernels that avoid the full workgroup fence, read from the
sources: a kernel whose waves store to LDS publishes it by barrier_lds (each
wave waits for its own stores first); barrier_nofence alone is for kernels
whose LDS is written by direct global->LDS loads only.  No run can show a
missing wait dependably, so the call sites are checked instead."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2607_25422_amd", "csrc")


def kernel_body(source, name):
    """Text of kernel `name`, from its name to the brace that closes it."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, source)).read())
    m = re.search(r"__global__[^;{]*\b" + name + r"\s*\(", text)
    assert m, name
    i = text.index("{", m.end())
    depth, j = 1, i + 1
    while depth:
        depth += {"{": 1, "}": -1}.get(text[j], 0)
        j += 1
    return text[i:j]


@pytest.mark.parametrize("source,name", [("mlp.hip", "mlp_score_kernel"),
                                         ("attn.hip", "attn_sparse_kernel")])
def test_kernels_that_store_to_lds_wait_for_their_stores(source, name):
    body = kernel_body(source, name)
    assert "barrier_lds()" in body
    assert "barrier_nofence()" not in body and "builtin_amdgcn_s_barrier" not in body


@pytest.mark.parametrize("name", ["proj_gemm_kernel", "proj_wide_kernel"])
def test_the_plain_barrier_only_publishes_direct_loads(name):
    """The projection tiles' one LDS array is filled by lds_dma16 alone."""
    body = kernel_body("proj.hip", name)
    assert "barrier_nofence()" in body
    assert re.findall(r"__shared__[^;]*\b(\w+)\[", body) == ["Ar"]
    assert not re.search(r"\b(Ar|At)\b[^;=]*[^=!<>]=[^=]", body.replace("const bf16_t* At = Ar", ""))


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
