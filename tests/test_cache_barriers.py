"""Waits and barriers of the paged cache's attention, read from the source (no run can
show a missing one dependably)."""
import os
import re

from test_lds_barriers import CSRC


def code(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"\s+", "", re.sub(r"//[^\n]*", "", text))


def test_tiles_are_overwritten_behind_a_barrier():
    """A tile's place is loaded anew (by direct loads, which nothing else orders) only
    behind a barrier that every wave reaches with its reads of that place done."""
    text = code("skip_cache_tall.h")
    assert "barrier_nofence" not in text
    loop = text[text.index("for(inti=it.i0;i<it.i1;++i){"):]
    loop = loop[:loop.index("if(!any)return;")]
    wait, barrier, fetch = (loop.index(x) for x in ("elsewait_vmcnt<0>();barrier_lds();",
                                                    "barrier_lds();", "fetch("))
    assert wait < barrier < fetch
    first = text[text.index("if(it.i0<it.i1){load_pages();"):]
    assert first.index("barrier_lds();") < first.index("fetch(")


def test_cleaned_values_are_published():
    """What the waves put into a tile, and their findings, are read behind a barrier
    that waits for their stores; the next tile's are written behind the next one."""
    text = code("skip_cache_tall.h")
    assert text.count("clean(t,miss);") == 1
    assert "clean(t,miss);barrier_lds();odd=flags[0]|flags[1]|flags[2]|flags[3];" in text


def test_results_and_keys_take_turns_in_lds():
    """The waves' results are read by all of them behind a barrier, and the next item's
    keys take their place behind another; likewise between prefixes and own tokens."""
    text = code("skip_cache_rows.h")
    assert "if(SOLO)wait_lgkm0();else__syncthreads();constexprintNC4" in text
    assert "if(SOLO)wait_lgkm0();elseif(!a.direct)__syncthreads();};" in text
    shared = code("attn_cache_tall.hip")
    shared = shared[shared.index("cache_shared_kernel(TallArgspre"):]
    assert (shared.index("cache_tall_work<") < shared.index("__syncthreads();")
            < shared.index("cache_rows<"))
