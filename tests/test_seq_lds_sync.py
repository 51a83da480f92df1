"""Static check of the attention kernels' LDS synchronisation (no GPU): their tiles are loaded
straight from global memory into LDS, over the ones that were read before the last barrier, so at
every barrier no LDS read that a wavefront has issued may be pending, and none of its loads into
LDS either (the barrier tells the others that they have landed)."""
import re

import pytest

from test_gemm_lds_sync import body_of, compiled, is_barrier, is_lds_load, no_hipcc, pending_reads


def pending_loads(asm):
    """barriers reached with loads into LDS that no vmcnt(0) has waited for"""
    bad, pending = 0, 0
    for line in asm.split("\n"):
        t = line.strip()
        if not t or t.startswith((";", ".")):
            continue
        if is_lds_load(t):
            pending += 1
        elif re.match(r"s_waitcnt\b.*vmcnt\(0\)", t):
            pending = 0
        elif is_barrier(t):
            bad += pending > 0
    return bad


def test_scan_flags_a_pending_load():
    load, wait, barrier = "  global_load_lds_dwordx4 v[0:1], off", "  s_waitcnt vmcnt(0) lgkmcnt(0)", "  s_barrier"
    assert pending_loads("\n".join([load, wait, barrier])) == 0
    assert pending_loads("\n".join([load, "  s_waitcnt vmcnt(4)", barrier])) == 1


@no_hipcc
@pytest.mark.parametrize("source,kernel,count", [("attn_fwd.hip", "k_attn_many|k_attn_few", 4),
                                                 ("attn_bwd.hip", "k_attn_dq|k_attn_dkv", 4)])
def test_tiles_are_refilled_after_their_reads(tmp_path, source, kernel, count):
    asm, n = body_of(compiled(tmp_path, source), kernel)
    assert n == count
    lines = [l.strip() for l in asm.split("\n") if l.strip()]
    assert sum(map(is_lds_load, lines)) > 0 and sum(l.split()[0] == "s_barrier" for l in lines) > 0
    assert pending_reads(asm, is_barrier) == {}
    assert pending_loads(asm) == 0
