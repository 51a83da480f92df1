"""Group-norm and dropout calls through the sanitized host-only library (run with
the ASan runtime preloaded; tests/test_gn_launches.py does that).

    LD_PRELOAD=<asan runtime> python tests/hostcheck/gn.py < <calls as JSON>

Reads a list of calls [n, hw, c, groups, x, g, d, act, p, forward, backward, pad, short],
issues each on fake device buffers of the sizes the ABI documents, the workspace
`short` bytes below (op_gn_apply with every forward, op_dropout of g to d with every
backward), and prints as JSON the mangled names of the library's group-norm and dropout
kernels, with how often each was launched, and the checker's errors.
"""
from __future__ import annotations

import ctypes as C
import json
import os
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(os.path.dirname(HERE))
LIB = C.CDLL(os.path.join(ROOT, "_build", "hostcheck", "libckpt_hostcheck.so"))
vp, i64, i32, u64 = C.c_void_p, C.c_int64, C.c_int32, C.c_uint64


class Dropout(C.Structure):
    _fields_ = [("rng", vp), ("site", C.c_uint32), ("reserved", C.c_uint32), ("p", C.c_double)]


class Desc(C.Structure):
    _fields_ = ([(k, i64) for k in ("n", "hw")] +
                [(k, i32) for k in ("c", "groups", "act", "xtype", "gtype", "dtype")] +
                [(k, i64) for k in ("ldx", "ldy", "ldg", "ldd")] + [("eps", C.c_float), ("reserved", i32)])


DP, RP = C.POINTER(Desc), C.POINTER(Dropout)
LIB.hc_alloc.restype, LIB.hc_alloc.argtypes = vp, [u64, C.c_char_p]
LIB.hc_kernel.restype, LIB.hc_kernel.argtypes = C.c_char_p, [u64, C.POINTER(u64)]
LIB.ckpt_last_error.restype = C.c_char_p
LIB.op_gn_workspace_bytes.argtypes = [DP, i32, C.POINTER(u64)]
LIB.op_gn_forward.argtypes = [DP, vp, vp, vp, RP, vp, vp, vp, u64, vp]
LIB.op_gn_apply.argtypes = [DP, vp, vp, vp, vp, RP, vp, vp]
LIB.op_gn_backward.argtypes = [DP, vp, vp, vp, vp, vp, RP, vp, vp, vp, vp, u64, vp]
LIB.op_dropout.argtypes = [i64, i64, i32, vp, i64, vp, i64, i32, vp, i64, RP, vp]

SIZE, CODE = {"f32": 4, "bf16": 2}, {"f32": 0, "bf16": 1}
ACT = {"none": 0, "relu": 1, "silu": 2}


def ok(rc):
    if rc != 0:
        raise RuntimeError(f"{rc}: {LIB.ckpt_last_error().decode()}")


def rows(n, ld, c, t):
    return LIB.hc_alloc(((n - 1) * ld + c) * SIZE[t], b"rows")


def workspace(nbytes, short):
    return LIB.hc_alloc(nbytes - min(nbytes, short), b"workspace") if nbytes else None


def main():
    failures = []
    for call in json.load(sys.stdin):
        n, hw, c, groups, x, g, d, act, p, forward, backward, pad, short = call
        LIB.hc_free_all()
        ld, pixels = c + pad, n * hw
        desc = Desc(n, hw, c, groups, ACT[act], CODE[x], CODE[g], CODE[d], ld, ld, ld, ld, 1e-5, 0)
        rng = LIB.hc_alloc(16, b"seed and step")
        drop = C.byref(Dropout(rng, 3, 0, p)) if p else None
        X, Y = rows(pixels, ld, c, x), rows(pixels, ld, c, x)
        ga, be = LIB.hc_alloc(4 * c, b"gamma"), LIB.hc_alloc(4 * c, b"beta")
        st = LIB.hc_alloc(8 * n * groups, b"statistics")
        nb = u64()
        try:
            if forward:
                ok(LIB.op_gn_workspace_bytes(desc, 0, nb))
                ok(LIB.op_gn_forward(desc, X, ga, be, drop, Y, st, workspace(nb.value, short), nb.value, None))
                ok(LIB.op_gn_apply(desc, X, st, ga, be, drop, Y, None))
            if backward:
                G, D = rows(pixels, ld, c, g), rows(pixels, ld, c, d)
                dg, db = LIB.hc_alloc(4 * c, b"dgamma"), LIB.hc_alloc(4 * c, b"dbeta")
                ok(LIB.op_gn_workspace_bytes(desc, 1, nb))
                ok(LIB.op_gn_backward(desc, G, X, st, ga, be, drop, D, dg, db, workspace(nb.value, short),
                                      nb.value, None))
                if p:
                    ok(LIB.op_dropout(pixels, c, CODE[g], G, ld, None, 0, CODE[d], D, ld, drop, None))
        except RuntimeError as e:
            failures.append([call, str(e)])
    launches = u64()
    kernels, i = {}, 0
    while True:
        name = LIB.hc_kernel(i, launches)
        if name is None:
            break
        if b"k_gn_" in name or b"k_dropout" in name:
            kernels[name.decode()] = launches.value
        i += 1
    counts = [u64() for _ in range(4)]
    LIB.hc_counters(*(C.byref(v) for v in counts))
    print(json.dumps(dict(kernels=kernels, errors=counts[1].value, extents=counts[3].value, failures=failures[:20])))


if __name__ == "__main__":
    main()
