"""The token models' operators through the sanitized host-only library (run with the ASan
runtime preloaded; tests/test_seq_launches.py does that).

    LD_PRELOAD=<asan runtime> python tests/hostcheck/seq.py < <calls as JSON>

Reads a list of calls [kind, descriptor's fields, workspace's shortage], issues each with its
backward on fake device buffers that end where the ABI lets them, and prints as JSON the mangled names
of the operators' kernels, with how often each was launched, the return codes other than 0, and the
checker's errors.
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


def struct(*fields):
    return type("Desc", (C.Structure,), dict(_fields_=[(n, t) for t, names in fields for n in names.split()]))


Rms = struct((i64, "rows"), (i32, "c qgroup xtype htype ytype gtype dtype"), (C.c_float, "eps"),
             (i64, "ldx ldh ldy ldg ldd"))
Embed = struct((i64, "tokens vocab"), (i32, "c ids64 wtype ytype gtype dtype accumulate"), (C.c_float, "scale"),
               (i64, "ldw ldy ldg"))
Attn = struct((i64, "tq tk"), (i32, "seqs heads kv_heads dim causal"), (C.c_float, "scale"),
              (i64, "ldq hsq ldk hsk ldv hsv ldo hso"))
LIB.hc_alloc.restype, LIB.hc_alloc.argtypes = vp, [u64, C.c_char_p]
LIB.hc_kernel.restype, LIB.hc_kernel.argtypes = C.c_char_p, [u64, C.POINTER(u64)]
LIB.ckpt_last_error.restype = C.c_char_p
for name, pointers, ws in (("rms_forward", 7, 0), ("rms_apply", 5, 0), ("rms_backward", 7, 1), ("embed_forward", 3, 0),
                           ("embed_backward", 3, 1), ("attn_forward", 7, 1), ("attn_backward", 11, 1)):
    getattr(LIB, "op_" + name).argtypes = [vp] + [vp] * pointers + [vp, u64] * ws + [vp]
SIZE = [4, 2, 1]


class Refused(Exception):
    pass


def ok(rc):
    if rc != 0:
        raise Refused(rc, LIB.ckpt_last_error().decode())


def alloc(nbytes):
    return LIB.hc_alloc(nbytes, b"tensor") if nbytes else None


def rows(n, ld, c, t):
    return alloc(((n - 1) * (ld or c) + c) * SIZE[t])


def workspace(call, *args, short):
    nb = u64()
    ok(call(*args, C.byref(nb)))
    return alloc(nb.value - min(nb.value, short)), nb.value


def rms(d, short):
    n, c = d.rows, d.c
    groups = -(-c // d.qgroup) if d.qgroup else 1
    w, st, ys = alloc(4 * c), alloc(4 * n), alloc(4 * n * groups) if d.ytype == 2 else None
    y, h = rows(n, d.ldy, c, d.ytype), rows(n, d.ldh, c, d.htype)
    r = C.byref(d)
    if d.xtype == d.htype:
        ok(LIB.op_rms_forward(r, rows(n, d.ldx, c, d.xtype), None, w, None, y, ys, st, None))
    ok(LIB.op_rms_forward(r, rows(n, d.ldx, c, d.xtype), rows(n, d.ldh, c, d.htype), w, h, y, ys, st, None))
    ok(LIB.op_rms_apply(r, h, st, w, y, ys, None))
    ws = workspace(LIB.op_rms_workspace_bytes, r, short=short)
    for gh in (None, rows(n, d.ldd, c, d.dtype)):
        ok(LIB.op_rms_backward(r, rows(n, d.ldg, c, d.gtype), gh, h, st, w, rows(n, d.ldd, c, d.dtype), alloc(4 * c), *ws,
                               None))


def embed(d, short):
    ids, r = alloc(d.tokens * (8 if d.ids64 else 4)), C.byref(d)
    ok(LIB.op_embed_forward(r, ids, rows(d.vocab, d.ldw, d.c, d.wtype), rows(d.tokens, d.ldy, d.c, d.ytype), None))
    ok(LIB.op_embed_backward(r, ids, rows(d.tokens, d.ldg, d.c, d.gtype), rows(d.vocab, d.ldw, d.c, d.dtype),
                             *workspace(LIB.op_embed_workspace_bytes, r, short=short), None))


def attn(d, short):
    def heads(t, n, ld, hs):
        return alloc(2 * ((t - 1) * (ld or n * d.dim) + (n - 1) * (hs or d.dim) + d.dim)) if t else None

    r, off = C.byref(d), alloc(4 * (d.seqs + 1))
    q, o, dq, g = (heads(d.tq, d.heads, *s) for s in ((d.ldq, d.hsq), (d.ldo, d.hso), (d.ldq, d.hsq), (d.ldo, d.hso)))
    k, v, dk, dv = (heads(d.tk, d.kv_heads, *s) for s in ((d.ldk, d.hsk), (d.ldv, d.hsv)) * 2)
    lse = alloc(4 * d.heads * d.tq)
    ok(LIB.op_attn_forward(r, q, k, v, off, off, o, lse, *workspace(LIB.op_attn_workspace_bytes, r, 0, short=short), None))
    ok(LIB.op_attn_backward(r, g, q, k, v, o, lse, off, off, dq, dk, dv,
                            *workspace(LIB.op_attn_workspace_bytes, r, 1, short=short), None))


def main():
    refused = []
    for kind, fields, short in json.load(sys.stdin):
        LIB.hc_free_all()
        make, call = dict(rms=(Rms, rms), embed=(Embed, embed), attn=(Attn, attn))[kind]
        try:
            call(make(**fields), short)
        except Refused as e:
            refused.append([kind, fields, *e.args])
    launches, kernels, i = u64(), {}, 0
    while (name := LIB.hc_kernel(i, launches)) is not None:
        if any(k in name for k in (b"k_rms_", b"k_embed_", b"k_attn_")):
            kernels[name.decode()] = launches.value
        i += 1
    counts = [u64() for _ in range(4)]
    LIB.hc_counters(*(C.byref(v) for v in counts))
    print(json.dumps(dict(kernels=kernels, errors=counts[1].value, extents=counts[3].value, refused=refused)))


if __name__ == "__main__":
    main()
