"""Launches of the token models' operators stay in the buffers the ABI documents, up to the largest
sizes, and every kernel that is compiled is reached (CPU: the sanitized host-only library of
tests/hostcheck)."""
import itertools
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.join(HERE, "hostcheck"))

import build as HB  # noqa: E402

F32, BF16, E4M3 = 0, 1, 2


def run(calls, clean=True):
    if HB.stale():
        HB.build()
    e = dict(os.environ, LD_PRELOAD=HB.runtime(), ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
             UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, os.path.join(HERE, "hostcheck", "seq.py")], env=e, input=json.dumps(calls),
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    res = json.loads(r.stdout.strip().splitlines()[-1])
    assert not clean or res["errors"] == 0 and res["extents"] > 0, r.stderr[-4000:]
    return res


def rms(rows, c, x=BF16, h=BF16, y=BF16, g=BF16, d=BF16, q=0, short=0, **ld):
    return ["rms", dict(rows=rows, c=c, qgroup=q, xtype=x, htype=h, ytype=y, gtype=g, dtype=d, eps=1e-5, **ld), short]


def embed(tokens, vocab, c, w=BF16, y=BF16, g=BF16, d=F32, ids64=0, accumulate=0, short=0, **ld):
    return ["embed", dict(tokens=tokens, vocab=vocab, c=c, ids64=ids64, wtype=w, ytype=y, gtype=g, dtype=d,
                          accumulate=accumulate, scale=1.0, **ld), short]


def attn(tq, tk, seqs, heads, kv, dim, causal=1, short=0, **ld):
    return ["attn", dict(tq=tq, tk=tk, seqs=seqs, heads=heads, kv_heads=kv, dim=dim, causal=causal, scale=0.0, **ld), short]


TYPES = list(itertools.product((F32, BF16), repeat=3))
CALLS = ([rms(37, c, x=x, h=h, y=y, g=g, d=d) for c in (1, 509, 1000, 2048, 4090, 8192, 16384) for x, h, g in TYPES
          for y, d in ((F32, F32), (BF16, BF16), (E4M3, BF16), (E4M3, F32))] +
         [rms(9001, 333, y=E4M3, q=q, ldx=340, ldh=336, ldy=334, ldg=333, ldd=352) for q in (8, 64, 512)] +
         [embed(n, v, c, w=w, y=g, g=g, d=w, ids64=n % 2, accumulate=c % 2, ldw=c + 3)
          for n, v, c in ((1, 1, 1), (70, 3, 8), (5001, 97, 333), (4096, 200001, 1024), (300000, 5, 64)) for w in (F32, BF16)
          for g in (F32, BF16)] +
         [attn(*s, causal) for causal in (0, 1) for s in
          ((1, 1, 1, 1, 1, 8), (0, 9, 2, 4, 2, 64), (9, 0, 2, 4, 2, 128), (16, 90000, 16, 32, 8, 128), (3, 5000, 3, 8, 8, 64),
           (2000, 2000, 3, 8, 1, 72), (8192, 8192, 1, 16, 4, 128), (4000, 4100, 150, 12, 12, 40), (200, 70000, 1, 4, 4, 64))])
# as large as the header allows, or nearly (buffers of up to a terabyte in all)
LARGEST = [rms((1 << 31) - 1, 1), rms(1 << 20, 16384, y=E4M3, q=8), embed(1 << 30, 1, 8), embed(1 << 16, 1 << 10, (1 << 20) - 1),
           embed(1 << 10, (1 << 31) - 1, 8), embed((1 << 30), 1 << 20, 63, d=BF16),
           attn(1 << 26, 1 << 26, 1, 12, 12, 8), attn(1 << 30, 1, 1, 1, 1, 8), attn(1, 1 << 30, 1, 1, 1, 8),
           attn(4, 1 << 28, 4, 128, 1, 8), attn((1 << 20) - 1, 1 << 20, (1 << 20) - 1, 4, 4, 8),
           attn(1 << 17, 1 << 22, 1 << 16, 4096, 32, 8)]


def test_every_kernel_is_launched_within_its_buffers():
    res = run(CALLS)
    assert not res["refused"], res["refused"][:5]
    missing = sorted(k for k, n in res["kernels"].items() if not n)
    assert len(res["kernels"]) > 200 and not missing, (len(missing), missing[:20])


@pytest.mark.parametrize("call", LARGEST, ids=[str(k) for k in range(len(LARGEST))])
def test_largest_sizes(call):
    assert not run([call])["refused"]


@pytest.mark.parametrize("call", [rms(9001, 333, short=16), embed(5001, 97, 333, short=16),
                                  attn(16, 90000, 16, 32, 8, 128, short=16), attn(8192, 8192, 1, 16, 4, 128, short=16)],
                         ids=["rms", "embed", "split", "parts"])
def test_the_checker_sees_a_short_workspace(call):
    assert run([call[:2] + [0]])["errors"] == 0
    assert run([call], False)["errors"] > 0
