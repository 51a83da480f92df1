"""Every group-norm and dropout kernel that is compiled is launched by a shape that
the GPU tests run, and every launch stays in the buffers the ABI documents (CPU:
the sanitized host-only library of tests/hostcheck)."""
import json
import os
import re
import subprocess
import sys

import pytest

import gn_cases as R

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.join(HERE, "hostcheck"))

import build as HB  # noqa: E402


def run(calls, clean=True):
    if HB.stale():
        HB.build()
    e = dict(os.environ, LD_PRELOAD=HB.runtime(), ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
             UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, os.path.join(HERE, "hostcheck", "gn.py")], env=e, input=json.dumps(calls),
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    res = json.loads(r.stdout.strip().splitlines()[-1])
    assert not res["failures"], res["failures"]
    assert not clean or res["errors"] == 0 and res["extents"] > 0, r.stderr[-4000:]
    return res


def gpu_calls():
    """What the GPU tests call: [n, hw, c, groups, x, g, d, act, p, forward, backward, pad, short]."""
    torch_tests = pytest.importorskip("test_gpu_gn")
    out = []
    for k, s in enumerate(torch_tests.SHAPES.values()):
        act, p = ["silu", "relu", "none"][k % 3], [0.0, 0.2][(k // 3) % 2]
        for x, gd in R.GRADIENTS.items():
            for g, d in gd:
                out.append([*s, x, g, d, act, p, g == gd[0][0], True, 0, 0])
    for k, s in enumerate(list(R.RANGES.values()) + list(R.FORWARD.values())):
        for act, p in R.combos(k):
            for x, gd in R.GRADIENTS.items():
                for g, d in gd if k < len(R.RANGES) else gd[:1]:
                    out.append([*s, x, g, d, act, p, True, k < len(R.RANGES), 0, 0])
    for k, s in enumerate(R.MANY.values()):
        act, p = R.COMBOS[k % 4]
        for x, gd in R.GRADIENTS.items():
            for g, d in gd:
                out.append([*s, x, g, d, act, p, g == gd[0][0], True, 8 * (k % 2), 0])
    return out


def kind(name):
    """A kernel without its last two flags (SiLU, dropout) where it has them: they
    choose element code, which every shape runs in two of its four forms."""
    m = re.search(r"k_(gn_fwd|gn_bwd)I", name)
    return re.sub(r"Lb[01]ELb[01]E(EEv)", r"\1", name) if m else name


def test_every_kernel_is_launched_by_a_gpu_test():
    kernels = run(gpu_calls())["kernels"]
    assert len(kernels) > 300
    launched = {kind(k) for k, n in kernels.items() if n}
    missing = sorted({kind(k) for k in kernels} - launched)
    assert not missing, (len(missing), missing[:20])


def test_every_choice_of_activation_and_dropout_is_launched():
    kernels = run(gpu_calls())["kernels"]
    for kernel in ("gn_fwd", "gn_bwd"):
        flags = {re.search(r"Lb([01])ELb([01])EEEv", k).groups() for k, n in kernels.items()
                 if n and re.search(rf"k_{kernel}I", k)}
        assert len(flags) == 4


def test_the_checker_sees_a_short_workspace():
    """Chunks, records and group sums that end 16 bytes past their buffer."""
    for s, forward in [((2, 3136, 64, 32), True), ((300, 1, 1024, 16), False), ((1, 9000, 256, 2), False)]:
        # 256: a workspace's parts are rounded up to that
        assert run([[*s, "bf16", "bf16", "bf16", "none", 0.0, forward, not forward, 0, 0]])["errors"] == 0
        assert run([[*s, "bf16", "bf16", "bf16", "none", 0.0, forward, not forward, 0, 272]], False)["errors"] > 0
