"""Accuracy of group norm where its range makes it hard: a first value far from
the others.  Bars are worst cases of the fp32 operations, counted beside each test.
"""
import numpy as np
import pytest

from oracle import norm as N
from test_gpu_gn import DEV, EPS, L, _K, host, rounded, torch, types

pytestmark = pytest.mark.gpu

U = 2.0 ** -24  # half a step of fp32


# ------------------------------------------------------- an outlying value --
# sums of the differences from a value far from all the others cancel by the count of
# the values, so that count may not grow with the sample
OUTLIER_SHAPES = {
    "stage1_512": (512, 3136, 64, 8),          # a chunk is a whole sample: 784 values a thread in bf16
    "stage1_128": (128, 12544, 64, 8),
    "stem_512": (512, 12544, 64, 8),           # 3136 values a thread in bf16
    "several_groups_a_vector": (512, 3136, 64, 16),
    "odd_groups": (512, 3136, 72, 24),
    "element_by_element": (1024, 3136, 7, 1),
}


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("shape", list(OUTLIER_SHAPES))
def test_statistics_with_an_outlying_first_value(shape, x):
    """Eight different samples, pixel 0 of each scaled, repeated through the batch.

    The variance's relative error: a thread adds at most 256 values in turn before
    it takes the running mean as its new pivot; the sum of squares is then at most
    twice what it contributes (four times for the first 32 values, whose pivot is a
    mean of eight of them; sixteen times for the first 16 single ones): 2 256 = 512 at
    most.  Those sums are added up in at most 50 steps and the threads' in at most 64:
    626 in all, half of it for 1 / std: 320 with the distance of 313 to it for the few
    operations before and after."""
    K = _K()
    n, hw, c, groups = OUTLIER_SHAPES[shape]
    print(f"[gn outlier] {shape} {x}", flush=True)
    rng = np.random.default_rng(41)
    scales = np.array([1.0, 30.0, 300.0, 1e3, 3e3, 1e4, 3e4, -1e4])
    base = rounded(rng.standard_normal((8, hw, c)), x)
    base[:, 0] = rounded(base[:, 0] * scales[:, None], x)
    mean, rstd = N.group_stats(base, groups, EPS)
    code, dt, _ = types()[x]
    b = torch.from_numpy(base).to(DEV).to(dt)
    xs = b.repeat(n // 8, 1, 1)
    y = torch.empty_like(xs)
    d = K.gn_desc(n, hw, c, groups, xtype=code, eps=EPS)
    st = torch.full((2 * n * groups,), float("nan"), device=DEV)
    nb = K.op_gn_workspace_bytes(d, False)
    ws = torch.empty(max(16, nb), dtype=torch.uint8, device=DEV)
    ga, be = torch.ones(c, device=DEV), torch.zeros(c, device=DEV)
    K.op_gn_forward(d, xs, ga, be, y, st, ws, nb)
    torch.cuda.synchronize()
    st = st.view(2, n // 8, 8, groups)
    assert bool((st == st[:, :1]).all()), "equal samples, equal statistics"
    assert torch.equal(y.view(n // 8, 8, hw, c)[-1], y.view(n // 8, 8, hw, c)[0])
    s = host(st[:, 0])
    err = np.abs(s[1] / rstd - 1)
    print("    1 / std, worst of each sample:", " ".join(f"{v:.1e}" for v in err.max(1)), flush=True)
    absmean = np.abs(base.astype(np.float64)).reshape(8, hw, groups, -1).mean((1, 3))
    assert (np.abs(s[0] - mean) <= U * np.abs(mean) + L * absmean).all()
    assert (err <= 320 * U).all()
