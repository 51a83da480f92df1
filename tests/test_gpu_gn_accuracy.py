"""Accuracy of group norm where its range makes it hard: a first value far from
the others, a mean far from zero, sums over many samples, SiLU far below zero.
Bars are worst cases of the fp32 operations, counted beside each test.
"""
import numpy as np
import pytest

from oracle import norm as N
from test_gpu_gn import DEV, EPS, L, Case, _K, f32, host, rounded, torch, types

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


# ------------------------------------------------- a mean far from zero ------
FAR_SHAPES = {
    "rows": (300, 1, 1024, 16),
    "rows_packed": (4100, 1, 64, 4),
    "layer_rows": (1500, 1, 1024, 1),
    "layer_rows_fours": (700, 1, 1000, 2),
    "wave_two_vectors": (2048, 16, 64, 8),
    "wave_fours": (2048, 16, 64, 16),
    "resident": (32, 196, 256, 32),
    "resident_odd_groups": (5, 100, 120, 12),
    "resident_eight_vectors": (64, 784, 64, 8),
    "split": (2, 3136, 64, 32),
    "split_many_chunks": (1, 40000, 64, 8),
    "split_odd_groups": (3, 2777, 72, 6),
    "scalar": (7, 65, 37, 37),
    "scalar_rows": (1500, 1, 515, 5),
    "scalar_split": (2, 9001, 6, 2),
}


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("shape", list(FAR_SHAPES))
def test_one_offset_for_all_values(shape, x):
    """A spread of one on a level of a thousand (bf16: of 64, where its steps are
    still a quarter of the spread) that all channels share.  1 / std from the squares
    of the differences: L for the sums, and the square of the mean's error in
    standard deviations; a difference of the squares' mean and the mean's square is
    off by a hundred times that."""
    level = 1000.0 if x == "f32" else 64.0
    print(f"[gn far] {shape} {x}", flush=True)
    c = Case(*FAR_SHAPES[shape], x=x, level=0.0, seed=43)
    v = rounded(np.random.default_rng(44).standard_normal(c.xv.shape) + level, x)
    c.xv, c.x3 = v, v.reshape(c.n, c.hw, c.c)
    c.X.m.copy_(torch.from_numpy(v))
    mean, rstd = N.group_stats(c.x3, c.groups, EPS)
    # the groups have eight values or more
    assert (1 / (rstd * mean)).max() <= (3e-3 if x == "f32" else 5e-2)
    s = host(c.check_forward()).reshape(2, c.n, c.groups)
    off = np.abs(s[1] / rstd - 1)
    bar = U + L + (L * mean * rstd) ** 2
    print(f"    1 / std: {(off / bar).max():.3f} of its bar", flush=True)
    assert (off <= bar).all()


# ------------------------------------------------ sums over many samples ----
def test_gradients_of_shift_over_many_samples():
    """dbeta over 100000 samples of 200 pixels whose gradient is one number a channel:
    a chain of equal terms rounds the same way at every step, and these numbers are
    ones for which a chain over 1563 of the samples' sums, exact each,
    loses more than L of itself.  As bounded in test_gpu_gn.py: 256 operations."""
    K = _K()
    n, hw, c = 100000, 200, 8
    print(f"[gn many samples] {n} x {hw} x {c}", flush=True)
    v = np.array([56553, 53865, 64279, 33911, 33673, 41719, 57459, 47629]) / 32768
    g = f32(v).expand(n * hw, c).contiguous()
    x = torch.zeros(n * hw, c, dtype=torch.bfloat16, device=DEV)
    d = K.gn_desc(n, hw, c, 1, gtype=K.TYPE_F32)
    st = torch.cat([torch.zeros(n, device=DEV), torch.ones(n, device=DEV)])
    dx, dg, db = torch.empty_like(x), torch.empty(c, device=DEV), torch.empty(c, device=DEV)
    nb = K.op_gn_workspace_bytes(d, True)
    ws = torch.empty(max(16, nb), dtype=torch.uint8, device=DEV)
    K.op_gn_backward(d, g, x, st, torch.ones(c, device=DEV), torch.zeros(c, device=DEV), dx, dg, db, ws, nb)
    err = np.abs(host(db) / (v * (n * hw)) - 1)
    print(f"    {err.max() / L:.3f} of its bar", flush=True)
    assert (err <= L).all() and bool((dg == 0).all())


# ------------------------------------------------------------------- SiLU --
def _levels():
    """u from -80 (where silu' = u e^u is still a normal number) to 80."""
    rng = np.random.default_rng(45)
    u = np.concatenate([np.linspace(-80, 80, 4001), rng.uniform(-80, 0, 4000), rng.uniform(-2, 2, 2000), [0.0]])
    return u.astype(np.float32)


def _identity(u, dt):
    """Statistics, scale and shift that make u of a bf16 or fp32 x exactly x."""
    c = u.size
    K = _K()
    code = {torch.float32: K.TYPE_F32, torch.bfloat16: K.TYPE_BF16}[dt]
    d = K.gn_desc(1, 1, c, c, act=K.ACT_SILU, xtype=code, gtype=K.TYPE_F32, dtype=K.TYPE_F32)
    st = f32(np.concatenate([np.zeros(c), np.ones(c)]))
    return d, torch.from_numpy(u).to(DEV).to(dt).view(1, c), st, torch.ones(c, device=DEV), torch.zeros(c, device=DEV)


def _pad8(u, n):
    return u[:u.size // 8 * 8] if n == 8 else u[:u.size // 8 * 8 - 1]


@pytest.mark.parametrize("vec", [8, 1])
def test_silu_of_fp32(vec):
    """x sigmoid(x) relative to itself: the exponential (a step and a half at most),
    the sum, the reciprocal (a step) and the product are below 8 half steps."""
    K = _K()
    print(f"[gn silu] {vec}", flush=True)
    u = _pad8(_levels(), vec)
    d, x, st, ga, be = _identity(u, torch.float32)
    y = torch.empty_like(x)
    K.op_gn_apply(d, x, st, ga, be, y)
    want = u.astype(np.float64) * N.sigmoid(u.astype(np.float64))
    err = np.abs(host(y).reshape(-1) - want)
    print(f"    {np.max(err[want != 0] / np.abs(want[want != 0])) / U:.1f} half steps", flush=True)
    assert (err <= 8 * U * np.abs(want)).all()


@pytest.mark.parametrize("vec", [8, 1])
@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_silu_slope(vec, x):
    """The shift's gradient of a single pixel is g silu'(u) itself: q (1 + u (1 - q))
    with q = sigmoid(u) to 6 half steps, three operations more and the product with g,
    relative to q (1 + |u| (1 - q)); 1 - q to four half steps of 1.  A bf16 x takes the
    exponential whose relative error is 1.25 |u| half steps and two more."""
    K = _K()
    print(f"[gn silu'] {vec} {x}", flush=True)
    u = _pad8(rounded(_levels(), x), vec)
    d, xd, st, ga, be = _identity(u, torch.float32 if x == "f32" else torch.bfloat16)
    g = np.random.default_rng(46).standard_normal(u.size).astype(np.float32)
    dx, dg, db = torch.empty(1, u.size, device=DEV), torch.empty(u.size, device=DEV), torch.empty(u.size, device=DEV)
    nb = K.op_gn_workspace_bytes(d, True)
    ws = torch.empty(max(16, nb), dtype=torch.uint8, device=DEV)
    K.op_gn_backward(d, f32(g).view(1, -1), xd, st, ga, be, dx, dg, db, ws, nb)
    w = u.astype(np.float64)
    q = N.sigmoid(w)
    want = g * (q * (1 + w * (1 - q)))
    steps = 24.0 if x == "f32" else 24.0 + 2 * (1.25 * np.abs(w) + 2)
    bar = U * np.abs(g) * q * (steps * (1 + np.abs(w) * (1 - q)) + 4 * np.abs(w))
    err = np.abs(host(db) - want)
    print(f"    {np.max(err / (bar + 1e-37)):.3f} of its bar", flush=True)
    assert (err <= bar + 1e-37).all()


@pytest.mark.parametrize("vec", [8, 1])
@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_silu_of_extremes(vec, x):
    """Where the exponential under- or overflows: u itself or zero, and slopes of one or
    zero; NaN and infinity stay what u / (1 + exp(-u)) makes of them."""
    K = _K()
    print(f"[gn silu extremes] {vec} {x}", flush=True)
    big = [200.0, 1e4, 1e30, 2.0 ** 127, 3e38, float("inf")]
    u = rounded(np.array(big + [-v for v in big[:-1]] + [float("nan"), float("-inf")] + [0.0] * (vec + 2)), x)
    u = _pad8(u, vec)
    d, xd, st, ga, be = _identity(u, types()[x][1])
    y = torch.empty_like(xd)
    K.op_gn_apply(d, xd, st, ga, be, y)
    got = host(y.float()).reshape(-1)
    assert np.array_equal(got[:6], u[:6].astype(np.float64)) and (got[6:11] == 0).all()
    assert np.isnan(got[11:13]).all() and (got[13:] == 0).all()
    dx, dg, db = (torch.empty(u.size, device=DEV) for _ in range(3))
    nb = K.op_gn_workspace_bytes(d, True)
    ws = torch.empty(max(16, nb), dtype=torch.uint8, device=DEV)
    K.op_gn_backward(d, torch.full((u.size,), 3.0, device=DEV), xd, st, ga, be, dx, dg, db, ws, nb)
    got = host(db)
    assert (got[:5] == 3).all() and (got[6:11] == 0).all() and np.isnan(got[11]) and (got[13:] == 1.5).all()
