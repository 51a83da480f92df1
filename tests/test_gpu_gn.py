"""GPU parity of group norm, its activation and dropout (op_gn_*, op_dropout)
with the float64 oracle on the same inputs.

Bars, per element: half a step of the output's type at the exact value (bf16
2^-8 of it, fp32 2^-24) for the one rounding at the end, plus
L 2^-24 times the sum of the magnitudes that enter the element, for the fp32
arithmetic.  L bounds the operations an input passes: a sum runs over at most
128 values in a thread (16 vectors of 8; the chunks of the sizes here are no
longer), then trees of eight of at most 1024 threads, 16 wavefronts or 64
columns, and 64 records in turn, below 256 in all; the few operations before and
after it are covered by the distance of 256 to these 240.  ReLU's decisions are the documented fp32 ones (oracle.affine_f32).
"""
import numpy as np
import pytest

from oracle import norm as N
from oracle import units as U

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DEV = "cuda:0"
L = 256 * 2.0 ** -24
EPS = 1e-5


def _K():
    from paper_1604_06174_amd import ckpt as K
    return K


def types():
    K = _K()
    return {"bf16": (K.TYPE_BF16, torch.bfloat16, 2.0 ** -8), "f32": (K.TYPE_F32, torch.float32, 2.0 ** -24)}


def acts():
    K = _K()
    return {"none": K.ACT_NONE, "relu": K.ACT_RELU, "silu": K.ACT_SILU}


def rounded(v, t):
    v = np.asarray(v, np.float32)
    return v if t == "f32" else U.bf16_round(v).astype(np.float32)


class Rows:
    """[rows, cols] of a type with `pad` elements between the rows, `shift`
    elements from an aligned address; the gaps and both ends hold a value that no
    call may change."""

    def __init__(self, rows, cols, t, pad=0, shift=0, data=None):
        self.rows, self.cols, self.ld, self.t = rows, cols, cols + pad, t
        self.all = torch.full((shift + rows * self.ld + 16,), -77.0, dtype=types()[t][1], device=DEV)
        self.m = self.all[shift:shift + rows * self.ld].view(rows, self.ld)[:, :cols]
        if data is not None:
            self.m.copy_(torch.from_numpy(np.ascontiguousarray(np.asarray(data, np.float32).reshape(rows, cols))))

    def data_ptr(self):
        return self.m.data_ptr()

    def host(self):
        torch.cuda.synchronize()
        v = self.m.float().cpu().numpy().astype(np.float64)
        rest = self.all.clone()
        n = self.m.storage_offset()
        rest[n:n + self.rows * self.ld].view(self.rows, self.ld)[:, :self.cols] = -77.0
        assert bool((rest == -77.0).all()), "written outside its rows"
        return v


def f32(v):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(v, np.float32))).to(DEV)


def host(t):
    torch.cuda.synchronize()
    return t.cpu().numpy().astype(np.float64)


def close(name, got, want, mag, step):
    want = np.asarray(want, np.float64).reshape(got.shape)
    tol = step * np.abs(want) + L * np.asarray(mag, np.float64).reshape(got.shape) + 1e-30
    err = np.abs(got - want)
    worst = float(np.max(err / tol))
    print(f"    {name}: {worst:.3f} of its bar", flush=True)
    assert np.isfinite(got).all(), name
    assert worst <= 1.0, (name, worst, int(np.argmax(err / tol)))


class Case:
    def __init__(self, n, hw, c, groups, act="none", x="bf16", g=None, d=None, pad=0, shift=0, p=0.0, level=0.5,
                 seed=1):
        K = _K()
        self.__dict__.update(n=n, hw=hw, c=c, groups=groups, act=act, x=x, p=p)
        self.g, self.d = g or x, d or x
        rng = np.random.default_rng(seed)
        rows = n * hw
        self.xv = rounded(rng.standard_normal((rows, c)) * (0.5 + rng.random(c)) + level * rng.standard_normal(c), x)
        self.gv = rounded(rng.standard_normal((rows, c)), self.g)
        self.gamma = (1 + 0.2 * rng.standard_normal(c)).astype(np.float32)
        self.beta = (0.2 * rng.standard_normal(c)).astype(np.float32)
        self.X = Rows(rows, c, x, pad, shift, self.xv)
        self.G = Rows(rows, c, self.g, pad, shift, self.gv)
        self.Y, self.D = Rows(rows, c, x, pad, shift), Rows(rows, c, self.d, pad, shift)
        self.ga, self.be = f32(self.gamma), f32(self.beta)
        ty = types()
        self.desc = K.gn_desc(n, hw, c, groups, act=acts()[act], xtype=ty[x][0], gtype=ty[self.g][0],
                              dtype=ty[self.d][0], ldx=self.X.ld, ldy=self.Y.ld, ldg=self.G.ld, ldd=self.D.ld, eps=EPS)
        self.seed, self.step, self.site = 0xFEDCBA9876543210, (3 << 32) + 17, 5
        self.rng = torch.tensor([self.seed - (1 << 64), self.step], dtype=torch.int64, device=DEV)
        self.drop = K.dropout(self.rng, p, self.site) if p else None
        self.factor = N.dropout_factor(rows * c, p, self.seed, self.step, self.site) if p else None
        self.x3 = self.xv.reshape(n, hw, c)

    def workspace(self, backward):
        nb = _K().op_gn_workspace_bytes(self.desc, backward)
        return torch.full((nb + 256,), 255, dtype=torch.uint8, device=DEV), nb

    def forward(self, stream=None):
        K = _K()
        st = torch.full((2 * self.n * self.groups,), float("nan"), device=DEV)
        ws, nb = self.workspace(False)
        K.op_gn_forward(self.desc, self.X, self.ga, self.be, self.Y, st, ws, nb, drop=self.drop, stream=stream)
        torch.cuda.synchronize()
        assert bool((ws[nb:] == 255).all())
        return st

    def backward(self, st, stream=None):
        K = _K()
        dg, db = (torch.full((self.c,), float("nan"), device=DEV) for _ in range(2))
        ws, nb = self.workspace(True)
        K.op_gn_backward(self.desc, self.G, self.X, st, self.ga, self.be, self.D, dg, db, ws, nb, drop=self.drop,
                         stream=stream)
        torch.cuda.synchronize()
        assert bool((ws[nb:] == 255).all())
        return dg, db

    def spread(self, v):
        return np.repeat(v, self.c // self.groups, 1)[:, None, :]

    def check_forward(self):
        K = _K()
        st = self.forward()
        y = self.Y.host()
        mean, rstd = N.group_stats(self.x3, self.groups, EPS)
        s = host(st).reshape(2, self.n, self.groups)
        absmean = np.abs(self.x3.astype(np.float64)).reshape(self.n, self.hw, self.groups, -1).mean((1, 3))
        close("mean", s[0], mean, absmean, 2.0 ** -24)
        # the variance's relative error: L, and twice that of the mean times |mean| / std
        close("rstd", s[1], rstd, rstd * (1 + 2 * absmean * rstd), 2.0 ** -24)
        xhat = (self.x3 - self.spread(mean)) * self.spread(rstd)
        mag = (np.abs(xhat * self.gamma) * (1 + 2 * self.spread(absmean * rstd)) + np.abs(self.beta) +
               np.abs(self.gamma) * self.spread(absmean * rstd))
        # |silu'| <= 1.1; the scale of kept elements
        scale = 1.1 if self.factor is None else 1.1 * max(1.0, self.factor.max())
        close("y", y, N.gn_apply(self.x3, mean, rstd, self.gamma, self.beta, self.act, self.factor), scale * mag,
              types()[self.x][2])
        again = Rows(self.Y.rows, self.c, self.x, self.Y.ld - self.c, self.Y.m.storage_offset())
        K.op_gn_apply(self.desc, self.X, st, self.ga, self.be, again, drop=self.drop)
        torch.cuda.synchronize()
        assert torch.equal(again.all, self.Y.all), "re-run from the statistics"
        return st

    def check_backward(self):
        mean, rstd = N.group_stats(self.x3, self.groups, EPS)
        st = np.concatenate([mean.reshape(-1), rstd.reshape(-1)]).astype(np.float32)
        dg, db = self.backward(f32(st))
        mean, rstd = st.reshape(2, self.n, self.groups)
        pos = N.affine_f32(self.x3, mean, rstd, self.gamma, self.beta) > 0
        mean, rstd = mean.astype(np.float64), rstd.astype(np.float64)
        g3 = self.gv.reshape(self.x3.shape)
        d, dgo, dbo = N.gn_backward(g3, self.x3, mean, rstd, self.gamma, self.beta, self.act, self.factor, pos)
        # magnitudes: |act'| <= 1.1 on the dropped-out gradient, with the error of u (a few steps of its terms) times
        # |act''| <= 0.5 inside the factor
        f = 1.0 if self.factor is None else self.factor.reshape(g3.shape)
        xhat = (self.x3 - self.spread(mean)) * self.spread(rstd)
        live = pos if self.act == "relu" else 1.0
        du = 1.1 * np.abs(g3) * f * live * (1 + np.abs(xhat * self.gamma) + np.abs(self.beta))
        gd, ax = du * np.abs(self.gamma), np.abs(xhat)
        mean_of = lambda v: self.spread(v.reshape(self.n, self.hw, self.groups, -1).mean((1, 3)))
        close("d", self.D.host(), d, self.spread(rstd) * (gd + mean_of(gd) + ax * mean_of(gd * ax)),
              types()[self.d][2])
        close("dgamma", host(dg), dgo, (du * ax).sum((0, 1)), 2.0 ** -24)
        close("dbeta", host(db), dbo, du.sum((0, 1)), 2.0 ** -24)


# what each shape is there for
SHAPES = {
    "one_pixel_row": (3, 1, 64, 1),
    "rows": (300, 1, 1024, 16),
    "rows_many": (5000, 1, 136, 17),      # wavefront teams, columns no power of two
    "rows_two_pixels": (4200, 2, 32, 2),  # wavefront teams, two pixels each
    "b1_7x7": (1, 49, 512, 32),
    "wave_49": (520, 49, 64, 8),          # wavefront teams over seven vectors a thread
    "resident": (32, 196, 256, 32),
    "resident_2perGroup": (4, 784, 64, 32),
    "resident_odd_groups": (5, 100, 120, 12),
    "resident_3perGroup": (9, 33, 24, 8),
    "instance": (2, 37, 16, 16),          # one channel a group
    "layer": (2, 37, 1024, 1),            # all channels one group
    "widest_group": (1, 5, 4096, 1),
    "split": (2, 3136, 64, 32),
    "split_one_group": (1, 5000, 40, 1),
    "split_odd_groups": (3, 2777, 72, 6),
    "split_partial_tile": (2, 2900, 168, 21),
    "scalar": (7, 65, 37, 37),
    "scalar_rows": (4500, 1, 9, 3),
    "scalar_split": (2, 9001, 6, 2),
    "scalar_wide": (1, 130, 515, 1),
    "one_channel": (3, 50, 1, 1),
    "last_tile_short": (2, 60, 200, 25),
    "rows_packed": (4100, 1, 64, 4),       # eight samples of one pixel a wavefront
    "rows_packed_fours": (2101, 1, 32, 8),
    "rows_packed_pairs": (3003, 1, 16, 8),
    "fours": (3, 300, 64, 16),             # groups of four channels, two in a vector
    "padded_columns": (2, 100, 320, 32),   # ten channels a group: 15 of 16 columns in use
    "padded_one_group": (3, 70, 40, 1),
    "split_many_chunks": (1, 40000, 64, 8),
    "split_wide_groups": (1, 9000, 256, 2),
    "split_one_wide": (1, 3000, 1024, 1),
}


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_forward(shape, x):
    k = list(SHAPES).index(shape)
    print(f"[gn forward] {shape} {x}", flush=True)
    Case(*SHAPES[shape], act=["silu", "relu", "none"][k % 3], x=x, p=[0.0, 0.2][(k // 3) % 2], seed=k).check_forward()


@pytest.mark.parametrize("types_", ["bf16-bf16-bf16", "bf16-f32-bf16", "bf16-f32-f32", "bf16-bf16-f32", "f32-f32-f32"])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_backward(shape, types_):
    k = list(SHAPES).index(shape)
    x, g, d = types_.split("-")
    print(f"[gn backward] {shape} {types_}", flush=True)
    Case(*SHAPES[shape], act=["silu", "relu", "none"][k % 3], x=x, g=g, d=d, p=[0.0, 0.2][(k // 3) % 2],
         seed=k).check_backward()


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5])
@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_activations_and_dropout(act, p, x):
    print(f"[gn act] {act} {p} {x}", flush=True)
    c = Case(4, 130, 96, 8, act=act, x=x, p=p, seed=11)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("pad,shift", [(8, 0), (5, 0), (3, 1), (0, 3), (64, 5)])
@pytest.mark.parametrize("shape", ["resident", "split_odd_groups", "rows_many", "scalar"])
def test_strides_and_addresses(shape, pad, shift, x):
    print(f"[gn strides] {shape} {pad} {shift} {x}", flush=True)
    c = Case(*SHAPES[shape], act="silu", x=x, p=0.2, pad=pad, shift=shift, seed=12)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("shape", ["resident", "split", "wave_49", "scalar_split"])
def test_mean_far_from_zero(shape):
    """A spread of one on a level of a thousand."""
    print(f"[gn far mean] {shape}", flush=True)
    Case(*SHAPES[shape], x="f32", level=1000.0, seed=13).check_forward()


@pytest.mark.parametrize("shape", ["resident", "split", "wave_49", "scalar", "resident_odd_groups"])
def test_special_values_stay_in_their_group(shape):
    K = _K()
    print(f"[gn special] {shape}", flush=True)
    n, hw, c, groups = SHAPES[shape]
    cg = c // groups
    ref = Case(n, hw, c, groups, act="relu", x="f32", seed=14)
    bad = Case(n, hw, c, groups, act="relu", x="f32", seed=14)
    m = bad.X.m.view(n, hw, c)
    m[0, 0, 0] = float("nan")
    m[n - 1, hw - 1, c - 1] = float("inf")
    m[0, :, cg:2 * cg] = 3.5  # a constant group: variance zero
    sr, sb = ref.forward(), bad.forward()
    y, yr = bad.Y.m.view(n, hw, groups, cg), ref.Y.m.view(n, hw, groups, cg)
    touched = torch.zeros(n, groups, dtype=torch.bool, device=DEV)
    touched[0, 0] = touched[n - 1, groups - 1] = touched[0, 1] = True
    same = (y == yr).all(3).all(1)
    assert bool(same[~touched].all())
    assert bool(torch.isnan(y[0, :, 0]).all()) and bool(torch.isnan(y[n - 1, :, groups - 1]).all())
    want = torch.relu(bad.be[cg:2 * cg]).expand(hw, cg)
    assert torch.equal(y[0, :, 1], want)
    assert abs(float(sb[n * groups + 1]) * np.sqrt(EPS) - 1) < 2.0 ** -22
    # a dropped element is zero whatever reaches it, forward and backward
    for p in (0.5, 1.0):
        q = Case(n, hw, c, groups, act="silu", x="f32", p=p, seed=14)
        zero = torch.from_numpy(q.factor.reshape(n * hw, c) == 0).to(DEV)
        st = q.forward()
        assert bool((q.Y.m[zero] == 0).all())
        q.G.m[zero] = float("nan")
        dg, db = q.backward(st)
        assert bool(torch.isfinite(q.D.m).all()) and bool(torch.isfinite(dg).all()) and bool(torch.isfinite(db).all())


@pytest.mark.parametrize("shape", ["resident", "split", "rows_many", "scalar_split"])
def test_same_bits_and_in_place(shape):
    """Two runs, a run on another stream and runs over their inputs agree bit for bit."""
    print(f"[gn bits] {shape}", flush=True)
    K = _K()
    a, b = (Case(*SHAPES[shape], act="silu", p=0.2, seed=15) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    sa, sb = a.forward(), b.forward(side)
    assert torch.equal(sa, sb) and torch.equal(a.Y.all, b.Y.all)
    (dga, dba), (dgb, dbb) = a.backward(sa), b.backward(sb, side)
    assert torch.equal(a.D.all, b.D.all) and torch.equal(dga, dgb) and torch.equal(dba, dbb)
    keep = b.X.all.clone()
    b.G.all.copy_(a.G.all)
    b.D = b.G
    dgb, dbb = b.backward(sb)
    assert torch.equal(a.D.all, b.G.all) and torch.equal(dga, dgb) and torch.equal(dba, dbb)
    b.Y = b.X
    st = b.forward()
    assert torch.equal(st, sa) and torch.equal(b.X.all, a.Y.all)
    b.X.all.copy_(keep)
    b.Y = b.X
    K.op_gn_apply(b.desc, b.X, sb, b.ga, b.be, b.X, drop=b.drop)
    torch.cuda.synchronize()
    assert torch.equal(b.X.all, a.Y.all)


# ----------------------------------------------------------------- dropout --
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 7, 0), (3, 8, 0), (37, 250, 0), (37, 250, 6), (64, 1024, 0),
                                           (64, 1024, 8), (129, 40, 3), (1000, 33, 0), (3211, 3, 5), (5, 1, 9)])
@pytest.mark.parametrize("xt,yt", [("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "f32")])
def test_dropout(rows, cols, pad, xt, yt):
    """The products and sums of one element are exact in float64: fp32 arithmetic
    is two roundings, a bf16 output a third."""
    K = _K()
    print(f"[dropout] {rows} x {cols} + {pad} {xt} {yt}", flush=True)
    rng = np.random.default_rng(21)
    xv, rv = rounded(rng.standard_normal((rows, cols)), xt), rounded(rng.standard_normal((rows, cols)), yt)
    seed, step = 0x0123456789ABCDEF, 41
    dev_rng = torch.tensor([seed, step], dtype=torch.int64, device=DEV)
    for p, site, res in [(0.1, 0, True), (0.5, 0xFFFFFFFF, False), (0.0, 1, True), (1.0, 2, True), (1.0, 3, False)]:
        X, R, Y = (Rows(rows, cols, t, pad, 1, v) for t, v in ((xt, xv), (yt, rv), (yt, None)))
        K.op_dropout(rows, cols, X, Y, K.dropout(dev_rng, p, site), res=R if res else None, xtype=types()[xt][0],
                     ytype=types()[yt][0], ldx=X.ld, ldr=R.ld, ldy=Y.ld)
        f = N.dropout_factor(rows * cols, p, seed, step, site).reshape(rows, cols)
        kept = xv.astype(np.float64) * f
        want = kept + rv if res else kept
        got = Y.host()
        # the scale's own rounding, the product's, the sum's
        tol = types()[yt][2] * np.abs(want) + 2.0 ** -24 * (2 * np.abs(kept) + np.abs(want)) * (1 + 2.0 ** -7)
        assert (np.abs(got - want) <= tol).all()
        if not res:
            assert np.array_equal(got == 0, (f == 0) | (xv == 0))


def test_dropped_elements_are_zero_whatever_they_were():
    K = _K()
    rows, cols = 50, 64
    x = torch.full((rows, cols), float("inf"), device=DEV)
    x[1::2] = float("nan")
    rng = torch.tensor([5, 6], dtype=torch.int64, device=DEV)
    y, r = torch.empty_like(x), torch.full_like(x, 2.0)
    K.op_dropout(rows, cols, x, y, K.dropout(rng, 0.4, 1), res=r, xtype=K.TYPE_F32)
    f = torch.from_numpy(N.dropout_factor(rows * cols, 0.4, 5, 6, 1).reshape(rows, cols) == 0).to(DEV)
    torch.cuda.synchronize()
    assert bool((y[f] == 2.0).all()) and not bool(torch.isfinite(y[~f]).any())


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_dropout_in_place(t):
    K = _K()
    ty, dt, _ = types()[t]
    x = torch.randn(77, 123, device=DEV).to(dt)
    r = torch.randn(77, 123, device=DEV).to(dt)
    d = K.dropout(torch.tensor([9, 9], dtype=torch.int64, device=DEV), 0.3, 1)
    y = torch.empty_like(x)
    K.op_dropout(77, 123, x, y, d, res=r, xtype=ty)
    a, b = x.clone(), r.clone()
    K.op_dropout(77, 123, a, a, d, res=r, xtype=ty)
    K.op_dropout(77, 123, x, b, d, res=b, xtype=ty)
    torch.cuda.synchronize()
    assert torch.equal(a, y) and torch.equal(b, y)


def test_offsets_past_32_bits():
    """Elements past 2^32, and rows whose stride passes 2^31 elements."""
    K = _K()
    print("[dropout] past 2^32", flush=True)
    cols = (1 << 32) + 8 * 1003
    x = torch.ones(cols, dtype=torch.bfloat16, device=DEV)
    rng = torch.tensor([3, 4], dtype=torch.int64, device=DEV)
    K.op_dropout(1, cols, x, x, K.dropout(rng, 0.5, 7))
    tail = 8 * 1003 + 64
    want = N.dropout_factor(tail, 0.5, 3, 4, 7, cols - tail)
    assert np.array_equal(host(x[-tail:].float()), want)
    assert np.array_equal(host(x[:64].float()), N.dropout_factor(64, 0.5, 3, 4, 7))
    del x
    ld = (1 << 31) + 24
    wide = torch.empty(2 * ld + 64, dtype=torch.bfloat16, device=DEV)
    rows = torch.stack([wide[k * ld:k * ld + 64] for k in range(3)])
    v = torch.randn(3, 64, device=DEV).to(torch.bfloat16)
    for k in range(3):
        wide[k * ld:k * ld + 64] = v[k]
    y, z = torch.empty_like(v), torch.empty_like(v)
    K.op_dropout(3, 64, wide, y, K.dropout(rng, 0.5, 7), ldx=ld)
    K.op_dropout(3, 64, v, z, K.dropout(rng, 0.5, 7))
    torch.cuda.synchronize()
    assert torch.equal(y, z)
    # the same rows as pixels of a group norm: resident, apply and backward
    ga, be = torch.ones(64, device=DEV), torch.zeros(64, device=DEV)
    outs = []
    for x_, ld_ in ((wide, ld), (v, 64)):
        d = K.gn_desc(1, 3, 64, 4, act=K.ACT_SILU, ldx=ld_)
        yy, st, dd = torch.empty_like(v), torch.empty(8, device=DEV), torch.empty_like(v)
        dg, db = torch.empty(64, device=DEV), torch.empty(64, device=DEV)
        ws = torch.empty(max(16, K.op_gn_workspace_bytes(d, True)), dtype=torch.uint8, device=DEV)
        K.op_gn_forward(d, x_, ga, be, yy, st, ws, ws.numel())
        K.op_gn_backward(d, v, x_, st, ga, be, dd, dg, db, ws, ws.numel())
        outs.append((yy, st, dd, dg, db))
    torch.cuda.synchronize()
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    del rows


# ---------------------------------------------------------------- together --
class Unit:
    """conv 3x3 - group norm - SiLU - dropout - conv 1x1 - dropout + shortcut, on
    the framework's bf16 convolutions: forward, and the backward from kept or
    re-run activations."""

    def __init__(self, rng, n=4, side=14, c=64, groups=8, p=0.25):
        K = _K()
        self.n, self.side, self.c, self.groups = n, side, c, groups
        self.P = n * side * side
        bf = lambda *s, scale=1.0: (torch.randn(*s, device=DEV) * scale).to(torch.bfloat16)
        self.w1, self.w2 = bf(c, 3, 3, c, scale=0.06), bf(c, 1, 1, c, scale=0.15)
        self.gamma, self.beta = 1 + 0.1 * torch.randn(c, device=DEV), 0.1 * torch.randn(c, device=DEV)
        self.g1, self.g2 = K.conv_geo(n, side, side, c, side, side, c, 3, 1, 1), K.conv_geo(n, side, side, c, side, side, c, 1, 1, 0)
        self.desc = K.gn_desc(n, side * side, c, groups, act=K.ACT_SILU, gtype=K.TYPE_F32)
        self.rng, self.d1, self.d2 = rng, K.dropout(rng, p, 1), K.dropout(rng, p, 2)
        self.stats = torch.empty(K.op_gemm_bf16_blocks(self.P, c)[0] * 2 * c, dtype=torch.float64, device=DEV)
        self.ws = torch.empty(max(16, K.op_gn_workspace_bytes(self.desc, False), K.op_gn_workspace_bytes(self.desc, True)),
                              dtype=torch.uint8, device=DEV)
        e = lambda t=torch.bfloat16: torch.empty(self.P, c, dtype=t, device=DEV)
        self.h, self.a, self.b, self.y, self.db_, self.dh = e(), e(), e(), e(), e(), e()
        self.da, self.dx = e(torch.float32), e(torch.float32)
        self.st = torch.empty(2 * n * groups, device=DEV)
        self.dw1, self.dw2 = (torch.empty(w.shape, device=DEV) for w in (self.w1, self.w2))
        self.dgamma, self.dbeta = torch.empty(c, device=DEV), torch.empty(c, device=DEV)

    def forward(self, x, rerun=False, s=None):
        K = _K()
        K.op_conv_bf16_fwd(self.g1, x, self.w1, self.h, self.stats, s)
        if rerun:
            K.op_gn_apply(self.desc, self.h, self.st, self.gamma, self.beta, self.a, drop=self.d1, stream=s)
            return
        K.op_gn_forward(self.desc, self.h, self.gamma, self.beta, self.a, self.st, self.ws, self.ws.numel(),
                        drop=self.d1, stream=s)
        K.op_conv_bf16_fwd(self.g2, self.a, self.w2, self.b, self.stats, s)
        K.op_dropout(self.P, self.c, self.b, self.y, self.d2, res=x, stream=s)

    def backward(self, x, g, s=None):
        """From g = dL/dy (f32): dw1, dw2, dgamma, dbeta and dx = g + the branch's."""
        K = _K()
        K.op_dropout(self.P, self.c, g, self.db_, self.d2, xtype=K.TYPE_F32, ytype=K.TYPE_BF16, stream=s)
        K.op_conv_bf16_wgrad(self.g2, self.a, self.db_, None, 1, self.dw2, s)
        K.op_conv_bf16_dgrad(self.g2, self.db_, self.w2, self.da, stream=s)
        K.op_gn_backward(self.desc, self.da, self.h, self.st, self.gamma, self.beta, self.dh, self.dgamma, self.dbeta,
                         self.ws, self.ws.numel(), drop=self.d1, stream=s)
        K.op_conv_bf16_wgrad(self.g1, x, self.dh, None, 1, self.dw1, s)
        K.op_conv_bf16_dgrad(self.g1, self.dh, self.w1, self.dx, K.EPI_ADD, d=g, stream=s)

    def grads(self):
        return [t.clone() for t in (self.dx, self.dw1, self.dw2, self.dgamma, self.dbeta)]


def test_unit_rerun_gives_the_first_forwards_gradients():
    """A segment of two units: back-propagation through kept activations and through
    activations formed again from the boundary and the statistics agree bit for bit,
    and the gradients match the oracle's."""
    print("[unit] re-run", flush=True)
    torch.manual_seed(5)
    rng = torch.tensor([77, 5], dtype=torch.int64, device=DEV)
    u = Unit(rng)
    x = torch.randn(u.P, u.c, device=DEV).to(torch.bfloat16)
    g = torch.randn(u.P, u.c, device=DEV)
    u.forward(x)
    u.backward(x, g)
    kept = u.grads()
    y, h, a = u.y.clone(), u.h.clone(), u.a.clone()
    for t in (u.h, u.a, u.b, u.y):
        t.fill_(float("nan"))
    u.forward(x, rerun=True)
    assert torch.equal(u.h, h) and torch.equal(u.a, a)
    u.backward(x, g)
    torch.cuda.synchronize()
    for p, q in zip(kept, u.grads()):
        assert torch.equal(p, q)
    # the oracle on the stored tensors: each operator's input is the GPU's own output of the one before
    n, side, c = u.n, u.side, u.c
    nhwc = lambda t: host(t.float()).reshape(n, side, side, c)
    f1, f2 = (N.dropout_factor(u.P * c, 0.25, 77, 5, s) for s in (1, 2))
    mean, rstd = host(u.st).reshape(2, n, u.groups)
    ga, be = host(u.gamma), host(u.beta)
    want = N.gn_apply(nhwc(h).reshape(n, -1, c), mean, rstd, ga, be, "silu", f1)
    got = nhwc(a).reshape(want.shape)
    assert np.abs(got - want).max() <= 2.0 ** -8 * np.abs(want).max()
    b2 = U.conv2d(nhwc(a), host(u.w2.float()), 1, 0)
    want = nhwc(x) + b2 * f2.reshape(b2.shape)
    # two bf16 roundings: of b (times the scale) and of y
    assert (np.abs(nhwc(y) - want) <= 2.0 ** -8 * (np.abs(want) + 1.4 * np.abs(b2)) + 1e-3).all()
    db_ = host(u.db_.float()).reshape(n, side, side, c)
    assert np.abs(db_ - host(g).reshape(db_.shape) * f2.reshape(db_.shape)).max() <= 2.0 ** -8 * np.abs(db_).max()
    da = host(u.da).reshape(n, -1, c)
    d, dga, dbe = N.gn_backward(da, nhwc(h).reshape(n, -1, c), mean, rstd, ga, be, "silu", f1)
    assert np.abs(host(u.dh.float()).reshape(d.shape) - d).max() <= (2.0 ** -8 + 1e-4) * np.abs(d).max()
    assert np.abs(host(kept[3]) - dga).max() <= 1e-4 * np.abs(dga).max()
    assert np.abs(host(kept[4]) - dbe).max() <= 1e-4 * np.abs(dbe).max()
    dh = host(u.dh.float()).reshape(n, side, side, c)
    dx = U.conv2d_dgrad(dh, host(u.w1.float()), (n, side, side, c), 1, 1) + host(g).reshape(n, side, side, c)
    assert np.abs(host(kept[0]).reshape(dx.shape) - dx).max() <= 1e-4 * np.abs(dx).max()


def test_captured_unit_takes_a_new_mask_at_every_step():
    """Forward, re-run and backward of a unit in one graph; the step's number is
    written between replays."""
    print("[unit] captured", flush=True)
    torch.manual_seed(6)
    rng = torch.tensor([78, 0], dtype=torch.int64, device=DEV)
    u, e = Unit(rng, n=2, side=7), None
    torch.manual_seed(6)
    rng_e = torch.tensor([78, 0], dtype=torch.int64, device=DEV)
    e = Unit(rng_e, n=2, side=7)
    x = torch.randn(u.P, u.c, device=DEV).to(torch.bfloat16)
    g = torch.randn(u.P, u.c, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        u.forward(x, s=side)
        u.backward(x, g, s=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        u.forward(x, s=side)
        u.forward(x, rerun=True, s=side)
        u.backward(x, g, s=side)
    seen = []
    for step in (1, 2, 7, 2):
        rng[1] = step
        rng_e[1] = step
        x.copy_(torch.randn(u.P, u.c, device=DEV))
        g.copy_(torch.randn(u.P, u.c, device=DEV))
        graph.replay()
        e.forward(x)
        e.backward(x, g)
        torch.cuda.synchronize()
        assert torch.equal(u.y, e.y)
        for p, q in zip(u.grads(), e.grads()):
            assert torch.equal(p, q)
        seen.append((u.a == 0).clone())
    assert not torch.equal(seen[0], seen[1])


def test_two_calls_at_once():
    """Two streams, each with its own workspace, many calls in flight."""
    print("[gn] two streams", flush=True)
    K = _K()
    cs = [Case(*SHAPES["split"], act="silu", p=0.1, seed=s) for s in (31, 32)]
    want = []
    for c in cs:
        st = c.forward()
        want.append((st, c.Y.all.clone()) + c.backward(st) + (c.D.all.clone(),))
    streams = [torch.cuda.Stream() for _ in cs]
    outs = []
    bufs = []
    for c, s in zip(cs, streams):
        st = torch.empty(2 * c.n * c.groups, device=DEV)
        dg, db = torch.empty(c.c, device=DEV), torch.empty(c.c, device=DEV)
        bufs.append((st, dg, db, c.workspace(False), c.workspace(True)))
        c.Y.m.fill_(0)
        c.D.m.fill_(0)
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        for c, s, (st, dg, db, wf, wb) in zip(cs, streams, bufs):
            K.op_gn_forward(c.desc, c.X, c.ga, c.be, c.Y, st, *wf, drop=c.drop, stream=s)
            K.op_gn_backward(c.desc, c.G, c.X, st, c.ga, c.be, c.D, dg, db, *wb, drop=c.drop, stream=s)
    torch.cuda.synchronize()
    for c, (st, dg, db, _, _), w in zip(cs, bufs, want):
        for a, b in zip((st, c.Y.all, dg, db, c.D.all), w):
            assert torch.equal(a, b)
    del outs
