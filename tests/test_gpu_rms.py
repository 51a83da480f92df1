"""GPU parity of the RMS norm (op_rms_*) with the float64 oracle on the same inputs.

Bars, per element: half a step of the output's type for the rounding at the end, plus
L 2^-24 times the magnitudes that enter it for the fp32 arithmetic.  A row's sum
runs over at most 16 values in a thread and trees of 64 lanes and 16 wavefronts (below
16 + 6 + 16 operations), a column's over at most 40 rows here in a team, 4 teams, 32
records and 16 wavefronts; the few operations before and after are covered by the distance to 256.
"""
import numpy as np
import pytest

from oracle import seq as S
from seq_cases import DEV, STEP, K, Rows, close, code, dtype, f32, host, rounded

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

L = 256 * 2.0 ** -24
EPS = 1e-5
# widths of every team and vector count, full and not, and odd ones
WIDTHS = [1, 7, 8, 64, 333, 512, 513, 1000, 1024, 1025, 2047, 2048, 2049, 4096, 4100, 8192, 8200, 16381, 16384]


class Case:
    def __init__(self, rows, c, x="bf16", h="bf16", y="bf16", g="bf16", d=None, res=True, group=0, pad=0, shift=0, seed=1,
                 level=1.0):
        d = d or h
        rng = np.random.default_rng(seed)
        self.__dict__.update(rows=rows, c=c, x=x, h=h, y=y, g=g, d=d, res=res, group=group)
        n = lambda: rng.standard_normal((rows, c)) * np.exp(0.5 * rng.standard_normal(c)) * level
        self.xv = rounded(n(), x)
        self.rv = rounded(n(), h) if res else None
        self.hv = rounded((self.xv.astype(np.float32) + self.rv.astype(np.float32)), h) if res else self.xv
        self.gv, self.ghv = rounded(rng.standard_normal((rows, c)), g), rounded(rng.standard_normal((rows, c)), d)
        self.w = rounded(1 + 0.3 * rng.standard_normal(c), "f32")
        self.X, self.R = Rows(rows, c, x, pad, shift, self.xv), Rows(rows, c, h, pad, shift, self.rv) if res else None
        self.H = Rows(rows, c, h, pad, shift) if res else None
        self.Y, self.G = Rows(rows, c, y, pad, shift), Rows(rows, c, g, pad, shift, self.gv)
        self.D, self.GH = Rows(rows, c, d, pad, shift), Rows(rows, c, d, pad, shift, self.ghv) if res else None
        self.W, self.ST = f32(self.w), torch.full((rows,), -7.0, device=DEV)
        self.groups = -(-c // (group or c))
        self.YS = torch.full((rows, self.groups), -7.0, device=DEV) if y == "f8" else None
        ld = c + pad
        self.desc = K().rms_desc(rows, c, xtype=code(x), htype=code(h), ytype=code(y), gtype=code(g), dtype=code(d),
                                 qgroup=group, ldx=ld, ldh=ld, ldy=ld, ldg=ld, ldd=ld, eps=EPS)

    def forward(self):
        K().op_rms_forward(self.desc, self.X, self.W, self.Y, self.ST, res=self.R, h=self.H, ys=self.YS)

    def backward(self, dw=None):
        nb = K().op_rms_workspace_bytes(self.desc)
        ws = torch.full((nb + 64,), 255, dtype=torch.uint8, device=DEV)
        self.DW = torch.full((self.c,), -7.0, device=DEV)
        K().op_rms_backward(self.desc, self.G, self.H or self.X, self.ST, self.W, self.D, self.DW, ws, nb, gh=self.GH)
        torch.cuda.synchronize()
        assert bool((ws[nb:] == 255).all()), "written past the workspace"

    def check_y(self, st):
        u = S.rms_apply(self.hv, st, self.w)
        if self.y != "f8":
            close("y", self.Y.host(), u, (STEP[self.y] + L) * np.abs(u))
            return
        scale, ys = S.group_scales(u, self.group), host(self.YS)
        close("scales", ys, scale, L * scale)
        wide = np.repeat(ys, self.group or self.c, 1)[:, :self.c]
        # half a step: 2^-4 of a normal value, 2^-10 of the scale below 2^-6 scales
        close("y", self.Y.host() * wide, u, (2.0 ** -4 + L) * np.abs(u) + 2.0 ** -10 * wide)

    def check_forward(self):
        st = S.rms_stat(self.hv, EPS)
        close("st", host(self.ST), st, L * st)
        if self.res:
            assert np.array_equal(self.H.host(), self.hv)
        self.check_y(st)

    def check_backward(self):
        st = host(self.ST)
        d, dw, md, mw = S.rms_backward(self.gv, self.ghv if self.res else None, self.hv, st, self.w)
        close("d", self.D.host(), d, STEP[self.d] * np.abs(d) + L * md)
        close("dw", host(self.DW), dw, L * mw + 2.0 ** -24 * np.abs(dw))


@pytest.mark.parametrize("c", WIDTHS)
def test_widths(c):
    rows = 67 if c <= 4100 else 9
    for kw in (dict(y="bf16"), dict(y="f8", res=False), dict(x="f32", h="f32", y="f32", g="f32", pad=3, shift=1)):
        t = Case(rows, c, **kw)
        t.forward()
        t.check_forward()
        t.backward()
        t.check_backward()


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("h", ["bf16", "f32"])
@pytest.mark.parametrize("y", ["bf16", "f32", "f8"])
def test_types(x, h, y):
    for res in ((True, False) if x == h else (True,)):
        t = Case(33, 200, x=x, h=h, y=y, res=res, pad=8)
        t.forward()
        t.check_forward()


@pytest.mark.parametrize("g", ["bf16", "f32"])
@pytest.mark.parametrize("h", ["bf16", "f32"])
@pytest.mark.parametrize("d", ["bf16", "f32"])
def test_gradient_types(g, h, d):
    for res in (True, False):
        t = Case(70, 264, x=h, h=h, g=g, d=d, res=res, pad=5, shift=3)
        t.forward()
        t.backward()
        t.check_backward()


@pytest.mark.parametrize("group", [0, 8, 16, 32, 64, 128, 256, 512])
@pytest.mark.parametrize("c", [40, 1000, 1024, 4600])
def test_8_bit_groups(group, c):
    t = Case(19, c, y="f8", group=group, pad=1)
    t.forward()
    t.check_forward()


@pytest.mark.parametrize("rows", [1, 2, 3, 5, 2049, 70001])
def test_row_counts(rows):
    t = Case(rows, 72)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()


@pytest.mark.parametrize("y,group,c", [("bf16", 0, 1000), ("f8", 128, 1024), ("f8", 0, 4104), ("f32", 0, 12000)])
def test_rerun_gives_the_same_bits(y, group, c):
    t = Case(21, c, y=y, group=group)
    t.forward()
    again, ys = Rows(t.rows, c, y), torch.empty_like(t.YS) if t.YS is not None else None
    K().op_rms_apply(t.desc, t.H, t.ST, t.W, again, ys=ys)
    assert np.array_equal(again.host(), t.Y.host())
    if ys is not None:
        assert torch.equal(ys, t.YS)


def test_rows_of_zeros_and_of_tiny_values():
    t = Case(4, 96, y="f8", group=32, res=False)
    t.X.m[0].zero_()
    t.X.m[1].fill_(1e-37)
    t.X.m[2, :40].zero_()
    t.xv = t.hv = t.X.host()
    t.forward()
    t.check_forward()
    assert host(t.YS)[0].max() <= 1e-30 / 448 * (1 + L)


def test_special_values_stay_in_their_row_and_group():
    t = Case(5, 256, y="f8", group=64)
    t.X.m[1, 70] = float("nan")
    t.X.m[3, 200] = float("inf")
    t.forward()
    y = t.Y.host() * np.repeat(host(t.YS), 64, 1)
    assert np.isnan(y[1]).all()  # the row's statistic is NaN
    assert np.isnan(y[3, 192:]).all()  # infinite mean square: st = 0, inf 0
    for r in (0, 2, 4):
        u = S.rms_apply(t.hv, S.rms_stat(t.hv, EPS), t.w)[r]
        close("y", y[r], u, (2.0 ** -4 + L) * np.abs(u) + 2.0 ** -10 * np.repeat(host(t.YS), 64, 1)[r])


def test_outputs_over_inputs():
    t = Case(37, 520)
    t.forward()
    t.check_forward()
    k, want, hsum = K(), t.Y.host(), t.H.host()
    k.op_rms_forward(t.desc, t.X, t.W, t.X, t.ST, res=t.R, h=t.R)  # y over x, h over res
    assert np.array_equal(t.X.host(), want) and np.array_equal(t.R.host(), hsum)
    t.backward()
    d = t.D.host()
    nb = k.op_rms_workspace_bytes(t.desc)
    ws = torch.empty(nb, dtype=torch.uint8, device=DEV)
    for over in (t.G, t.GH, t.H):
        keep = over.m.clone()
        k.op_rms_backward(t.desc, t.G, t.H, t.ST, t.W, over, t.DW, ws, nb, gh=t.GH)
        assert np.array_equal(over.host(), d)
        over.m.copy_(keep)


def test_captured_and_replayed():
    t = Case(300, 1024, y="f8", group=128)
    k = K()
    nb = k.op_rms_workspace_bytes(t.desc)
    ws, dw = torch.empty(nb, dtype=torch.uint8, device=DEV), torch.empty(t.c, device=DEV)
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()

    def run(stream):
        k.op_rms_forward(t.desc, t.X, t.W, t.Y, t.ST, res=t.R, h=t.H, ys=t.YS, stream=stream)
        k.op_rms_backward(t.desc, t.G, t.H, t.ST, t.W, t.D, dw, ws, nb, gh=t.GH, stream=stream)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        run(torch.cuda.current_stream())
    for seed in range(3):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        t.X.m.copy_(torch.randn(t.rows, t.c, generator=gen, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone().view(torch.uint8) for v in (t.Y.m, t.YS, t.ST, t.H.m, t.D.m, dw)]
        run(None)
        torch.cuda.synchronize()
        for a, b in zip(got, (t.Y.m, t.YS, t.ST, t.H.m, t.D.m, dw)):
            assert torch.equal(a, b.clone().view(torch.uint8))


def test_offsets_past_32_bits():
    # a row 2^32 elements behind the first
    c, ld = 64, 1 << 31
    big = torch.empty(2 * ld + c, dtype=torch.bfloat16, device=DEV)
    m = big.as_strided((3, c), (ld, 1))
    v = torch.randn(3, c, device=DEV).to(torch.bfloat16)
    m.copy_(v)
    y, st, w = torch.empty(3, c, device=DEV), torch.empty(3, device=DEV), torch.ones(c, device=DEV)
    desc = K().rms_desc(3, c, ytype=K().TYPE_F32, ldx=ld, eps=EPS)
    K().op_rms_forward(desc, big, w, y, st)
    h = host(v)
    u = S.rms_apply(h, S.rms_stat(h, EPS), np.ones(c))
    close("y", host(y), u, L * np.abs(u))
