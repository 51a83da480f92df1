"""GPU parity of attention over packed sequences (op_attn_*) with the float64 oracle, whose bounds
of rounding (oracle.seq) are the bars."""
import numpy as np
import pytest

from oracle import seq as S
from seq_cases import DEV, K, close, host, rounded

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

GUARD = 1232.0  # a value of bf16


class Case:
    """lens: (queries, keys) of each sequence; layout: how the heads lie in memory; before and
    after: rows of no sequence at the tensors' ends."""

    def __init__(self, lens, heads, kv, dim, causal=True, scale=0.0, layout="rows", before=0, after=0, seed=1, amp=1.0):
        rng = np.random.default_rng(seed)
        self.heads, self.kv, self.dim, self.causal = heads, kv, dim, causal
        self.scale = float(np.float32(scale or dim ** -0.5))
        self.qoff = np.concatenate([[0], np.cumsum([a for a, _ in lens])]) + before
        self.koff = np.concatenate([[0], np.cumsum([b for _, b in lens])]) + before
        self.tq, self.tk = int(self.qoff[-1]) + after, int(self.koff[-1]) + after
        self.dims = dict(q=(self.tq, heads), k=(self.tk, kv), v=(self.tk, kv), o=(self.tq, heads))
        self.st, self.buf = {}, {}
        for n, (t, h) in self.dims.items():
            self.st[n] = dict(rows=(h * dim, dim), heads=(dim, max(t, 1) * dim + 8), wide=(h * (dim + 8) + 16, dim + 8))[layout]
        self.v = {n: rounded(rng.standard_normal((t, h, dim)) * amp, "bf16") for n, (t, h) in self.dims.items()}
        self.v["g"] = rounded(rng.standard_normal((self.tq, heads, dim)), "bf16")
        self.d = {n: self.tensor(n, self.v[n]) for n in "qkv"}
        self.d["g"] = self.tensor("o", self.v["g"])
        self.d["o"] = self.tensor("o")
        self.lse = torch.full((heads, self.tq), GUARD, device=DEV)
        off = lambda v: torch.from_numpy(v.astype(np.int32)).to(DEV)
        self.dqoff, self.dkoff = off(self.qoff), off(self.koff)
        k = K()
        self.desc = k.attn_desc(self.tq, self.tk, len(lens), heads, kv, dim, causal=causal, scale=scale,
                                **{p + n: s for n in "qkvo" for p, s in zip(("ld", "hs"), self.st[n])})

    def tensor(self, n, data=None):
        t, h = self.dims[n]
        a, b = self.st[n]
        buf = torch.full((a * max(t, 1) + b * h + 64,), GUARD, dtype=torch.bfloat16, device=DEV)
        m = buf.as_strided((t, h, self.dim), (a, b, 1))
        if data is not None:
            m.copy_(torch.from_numpy(np.ascontiguousarray(data)))
        self.buf[m.data_ptr()] = buf
        return m

    def whole(self, m):
        """The tensor's values; what lies between them is checked to be as it was."""
        torch.cuda.synchronize()
        v = m.double().cpu().numpy()
        rest = self.buf[m.data_ptr()].clone()
        rest.as_strided(m.shape, m.stride()).fill_(GUARD)
        assert bool((rest == GUARD).all()), "written outside its rows"
        return v

    def workspace(self, backward):
        nb = K().op_attn_workspace_bytes(self.desc, backward)
        return torch.full((nb + 64,), 255, dtype=torch.uint8, device=DEV), nb

    def forward(self, stream=None):
        ws, nb = self.workspace(False)
        d = self.d
        K().op_attn_forward(self.desc, d["q"], d["k"], d["v"], self.dqoff, self.dkoff, d["o"], self.lse, ws, nb, stream=stream)
        torch.cuda.synchronize()
        assert bool((ws[nb:] == 255).all()), "written past the workspace"

    def backward(self):
        ws, nb = self.workspace(True)
        d = self.d
        self.grads = [self.tensor(n) for n in "qkv"]
        K().op_attn_backward(self.desc, d["g"], d["q"], d["k"], d["v"], d["o"], self.lse, self.dqoff, self.dkoff,
                             *self.grads, ws, nb)
        torch.cuda.synchronize()
        assert bool((ws[nb:] == 255).all()), "written past the workspace"

    def outside(self, got, want, name):
        """Rows of no sequence (NaN in the oracle) hold what they held."""
        none = np.isnan(want)
        assert (got[none] == GUARD).all(), name
        return np.where(none, 0.0, got), np.where(none, 0.0, want)

    def check_forward(self):
        o, lse, eo, el = S.attention(self.v["q"], self.v["k"], self.v["v"], self.qoff, self.koff, self.causal, self.scale)
        g, w = self.outside(self.whole(self.d["o"]), o, "o")
        close("o", g, w, np.nan_to_num(eo))
        g, w = self.outside(host(self.lse), lse, "lse")
        close("lse", g, w, np.nan_to_num(el) + 1e-30)

    def check_backward(self):
        o, lse = self.whole(self.d["o"]), host(self.lse)
        want, err = S.attention_backward(self.v["g"], self.v["q"], self.v["k"], self.v["v"], o, lse, self.qoff,
                                         self.koff, self.causal, self.scale)
        for n, got, w, e in zip(("dq", "dk", "dv"), self.grads, want, err):
            a, b = self.outside(self.whole(got), w, n)
            close(n, a, b, np.nan_to_num(e))

    def check(self):
        self.forward()
        self.check_forward()
        self.backward()
        self.check_backward()


SAME = lambda *n: [(k, k) for k in n]

SHAPES = {
    "one_token": (SAME(1), 1, 1, 8),
    "one_tile": (SAME(128), 2, 1, 128),
    "odd": (SAME(77), 3, 3, 64),
    "two_tiles_and_one": (SAME(129), 2, 2, 128),
    "long": (SAME(700), 4, 1, 128),
    "long_narrow": (SAME(643), 2, 2, 40),
    "ragged": (SAME(1, 64, 63, 200, 2, 0, 131, 1), 6, 2, 64),
    "ragged_wide": (SAME(5, 190, 31, 0, 0, 66), 8, 2, 128),
    "many_short": (SAME(*([3, 1, 7, 2] * 40)), 4, 4, 72),
    "groups_of_three": (SAME(150, 20), 9, 3, 96),
    "one_key_head": (SAME(90, 33), 16, 1, 128),
    "after_earlier": ([(1, 300), (5, 77), (64, 64), (33, 1000)], 8, 2, 128),
    "single_tokens": ([(1, n) for n in (1, 64, 127, 128, 129, 1000, 33)], 8, 2, 128),
    "single_tokens_narrow": ([(1, n) for n in (5, 256, 700)], 4, 4, 48),
    "more_queries_than_keys": ([(100, 30), (5, 0), (40, 39), (0, 12)], 4, 2, 64),
    "widest_group": (SAME(3, 40), 40, 1, 32),
}


@pytest.mark.parametrize("name", SHAPES)
@pytest.mark.parametrize("causal", [True, False])
def test_shapes(name, causal):
    lens, heads, kv, dim = SHAPES[name]
    Case(lens, heads, kv, dim, causal).check()


@pytest.mark.parametrize("dim", range(8, 129, 8))
def test_widths(dim):
    Case(SAME(70, 9), 2, 1, dim, seed=dim).check()


@pytest.mark.parametrize("layout", ["rows", "heads", "wide"])
@pytest.mark.parametrize("dim", [24, 64, 128])
def test_layouts_and_rows_of_no_sequence(layout, dim):
    Case(SAME(40, 0, 150), 6, 3, dim, layout=layout, before=5, after=70).check()
    Case([(1, 400), (1, 3), (1, 0)], 6, 3, dim, layout=layout, before=3, after=9).check()


@pytest.mark.parametrize("scale", [0.01, 1.0, 3.0])
def test_scales(scale):
    Case(SAME(130), 2, 2, 64, scale=scale).check()


def test_keys_split_over_workgroups():
    """Few rows with many keys: unfinished rows are joined."""
    for lens, heads, kv, dim in (([(1, 5000)], 8, 2, 128), ([(1, 3000), (1, 1), (1, 0), (1, 2222)], 4, 4, 64),
                                 ([(300, 4000)], 2, 1, 128)):
        t = Case(lens, heads, kv, dim)
        assert t.workspace(False)[1] > 0
        t.check()


def test_large_scores():
    """Scores of hundreds: the running maximum keeps the exponentials in range."""
    Case(SAME(300), 2, 1, 64, amp=6.0).check()


def test_falling_and_rising_scores():
    """The maximum moves in every tile, or never after the first."""
    for sign in (1.0, -1.0):
        t = Case(SAME(400), 1, 1, 64)
        t.v["q"][:] = 0
        t.v["q"][:, :, 0] = 8.0
        t.v["k"][:, :, 0] = rounded(sign * np.arange(400)[:, None] / 8.0, "bf16")
        for n in "qk":
            t.d[n].copy_(torch.from_numpy(t.v[n]))
        t.check()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_hidden_values_have_no_part(bad):
    """Keys and values that a query does not see, and gradients of queries that a key is not
    seen by, may hold anything: here the last key's rows and the first queries' gradients are so,
    and what does not see them comes out as without them."""
    n = 200
    clean = Case(SAME(n), 4, 2, 128)
    clean.forward()
    o, lse, eo, el = S.attention(clean.v["q"], clean.v["k"], clean.v["v"], clean.qoff, clean.koff, True, clean.scale)
    t = Case(SAME(n), 4, 2, 128)
    t.d["k"][n - 1], t.d["v"][n - 1] = bad, bad
    t.forward()
    close("o", t.whole(t.d["o"])[:n - 1], o[:n - 1], eo[:n - 1])
    assert torch.equal(t.lse[:, :n - 1], clean.lse[:, :n - 1])
    t.d["o"].copy_(clean.d["o"])
    t.lse.copy_(clean.lse)
    t.backward()
    want, err = S.attention_backward(clean.v["g"], clean.v["q"], clean.v["k"], clean.v["v"], clean.whole(clean.d["o"]),
                                     host(clean.lse), clean.qoff, clean.koff, True, clean.scale)
    close("dq", t.whole(t.grads[0])[:n - 1], want[0][:n - 1], err[0][:n - 1])
    t = Case(SAME(n), 4, 2, 128)
    t.d["o"].copy_(clean.d["o"])
    t.lse.copy_(clean.lse)
    t.d["q"][0], t.d["g"][0] = bad, bad
    t.backward()
    close("dk", t.whole(t.grads[1])[1:], want[1][1:], err[1][1:])
    close("dv", t.whole(t.grads[2])[1:], want[2][1:], err[2][1:])


@pytest.mark.parametrize("causal,n,heads,kv", [(True, 200, 2, 1), (True, 333, 2, 2), (False, 150, 4, 2), (True, 1, 2, 1)])
@pytest.mark.parametrize("dim", [64, 128])
def test_special_values_that_are_seen(causal, n, heads, kv, dim):
    """An infinity or a NaN among the values reaches the rows that see it, and no others; among
    the gradients, the keys that are seen by its query; wherever in a tile it lies."""
    rng = np.random.default_rng(n + dim)
    for at in sorted({0, n - 1, *rng.integers(0, n, 12).tolist()}):
        t = Case(SAME(n), heads, kv, dim, causal)
        bad = float(rng.choice([np.nan, np.inf, -np.inf]))
        t.d["v"][at, :, 3] = bad
        t.forward()
        o = t.whole(t.d["o"])
        see = np.arange(n) >= at if causal else np.ones(n, bool)
        assert np.array_equal(o[see, :, 3], np.full((see.sum(), heads), bad), equal_nan=True)
        assert np.isfinite(o[~see]).all() and np.isfinite(np.delete(o, 3, 2)).all()
        t = Case(SAME(n), heads, kv, dim, causal)
        t.forward()
        t.d["g"][at, :, 5] = bad
        t.backward()
        dq, dk, dv = (t.whole(x) for x in t.grads)
        see = np.arange(n) <= at if causal else np.ones(n, bool)
        assert not np.isfinite(dv[see, :, 5]).any() and np.isfinite(dv[~see]).all()
        assert np.isfinite(np.delete(dv, 5, 2)).all()
        # g v^T and its row's sum are infinite or NaN, their difference too
        assert not np.isfinite(dk[see]).any() and np.isfinite(dk[~see]).all()
        assert not np.isfinite(dq[at]).any() and np.isfinite(np.delete(dq, at, 0)).all()


def test_values_behind_a_sequence_have_no_part():
    """The rows behind a sequence's last, in its last tile, are the next sequence's or nobody's."""
    for causal in (True, False):
        a = Case(SAME(100, 40), 4, 2, 64, causal, after=30)
        a.forward()
        a.backward()
        b = Case(SAME(100, 40), 4, 2, 64, causal, after=30)
        for n in "qkvg":
            b.d[n][100:] = float("nan")
        b.forward()
        b.lse[:, 100:].fill_(float("nan"))
        b.d["o"][100:] = float("nan")
        b.backward()
        for x, y in zip((a.d["o"], *a.grads), (b.d["o"], *b.grads)):
            assert torch.equal(x[:100], y[:100])
        assert torch.equal(a.lse[:, :100], b.lse[:, :100])


def test_the_same_bits_again():
    t = Case(SAME(300, 77, 190), 8, 2, 128)
    t.check()
    first = [x.clone() for x in (t.d["o"], t.lse, *t.grads)]
    for _ in range(3):
        t.forward()
        t.backward()
        for a, b in zip(first, (t.d["o"], t.lse, *t.grads)):
            assert torch.equal(a, b)


def test_captured_replayed_with_other_lengths():
    """Offsets are read when the kernels run; two graphs with workspaces of their own."""
    k, graphs = K(), []
    cases = [Case(SAME(100, 60, 40), 4, 2, 64), Case([(1, 900), (1, 500)], 4, 2, 64)]
    for t in cases:
        ws = [t.workspace(b) for b in (False, True)]
        t.grads = [t.tensor(n) for n in "qkv"]
        t.keep = ws
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            s, d = torch.cuda.current_stream(), t.d
            k.op_attn_forward(t.desc, d["q"], d["k"], d["v"], t.dqoff, t.dkoff, d["o"], t.lse, *ws[0], stream=s)
            k.op_attn_backward(t.desc, d["g"], d["q"], d["k"], d["v"], d["o"], t.lse, t.dqoff, t.dkoff, *t.grads,
                               *ws[1], stream=s)
        graphs.append(graph)
    for qoff, koff in (([0, 100, 160, 200], [0, 900, 1400]), ([0, 0, 199, 200], [0, 3, 1400]), ([0, 64, 128, 200], [0, 700, 1400])):
        cases[0].qoff = cases[0].koff = np.array(qoff)
        cases[1].koff = np.array(koff)
        for t in cases:
            t.dqoff.copy_(torch.from_numpy(t.qoff.astype(np.int32)))
            t.dkoff.copy_(torch.from_numpy(t.koff.astype(np.int32)))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for t in cases:
            t.check_forward()
            t.check_backward()


def test_offsets_past_32_bits():
    """A cache whose last rows lie behind 2^32 elements."""
    lk, heads, dim = 300, 1, 64
    ld = (1 << 32) // 296 // 8 * 8
    big = torch.empty(lk * ld + 64, dtype=torch.bfloat16, device=DEV)
    rng = np.random.default_rng(2)
    q, kv = rounded(rng.standard_normal((2, heads, dim)), "bf16"), rounded(rng.standard_normal((lk, heads, dim)), "bf16")
    big.as_strided((lk, heads, dim), (ld, dim, 1)).copy_(torch.from_numpy(kv))
    dq = torch.from_numpy(q).to(torch.bfloat16).to(DEV)
    o, lse = torch.empty_like(dq), torch.empty(heads, 2, device=DEV)
    k = K()
    desc = k.attn_desc(2, lk, 1, heads, heads, dim, ldk=ld, ldv=ld)
    off = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    nb = k.op_attn_workspace_bytes(desc, False)
    ws = torch.empty(max(nb, 16), dtype=torch.uint8, device=DEV)
    k.op_attn_forward(desc, dq, big, big, off(0, 2), off(0, lk), o, lse, ws, nb)
    wo, wl, eo, el = S.attention(q, kv, kv, np.array([0, 2]), np.array([0, lk]), True, dim ** -0.5)
    close("o", host(o), wo, eo)
    close("lse", host(lse), wl, el)


@pytest.mark.parametrize("lens,heads,kv,dim", [(SAME(200, 1, 33, 1, 129), 4, 2, 64), (SAME(1, 1, 2, 1), 8, 2, 128),
                                               ([(40, 1), (9, 9), (1, 3000)], 2, 2, 40)], ids=["many", "few", "split"])
def test_a_row_that_sees_one_key_gets_its_value(lens, heads, kv, dim):
    """Whatever the score and the rounding of its exponential."""
    t = Case(lens, heads, kv, dim, seed=11, amp=3.0)
    t.forward()
    o, n = t.whole(t.d["o"]), 0
    for a, b, c, d in zip(t.qoff, t.qoff[1:], t.koff, t.koff[1:]):
        i = a + (b - a) - (d - c)  # the query that sees the first key alone
        if a <= i < b:
            assert np.array_equal(o[i], np.repeat(t.v["v"][c], heads // kv, 0))
            n += 1
    assert n >= 2


@pytest.mark.parametrize("keys", [300, 1025, 3400, 15873, 16400])
def test_numbers_of_splits(keys):
    """1, 4, 13, 62 and 64 of them for one head."""
    t = Case([(1, keys)], 1, 1, 64, seed=keys)
    t.forward()
    t.check_forward()


@pytest.mark.parametrize("at,score", [(0, 0.0), (2000, 0.0), (4095, 0.0), (2000, 400.0)])
def test_a_seen_nan_in_one_split(at, score):
    """The only finite score of a split or not, and however far below another split's it is."""
    t = Case([(1, 4096)], 2, 1, 64, seed=5)
    t.d["q"].fill_(1.0)
    t.d["k"].fill_(0.0)
    t.d["k"][1000, 0] = score / 8
    t.d["k"][at, 0, 3] = float("nan")
    t.forward()
    torch.cuda.synchronize()
    assert bool(t.d["o"].isnan().all()) and bool(t.lse.isnan().all())


def test_a_past_of_more_tiles_than_32_bits_hold():
    """Four single tokens of 128 heads on one key head, one of them behind 2^29 keys: one key has a
    score of 40 and the others of 0, so the answer is its value (they add 2^29 exp(-40) < 2^-28 of it)."""
    n, heads, dim, at = 1 << 29, 128, 8, (1 << 29) - 12345
    k = torch.zeros(n + 3, 1, dim, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    k[at], v[at] = 5.0, torch.arange(1.0, dim + 1, device=DEV).to(torch.bfloat16)
    v[n:] = 3.0
    q = torch.ones(4, heads, dim, dtype=torch.bfloat16, device=DEV)
    o, lse = torch.full_like(q, GUARD), torch.full((heads, 4), GUARD, device=DEV)
    c = K()
    desc = c.attn_desc(4, n + 3, 4, heads, 1, dim, scale=1.0)
    off = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    nb = c.op_attn_workspace_bytes(desc, False)
    ws = torch.empty(max(nb, 16), dtype=torch.uint8, device=DEV)
    c.op_attn_forward(desc, q, k, v, off(0, 1, 2, 3, 4), off(0, n, n + 1, n + 2, n + 3), o, lse, ws, nb)
    want = np.full((4, heads, dim), 3.0)
    want[0] = np.arange(1, dim + 1)
    # the probability and the output are rounded to bf16, half a step each
    close("o", host(o), want, (2 * S.U16 + 2.0 ** -20) * want)
    wl = np.zeros((heads, 4))
    wl[:, 0] = 40.0
    # a logarithm of a few operations on numbers up to 40 / ln 2, and 2^-28 of the others
    close("lse", host(lse), wl, np.where(wl > 0, 64 * 8 * S.U24, 8 * S.U24))
