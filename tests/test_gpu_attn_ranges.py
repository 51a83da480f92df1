"""Attention over packed sequences (op_attn_*) where values go to their limits: special values, in split
keys too, values near the largest, scores of -inf and huge ones.  Against the float64 oracle (oracle.seq)."""
import numpy as np
import pytest

from oracle import seq as S
from seq_cases import host, rounded
from test_gpu_attn import SAME, Case

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# rows for each of the forward's forms: tiles of 128, of 32, and keys split over workgroups
FORMS = {"many": (SAME(200, 77), 4, 2, 64), "few": ([(1, 300), (2, 290)], 4, 2, 128), "split": ([(1, 4096), (1, 3000)], 2, 1, 64)}


def form(name, causal=True, seed=1):
    lens, heads, kv, dim = FORMS[name]
    t = Case(lens, heads, kv, dim, causal, seed=seed)
    assert (t.workspace(False)[1] > 0) == (name == "split")
    return t


def put(t, **tensors):
    for n, v in tensors.items():
        t.v[n] = rounded(v, "bf16")
        t.d[n].copy_(torch.from_numpy(t.v[n]))


def scored(t, scores):
    """Queries and keys whose score is `scores[j]` for each key j of a sequence, or that in bf16."""
    q, k = np.zeros_like(t.v["q"]), np.zeros_like(t.v["k"])
    q[:, :, 0] = 1.0 / t.scale if t.dim == 64 else 8.0
    for c, d in zip(t.koff, t.koff[1:]):
        k[c:d, :, 0] = scores[:d - c, None] * (1.0 if t.dim == 64 else 1.0 / (8.0 * t.scale))
    put(t, q=q, k=k)


def against_oracle(t):
    """o and lse, where the oracle has NaNs too."""
    o, lse, eo, el = S.attention(t.v["q"], t.v["k"], t.v["v"], t.qoff, t.koff, t.causal, t.scale)
    for got, want, err in ((t.whole(t.d["o"]), o, eo), (host(t.lse), lse, el)):
        ok = ~np.isnan(want)
        assert np.array_equal(np.isnan(got), ~ok) and (np.abs(got - want)[ok] <= err[ok] + 1e-30).all()
    return np.isnan(o)


# ------------------------------------------------------- special values --
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("at,score", [(at, s) for s in (0.0, 400.0) for at in (0, 1010, 2000, 4095)])
def test_a_special_value_in_one_split_reaches_the_row(bad, at, score):
    """Whatever another split's score: its probability may be so small that 32 bits hold it as zero,
    times which an infinity is a NaN."""
    t = Case([(1, 4096)], 2, 1, 64, seed=5)
    assert t.workspace(False)[1] > 0
    scores = np.zeros(4096)
    scores[1000] = score
    scored(t, scores)
    t.v["v"][at, 0, 3] = bad
    t.d["v"].copy_(torch.from_numpy(t.v["v"]))
    t.forward()
    o = t.whole(t.d["o"])
    assert not np.isfinite(o[:, :, 3]).any()
    if score == 0.0:
        assert np.array_equal(o[:, :, 3], np.full((1, 2), bad), equal_nan=True)
    assert np.isfinite(np.delete(o, 3, 2)).all() and bool(t.lse.isfinite().all())


@pytest.mark.parametrize("name", FORMS)
@pytest.mark.parametrize("what", ["k", "v"])
def test_special_values_against_the_oracle(name, what):
    t = form(name, seed=7)
    rng = np.random.default_rng(8)
    for at in rng.integers(t.tk // 2, t.tk, 3):
        t.v[what][at, 0, 5] = np.nan
    t.d[what].copy_(torch.from_numpy(t.v[what]))
    t.forward()
    assert against_oracle(t).any()


# --------------------------------------------------------- large values --
@pytest.mark.parametrize("name", FORMS)
@pytest.mark.parametrize("score", [0.0, 2.0, 5.1875, 40.0])
def test_values_near_the_largest(name, score):
    """One key's value near the largest of the type, its score above those that come by before it: o is
    a weighted mean, so it is finite, as it is with exponentials of at most 1."""
    t = form(name)
    scores = np.zeros(4096)
    scores[70] = score  # not in its wavefront's first turn
    scored(t, scores)
    v = t.v["v"] * 1e30
    for c, d in zip(t.koff, t.koff[1:]):
        v[c + 70] = 3.3e38 * np.sign(v[c + 70])
    put(t, v=v)
    t.forward()
    t.check_forward()
    assert np.abs(t.whole(t.d["o"])).max() > 1e34


# ------------------------------------------------------ scores of -inf --
@pytest.mark.parametrize("name", FORMS)
@pytest.mark.parametrize("causal", [True, False])
def test_rows_whose_scores_are_all_minus_infinity(name, causal):
    """exp(-inf) over a sum of such: NaN, and so are the gradients of what such a row sees; what sees no
    such score is as without them."""
    t = form(name, causal)
    k, q = t.v["k"].copy(), t.v["q"].copy()
    k[:, :, 0] = 1.0
    rows = [int(b) - 1 for b in t.qoff[1:2]]  # the first sequence's last query
    for i in rows:
        q[i] = 0.0
        q[i, :, 0] = -np.inf
    t.v["k"], t.v["q"] = k, q
    for n in "qk":
        t.d[n].copy_(torch.from_numpy(t.v[n]))
    t.forward()
    assert against_oracle(t)[rows].all()
    t.backward()
    dq, dk, dv = (t.whole(x) for x in t.grads)
    n = t.koff[1]
    assert np.isnan(dq[rows]).all() and np.isnan(dv[:n]).all() and np.isnan(dk[:n]).all()
    assert np.isfinite(np.delete(dq, rows, 0)).all() and np.isfinite(dv[n:]).all() and np.isfinite(dk[n:]).all()


@pytest.mark.parametrize("name", FORMS)
def test_some_scores_of_minus_infinity(name):
    """They have no part, however many tiles or splits hold nothing else; rows that see nothing else are NaN."""
    t = form(name)
    first = {"many": 130, "few": 65, "split": 1100}[name]
    q, k = np.abs(t.v["q"]) + 0.25, t.v["k"].copy()
    t.v["q"] = rounded(q, "bf16")
    for c, d in zip(t.koff, t.koff[1:]):
        k[c:min(d, c + first), :, 0] = -np.inf
    t.v["k"] = k
    for n in "qk":
        t.d[n].copy_(torch.from_numpy(t.v[n]))
    t.forward()
    o, lse = t.whole(t.d["o"]), host(t.lse)
    i = 0
    for a, b, c, d in zip(t.qoff, t.qoff[1:], t.koff, t.koff[1:]):
        for r in range(a, b):
            lim = r - a + (d - c) - (b - a) + 1
            if lim <= first:
                assert np.isnan(o[r]).all() and np.isnan(lse[:, r]).all()
                continue
            for h in range(t.heads):
                kh = h // (t.heads // t.kv)
                keys, v, query = t.v["k"][c + first:c + lim, kh], t.v["v"][c + first:c + lim, kh], t.v["q"][r, h]
                e = keys @ query * t.scale
                p = np.exp(e - e.max())
                # a score is a sum of dim products; weights and the output are rounded to bf16
                rel = (t.dim + 16) * S.U24 * 2 * ((np.abs(keys) @ query).max() * t.scale + abs(e.max())) + (lim + 64) * S.U24
                want, mag = p @ v / p.sum(), p @ np.abs(v) / p.sum()
                assert (np.abs(o[r, h] - want) <= (S.U16 + 2 * rel) * mag + 2 * S.U16 * np.abs(want)).all()
                log = e.max() + np.log(p.sum())
                assert abs(lse[h, r] - log) <= rel + 4 * S.U24 * abs(log)
            i += 1
    assert i > 0


def test_rows_that_see_no_key_are_zeros_beside_them():
    t = Case([(9, 4), (1, 0), (1, 5)], 2, 1, 64)
    t.check()
    assert not t.whole(t.d["o"])[[0, 1, 2, 3, 4, 9]].any() and bool(t.lse[:, [0, 1, 2, 3, 4, 9]].isneginf().all())


# --------------------------------------------------------- huge scores --
@pytest.mark.parametrize("name", FORMS)
@pytest.mark.parametrize("size", [300.0, 3000.0, 20000.0, 30000.0, 1e8, 1e15])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_huge_scores(name, size, sign):
    """Scores that 32 bits hold to many whole numbers only, up to 1e31: equal ones have equal
    weights, those far below have none, and nothing overflows."""
    t = form(name)
    q, k = np.full_like(t.v["q"], size), np.full_like(t.v["k"], sign * size)
    rng = np.random.default_rng(3)
    low = rng.random(t.tk) < 0.5
    low[t.koff[:-1]] = False  # a key that every query sees
    k[low] *= -sign if sign > 0 else 4.0  # all below the others
    put(t, q=q, k=k)
    t.forward()
    o, lse = t.whole(t.d["o"]), host(t.lse)
    top = t.dim * t.v["q"][0, 0, 0] * t.v["k"][t.koff[0], 0, 0] * t.scale
    for a, b, c, d in zip(t.qoff, t.qoff[1:], t.koff, t.koff[1:]):
        for r in range(a, b):
            lim = r - a + (d - c) - (b - a) + 1
            v = np.repeat(t.v["v"][c:c + lim][~low[c:c + lim]], t.heads // t.kv, 1)
            # weights and the output rounded to bf16, fp32 sums of at most 4096 values
            want, mag = v.mean(0), np.abs(v).mean(0)
            assert (np.abs(o[r] - want) <= S.U16 * (mag + 2 * np.abs(want)) + (lim + 64) * S.U24 * mag).all()
            # a score is a sum of dim products, scaled and taken to base 2 and back
            assert (np.abs(lse[:, r] - (top + np.log(len(v)))) <= (t.dim + 8) * S.U24 * abs(top) + 1e-4).all()


@pytest.mark.parametrize("size", [1.0, 30000.0, 1e8])
def test_huge_scores_beside_rows_that_see_nothing(size):
    """In one wavefront: rows without keys, rows of small scores, and rows of huge ones."""
    t = Case([(100, 61), (70, 70)], 2, 2, 64)
    q = t.v["q"].copy()
    q[::3] *= size
    put(t, q=q)
    t.forward()
    o, lse = t.whole(t.d["o"]), host(t.lse)
    assert not o[:39].any() and np.isneginf(lse[:, :39]).all()
    assert np.isfinite(o).all() and np.isfinite(lse[:, 39:]).all()
    want, wl, eo, el = S.attention(t.v["q"], t.v["k"], t.v["v"], t.qoff, t.koff, True, t.scale)
    small = np.arange(170) % 3 != 0
    assert (np.abs(o - want)[small] <= eo[small] + 1e-30).all()
    some = np.flatnonzero(small)[np.flatnonzero(small) >= 39]
    assert (np.abs(lse[:, some] - wl[:, some]) <= el[:, some]).all()


@pytest.mark.parametrize("size", [3.0, 30.0, 100.0, 300.0])
def test_gradients_of_large_scores(size):
    """Of a row that sees one key p is 1, off by the roundings of its lse: half a step of fp32 each where it is
    stored and taken to base 2 and back, and of the score, below 4 of them.  dv = p g."""
    t = Case(SAME(*[1] * 40), 2, 2, 64)
    put(t, q=np.full_like(t.v["q"], size), k=np.full_like(t.v["k"], size))
    t.forward()
    t.backward()
    g, lse = t.v["g"], host(t.lse).T[:, :, None]
    # p and dv are rounded to bf16
    assert (np.abs(t.whole(t.grads[2]) - g) <= (lse * 4 * S.U24 + 2.1 * S.U16) * np.abs(g)).all()
