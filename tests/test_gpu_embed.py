"""GPU parity of the embedding and its gradient (op_embed_*) with the float64 oracle.

Bars: half a step of the output's type, plus for a gradient the chain of sums that a row
of n tokens of one id may pass, 2^-24 of the sum of magnitudes each: at most 64 in a wavefront,
then ceil(n / 16) pieces at most, dealt to eight wavefronts if there are more than 16, the
eight sums, and three more for the scale, the addition and the store.
"""
import numpy as np
import pytest

from oracle import seq as S
from seq_cases import DEV, STEP, K, Rows, close, code, host, rounded

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def chain(ids):
    n = int(np.bincount(ids[ids >= 0]).max()) if (ids >= 0).any() else 1
    pieces = -(-n // 16)
    return (64 + (pieces if pieces <= 16 else -(-pieces // 8)) + 8 + 3) * 2.0 ** -24


def device_ids(ids, wide):
    return torch.from_numpy(np.asarray(ids, np.int64)).to(torch.int64 if wide else torch.int32).to(DEV)


def words(rng, n, vocab, bad=0.05):
    """Unevenly distributed ids, some outside the vocabulary."""
    ids = (np.exp(rng.random(n) * np.log(vocab + 1e-9)) - 1).astype(np.int64).clip(0, vocab - 1)
    ids = rng.permutation(vocab)[ids]
    out = rng.random(n) < bad
    ids[out] = rng.choice([-1, vocab, -7, vocab + 5, 2 ** 31 - 1, -2 ** 31], out.sum())
    return ids


def backward(ids, g, vocab, scale=1.0, gt="f32", dt="f32", pad=0, shift=0, wide=False, accumulate=None):
    n, c = g.shape
    k = K()
    desc = k.embed_desc(n, vocab, c, gtype=code(gt), dtype=code(dt), scale=scale, ids64=wide,
                        accumulate=accumulate is not None, ldw=c + pad, ldg=c + pad)
    G, D = Rows(n, c, gt, pad, shift, g), Rows(vocab, c, dt, pad, shift, accumulate)
    nb = k.op_embed_workspace_bytes(desc)
    ws = torch.full((nb + 64,), 255, dtype=torch.uint8, device=DEV)
    k.op_embed_backward(desc, device_ids(ids, wide), G, D, ws, nb)
    torch.cuda.synchronize()
    assert bool((ws[nb:] == 255).all()), "written past the workspace"
    return D.host()


def check(ids, g, vocab, scale=1.0, gt="f32", dt="f32", accumulate=None, **kw):
    g = rounded(g, gt)
    scale = float(np.float32(scale))
    got = backward(ids, g, vocab, scale, gt, dt, accumulate=accumulate, **kw)
    want, mag = S.embed_backward(np.asarray(ids), g, vocab, scale)
    if accumulate is not None:
        want, mag = want + accumulate, mag + np.abs(accumulate)
    close("dw", got, want, STEP[dt] * np.abs(want) + chain(np.asarray(ids)[np.asarray(ids) < vocab]) * mag)


@pytest.mark.parametrize("tokens,vocab,c", [(1, 1, 1), (1, 50, 7), (7, 3, 9), (64, 5, 8), (65, 2, 520), (1000, 40, 333),
                                            (4099, 97, 64), (5000, 30011, 40), (300, 300000, 16), (20011, 1030, 1030),
                                            (60000, 2, 8), (60000, 1, 24), (64, 1, 8), (65, 1, 8), (129, 2, 600), (640, 10, 9),
                                            (6400, 100, 17)])
def test_gradient_sizes(tokens, vocab, c):
    rng = np.random.default_rng(tokens + vocab)
    check(words(rng, tokens, vocab), rng.standard_normal((tokens, c)), vocab, scale=3.7)


@pytest.mark.parametrize("gt", ["f32", "bf16"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("wide", [False, True])
def test_gradient_types_strides_and_accumulation(gt, dt, wide):
    rng = np.random.default_rng(5)
    n, vocab, c = 777, 210, 75
    ids, g = words(rng, n, vocab), rng.standard_normal((n, c))
    check(ids, g, vocab, gt=gt, dt=dt, pad=3, shift=1, wide=wide)
    check(ids, g, vocab, 0.25, gt=gt, dt=dt, pad=5, shift=3, wide=wide, accumulate=rounded(rng.standard_normal((vocab, c)), dt))


def test_ids_of_64_bits_are_compared_whole():
    ids = np.array([3, 3 + (1 << 32), -(1 << 32) + 3, 1 << 62, 4], np.int64)
    g = np.ones((5, 8))
    got = backward(ids, g, 6, wide=True)
    assert np.array_equal(got[:, 0], [0, 0, 0, 1, 1, 0])


def test_no_valid_id():
    assert not backward(np.full(100, -1), np.ones((100, 8)), 12).any()
    keep = np.arange(96.0).reshape(12, 8)
    assert np.array_equal(backward(np.full(100, 12), np.ones((100, 8)), 12, accumulate=keep), keep)


def test_each_id_is_added_in_the_order_of_its_tokens():
    # sums whose value depends on the order: of few tokens they are a running sum
    rng = np.random.default_rng(3)
    n, vocab = 600, 40
    ids = np.repeat(np.arange(40), 15)[rng.permutation(600)]
    g = (rng.standard_normal((n, 8)) * 10.0 ** rng.integers(-4, 5, (n, 1))).astype(np.float32)
    got = backward(ids, g.astype(np.float64), vocab)
    order, p = np.argsort(ids, kind="stable"), 0
    for v in range(vocab):
        rows = order[p:p + 15]
        s = np.zeros(8, np.float32)
        for i in rows:
            s = s + g[i]
        assert np.array_equal(got[v], s.astype(np.float64))
        p += 15


@pytest.mark.parametrize("wt", ["f32", "bf16"])
@pytest.mark.parametrize("yt", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,vocab,c,pad", [(1, 3, 1, 0), (5, 2, 1000, 0), (1001, 77, 64, 0), (333, 50, 67, 5),
                                                (4, 9, 8, 8)])
def test_lookup(wt, yt, tokens, vocab, c, pad):
    rng = np.random.default_rng(tokens)
    k, ids, w = K(), words(rng, tokens, vocab, 0.1), rounded(rng.standard_normal((vocab, c)), wt)
    W, Y = Rows(vocab, c, wt, pad, 1, w), Rows(tokens, c, yt, pad, 1)
    for wide in (False, True):
        desc = k.embed_desc(tokens, vocab, c, wtype=code(wt), ytype=code(yt), scale=0.3, ids64=wide, ldw=c + pad,
                            ldy=c + pad)
        k.op_embed_forward(desc, device_ids(ids, wide), W, Y)
        want = S.embed(ids, w, float(np.float32(0.3)))
        close("y", Y.host(), want, (STEP[yt] + 2.0 ** -24) * np.abs(want))


def test_captured_and_replayed():
    rng = np.random.default_rng(9)
    n, vocab, c, k = 3000, 500, 128, K()
    desc = k.embed_desc(n, vocab, c, scale=2.0)
    nb = k.op_embed_workspace_bytes(desc)
    ws = torch.empty(nb, dtype=torch.uint8, device=DEV)
    ids, g = device_ids(words(rng, n, vocab), False), torch.randn(n, c, device=DEV).to(torch.bfloat16)
    w = torch.randn(vocab, c, device=DEV).to(torch.bfloat16)
    y, dw = torch.empty(n, c, dtype=torch.bfloat16, device=DEV), torch.empty(vocab, c, device=DEV)
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()

    def run(stream):
        k.op_embed_forward(desc, ids, w, y, stream=stream)
        k.op_embed_backward(desc, ids, g, dw, ws, nb, stream=stream)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        run(torch.cuda.current_stream())
    for seed in range(3):
        ids.copy_(device_ids(words(np.random.default_rng(seed), n, vocab), False))
        graph.replay()
        torch.cuda.synchronize()
        a, b = y.clone(), dw.clone()
        run(None)
        torch.cuda.synchronize()
        assert torch.equal(a, y) and torch.equal(b, dw)
