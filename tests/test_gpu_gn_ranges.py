"""Group norm through every kernel it is compiled to, and through offsets past 32
bits (the checks and bars are those of test_gpu_gn.py)."""
import numpy as np
import pytest

import gn_cases as R
import test_gpu_gn as B
from oracle import norm as N
from test_gpu_gn import DEV, Case, _K, f32, host, torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("shape", list(R.RANGES) + list(R.FORWARD))
def test_forward(shape, x):
    table = {**R.RANGES, **R.FORWARD}
    k = list(table).index(shape)
    for act, p in R.combos(k):
        print(f"[gn ranges forward] {shape} {x} {act} {p}", flush=True)
        Case(*table[shape], act=act, x=x, p=p, seed=100 + k).check_forward()


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("shape", list(R.RANGES))
def test_backward(shape, x):
    k = list(R.RANGES).index(shape)
    for act, p in R.combos(k):
        for g, d in R.GRADIENTS[x]:
            print(f"[gn ranges backward] {shape} {x} {g} {d} {act} {p}", flush=True)
            Case(*R.RANGES[shape], act=act, x=x, g=g, d=d, p=p, seed=100 + k).check_backward()


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("shape", list(R.MANY))
def test_many_samples(shape, x):
    k = list(R.MANY).index(shape)
    act, p = R.COMBOS[k % 4]
    for i, (g, d) in enumerate(R.GRADIENTS[x]):
        print(f"[gn many] {shape} {x} {g} {d} {act} {p}", flush=True)
        c = Case(*R.MANY[shape], act=act, x=x, g=g, d=d, p=p, pad=8 * (k % 2), seed=200 + k)
        if i == 0:
            c.check_forward()
        c.check_backward()


# teams that the shapes of these checks in test_gpu_gn.py leave out
TEAMS = {
    "wave_two_vectors": (2048, 16, 64, 8),
    "wave_fours": (2048, 16, 64, 16),
    "wave_padded": (1039, 9, 40, 4),
    "wave_packed": (4100, 1, 64, 4),
    "wave_packed_fours": (2101, 1, 32, 8),
    "loop_rows": (1203, 1, 2048, 2),
    "loop_rows_halves": (2300, 1, 1000, 2),
    "loop_rows_s": (1203, 2, 1030, 2),
    "loop_four_pixels": (1301, 4, 1024, 2),
    "resident_sixteen_vectors": (66, 130, 264, 8),
}


@pytest.mark.parametrize("shape", list(TEAMS))
def test_special_values_stay_in_their_group(shape, monkeypatch):
    monkeypatch.setitem(B.SHAPES, shape, TEAMS[shape])
    B.test_special_values_stay_in_their_group(shape)


@pytest.mark.parametrize("shape", list(TEAMS))
def test_same_bits_and_in_place(shape, monkeypatch):
    monkeypatch.setitem(B.SHAPES, shape, TEAMS[shape])
    B.test_same_bits_and_in_place(shape)


def _wide(rows, ld, dtype):
    """A tensor of `rows` rows `ld` elements apart, and its rows alone."""
    t = torch.empty((rows - 1) * ld + 64, dtype=dtype, device=DEV)
    return t, t.as_strided((rows, 64), (ld, 1))


@pytest.mark.parametrize("n,hw,rows", [(1, 3, 3), (3, 1, 3), (1, 4500, 4500), (2, 70, 140)])
def test_offsets_past_31_bits(n, hw, rows):
    """Pixel strides with which x, g, y and d pass 2^31 elements, forward, re-run and
    backward, resident, split and by rows: the packed tensors' results."""
    K = _K()
    ld = (1 << 31) // (rows - 1) + 27
    print(f"[gn far offsets] {n} x {hw}, stride {ld}", flush=True)
    assert (rows - 1) * ld > 1 << 31
    torch.manual_seed(9)
    ga, be = 1 + 0.1 * torch.randn(64, device=DEV), 0.1 * torch.randn(64, device=DEV)
    v, w = (torch.randn(rows, 64, device=DEV).to(torch.bfloat16) for _ in range(2))
    drop = K.dropout(torch.tensor([3, 4], dtype=torch.int64, device=DEV), 0.3, 7)
    wides = [_wide(rows, ld, torch.bfloat16) for _ in range(2)]
    (wx, mx), (wo, mo) = wides
    outs = []
    for far in (False, True):
        l = ld if far else 64
        d = K.gn_desc(n, hw, 64, 8, act=K.ACT_SILU, ldx=l, ldy=l, ldg=l, ldd=l)
        nb = max(16, K.op_gn_workspace_bytes(d, False), K.op_gn_workspace_bytes(d, True))
        ws = torch.empty(nb, dtype=torch.uint8, device=DEV)
        st, dg, db = torch.empty(2 * n * 8, device=DEV), torch.empty(64, device=DEV), torch.empty(64, device=DEV)
        out = torch.empty_like(v)
        x, o, oo = (wx, wo, mo) if far else (v, out, out)
        mx.copy_(v)
        got = [st, dg, db]
        K.op_gn_forward(d, x, ga, be, o, st, ws, nb, drop=drop)
        got.append(oo.clone())
        oo.fill_(0)
        K.op_gn_apply(d, x, st, ga, be, o, drop=drop)
        got.append(oo.clone())
        # the gradient in the output's place: d may be written over it
        oo.copy_(w)
        K.op_gn_backward(d, o, x, st, ga, be, o, dg, db, ws, nb, drop=drop)
        got.append(oo.clone())
        torch.cuda.synchronize()
        outs.append(got)
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert torch.equal(outs[0][3], outs[0][4])


@pytest.mark.parametrize("hw,c", [((1 << 26) + 3, 72), ((1 << 29) + 3, 9)])
def test_elements_past_32_bits(hw, c):
    """Element numbers past 2^32: the mask of the last pixels, in the forward and in
    the backward (whose shift gradient counts the kept elements of a channel)."""
    K = _K()
    print(f"[gn far elements] {hw} x {c}", flush=True)
    assert hw * c > 1 << 32
    seed, step, site = 11, 12, 13
    drop = K.dropout(torch.tensor([seed, step], dtype=torch.int64, device=DEV), 0.5, site)
    x = torch.zeros(hw, c, dtype=torch.bfloat16, device=DEV)
    d = K.gn_desc(1, hw, c, 1, ldg=c)
    nb = max(16, K.op_gn_workspace_bytes(d, False), K.op_gn_workspace_bytes(d, True))
    ws = torch.empty(nb, dtype=torch.uint8, device=DEV)
    st, dg, db = torch.empty(2, device=DEV), torch.empty(c, device=DEV), torch.empty(c, device=DEV)
    ga, be = torch.ones(c, device=DEV), torch.ones(c, device=DEV)
    # a constant sample: every output is the shift, 1, before dropout
    tail = 999
    want = N.dropout_factor(tail * c, 0.5, seed, step, site, (hw - tail) * c).reshape(tail, c)
    K.op_gn_forward(d, x, ga, be, x, st, ws, nb, drop=drop)
    assert np.array_equal(host(x[-tail:].float()), want)
    x.zero_()
    K.op_gn_apply(d, x, st, ga, be, x, drop=drop)
    assert np.array_equal(host(x[-tail:].float()), want)
    # a gradient of ones on the last pixels alone
    g = x
    g.zero_()
    g[-tail:] = 1
    y = torch.zeros(hw, c, dtype=torch.bfloat16, device=DEV)
    K.op_gn_backward(d, g, y, st, ga, be, g, dg, db, ws, nb, drop=drop)
    # whole numbers below 2^24
    assert np.array_equal(host(db), want.sum(0))
