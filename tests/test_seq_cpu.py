"""RMS norm, embedding and attention without a GPU: the oracle's gradients against
differences, and the calls' refusals (nothing is launched for an invalid one)."""
import ctypes as C

import numpy as np
import pytest

from oracle import seq as S

K = pytest.importorskip("paper_1604_06174_amd.ckpt")
torch = pytest.importorskip("torch")


# ------------------------------------------------------------------ oracle --
def differences(loss, args, which, h=1e-6):
    base = args[which]
    out = np.zeros(base.size)
    for e in range(base.size):
        vals = []
        for s in (h, -h):
            v = base.copy()
            v.reshape(-1)[e] += s
            vals.append(loss(*[v if k == which else a for k, a in enumerate(args)]))
        out[e] = (vals[0] - vals[1]) / (2 * h)
    return out.reshape(base.shape)


# truncation h^2 |f'''| / 6 and rounding 2^-53 |f| / h, both below 1e-8 here (|f'''| < 1e3, |f| < 1e2)
ATOL = 1e-7


@pytest.mark.parametrize("res", [False, True])
def test_rms_gradients_against_differences(res):
    rng = np.random.default_rng(1)
    h, g, gh = rng.standard_normal((3, 4, 6))
    w = 1 + 0.3 * rng.standard_normal(6)

    def loss(h, w):
        return (g * S.rms_apply(h, S.rms_stat(h, 1e-2), w)).sum() + ((gh * h).sum() if res else 0)
    d, dw, _, _ = S.rms_backward(g, gh if res else None, h, S.rms_stat(h, 1e-2), w)
    np.testing.assert_allclose(d, differences(loss, [h, w], 0), atol=ATOL)
    np.testing.assert_allclose(dw, differences(loss, [h, w], 1), atol=ATOL)


def test_embedding_gradient_against_differences():
    rng = np.random.default_rng(2)
    ids = np.array([3, 0, 3, -1, 5, 4, 3])
    w, g = rng.standard_normal((5, 4)), rng.standard_normal((7, 4))
    d, _ = S.embed_backward(ids, g, 5, 1.7)
    np.testing.assert_allclose(d, differences(lambda w: (g * S.embed(ids, w, 1.7)).sum(), [w], 0), atol=ATOL)


@pytest.mark.parametrize("causal", [True, False])
def test_attention_gradients_against_differences(causal):
    rng = np.random.default_rng(3)
    q, k, v = (rng.standard_normal((t, h, 6)) for t, h in ((9, 4), (11, 2), (11, 2)))
    g, lens = rng.standard_normal(q.shape), (np.array([0, 3, 7, 9]), np.array([0, 2, 9, 11]))

    def loss(q, k, v):
        return (g * S.attention(q, k, v, *lens, causal, 0.4)[0]).sum()
    o, lse, _, _ = S.attention(q, k, v, *lens, causal, 0.4)
    got, _ = S.attention_backward(g, q, k, v, o, lse, *lens, causal, 0.4)
    for n in range(3):
        np.testing.assert_allclose(got[n], differences(loss, [q, k, v], n), atol=ATOL)


def test_attention_rows_that_see_nothing():
    rng = np.random.default_rng(4)
    q, k, v = rng.standard_normal((5, 1, 4)), rng.standard_normal((2, 1, 4)), rng.standard_normal((2, 1, 4))
    o, lse, _, _ = S.attention(q, k, v, np.array([0, 5]), np.array([0, 2]), True, 1.0)
    assert not o[:3].any() and np.isneginf(lse[0, :3]).all() and np.isfinite(lse[0, 3:]).all()


# ---------------------------------------------------------------- refusals --
A = 0x1000  # an aligned address that nothing reads


def refused(code, call, *args, **kw):
    with pytest.raises(K.CkptError) as e:
        call(*args, **kw)
    assert e.value.code == code, e.value


def rms_all(code, **kw):
    d = K.rms_desc(**{**dict(rows=4, c=16), **kw})
    ys = A if d.ytype == K.TYPE_E4M3 else None
    refused(code, K.op_rms_forward, d, A, A, A, A, res=A, h=A, ys=ys)
    refused(code, K.op_rms_apply, d, A, A, A, A, ys=ys)
    refused(code, K.op_rms_workspace_bytes, d)
    refused(code, K.op_rms_backward, d, A, A, A, A, A, A, A, 1 << 30)


@pytest.mark.parametrize("kw", [dict(rows=0), dict(rows=-1), dict(c=0), dict(xtype=2), dict(htype=3), dict(ytype=7),
                                dict(gtype=2), dict(dtype=-1), dict(eps=0.0), dict(eps=float("nan")),
                                dict(eps=float("inf")), dict(ldx=15), dict(ldh=15), dict(ldy=15), dict(ldg=-16),
                                dict(ldd=15), dict(qgroup=8), dict(ytype=K.TYPE_E4M3, qgroup=4),
                                dict(ytype=K.TYPE_E4M3, qgroup=24), dict(ytype=K.TYPE_E4M3, qgroup=1024)])
def test_rms_invalid(kw):
    rms_all(K.E_INVALID, **kw)


@pytest.mark.parametrize("kw", [dict(rows=1 << 31), dict(c=16385), dict(ldx=1 << 60)])
def test_rms_unsupported(kw):
    rms_all(K.E_UNSUPPORTED, **kw)


def test_rms_arguments():
    d = K.rms_desc(4, 16)
    f, b = K.op_rms_forward, K.op_rms_backward
    for k in range(4):
        a = [A] * 4
        a[k] = None
        refused(K.E_INVALID, f, d, *a, res=A, h=A)
    refused(K.E_INVALID, f, d, A, A, A, A, res=A)          # h missing
    refused(K.E_INVALID, f, d, A, A, A, A, h=A)            # res missing
    refused(K.E_INVALID, f, d, A, A, A, A, ys=A)           # scales of a 16-bit y
    refused(K.E_INVALID, f, d, A + 1, A, A, A)             # misaligned
    refused(K.E_INVALID, f, d, A, A + 2, A, A)
    refused(K.E_INVALID, f, K.rms_desc(4, 16, htype=K.TYPE_F32), A, A, A, A)  # x alone, of another type
    refused(K.E_INVALID, f, K.rms_desc(4, 16, ytype=K.TYPE_E4M3, gtype=K.TYPE_BF16), A, A, A, A)  # scales missing
    for k in range(6):
        a = [A] * 6
        a[k] = None
        refused(K.E_INVALID, b, d, *a, A, 1 << 20)
    nb = K.op_rms_workspace_bytes(d)
    refused(K.E_INVALID, b, d, A, A, A, A, A, A, None, nb)
    refused(K.E_INVALID, b, d, A, A, A, A, A, A, A + 8, nb)
    refused(K.E_WORKSPACE, b, d, A, A, A, A, A, A, A, nb - 1)
    refused(K.E_INVALID, b, d, A, A, A, A, A, A, A, -1)
    refused(K.E_INVALID, f, d, torch.zeros(4, 16), A, A, A)  # fp32, described as bf16
    refused(K.E_INVALID, f, d, A, torch.zeros(16, dtype=torch.bfloat16), A, A)
    refused(K.E_INVALID, K.rms_desc, 4, -(1 << 33))
    refused(K.E_UNSUPPORTED, K.rms_desc, 4, 1 << 33)


def embed_all(code, **kw):
    d = K.embed_desc(**{**dict(tokens=5, vocab=9, c=16), **kw})
    refused(code, K.op_embed_forward, d, A, A, A)
    refused(code, K.op_embed_workspace_bytes, d)
    refused(code, K.op_embed_backward, d, A, A, A, A, 1 << 30)


@pytest.mark.parametrize("kw", [dict(tokens=0), dict(vocab=0), dict(c=0), dict(vocab=-4), dict(wtype=2), dict(ytype=2),
                                dict(gtype=3), dict(dtype=2), dict(scale=float("nan")), dict(scale=float("inf")),
                                dict(ldw=15), dict(ldy=15), dict(ldg=15)])
def test_embedding_invalid(kw):
    embed_all(K.E_INVALID, **kw)


@pytest.mark.parametrize("kw", [dict(tokens=1 << 31), dict(vocab=1 << 31), dict(c=(1 << 20) + 1), dict(ldw=1 << 60),
                                dict(tokens=1 << 25, c=1 << 16), dict(tokens=(1 << 30) + 1), dict(tokens=1 << 20, c=1 << 16)])
def test_embedding_unsupported(kw):
    embed_all(K.E_UNSUPPORTED, **kw)


def test_embedding_arguments():
    d = K.embed_desc(5, 9, 16)
    for k in range(3):
        a = [A] * 3
        a[k] = None
        refused(K.E_INVALID, K.op_embed_forward, d, *a)
        refused(K.E_INVALID, K.op_embed_backward, d, *a, A, 1 << 20)
        a[k] = A + 1
        refused(K.E_INVALID, K.op_embed_forward, d, *a)
    refused(K.E_INVALID, K.op_embed_forward, K.embed_desc(5, 9, 16, ids64=True), A + 4, A, A)
    nb = K.op_embed_workspace_bytes(d)
    refused(K.E_WORKSPACE, K.op_embed_backward, d, A, A, A, A, nb - 1)
    refused(K.E_INVALID, K.op_embed_backward, d, A, A, A, None, nb)
    refused(K.E_INVALID, K.op_embed_backward, d, A, A, A, A + 4, nb)
    refused(K.E_INVALID, K.op_embed_forward, d, torch.zeros(5, dtype=torch.int64), A, A)
    refused(K.E_INVALID, K.op_embed_forward, d, torch.zeros(10, dtype=torch.int32)[::2], A, A)
    refused(K.E_INVALID, K.op_embed_forward, d, torch.zeros(5), A, A)


def attn_all(code, **kw):
    d = K.attn_desc(**{**dict(tq=10, tk=12, seqs=2, heads=4, kv_heads=2, dim=16), **kw})
    for b in (False, True):
        refused(code, K.op_attn_workspace_bytes, d, b)
    refused(code, K.op_attn_forward, d, A, A, A, A, A, A, A, A, 1 << 30)
    refused(code, K.op_attn_backward, d, A, A, A, A, A, A, A, A, A, A, A, A, 1 << 30)


@pytest.mark.parametrize("kw", [dict(tq=-1), dict(tk=-1), dict(seqs=0), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3),
                                dict(dim=0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
                                dict(ldq=8), dict(hsk=8), dict(ldv=-64), dict(hso=8)])
def test_attention_invalid(kw):
    attn_all(K.E_INVALID, **kw)


@pytest.mark.parametrize("kw", [dict(dim=12), dict(dim=136), dict(tq=1 << 31), dict(tk=1 << 31), dict(seqs=1 << 20),
                                dict(heads=8192), dict(ldq=66), dict(hsv=20), dict(ldk=1 << 60),
                                dict(tq=1 << 30, heads=64), dict(tq=(1 << 30) + 1, heads=1, kv_heads=1),
                                dict(tk=1 << 30, seqs=1), dict(seqs=1 << 19, heads=32, kv_heads=32)])
def test_attention_unsupported(kw):
    attn_all(K.E_UNSUPPORTED, **kw)


def test_attention_arguments():
    d = K.attn_desc(10, 12, 2, 4, 2, 16)
    for k in range(7):
        a = [A] * 7
        a[k] = None
        refused(K.E_INVALID, K.op_attn_forward, d, *a)
        a[k] = A + 2
        refused(K.E_INVALID, K.op_attn_forward, d, *a)
    for k in range(11):
        a = [A] * 11
        a[k] = None
        refused(K.E_INVALID, K.op_attn_backward, d, *a, A, 1 << 20)
    nb = K.op_attn_workspace_bytes(d, True)
    refused(K.E_WORKSPACE, K.op_attn_backward, d, *[A] * 11, A, nb - 1)
    refused(K.E_INVALID, K.op_attn_backward, d, *[A] * 11, None, nb)
    split = K.attn_desc(2, 100000, 2, 4, 2, 16)
    nb = K.op_attn_workspace_bytes(split, False)
    assert nb > 0
    refused(K.E_WORKSPACE, K.op_attn_forward, split, *[A] * 7, A, nb - 1)
    refused(K.E_INVALID, K.op_attn_forward, split, *[A] * 7, None, nb)
    refused(K.E_INVALID, K.op_attn_forward, d, torch.zeros(10, 64), *[A] * 6)       # fp32
    refused(K.E_INVALID, K.op_attn_forward, d, A, A, A, torch.zeros(3, dtype=torch.int64), A, A, A)
    refused(K.E_INVALID, K.attn_desc, 10, 12, 2, 4, 2, -(1 << 40))


def test_tensors_of_another_device():
    """Host memory would be a fault on the GPU."""
    z = torch.zeros(16 * 16, dtype=torch.bfloat16)
    f, i = torch.zeros(16), torch.zeros(16, dtype=torch.int32)
    for bad in ((z, A, A, A), (A, f, A, A), (A, A, z, A), (A, A, A, f)):
        refused(K.E_INVALID, K.op_rms_forward, K.rms_desc(4, 16), *bad)
    for bad in ((i, A, A), (A, z, A), (A, A, z)):
        refused(K.E_INVALID, K.op_embed_forward, K.embed_desc(5, 9, 16), *bad)
    d = K.attn_desc(10, 12, 2, 4, 2, 16)
    for bad in ((z, A, A, A, A, A, A), (A, A, A, i, A, A, A), (A, A, A, A, A, A, f), (A, A, A, A, A, A, A, z)):
        refused(K.E_INVALID, K.op_attn_forward, d, *bad)


def test_descriptors_match_the_header():
    """Sizes of the structures as the library's compiler lays them out: a field shifted by
    a missing one would be refused or read as another."""
    assert C.sizeof(K.RmsDesc) == 8 + 7 * 4 + 4 + 5 * 8
    assert C.sizeof(K.EmbedDesc) == 16 + 7 * 4 + 4 + 24
    assert C.sizeof(K.AttnDesc) == 16 + 5 * 4 + 4 + 64
