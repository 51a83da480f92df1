"""The token models' operators together, as a block of such a model uses them: embedding, norm,
product, attention over packed sequences, product, residual and norm (8-bit output), and the
whole backward, of a segment that keeps the stream's rows and statistics alone and runs the rest
again.  Every stage is held to the float64 oracle on the values that reached it; the run is on a stream of its
own, then captured and replayed with other tokens."""
import numpy as np
import pytest

from oracle import seq as S
from seq_cases import DEV, K, close, f32, host, rounded

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U16, U24 = S.U16, S.U24
EPS = 1e-5


class Block:
    def __init__(self, vocab, c, heads, kv, dim, lens, seed=3):
        rng = np.random.default_rng(seed)
        self.k, self.vocab, self.c, self.heads, self.kv, self.dim = K(), vocab, c, heads, kv, dim
        self.n, self.off = sum(lens), np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        self.wide = (heads + 2 * kv) * dim  # a row of q, k and v side by side
        k, n = self.k, self.n
        bf = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=DEV)
        f = lambda *s: torch.empty(*s, device=DEV)
        self.v = dict(table=rounded(rng.standard_normal((vocab, c)), "bf16"),
                      w0=rounded(rng.uniform(0.5, 1.5, c), "f32"), w1=rounded(rng.uniform(0.5, 1.5, c), "f32"),
                      wqkv=rounded(rng.standard_normal((self.wide, c)) * c ** -0.5, "bf16"),
                      wo=rounded(rng.standard_normal((c, heads * dim)) * (heads * dim) ** -0.5, "bf16"),
                      g1=rounded(rng.standard_normal((n, c)), "bf16"), gh=rounded(rng.standard_normal((n, c)), "bf16"))
        self.d = {m: f32(a) if m in ("w0", "w1") else f32(a).to(torch.bfloat16) for m, a in self.v.items()}
        d = self.d
        d.update(ids=torch.empty(n, dtype=torch.int32, device=DEV), off=torch.from_numpy(self.off).to(DEV),
                 h0=bf(n, c), st0=f(n), y0=bf(n, c), qkv32=f(n, self.wide), qkv=bf(n, self.wide), o=bf(n, heads * dim),
                 lse=f(heads, n), x1=f(n, c), h1=bf(n, c), st1=f(n), y1=bf(n, c).to(torch.float8_e4m3fn), ys1=f(n, 1),
                 d1=bf(n, c), dw1=f(c), go32=f(n, heads * dim), go=bf(n, heads * dim), dqkv=bf(n, self.wide),
                 gy32=f(n, c), gy=bf(n, c), d0=bf(n, c), dw0=f(c), dtable=f(vocab, c), dwqkv=f(self.wide, c))
        self.emb = k.embed_desc(n, vocab, c)
        self.rms0 = k.rms_desc(n, c, eps=EPS)
        self.rms1 = k.rms_desc(n, c, eps=EPS, xtype=k.TYPE_F32, htype=k.TYPE_BF16, ytype=k.TYPE_E4M3)
        self.att = k.attn_desc(n, n, len(lens), heads, kv, dim, ldq=self.wide, ldk=self.wide, ldv=self.wide)
        sizes = dict(emb=k.op_embed_workspace_bytes(self.emb), rms=k.op_rms_workspace_bytes(self.rms0),
                     fwd=k.op_attn_workspace_bytes(self.att, False), bwd=k.op_attn_workspace_bytes(self.att, True))
        self.ws = {m: (torch.empty(max(s, 16), dtype=torch.uint8, device=DEV), s) for m, s in sizes.items()}

    def tokens(self, seed):
        self.ids = np.random.default_rng(seed).integers(-2, self.vocab + 2, self.n)
        self.d["ids"].copy_(torch.from_numpy(self.ids.astype(np.int32)))

    def qkv_of(self, m):
        a, b = self.heads * self.dim, (self.heads + self.kv) * self.dim
        return m[:, :a], m[:, a:b], m[:, b:]

    def mid(self, s):
        """from y0 on to the block's product"""
        k, d, n = self.k, self.d, self.n
        k.op_gemm_bf16(n, self.wide, self.c, d["y0"], self.c, True, d["wqkv"], self.c, True, d["qkv32"], self.wide, stream=s)
        d["qkv"].copy_(d["qkv32"])
        k.op_attn_forward(self.att, *map(torch.Tensor.data_ptr, self.qkv_of(d["qkv"])), d["off"], d["off"], d["o"], d["lse"],
                          *self.ws["fwd"], stream=s)

    def run(self, s, rerun):
        k, d, n, c, e = self.k, self.d, self.n, self.c, self.heads * self.dim
        k.op_embed_forward(self.emb, d["ids"], d["table"], d["h0"], stream=s)
        k.op_rms_forward(self.rms0, d["h0"], d["w0"], d["y0"], d["st0"], stream=s)
        self.mid(s)
        k.op_gemm_bf16(n, c, e, d["o"], e, True, d["wo"], e, True, d["x1"], c, stream=s)
        k.op_rms_forward(self.rms1, d["x1"], d["w1"], d["y1"], d["st1"], d["h0"], d["h1"], d["ys1"], stream=s)
        if rerun:
            for m in ("y0", "qkv32", "qkv", "o", "lse"):
                d[m].zero_()
            k.op_rms_apply(self.rms0, d["h0"], d["st0"], d["w0"], d["y0"], stream=s)
            self.mid(s)
        k.op_rms_backward(self.rms1, d["g1"], d["h1"], d["st1"], d["w1"], d["d1"], d["dw1"], *self.ws["rms"], gh=d["gh"],
                          stream=s)
        k.op_gemm_bf16(n, e, c, d["d1"], c, True, d["wo"], e, False, d["go32"], e, stream=s)
        d["go"].copy_(d["go32"])
        k.op_attn_backward(self.att, d["go"], *map(torch.Tensor.data_ptr, self.qkv_of(d["qkv"])), d["o"], d["lse"], d["off"],
                           d["off"], *map(torch.Tensor.data_ptr, self.qkv_of(d["dqkv"])), *self.ws["bwd"], stream=s)
        k.op_gemm_bf16(self.wide, c, n, d["dqkv"], self.wide, False, d["y0"], c, False, d["dwqkv"], c, stream=s)
        k.op_gemm_bf16(n, c, self.wide, d["dqkv"], self.wide, True, d["wqkv"], c, False, d["gy32"], c, stream=s)
        d["gy"].copy_(d["gy32"])
        k.op_rms_backward(self.rms0, d["gy"], d["h0"], d["st0"], d["w0"], d["d0"], d["dw0"], *self.ws["rms"], gh=d["d1"],
                          stream=s)
        k.op_embed_backward(self.emb, d["ids"], d["d0"], d["dtable"], *self.ws["emb"], stream=s)

    OUTS = ("y1", "ys1", "h1", "st1", "dw1", "dqkv", "dwqkv", "dw0", "dtable")

    def outs(self):
        torch.cuda.synchronize()
        return {m: self.d[m].view(torch.uint8).clone() for m in self.OUTS}

    def check(self):
        """Each stage on the values that reached it."""
        c, n, heads, kv, dim = self.c, self.n, self.heads, self.kv, self.dim
        D = {m: (host(t.float()) if t.is_floating_point() else None) for m, t in self.d.items()}
        v = self.v
        close("h0", D["h0"], S.embed(self.ids, v["table"], 1.0), 1e-30)

        def product(name, a, b):
            close(name, D[name], a @ b, (a.shape[1] + 2) * U24 * (np.abs(a) @ np.abs(b)) + 1e-30)

        def norm(h, st, w, name):  # a sum of c squares, its root and the two products
            want = S.rms_stat(h, EPS)
            close(st, D[st], want, (c + 8) * U24 * want)
            return S.rms_apply(h, want, v[w])

        u = norm(D["h0"], "st0", "w0", "y0")
        close("y0", D["y0"], u, (U16 + (c + 16) * U24) * np.abs(u) + 1e-30)
        product("qkv32", D["y0"], v["wqkv"].T)
        q, k, val = (m.reshape(n, -1, dim) for m in self.qkv_of(D["qkv"]))
        o, lse, eo, el = S.attention(q, k, val, self.off, self.off, True, dim ** -0.5)
        close("o", D["o"].reshape(n, heads, dim), o, eo)
        close("lse", D["lse"], lse, el)
        product("x1", D["o"], v["wo"].T)
        sum1 = D["x1"] + D["h0"]
        close("h1", D["h1"], sum1, (U16 + 2 * U24) * np.abs(sum1) + 1e-30)
        u = norm(D["h1"], "st1", "w1", "y1")
        top = S.group_scales(u, 0)
        close("ys1", D["ys1"], top, (c + 32) * U24 * top)
        # half a step of e4m3: 2^-4 of the value, 2^-10 of the scale below its normal values
        close("y1", D["y1"] * D["ys1"], u, (2.0 ** -4 + (2 * c + 64) * U24) * np.abs(u) + 2.0 ** -10 * 1.001 * top)

        def grad(g, gh, h, st, w, dname, dwname):
            want, dw, mag, dwmag = S.rms_backward(g, gh, h, D[st], v[w])
            close(dname, D[dname], want, U16 * np.abs(want) + (c + 32) * U24 * mag + 1e-30)
            close(dwname, D[dwname], dw, (n + 32) * U24 * dwmag + 1e-30)

        grad(v["g1"], v["gh"], D["h1"], "st1", "w1", "d1", "dw1")
        product("go32", D["d1"], v["wo"])
        want, err = S.attention_backward(D["go"].reshape(n, heads, dim), q, k, val, D["o"].reshape(n, heads, dim), D["lse"],
                                         self.off, self.off, True, dim ** -0.5)
        for name, got, a, b in zip(("dq", "dk", "dv"), self.qkv_of(D["dqkv"]), want, err):
            close(name, got.reshape(a.shape), a, b)
        product("dwqkv", D["dqkv"].T, D["y0"])
        product("gy32", D["dqkv"], v["wqkv"])
        grad(D["gy"], D["d1"], D["h0"], "st0", "w0", "d0", "dw0")
        want, mag = S.embed_backward(self.ids, D["d0"], self.vocab, 1.0)
        close("dtable", D["dtable"], want, (n + 32) * U24 * mag + 1e-30)


SHAPES = [dict(vocab=61, c=64, heads=4, kv=2, dim=16, lens=(1, 37, 0, 130, 64)),
          dict(vocab=500, c=256, heads=4, kv=1, dim=64, lens=(200, 7, 300))]


@pytest.mark.parametrize("shape", SHAPES, ids=["small", "wide"])
def test_block(shape):
    b = Block(**shape)
    b.tokens(1)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        b.run(stream, rerun=False)
    first = b.outs()
    b.check()
    with torch.cuda.stream(stream):
        b.run(stream, rerun=True)
    again = b.outs()
    for m in first:
        assert torch.equal(first[m], again[m]), m


def test_captured_block():
    """Replays with other tokens, with eager work of a second block on another stream between them."""
    b, other = Block(**SHAPES[0]), Block(**SHAPES[0], seed=4)
    b.tokens(1)
    other.tokens(9)
    torch.cuda.synchronize()
    stream, side = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(stream):
        b.run(stream, rerun=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        b.run(stream, rerun=True)
    want = None
    for seed in (5, 6, 7):
        b.tokens(seed)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            other.run(side, rerun=False)
        b.outs()
        b.check()
        got = other.outs()
        for m in want or ():
            assert torch.equal(want[m], got[m]), m
        want = got
