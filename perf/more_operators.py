"""The operators of a token model's units whose speed matters, case by case.

Kinds:
  rms_fwd    root-mean-square norm, of a sum with the residual stream or of x
             alone, out in 32, 16 or 8 bits (`op_rms_forward`)
  rms_apply  the same with the statistics known: the re-run of a checkpointed
             unit (`op_rms_apply`)
  rms_bwd    its backward: gradient of the sum, of the weight (`op_rms_backward`)
  emb_fwd    embedding lookup with a scale (`op_embed_forward`)
  emb_bwd    the table's gradient, rows added up by sorted tokens (`op_embed_backward`)
  att_fwd    attention of packed sequences, grouped heads (`op_attn_forward`)
  att_bwd    its backward (`op_attn_backward`)

A sequence of an attention case has lq queries, which are the last of its lk
keys' positions: lk = lq where a whole sequence attends to itself, more where
tokens go on from earlier ones.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "f8": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "f32": 4, "f8": 1}
TINY = 1e-30  # least amplitude that a scale of 8-bit values stands for


def listed():
    return [
        # the hidden states of eight sequences' current tokens: generation, where latency counts
        dict(name="rms_fwd_tokens", kind="rms_fwd", rows=8, c=1024, x="bf16", h="bf16", y="bf16", res=1, group=0,
             pad=0),
        # a unit's entry at training size: branch added to the stream, normalised, out in 8 bits for the next product
        dict(name="rms_fwd_res_f8", kind="rms_fwd", rows=16384, c=4096, x="bf16", h="bf16", y="f8", res=1, group=128,
             pad=0),
        # the re-run of a checkpointed segment with a float32 stream, odd width in a wider tensor
        dict(name="rms_apply_odd", kind="rms_apply", rows=5003, c=1001, x="bf16", h="f32", y="bf16", res=1, group=0,
             pad=24),
        # backward at training size, the stream's gradient joined
        dict(name="rms_bwd", kind="rms_bwd", rows=16384, c=2048, x="bf16", h="bf16", g="bf16", d="bf16", res=1, pad=0),
        # a batch's tokens looked up
        dict(name="emb_fwd", kind="emb_fwd", tokens=32768, vocab=32000, c=1024, w="bf16", y="bf16", pad=0),
        # the table's gradient of the same batch, tokens as unevenly distributed as words are
        dict(name="emb_bwd_words", kind="emb_bwd", tokens=65536, vocab=50000, c=1024, g="bf16", d="f32", pad=0),
        # characters of a small corpus, a float32 net of odd width: few rows, each with many tokens
        dict(name="emb_bwd_chars", kind="emb_bwd", tokens=4099, vocab=97, c=333, g="f32", d="f32", pad=0),
        # one token for each of 16 sequences against what came before
        dict(name="att_fwd_tokens", kind="att_fwd", seqs=16, q=16, past=8192, heads=32, kv_heads=8, dim=128, causal=1,
             split=1, fused=0),
        # training: sequences of different lengths in one packed batch
        dict(name="att_fwd_packed", kind="att_fwd", seqs=7, q=16384, past=0, heads=16, kv_heads=4, dim=128, causal=1,
             split=2, fused=1),
        # short sequences that attend both ways, odd lengths, narrow heads, each with its own keys
        dict(name="att_fwd_short", kind="att_fwd", seqs=61, q=5003, past=0, heads=12, kv_heads=12, dim=40, causal=0,
             split=3, fused=0),
        # training's backward of one long sequence
        dict(name="att_bwd_long", kind="att_bwd", seqs=1, q=8192, past=0, heads=16, kv_heads=4, dim=128, causal=1,
             split=4, fused=0),
        # and of a packed batch of narrower heads
        dict(name="att_bwd_packed", kind="att_bwd", seqs=19, q=8201, past=0, heads=16, kv_heads=16, dim=64, causal=1,
             split=5, fused=1),
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], uniform in its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


LIMIT = 16384 * 4096     # elements of a drawn norm
PAIRS = 16 * 8192 ** 2 // 2 * 128  # (query, key, head) pairs of a drawn attention, times the head's width


def draw(rng):
    kind = rng.choice(["rms_fwd", "rms_fwd", "rms_apply", "rms_bwd", "emb_fwd", "emb_bwd", "emb_bwd", "att_fwd",
                       "att_fwd", "att_fwd", "att_bwd", "att_bwd"])
    if kind.startswith("rms"):
        c = rng.choice([8 * _log(rng, 8, 1024), 128 * _log(rng, 1, 64), _log(rng, 1, 9000)])
        h = rng.choice(["bf16", "bf16", "f32"])
        res = rng.randint(0, 1)
        x = rng.choice(["bf16", "f32"]) if res else h
        case = dict(kind=kind, rows=_log(rng, 1, max(1, LIMIT // c // (2 if "f32" in (x, h) else 1))), c=c, x=x, h=h)
        if kind == "rms_bwd":
            case.update(g=rng.choice(["bf16", "f32"]), d=h)
        else:
            case.update(y=rng.choice(["bf16", "bf16", "f32", "f8", "f8"]))
            case.update(group=rng.choice([0, 32, 128, 512]) if case["y"] == "f8" else 0)
        case.update(res=res, pad=rng.choice([0, 0, 0, 8, 5]))
        return case
    if kind.startswith("emb"):
        c = rng.choice([8 * _log(rng, 8, 512), 64 * _log(rng, 1, 64), _log(rng, 1, 3000)])
        a, b = rng.choice(["bf16", "f32"]), rng.choice(["bf16", "f32"])
        case = dict(kind=kind, tokens=_log(rng, 1, min(65536, LIMIT // 2 // c)),
                    vocab=_log(rng, 2, min(131072, LIMIT // c)), c=c)
        case.update(dict(w=a, y=b) if kind == "emb_fwd" else dict(g=a, d=b))
        case.update(pad=rng.choice([0, 0, 0, 8, 5]))
        return case
    kv = rng.choice([1, 2, 4, 8, 12, 16])
    dim = rng.choice([128, 128, 64, 64, 8 * rng.randint(1, 16)])
    case = dict(kind=kind, seqs=_log(rng, 1, 64), q=0, past=0, heads=kv * rng.choice([1, 1, 2, 3, 4, 8]), kv_heads=kv,
                dim=dim, causal=rng.choice([1, 1, 1, 0]), split=rng.randint(1, 1 << 20), fused=rng.randint(0, 1))
    if kind == "att_fwd" and rng.random() < 0.35:  # tokens after earlier ones
        case.update(q=case["seqs"] * rng.choice([1, 1, 2, 5]), past=_log(rng, 1, 16384), fused=0)
    else:
        # several tokens a sequence: a gradient through a single key is rounding alone
        case.update(q=max(4 * case["seqs"], _log(rng, 16, 16384)))
        if kind == "att_fwd" and rng.random() < 0.3:
            case.update(past=_log(rng, 1, 4096), fused=0)
    while _pairs(case) * case["heads"] * dim > PAIRS // (1 if kind == "att_bwd" else 2):
        case["q"] = max(1, case["q"] // 2)
        case["past"] //= 2
        case["seqs"] = min(case["seqs"], max(1, case["q"] // 4) if kind == "att_bwd" else case["q"])
    return case


# ------------------------------------------------------------------ inputs --
def _lengths(case):
    """Queries and keys of each sequence: a random partition of `q`, at most `past` earlier keys."""
    rng = random.Random(case["split"])
    n, q = case["seqs"], case["q"]
    if q // n <= 8:
        lq = [q // n + (k < q % n) for k in range(n)]
    else:
        share = [rng.random() + 0.05 for _ in range(n)]
        cuts = [int(sum(share[:k]) / sum(share) * (q - n)) + k for k in range(n)] + [q]
        lq = [b - a for a, b in zip(cuts, cuts[1:])]
    return lq, [v + (rng.randint(0, case["past"]) if case["past"] else 0) for v in lq]


def _pairs(case):
    """Visible pairs of a query and a key."""
    return sum(a * b - (a * (a - 1) // 2 if case["causal"] else 0) for a, b in zip(*_lengths(case)))


def _matrix(gen, rows, cols, pad, dtype, scale=1.0):
    """A [rows, cols] matrix of normal values, `pad` elements between its rows."""
    wide = torch.randn(rows, cols + pad, generator=gen, device=DEV)
    return (wide * scale).to(dtype)[:, :cols]


def _prepare_rms(case, s, gen):
    rows, c, pad = case["rows"], case["c"], case["pad"]
    # a few of a stream's channels are much larger than the others
    spread = torch.exp(0.5 * torch.randn(c, generator=gen, device=DEV))
    s["w"] = 1.0 + 0.2 * torch.randn(c, generator=gen, device=DEV)
    if case["kind"] == "rms_fwd":
        s["x"] = _matrix(gen, rows, c, pad, TYPES[case["x"]], torch.nn.functional.pad(spread, (0, pad)))
        s["res"] = _matrix(gen, rows, c, 0, TYPES[case["h"]], 2.0 * spread) if case["res"] else None
    else:
        s["h"] = _matrix(gen, rows, c, pad, TYPES[case["h"]], torch.nn.functional.pad(spread, (0, pad)))
        s["st"] = (s["h"].double().square().mean(1) + EPS).rsqrt().float()
    if case["kind"] == "rms_bwd":
        s["g"] = _matrix(gen, rows, c, pad, TYPES[case["g"]])
        s["gh"] = _matrix(gen, rows, c, 0, TYPES[case["d"]]) if case["res"] else None
    if not own:
        return
    from paper_1604_06174_amd import ckpt as K
    code = {"bf16": K.TYPE_BF16, "f32": K.TYPE_F32, "f8": K.TYPE_E4M3}
    ld = c + pad
    empty = lambda t, *shape: torch.empty(*shape, dtype=TYPES[t], device=DEV)
    s["desc"] = K.rms_desc(rows, c, xtype=code[case["x"]], htype=code[case["h"]], ytype=code[case.get("y", case["h"])],
                           gtype=code[case.get("g", "bf16")], dtype=code[case.get("d", case["h"])],
                           qgroup=case.get("group", 0), ldx=ld, ldh=c if case["kind"] == "rms_fwd" else ld, ldg=ld,
                           eps=EPS)
    if case["kind"] == "rms_bwd":
        nb = K.op_rms_workspace_bytes(s["desc"])
        s["ws"] = torch.empty(max(nb, 1), dtype=torch.uint8, device=DEV)
        s["d"], s["dw"] = empty(case["d"], rows, c), empty("f32", c)
        return
    s["y"] = empty(case["y"], rows, c)
    s["ys"] = empty("f32", rows, -(-c // (case["group"] or c))) if case["y"] == "f8" else None
    if case["kind"] == "rms_fwd":
        s["hsum"] = empty(case["h"], rows, c) if case["res"] else None
        s["st"] = empty("f32", rows)


def _prepare_emb(case, s, gen):
    n, vocab, c, pad = (case[k] for k in ("tokens", "vocab", "c", "pad"))
    # ranks uniform in their logarithm, as those of words nearly are, in a shuffled vocabulary
    rank = torch.exp(torch.rand(n, generator=gen, device=DEV, dtype=torch.float64) * math.log(vocab)).long() - 1
    s["ids"] = torch.randperm(vocab, generator=gen, device=DEV)[rank.clamp(0, vocab - 1)].to(torch.int32)
    s["scale"] = math.sqrt(c)
    if case["kind"] == "emb_fwd":
        s["w"] = _matrix(gen, vocab, c, 0, TYPES[case["w"]], 0.02)
    else:
        s["g"] = _matrix(gen, n, c, pad, TYPES[case["g"]])
    if not own:
        return
    from paper_1604_06174_amd import ckpt as K
    code = {"bf16": K.TYPE_BF16, "f32": K.TYPE_F32}
    if case["kind"] == "emb_fwd":
        s["desc"] = K.embed_desc(n, vocab, c, wtype=code[case["w"]], ytype=code[case["y"]], scale=s["scale"],
                                 ldy=c + pad)
        s["y"] = torch.empty(n, c + pad, dtype=TYPES[case["y"]], device=DEV)[:, :c]
    else:
        s["desc"] = K.embed_desc(n, vocab, c, gtype=code[case["g"]], dtype=code[case["d"]], scale=s["scale"],
                                 ldg=c + pad)
        nb = K.op_embed_workspace_bytes(s["desc"])
        s["ws"] = torch.empty(max(nb, 1), dtype=torch.uint8, device=DEV)
        s["dw"] = torch.empty(vocab, c, dtype=TYPES[case["d"]], device=DEV)


def _prepare_att(case, s, gen):
    heads, kv, dim = case["heads"], case["kv_heads"], case["dim"]
    s["lq"], s["lk"] = _lengths(case)
    tq, tk = sum(s["lq"]), sum(s["lk"])
    acc = lambda v: torch.tensor([sum(v[:k]) for k in range(len(v) + 1)], dtype=torch.int32, device=DEV)
    s["qoff"], s["koff"] = acc(s["lq"]), acc(s["lk"])
    if case["fused"]:  # slices of one projection's output
        qkv = torch.randn(tq, heads + 2 * kv, dim, generator=gen, device=DEV).to(torch.bfloat16)
        s["q"], s["k"], s["v"] = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    else:
        part = lambda t, n: torch.randn(t, n, dim, generator=gen, device=DEV).to(torch.bfloat16)
        s["q"], s["k"], s["v"] = part(tq, heads), part(tk, kv), part(tk, kv)
    if case["kind"] == "att_bwd":
        s["g"] = torch.randn(tq, heads, dim, generator=gen, device=DEV).to(torch.bfloat16)
        s["o"], s["lse"] = _att_forward(case, s)
    if not own:
        return
    from paper_1604_06174_amd import ckpt as K
    st = lambda t: (t.stride(0), t.stride(1))
    (ldq, hsq), (ldk, hsk), (ldv, hsv) = st(s["q"]), st(s["k"]), st(s["v"])
    s["desc"] = K.attn_desc(tq, tk, case["seqs"], heads, kv, dim, causal=bool(case["causal"]), ldq=ldq, hsq=hsq,
                            ldk=ldk, hsk=hsk, ldv=ldv, hsv=hsv)
    nb = K.op_attn_workspace_bytes(s["desc"], case["kind"] == "att_bwd")
    s["ws"] = torch.empty(max(nb, 1), dtype=torch.uint8, device=DEV)
    if case["kind"] == "att_fwd":
        s["o"] = torch.empty(tq, heads, dim, dtype=torch.bfloat16, device=DEV)
        s["lse"] = torch.empty(heads, tq, device=DEV)
    else:
        if case["fused"]:
            d = torch.empty(tq, heads + 2 * kv, dim, dtype=torch.bfloat16, device=DEV)
            s["dq"], s["dk"], s["dv"] = d[:, :heads], d[:, heads:heads + kv], d[:, heads + kv:]
        else:
            s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[k]) for k in "qkv")


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(case=case)
    {"rms": _prepare_rms, "emb": _prepare_emb, "att": _prepare_att}[case["kind"][:3]](case, s, gen)
    return s


# -------------------------------------------------------------- plain form --
def _to_8_bits(u, group):
    """Values of e4m3 with one scale for each `group` columns (0: a row) and the scales."""
    rows, c = u.shape
    group = group or c
    wide = torch.nn.functional.pad(u, (0, -c % group)).reshape(rows, -1, group)
    top = wide.abs().amax(2).clamp(min=TINY)
    v = (wide * (448.0 / top)[:, :, None]).reshape(rows, -1)[:, :c]
    return v.to(torch.float8_e4m3fn), top / 448.0


def _plain_rms(case, s):
    if case["kind"] == "rms_bwd":
        h, g, st = s["h"].float(), s["g"].float(), s["st"][:, None]
        xhat = h * st
        du = g * s["w"]
        d = st * (du - xhat * (du * xhat).mean(1, keepdim=True))
        if s["gh"] is not None:
            d = d + s["gh"].float()
        return d.to(TYPES[case["d"]]), (g * xhat).sum(0)
    if case["kind"] == "rms_fwd":
        h = s["x"]
        if s["res"] is not None:
            h = (h.float() + s["res"].float()).to(TYPES[case["h"]])
        st = 1.0 / torch.sqrt(h.float().square().mean(1) + EPS)
    else:
        h, st = s["h"], s["st"]
    u = h.float() * st[:, None] * s["w"]
    y = _to_8_bits(u, case["group"]) if case["y"] == "f8" else (u.to(TYPES[case["y"]]),)
    if case["kind"] == "rms_apply":
        return y
    return y + (st,) + ((h,) if s["res"] is not None else ())


def _plain_emb(case, s):
    ids = s["ids"].long()
    if case["kind"] == "emb_fwd":
        return (s["w"][ids].float() * s["scale"]).to(TYPES[case["y"]])
    order = torch.argsort(ids, stable=True)
    count = torch.bincount(ids, minlength=case["vocab"])
    # sums of rows that a running sum in 64 bits differs by
    total = torch.cumsum(s["g"][order].double(), 0)
    total = torch.cat([torch.zeros_like(total[:1]), total])
    end = torch.cumsum(count, 0)
    return ((total[end] - total[end - count]) * s["scale"]).to(TYPES[case["d"]])


def _scores(case, q, k):
    """Scores of queries [heads, lq, dim] with keys [kv_heads, lk, dim], hidden ones -inf."""
    lq, lk, rep = q.shape[1], k.shape[1], case["heads"] // case["kv_heads"]
    a = torch.matmul(q, k.repeat_interleave(rep, 0).transpose(1, 2).contiguous()) * (1.0 / math.sqrt(case["dim"]))
    if case["causal"]:
        i, j = torch.arange(lq, device=DEV)[:, None], torch.arange(lk, device=DEV)[None]
        a = a.masked_fill(j > i + (lk - lq), -math.inf)
    return a


def _sequences(s):
    a = b = 0
    for n, m in zip(s["lq"], s["lk"]):
        yield slice(a, a + n), slice(b, b + m)
        a, b = a + n, b + m


def _heads_first(t):
    return t.float().transpose(0, 1).contiguous()


def _att_forward(case, s):
    heads, rep = case["heads"], case["heads"] // case["kv_heads"]
    o = torch.empty(s["q"].shape[0], heads, case["dim"], dtype=torch.bfloat16, device=DEV)
    lse = torch.empty(heads, s["q"].shape[0], device=DEV)
    for qs, ks in _sequences(s):
        a = _scores(case, _heads_first(s["q"][qs]), _heads_first(s["k"][ks]))
        top = a.amax(2, keepdim=True)
        p = torch.exp(a - top)
        z = p.sum(2, keepdim=True)
        v = _heads_first(s["v"][ks]).repeat_interleave(rep, 0)
        o[qs] = (torch.matmul(p, v) / z).transpose(0, 1).to(torch.bfloat16)
        lse[:, qs] = (top + torch.log(z))[:, :, 0]
    return o, lse


def _plain_att(case, s):
    if case["kind"] == "att_fwd":
        return _att_forward(case, s)
    heads, kv, dim = case["heads"], case["kv_heads"], case["dim"]
    rep, scale = heads // kv, 1.0 / math.sqrt(dim)
    dq, dk, dv = (torch.empty(s[n].shape, dtype=torch.bfloat16, device=DEV) for n in "qkv")
    for qs, ks in _sequences(s):
        q, k, g, o = (_heads_first(t) for t in (s["q"][qs], s["k"][ks], s["g"][qs], s["o"][qs]))
        v = _heads_first(s["v"][ks]).repeat_interleave(rep, 0)
        p = torch.exp(_scores(case, q, k) - s["lse"][:, qs, None])
        shared = lambda t: t.reshape(kv, rep, -1, dim).sum(1).transpose(0, 1).to(torch.bfloat16)
        dv[ks] = shared(torch.matmul(p.transpose(1, 2).contiguous(), g))
        dp = torch.matmul(g, v.transpose(1, 2).contiguous()) - (g * o).sum(2, keepdim=True)
        ds = p * dp * scale
        dq[qs] = torch.matmul(ds, k.repeat_interleave(rep, 0)).transpose(0, 1).to(torch.bfloat16)
        dk[ks] = shared(torch.matmul(ds.transpose(1, 2).contiguous(), q))
    return dq, dk, dv


# --------------------------------------------------------------- one pass --
def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        return {"rms": _plain_rms, "emb": _plain_emb, "att": _plain_att}[kind[:3]](case, s)
    from paper_1604_06174_amd import ckpt as K
    st = torch.cuda.current_stream()
    if kind == "rms_bwd":
        K.op_rms_backward(s["desc"], s["g"], s["h"], s["st"], s["w"], s["d"], s["dw"], s["ws"], s["ws"].numel(),
                          gh=s["gh"], stream=st)
        return s["d"], s["dw"]
    if kind.startswith("rms"):
        if kind == "rms_fwd":
            K.op_rms_forward(s["desc"], s["x"], s["w"], s["y"], s["st"], res=s["res"], h=s["hsum"], ys=s["ys"],
                             stream=st)
        else:
            K.op_rms_apply(s["desc"], s["h"], s["st"], s["w"], s["y"], ys=s["ys"], stream=st)
        y = (s["y"], s["ys"]) if case["y"] == "f8" else (s["y"],)
        if kind == "rms_apply":
            return y
        return y + (s["st"],) + ((s["hsum"],) if s["res"] is not None else ())
    if kind == "emb_fwd":
        K.op_embed_forward(s["desc"], s["ids"], s["w"], s["y"], stream=st)
        return s["y"]
    if kind == "emb_bwd":
        K.op_embed_backward(s["desc"], s["ids"], s["g"], s["dw"], s["ws"], s["ws"].numel(), stream=st)
        return s["dw"]
    if kind == "att_fwd":
        K.op_attn_forward(s["desc"], s["q"], s["k"], s["v"], s["qoff"], s["koff"], s["o"], s["lse"], s["ws"],
                          s["ws"].numel(), stream=st)
        return s["o"], s["lse"]
    K.op_attn_backward(s["desc"], s["g"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["qoff"], s["koff"], s["dq"],
                       s["dk"], s["dv"], s["ws"], s["ws"].numel(), stream=st)
    return s["dq"], s["dk"], s["dv"]


# ------------------------------------------------------------- definition --
def _exact_att(case, s):
    """Sums written out over one query head at a time."""
    rep, scale = case["heads"] // case["kv_heads"], case["dim"] ** -0.5
    wide = {n: s[n].double() for n in "qkvgo" if n in s}
    out = {n: torch.zeros_like(wide[n]) for n in ("qkv" if case["kind"] == "att_bwd" else "q")}
    lse = torch.zeros(case["heads"], s["q"].shape[0], dtype=torch.float64, device=DEV)
    a = b = 0
    for n, m in zip(s["lq"], s["lk"]):
        seen = torch.ones(n, m, dtype=torch.bool, device=DEV)
        if case["causal"]:
            seen = seen.tril(m - n)
        for h in range(case["heads"]):
            kq, kk = (slice(a, a + n), h), (slice(b, b + m), h // rep)
            e = (wide["q"][kq] @ wide["k"][kk].T) * scale
            if case["kind"] == "att_fwd":
                e = torch.where(seen, e, torch.full_like(e, -math.inf))
                lse[h, a:a + n] = torch.logsumexp(e, 1)
                out["q"][kq] = torch.softmax(e, 1) @ wide["v"][kk]
                continue
            p = torch.where(seen, torch.exp(e - s["lse"][h, a:a + n].double()[:, None]), torch.zeros_like(e))
            inner = (wide["g"][kq] * wide["o"][kq]).sum(1)
            ds = p * (wide["g"][kq] @ wide["v"][kk].T - inner[:, None])
            out["q"][kq] = ds @ wide["k"][kk] * scale
            out["k"][kk] += ds.T @ wide["q"][kq] * scale
            out["v"][kk] += p.T @ wide["g"][kq]
        a, b = a + n, b + m
    return (out["q"], lse) if case["kind"] == "att_fwd" else (out["q"], out["k"], out["v"])


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind.startswith("att"):
        return _exact_att(case, s)
    if kind == "emb_fwd":
        return s["w"].double().index_select(0, s["ids"].long()) * s["scale"]
    if kind == "emb_bwd":
        d = torch.zeros(case["vocab"], case["c"], dtype=torch.float64, device=DEV)
        return d.index_add_(0, s["ids"].long(), s["g"].double() * s["scale"])
    w = s["w"].double()
    if kind == "rms_bwd":
        h, g, r = s["h"].double(), s["g"].double(), s["st"].double().unsqueeze(1)
        inner = torch.einsum("rc,rc,c->r", g, h, w).unsqueeze(1) / case["c"]
        d = g * w * r - h * inner * r ** 3
        return (d if s["gh"] is None else d + s["gh"].double()), (g * h * r).sum(0)
    if kind == "rms_fwd":
        h = s["x"].double()
        if s["res"] is not None:  # the stream is kept in its own type, and that is what is normalised
            h = (h + s["res"].double()).to(TYPES[case["h"]]).double()
        st = (h.square().mean(1) + EPS).pow(-0.5)
    else:
        h, st = s["h"].double(), s["st"].double()
    u = h * st.unsqueeze(1) * w
    y = (u,)
    if case["y"] == "f8":
        cols = torch.split(u.abs(), case["group"] or case["c"], 1)
        each = [t.max(1, keepdim=True).values.clamp(min=TINY) / 448 for t in cols]
        y = (torch.cat([a / b for a, b in zip(torch.split(u, case["group"] or case["c"], 1), each)], 1), torch.cat(each, 1))
    if kind == "rms_apply":
        return y
    return y + (st,) + ((h,) if s["res"] is not None else ())


def work(case):
    kind = case["kind"]
    if kind.startswith("rms"):
        e, rows, c = case["rows"] * case["c"], case["rows"], case["c"]
        if kind == "rms_bwd":
            b = e * (SIZE[case["h"]] + SIZE[case["g"]] + SIZE[case["d"]] * (1 + case["res"])) + 4 * rows + 8 * c
            return {"bytes": b, "flops": e * (10 + case["res"])}
        b = e * SIZE[case["y"]] + 4 * rows + 4 * c
        if case["y"] == "f8":
            b += 4 * rows * -(-c // (case["group"] or c))
        if kind == "rms_apply":
            b += e * SIZE[case["h"]]
        else:
            b += e * (SIZE[case["x"]] + (2 * SIZE[case["h"]] if case["res"] else 0))
        return {"bytes": b, "flops": e * ((4 if kind == "rms_fwd" else 2) + case["res"] + (2 if case["y"] == "f8" else 0))}
    if kind.startswith("emb"):
        n, vocab, c = case["tokens"], case["vocab"], case["c"]
        if kind == "emb_bwd":
            return {"bytes": n * (4 + c * SIZE[case["g"]]) + vocab * c * SIZE[case["d"]], "flops": (n + vocab) * c}
        # rows that are looked up: at most each of the table's once
        return {"bytes": 4 * n + min(n, vocab) * c * SIZE[case["w"]] + n * c * SIZE[case["y"]], "flops": n * c}
    lq, lk = _lengths(case)
    rows = sum(lq) * case["heads"] * case["dim"] * 2
    kv = 2 * sum(lk) * case["kv_heads"] * case["dim"] * 2
    products = 2 * case["dim"] * case["heads"] * _pairs(case)
    lse = 4 * sum(lq) * case["heads"]
    if kind == "att_fwd":
        return {"bytes": 2 * rows + kv + lse, "flops": 2 * products}
    return {"bytes": 4 * rows + 2 * kv + lse, "flops": 5 * products}
