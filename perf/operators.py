"""The normalisation and dropout operators whose speed matters, case by case.

Kinds:
  fwd      group norm - activation [- dropout], statistics formed (`op_gn_forward`)
  apply    the same with the statistics known: the re-run of a checkpointed unit (`op_gn_apply`)
  bwd      its backward: data gradient, scale and shift gradients (`op_gn_backward`)
  dropout  dropout [+ residual], forward or (no residual) backward (`op_dropout`)

Tensors are channels last: n samples of hw pixels of c channels, `pad` elements
between the pixels of the inputs (a channel slice of a wider tensor).  Dropout
takes the 16-bit half e % 8 of block e / 8 of Philox4x32-10 (Salmon et al.,
"Parallel random numbers: as easy as 1, 2, 3", 2011) for element e of the
tensor in row-major order.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one image at the last stage of the ImageNet-shaped ResNet: evaluation or debugging, where latency counts
        dict(name="gn_fwd_7x7_b1", kind="fwd", n=1, hw=49, c=512, groups=32, act="relu", x="bf16", pad=0, p=0.0),
        # that network's stem output at its training batch: few channels, two per group, many pixels
        dict(name="gn_fwd_stem", kind="fwd", n=32, hw=12544, c=64, groups=32, act="relu", x="bf16", pad=0, p=0.0),
        # a channel slice of a wider float32 tensor, odd image, groups that no vector width divides
        dict(name="gn_fwd_odd_f32", kind="fwd", n=5, hw=1131, c=120, groups=12, act="silu", x="f32", pad=32, p=0.0),
        # norm - activation - dropout of a unit of stage 2
        dict(name="gn_drop_fwd_s2", kind="fwd", n=32, hw=784, c=512, groups=32, act="silu", x="bf16", pad=0, p=0.1),
        # the re-run of a unit of stage 1 whose statistics the first forward kept
        dict(name="gn_apply_s1", kind="apply", n=32, hw=3136, c=64, groups=32, act="relu", x="bf16", pad=0, p=0.0),
        # backward of the expansion of stage 3: the float32 gradient of a convolution in, the bfloat16 one of the
        # next out
        dict(name="gn_bwd_s3", kind="bwd", n=32, hw=196, c=1024, groups=32, act="relu", x="bf16", g="f32", d="bf16",
             pad=0, p=0.0),
        # backward of the largest activations, with dropout
        dict(name="gn_drop_bwd_s1", kind="bwd", n=32, hw=3136, c=256, groups=32, act="silu", x="bf16", g="bf16",
             d="bf16", pad=0, p=0.1),
        # rows of hidden states: 256 steps of the speech-sized LSTM at batch 64, one pixel per sample
        dict(name="gn_bwd_rows", kind="bwd", n=16384, hw=1, c=1024, groups=16, act="none", x="bf16", g="bf16",
             d="bf16", pad=0, p=0.0),
        # the CIFAR-shaped network's first stage, float32
        dict(name="gn_bwd_cifar_f32", kind="bwd", n=128, hw=1024, c=16, groups=4, act="relu", x="f32", g="f32",
             d="f32", pad=0, p=0.0),
        # a residual block's output of stage 1: shortcut + dropout(branch)
        dict(name="dropout_res_s1", kind="dropout", rows=100352, cols=256, x="bf16", y="bf16", res=1, pad=0, p=0.1),
        # a block of the residual MLP (width 1024, batch 256), float32
        dict(name="dropout_mlp_f32", kind="dropout", rows=256, cols=1024, x="f32", y="f32", res=0, pad=0, p=0.5),
        # a float32 gradient of odd width out of a wider tensor, rounded for the next product
        dict(name="dropout_bwd_odd", kind="dropout", rows=3211, cols=333, x="f32", y="bf16", res=0, pad=19, p=0.2),
    ]


LIMIT = 32 * 3136 * 250  # elements of a drawn case: the largest listed one's, less its statistics


def _log(rng, lo, hi):
    """An integer of [lo, hi], uniform in its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["fwd", "fwd", "apply", "bwd", "bwd", "dropout"])
    p = rng.choice([0.0, 0.0, 0.1, 0.25, 0.5])
    pad = rng.choice([0, 0, 0, 8, 64, 5])
    if kind == "dropout":
        cols = rng.choice([_log(rng, 1, 4096), 8 * _log(rng, 1, 512)])
        x = rng.choice(["bf16", "f32"])
        return dict(kind=kind, rows=_log(rng, 1, min(100352, LIMIT // 2 // cols)), cols=cols, x=x,
                    y=rng.choice([x, x, "bf16", "f32"]), res=rng.randint(0, 1), pad=pad,
                    p=rng.choice([0.1, 0.25, 0.5]))
    x = rng.choice(["bf16", "bf16", "f32"])
    limit = LIMIT // 2 if x == "f32" else LIMIT
    if kind == "bwd":
        g, d = ("f32", "f32") if x == "f32" else (rng.choice(["bf16", "f32"]), rng.choice(["bf16", "bf16", "f32"]))
        limit //= 2 if g == "f32" or d == "f32" else 1
    c = rng.choice([8 * _log(rng, 1, 256), 1 << rng.randint(4, 11), _log(rng, 8, 600)])
    if rng.random() < 0.2:
        hw = rng.choice([1, 1, 2, 3])
        n = _log(rng, 1, min(16384, limit // (hw * c)))
    else:
        hw = rng.choice([_log(rng, 4, 12544), rng.choice([7, 13, 14, 28, 31, 56, 112]) ** 2])
        hw = min(hw, limit // c)
        n = _log(rng, 1, max(1, min(128, limit // (hw * c))))
    # groups of eight values at least: with two or three, what is left of a gradient is rounding
    groups = rng.choice([k for k in range(1, min(c, 64) + 1) if c % k == 0 and hw * (c // k) >= 8])
    case = dict(kind=kind, n=n, hw=hw, c=c, groups=groups, act=rng.choice(["none", "relu", "silu"]), x=x, pad=pad, p=p)
    if kind == "bwd":
        case.update(g=g, d=d)
    return case


# ------------------------------------------------------------------ inputs --
def _matrix(gen, rows, cols, pad, dtype, scale=1.0, shift=0.0):
    """A [rows, cols] matrix of normal values, `pad` elements between its rows."""
    wide = torch.randn(rows, cols + pad, generator=gen, device=DEV)
    wide[:, :cols].mul_(scale).add_(shift)
    return wide.to(dtype)[:, :cols]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(case=case)
    s["site"] = 3 + seed % 5
    s["rng"] = torch.tensor([(seed * 0x9E3779B97F4A7C15 + 12345) % (1 << 63), 100 + seed % 1000], dtype=torch.int64,
                            device=DEV)
    if case["kind"] == "dropout":
        rows, cols = case["rows"], case["cols"]
        s["x"] = _matrix(gen, rows, cols, case["pad"], TYPES[case["x"]])
        s["res"] = _matrix(gen, rows, cols, 0, TYPES[case["y"]]) if case["res"] else None
        if own:
            from paper_1604_06174_amd import ckpt as K
            s["y"] = torch.empty(rows, cols, dtype=TYPES[case["y"]], device=DEV)
            s["drop"] = K.dropout(s["rng"], case["p"], s["site"])
        return s
    n, hw, c, groups = (case[k] for k in ("n", "hw", "c", "groups"))
    rows = n * hw
    # channels of a convolution's output differ in level and spread
    scale = 0.5 + torch.rand(c, generator=gen, device=DEV)
    shift = 0.5 * torch.randn(c, generator=gen, device=DEV)
    s["x"] = _matrix(gen, rows, c, case["pad"], TYPES[case["x"]], scale, shift)
    s["gamma"] = 1.0 + 0.2 * torch.randn(c, generator=gen, device=DEV)
    s["beta"] = 0.2 * torch.randn(c, generator=gen, device=DEV)
    if case["kind"] == "bwd":
        s["g"] = _matrix(gen, rows, c, case["pad"], TYPES[case["g"]])
    if case["kind"] != "fwd":
        v = s["x"].reshape(n, hw, groups, c // groups).double()
        mean = v.mean((1, 3))
        var = ((v - mean[:, None, :, None]) ** 2).mean((1, 3))
        s["st"] = torch.cat([mean.reshape(-1), (var + EPS).rsqrt().reshape(-1)]).float()
    if own:
        from paper_1604_06174_amd import ckpt as K
        types = {"bf16": K.TYPE_BF16, "f32": K.TYPE_F32}
        ld = c + case["pad"]
        s["desc"] = K.gn_desc(n, hw, c, groups, act={"none": K.ACT_NONE, "relu": K.ACT_RELU, "silu": K.ACT_SILU}[case["act"]],
                              xtype=types[case["x"]], gtype=types[case.get("g", case["x"])],
                              dtype=types[case.get("d", case["x"])], ldx=ld, ldg=ld, eps=EPS)
        s["drop"] = K.dropout(s["rng"], case["p"], s["site"]) if case["p"] > 0 else None
        nb = K.op_gn_workspace_bytes(s["desc"], case["kind"] == "bwd")
        s["ws"] = torch.empty(max(nb, 1), dtype=torch.uint8, device=DEV)
        if case["kind"] == "bwd":
            s["out"] = torch.empty(rows, c, dtype=TYPES[case["d"]], device=DEV)
            s["dgamma"] = torch.empty(c, device=DEV)
            s["dbeta"] = torch.empty(c, device=DEV)
        else:
            s["out"] = torch.empty(rows, c, dtype=TYPES[case["x"]], device=DEV)
            if case["kind"] == "fwd":
                s["st"] = torch.empty(2 * n * groups, device=DEV)
    return s


# -------------------------------------------------------------- plain form --
def _keep(count, p, rng, site):
    """The mask of `count` elements and the scale of the kept ones."""
    T = math.floor(65536 * p + 0.5)
    blk = torch.arange((count + 7) // 8, device=rng.device, dtype=torch.int64)
    low = 0xFFFFFFFF
    k0, k1 = rng[0] & low, (rng[0] >> 32) & low
    c = [blk, torch.full_like(blk, site), (rng[1] & low).expand_as(blk), ((rng[1] >> 32) & low).expand_as(blk)]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((b >> 32) & low) ^ c[1] ^ k0, b & low, ((a >> 32) & low) ^ c[3] ^ k1, a & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    w = torch.stack(c, 1)
    half = torch.stack([w & 0xFFFF, w >> 16], 2).reshape(-1)[:count]
    return half >= T, (65536.0 / (65536 - T) if T < 65536 else 0.0)


def _drop(v, case, s):
    if case["p"] == 0:
        return v
    keep, scale = _keep(v.numel(), case["p"], s["rng"], s["site"])
    return torch.where(keep.reshape(v.shape), v * scale, torch.zeros_like(v))


def _plain(s):
    case = s["case"]
    if case["kind"] == "dropout":
        v = _drop(s["x"].float(), case, s)
        if s["res"] is not None:
            v = s["res"].float() + v
        return v.to(TYPES[case["y"]])
    n, hw, c, groups = (case[k] for k in ("n", "hw", "c", "groups"))
    cg = c // groups
    x = s["x"].float().reshape(n, hw, groups, cg)
    gamma, beta = s["gamma"].reshape(groups, cg), s["beta"].reshape(groups, cg)
    if case["kind"] == "fwd":
        mean = x.mean((1, 3))
        var = ((x - mean[:, None, :, None]) ** 2).mean((1, 3))
        rstd = 1.0 / torch.sqrt(var + EPS)
    else:
        mean, rstd = s["st"].reshape(2, n, groups)
    mean, rstd = mean[:, None, :, None], rstd[:, None, :, None]
    t = x - mean
    u = t * (gamma * rstd) + beta
    if case["kind"] != "bwd":
        if case["act"] == "relu":
            u = torch.relu(u)
        elif case["act"] == "silu":
            u = u / (1.0 + torch.exp(-u))
        y = _drop(u, case, s).reshape(n * hw, c).to(TYPES[case["x"]])
        if case["kind"] == "apply":
            return y
        return y, torch.cat([mean.reshape(-1), rstd.reshape(-1)])
    du = _drop(s["g"].float().reshape(n, hw, groups, cg), case, s)
    if case["act"] == "relu":
        du = torch.where(u > 0, du, torch.zeros_like(du))
    elif case["act"] == "silu":
        sg = 1.0 / (1.0 + torch.exp(-u))
        du = du * (sg * (1.0 + u * (1.0 - sg)))
    xhat = t * rstd
    dgamma = (du * xhat).sum((0, 1)).reshape(-1)
    dbeta = du.sum((0, 1)).reshape(-1)
    dx = du * gamma
    d = rstd * (dx - dx.mean((1, 3), keepdim=True) - xhat * (dx * xhat).mean((1, 3), keepdim=True))
    return d.reshape(n * hw, c).to(TYPES[case["d"]]), dgamma, dbeta


# --------------------------------------------------------------- one pass --
def run(s):
    if not own:
        return _plain(s)
    from paper_1604_06174_amd import ckpt as K
    case, st = s["case"], torch.cuda.current_stream()
    kind = case["kind"]
    if kind == "dropout":
        K.op_dropout(case["rows"], case["cols"], s["x"], s["y"], s["drop"], res=s["res"], xtype=K.type_of(s["x"]),
                     ytype=K.type_of(s["y"]), ldx=case["cols"] + case["pad"], stream=st)
        return s["y"]
    if kind == "fwd":
        K.op_gn_forward(s["desc"], s["x"], s["gamma"], s["beta"], s["out"], s["st"], s["ws"], s["ws"].numel(),
                        drop=s["drop"], stream=st)
        return s["out"], s["st"]
    if kind == "apply":
        K.op_gn_apply(s["desc"], s["x"], s["st"], s["gamma"], s["beta"], s["out"], drop=s["drop"], stream=st)
        return s["out"]
    K.op_gn_backward(s["desc"], s["g"], s["x"], s["st"], s["gamma"], s["beta"], s["out"], s["dgamma"], s["dbeta"],
                     s["ws"], s["ws"].numel(), drop=s["drop"], stream=st)
    return s["out"], s["dgamma"], s["dbeta"]


# ------------------------------------------------------------- definition --
def _philox_halves(count, seed, step, site):
    """The first `count` 16-bit halves, in 64-bit unsigned integers on the host."""
    u = np.uint64
    sh, lo = u(32), u(0xFFFFFFFF)
    x0 = np.arange(-(-count // 8), dtype=u)
    x1 = np.full_like(x0, site)
    x2 = np.full_like(x0, step % (1 << 32))
    x3 = np.full_like(x0, step >> 32)
    for r in range(10):
        key0 = u((seed % (1 << 32) + r * 0x9E3779B9) % (1 << 32))
        key1 = u(((seed >> 32) + r * 0xBB67AE85) % (1 << 32))
        pa, pb = x0 * u(0xD2511F53), x2 * u(0xCD9E8D57)
        x0, x1, x2, x3 = (pb >> sh) ^ x1 ^ key0, pb & lo, (pa >> sh) ^ x3 ^ key1, pa & lo
    words = np.stack([x0, x1, x2, x3], -1).astype("<u4")
    return words.view("<u2").reshape(-1)[:count]


def exact(case, seed):
    s = prepare(case, seed)
    factor = None
    if case["p"] > 0:
        T = math.floor(65536 * case["p"] + 0.5)
        seed64, step = (int(v) for v in s["rng"].tolist())
        half = torch.from_numpy(_philox_halves(s["x"].numel(), seed64, step, s["site"]).astype(np.int32)).to(DEV)
        factor = (half >= T).double().reshape(s["x"].shape) * (65536 / (65536 - T))
    if case["kind"] == "dropout":
        y = s["x"].double() * factor
        return y if s["res"] is None else y + s["res"].double()
    n, hw, c, groups = (case[k] for k in ("n", "hw", "c", "groups"))
    rep = lambda v: v.repeat_interleave(c // groups, 1)[:, None, :]  # [n, groups] -> [n, 1, c]
    pool = lambda v: v.reshape(n, groups, c // groups).sum(2) / (hw * (c // groups))
    x = s["x"].double().reshape(n, hw, c)
    gamma, beta = s["gamma"].double(), s["beta"].double()
    if case["kind"] == "fwd":
        mean = pool(x.sum(1))
        rstd = (pool((x - rep(mean)).square().sum(1)) + EPS) ** -0.5
    else:
        mean, rstd = s["st"].double().reshape(2, n, groups)
    xhat = (x - rep(mean)) * rep(rstd)
    u = xhat * gamma + beta
    if case["kind"] != "bwd":
        y = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "silu": lambda v: v * torch.sigmoid(v)}[case["act"]](u)
        y = y.reshape(n * hw, c)
        y = y if factor is None else y * factor
        return y if case["kind"] == "apply" else (y, torch.cat([mean.flatten(), rstd.flatten()]))
    du = s["g"].double() if factor is None else s["g"].double() * factor
    du = du.reshape(n, hw, c)
    if case["act"] == "relu":
        du = du * (u > 0)
    elif case["act"] == "silu":
        q = torch.sigmoid(u)
        du = du * (q + u * q * (1 - q))
    dx = du * gamma
    d = (dx - rep(pool(dx.sum(1))) - xhat * rep(pool((dx * xhat).sum(1)))) * rep(rstd)
    return d.reshape(n * hw, c), (du * xhat).sum((0, 1)), du.sum((0, 1))


def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["kind"] == "dropout":
        e = case["rows"] * case["cols"]
        return {"bytes": e * (size[case["x"]] + size[case["y"]] * (1 + case["res"])), "flops": e * (1 + case["res"])}
    e, ng, c = case["n"] * case["hw"] * case["c"], case["n"] * case["groups"], case["c"]
    extra = {"none": 0, "relu": 1, "silu": 4}[case["act"]] + (1 if case["p"] > 0 else 0)
    if case["kind"] == "bwd":
        return {"bytes": e * (size[case["x"]] + size[case["g"]] + size[case["d"]]) + 8 * ng + 16 * c,
                "flops": e * (14 + extra)}
    return {"bytes": 2 * e * size[case["x"]] + 8 * ng + 8 * c, "flops": e * ((7 if case["kind"] == "fwd" else 3) + extra)}
