"""Helpers of the tests of the token models' operators: strided device tensors with
guarded surroundings, and comparison with a bound for each element."""
import numpy as np

from oracle import units as U

DEV = "cuda:0"
STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # half a step, of the value
GUARD = -77.0


def K():
    from paper_1604_06174_amd import ckpt
    return ckpt


def dtype(t):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32, "f8": torch.float8_e4m3fn}[t]


def code(t):
    k = K()
    return {"bf16": k.TYPE_BF16, "f32": k.TYPE_F32, "f8": k.TYPE_E4M3}[t]


def rounded(v, t):
    """float64 -> the type's values, as float64 (through fp32, as a sum formed in fp32 is)."""
    v = np.asarray(v, np.float32)
    return (v if t == "f32" else U.bf16_round(v)).astype(np.float64)


class Rows:
    """[rows, cols] of a type, `pad` elements between the rows and `shift` before the first;
    what is not a row's holds a value that no call may change."""

    def __init__(self, rows, cols, t, pad=0, shift=0, data=None):
        import torch
        self.rows, self.cols, self.ld, self.t = rows, cols, cols + pad, t
        self.all = torch.full((shift + rows * self.ld + 16,), GUARD, dtype=torch.float32, device=DEV).to(dtype(t))
        self.shift = shift
        self.m = self.all[shift:shift + rows * self.ld].view(rows, self.ld)[:, :cols]
        if data is not None:
            self.m.copy_(torch.from_numpy(np.ascontiguousarray(np.asarray(data, np.float32).reshape(rows, cols))))

    def data_ptr(self):
        return self.m.data_ptr()

    def host(self):
        import torch
        torch.cuda.synchronize()
        v = self.m.float().cpu().numpy().astype(np.float64)
        rest = self.all.clone().float()
        fill = float(torch.full((1,), GUARD).to(dtype(self.t)).float())
        rest[self.shift:self.shift + self.rows * self.ld].view(self.rows, self.ld)[:, :self.cols] = fill
        assert bool((rest == fill).all()), "written outside its rows"
        return v


def f32(v):
    import torch
    return torch.from_numpy(np.ascontiguousarray(np.asarray(v, np.float32))).to(DEV)


def host(t):
    import torch
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def close(name, got, want, tol):
    """Every element within its bound; where `want` is not finite, the same value."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    fin = np.isfinite(want)
    assert np.array_equal(got[~fin], want[~fin], equal_nan=True), f"{name}: special values"
    if not fin.any():
        return
    assert np.isfinite(got[fin]).all(), f"{name}: not finite"
    rel = np.abs(got[fin] - want[fin]) / (np.broadcast_to(tol, want.shape)[fin] + 1e-38)
    print(f"    {name}: {rel.max():.3f} of its bar", flush=True)
    assert rel.max() <= 1.0, (name, float(rel.max()), int(rel.argmax()))
