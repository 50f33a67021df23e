"""Shared by the tests of dense layers and layer norm: guarded matrices, 64-bit formulas, and the error bounds of the fp32
arithmetic in between, from which the tests' tolerances come."""
import math

import torch

HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # of a rounding, relative
HALF_TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}  # ... among the subnormals
U32 = 2.0 ** -23               # one step of fp32, relative: what an addition on the tensor core may lose (it may cut off)
GUARD = 7168.0                 # exact in every type


class Guarded:
    """A [rows, cols] matrix inside a larger buffer: rows `ld` apart, whole rows before and after it.  What lies around the matrix is
    NaN for an input (reading it shows in the results) and GUARD for an output (writing there shows in check())."""

    def __init__(self, rows, cols, dtype, ld=None, values=None, offset=0):
        ld = ld or (cols + 7) // 8 * 8
        fill = math.nan if values is not None else GUARD
        self.buffer = torch.full(((rows + 4) * ld + 8,), fill, device="cuda", dtype=dtype)
        self.t = torch.as_strided(self.buffer, (rows, cols), (ld, 1), 2 * ld + offset)
        if values is not None:
            self.t.copy_(values)

    def check(self):
        outside = self.buffer.clone()
        torch.as_strided(outside, self.t.shape, self.t.stride(), self.t.storage_offset()).fill_(GUARD)
        assert torch.all(outside == GUARD), "written outside the matrix"
        return self.t


def act(name, z):
    """(act(z), act'(z), p, u', |u|): p the logistic function of the argument u."""
    zero, one = torch.zeros_like(z), torch.ones_like(z)
    if name == "none":
        return z, one, one, zero, zero
    if name == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype), one, zero, zero
    if name == "silu":
        u, slope = z, one
    else:
        c = 2 * math.sqrt(2 / math.pi)
        u, slope = c * (z + 0.044715 * z ** 3), c * (1 + 3 * 0.044715 * z ** 2)
    p = torch.sigmoid(u)
    return z * p, p + z * p * (1 - p) * slope, p, slope, u.abs()


def act_error(name, z):
    """Bound of the error of act(z) taken in fp32.  exp2 and 1/x by the approximate units: 2 steps each, and the argument u,
    of a few operations, is off by 4 steps, so p by p (1 - p) 4 |u| steps and 6 steps of itself."""
    if name in ("none", "relu"):
        return torch.zeros_like(z)
    _, _, p, _, u = act(name, z)
    return z.abs() * U32 * (p * (1 - p) * 4 * u + 7 * p) + 1e-36


def act_grad_error(name, z):
    """The same of act'(z) = p + z p (1 - p) u': the error of p enters twice, and 1 - p is off by a step of 1."""
    if name in ("none", "relu"):
        return torch.zeros_like(z)
    _, _, p, slope, u = act(name, z)
    dp = U32 * (p * (1 - p) * 4 * u + 6 * p)
    return dp + (z * slope).abs() * (dp * (1 - p) + p * (dp + U32) + 4 * U32 * p * (1 - p)) + 1e-24


def close(got, want, bound, what):
    got, want = got.double(), want.double()
    assert got.shape == want.shape
    off = (got - want).abs() - bound
    assert bool(torch.all(off <= 0)), f"{what}: {float((got - want).abs().max())} off, {float(off.max())} more than the bound allows"
