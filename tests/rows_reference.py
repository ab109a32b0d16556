"""Plain 64-bit forms of group norm, rows in 8 bits and their products, and the error bounds that the tests hold the
kernels to: (value, bound) as in block_reference. u = 2^-24 is fp32's half step, relative to the value."""
import numpy as np
import torch

from block_reference import HALF, U, activation

SLOPE = 1.13      # of every activation, at most


def moments(x, groups, together):
    """x [M][N][C] in 64 bits -> mean, variance and largest magnitude of each run of frames and group,
    [M / together][groups], by two passes."""
    M, N, C = x.shape
    v = x.reshape(M // together, together * N, groups, C // groups)
    mean = v.mean((1, 3))
    var = (v - mean[:, None, :, None]).square().mean((1, 3))
    return mean, var, v.abs().amax((1, 3))


def group_norm(x, groups, weight=None, bias=None, eps=1e-5, act="none", together=1):
    """x [M][N][C]; weight and bias [C] or [M][C] (of the listed frames) -> [M][N][C] fp32 results before their rounding
    to the type, and their bound.

    A is a group's largest magnitude, s = sqrt(var + eps). Means: a thread adds eight rows at a time (8 u A) and joins
    that sum's mean to its own (a rounding of u A each, at most 15 times where a run has up to 120 rows of a thread: the
    kernels' runs of the tests' sizes), then up to 8 times in the tree of threads, and sums the channels of a group (8 u A: a
    lane's channels and six halvings, by way of sums of at most 64 u A / 8); totals are in 64 bits and rounded once: 42 u A.
    Squared deviations are about such means, so that each deviation is off by as much and their mean square by
    2 s 42 u A; their sums add 42 u relative: 1 / s is off by (42 A / s + 42) u relative. The result is three fp32
    operations more. An activation has a slope of 1.13 at most and is worth 32 u of its argument."""
    x = x.double()
    M, N, C = x.shape
    per = C // groups
    mean, var, A = (t.repeat_interleave(per, 1).repeat_interleave(together, 0)[:, None] for t in moments(x, groups, together))
    s = torch.sqrt(var + eps)
    z = (x - mean) / s
    one = lambda t: torch.ones(1, 1, 1, dtype=torch.float64, device=x.device) if t is None else t.double().reshape(-1, 1, C)  # noqa: E731
    w = one(weight)
    y = z * w
    err = U * (42 * A / s * w.abs() + y.abs() * (42 * A / s + 46))
    if bias is not None:
        y = y + one(bias)
        err = err + U * y.abs()
    if act != "none":
        err = SLOPE * err + 32 * U * y.abs()
        y = activation(act, y)
    return y, err


def rounded(y, err, dtype):
    return y, err + HALF[dtype] * 1.01 * (y.abs() + err)


def rows8(x):
    """The definition, bit by bit, on the host: int8 and float32 arrays of x [rows][features]."""
    v = x.detach().float().cpu().numpy()
    with np.errstate(all="ignore"):
        top = np.abs(v).max(1)
        bad = ~np.isfinite(v).all(1)
        tiny = top < np.float32(2.0 ** -100)
        scale = (top / np.float32(127)).astype(np.float32)
        inverse = (np.float32(127) / top).astype(np.float32)
        q = np.rint((v * inverse[:, None]).astype(np.float32))
    q[bad | tiny] = 0
    scale[tiny] = 0
    scale[bad] = np.nan
    return torch.from_numpy(q.astype(np.int8)), torch.from_numpy(scale)


def linear_i8(xq, xs, wq, ws, bias=None, act="none", gate=None, residual=None, dtype=torch.float32):
    """The sum is exact; its fp32 form and the two scales are three roundings, and the rest as block_reference.linear."""
    z = torch.mm(xq.double(), wq.double().t().contiguous()) * xs.double()[:, None] * ws.double()
    err = 3.01 * U * z.abs()
    if bias is not None:
        z = z + bias.double()
        err = err + U * (z.abs() + bias.double().abs())
    y = activation(act, z)
    if act != "none":
        err = SLOPE * err + 32 * U * z.abs()
    if gate is not None:
        y, err = y * gate.double(), err * gate.double().abs() + U * (y * gate.double()).abs()
    if residual is not None:
        err = err + U * (y.abs() + residual.double().abs())
        y = y + residual.double()
    return y, err + HALF[dtype] * 1.01 * (y.abs() + err)
