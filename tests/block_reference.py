"""Plain 64-bit forms of a block's operators and the error bounds that the tests hold the kernels to.

Every reference takes torch tensors on any device and returns (value, bound), both float64: the operator's
definition evaluated in 64 bits, and how far a result may be off given which roundings the kernels make.
u = 2^-24 is fp32's half step, relative to the value; bf16's is 2^-8 (finfo.eps / 2).
"""
import math

import torch

U = 2.0 ** -24
HALF = {torch.float64: 2.0 ** -53, torch.float32: U, torch.bfloat16: 2.0 ** -8}


def positions(ids, N, device):
    ids = torch.as_tensor([int(i) for i in ids], device=device)
    return (ids[:, None] * N + torch.arange(N, device=device)[None, :]).reshape(-1)


def rotary(x, ids, H, W, dims, theta=(10000.0,) * 3, origin=(0.0,) * 3, step=(1.0,) * 3, halves=False, inverse=False):
    """x: compact rows [M*H*W][heads][d]. The angle is reduced in double and rounded to fp32 as a half turn in
    [-1, 1] (pi u at most), sine and cosine are then off by 2 of their last places (4 u) at most, and the two
    products and their sum by 2 u more: (|a| + |b|) (pi + 4 + 2) u. Then one rounding to the type."""
    N, dev = H * W, x.device
    tok = torch.arange(N, device=dev)
    y = x.double().clone()
    R = sum(dims)
    size = y.abs()
    bound = torch.zeros_like(y)
    pair = 0
    for a in range(3):
        for j in range(dims[a] // 2):
            freq = theta[a] ** (-2.0 * j / dims[a])
            lo, hi = (pair, pair + R // 2) if halves else (2 * pair, 2 * pair + 1)
            pair += 1
            for m, f in enumerate(ids):
                index = (torch.full_like(tok, int(f)), tok // W, tok % W)[a].double()
                phi = (origin[a] + step[a] * index) * freq * (-1.0 if inverse else 1.0)
                c, s = phi.cos()[:, None], phi.sin()[:, None]
                r = slice(m * N, (m + 1) * N)
                p, q = x[r, :, lo].double(), x[r, :, hi].double()
                y[r, :, lo], y[r, :, hi] = p * c - q * s, p * s + q * c
                bound[r, :, lo] = bound[r, :, hi] = (size[r, :, lo] + size[r, :, hi]) * 10 * U
    # dimensions past R pass as they are
    turned = torch.zeros(x.shape[2], dtype=torch.bool, device=dev)
    turned[:R] = True
    bound = bound + turned * y.abs() * HALF[x.dtype] * 1.01
    return y, bound


def cross(q, k, v, lengths=None, mask=None):
    """A score is a sum of d products in fp32, off by d u sum |q k| / sqrt(d), the softmax's argument by 4 u of the
    largest score more; e^x and its argument's rounding add 8 u. In bf16 each probability is rounded (2^-8) and the
    sum adds the rounded ones. An error of e in every weight moves the mean of v by e sum w |v - out| at most, twice
    that for weights over their sum. Sums over n keys: n u. Then one rounding to the type."""
    B, Lq, heads, d = q.shape
    Lk, group = k.shape[1], heads // k.shape[2]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(out)
    half = HALF[q.dtype]
    for b in range(B):
        n = Lk if lengths is None else max(0, min(Lk, int(lengths[b])))
        keys = torch.arange(n, device=q.device)
        if mask is not None:
            keys = keys[mask[b][:n].to(q.device) != 0]
        if keys.numel() == 0:
            continue
        for h in range(heads):
            kk, vv = k[b, :, h // group].double()[keys], v[b, :, h // group].double()[keys]
            qq = q[b, :, h].double()
            s = torch.mm(qq, kk.t().contiguous()) / math.sqrt(d)
            w = torch.softmax(s, -1)
            o = torch.mm(w, vv)
            spread = torch.mm(w, vv.abs()) + o.abs()
            score_err = d * U * torch.mm(qq.abs(), kk.abs().t().contiguous()).amax(1, keepdim=True) / math.sqrt(d)
            e = 2 * (score_err + 4 * U * s.abs().amax(1, keepdim=True) + 8 * U) + (keys.numel() + d) * U
            if q.dtype == torch.bfloat16:
                e = e + half
            out[b, :, h] = o
            bound[b, :, h] = e * spread + half * o.abs() * 1.01
    return out, bound


def activation(name, z):
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z / math.sqrt(2.0)))
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def linear(x, w, bias=None, act="none", gate=None, residual=None):
    """x, gate and residual: the product's own rows (gate may be one row). A sum of K products in fp32 is off by K u
    sum |x w|; the activations' slopes are at most 1.13; the activation itself is worth 32 u |z| (its exponential's
    argument and the quotients) and the rest of the epilogue 4 u of its terms. Then one rounding to the type."""
    z = torch.mm(x.double(), w.double().t().contiguous())
    err = (x.shape[1] + 2) * U * torch.mm(x.double().abs(), w.double().abs().t().contiguous())
    if bias is not None:
        z = z + bias.double()
        err = err + U * (z.abs() + bias.double().abs())
    y = activation(act, z)
    if act != "none":
        err = 1.13 * err + 32 * U * z.abs()
    if gate is not None:
        y, err = y * gate.double(), err * gate.double().abs() + U * (y * gate.double()).abs()
    if residual is not None:
        err = err + U * (y.abs() + residual.double().abs())
        y = y + residual.double()
    return y, err + HALF[x.dtype] * 1.01 * y.abs()


def assert_within(got, want, bound, what=""):
    """Every element within its bound (a subnormal rounding besides)."""
    got = got.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert bool(torch.isfinite(got).all()), f"{what}: not finite"
    over = (got - want).abs() - bound - 1e-38
    worst = float(over.max()) if over.numel() else 0.0
    if worst > 0:
        at = int(over.reshape(-1).argmax())
        raise AssertionError(f"{what}: element {at} is {float(got.reshape(-1)[at])}, {float(want.reshape(-1)[at])} "
                             f"within {float(bound.reshape(-1)[at])}; {int((over > 0).sum())} of {over.numel()} are over")
