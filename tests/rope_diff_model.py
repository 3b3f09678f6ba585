"""Position rotation and differential attention in 64 bits, from their definitions, and the errors that the kernels'
roundings allow.

A rounding to bf16 is off by at most 2^-8 of the value (EB), one to e4m3 by 2^-4 (E8)."""
import math

import torch

EB, E8 = 2.0 ** -8, 2.0 ** -4


def rotated(x, pos, freq, axis=None, interleaved=False, scale=1.0):
    """x [..][N][H][d], pos [axes][N] (integers).  Returns (value, bound on what 32 bits get wrong), fp64.  The angle errs by
    pi 2^-25 (its 32 bits as a float), cosine and sine by 2^-23 each, products and sums by 2^-24: below 2^-20 (|a| + |b|)."""
    x, n = x.double(), len(freq)
    axis = axis or [0] * n
    f = torch.tensor(freq, dtype=torch.float64, device=x.device)
    far = pos.abs().max().item() if pos.numel() else 0
    angle = (pos.double()[axis].t() * f)[:, None]           # [N][1][pairs]
    one, two = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    a, b, c, s = x[..., one], x[..., two], angle.cos(), angle.sin()
    y, e = x.clone(), torch.zeros_like(x)
    y[..., one], y[..., two] = scale * (a * c - b * s), scale * (b * c + a * s)
    e[..., one] = e[..., two] = abs(scale) * (a.abs() + b.abs()) * (2.0 ** -20 + 1e-15 * far)
    return y, e


def check_rotated(got, want, err):
    excess = (got.double() - want).abs() - (EB * want.abs() + err + 2.0 ** -134)
    assert (excess <= 0).all(), excess.max().item()


def page_scale(a):
    """2^e of pages whose largest magnitude is a, fp64: the least e >= -126 with a <= 448 2^e."""
    e = torch.ceil(torch.log2(a.clamp(min=2.0 ** -200) / 448))
    e = torch.where(a > 448 * torch.exp2(e), e + 1, torch.where(a <= 448 * torch.exp2(e - 1), e - 1, e))
    return torch.exp2(e.clamp(min=-126))


def diff_attention(q, k, v, lam, gain, eps, scale, group):
    """One sequence: q [n][Hq][d], its last n positions; k, v [T][Hkv][d]; all fp64.  Returns (out [n][Hq/2][2d], bound).

    What the kernel rounds: each weight to bf16 (EB), in the sum as in the product, so a map's output is off by at most
    2 EB times B = sum of weight |V|; the rest is in 32 bits (scores of a few hundred units in log2: 2^-14 of a weight at
    most); the output once."""
    n, hq, d = q.shape
    T = k.shape[0]
    seen = torch.arange(T, device=q.device)[None] <= torch.arange(T - n, T, device=q.device)[:, None]
    out = torch.empty((n, hq // 2, 2 * d), dtype=torch.float64, device=q.device)
    bound = torch.empty_like(out)
    for h in range(hq // 2):
        j = h // group
        val = torch.cat([v[:, 2 * j], v[:, 2 * j + 1]], dim=1)
        o, D = 0.0, 0.0
        for m in range(2):
            s = (q[:, 2 * h + m] @ k[:, 2 * j + m].t() * scale).masked_fill(~seen, -math.inf)
            w = torch.softmax(s, dim=1)
            part = 1.0 if m == 0 else -lam[h]
            # (what a row does not see has no part in it, whatever it is: 0 infinity is 0 here)
            clean = torch.nan_to_num(val, nan=0.0, posinf=0.0, neginf=0.0)
            odd = (seen.double() @ (~torch.isfinite(val)).double()) > 0
            o = o + part * torch.where(odd, torch.full_like(w @ clean, math.nan), w @ clean)
            D = D + abs(float(part)) * (2 * EB * 1.02 + 2.0 ** -13) * (w @ clean.abs())
        if gain is not None:
            r = 1.0 / torch.sqrt((o * o).mean(dim=1, keepdim=True) + eps)
            delta = (D * D).mean(dim=1, keepdim=True).sqrt() * r
            delta = torch.where(delta < 0.5, delta / (1 - delta), torch.full_like(delta, math.inf))
            D = gain.abs() * r * (D + (o.abs() + D) * delta)
            o = o * r * gain
        out[:, h], bound[:, h] = o, D + EB * (o.abs() + D) + 1e-30
    return out, bound


def check_diff(got, want, bound, what=""):
    got = got.double()
    nan = torch.isnan(want)
    assert not torch.isfinite(got[nan]).any(), f"{what}: a row that sees an infinity or NaN is finite"
    got, want, bound = got[~nan], want[~nan], bound[~nan]
    assert torch.isfinite(got).all(), f"{what}: not finite"
    excess = (got - want).abs() - bound
    assert excess.numel() == 0 or excess.max().item() <= 0, f"{what}: {excess.max().item():.3e} over the bound"
    if got.numel() > 4096:  # the roundings are independent: on average far below the bound
        off = ((got - want).norm() / want.norm()).item()
        assert off <= 2 * EB, f"{what}: {off:.2e} off in the 2-norm"
