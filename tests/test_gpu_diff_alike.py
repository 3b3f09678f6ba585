"""Differential attention of maps that are nearly alike: what they share cancels, and an error of a map's weights stays while the
result shrinks.

Tolerance, of the 2-norm of all outputs' errors.  The output's rounding to bf16 is off by at most EB of the value, spread evenly:
EB / sqrt(3) in the mean square.  A weight goes to the product as two bf16 parts (off by EB^2 = 2^-16) from a score in 32 bits:
d products added one by one, each sum off by 2^-23 of at most their magnitudes' sum S: in the mean square sqrt(d) 2^-23 S / 2
(half of that sum has been added on average), times ln 2 log2(e) = 1.  The errors of different keys are independent, so a map's
output is off by tol sqrt(sum (weight V)^2) in the mean square; the norm multiplies that, and adds an error of the whole row no
larger than its own.  A quarter more for what a finite number of errors strays."""
import math

import pytest
import torch

import rope_diff_model as model
from test_gpu_diff import Setup
from test_gpu_rope import cu_of, randn

pytestmark = pytest.mark.gpu
pe = pytest.importorskip("paper_2609_04875_gb300")


def alike(lens, counts, hq, hkv, d, ps, c, seed, bits=16):
    """A cache whose kv-heads 2j + 1 are the heads 2j and noise of c times their size, and queries likewise."""
    s = Setup(lens, hkv, d, ps, seed=seed, bits=bits, outliers=0.0)
    K = s.K.float()
    K[:, :, 1::2] = K[:, :, 0::2] + c * K[:, :, 1::2]
    s.cache.crop_batch(s.seqs, [1] * len(lens))
    s.cache.append_kv_batch(s.seqs, K.to(torch.bfloat16), s.V, cu_of(lens))
    q = randn(s.g, sum(counts), hq, d).float()
    q[:, 1::2] = q[:, 0::2] + c * q[:, 1::2]
    return s, q.to(torch.bfloat16)


def tolerance(q, k, v, lam, gain, eps, group):
    """(sum of squares of the outputs, sum of squares of their expected errors)."""
    n, hq, d = q.shape
    T, scale = k.shape[0], d ** -0.5
    seen = torch.arange(T, device=q.device)[None] <= torch.arange(T - n, T, device=q.device)[:, None]
    size = err = 0.0
    for h in range(hq // 2):
        j = h // group
        val = torch.cat([v[:, 2 * j], v[:, 2 * j + 1]], dim=1)
        o = var = 0.0
        for m in range(2):
            s = (q[:, 2 * h + m] @ k[:, 2 * j + m].t() * scale).masked_fill(~seen, -math.inf)
            w = torch.softmax(s, dim=1)
            S = (q[:, 2 * h + m].abs() @ k[:, 2 * j + m].abs().t()) * scale
            tol = model.EB ** 2 + math.sqrt(d) * 2.0 ** -24 * S + 2.0 ** -20
            part = 1.0 if m == 0 else -lam[h]
            o = o + part * (w @ val)
            var = var + part ** 2 * ((w * tol) ** 2 @ val ** 2)
        r = 1.0 if gain is None else gain / torch.sqrt((o * o).mean(dim=1, keepdim=True) + eps)
        y, e = o * r, var * r * r * (1 if gain is None else 2)
        size += (y * y).sum().item()
        err += (e + (model.EB ** 2 / 3) * y * y).sum().item()
    return size, err


# lens, counts, hq, hkv, d, ps
CASES = [
    ([900], [1], 64, 2, 64, 16),
    ([6000], [4], 32, 4, 128, 16),
    ([12000, 700], [16, 16], 8, 2, 128, 64),
    ([500, 800], [60, 20], 4, 4, 64, 32),
    ([700], [300], 8, 4, 128, 16),
    ([3000], [200], 8, 2, 64, 16),
    ([515, 300], [515, 300], 4, 2, 128, 16),
    ([5000], [700], 8, 2, 128, 128),
]


@pytest.mark.parametrize("c,lam_", [(0.1, 0.8), (0.1, 0.95), (0.02, 0.8), (0.02, 0.95)])
@pytest.mark.parametrize("lens,counts,hq,hkv,d,ps", CASES)
def test_maps_alike(lens, counts, hq, hkv, d, ps, c, lam_):
    s, q = alike(lens, counts, hq, hkv, d, ps, c, seed=sum(lens) + hq)
    lam = torch.full((hq // 2,), lam_, device="cuda")
    gain = 0.2 * (1 + 0.1 * torch.randn(2 * d, generator=s.g, device="cuda"))
    cu = cu_of(counts)
    for g in (None, gain):
        out = s.cache.diff_attn_batch(s.seqs, 0, q, cu, lam, gain=g)
        off = size = err = 0.0
        for i, x in enumerate(s.seqs):
            a, b = cu[i], cu[i + 1]
            k, v = [t[0].double() for t in s.cache.read_kv(x)]
            gd = None if g is None else g.double()
            want, _ = model.diff_attention(q[a:b].double(), k, v, lam.double(), gd, 1e-5, d ** -0.5, hq // hkv)
            off += ((out[a:b].double() - want) ** 2).sum().item()
            more = tolerance(q[a:b].double(), k, v, lam.double(), gd, 1e-5, hq // hkv)
            size, err = size + more[0], err + more[1]
        off, tol = math.sqrt(off / size), 1.25 * math.sqrt(err / size)
        assert off <= tol, f"{'norm' if g is not None else 'no norm'}: {off:.2e} off in the 2-norm, {tol:.2e} allowed"


@pytest.mark.parametrize("n", [1, 50, 200])
def test_maps_alike_in_8_bits(n):
    s, q = alike([1000], [n], 16, 2, 64, 16, 0.02, seed=n, bits=8)
    lam, gain = torch.full((8,), 0.9, device="cuda"), torch.full((128,), 0.2, device="cuda")
    out = s.cache.diff_attn(s.seqs[0], 0, q, lam, gain=gain)
    k, v = [t[0].double() for t in s.cache.read_kv(s.seqs[0])]
    want, _ = model.diff_attention(q.double(), k, v, lam.double(), gain.double(), 1e-5, 0.125, 8)
    size, err = tolerance(q.double(), k, v, lam.double(), gain.double(), 1e-5, 8)
    off = ((out.double() - want) ** 2).sum().item()
    assert off <= 1.25 ** 2 * err, f"{math.sqrt(off / size):.2e} off, {1.25 * math.sqrt(err / size):.2e} allowed"
