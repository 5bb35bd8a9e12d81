"""Attention over a live cache in 64 bits, with windows and caches held in 8 bits, and how far a kernel may be from it.

A rounding to bf16 is off by at most 2^-8 of the value (half a step).  The kernels round queries and keys after their
rotation, weights before they meet the values, and the output once.  A score's two rounded factors move it by at most
e = (2 * 2^-8 + 2^-16) sum_d |q_d k_d| / sqrt(D), all weights together by a factor in [exp(-2e), exp(2e)]; so an output
moves by at most 2^-8 |o| + (2^-8 + expm1(2e)) sum_j p_j |v_j|, and fp32 sums add less than 1e-5 of the same.
"""
import math

import torch

THETA = 1.0e4


def rope(x, pos, rot, theta=THETA):
    """Rows x [n][heads][d] in 64 bits rotated at pos [n], pairs (i, i + rot / 2)."""
    half = rot // 2
    freq = theta ** (-2.0 * torch.arange(half, dtype=torch.float64, device=x.device) / max(rot, 1))
    ang = pos.double().to(x.device)[:, None, None] * freq
    a, b = x[..., :half], x[..., half:rot]
    return torch.cat([a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin(), x[..., rot:]], -1)


def in_sight(at, n_keys, window=0, n_sink=0):
    """[rows][n_keys]: which keys the rows at live indices `at` see."""
    at = torch.as_tensor(at).cuda()[:, None]
    j = torch.arange(n_keys, device="cuda")
    ok = j <= at
    if window:
        ok &= (j > at - window) | (j < n_sink)
    return ok


def attend(q, K, V, seen, rounded=2):
    """q [n][Hq][d], K, V [Hkv][keys][d] in 64 bits, seen [n][keys]: (outputs, how far each element may be off).  `rounded`: of a
    score's factors how many are rounded to bf16 on their way."""
    n, hq, d = q.shape
    g = hq // K.shape[0]
    want, off = torch.empty_like(q), torch.empty_like(q)
    u = 2.0 ** -8
    for h in range(hq):
        k, v = K[h // g], V[h // g]
        s = (q[:, h] @ k.T) / math.sqrt(d)
        p = torch.softmax(s.masked_fill(~seen, -math.inf), -1)
        e = ((1 + u) ** rounded - 1) * ((q[:, h].abs() @ k.abs().T) / math.sqrt(d) * seen).amax(-1, keepdim=True)
        want[:, h] = p @ v
        off[:, h] = u * want[:, h].abs() + (u + torch.expm1(2 * e) + 1e-5) * (p @ v.abs())
    return want, off


def inside(got, want, off, what=""):
    """Every element within its bound, and no row as a whole further off than the roundings' own size."""
    got = got.double()
    assert torch.isfinite(got).all(), what
    bad = (got - want).abs() > off + 1e-30
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), float(((got - want).abs() / (off + 1e-30)).max()))
    return float(torch.linalg.norm(got - want) / torch.linalg.norm(want).clamp(min=1e-300))
