"""What finch_rotate, finch_quantize and finch_attend compute, written out in 64 bits on the CPU, with the bounds that
a correct 32-bit calculation keeps (tests only; no code in common with the library)."""
from __future__ import annotations

import math

import torch

# a rounding is off by half a step at most, relative to the value
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def host(t):
    return t.detach().cpu().to(torch.float64)


def attention(q, k, v, causal):
    """q [n][G][d], k and v [N][d] (any type) -> out [n][G][d], lse [G][n] in 64 bits, and per output the sum of weights times |v|
    and per row the largest sum |q_c k_c| / sqrt(d) of a key."""
    q, k, v = host(q), host(k), host(v)
    n, G, d = q.shape
    N = k.shape[0]
    out, mag = torch.zeros(n, G, d, dtype=torch.float64), torch.zeros(n, G, d, dtype=torch.float64)
    lse, size = torch.full((G, n), -math.inf, dtype=torch.float64), torch.zeros(G, n, dtype=torch.float64)
    for i in range(n):
        sees = max(0, min(N, N - n + i + 1)) if causal else N
        if sees == 0:
            continue
        for g in range(G):
            s = k[:sees] @ q[i, g] / math.sqrt(d)
            z = torch.logsumexp(s, 0)
            w = torch.exp(s - z)
            out[i, g], mag[i, g] = w @ v[:sees], w @ v[:sees].abs()
            lse[g, i] = z
            size[g, i] = (k[:sees].abs() @ q[i, g].abs()).max() / math.sqrt(d)
    return out, lse, mag, size


def check_attention(got, got_lse, q, k, v, causal, what):
    """Bounds, per element.  A logit is a sum of d products (error d * 2^-24 of the sum of their sizes, S) times a rounded factor;
    its exponential and the difference from the reference add 4 * 2^-24 * S * log2(e) and a few 2^-23: weights are off by
    e = 2^-24 * ((d + 8) * S * 1.5 + 16) of themselves, N of them summed one after the other by N * 2^-24 more, and both sums
    count.  bf16: weights are rounded once (2^-8), and so is the output."""
    want, lse, mag, size = attention(q, k, v, causal)
    n, G, d = q.shape
    N = k.shape[0]
    e = 2.0 ** -24 * ((d + 8) * size * 1.5 + 16)            # [G][n]
    rel = (2 * e + 2 * (N + 32) * 2.0 ** -24).T[..., None]  # [n][G][1]
    half = HALF[q.dtype]
    if q.dtype == torch.bfloat16:
        rel = rel + half
    off = (host(got) - want).abs()
    bound = rel * mag + half * (want.abs() + rel * mag) + 1e-30
    assert torch.isfinite(host(got)).all(), f"{what}: not finite"
    worst = float((off / bound).max()) if off.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3g} times the bound"
    if got_lse is not None:
        g = host(got_lse).view(G, n)
        empty = torch.isinf(lse)
        assert torch.equal(torch.isinf(g), empty) and bool((g[empty] < 0).all()), f"{what}: lse of empty rows"
        far = ((g - lse).abs()[~empty] / (e + (N + 32) * 2.0 ** -24 + 2.0 ** -22 * lse.abs())[~empty])
        assert far.numel() == 0 or float(far.max()) <= 1.0, f"{what}: lse {float(far.max()):.3g} times the bound"
    return worst


def rotated(x, pos, pairing, dims, freq, gain, weight, eps):
    """x [n][heads][d] -> the same rows after norm and rotation, and the size of what each element was made of."""
    y = host(x)
    if weight is not None:
        y = y / torch.sqrt(y.square().mean(2, keepdim=True) + eps) * host(weight)
    size = y.abs().clone()
    if pairing:
        a = torch.tensor(pos, dtype=torch.float64)[:, None] * torch.tensor(freq, dtype=torch.float64)[None]
        c, s = gain * torch.cos(a)[:, None], gain * torch.sin(a)[:, None]
        u, w = (slice(0, dims // 2), slice(dims // 2, dims)) if pairing == 1 else (slice(0, dims, 2), slice(1, dims, 2))
        p, q = y[..., u].clone(), y[..., w].clone()
        y[..., u], y[..., w] = p * c - q * s, q * c + p * s
        size[..., u] = size[..., w] = abs(gain) * (p.abs() + q.abs())
    return y, size


def check_rotated(got, x, pos, pairing, dims, freq, gain, weight, eps, what):
    """The norm's sum of d squares is off by d * 2^-24 of itself, its root by half of that, a few roundings beside it; sine and
    cosine by 2^-22, and their products and the sum by 4 * 2^-24: together under 2^-24 * (d / 2 + 24) of the parts' sizes;
    one rounding of the result."""
    want, size = rotated(x, pos, pairing, dims, freq, gain, weight, eps)
    d = x.shape[2]
    bound = 2.0 ** -24 * (d / 2 + 24) * size
    bound = bound + HALF[x.dtype] * (want.abs() + bound) + 1e-37
    worst = float(((host(got) - want).abs() / bound).max()) if want.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3g} times the bound"


def e4m3_table():
    """Values of the bytes 0 .. 126."""
    t = [((1 + (b & 7) / 8) * 2.0 ** ((b >> 3) - 7) if b >> 3 else (b & 7) / 8 * 2.0 ** -6) for b in range(127)]
    return torch.tensor(t, dtype=torch.float64)


def e4m3_values(b):
    b = b.detach().cpu().view(torch.uint8).long()
    v = torch.cat([e4m3_table(), torch.tensor([math.nan], dtype=torch.float64)])[b & 127]
    return torch.where(b >= 128, -v, v)


def quantized(x, block):
    """[n][d] -> values without the powers of two [n][d], exponents per block."""
    x = host(x)
    n = x.shape[0]
    got, exps, t = torch.zeros_like(x), [], e4m3_table()
    for b in range(0, n, block):
        y = x[b:b + block]
        top = float(y.abs().max())
        e = 0
        if top > 0:
            e = -100
            while math.ldexp(448.0, e) < top:
                e += 1
        y = y * math.ldexp(1.0, -e)
        hi = torch.searchsorted(t, y.abs()).clamp(max=126)
        lo = (hi - 1).clamp(min=0)
        up, down = t[hi] - y.abs(), y.abs() - t[lo]
        pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
        got[b:b + block] = torch.where(y < 0, -t[pick], t[pick])
        exps.append(e)
    return got, exps


def dequantized(rows, scale, block):
    v = e4m3_values(rows)
    e = scale.detach().cpu().long()[torch.arange(rows.shape[0]) // block]
    return v * torch.pow(torch.tensor(2.0, dtype=torch.float64), (e - 127).double())[:, None]
