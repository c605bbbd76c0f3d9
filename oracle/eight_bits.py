"""Plain CPU forms, in 64 bits, of a cache in 8 bits, of the attention over it, and of the norms and rotation before it.  Written from the
definitions; test infrastructure only."""
from __future__ import annotations

import math

import torch

BLOCK = 32


def nearest(x):
    """The nearest e4m3 value (ties to even) of each number, largest magnitude 448; NaN for what is not finite."""
    def one(v):
        if not math.isfinite(v):
            return math.nan
        step = 2.0 ** max(math.frexp(v)[1] - 4, -9)     # three bits behind the first; 2^-9 below 2^-6
        return math.copysign(min(abs(round(v / step) * step), 448.0), v)
    return torch.tensor([one(v) for v in x.double().flatten().tolist()], dtype=torch.float64).view(x.shape)


def exponent(x):
    """The smallest E, from 1 to 246, with which no finite number is above 448 * 2^(E - 127)."""
    most = max([abs(v) for v in x.double().flatten().tolist() if math.isfinite(v)], default=0.0)
    E = 1
    while E < 246 and most > 448.0 * 2.0 ** (E - 127):
        E += 1
    return E


def append(suf, cache, scale, count, prefix_len):
    """suf [B,S,H,D], cache e4m3 [B,C,H,D], scale [B,H,blocks] -> (e4m3 values in 64 bits, scales), new tensors."""
    val, scale = cache.double().clone(), scale.clone().to(torch.int64)
    B, S, H, _ = suf.shape
    for b in range(B):
        P = min(max(int(prefix_len[b]), 0), cache.shape[1])
        n = min(max(int(count[b]), 0), S, P)
        for g in range(H):
            for j in range((P - n) // BLOCK, -(-P // BLOCK) if n else 0):
                a, z = max(j * BLOCK, P - n), min((j + 1) * BLOCK, P)
                new = suf[b, a - (P - n):z - (P - n), g].double()
                E = exponent(new)
                if a > j * BLOCK:
                    old = int(scale[b, g, j])
                    if E > old:
                        val[b, j * BLOCK:a, g] = nearest(val[b, j * BLOCK:a, g] * 2.0 ** (old - E))
                    E = max(E, old)
                val[b, a:z, g] = nearest(new * 2.0 ** (127 - E))
                scale[b, g, j] = E
    return val, scale


def values(val, scale):
    """What a cache stands for, in 64 bits."""
    E = scale.to(torch.int64).repeat_interleave(BLOCK, dim=2)[:, :, :val.shape[1]]
    return val.double() * torch.pow(torch.tensor(2.0, dtype=torch.float64), (E - 127).double()).transpose(1, 2).unsqueeze(-1)


def attention(q, k_suf, v_suf, k_val, v_val, prefix_len, suffix_len, scale=0.0):
    """k_val, v_val [B,C,Hkv,D]: what the cached rows stand for.  -> (out, the same sum of |v|), NaN in rows that are not active."""
    B, S, Hq, D = q.shape
    rep = Hq // k_suf.shape[2]
    out, mass = (torch.full(q.shape, math.nan, dtype=torch.float64) for _ in range(2))
    for b in range(B):
        P, N = min(max(int(prefix_len[b]), 0), k_val.shape[1]), min(max(int(suffix_len[b]), 0), S)
        for h in range(Hq if N else 0):
            k, v = (torch.cat([c[b, :P, h // rep], x[b, :N, h // rep].double()]) for c, x in ((k_val, k_suf), (v_val, v_suf)))
            p = torch.softmax(q[b, :N, h].double() @ k.T * (scale or 1 / math.sqrt(D)), dim=1)
            out[b, :N, h], mass[b, :N, h] = p @ v, p @ v.abs()
    return out, mass


def norm_rope(q, k, inv_freq, q_weight=None, k_weight=None, eps=1e-6, prefix_len=None, suffix_len=None, positions=None, interleaved=False):
    """-> (q, k, and for each the sum of the magnitudes that an element is made of); NaN in rows that are not active."""
    B, S, _, D = q.shape
    half = inv_freq.shape[0]
    pos = torch.arange(S).expand(B, S).double() if prefix_len is None else prefix_len.view(B, 1).double() + torch.arange(S)
    if positions is not None:
        pos = positions.double()
    angle = pos.unsqueeze(-1) * inv_freq.double()
    c, s = angle.cos().unsqueeze(2), angle.sin().unsqueeze(2)
    at = torch.arange(half)
    one, two = (2 * at, 2 * at + 1) if interleaved else (at, at + half)
    res = []
    for x, w in ((q, q_weight), (k, k_weight)):
        y = x.double()
        if w is not None:
            y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * w.double()
        z, size = y.clone(), y.abs()
        z[..., one], z[..., two] = y[..., one] * c - y[..., two] * s, y[..., two] * c + y[..., one] * s
        size[..., one] = size[..., two] = y[..., one].abs() + y[..., two].abs()
        if suffix_len is not None:
            for b in range(B):
                z[b, max(int(suffix_len[b]), 0):] = math.nan
        res.append((z, size))
    return res
