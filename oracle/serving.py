"""Plain CPU forms, in 64 bits, of what a serving loop adds to a scheduler step: scores of tokens, the attention mass of the keys, and
the eviction that goes by it.  Written from the definitions; test infrastructure only."""
from __future__ import annotations

import math

import torch


def token_scores(logits, token_id=None, suffix_len=None, num_alt=0):
    """-> (logprob, entropy, alt_id, alt_logprob); rows that are not active hold NaN / -2."""
    B, S, V = logits.shape
    logprob, entropy = torch.full((B, S), math.nan, dtype=torch.float64), torch.full((B, S), math.nan, dtype=torch.float64)
    alt_id, alt = torch.full((B, S, num_alt), -2, dtype=torch.int32), torch.full((B, S, num_alt), math.nan, dtype=torch.float64)
    for b in range(B):
        for i in range(S if suffix_len is None else int(suffix_len[b])):
            z = logits[b, i].double()
            d = z - z.max()     # (first: next to 3e38 a logarithm is lost in 64 bits too)
            lp = d - torch.logsumexp(d, 0) if z.max() > -math.inf else torch.full_like(z, -math.inf)
            p = lp.exp()
            entropy[b, i] = -(p[p > 0] * lp[p > 0]).sum()
            if token_id is not None:
                v = int(token_id[b, i])
                logprob[b, i] = lp[v] if 0 <= v < V else -math.inf
            order = torch.sort(z, descending=True, stable=True).indices[:num_alt]
            alt_id[b, i], alt[b, i] = -1, -math.inf
            alt_id[b, i, :len(order)], alt[b, i, :len(order)] = order.to(torch.int32), lp[order]
    return logprob if token_id is not None else None, entropy, alt_id, alt


def key_weights(q, k_suf, k_cache, prefix_len, suffix_len, weights, decay=1.0, scale=0.0):
    """One layer: weights [B,Hkv,C] after the step, in 64 bits."""
    B, S, Hq, D = q.shape
    Hkv, C = k_suf.shape[2], k_cache.shape[1]
    w, scale = weights.double().clone(), scale or 1 / math.sqrt(D)
    for b in range(B):
        P, N = min(max(int(prefix_len[b]), 0), C), min(max(int(suffix_len[b]), 0), S)
        if N == 0:
            continue
        for g in range(Hkv):
            k = torch.cat([k_cache[b, :P, g], k_suf[b, :N, g]]).double()
            mass = torch.zeros(P + N, dtype=torch.float64)
            for h in range(g * (Hq // Hkv), (g + 1) * (Hq // Hkv)):
                mass += torch.softmax(q[b, :N, h].double() @ k.T * scale, dim=1).sum(0)
            w[b, g, :P] = mass[:P] + (decay * w[b, g, :P] if decay else 0)
            w[b, g, P:P + N] = mass[P:min(P + N, C)]
    return w


BY_PLACE = -2 ** 31


def evict(weights, prefix_len, keep, high=None, first=0, recent=0, caches=(), positions=None, token_len=None):
    """weights [L,B,H,C]; caches: tensors [L,B,C,H,D], rows moved in place.  -> (new weights, new lengths, kept index).
    positions [L,B,H,C], updated in place, with token_len [B]: `recent` goes by them, and not by the places."""
    L, B, H, C = weights.shape
    high = keep if high is None else high
    new, length = weights.clone(), prefix_len.clone()
    index = torch.full((L, B, H, keep), -1, dtype=torch.int32)
    for b in range(B):
        P = min(max(int(prefix_len[b]), 0), C)
        length[b] = keep if P > high else P
        for l in range(L):
            for h in range(H):
                at = list(range(min(P, keep)))
                if P > high:
                    w = weights[l, b, h].tolist()
                    new_rows = set(range(P - recent, P))
                    if positions is not None:
                        T = int(token_len[b])
                        where = [T - (P - t) if p == BY_PLACE else p for t, p in enumerate(positions[l, b, h, :P].tolist())]
                        young = {t for t in range(first, P) if T - where[t] <= recent}
                        new_rows = young if len(young) <= keep - first else new_rows
                    free = sorted(set(range(first, P)) - new_rows, key=lambda t: (math.isnan(w[t]), -w[t], t))
                    stay = set(range(first)) | new_rows | set(free[:keep - first - len(new_rows)])
                    come = sorted(t for t in stay if t >= keep)
                    for hole, t in zip([t for t in range(keep) if t not in stay], come):
                        at[hole] = t
                    if positions is not None:
                        positions[l, b, h, :P] = torch.tensor([where[t] for t in at] + [BY_PLACE] * (P - keep), dtype=torch.int32)
                    for j, t in enumerate(at):
                        if j != t:
                            new[l, b, h, j] = weights[l, b, h, t]
                            for c in caches:
                                c[l, b, j, h] = c[l, b, t, h].clone()
                index[l, b, h, :len(at)] = torch.tensor(at, dtype=torch.int32)
    return new, length, index
