"""Timed cases of the operators of a serving loop with a bounded cache: what a step says about its tokens
(`token_scores`), what its attention says about the cached rows (`attn_key_weights`), and the eviction that goes by it
(`kv_evict`).

Shapes are those of the repository's own workloads (an LLaDA-8B-like decoder: 32 layers, 32 heads of 128, vocabulary 126464; a
Dream-7B-like one: 28 query / 4 KV heads of 128, vocabulary 152064; a small fp32 configuration with 4 heads of 64) and values
between and below them; `draw` covers the same ranges at other sizes.

A decode loop keeps suffix buffers of S rows and shrinks the number of ACTIVE rows: `active` is the longest suffix left in the
batch, sequence b has N_b rows left (between half of `active` and `active`) and P_b = P + S - N_b rows in its cache.

Where `own` is false, `run` computes the operators in elementary torch operations, in 32 bits; where it is true, it makes the
library's calls.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda"
LLADA = dict(Hq=32, Hkv=32, D=128, dtype="bf16")
DREAM = dict(Hq=28, Hkv=4, D=128, dtype="bf16")
SMALL = dict(Hq=4, Hkv=4, D=64, dtype="f32")
LLADA_V, DREAM_V = 126464, 152064
NEG = float("-inf")


def listed():
    return [
        # the last position of one user's answer: launch, latency and the trip through one row
        dict(name="scores_one_row", kind="scores", B=1, S=1, active=1, V=LLADA_V, K=5, dtype="bf16"),
        # late in a batch's loop: a few rows left of large buffers, twenty alternatives (what serving interfaces offer)
        dict(name="scores_few_rows", kind="scores", B=4, S=256, active=37, V=LLADA_V, K=20, dtype="bf16"),
        # fp32 logits of a small vocabulary, odd sizes, ragged
        dict(name="scores_f32_odd", kind="scores", B=3, S=189, active=150, V=30001, K=8, dtype="f32"),
        # a large batch's whole suffixes at the larger vocabulary: the logits have to be read once
        dict(name="scores_large", kind="scores", B=8, S=1024, active=1024, V=DREAM_V, K=20, dtype="bf16"),
        # the smallest configuration: four fp32 heads of 64, one short prompt
        dict(name="weights_f32_tiny", kind="weights", layers=1, B=1, S=64, active=64, P=128, decay=1.0, **SMALL),
        # one layer with grouped KV heads, odd lengths, ragged batch
        dict(name="weights_gqa_ragged", kind="weights", layers=1, B=4, S=509, active=497, P=1021, decay=0.9, **DREAM),
        # long context: two products of every query with every key
        dict(name="weights_long", kind="weights", layers=1, B=8, S=1024, active=1024, P=4096, decay=1.0, **LLADA),
        # the end of a decode loop: a few rows left, the keys of several layers have to be read
        dict(name="weights_tail", kind="weights", layers=8, B=16, S=1024, active=21, P=512, decay=0.9, **LLADA),
        # one layer of grouped heads for one user: a selection's latency
        dict(name="evict_one_layer", kind="evict", layers=1, B=1, P=700, spread=0, keep=512, first=4, recent=64, Hkv=4, D=128, dtype="bf16"),
        # fp32 caches of odd lengths, some sequences below the mark at which rows leave
        dict(name="evict_f32_ragged", kind="evict", layers=4, B=5, P=1201, spread=500, keep=797, first=1, recent=33, Hkv=4, D=64, dtype="f32"),
        # all layers of one user's cache, cut back to the budget
        dict(name="evict_single", kind="evict", layers=32, B=1, P=1280, spread=0, keep=1024, first=4, recent=128, Hkv=32, D=128, dtype="bf16"),
        # a long batch
        dict(name="evict_long", kind="evict", layers=8, B=8, P=5120, spread=512, keep=4096, first=4, recent=256, Hkv=32, D=128, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["scores", "weights", "evict"])
    if kind == "scores":
        S = _log_int(rng, 1, 1024)
        return dict(kind=kind, B=_log_int(rng, 1, 8), S=S, active=S if rng.random() < 0.5 else _log_int(rng, 1, S),
                    V=rng.choice([LLADA_V, DREAM_V, _log_int(rng, 1024, DREAM_V)]), K=rng.choice([0, 1, 5, 20, rng.randint(2, 32)]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]) if S <= 512 else "bf16")
    if kind == "weights":
        model = rng.choice([LLADA, LLADA, DREAM, SMALL])
        S = _log_int(rng, 1, 256 if model is SMALL else 1024)
        c = dict(kind=kind, layers=rng.choice([1, 1, 4]), B=_log_int(rng, 1, 8), S=S, active=S if rng.random() < 0.5 else _log_int(rng, 1, S),
                 P=_log_int(rng, 32, 1024 if model is SMALL else 4096), decay=rng.choice([1.0, 0.9, 0.0]), **model)
        while work(c)["flops"] > 6e11:
            c.update(layers=1, B=max(1, c["B"] - 1), P=c["P"] - c["P"] // 8)
        return c
    model = rng.choice([dict(Hkv=32, D=128, dtype="bf16"), dict(Hkv=4, D=128, dtype="bf16"), dict(Hkv=4, D=64, dtype="f32")])
    keep = _log_int(rng, 32, 4096)
    more = _log_int(rng, 1, keep)
    c = dict(kind=kind, layers=rng.choice([1, 4, 16, 32]), B=_log_int(rng, 1, 8), P=keep + more, spread=rng.choice([0, rng.randint(0, more + keep // 2)]),
             keep=keep, first=rng.choice([0, 1, 4]), recent=rng.randint(0, keep // 4), **model)
    while c["layers"] * c["B"] * c["P"] * c["Hkv"] * c["D"] > 1.2e9:
        c["layers"] = max(1, c["layers"] // 2)
        c["B"] = max(1, c["B"] - 1)
    return c


# --------------------------------------------------------------------------- #
# inputs
# --------------------------------------------------------------------------- #
def _lengths(c):
    """(P_b, N_b) of every sequence; they belong to the case, not to the seed."""
    B = c["B"]
    if c["kind"] == "evict":        # sequence b is up to `spread` rows shorter than the longest
        r = random.Random(31 * B + 1009 * c["P"] + c["spread"])
        return [c["P"]] + [c["P"] - r.randint(0, c["spread"]) for _ in range(B - 1)], [0] * B
    S, act = c["S"], c["active"]
    if act >= S:
        return [c.get("P", 0)] * B, [S] * B
    r = random.Random(1000003 * B + 1009 * S + act)
    n = [act] + [r.randint((act + 1) // 2, act) for _ in range(B - 1)]
    return [c.get("P", 0) + S - x for x in n], n


def _dt(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def prepare(case, seed):
    c, g, dt = case, torch.Generator(device=DEV).manual_seed(seed), _dt(case)
    p, n = _lengths(c)
    s = dict(c, lens=torch.tensor([p, n], dtype=torch.int32, device=DEV))
    B = c["B"]
    if c["kind"] == "scores":
        S, V, K = c["S"], c["V"], c["K"]
        z = torch.randn((B, S, V), generator=g, device=DEV, dtype=dt).clamp_(max=5.0)
        ids = torch.randint(0, V, (B, S), generator=g, device=DEV)
        # a sure token at most positions, none at the others
        sure = torch.where(torch.rand((B, S), generator=g, device=DEV) < 0.7, 12.0, 0.0)
        z.scatter_add_(2, ids.unsqueeze(-1), sure.unsqueeze(-1).to(dt))
        rows = torch.cat([torch.arange(S)[:k] + b * S for b, k in enumerate(n)]).to(DEV)
        f, i = dict(device=DEV), dict(device=DEV, dtype=torch.int32)
        out = (torch.zeros((B, S), **f), torch.zeros((B, S), **f), torch.zeros((B, S, K), **i), torch.zeros((B, S, K), **f))
        s.update(logits=z, ids=ids.to(torch.int32), rows=rows, out=out if K else (*out[:2], None, None))
        return s
    L, Hkv, D = c["layers"], c["Hkv"], c["D"]
    if c["kind"] == "weights":
        S, Hq, C = c["S"], c["Hq"], c["P"] + c["S"]
        q = torch.randn((L, B, S, Hq, D), generator=g, device=DEV, dtype=dt)
        k, v = (torch.randn((L, B, S, Hkv, D), generator=g, device=DEV, dtype=dt) for _ in range(2))
        kc, vc = (torch.randn((L, B, C, Hkv, D), generator=g, device=DEV, dtype=dt) for _ in range(2))
        # what a few steps before this one left
        w = torch.rand((L, B, Hkv, C), generator=g, device=DEV) * (4.0 * Hq // Hkv * max(n) / (c["P"] + S))
        s.update(q=q, k=k, kc=kc, most=(max(p), max(n)), w=w,
                 layers_of=[list(t.unbind(0)) for t in (q, k, v, kc, vc, torch.zeros_like(q))])
        return s
    C, S = c["P"] + 16, 16
    k, v = (torch.zeros((L, B, S, Hkv, D), device=DEV, dtype=dt) for _ in range(2))
    kc, vc = (torch.randn((L, B, C, Hkv, D), generator=g, device=DEV, dtype=dt) for _ in range(2))
    # accumulated weights: a few rows have most of it
    w = torch.randn((L, B, Hkv, C), generator=g, device=DEV).mul_(1.5).exp_()
    s.update(kc=kc, vc=vc, w=w, new_w=torch.zeros_like(w), new_len=torch.zeros(B, dtype=torch.int32, device=DEV),
             kept=torch.zeros((L, B, Hkv, c["keep"]), dtype=torch.int32, device=DEV), most=max(p),
             layers_of=[list(t.unbind(0)) for t in (k, v, kc, vc)])
    return s


# --------------------------------------------------------------------------- #
# plain forms
# --------------------------------------------------------------------------- #
def _plain_scores(s):
    V, K, rows = s["V"], s["K"], s["rows"]
    logprob, entropy, alt_id, alt_logprob = s["out"]
    z = s["logits"].view(-1, V)[rows].float()
    ids = s["ids"].view(-1)[rows].long()
    m = z.max(-1, keepdim=True).values
    d = z - m
    e = d.exp()
    tot = e.sum(-1)
    log_tot = tot.log()
    logprob.view(-1)[rows] = torch.gather(d, 1, ids.unsqueeze(1)).squeeze(1) - log_tot
    entropy.view(-1)[rows] = log_tot - (e * d).sum(-1) / tot
    if K:
        # one whole number for an entry: its value's order above, its place below, so that ties go to the lowest index
        bits = z.view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7fffffff, bits)
        top = torch.topk((order.long() << 32) + (V - 1 - torch.arange(V, device=DEV)), K, dim=-1).values
        at = V - 1 - (top & 0xffffffff)
        alt_id.view(-1, K)[rows] = at.to(torch.int32)
        alt_logprob.view(-1, K)[rows] = torch.gather(d, 1, at) - log_tot.unsqueeze(1)
    return s["out"]


def _heads_first(t):
    """[L, B, T, H, D] -> [L, B, H, T, D], dense, in 32 bits."""
    return t.permute(0, 1, 3, 2, 4).float().contiguous()


def _scores_of(s):
    """Scaled scores of the batch's active queries (all heads of a group, one after the other) with its keys, [L, B, Hkv, G N, P + N], keys that are
    not there at -inf, and the rows that are there."""
    L, B, Hq, Hkv, D = s["layers"], s["B"], s["Hq"], s["Hkv"], s["D"]
    P, N = s["most"]
    q = _heads_first(s["q"][:, :, :N]).view(L, B, Hkv, Hq // Hkv * N, D)
    k = _heads_first(torch.cat([s["kc"][:, :, :P], s["k"][:, :, :N]], dim=2))
    z = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    there = torch.cat([torch.arange(P, device=DEV) < s["lens"][0].unsqueeze(1), torch.arange(N, device=DEV) < s["lens"][1].unsqueeze(1)], dim=1)
    z = torch.where(there[:, None, None, :], z, NEG)
    rows = (torch.arange(N, device=DEV) < s["lens"][1].unsqueeze(1)).repeat(1, Hq // Hkv)
    return z, rows[:, None, :, None]


def _taken_over(s, mass, w):
    """Cached rows add this step's mass to what is left of theirs; active rows, which may be cached next, begin with it."""
    P, N = s["most"]
    C = w.shape[-1]
    t = torch.arange(C, device=DEV)
    p, n = s["lens"][0].view(-1, 1, 1), s["lens"][1].view(-1, 1, 1)
    old = torch.nn.functional.pad(mass[..., :P], (0, C - P))
    u = (t - p).clamp(0, N - 1).expand(w.shape)
    new = torch.gather(mass[..., P:], -1, u)
    got = torch.where(t < p, old + (w * s["decay"] if s["decay"] else 0.0), torch.where(t < p + n, new, w))
    return torch.where(n > 0, got, w)


def _plain_weights(s):
    z, rows = _scores_of(s)
    e = (z - z.max(-1, keepdim=True).values).exp()
    mass = torch.where(rows, e / e.sum(-1, keepdim=True), 0.0).sum(-2)
    s["w"].copy_(_taken_over(s, mass, s["w"]))
    return s["w"]


def _plain_evict(s):
    L, B, H, keep, most = s["layers"], s["B"], s["Hkv"], s["keep"], s["most"]
    p = s["lens"][0].view(B, 1, 1)
    t = torch.arange(most, device=DEV)
    w = s["w"][..., :most]
    valid, leaves = t < p, p > keep
    safe = valid & ((t < s["first"]) | (t >= p - s["recent"]))
    best = torch.sort(torch.where(safe, math.inf, torch.where(valid, w, NEG)), dim=-1, descending=True, stable=True).indices[..., :keep]
    kept = torch.zeros((L, B, H, most), dtype=torch.bool, device=DEV).scatter_(-1, best, True)
    kept = torch.where(leaves, kept, valid)
    hole = leaves & ~kept[..., :keep]
    moved = leaves & kept[..., keep:]
    m = min(keep, most - keep)
    none = most     # (sorts behind every row)
    src = torch.sort(torch.where(moved, t[keep:], none), dim=-1).values[..., :m]
    dst = torch.sort(torch.where(hole, t[:keep], none), dim=-1).values[..., :m]
    # the n-th hole takes the n-th row from behind
    if m:
        comes = torch.gather(src, -1, (hole.cumsum(-1) - 1).clamp(0, m - 1))
        index = torch.where(hole, comes, t[:keep])
        a, b = torch.where(src < none, src, keep), torch.where(dst < none, dst, keep)     # nothing more to move: a row behind onto itself
        l, q, h = torch.arange(L, device=DEV).view(L, 1, 1, 1), torch.arange(B, device=DEV).view(B, 1, 1), torch.arange(H, device=DEV).view(H, 1)
        s["kc"][l, q, b, h] = s["kc"][l, q, a, h]
        s["vc"][l, q, b, h] = s["vc"][l, q, a, h]
    else:
        index = t[:keep].expand(L, B, H, keep)
    s["kept"].copy_(torch.where(t[:keep] < p, index, -1))
    s["new_w"][..., :keep] = torch.where(t[:keep] < p, torch.gather(w, -1, index), s["new_w"][..., :keep])
    behind = valid[..., keep:] & ~leaves
    s["new_w"][..., keep:most] = torch.where(behind, w[..., keep:], s["new_w"][..., keep:most])
    s["new_len"].copy_(s["lens"][0].clamp(max=keep))
    return dict(new_len=s["new_len"], kept=s["kept"], new_w=s["new_w"], kc=s["kc"], vc=s["vc"])


def run(state):
    s, kind = state, state["kind"]
    if not own:
        return {"scores": _plain_scores, "weights": _plain_weights, "evict": _plain_evict}[kind](s)
    import paper_2603_05454_amd as lsp
    if kind == "scores":
        return lsp.token_scores(s["logits"], s["ids"], s["lens"][1], num_alt=s["K"], out=s["out"])
    if kind == "weights":
        if s["layers"] == 1:
            q, k, _, kc, _, _ = s["layers_of"]
            return lsp.attn_key_weights(q[0], k[0], kc[0], s["lens"][0], s["lens"][1], s["w"][0], decay=s["decay"]).unsqueeze(0)
        table = lsp.AttnLayerTable(*s["layers_of"])
        return lsp.attn_key_weights_layers(table, s["lens"][0], s["lens"][1], s["w"], decay=s["decay"])
    table = lsp.LayerTable(*s["layers_of"])
    lsp.kv_evict(s["w"], s["lens"][0], table, keep=s["keep"], first=s["first"], recent=s["recent"], new_weights=s["new_w"], new_len=s["new_len"],
                 kept_index=s["kept"])
    return dict(new_len=s["new_len"], kept=s["kept"], new_w=s["new_w"], kc=s["kc"], vc=s["vc"])


# --------------------------------------------------------------------------- #
# the definitions in 64 bits, and what a pass cannot do without
# --------------------------------------------------------------------------- #
def exact(case, seed):
    if case["kind"] == "evict":     # whole numbers and copies: nothing is computed
        return None
    s = prepare(case, seed)
    if case["kind"] == "weights":
        w, group, decay = s["w"].double(), s["Hq"] // s["Hkv"], s["decay"]
        for l in range(s["layers"]):
            for b, (p, n) in enumerate(zip(*_lengths(case))):
                q = s["q"][l, b, :n].double().view(n, s["Hkv"], group, -1).permute(1, 2, 0, 3).flatten(1, 2)
                k = torch.cat([s["kc"][l, b, :p], s["k"][l, b, :n]]).double().permute(1, 2, 0).contiguous()
                mass = torch.softmax(q.contiguous() @ k / math.sqrt(s["D"]), dim=-1).sum(1)
                w[l, b, :, :p] = mass[:, :p] + (decay * w[l, b, :, :p] if decay else 0.0)
                w[l, b, :, p:p + n] = mass[:, p:]
        return w
    B, S, V, K, rows = s["B"], s["S"], s["V"], s["K"], s["rows"]
    x = s["logits"].reshape(B * S, V).index_select(0, rows).double()
    lp = torch.log_softmax(x, dim=1)
    del x
    logprob, entropy, alt = torch.zeros(B * S, device=DEV).double(), torch.zeros(B * S, device=DEV).double(), torch.zeros(B * S, K, device=DEV).double()
    logprob[rows] = lp.gather(1, s["ids"].reshape(-1)[rows].long()[:, None])[:, 0]
    if K:
        alt[rows] = lp.topk(K, dim=1).values
    entropy[rows] = -(lp.exp().mul_(lp)).sum(1)
    return (logprob.view(B, S), entropy.view(B, S), None, alt.view(B, S, K) if K else None)


def work(case):
    c = case
    es = 4.0 if c["dtype"] == "f32" else 2.0
    p, n = _lengths(c)
    if c["kind"] == "scores":       # every entry: a difference, an exponential, two sums
        return dict(bytes=sum(n) * (c["V"] * es + 12.0 + 8.0 * c["K"]), flops=sum(n) * c["V"] * 5.0)
    L, Hkv, D = c["layers"], c["Hkv"], c["D"]
    if c["kind"] == "weights":      # Q, K and the weights read, the weights written; the product of every query with every key
        rows = sum(n)
        keys = sum(a + b for a, b in zip(p, n))
        flops = L * sum(2.0 * c["Hq"] * b * (a + b) * D for a, b in zip(p, n))
        return dict(bytes=L * (es * D * (rows * c["Hq"] + keys * Hkv) + 4.0 * Hkv * (keys + sum(p) * (c["decay"] > 0))), flops=flops)
    nbytes = 0.0
    for a in p:
        nbytes += 8.0 * Hkv * min(a, c["keep"]) + 4.0 * Hkv * a         # index and weights written, weights read
        if a > c["keep"]:           # rows that leave lie anywhere in the part that is not protected: those below `keep` are holes
            free = a - c["first"] - c["recent"]
            holes = (a - c["keep"]) * min(1.0, max(0, min(c["keep"], a - c["recent"]) - c["first"]) / free)
            nbytes += 4.0 * Hkv * holes * D * es                        # K and V, read and written
    return dict(bytes=L * nbytes, flops=0)
