"""Timed cases of the operators of a cache that is held in 8 bits: norms and rotation of a step's queries and keys (`qk_norm_rope`),
the committed rows quantised as they are written and read back (`kv_append_q8`, `kv_read_q8`), and the attention over such a
cache (`attn_step_q8`).

Shapes are those of the repository's own workloads (an LLaDA-8B-like decoder: 32 layers, 32 heads of 128; a Dream-7B-like one: 28
query / 4 KV heads of 128; a small configuration with 4 heads of 64) and values between and around them; `draw` covers the same
ranges at other sizes.

A cache row is e4m3 values; 32 rows of one head (rows 32 j to 32 j + 31) share an exponent byte E and stand for e4m3 * 2^(E - 127). E is
the smallest with which the largest magnitude of the block is at most 448 * 2^(E - 127), from 1 to 246; where rows are added to a
block that has some, it keeps the larger of both and what is there is rounded again.

Where `own` is false, `run` computes the operators in elementary torch operations, in 32 bits; where it is true, it makes the
library's calls.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda"
BLOCK = 32
LLADA = dict(Hq=32, Hkv=32, D=128, dtype="bf16")
DREAM = dict(Hq=28, Hkv=4, D=128, dtype="bf16")
SMALL = dict(Hq=4, Hkv=4, D=64, dtype="f32")
SMALL16 = dict(SMALL, dtype="bf16")
NEG = float("-inf")


def listed():
    return [
        # one user, one layer of grouped heads: the last position of a denoising step goes into the cache; latency
        dict(name="append_one_row", kind="append", layers=1, B=1, P=700, spread=0, new=1, S=64, **DREAM),
        # the commit of one step of a batch, all layers
        dict(name="append_step", kind="append", layers=32, B=8, P=1500, spread=400, new=64, S=256, **LLADA),
        # fp32 projections of small heads, odd lengths, blocks that are partly there
        dict(name="append_f32_odd", kind="append", layers=4, B=5, P=1201, spread=77, new=333, S=501, **SMALL),
        # prompts: everything is new, written once and read back once
        dict(name="append_prompt", kind="append", layers=2, B=4, P=0, spread=0, new=4096, S=4096, **LLADA),
        # the last position of one user's answer
        dict(name="attn_one_row", kind="attn", layers=1, B=1, S=1, active=1, P=700, **DREAM),
        # the end of a batch's decode loop: a few rows left, all keys of several layers have to be read
        dict(name="attn_tail", kind="attn", layers=8, B=16, S=1024, active=21, P=512, **LLADA),
        # few rows on long documents
        dict(name="attn_long_cache", kind="attn", layers=1, B=4, S=16, active=16, P=32768, **LLADA),
        # one layer with grouped KV heads, odd lengths, ragged batch
        dict(name="attn_gqa_ragged", kind="attn", layers=1, B=4, S=509, active=497, P=1021, **DREAM),
        # a long batch's first step: two products of every query with every key
        dict(name="attn_full", kind="attn", layers=1, B=8, S=1024, active=1024, P=4096, **LLADA),
        # rotation alone (a decoder without norms of heads), one row far into a document
        dict(name="rope_one_row", kind="rope", B=1, S=1, active=1, P=100003, R=128, norm=False, interleaved=False, **DREAM),
        # small fp32 heads, half of each head rotated, neighbours paired, ragged
        dict(name="rope_f32_partial", kind="rope", B=5, S=203, active=190, P=777, R=32, norm=True, interleaved=True, **SMALL),
        # norms and rotation of a long batch's step
        dict(name="rope_full", kind="rope", B=8, S=1024, active=1024, P=4096, R=128, norm=True, interleaved=False, **LLADA),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "attn", "attn", "rope"])
    if kind == "append":
        model = rng.choice([LLADA, DREAM, SMALL, SMALL16])
        P = rng.choice([0, _log_int(rng, 1, 4096)])
        new = _log_int(rng, 1, 2048)
        c = dict(kind=kind, layers=rng.choice([1, 1, 4, 32]), B=_log_int(rng, 1, 8), P=P, spread=rng.randint(0, P // 2), new=new,
                 S=new + rng.choice([0, rng.randint(1, 300)]), **model)
        while c["layers"] * c["B"] * max(c["S"], c["new"] + BLOCK, c["P"] // 4) * c["Hkv"] * c["D"] > 1.2e8:
            c["layers"] = max(1, c["layers"] // 2)
            c["B"] = max(1, c["B"] - 1)
            if c["layers"] == c["B"] == 1:
                break
        return c
    if kind == "rope":
        model = rng.choice([LLADA, DREAM, SMALL, SMALL16])
        S = _log_int(rng, 1, 1024)
        return dict(kind=kind, B=_log_int(rng, 1, 8), S=S, active=S if rng.random() < 0.5 else _log_int(rng, 1, S), P=_log_int(rng, 1, 200000),
                    R=rng.choice([model["D"], model["D"], model["D"] // 2, 16]), norm=rng.random() < 0.6, interleaved=rng.random() < 0.3, **model)
    model = rng.choice([LLADA, LLADA, DREAM, DREAM, SMALL16])
    S = _log_int(rng, 1, 1024)
    c = dict(kind=kind, layers=rng.choice([1, 1, 4]), B=_log_int(rng, 1, 8), S=S, active=S if rng.random() < 0.5 else _log_int(rng, 1, S),
             P=_log_int(rng, 16, 32768 if S <= 64 else 4096), **model)
    while work(c)["flops"] > 6e11 or work(c)["bytes"] > 1e9:
        c.update(layers=1, B=max(1, c["B"] - 1), P=c["P"] - c["P"] // 8)
    return c


# --------------------------------------------------------------------------- #
# inputs
# --------------------------------------------------------------------------- #
def _lengths(c):
    """Cached and active rows of every sequence (append: cached rows before and new ones); they belong to the case, not to the seed."""
    B = c["B"]
    if c["kind"] == "append":
        r = random.Random(31 * B + 1009 * c["P"] + 7 * c["spread"] + c["new"])
        p = [c["P"]] + [c["P"] - r.randint(0, c["spread"]) for _ in range(B - 1)]
        return p, [c["new"]] + [r.randint((c["new"] + 1) // 2, c["new"]) if c["spread"] else c["new"] for _ in range(B - 1)]
    S, act = c["S"], c["active"]
    if act >= S:
        return [c["P"]] * B, [S] * B
    r = random.Random(1000003 * B + 1009 * S + act)
    n = [act] + [r.randint((act + 1) // 2, act) for _ in range(B - 1)]
    return [c["P"] + S - x for x in n], n


def _read_back(c):
    """First and last row of what is read back: from the beginning of the first block that was written to."""
    p, n = _lengths(c)
    return [a // BLOCK * BLOCK for a in p], [a + b for a, b in zip(p, n)]


def _dt(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _projection(shape, g, dt):
    """Keys or values: some dimensions are larger than others."""
    loud = torch.randn(shape[-2:], generator=g, device=DEV).mul_(0.5).exp_()
    return torch.randn(shape, generator=g, device=DEV).mul_(loud).to(dt)


def _blocks(x, C):
    """[..., C, H, D] -> [..., blocks, BLOCK, H, D], padded with zeros."""
    pad = -C % BLOCK
    x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, pad)) if pad else x
    return x.unflatten(-3, (-1, BLOCK))


def _exponent(amax):
    """The smallest e with amax <= 448 * 2^e, from -126 to 119."""
    m, x = torch.frexp(amax)
    e = torch.where(m > 0.875, x - 8, x - 9)
    return torch.where(amax == 0, -126, e).clamp(-126, 119)


def _pow2(e):
    """2^e in 32 bits, e from -126 to 127."""
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _round8(x):
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _cache(shape, g):
    """A cache that holds rows of a projection: values [B, C, H, D] and exponent bytes [B, H, blocks]."""
    B, C, H, D = shape
    x = _blocks(_projection(shape, g, torch.bfloat16).float(), C)
    e = _exponent(x.abs().amax((2, 4)))                                 # [B, blocks, H]
    q = _round8(x * _pow2(-e)[:, :, None, :, None]).flatten(1, 2)[:, :C].contiguous()
    return q, (e + 127).to(torch.uint8).transpose(1, 2).contiguous()


def _caches(c, C, g):
    made = [[_cache((c["B"], C, c["Hkv"], c["D"]), g) for _ in range(c["layers"])] for _ in range(2)]
    kc, vc = (torch.stack([a.view(torch.uint8) for a, _ in m]).view(torch.float8_e4m3fn) for m in made)
    return kc, vc, *(torch.stack([e for _, e in m]) for m in made)


def prepare(case, seed):
    c, g, dt = case, torch.Generator(device=DEV).manual_seed(seed), _dt(case)
    p, n = _lengths(c)
    B, S, Hq, Hkv, D = c["B"], c["S"], c["Hq"], c["Hkv"], c["D"]
    s = dict(c, lens=torch.tensor([p, n], dtype=torch.int32, device=DEV), p=p, n=n)
    if c["kind"] == "rope":
        q, k = _projection((B, S, Hq, D), g, dt), _projection((B, S, Hkv, D), g, dt)
        R = c["R"]
        inv_freq = torch.pow(torch.tensor(500000.0, dtype=torch.float64), -torch.arange(0, R, 2, dtype=torch.float64) / R).float().to(DEV)
        w = [1 + 0.3 * torch.randn(D, generator=g, device=DEV) for _ in range(2)] if c["norm"] else [None, None]
        s.update(q=q, k=k, inv_freq=inv_freq, q_weight=w[0], k_weight=w[1], out=(torch.zeros_like(q), torch.zeros_like(k)))
        return s
    L = c["layers"]
    C = c["P"] + (c["new"] if c["kind"] == "append" else S) + 13
    k, v = (_projection((L, B, S, Hkv, D), g, dt) for _ in range(2))
    kc, vc, ke, ve = _caches(c, C, g)
    s.update(k=k, v=v, kc=kc, vc=vc, ke=ke, ve=ve, C=C)
    layers_of = [list(t.unbind(0)) for t in (k, v, kc, vc, ke, ve)]
    if c["kind"] == "append":
        first, end = _read_back(c)
        R = max(b - a for a, b in zip(first, end))
        outs = [torch.zeros((L, B, R, Hkv, D), dtype=dt, device=DEV) for _ in range(2)]
        s.update(outs=outs, outs_of=[list(t.unbind(0)) for t in outs], after=s["lens"].sum(0, dtype=torch.int32),
                 rows=torch.tensor([first, end], dtype=torch.int32, device=DEV))
    else:
        q = torch.randn((L, B, S, Hq, D), generator=g, device=DEV).to(dt)
        out = torch.zeros_like(q)
        s.update(q=q, out=out, q_of=list(q.unbind(0)), out_of=list(out.unbind(0)))
    s["layers_of"] = layers_of
    return s


# --------------------------------------------------------------------------- #
# plain forms
# --------------------------------------------------------------------------- #
def _values(q, e, first, end):
    """Rows first..end of a cache [L, C, H, D] with exponents [L, H, blocks], in 32 bits."""
    scale = _pow2(e.to(torch.int32) - 127).transpose(1, 2)
    block = torch.arange(first, end, device=DEV) // BLOCK
    return q[:, first:end].float() * scale[:, block, :, None]


def _plain_append(s):
    first, end = _read_back(s)
    for new, q, e, out in ((s["k"], s["kc"], s["ke"], s["outs"][0]), (s["v"], s["vc"], s["ve"], s["outs"][1])):
        for b, (p, n) in enumerate(zip(s["p"], s["n"])):
            a, z = first[b], end[b]
            x = torch.cat([_values(q[:, b], e[:, b], a, p), new[:, b, :n].float()], dim=1)
            fresh = _blocks(torch.cat([torch.zeros_like(x[:, :p - a]), x[:, p - a:]], dim=1), z - a)
            exps = _exponent(fresh.abs().amax((2, 4)))                   # [L, blocks, H]
            j = a // BLOCK
            if p > a:       # rows from before in the first block
                exps[:, 0] = torch.maximum(exps[:, 0], e[:, b, :, j].to(torch.int32) - 127)
            x8 = _round8(_blocks(x, z - a) * _pow2(-exps)[:, :, None, :, None]).flatten(1, 2)[:, :z - a]
            q.view(torch.uint8)[:, b, a:z] = x8.contiguous().view(torch.uint8)
            e[:, b, :, j:j + exps.shape[1]] = (exps + 127).to(torch.uint8).transpose(1, 2)
            out[:, b, :z - a] = _values(q[:, b], e[:, b], a, z).to(out.dtype)
    return dict(k=s["outs"][0], v=s["outs"][1], ke=s["ke"], ve=s["ve"])


def _plain_attn(s):
    group = s["Hq"] // s["Hkv"]
    P, N = max(s["p"]), max(s["n"])
    lens = s["lens"]
    there = torch.cat([torch.arange(P, device=DEV) < lens[0].unsqueeze(1), torch.arange(N, device=DEV) < lens[1].unsqueeze(1)], dim=1)
    rows = torch.arange(N, device=DEV) < lens[1].unsqueeze(1)
    block = torch.arange(P, device=DEV) // BLOCK
    for l in range(s["layers"]):
        def keys(q, e, new):      # [B, Hkv, P + N, D]
            scale = _pow2(e.to(torch.int32) - 127)[:, :, block].unsqueeze(-1)
            return torch.cat([q[:, :P].float().transpose(1, 2) * scale, new[:, :N].float().transpose(1, 2)], dim=2)
        k, v = keys(s["kc"][l], s["ke"][l], s["k"][l]), keys(s["vc"][l], s["ve"][l], s["v"][l])
        q = s["q"][l, :, :N].float().unflatten(2, (s["Hkv"], group)).permute(0, 2, 3, 1, 4).flatten(2, 3).contiguous()   # [B, Hkv, group N, D]
        z = torch.matmul(q, k.transpose(-1, -2).contiguous()) * (1.0 / math.sqrt(s["D"]))
        z = torch.where(there[:, None, None, :], z, NEG)
        z = (z - z.max(-1, keepdim=True).values).exp_()
        o = torch.matmul(z, v) / z.sum(-1, keepdim=True)
        o = o.unflatten(2, (group, N)).permute(0, 3, 1, 2, 4).flatten(2, 3)
        to = s["out"][l, :, :N]
        to.copy_(torch.where(rows[:, :, None, None], o.to(to.dtype), to))
    return s["out"]


def _plain_rope(s):
    S, R, D = s["S"], s["R"], s["D"]
    u = torch.arange(S, device=DEV)
    rows = (u < s["lens"][1].unsqueeze(1))[:, :, None, None]
    angle = (s["lens"][0].unsqueeze(1) + u).double().unsqueeze(-1) * s["inv_freq"].double()
    cos, sin = angle.cos().float().unsqueeze(2), angle.sin().float().unsqueeze(2)
    for x, w, to in ((s["q"], s["q_weight"], s["out"][0]), (s["k"], s["k_weight"], s["out"][1])):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6) * w
        if s["interleaved"]:
            a, b = y[..., 0:R:2], y[..., 1:R:2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
        else:
            a, b = y[..., :R // 2], y[..., R // 2:R]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
        y = torch.cat([turned, y[..., R:]], dim=-1) if R < D else turned
        to.copy_(torch.where(rows, y.to(to.dtype), to))
    return s["out"]


def run(state):
    s, kind = state, state["kind"]
    if not own:
        return {"append": _plain_append, "attn": _plain_attn, "rope": _plain_rope}[kind](s)
    import paper_2603_05454_amd as lsp
    if kind == "rope":
        return lsp.qk_norm_rope(s["q"], s["k"], s["inv_freq"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6, prefix_len=s["lens"][0],
                                suffix_len=s["lens"][1], interleaved=s["interleaved"], out=s["out"])
    if kind == "append":
        table = lsp.Q8LayerTable(*s["layers_of"])
        lsp.kv_append_q8(table, s["lens"][1], s["after"])
        lsp.kv_read_q8(table, s["rows"][0], s["rows"][1], *s["outs_of"])
        return dict(k=s["outs"][0], v=s["outs"][1], ke=s["ke"], ve=s["ve"])
    if s["layers"] == 1:
        k, v, kc, vc, ke, ve = (t[0] for t in s["layers_of"])
        lsp.attn_step_q8(s["q_of"][0], k, v, kc, vc, ke, ve, s["lens"][0], s["lens"][1], out=s["out_of"][0])
        return s["out"]
    table = lsp.Q8LayerTable(*s["layers_of"], q=s["q_of"], out=s["out_of"])
    lsp.attn_step_q8_layers(table, s["lens"][0], s["lens"][1])
    return s["out"]


# --------------------------------------------------------------------------- #
# the definitions in 64 bits, and what a pass cannot do without
# --------------------------------------------------------------------------- #
def _unit(e):
    """2^e in 64 bits, from a table (an exponential may be a rounding off)."""
    return torch.tensor([2.0 ** k for k in range(-160, 160)], dtype=torch.float64, device=DEV)[e.long() + 160]


def _nearest8(x):
    """The e4m3 value nearest to each (ties to even), in 64 bits: three bits behind the first, steps of 2^-9 below 2^-6."""
    x = x.clamp(-448.0, 448.0)
    _, e = torch.frexp(x.abs().clamp_min(2.0 ** -6))
    step = _unit(e - 4)
    return torch.round(x / step) * step


def _exact_append(case, seed):
    s = prepare(case, seed)
    first, end = _read_back(case)
    got = []
    for new, q, e, out in ((s["k"], s["kc"], s["ke"], s["outs"][0]), (s["v"], s["vc"], s["ve"], s["outs"][1])):
        res = torch.zeros(out.shape, dtype=torch.float64, device=DEV)
        for b in range(case["B"]):
            p, n = s["p"][b], s["n"][b]
            for a in range(first[b], end[b], BLOCK):
                z = min(a + BLOCK, end[b])
                x = new[:, b, max(a, p) - p:z - p].double()
                most = x.abs().amax((1, 3)).clamp_min(1e-37) / 448.0
                E = torch.ceil(torch.log2(most))                # (a logarithm may be a rounding off at powers of two)
                E = (E + (most > _unit(E)).double() - (most <= _unit(E - 1)).double()).clamp(-126, 119)
                if p > a:
                    was = e[:, b, :, a // BLOCK].double() - 127.0
                    E = torch.maximum(E, was)
                    x = torch.cat([q[:, b, a:p].double() * _unit(was)[:, None, :, None], x], dim=1)
                unit = _unit(E)[:, None, :, None]
                res[:, b, a - first[b]:z - first[b]] = _nearest8(x / unit) * unit
        got.append(res)
    return dict(k=got[0], v=got[1], ke=None, ve=None)


def exact(case, seed):
    if case["kind"] == "append":
        return _exact_append(case, seed)
    s = prepare(case, seed)
    if case["kind"] == "attn":
        group, out = s["Hq"] // s["Hkv"], torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
        for l in range(s["layers"]):
            for b, (p, n) in enumerate(zip(s["p"], s["n"])):
                for h in range(s["Hkv"]):
                    k, v = (torch.cat([t[l, b, :p, h].double() * _unit(e[l, b, h].long() - 127).repeat_interleave(BLOCK)[:p, None],
                                       x[l, b, :n, h].double()]) for t, e, x in ((s["kc"], s["ke"], s["k"]), (s["vc"], s["ve"], s["v"])))
                    for m in range(h * group, (h + 1) * group):
                        w = torch.softmax(s["q"][l, b, :n, m].double() @ k.T.contiguous() / math.sqrt(s["D"]), dim=-1)
                        out[l, b, :n, m] = w @ v
        return out
    R, res = s["R"], []
    pair = torch.arange(R // 2, device=DEV)
    one, two = (2 * pair, 2 * pair + 1) if s["interleaved"] else (pair, pair + R // 2)
    for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        y = torch.zeros(x.shape, dtype=torch.float64, device=DEV)
        for b, (p, n) in enumerate(zip(s["p"], s["n"])):
            row = x[b, :n].double()
            if w is not None:
                row = row / ((row ** 2).mean(-1, keepdim=True) + 1e-6).sqrt() * w.double()
            z = torch.polar(torch.ones(n, R // 2, dtype=torch.float64, device=DEV), torch.outer(torch.arange(p, p + n, device=DEV).double(), s["inv_freq"].double()))
            turned = torch.complex(row[..., one], row[..., two]) * z.unsqueeze(1)
            row = row.clone()
            row[..., one], row[..., two] = turned.real, turned.imag
            y[b, :n] = row
        res.append(y)
    return tuple(res)


def work(case):
    c = case
    es = 4.0 if c["dtype"] == "f32" else 2.0
    p, n = _lengths(c)
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    if c["kind"] == "rope":         # queries and keys read and written
        return dict(bytes=sum(n) * (Hq + Hkv) * D * 2 * es + 2.0 * c["R"], flops=sum(n) * (Hq + Hkv) * (3.0 * c["R"] + (4.0 * D if c["norm"] else 0.0)))
    L = c["layers"]
    if c["kind"] == "append":       # new rows read, rows of 8 bits (those of the first block that are there) read or written, all read back
        first, end = _read_back(c)
        rows = sum(b - a for a, b in zip(first, end))
        old = sum(a - f for a, f in zip(p, first))
        return dict(bytes=2.0 * L * Hkv * D * (sum(n) * (es + 1.0) + old + rows * es), flops=2.0 * L * Hkv * D * (sum(n) * 3.0 + rows))
    # queries read, the result written, the cache in 8 bits, the suffix's keys and values; two products of every query with every key
    nbytes = sum(2.0 * es * b * Hq * D + 2.0 * Hkv * D * (a * (1.0 + 1.0 / (BLOCK * D)) + b * es) for a, b in zip(p, n))
    return dict(bytes=L * nbytes, flops=L * sum(4.0 * Hq * b * (a + b) * D for a, b in zip(p, n)))
