"""The calls of caches in 8 bits together, as a decoder makes them, and in decode_loop."""
import pytest
import torch

import workloads as W
from oracle import eight_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsp():
    import paper_2603_05454_amd as m
    assert torch.cuda.is_available()
    return m


def _work(G=96, P=40, D=64):
    return W.scaled(W.C5, B=3, S=G, V=4096, P=P, gen_len=G, C=P + G + 20, layers=2, Hq=4, Hkv=2, D=D)


def _start(lsp, w):
    """Sequences whose prompts are in caches of both kinds: the plain ones are what was quantised."""
    pl, sl = (t.cuda() for t in W.make_lengths(w))
    plain = [{k: v.cuda() for k, v in W.make_layer_kv(w, l).items()} for l in range(w.layers)]
    eight = []
    for L in plain:
        kc, vc, ke, ve = lsp.q8_cache(w.B, w.C, w.Hkv, w.D)
        lsp.kv_append_q8(lsp.Q8LayerTable([L["k_cache"]], [L["v_cache"]], [kc], [vc], [ke], [ve]), pl, pl)
        eight.append(dict(q=L["q"], k_suf=L["k_suf"], v_suf=L["v_suf"], k_cache=kc, v_cache=vc, k_scale=ke, v_scale=ve))
    return dict(bitmap=W.make_delimiters(w)[1].cuda(), prefix_len=pl, suffix_len=sl, tokens=W.make_tokens(w, w.C).cuda(), plain=plain, eight=eight)


def _loop(w, s, kv, **kw):
    from paper_2603_05454_amd.loop import decode_loop
    fn = lambda step, p: W.make_logits(w, step=step, prefix_len=p.cpu())[0].cuda()      # noqa: E731
    return decode_loop(fn, s["bitmap"], w.V, w.tau, w.window, 1, 1, s["prefix_len"], s["suffix_len"], s["tokens"], kv_layers=kv, gen_len=w.gen_len, **kw)


def _caches(kv):
    return [L[k].cpu().view(torch.uint8) for L in kv for k in ("k_cache", "v_cache", "k_scale", "v_scale")]


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_loop(lsp, graph, D):
    """Tokens and lengths are those of plain caches (logits are the caller's); the caches what appending every step's rows leaves, byte for byte; the
    attention that of the caches before each step's rows."""
    import paper_2603_05454_amd.loop as loop
    w = _work(D=D)
    s, plain = _start(lsp, w), _start(lsp, w)
    want = [[[L[f"{x}_suf"].cpu(), L[f"{x}_cache"].cpu().double(), L[f"{x}_scale"].cpu()] for x in "kv"] for L in s["eight"]]
    before = [s["prefix_len"].cpu().clone(), s["suffix_len"].cpu().clone()]
    seen, tables = [], []

    def attend(table, prefix_len, suffix_len, workspace=None):
        tables.append(table)
        return lsp.attn_step_q8_layers(table, prefix_len, suffix_len, workspace=workspace)

    def observer(step, z, conf, out):
        P, N = before
        if step in (0, 1, 7):
            for l, L in enumerate(want):
                q = s["eight"][l]["q"].cpu()
                o, mass = eight_bits.attention(q, L[0][0], L[1][0], *[eight_bits.values(x[1], x[2]) for x in L], P, N)
                got = tables[0].out[l].cpu().double()
                for b in range(w.B):
                    n = int(N[b])
                    # the bound of the call's own test
                    assert ((got[b, :n] - o[b, :n]).abs() <= (2.0 ** -8 + 2.0 ** -12) * mass[b, :n] + 2.0 ** -8 * o[b, :n].abs()).all()
        count, P = out["commit_len"].cpu(), s["prefix_len"].cpu()
        for L in want:
            for x in L:
                x[1], e = eight_bits.append(x[0], x[1], x[2], count, P)
                x[2] = e.to(torch.uint8)
        before[0], before[1] = P.clone(), s["suffix_len"].cpu().clone()
        seen.append(count.clone())
    keep = loop.attn_step_q8_layers
    loop.attn_step_q8_layers = attend
    try:
        res = _loop(w, s, s["eight"], run_attention=True, graph=graph, observer=observer)
    finally:
        loop.attn_step_q8_layers = keep
    ref = _loop(w, plain, plain["plain"], run_attention=True, graph=graph)
    assert res["steps"] == ref["steps"] == len(seen) > 8 and res["flips"] == ref["flips"] and res["committed"] == int(sum(seen).sum())
    assert all(torch.equal(s[k], plain[k]) for k in ("prefix_len", "suffix_len", "tokens")) and s["suffix_len"].max() == 0
    for l, L in enumerate(s["eight"]):
        for x, (_, val, scale) in zip("kv", want[l]):
            assert torch.equal(L[f"{x}_cache"].cpu().double(), val) and torch.equal(L[f"{x}_scale"].cpu(), scale)


def test_loop_stopped_and_resumed_with_scores(lsp):
    w = _work()
    whole, parts = _start(lsp, w), _start(lsp, w)
    scores = [dict(logprob=torch.full((w.B, w.C), 7.0, device="cuda")) for _ in range(2)]
    a = _loop(w, whole, whole["eight"], run_attention=True, scores=scores[0])
    r = _loop(w, parts, parts["eight"], stop_after=4, scores=scores[1])
    b = _loop(w, parts, parts["eight"], state=r["state"], run_attention=True, graph=True, scores=scores[1])
    assert a["steps"] == b["steps"] and a["flips"] == b["flips"] and torch.equal(scores[0]["logprob"], scores[1]["logprob"])
    assert all(torch.equal(x, y) for x, y in zip(_caches(whole["eight"]), _caches(parts["eight"])))


def test_loop_refusals(lsp):
    w = _work()
    s = _start(lsp, w)

    def refused(word, kv, **kw):
        before = [s[k].clone() for k in ("prefix_len", "suffix_len", "tokens")]
        caches = _caches(s["eight"])
        with pytest.raises(lsp.LspError, match=word):
            _loop(w, s, kv, **kw)
        assert all(torch.equal(a, s[k]) for a, k in zip(before, ("prefix_len", "suffix_len", "tokens")))
        assert all(torch.equal(a, b) for a, b in zip(caches, _caches(s["eight"])))
    eight = s["eight"]
    refused("not cut back", eight, run_attention=True, cache_budget=dict(keep=64))
    refused("come together", [{k: v for k, v in L.items() if k != "v_scale"} for L in eight])
    refused("come together", [eight[0], s["plain"][1]])
    refused("v_cache|e4m3|float8", [{**L, "v_cache": s["plain"][0]["v_cache"]} for L in eight])
    refused("rows for token buffers", [dict(L, **dict(zip(("k_cache", "v_cache", "k_scale", "v_scale"), lsp.q8_cache(w.B, w.C - 1, w.Hkv, w.D)))) for L in eight])
    refused("sequences for", [{k: v[:2] for k, v in L.items()} for L in eight])
    refused("bf16|bfloat16|dtype", [{k: v.float() if k in ("q", "k_suf", "v_suf") else v for k, v in L.items()} for L in eight], run_attention=True)


def test_a_decoder_s_step(lsp):
    """A step of a small decoder: heads normed and rotated, attention over the cache, the output head, the commit, its rows quantised; every call's result
    against its definition on what the call before it left.  Then the same from one captured graph, and the bytes are the same."""
    w = _work(P=37, D=128)
    B, S, H, Hkv, D, V = w.B, w.S, w.Hq, w.Hkv, w.D, w.V
    g = torch.Generator().manual_seed(4)
    raw = [torch.randn((w.layers, B, S, h, D), generator=g).to(torch.bfloat16).cuda() for h in (H, Hkv, Hkv)]
    weights = [(1 + 0.1 * torch.randn(D, generator=g)).cuda() for _ in range(2)]
    inv = (10000.0 ** (-torch.arange(0, D, 2) / D)).float().cuda()
    head = (torch.randn((V, H * D), generator=g) / 8).to(torch.bfloat16).cuda()
    bitmap = W.make_delimiters(w)[1].cuda()

    def fresh():
        s = _start(lsp, w)
        kv = s["eight"]
        s["table"] = lsp.Q8LayerTable([torch.zeros_like(raw[1][0]) for _ in kv], list(raw[2].unbind(0)), *[[L[k] for L in kv] for k in
                                      ("k_cache", "v_cache", "k_scale", "v_scale")], q=[torch.zeros_like(raw[0][0]) for _ in kv],
                                      out=[torch.zeros_like(raw[0][0]) for _ in kv])
        s["ws"] = torch.zeros(max(16, lsp.attn_q8_workspace_bytes(B, S, H, Hkv, D, w.C, w.layers)), dtype=torch.uint8, device="cuda")
        s["cws"] = torch.zeros(lsp.lm_head_confidence_workspace_bytes(B, S, V), dtype=torch.uint8, device="cuda")
        s["conf"] = s["commit"] = None
        return s

    def heads(s):
        t = s["table"]
        for l in range(w.layers):
            lsp.qk_norm_rope(raw[0][l], raw[1][l], inv, q_weight=weights[0], k_weight=weights[1], prefix_len=s["prefix_len"], suffix_len=s["suffix_len"],
                             out=(t.keep[6][l], t.keep[0][l]))

    def rest(s):
        lsp.attn_step_q8_layers(s["table"], s["prefix_len"], s["suffix_len"], workspace=s["ws"])
        s["conf"] = lsp.lm_head_confidence(s["table"].out[-1].view(B, S, H * D), head, s["suffix_len"], out=s["conf"], workspace=s["cws"])
        s["commit"] = lsp.commit(s["conf"][2], s["conf"][0], bitmap, V, 0.02, w.window, 2, 1, s["prefix_len"], s["suffix_len"], tokens=s["tokens"],
                                 C=w.C, out=s["commit"])
        lsp.kv_append_q8(s["table"], s["commit"]["commit_len"], s["prefix_len"])

    s, steps = fresh(), 6
    for step in range(steps):
        P, N = s["prefix_len"].cpu(), s["suffix_len"].cpu()
        heads(s)
        t = s["table"]
        val = [[x.cpu() for x in lst] for lst in t.keep[2:6]]
        for l in range(w.layers):
            want = eight_bits.norm_rope(raw[0][l].cpu(), raw[1][l].cpu(), inv.cpu(), *[x.cpu() for x in weights], prefix_len=P, suffix_len=N)
            for got, (ref, size) in zip((t.keep[6][l], t.keep[0][l]), want):
                for b in range(B):
                    n = int(N[b])     # the bound of the call's own test
                    assert ((got.cpu().double()[b, :n] - ref[b, :n]).abs() <= 21 * 2.0 ** -24 * size[b, :n] + 2.0 ** -8 * ref[b, :n].abs() + 1e-30).all()
        rest(s)
        n, P1 = s["commit"]["commit_len"].cpu(), s["prefix_len"].cpu()
        assert torch.equal(P1, P + n) and torch.equal(s["suffix_len"].cpu(), N - n) and n.max() > 0
        for l in range(w.layers):
            k_suf, v_suf, q = t.keep[0][l].cpu(), t.keep[1][l].cpu(), t.keep[6][l].cpu()
            o, mass = eight_bits.attention(q, k_suf, v_suf, eight_bits.values(val[0][l], val[2][l]), eight_bits.values(val[1][l], val[3][l]), P, N)
            got = t.out[l].cpu().double()
            for b in range(B):
                a = int(N[b])
                assert ((got[b, :a] - o[b, :a]).abs() <= (2.0 ** -8 + 2.0 ** -12) * mass[b, :a] + 2.0 ** -8 * o[b, :a].abs()).all()
            for x, suf, c, e in (("k", k_suf, 2, 4), ("v", v_suf, 3, 5)):
                v, scale = eight_bits.append(suf, val[c - 2][l].double(), val[e - 2][l], n, P1)
                assert torch.equal(t.keep[c][l].cpu().double(), v) and torch.equal(t.keep[e][l].cpu().long(), scale), (step, l, x)

    # eagerly once (workspaces and outputs are there then), and from a graph
    one, two = fresh(), fresh()
    for x in (one, two):
        heads(x)
        rest(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        heads(two)
        rest(two)
    for _ in range(steps - 1):
        heads(one)
        rest(one)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(one[k], two[k]) for k in ("prefix_len", "suffix_len", "tokens"))
        assert all(torch.equal(a, b) for a, b in zip(_caches(one["eight"]), _caches(two["eight"])))
    assert torch.equal(one["tokens"], s["tokens"]) and all(torch.equal(a, b) for a, b in zip(_caches(one["eight"]), _caches(s["eight"])))


def test_loop_refuses_suffix_buffers_that_lack_rows(lsp):
    """Rows that a step commits have to be there to be appended."""
    w = _work()
    s = _start(lsp, w)
    kept = [s[k].clone() for k in ("prefix_len", "suffix_len", "tokens")]
    for attend in (False, True):
        with pytest.raises(lsp.LspError, match="rows for logits"):
            _loop(w, s, [{k: v[:, :w.S - 1] if k in ("q", "k_suf", "v_suf") else v for k, v in L.items()} for L in s["eight"]], run_attention=attend)
    assert all(torch.equal(a, s[k]) for a, k in zip(kept, ("prefix_len", "suffix_len", "tokens")))
