"""A cache that is cut back step after step keeps the newest tokens, whatever their weights: rows carry their tokens' positions."""
import pytest
import torch

import workloads as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsp():
    import paper_2603_05454_amd as m
    assert torch.cuda.is_available()
    return m


def _work(G=96, P=40):
    return W.scaled(W.C5, B=3, S=G, V=4096, P=P, gen_len=G, C=P + G + 20, layers=2, Hq=4, Hkv=2, D=64, dtype="f32")


def _start(w):
    """V of cached row t holds t."""
    pl, sl = (t.cuda() for t in W.make_lengths(w))
    kv = [{k: v.cuda() for k, v in W.make_layer_kv(w, l).items()} for l in range(w.layers)]
    for layer in kv:
        layer["v_cache"].copy_(torch.arange(w.C, device="cuda").view(1, -1, 1, 1).float().expand_as(layer["v_cache"]))
    return dict(bitmap=W.make_delimiters(w)[1].cuda(), prefix_len=pl, suffix_len=sl, tokens=W.make_tokens(w, w.C).cuda(), kv_layers=kv)


def _loop(w, s, **kw):
    """The denoiser writes V of suffix row i as its token's position."""
    from paper_2603_05454_amd.loop import decode_loop

    def fn(step, p):
        for layer in s["kv_layers"]:
            at = p.view(-1, 1) + torch.arange(w.S, device="cuda")
            layer["v_suf"].copy_(at.float()[:, :, None, None].expand_as(layer["v_suf"]))
        return W.make_logits(w, step=step, prefix_len=p.cpu())[0].cuda()
    return decode_loop(fn, s["bitmap"], w.V, w.tau, w.window, 1, 1, s["prefix_len"], s["suffix_len"], s["tokens"], kv_layers=s["kv_layers"],
                       gen_len=w.gen_len, run_attention=True, **kw)


def _held(s, cache_len):
    """(prefix_len, positions held) of every layer, sequence and head."""
    for b, (n, t) in enumerate(zip(cache_len.tolist(), s["prefix_len"].tolist())):
        for layer in s["kv_layers"]:
            for h in range(layer["v_cache"].shape[2]):
                at = layer["v_cache"][b, :n, h, 0].cpu().long().tolist()
                assert len(set(at)) == n
                yield t, set(at)


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("keep,high,first,recent,decay", [(44, None, 2, 8, 1.0), (44, None, 0, 44, 1.0), (44, 50, 2, 8, 0.9), (44, 47, 0, 20, 0.5),
                                                          (30, None, 30, 0, 1.0), (45, 60, 5, 40, 1.0)])
def test_the_newest_tokens_stay(lsp, graph, keep, high, first, recent, decay):
    w = _work()
    s = _start(w)
    cache_len = s["prefix_len"].clone()
    steps = []

    def observer(step, z, conf, out):
        steps.append(step)
        for t, held in _held(s, cache_len):
            assert held >= set(range(max(t - recent, 0), t)) | set(range(first)), (step, t, sorted(held))
    res = _loop(w, s, graph=graph, observer=observer, cache_budget=dict(keep=keep, high=high, first=first, recent=recent, decay=decay, cache_len=cache_len))
    assert len(steps) > 20 and s["suffix_len"].max() == 0 and (res["cache_len"] <= (high or keep)).all()


def _calls(lsp, w, m, lens, budget):
    """The loop's calls one by one, every choice against the definition.  -> weights, positions, cache_len."""
    from oracle import serving
    L, kv = w.layers, m["kv_layers"]
    cols = {k: [x[k] for x in kv] for k in kv[0]}
    attn = lsp.AttnLayerTable(cols["q"], cols["k_suf"], cols["v_suf"], cols["k_cache"], cols["v_cache"], [torch.zeros_like(q) for q in cols["q"]])
    table = lsp.LayerTable(cols["k_suf"], cols["v_suf"], cols["k_cache"], cols["v_cache"])
    weights = torch.zeros((L, 3, w.Hkv, w.C), device="cuda")
    positions = torch.full((L, 3, w.Hkv, w.C), lsp.BY_PLACE, dtype=torch.int32, device="cuda")
    tokens, suffix_len = m["prefix_len"], m["suffix_len"].clone()
    cache_len = tokens.clone()
    rows = torch.arange(w.S, dtype=torch.int32, device="cuda").expand(3, w.S).contiguous()
    kw = {k: v for k, v in budget.items() if k != "decay"}
    for step, n in enumerate(lens):
        before, was, had = weights.cpu(), cache_len.cpu(), [k.cpu() for k in cols["k_cache"]]
        lsp.attn_key_weights_layers(attn, cache_len, suffix_len, weights, decay=budget["decay"])
        if step % 8 == 0:
            for l in range(L):
                want = serving.key_weights(cols["q"][l].cpu(), cols["k_suf"][l].cpu(), had[l], was, suffix_len.cpu(), before[l], budget["decay"])
                assert torch.allclose(weights[l].cpu().double(), want, rtol=1e-4, atol=1e-6)
        lsp.kv_gather_append(rows, n, cache_len, table)
        tokens += n
        suffix_len -= n
        given, length, at = weights.cpu(), cache_len.cpu(), positions.cpu()
        caches = [torch.stack(cols[k]).cpu() for k in ("k_cache", "v_cache")]
        lsp.kv_evict(weights, cache_len, table, positions=positions, token_len=tokens, **kw)
        new_w, new_len, _ = serving.evict(given, length, caches=caches, positions=at, token_len=tokens.cpu(), **kw)
        assert torch.equal(weights.cpu(), new_w) and torch.equal(cache_len.cpu(), new_len) and torch.equal(positions.cpu(), at)
        assert all(torch.equal(torch.stack(cols[k]).cpu(), c) for k, c in zip(("k_cache", "v_cache"), caches))
    return weights, positions, cache_len


def _plain(w, s, **kw):
    """The loop with suffix rows that stay as they are."""
    from paper_2603_05454_amd.loop import decode_loop
    fn = lambda step, p: W.make_logits(w, step=step, prefix_len=p.cpu())[0].cuda()      # noqa: E731
    return decode_loop(fn, s["bitmap"], w.V, w.tau, w.window, 1, 1, s["prefix_len"], s["suffix_len"], s["tokens"], kv_layers=s["kv_layers"],
                       gen_len=w.gen_len, run_attention=True, **kw)


BUDGET = dict(keep=44, high=50, first=2, recent=8, decay=0.9)


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("budget", [BUDGET, dict(keep=44, high=44, first=0, recent=20, decay=1.0)])
def test_a_bounded_cache_step_by_step(lsp, graph, dtype, budget):
    w = W.scaled(_work(), dtype=dtype)
    s, m = _start(w), _start(w)
    lens = []
    res = _plain(w, s, graph=graph, cache_budget=budget, observer=lambda step, z, conf, out: lens.append(out["commit_len"].clone()))
    weights, positions, cache_len = _calls(lsp, w, m, lens, budget)
    assert torch.equal(cache_len, res["cache_len"]) and torch.equal(weights, res["state"]["weights"]) and torch.equal(positions, res["state"]["positions"])
    for a, b in zip(s["kv_layers"], m["kv_layers"]):
        assert torch.equal(a["k_cache"], b["k_cache"]) and torch.equal(a["v_cache"], b["v_cache"])


def test_positions_of_the_callers_own_and_of_a_state(lsp):
    """Positions go on with a state, in the place of the budget's; a cache that was cut back without them cannot be told which of its rows are recent."""
    w = _work()
    whole, parts = _start(w), _start(w)

    def given():        # of the prompt's rows; the rows behind them are to come
        at = torch.arange(w.C, dtype=torch.int32, device="cuda").expand(w.layers, 3, w.Hkv, w.C)
        return torch.where(at < whole["prefix_len"].view(1, 3, 1, 1), at, lsp.BY_PLACE).contiguous()
    mine = given()
    again = given()
    a = _plain(w, whole, cache_budget=dict(BUDGET, positions=mine))
    assert a["state"]["positions"] is mine
    b = _plain(w, parts, cache_budget=BUDGET, stop_after=25)
    b = _plain(w, parts, cache_budget=dict(BUDGET, positions=again), state=b["state"])
    for n in range(w.layers):       # (given ones are not by place where nothing was evicted, but say the same)
        assert torch.equal(whole["kv_layers"][n]["k_cache"], parts["kv_layers"][n]["k_cache"])
    assert torch.equal(a["state"]["weights"], b["state"]["weights"]) and torch.equal(a["cache_len"], b["cache_len"])
    s = _start(w)
    c = _plain(w, s, cache_budget=dict(keep=44), stop_after=20)
    assert "positions" not in c["state"]
    with pytest.raises(lsp.LspError, match="without positions"):
        _plain(w, s, cache_budget=dict(keep=44, recent=4), state=c["state"])
    c = _plain(w, s, cache_budget=dict(keep=44), state=c["state"])
    assert (c["cache_len"] <= 44).all()
    with pytest.raises(lsp.LspError, match="positions must"):
        _plain(w, _start(w), cache_budget=dict(keep=44, recent=4, positions=mine[:1]))
