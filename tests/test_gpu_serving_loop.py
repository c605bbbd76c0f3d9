"""Token scores, key weights and eviction together, as a decode loop uses them: an answer's log probabilities, and caches of bounded length."""
import pytest
import torch

import workloads as W
from oracle import serving

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsp():
    import paper_2603_05454_amd as m
    assert torch.cuda.is_available()
    return m


def _work(G=96, P=40, dtype="bf16"):
    return W.scaled(W.C5, B=3, S=G, V=4096, P=P, gen_len=G, C=P + G + 20, layers=2, Hq=4, Hkv=2, D=64, dtype=dtype)


def _start(w):
    pl, sl = (t.cuda() for t in W.make_lengths(w))
    return dict(bitmap=W.make_delimiters(w)[1].cuda(), prefix_len=pl, suffix_len=sl, tokens=W.make_tokens(w, w.C).cuda(),
                kv_layers=[{k: v.cuda() for k, v in W.make_layer_kv(w, l).items()} for l in range(w.layers)])


def _loop(w, s, **kw):
    from paper_2603_05454_amd.loop import decode_loop
    fn = lambda step, p: W.make_logits(w, step=step, prefix_len=p.cpu())[0].cuda()      # noqa: E731
    return decode_loop(fn, s["bitmap"], w.V, w.tau, w.window, 1, 1, s["prefix_len"], s["suffix_len"], s["tokens"], kv_layers=s["kv_layers"],
                       gen_len=w.gen_len, run_attention=True, **kw)


def _state(s):
    return [s["prefix_len"], s["suffix_len"], s["tokens"], *[L[k] for L in s["kv_layers"] for k in ("k_cache", "v_cache")]]


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("K", [0, 5])
def test_scores_of_the_tokens_that_were_committed(lsp, graph, K):
    w = _work()
    s, T = _start(w), w.C
    scores = dict(logprob=torch.full((3, T), 7.0, device="cuda"), entropy=torch.full((3, T), 7.0, device="cuda"))
    if K:
        scores.update(alt_id=torch.full((3, T, K), 7, dtype=torch.int32, device="cuda"), alt_logprob=torch.full((3, T, K), 7.0, device="cuda"))
    want = {k: v.cpu().double() if v.is_floating_point() else v.cpu().clone() for k, v in scores.items()}
    at = s["prefix_len"].cpu().clone()

    def observer(step, z, conf, out):
        n, z, ids = out["commit_len"].cpu(), z.cpu(), conf[0].cpu()
        lp, h, alt_id, alt = serving.token_scores(z, ids, n, K)
        for b in range(3):
            a, k = int(at[b]), int(n[b])
            want["logprob"][b, a:a + k], want["entropy"][b, a:a + k] = lp[b, :k], h[b, :k]
            if K:
                want["alt_id"][b, a:a + k], want["alt_logprob"][b, a:a + k] = alt_id[b, :k], alt[b, :k]
        at.add_(n)
    res = _loop(w, s, scores=scores, observer=observer, graph=graph)
    assert res["steps"] > 5 and s["suffix_len"].max() == 0
    for k, v in scores.items():     # (sums of 4096 terms: the same bound as the call's own test)
        assert torch.equal(v.cpu(), want[k]) if k == "alt_id" else (v.cpu().double() - want[k]).abs().max() < 1e-4, k
    plain = _start(w)
    _loop(w, plain, graph=graph)
    assert all(torch.equal(a, b) for a, b in zip(_state(s), _state(plain)))


@pytest.mark.parametrize("graph", [False, True])
def test_a_budget_changes_no_token(lsp, graph):
    """Nor the caches, as long as nothing is evicted: logits are the caller's."""
    w = _work()
    s, plain = _start(w), _start(w)
    a = _loop(w, s, graph=graph, cache_budget=dict(keep=w.C - w.gen_len))
    b = _loop(w, plain, graph=graph)
    assert a["steps"] == b["steps"] and a["flips"] == b["flips"]
    assert all(torch.equal(x, y) for x, y in zip(_state(s)[:3], _state(plain)[:3]))
    first, one = _start(w), _start(w)
    _loop(w, first, graph=graph, cache_budget=dict(keep=w.C - w.gen_len), stop_after=1)
    _loop(w, one, graph=graph, stop_after=1)
    assert all(torch.equal(x, y) for x, y in zip(_state(first), _state(one)))


BUDGET = dict(keep=44, high=50, first=2, recent=8, decay=0.9)


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_bounded_cache_step_by_step(lsp, graph, dtype):
    """The loop against its calls made one by one; the first steps' weights and choices against the definition."""
    w = _work(dtype=dtype)
    s, m = _start(w), _start(w)
    lens = []
    res = _loop(w, s, graph=graph, cache_budget=BUDGET, observer=lambda step, z, conf, out: lens.append(out["commit_len"].clone()))
    assert s["suffix_len"].max() == 0 and (res["cache_len"] <= 50).all() and (s["prefix_len"] > 50).all()

    L, kv = w.layers, m["kv_layers"]
    cols = {k: [x[k] for x in kv] for k in kv[0]}
    out = [torch.zeros_like(q) for q in cols["q"]]
    attn = lsp.AttnLayerTable(cols["q"], cols["k_suf"], cols["v_suf"], cols["k_cache"], cols["v_cache"], out)
    table = lsp.LayerTable(cols["k_suf"], cols["v_suf"], cols["k_cache"], cols["v_cache"])
    weights = torch.zeros((L, 3, w.Hkv, w.C), device="cuda")
    cache_len, suffix_len = m["prefix_len"].clone(), m["suffix_len"].clone()
    rows = torch.arange(w.S, dtype=torch.int32, device="cuda").expand(3, w.S).contiguous()
    for step, n in enumerate(lens):
        before, was, had = weights.cpu(), cache_len.cpu(), [k.cpu() for k in cols["k_cache"]]
        lsp.attn_key_weights_layers(attn, cache_len, suffix_len, weights, decay=0.9)
        if step < 4:
            for l in range(L):
                want = serving.key_weights(cols["q"][l].cpu(), cols["k_suf"][l].cpu(), had[l], was, suffix_len.cpu(), before[l], 0.9)
                assert torch.allclose(weights[l].cpu().double(), want, rtol=1e-4, atol=1e-6)
        lsp.kv_gather_append(rows, n, cache_len, table)
        given, length, caches = weights.cpu(), cache_len.cpu(), [torch.stack(cols[k]).cpu() for k in ("k_cache", "v_cache")]
        lsp.kv_evict(weights, cache_len, table, **{k: v for k, v in BUDGET.items() if k != "decay"})
        if step < 8:
            new_w, new_len, _ = serving.evict(given, length, 44, 50, 2, 8, caches=caches)
            assert torch.equal(weights.cpu(), new_w) and torch.equal(cache_len.cpu(), new_len)
            assert all(torch.equal(torch.stack(cols[k]).cpu(), c) for k, c in zip(("k_cache", "v_cache"), caches))
        suffix_len -= n
    assert torch.equal(cache_len, res["cache_len"]) and torch.equal(weights, res["state"]["weights"])
    for a, b in zip(s["kv_layers"], kv):
        assert torch.equal(a["k_cache"], b["k_cache"]) and torch.equal(a["v_cache"], b["v_cache"])


@pytest.mark.parametrize("graph", [False, True])
def test_stopping_and_resuming_a_bounded_loop(lsp, graph):
    w = _work()
    whole, parts = _start(w), _start(w)
    a = _loop(w, whole, graph=graph, cache_budget=BUDGET)
    b, calls = None, 0
    while parts["suffix_len"].max() > 0:
        b = _loop(w, parts, graph=graph, cache_budget=BUDGET, stop_after=3, state=None if b is None else b["state"])
        calls += 1
        with pytest.raises(lsp.LspError, match="cut back"):
            _loop(w, parts, graph=graph, state=b["state"])
    assert calls > 2 and a["steps"] == b["steps"] and torch.equal(a["cache_len"], b["cache_len"])
    assert torch.equal(a["state"]["weights"], b["state"]["weights"]) and all(torch.equal(x, y) for x, y in zip(_state(whole), _state(parts)))


def test_weights_and_lengths_of_the_callers_own(lsp):
    """A prompt's rows may begin with weights of their own, in a cache whose rows are already fewer than the tokens."""
    w = _work()
    s = _start(w)
    weights = torch.rand((2, 3, 2, w.C), device="cuda")
    cache_len = torch.tensor([30, 44, 12], dtype=torch.int32, device="cuda")
    res = _loop(w, s, cache_budget=dict(BUDGET, weights=weights, cache_len=cache_len))
    assert res["cache_len"] is cache_len and res["state"]["weights"] is weights and (cache_len <= 50).all() and (cache_len >= 44).all()


def test_refusals(lsp):
    w = _work()
    s = _start(w)
    f = torch.zeros((3, w.C), device="cuda")
    for kw, text in ((dict(cache_budget=dict(keep=w.C - 10)), "no room"), (dict(cache_budget=dict(keep=44, weights=f)), "weights must"),
                     (dict(cache_budget=dict(keep=44, cache_len=s["prefix_len"].long())), "cache_len must"),
                     (dict(cache_budget=dict(keep=44, cache_len=s["prefix_len"])), "buffer of its own"), (dict(scores=dict(margin=f)), "scores are"),
                     (dict(scores={}), "scores are"), (dict(scores=dict(logprob=f[:, 1:])), "must have shape"), (dict(scores=dict(alt_id=f)), "come together"),
                     (dict(scores=dict(logprob=f), lm_head_weight=f), "logits"), (dict(cache_budget=dict(keep=44, first=40, recent=5)), "first"),
                     (dict(cache_budget=dict(keep=44, decay=2)), "decay"), (dict(cache_budget=dict(keep=44, high=43)), "high")):
        with pytest.raises(lsp.LspError, match=text):
            _loop(w, s, **kw)
    with pytest.raises(lsp.LspError, match="run_attention"):
        from paper_2603_05454_amd.loop import decode_loop
        decode_loop(None, s["bitmap"], w.V, 0.9, 16, 1, 1, s["prefix_len"], s["suffix_len"], s["tokens"], cache_budget=dict(keep=4))


def test_a_states_weights_and_lengths_go_before_those_of_the_budget(lsp):
    """The same dictionary may be handed over at every call, though its tensors are copies that stayed behind."""
    w = _work()
    whole, parts = _start(w), _start(w)
    f = torch.rand((len(whole["kv_layers"]), whole["prefix_len"].shape[0], w.Hkv, w.C), device="cuda")
    given = lambda s: dict(BUDGET, weights=f.clone(), cache_len=torch.full_like(s["prefix_len"], 30))      # noqa: E731
    a = _loop(w, whole, cache_budget=given(whole))
    b = _loop(w, parts, cache_budget=given(parts), stop_after=4)
    b = _loop(w, parts, cache_budget=given(parts), state=b["state"])
    assert torch.equal(a["cache_len"], b["cache_len"]) and torch.equal(a["state"]["weights"], b["state"]["weights"])
    assert all(torch.equal(x, y) for x, y in zip(_state(whole), _state(parts)))
