"""Scores, key weights and eviction where element and byte offsets no longer fit 32 bits, on two streams at once, and in graphs that share a workspace."""
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


def test_scores_of_logits_beyond_2_31_elements(lsp):
    """20 x 1024 x 126464 bf16: rows at both ends, on either side of the marks of 2^31 elements and 2^32 bytes, and some between.  The logarithm of a sum
    of 126464 terms in chains of V / 64 (1976 additions of half a step, 2^-24) and results up to 120: below 2e-4 + 2e-5."""
    w = W.scaled(W.C4, B=20)
    z, _ = W.make_logits(w, device="cuda")
    assert z.numel() > 2**31
    g = torch.Generator().manual_seed(12)
    ids = torch.randint(0, w.V, (w.B, w.S), generator=g, dtype=torch.int32).cuda()
    lp, h, alt_id, alt = lsp.token_scores(z, ids, num_alt=8)
    R = w.B * w.S
    marks = [2**31 // w.V, 2**32 // (2 * w.V)]
    rows = torch.cat([torch.tensor([0, R - 1] + [r + d for r in marks for d in (-1, 0, 1)]), torch.randint(R // 2, R, (40,), generator=g)]).cuda()
    pick = lambda t: t.reshape(R, -1)[rows].cpu().unsqueeze(0)      # noqa: E731
    want = serving.token_scores(pick(z), pick(ids)[..., 0], num_alt=8)
    assert torch.equal(pick(alt_id), want[2])
    assert (pick(alt) - want[3]).abs().max() <= 2.2e-4 and (pick(lp)[..., 0] - want[0]).abs().max() <= 2.2e-4
    # (terms of the entropy weigh the same errors with their distance from the maximum, log V = 12 on average at most)
    assert (pick(h)[..., 0] - want[1]).abs().max() <= 14 * 2.2e-4


def _one_long_sequence(B, C):
    P = torch.tensor([3] * (B - 1) + [C - 16], dtype=torch.int32)
    return P, torch.tensor([0, 2] + [0] * (B - 3) + [16], dtype=torch.int32)


def test_key_weights_beyond_2_31_elements(lsp):
    """A cache of 8 x 300 000 rows of 32 heads (2.5e9 numbers, 20 GB) that 30 layers read, and their 2.3e9 weights.  Scores as in the tests of small
    shapes (1e-4), and chains of up to 2000 additions: 1.2e-4 more."""
    L, B, Hkv, D, C, S = 30, 8, 32, 128, 300_000, 16
    g = torch.Generator(device="cuda").manual_seed(5)
    cache = torch.empty((B, C, Hkv, D), dtype=torch.bfloat16, device="cuda")
    for b in range(B):
        cache[b].normal_(generator=g)
    q, k = (torch.empty((B, S, Hkv, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    weights = torch.full((L, B, Hkv, C), 0.25, device="cuda")
    assert cache.numel() > 2**31 and weights.numel() > 2**31
    P, N = _one_long_sequence(B, C)
    P[-1] -= 3
    table = lsp.AttnLayerTable([q] * L, [k] * L, [k] * L, [cache] * L, [cache] * L, [torch.empty_like(q)] * L)
    lsp.attn_key_weights_layers(table, P.cuda(), N.cuda(), weights, decay=0.5)
    for b in (1, B - 1):
        for h in (0, Hkv - 1):
            n = int(P[b])
            one = slice(b, b + 1), slice(None), slice(h, h + 1)
            want = serving.key_weights(q[one].cpu(), k[one].cpu(), cache[b:b + 1, :n, h:h + 1].cpu(), P[b:b + 1], N[b:b + 1],
                                       torch.full((1, 1, n), 0.25), 0.5)
            for layer in (0, L - 1):
                got = weights[layer, b, h].cpu().double()
                assert ((got[:n] - want[0, 0]).abs() <= 2.2e-4 * want[0, 0]).all()
                assert (got[n + int(N[b]):] == 0.25).all()
    assert (weights[:, 0] == 0.25).all() and torch.equal(weights[0], weights[L - 1])


def _kept(weights, P, keep, first, recent):
    return serving.evict(weights.cpu()[None, None, None], torch.tensor([P]), keep, first=first, recent=recent)[2][0, 0, 0]


def test_eviction_from_caches_beyond_2_31_elements(lsp):
    """8 x 73 728 rows of 32 heads (2.4e9 numbers each of K and V): every row of the first and the last sequence, and what is between unchanged."""
    B, Hkv, D, C, keep = 8, 32, 128, 73_728, 60_001
    g = torch.Generator(device="cuda").manual_seed(6)
    k = torch.empty((B, C, Hkv, D), dtype=torch.bfloat16, device="cuda")
    for b in range(B):
        k[b].normal_(generator=g)
    v = -k
    assert k.numel() > 2**31
    was = k.clone()
    P = torch.tensor([C - 5] + [keep] * (B - 2) + [C], dtype=torch.int32, device="cuda")
    w = torch.rand((1, B, Hkv, C), device="cuda", generator=g)
    wanted = {(b, h): _kept(w[0, b, h], int(P[b]), keep, 4, 100) for b in (0, B - 1) for h in (0, Hkv - 1)}
    index = torch.empty((1, B, Hkv, keep), dtype=torch.int32, device="cuda")
    suf = torch.zeros((B, 1, Hkv, D), dtype=torch.bfloat16, device="cuda")
    lsp.kv_evict(w, P, lsp.LayerTable([suf], [suf], [k], [v]), keep=keep, first=4, recent=100, kept_index=index)
    assert P.tolist() == [keep] * B
    for (b, h), at in wanted.items():
        assert torch.equal(index[0, b, h].cpu(), at)
    assert torch.equal(k[1:-1], was[1:-1])
    for b in (0, B - 1):
        for h in range(Hkv):
            assert torch.equal(k[b, :keep, h], was[b, index[0, b, h].long(), h])
        assert torch.equal(k[b, keep:], was[b, keep:])
    assert all(torch.equal(v[b], -k[b]) for b in range(B))


def test_eviction_by_more_than_2_31_weights(lsp):
    L, B, Hkv, D, C, keep = 30, 8, 32, 8, 300_000, 299_900
    g = torch.Generator(device="cuda").manual_seed(7)
    caches = [[torch.empty((B, C, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(L)] for _ in range(2)]
    for c in caches[0]:
        c[-1].normal_(generator=g)
    for c, d in zip(*caches):
        d[-1] = -c[-1]
    w = torch.zeros((L, B, Hkv, C), device="cuda")
    w[:, -1].uniform_(generator=g)
    assert w.numel() > 2**31
    P = torch.tensor([0] * (B - 1) + [C], dtype=torch.int32, device="cuda")
    some = [(0, 0), (L - 1, Hkv - 1)]
    wanted = [(_kept(w[l, -1, h], C, keep, 0, 0), w[l, -1, h].clone(), caches[0][l][-1, :, h].clone()) for l, h in some]
    suf = [torch.zeros((B, 1, Hkv, D), dtype=torch.bfloat16, device="cuda")] * L
    lsp.kv_evict(w, P, lsp.LayerTable(suf, suf, *caches), keep=keep)
    assert P.tolist() == [0] * (B - 1) + [keep]
    for (l, h), (at, weight, rows) in zip(some, wanted):
        at = at.long().cuda()
        assert torch.equal(w[l, -1, h, :keep], weight[at]) and torch.equal(w[l, -1, h, keep:], weight[keep:])
        assert torch.equal(caches[0][l][-1, :keep, h], rows[at]) and torch.equal(caches[1][l][-1, :keep, h], -rows[at])
    assert (w[:, :-1] == 0).all()


class _Work:
    """One call of each operator on operands of its own, all from the seed; results are kept apart from what they are made of."""

    def __init__(self, lsp, seed, workspaces=None):
        self.lsp = lsp
        g = torch.Generator().manual_seed(seed)
        B, S, V, Hq, Hkv, D, C, L = 2, 40 + seed, 40_000, 8, 2, 64, 900, 3
        self.z = torch.randn((B, S, V), generator=g).cuda()
        self.ids = torch.randint(0, V, (B, S), generator=g, dtype=torch.int32).cuda()
        n = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).cuda()      # noqa: E731
        self.q, self.k = [n(B, S, Hq, D) for _ in range(L)], [n(B, S, Hkv, D) for _ in range(L)]
        self.first = [n(B, C, Hkv, D) for _ in range(2 * L)]
        self.caches = [t.clone() for t in self.first]
        self.attn = lsp.AttnLayerTable(self.q, self.k, self.k, self.caches[:L], self.caches[L:], [torch.empty_like(t) for t in self.q])
        self.table = lsp.LayerTable(self.k, self.k, self.caches[:L], self.caches[L:])
        self.N = torch.tensor([S, 3], dtype=torch.int32).cuda()
        self.P0 = torch.tensor([800, 700 + seed], dtype=torch.int32).cuda()
        self.P, self.w = self.P0.clone(), torch.zeros((L, B, Hkv, C), device="cuda")
        self.out = (torch.zeros((B, S), device="cuda"), torch.zeros((B, S), device="cuda"), torch.zeros((B, S, 4), dtype=torch.int32, device="cuda"),
                    torch.zeros((B, S, 4), device="cuda"))
        sizes = (lsp.token_scores_workspace_bytes(B, S, V, 4), lsp.attn_key_weights_workspace_bytes(lsp.LSP_BF16, B, S, Hq, Hkv, D, C, L),
                 lsp.kv_evict_workspace_bytes(self.table, keep=500, recent=20))
        self.spaces = workspaces or [torch.full((max(n, 16) + 4096,), 7, dtype=torch.uint8, device="cuda") for n in sizes]

    def reset(self):
        self.P.copy_(self.P0)
        self.w.zero_()
        for c, f in zip(self.caches, self.first):
            c.copy_(f)
        for t in self.out:
            t.zero_()

    def run(self):
        self.lsp.token_scores(self.z, self.ids, self.N, num_alt=4, out=self.out, workspace=self.spaces[0])
        self.lsp.attn_key_weights_layers(self.attn, self.P, self.N, self.w, workspace=self.spaces[1])
        self.lsp.kv_evict(self.w, self.P, self.table, keep=500, recent=20, workspace=self.spaces[2])

    def results(self):
        return [t.clone() for t in (*self.out, self.w, self.P, *self.caches)]

    def alone(self):
        self.reset()
        self.run()
        torch.cuda.synchronize()
        return self.results()


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_two_streams_at_once(lsp):
    work = [_Work(lsp, 0), _Work(lsp, 5)]
    want = [w.alone() for w in work]
    streams = [torch.cuda.Stream() for _ in work]
    for _ in range(4):
        for w in work:
            w.reset()
        torch.cuda.synchronize()
        for w, s in zip(work, streams):
            with torch.cuda.stream(s):
                w.run()
        torch.cuda.synchronize()
        assert all(_same(w.results(), x) for w, x in zip(work, want))


def test_two_graphs_that_share_their_workspaces(lsp):
    work = [_Work(lsp, 5)]
    work.append(_Work(lsp, 0, work[0].spaces))
    want = [w.alone() for w in work]
    graphs = []
    for w in work:
        graphs.append(torch.cuda.CUDAGraph())
        w.reset()
        torch.cuda.synchronize()
        with torch.cuda.graph(graphs[-1]):
            w.run()
    for turn in (0, 1, 0, 0, 1):
        work[turn].reset()
        graphs[turn].replay()
        torch.cuda.synchronize()
        assert _same(work[turn].results(), want[turn])
        if turn:
            assert _same(work[0].alone(), want[0])      # eager, between the replays
