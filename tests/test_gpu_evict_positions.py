"""lsp_kv_evict_positions against its definition: rows, weights, positions, lengths and indices exactly, over evictions one after the other."""
import pytest
import torch

from oracle import serving

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsp():
    import paper_2603_05454_amd as m
    assert torch.cuda.is_available()
    return m


class _Cache:
    """On the device and, as the definition moves it, on the host; fp32 or bf16 rows of random numbers."""

    def __init__(self, lsp, L, B, H, D, C, P, T=None, dtype=torch.float32, seed=0):
        self.lsp, self.g = lsp, torch.Generator().manual_seed(seed)
        self.host = [torch.randn((L, B, C, H, D), generator=self.g).to(dtype) for _ in range(2)]
        self.w = torch.rand((L, B, H, C), generator=self.g)
        self.P = torch.tensor(P, dtype=torch.int32)
        self.T = self.P.clone() if T is None else torch.tensor(T, dtype=torch.int32)
        self.at = torch.full((L, B, H, C), lsp.BY_PLACE, dtype=torch.int32)
        self.dev = [t.cuda() for t in (*self.host, self.w, self.P, self.T, self.at)]
        suf = [torch.zeros((B, 1, H, D), dtype=dtype, device="cuda") for _ in range(L)]
        self.table = lsp.LayerTable(suf, suf, list(self.dev[0].unbind(0)), list(self.dev[1].unbind(0)))

    def append(self, n):
        """n[b] rows: their K, V and weights are what lies behind the end already; positions have nothing written."""
        n = torch.tensor(n, dtype=torch.int32)
        C = self.w.shape[-1]
        for b in range(len(n)):
            a, e = int(self.P[b]), int(self.P[b] + n[b])
            assert e <= C
            self.w[:, b, :, a:e] = torch.rand(self.w[:, b, :, a:e].shape, generator=self.g) * 0.3
            for c in self.host:
                c[:, b, a:e] = torch.randn(c[:, b, a:e].shape, generator=self.g).to(c.dtype)
        self.P, self.T = self.P + n, self.T + n
        for d, h in zip(self.dev, (*self.host, self.w, self.P, self.T)):
            d.copy_(h)

    def evict(self, keep, high=None, first=0, recent=0, out_of_place=False, **kw):
        L, B, H, C = self.w.shape
        w, P = self.dev[2:4]
        kept = torch.full((L, B, H, keep), -5, dtype=torch.int32, device="cuda")
        to = dict(new_weights=w.clone(), new_len=torch.full_like(P, -9)) if out_of_place else {}
        self.lsp.kv_evict(w, P, self.table, keep=keep, high=high, first=first, recent=recent, kept_index=kept, positions=self.dev[5], token_len=self.dev[4],
                          **to, **kw)
        torch.cuda.synchronize()
        self.w, self.P, index = serving.evict(self.w, self.P, keep, high, first, recent, caches=self.host, positions=self.at, token_len=self.T)
        if out_of_place:
            w.copy_(to["new_weights"])
            P.copy_(to["new_len"])
        assert torch.equal(kept.cpu(), index)
        for name, d, h in zip(("K", "V", "weights", "length", "tokens", "positions"), self.dev, (*self.host, self.w, self.P, self.T, self.at)):
            assert torch.equal(d.cpu(), h), name


CASES = [   # L, B, H, D, C, P, rows appended at each of three steps, keep, high, first, recent
    (1, 1, 1, 8, 12, [5], [3], 2, None, 0, 1), (2, 3, 2, 64, 90, [40, 20, 21], [9, 4, 1], 20, None, 2, 10), (2, 2, 2, 64, 400, [300, 250], [20, 3], 200, 220, 4, 180),
    (1, 2, 2, 64, 700, [600, 60], [1, 1], 500, None, 0, 500), (1, 1, 2, 128, 3000, [2600], [100], 1500, None, 500, 1000), (3, 1, 3, 64, 100, [90], [4], 40, None, 40, 0),
    # several workgroups of a unit, several launches, blocks of 8192 rows
    (1, 1, 1, 128, 8192, [8100], [30], 4096, None, 4, 256), (35, 1, 2, 64, 60, [50], [5], 30, None, 1, 8), (1, 2, 1, 64, 9000, [700, 650], [40, 4], 500, None, 2, 100),
    (1, 1, 2, 64, 20000, [19000], [900], 12000, None, 3, 2500), (33, 2, 1, 64, 8200, [8200, 4000], [1, 1], 3000, 3500, 0, 400),
]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("out_of_place", [False, True])
def test_one_eviction_after_the_other(lsp, case, out_of_place):
    L, B, H, D, C, P, n, keep, high, first, recent = CASES[case]
    c = _Cache(lsp, L, B, H, D, C, P, T=None if case % 2 else [p + 100 * b for b, p in enumerate(P)], seed=case)
    c.evict(keep, high, first, recent, out_of_place=out_of_place)
    for _ in range(3):
        c.append(n)
        c.evict(keep, high, first, recent, out_of_place=out_of_place)


def test_bf16_rows_and_many_small_steps(lsp):
    c = _Cache(lsp, 2, 3, 2, 128, 200, [150, 80, 100], dtype=torch.bfloat16)
    for step in range(30):
        c.append([1, 3, 2] if step else [0, 0, 0])
        c.evict(100, None, 3, 40)


def test_positions_of_every_kind(lsp):
    """The caller's own, in any order, some of them by place; repeated and meaningless ones, where the last places stay."""
    for kind in ("shuffled", "some", "repeated", "extreme", "before"):
        c = _Cache(lsp, 1, 2, 3, 64, 500, [500, 433], seed=5)
        g = torch.Generator().manual_seed(6)
        p = torch.stack([torch.randperm(500, generator=g) for _ in range(6)]).view(1, 2, 3, 500).to(torch.int32)
        c.T += 67
        if kind == "some":
            p[..., 200:] = c.lsp.BY_PLACE
            p[..., :200] = p[..., :200] % 3
        elif kind == "repeated":
            p.fill_(499)
        elif kind == "extreme":
            c.T.fill_(600)              # (down to ages that do not wrap, which would mean nothing)
            p = torch.where(torch.rand(p.shape, generator=g) < 0.05, torch.randint(590, 2 ** 31 - 1, p.shape, generator=g),
                            torch.randint(-2 ** 31 + 700, 0, p.shape, generator=g)).to(torch.int32)
        elif kind == "before":
            c.T.fill_(5)                # more rows than tokens
            p.fill_(c.lsp.BY_PLACE)
        c.at.copy_(p)
        c.dev[4].copy_(c.T)
        c.dev[5].copy_(c.at)
        c.evict(250, None, 2, 60)


def test_native_and_general_path_agree_and_refuse(lsp, monkeypatch):
    made = []
    for native in (True, False):
        c = _Cache(lsp, 1, 2, 2, 64, 60, [60, 41], seed=7)
        w, P, T, at = c.dev[2:]
        if native:
            assert lsp._nat.kv_evict(w, P, c.table, (30, 40, 1, 5), w, P, None, None, at, T) == 0
            assert lsp._nat.kv_evict(w, P, c.table, (30, 40, 1, 5), w, P, None, None, at.long(), T) is None
            for bad, text in ((dict(positions=at), "together"), (dict(token_len=T), "together"), (dict(positions=at.long(), token_len=T), "positions must"),
                              (dict(positions=at, token_len=T[:1]), "token_len must"), (dict(positions=at[..., 1:], token_len=T), "positions must"),
                              (dict(positions=at, token_len=P), "new_len")):
                with pytest.raises(lsp.LspError, match=text):
                    lsp.kv_evict(w, P, c.table, 30, **bad)
        else:
            monkeypatch.setattr(lsp, "_nat", None)
            lsp.kv_evict(w, P, c.table, 30, high=40, first=1, recent=5, positions=at, token_len=T)
        made.append(c.dev)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*made))


def test_graph_replays(lsp):
    """Evictions of one graph, with eager ones of the same cache in between."""
    c = _Cache(lsp, 2, 2, 2, 64, 300, [280, 260], seed=8)
    kw = dict(keep=200, first=2, recent=50)
    c.evict(**kw)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            lsp.kv_evict(c.dev[2], c.dev[3], c.table, positions=c.dev[5], token_len=c.dev[4], **kw)
    for step in range(5):
        c.append([7, 30])
        graph.replay()
        torch.cuda.synchronize()
        c.w, c.P, _ = serving.evict(c.w, c.P, caches=c.host, positions=c.at, token_len=c.T, **kw)
        for d, h in zip(c.dev, (*c.host, c.w, c.P, c.T, c.at)):
            assert torch.equal(d.cpu(), h)
        c.append([9, 1])
        c.evict(**kw)


def test_more_than_2_31_positions(lsp):
    """30 layers of 8 x 300 000 rows of 32 heads; the last sequence is cut, in the first and the last layer by the definition."""
    L, B, H, D, C, keep, recent = 30, 8, 32, 8, 300_000, 299_900, 5000
    g = torch.Generator(device="cuda").manual_seed(7)
    caches = [[torch.empty((B, C, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(L)] for _ in range(2)]     # (what moves there is not looked at)
    w = torch.zeros((L, B, H, C), device="cuda")
    w[:, -1].uniform_(generator=g)
    at = torch.full((L, B, H, C), lsp.BY_PLACE, dtype=torch.int32, device="cuda")
    assert at.numel() > 2**31
    some = [(0, 0), (L - 1, H - 1)]
    for l, h in some:
        at[l, -1, h] = torch.randperm(C, device="cuda", generator=g).to(torch.int32)
    P = torch.tensor([0] * (B - 1) + [C], dtype=torch.int32, device="cuda")
    T = P + 70
    wanted = []
    for l, h in some:
        p = at[l, -1, h].cpu().view(1, 1, 1, C).clone()
        wanted.append((*serving.evict(w[l, -1, h].cpu().view(1, 1, 1, C), P[-1:].cpu(), keep, recent=recent, positions=p, token_len=T[-1:].cpu()), p))
    suf = [torch.zeros((B, 1, H, D), dtype=torch.bfloat16, device="cuda")] * L
    lsp.kv_evict(w, P, lsp.LayerTable(suf, suf, *caches), keep=keep, recent=recent, positions=at, token_len=T)
    assert P.tolist() == [0] * (B - 1) + [keep]
    for (l, h), (weight, _, _, p) in zip(some, wanted):
        assert torch.equal(at[l, -1, h].cpu(), p[0, 0, 0]) and torch.equal(w[l, -1, h].cpu(), weight[0, 0, 0])
    assert (at[:, :-1] == lsp.BY_PLACE).all() and (at[1, -1, 0, keep:] == lsp.BY_PLACE).all() and (at[1, -1, 0, :keep] >= 70).all()
