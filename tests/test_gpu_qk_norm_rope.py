"""lsp_qk_norm_rope against the definition in 64 bits."""
import pytest
import torch

from oracle import eight_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsp():
    import paper_2603_05454_amd as m
    assert torch.cuda.is_available()
    return m


@pytest.fixture(params=["native", "general"])
def marshalled(request, lsp, monkeypatch):
    lsp.lib()
    if request.param == "general":
        monkeypatch.setattr(lsp, "_nat", None)


def _close(got, want, size, before, dtype, n):
    """A norm: at most 16 + 5 additions on the way of a square and one rounding of it, half of which is the root's, then the mean, the root, the quotient and
    two products, each 2^-24 of the value: 16 x 2^-24.  A rotation: sine and cosine within 2 x 2^-24, a product, a sum: 4 x 2^-24 of what the
    element is made of.  21 x 2^-24 in all, and the rounding to the type."""
    got = got.cpu().double()
    for b in range(got.shape[0]):
        k = min(max(int(n[b]), 0), got.shape[1])
        tol = 21 * 2.0 ** -24 * size[b, :k] + (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24) * want[b, :k].abs() + 1e-30
        err = (got[b, :k] - want[b, :k]).abs()
        assert (err <= tol).all(), (err / tol).max()
        assert torch.equal(got[b, k:], before[b, k:].cpu().double())


def _freq(R, theta=10000.0):
    return (theta ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)).float() if R else torch.zeros(0)


CASES = [   # B, S, Hq, Hkv, D, R, norm, prefix, suffix (None: not given)
    (1, 1, 1, 1, 64, 64, True, None, None), (1, 1, 28, 4, 128, 128, False, [100003], [1]), (2, 5, 3, 1, 64, 16, True, [0, 7], [5, 0]),
    (3, 33, 4, 2, 128, 64, True, [31, 999, 4095], [33, 1, 32]), (2, 7, 6, 2, 64, 48, False, [1 << 20, 12], [9, -2]), (1, 300, 5, 5, 128, 0, True, [3], None),
    (5, 250, 4, 4, 64, 64, True, [1, 2, 3, 4, 5], [250, 249, 0, 1, 100]), (2, 700, 7, 1, 128, 112, True, [2 ** 31 - 701, 0], [700, 3]),
    (1, 2, 70, 3, 64, 32, False, [5], [2]), (9, 130, 2, 1, 128, 128, False, list(range(9)), list(range(122, 131)))]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_the_definition(lsp, dtype, case, interleaved):
    B, S, Hq, H, D, R, norm, P, N = CASES[case]
    g = torch.Generator().manual_seed(case)
    q, k = ((torch.randn((B, S, h, D), generator=g) * torch.exp(torch.randn((B, S, h, 1), generator=g))).to(dtype) for h in (Hq, H))
    w = [torch.randn(D, generator=g) for _ in range(2)] if norm else [None, None]
    P, N = (None if x is None else torch.tensor(x, dtype=torch.int32) for x in (P, N))
    f = _freq(R)
    want = eight_bits.norm_rope(q, k, f, *w, eps=1e-5, prefix_len=P, suffix_len=N, interleaved=interleaved)
    dev = lambda t: None if t is None else t.cuda()      # noqa: E731
    out = (torch.full_like(q, 7.0).cuda(), torch.full_like(k, 7.0).cuda())
    before = [o.clone() for o in out]
    kw = dict(q_weight=dev(w[0]), k_weight=dev(w[1]), eps=1e-5, prefix_len=dev(P), suffix_len=dev(N), interleaved=interleaved)
    assert lsp.qk_norm_rope(q.cuda(), k.cuda(), f.cuda(), out=out, **kw) is out
    n = [S] * B if N is None else N
    for o, (y, size), x in zip(out, want, before):
        _close(o, y, size, x, dtype, n)
    # in place: the same bits
    a, b = q.cuda(), k.cuda()
    lsp.qk_norm_rope(a, b, f.cuda(), out=(a, b), **kw)
    for i in range(B):
        m = min(max(int(n[i]), 0), S)
        assert torch.equal(a[i, :m], out[0][i, :m]) and torch.equal(b[i, :m], out[1][i, :m])
        assert torch.equal(a[i, m:], q[i, m:].cuda()) and torch.equal(b[i, m:], k[i, m:].cuda())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_positions_and_strides(lsp, marshalled, dtype):
    """Positions of the caller's own; queries and keys as parts of one projection's output, turned where they are."""
    B, S, Hq, H, D, R = 2, 37, 6, 2, 128, 96
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn((B, S + 1, Hq + 2 * H, D), generator=g).to(dtype)
    pos = torch.randint(0, 1 << 30, (B, S), generator=g, dtype=torch.int32)
    w, f, N = [torch.randn(D, generator=g) for _ in range(2)], _freq(R), torch.tensor([37, 20], dtype=torch.int32)
    d = qkv.cuda()
    part = lambda t: (t[:, 1:, :Hq], t[:, 1:, Hq:Hq + H])       # noqa: E731
    want = eight_bits.norm_rope(*part(qkv), f, *w, suffix_len=N, positions=pos)
    q, k = part(d)
    lsp.qk_norm_rope(q, k, f.cuda(), w[0].cuda(), w[1].cuda(), suffix_len=N.cuda(), positions=pos.cuda(), out=(q, k))
    for o, (y, size), x in zip((q, k), want, part(qkv)):
        _close(o, y, size, x, dtype, N)
    assert torch.equal(d[:, 1:, Hq + H:].cpu(), qkv[:, 1:, Hq + H:]) and torch.equal(d[:, 0].cpu(), qkv[:, 0])


def test_positions_take_the_place_of_lengths(lsp, marshalled):
    q, k = torch.randn(2, 9, 3, 64, device="cuda"), torch.randn(2, 9, 1, 64, device="cuda")
    f, P = _freq(64).cuda(), torch.tensor([11, 500], dtype=torch.int32, device="cuda")
    a = lsp.qk_norm_rope(q, k, f, prefix_len=P)
    b = lsp.qk_norm_rope(q, k, f, prefix_len=P * 0, positions=(P.view(2, 1) + torch.arange(9, device="cuda")).int())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    c = lsp.qk_norm_rope(q, k, f)
    assert torch.equal(c[0][:, 0], q[:, 0])       # position 0


def test_many_rows(lsp):
    """Long batches take several rows to a workgroup: the same bits as row by row."""
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k = (torch.randn((3, 1000, h, 128), generator=g, device="cuda").to(torch.bfloat16) for h in (7, 2))
    f, w = _freq(128).cuda(), [torch.randn(128, generator=g, device="cuda") for _ in range(2)]
    N, P = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([1000, 999, 2], [5, 6, 7]))
    out = (torch.zeros_like(q), torch.zeros_like(k))
    lsp.qk_norm_rope(q, k, f, *w, prefix_len=P, suffix_len=N, out=out)
    for u in range(0, 1000, 111):
        o = (torch.zeros_like(q[:, u:u + 1]), torch.zeros_like(k[:, u:u + 1]))
        lsp.qk_norm_rope(q[:, u:u + 1], k[:, u:u + 1], f, *w, prefix_len=P + u, suffix_len=(N - u).clamp(max=1), out=o)
        assert torch.equal(o[0], out[0][:, u:u + 1]) and torch.equal(o[1], out[1][:, u:u + 1])


def test_graph(lsp):
    q, k = torch.randn(2, 30, 4, 64, device="cuda"), torch.randn(2, 30, 2, 64, device="cuda")
    f = _freq(64).cuda()
    P, N = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([5, 6], [30, 11]))
    out = (torch.zeros_like(q), torch.zeros_like(k))
    lsp.qk_norm_rope(q, k, f, prefix_len=P, suffix_len=N, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lsp.qk_norm_rope(q, k, f, prefix_len=P, suffix_len=N, out=out)
    for step in range(3):
        q.normal_()
        k.normal_()
        P.add_(3)
        N.sub_(1)
        want = (out[0].clone(), out[1].clone())
        lsp.qk_norm_rope(q, k, f, prefix_len=P, suffix_len=N, out=want)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_offsets_beyond_32_bits(lsp):
    """2.2e9 numbers, in place: rows on both sides of 2^31 elements and bytes."""
    B, S, Hq, H, D = 2, 8300, 1024, 1, 128
    g = torch.Generator().manual_seed(8)
    q, k = torch.zeros((B, S, Hq, D), dtype=torch.bfloat16, device="cuda"), torch.randn((B, S, H, D), generator=g).to(torch.bfloat16).cuda()
    rows = [(0, 0), (0, 4095), (0, 4096), (0, 8191), (0, 8192), (0, 8299), (1, 0), (1, 8083), (1, 8084), (1, 8298)]
    x = torch.randn((len(rows), Hq, D), generator=g).to(torch.bfloat16)
    for i, (b, u) in enumerate(rows):
        q[b, u] = x[i].cuda()
    q[1, 8299] = 3.0
    w = torch.randn(D, generator=g)
    f, lens = _freq(D), [torch.tensor(v, dtype=torch.int32) for v in ([5, 9], [S, S - 1])]
    lsp.qk_norm_rope(q, k, f.cuda(), q_weight=w.cuda(), k_weight=w.cuda(), eps=1e-5, prefix_len=lens[0].cuda(), suffix_len=lens[1].cuda(), out=(q, k))
    for i, (b, u) in enumerate(rows):
        pos = torch.tensor([[int(lens[0][b]) + u]], dtype=torch.int32)
        (want, size), _ = eight_bits.norm_rope(x[i].view(1, 1, Hq, D), x[i].view(1, 1, Hq, D), f, w, w, eps=1e-5, positions=pos)
        _close(q[b, u].view(1, 1, Hq, D), want, size, x[i].view(1, 1, Hq, D), torch.bfloat16, [1])
    assert (q[1, 8299] == 3.0).all()
    assert q[0, 1].abs().max() == 0 and q[1, 4000].abs().max() == 0
