"""lsp_token_scores against the definition in 64 bits: ids exactly, numbers to the error of fp32 sums."""
import math

import pytest
import torch

from oracle import serving

pytestmark = pytest.mark.gpu
NEG = -math.inf


@pytest.fixture(scope="module")
def lsp():
    import paper_2603_05454_amd as m
    assert torch.cuda.is_available()
    return m


def _bounds(V, entropy):
    """Errors of log p and entropy.  A term exp(z - m), |z - m| <= 30 where it matters, carries two roundings of the exponent (2 x 30 x 2^-24 at most)
    and one step of the exponential (2^-23); sums are chains of at most V / 64 terms and a dozen joins.  The entropy's second sum weighs the same
    errors with |z - m|, whose mean is log s - H <= log V.  The result's own rounding: values up to 120, half a step each of two operations."""
    sums = (min(V, V / 64 + 64) + 60 + 2 + 12) * 2.0 ** -24
    return sums + 2 * 120 * 2.0 ** -24, sums * (2 + math.log(V + 1) + entropy.abs())


def _check(got, want, token_id, K, V, N):
    B, S = want[1].shape
    there = torch.arange(S)[None] < N[:, None]
    lp, h, ids, alt = [None if t is None else t.cpu() for t in got]
    tol_p, tol_h = _bounds(V, want[1])

    def close(x, y, tol):
        x, fine = x.double(), torch.isfinite(y)
        assert torch.equal(x[~fine], y[~fine])
        assert ((x - y).abs()[fine] <= (tol if isinstance(tol, float) else tol[fine])).all(), (x - y).abs()[fine].max()

    close(h[there], want[1][there], tol_h[there])
    assert (h[~there] == -7).all()
    if token_id is not None:
        close(lp[there], want[0][there], tol_p)
        assert (lp[~there] == -7).all()
    if K:
        assert torch.equal(ids[there], want[2][there])
        close(alt[there], want[3][there], tol_p)
        assert (ids[~there] == -7).all() and (alt[~there] == -7).all()


def _out(B, S, K, token_id):
    f = lambda *s: torch.full(s, -7.0, device="cuda")      # noqa: E731
    return (None if token_id is None else f(B, S), f(B, S), torch.full((B, S, K), -7, dtype=torch.int32, device="cuda") if K else None,
            f(B, S, K) if K else None)


def _run(lsp, z, token_id, N, K, view=None, **kw):
    B, S, V = z.shape
    zg = z.cuda() if view is None else view(z)
    tg = None if token_id is None else token_id.cuda()
    got = lsp.token_scores(zg, tg, None if N is None else N.cuda(), num_alt=K, out=_out(B, S, K, token_id), **kw)
    torch.cuda.synchronize()
    n = torch.full((B,), S) if N is None else N
    _check(got, serving.token_scores(z, token_id, n, K), token_id, K, V, n)
    return got


def _ids(B, S, V, g):
    t = torch.randint(0, V, (B, S), generator=g, dtype=torch.int32)
    t[0, 0] = V - 1
    return t


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,S,V,K", [(1, 1, 1, 3), (1, 1, 2, 1), (2, 3, 7, 7), (1, 2, 63, 32), (3, 5, 64, 8), (2, 9, 1000, 20), (1, 4, 4099, 32),
                                     (2, 70, 513, 5), (1, 130, 2048, 20), (1, 3, 16384, 20), (2, 5, 16411, 1), (1, 2, 50001, 32), (1, 1, 126464, 20),
                                     (3, 2, 152064, 5), (1, 1, 400003, 32), (1, 600, 300, 4), (2, 3, 8192, 0)])
def test_random_rows(lsp, dtype, B, S, V, K):
    g = torch.Generator().manual_seed(B * 7 + S * 11 + V + K)
    z = (torch.randn((B, S, V), generator=g) * 2).to(dtype)
    N = torch.tensor([S, max(S - 2, 0), 0][:B])
    _run(lsp, z, _ids(B, S, V, g), N.to(torch.int32), K)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [5, 700, 9000, 130001])
def test_rows_of_every_shape(lsp, dtype, V):
    """Constant, rising, falling rows, a tied maximum at both ends, masked entries of either kind, nothing left, one entry left, one sure entry."""
    low = torch.finfo(dtype).min
    up = torch.arange(V, dtype=torch.float32) * (20.0 / V)
    rows = [torch.full((V,), 3.0), up, up.flip(0), torch.zeros(V), torch.zeros(V), torch.full((V,), NEG), torch.full((V,), NEG), torch.full((V,), low),
            torch.zeros(V), torch.zeros(V), torch.full((V,), low), torch.full((V,), -0.0)]
    rows[3][[0, V - 1]] = 9.0
    rows[4][torch.arange(V) % 3 != 1] = NEG
    rows[6][V // 2] = -4.0
    rows[8][V // 3] = 80.0
    rows[9][torch.arange(V) % 5 != 2] = low
    rows[10][:V // 2] = NEG
    rows[11][::2] = 0.0
    z = torch.stack(rows)[None].to(dtype)
    ids = torch.full((1, len(rows)), V // 3, dtype=torch.int32)
    ids[0, 2], ids[0, 3] = V, -1
    for K in (0, 1, 32):
        _run(lsp, z, ids, None, K)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_heavy_ties(lsp, dtype):
    g = torch.Generator().manual_seed(3)
    z = (torch.randn((2, 4, 70000), generator=g) * 2).round().to(dtype)
    _run(lsp, z, None, torch.tensor([4, 3], dtype=torch.int32), 32)


@pytest.mark.parametrize("V,row,start", [(1001, 1001, 0), (1001, 1003, 1), (5000, 5003, 3), (70001, 70001, 5), (4096, 4104, 0)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_and_alignment(lsp, dtype, V, row, start):
    """Rows that begin at any element, inside a buffer whose other elements are NaN."""
    g = torch.Generator().manual_seed(V)
    z = torch.randn((2, 3, V), generator=g).to(dtype)

    def view(z):
        flat = torch.full((start + 2 * 4 * row + 64,), math.nan, dtype=dtype, device="cuda")
        v = flat.as_strided((2, 3, V), (4 * row, row, 1), start)
        v.copy_(z)
        return v
    _run(lsp, z, _ids(2, 3, V, g), torch.tensor([3, 2], dtype=torch.int32), 20, view=view)


def test_inactive_rows_may_hold_anything(lsp):
    g = torch.Generator().manual_seed(8)
    z = torch.randn((3, 40, 20000), generator=g).bfloat16()
    N = torch.tensor([40, 1, 0], dtype=torch.int32)
    zg = z.cuda()
    for b in range(3):
        zg[b, int(N[b]):] = math.nan
    _run(lsp, z, _ids(3, 40, 20000, g), N, 20, view=lambda _: zg)


@pytest.mark.parametrize("shape", [(1, 3, 126464), (4, 64, 126464), (2, 300, 5000)])
def test_with_and_without_a_workspace_and_the_same_again(lsp, shape):
    """The numbers follow how a row is cut, the ids do not; the same call gives the same bits."""
    g = torch.Generator().manual_seed(5)
    z = torch.randn(shape, generator=g).bfloat16().cuda()
    ids = torch.randint(0, shape[2], shape[:2], generator=g, dtype=torch.int32).cuda()
    N = torch.full((shape[0],), min(5, shape[1]), dtype=torch.int32, device="cuda")
    need = lsp.token_scores_workspace_bytes(*shape, 20)
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
    a, b, c = (lsp.token_scores(z, ids, N, num_alt=20, out=_out(*shape[:2], 20, ids), workspace=w) for w in (ws, ws, None))
    L = lsp.lib()
    d = _out(*shape[:2], 20, ids)
    import ctypes
    p = lsp._ptr
    assert L.lsp_token_scores(1, p(z), *shape, ctypes.c_int64(0), ctypes.c_int64(0), p(N), p(ids), 20, p(d[0]), p(d[1]), p(d[2]), p(d[3]), None,
                              ctypes.c_size_t(0), lsp._stream()) == 0
    torch.cuda.synchronize()
    for x, y, v, u in zip(a, b, c, d):
        assert torch.equal(x, y) and torch.equal(x, v)
        assert torch.equal(x, u) if x.dtype == torch.int32 else torch.allclose(x, u, rtol=0, atol=float(_bounds(shape[2], torch.tensor(12.0))[1]))


def test_agrees_with_the_confidence_reduction(lsp):
    """The first alternative is the confidence call's id, its probability that call's."""
    z = torch.randn((2, 50, 30000), generator=torch.Generator().manual_seed(9)).bfloat16().cuda()
    ids, prob, margin = lsp.confidence(z)
    lp, h, alt_id, alt = lsp.token_scores(z, ids, num_alt=2)
    assert torch.equal(alt_id[..., 0], ids) and torch.equal(alt[..., 0], lp)
    assert torch.allclose(lp.exp(), prob, rtol=1e-4) and torch.allclose(alt[..., 0] - alt[..., 1], margin, atol=1e-5)


def test_graph_replays_and_other_streams(lsp):
    """Captured beside its own eager calls, which use other workspaces; every replay equals the eager result."""
    g = torch.Generator().manual_seed(4)
    z = torch.randn((2, 6, 100000), generator=g).cuda()
    ids = torch.randint(0, 100000, (2, 6), generator=g, dtype=torch.int32).cuda()
    N = torch.tensor([6, 4], dtype=torch.int32, device="cuda")
    out = _out(2, 6, 20, ids)
    want = lsp.token_scores(z, ids, N, num_alt=20, out=_out(2, 6, 20, ids))
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            lsp.token_scores(z, ids, N, num_alt=20, out=out)
            lsp.token_scores(z, ids, N, num_alt=20, out=out)
    for _ in range(4):
        for t in out:
            t.fill_(-7)
        z2 = lsp.token_scores(z * 2, ids, N, num_alt=20)        # other eager work
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert z2[0].shape == (2, 6)
    got = _out(2, 6, 20, ids)
    with torch.cuda.stream(side):
        lsp.token_scores(z, ids, N, num_alt=20, out=got)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_native_and_general_path_agree(lsp, monkeypatch):
    """The native module takes the ordinary calls and leaves the others to the checks in Python."""
    z = torch.randn((2, 5, 30000), generator=torch.Generator().manual_seed(1)).cuda()
    ids, N = torch.zeros((2, 5), dtype=torch.int32, device="cuda"), torch.tensor([5, 2], dtype=torch.int32, device="cuda")
    cases = [(ids, N, 3), (None, None, 0), (None, N, 32), (ids, None, 0)]
    for t, n, K in cases:
        out = _out(2, 5, K, t)
        assert lsp._nat.token_scores(z, t, n, K, out, None) == 0
        with monkeypatch.context() as m:
            m.setattr(lsp, "_nat", None)
            other = lsp.token_scores(z, t, n, num_alt=K, out=_out(2, 5, K, t))
        assert all(a is b is None or torch.equal(a, b) for a, b in zip(out, other))
    out = _out(2, 5, 3, ids)
    for bad in ((ids.long(), N, 3, out), (ids, N, 4, out), (ids, N, 33, out), (None, N, 3, out), (ids, N.long(), 3, out), (ids, N, 3, out[:3]),
                (ids, N, 3, (None, *out[1:]))):
        assert lsp._nat.token_scores(z, *bad, None) is None
        with pytest.raises(lsp.LspError):
            lsp.token_scores(z, bad[0], bad[1], num_alt=bad[2], out=bad[3])
    assert lsp._nat.token_scores(z[:1, :1].expand(2, 5, 30000), ids, N, 3, out, None) is None
