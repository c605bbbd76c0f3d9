"""lsp_attn_key_weights against the definition in 64 bits."""
import math

import pytest
import torch

from oracle import serving

pytestmark = pytest.mark.gpu
POISON = -1234.5


@pytest.fixture(scope="module")
def lsp():
    import paper_2603_05454_amd as m
    assert torch.cuda.is_available()
    return m


def _operands(B, S, Hq, Hkv, D, C, dtype, layers=1, seed=0, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    q = (torch.randn((layers, B, S, Hq, D), generator=g) * spread).to(dtype)
    k = torch.randn((layers, B, S, Hkv, D), generator=g).to(dtype)
    c = torch.randn((layers, B, C, Hkv, D), generator=g).to(dtype)
    w = torch.rand((layers, B, Hkv, C), generator=g)
    return q, k, c, w


def _close(got, want, before, P, N, C, spread=1.0):
    """A score of unit-variance operands is a sum of D products of mean magnitude 0.64 / sqrt(D): four deviations of a random walk of D roundings
    make 4 sqrt(D) 2^-24 x 0.64 sqrt(D) = 2e-5 at D = 128, twice over (the key's score, and the row's logarithm), as the relative error of a
    probability; a sum of n of them adds at most sqrt(n) roundings on average.  Over all weights these errors are independent."""
    got = got.cpu().double()
    err = (got - want).abs()
    assert (err <= 1e-4 * spread * want.abs() + 1e-9).all(), (err / want.abs().clamp(min=1e-9)).max()
    assert torch.linalg.vector_norm(err) <= 1e-5 * spread * torch.linalg.vector_norm(want)
    for b in range(got.shape[-3]):     # untouched: behind the last key, and sequences without queries
        t = (P[b] + N[b]).clamp(max=C) if N[b] > 0 else 0
        assert torch.equal(got[..., b, :, t:], before[..., b, :, t:].double())


CASES = [   # B, S, Hq, Hkv, D, C, prefix, suffix
    (1, 1, 1, 1, 64, 1, [0], [1]), (1, 1, 4, 4, 128, 40, [33], [1]), (2, 3, 4, 2, 64, 17, [17, 0], [3, 2]), (1, 64, 4, 4, 64, 200, [128], [64]),
    (3, 70, 8, 2, 128, 300, [129, 0, 300], [70, 33, 1]), (2, 33, 7, 1, 128, 100, [31, 64], [32, 33]), (1, 200, 2, 2, 64, 700, [513], [200]),
    (4, 17, 28, 4, 128, 90, [63, 65, 1, 32], [17, 0, 16, 1]), (1, 129, 3, 3, 128, 1300, [1025], [129]), (1, 5, 2, 1, 128, 5000, [4999], [5]),
    (2, 257, 4, 4, 128, 400, [255, 397], [257, 256]), (1, 20, 6, 2, 64, 2100, [2080], [20]), (16, 21, 4, 4, 128, 130, [100 + b for b in range(16)], [1 + b for b in range(16)]),
    # each side of what the kernels divide by: 32 and 64 rows on 768 and 2048 keys, and more of either
    (4, 32, 1, 1, 128, 2100, [2016, 2017, 992, 2100], [32, 32, 32, 1]), (4, 64, 1, 1, 64, 2100, [704, 705, 735, 2080], [64, 64, 33, 20]),
    (3, 65, 2, 1, 128, 1200, [1000, 959, 1200], [32, 33, 65]), (2, 9, 7, 1, 64, 3000, [2900, 950], [9, 9]), (1, 2, 28, 4, 128, 4500, [4400], [2]),
    (1, 600, 7, 1, 64, 300, [200], [600]), (2, 700, 3, 1, 128, 900, [130, 0], [700, 699]), (1, 1400, 4, 1, 64, 64, [40], [1399]),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_the_definition(lsp, dtype, case):
    B, S, Hq, Hkv, D, C, P, N = CASES[case]
    q, k, c, w = _operands(B, S, Hq, Hkv, D, C, dtype, seed=case)
    P, N = (torch.tensor(x, dtype=torch.int32) for x in (P, N))
    for decay in (1.0, 0.75):
        want = serving.key_weights(q[0], k[0], c[0], P, N, w[0], decay)
        got = lsp.attn_key_weights(q[0].cuda(), k[0].cuda(), c[0].cuda(), P.cuda(), N.cuda(), w[0].cuda(), decay=decay)
        _close(got, want, w[0], P, N, C)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_layers_strides_scale_and_steps(lsp, dtype):
    """Three layers in one call, operands that are parts of one projection's output, a scale of the caller's; weights accumulate over calls."""
    B, S, Hq, Hkv, D, C = 2, 50, 6, 2, 64, 120
    g = torch.Generator().manual_seed(1)
    qkv = torch.randn((3, B, S, Hq + 2 * Hkv, D), generator=g).to(dtype)
    cache = torch.randn((3, B, C + 3, Hkv + 1, D), generator=g).to(dtype)
    P, N = torch.tensor([70, 11], dtype=torch.int32), torch.tensor([50, 37], dtype=torch.int32)
    w = torch.rand((3, B, Hkv, C), generator=g)
    dq, dc, dw = qkv.cuda(), cache.cuda(), w.cuda()
    q, k, v = dq[..., :Hq, :], dq[..., Hq:Hq + Hkv, :], dq[..., Hq + Hkv:, :]
    c = dc[:, :, 2:2 + C, 1:]
    un = lambda t: list(t.unbind(0))       # noqa: E731
    table = lsp.AttnLayerTable(un(q), un(k), un(v), un(c), un(c), un(torch.zeros((3, B, S, Hq, D), dtype=dtype, device="cuda")))
    want = w.double()
    for _ in range(2):
        want = torch.stack([serving.key_weights(q[l].cpu(), k[l].cpu(), c[l].cpu(), P, N, want[l], 0.5, 0.2) for l in range(3)])
        lsp.attn_key_weights_layers(table, P.cuda(), N.cuda(), dw, decay=0.5, scale=0.2)
    _close(dw, want, w, P, N, C, spread=2.0)


def test_more_layers_than_one_launch_takes(lsp):
    q, k, c, w = _operands(1, 4, 2, 1, 64, 30, torch.bfloat16, layers=35, seed=2)
    P, N = torch.tensor([20], dtype=torch.int32), torch.tensor([4], dtype=torch.int32)
    dq, dk, dc = (list(t.cuda().unbind(0)) for t in (q, k, c))
    table = lsp.AttnLayerTable(dq, dk, dk, dc, dc, [torch.zeros_like(t) for t in dq])
    got = lsp.attn_key_weights_layers(table, P.cuda(), N.cuda(), w.cuda())
    _close(got, torch.stack([serving.key_weights(q[l], k[l], c[l], P, N, w[l]) for l in range(35)]), w, P, N, 30)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_what_is_not_there_may_hold_anything(lsp, dtype):
    """NaN and infinities in cache rows, suffix rows and weights behind the lengths; with decay 0 in all weights."""
    B, S, Hq, Hkv, D, C = 2, 40, 4, 2, 128, 150
    q, k, c, w = _operands(B, S, Hq, Hkv, D, C, dtype, seed=3)
    P, N = torch.tensor([77, 110], dtype=torch.int32), torch.tensor([33, 39], dtype=torch.int32)
    for b in range(B):
        q[0, b, N[b]:], k[0, b, N[b]:], c[0, b, P[b]:] = math.nan, math.inf, math.nan
    want = serving.key_weights(q[0], k[0], c[0], P, N, torch.full_like(w[0], POISON), 0.0)
    got = lsp.attn_key_weights(q[0].cuda(), k[0].cuda(), c[0].cuda(), P.cuda(), N.cuda(), torch.full_like(w[0], POISON).cuda(), decay=0.0)
    _close(got, want, torch.full_like(w[0], POISON), P, N, C)
    nan = torch.full_like(w[0], math.nan).cuda()
    again = lsp.attn_key_weights(q[0].cuda(), k[0].cuda(), c[0].cuda(), P.cuda(), N.cuda(), nan, decay=0.0)
    there = torch.arange(C)[None, None] < (P + N)[:, None, None].clamp(max=C)
    there = there.expand(B, Hkv, C)
    assert torch.equal(again.cpu()[there], got.cpu()[there]) and torch.isnan(again.cpu()[~there]).all()


def test_lengths_beyond_the_buffers_are_clamped(lsp):
    q, k, c, w = _operands(2, 9, 2, 2, 64, 20, torch.bfloat16, seed=4)
    P, N = torch.tensor([500, -3], dtype=torch.int32), torch.tensor([900, 9], dtype=torch.int32)
    got = lsp.attn_key_weights(q[0].cuda(), k[0].cuda(), c[0].cuda(), P.cuda(), N.cuda(), w[0].cuda())
    P, N = P.clamp(0, 20), N.clamp(0, 9)
    _close(got, serving.key_weights(q[0], k[0], c[0], P, N, w[0]), w[0], P, N, 20)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_far_apart_scores(lsp, dtype):
    """Scores of deviation 8: most rows' mass sits on a few keys, most others' is tiny."""
    q, k, c, w = _operands(1, 60, 4, 4, 64, 400, dtype, seed=5, spread=8.0)
    P, N = torch.tensor([333], dtype=torch.int32), torch.tensor([60], dtype=torch.int32)
    got = lsp.attn_key_weights(q[0].cuda(), k[0].cuda(), c[0].cuda(), P.cuda(), N.cuda(), w[0].cuda())
    _close(got, serving.key_weights(q[0], k[0], c[0], P, N, w[0]), w[0], P, N, 400, spread=8.0)


def test_the_same_bits_at_every_call_and_replay(lsp):
    q, k, c, w = (t[0].cuda() for t in _operands(3, 90, 8, 2, 128, 700, torch.bfloat16, seed=6))
    P, N = torch.tensor([600, 100, 0], dtype=torch.int32, device="cuda"), torch.tensor([90, 41, 7], dtype=torch.int32, device="cuda")
    need = lsp.attn_key_weights_workspace_bytes(lsp.LSP_BF16, 3, 90, 8, 2, 128, 700)
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
    want = lsp.attn_key_weights(q, k, c, P, N, w.clone(), workspace=ws)
    again = lsp.attn_key_weights(q, k, c, P, N, w.clone())
    assert torch.equal(want, again)
    got, graph, side = w.clone(), torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            lsp.attn_key_weights(q, k, c, P, N, got)
    for _ in range(4):
        got.copy_(w)
        lsp.attn_key_weights(q * 2, k, c, P, N, w.clone())
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_mass_of_a_long_batch_adds_up(lsp):
    """At a size where every kernel variant's tiles are many: each row's mass is 1, and sampled keys are those of the definition."""
    B, S, Hq, Hkv, D, C = 2, 520, 8, 8, 128, 2600
    q, k, c, w = _operands(B, S, Hq, Hkv, D, C, torch.bfloat16, seed=7)
    P, N = torch.tensor([2080, 1500], dtype=torch.int32), torch.tensor([520, 411], dtype=torch.int32)
    got = lsp.attn_key_weights(q[0].cuda(), k[0].cuda(), c[0].cuda(), P.cuda(), N.cuda(), torch.zeros_like(w[0]).cuda()).cpu().double()
    assert torch.allclose(got.sum(-1), N[:, None].double().expand(B, Hkv), rtol=1e-5)
    for h in (0, 7):
        want = serving.key_weights(q[0][:, :, h:h + 1], k[0][:, :, h:h + 1], c[0][:, :, h:h + 1], P, N, torch.zeros(B, 1, C))
        _close(got[:, h:h + 1], want, torch.zeros(B, 1, C), P, N, C)


def test_native_and_general_path_agree(lsp, monkeypatch):
    q, k, c, w = (t[0].cuda() for t in _operands(2, 9, 4, 2, 64, 30, torch.float32, seed=8))
    P, N = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([20, 3], [9, 4]))
    table = lsp.AttnLayerTable([q], [k], [k], [c], [c], [torch.zeros_like(q)])
    a, b = w.clone(), w.clone()[None]
    assert lsp._nat.attn_key_weights(q, k, c, P, N, a, 0.5, 0.1, None) == 0
    assert lsp._nat.attn_key_weights_layers(table.desc, 1, table.arrays, P, N, b, 0.5, 0.1, None) == 0
    assert lsp._nat.attn_key_weights(q, k, c, P, N.long(), a, 0.5, 0.1, None) is None
    assert lsp._nat.attn_key_weights(q, k, c, P, N, a[:, :, :29], 0.5, 0.1, None) is None
    assert lsp._nat.attn_key_weights(q, k, c.bfloat16(), P, N, a, 0.5, 0.1, None) is None
    monkeypatch.setattr(lsp, "_nat", None)
    x = lsp.attn_key_weights(q, k, c, P, N, w.clone(), decay=0.5, scale=0.1)
    y = lsp.attn_key_weights_layers(table, P, N, w.clone()[None], decay=0.5, scale=0.1)
    assert torch.equal(a, x) and torch.equal(b, y) and torch.equal(x, y[0])
    with pytest.raises(lsp.LspError, match="decay"):
        lsp.attn_key_weights(q, k, c, P, N, w, decay=-0.1)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_more_units_than_one_pass_of_the_grid(lsp, dtype):
    """Several units to a workgroup, ragged, some without rows, some with more rows than the others' kernel takes."""
    B, S, Hq, Hkv, D, C = 40, 70, 8, 8, 64, 150
    q, k, c, w = _operands(B, S, Hq, Hkv, D, C, dtype, seed=9)
    P = torch.tensor([(37 * b) % 151 for b in range(B)], dtype=torch.int32)
    N = torch.tensor([(29 * b) % 71 for b in range(B)], dtype=torch.int32)
    got = lsp.attn_key_weights(q[0].cuda(), k[0].cuda(), c[0].cuda(), P.cuda(), N.cuda(), w[0].cuda(), decay=0.5)
    _close(got, serving.key_weights(q[0], k[0], c[0], P, N, w[0], 0.5), w[0], P, N, C)


def test_a_second_launch_of_few_layers(lsp):
    """33 layers are a launch of 32 and one of 1, whose units are few enough to be divided further; the workspace is that of the first."""
    B, S, Hq, Hkv, D, C, L = 10, 70, 2, 2, 64, 600, 33
    q, k, c, w = _operands(B, S, Hq, Hkv, D, C, torch.bfloat16, layers=L, seed=10)
    P, N = torch.tensor([500 + b for b in range(B)], dtype=torch.int32), torch.full((B,), 70, dtype=torch.int32)
    dq, dk, dc = (list(t.cuda().unbind(0)) for t in (q, k, c))
    table = lsp.AttnLayerTable(dq, dk, dk, dc, dc, [torch.zeros_like(t) for t in dq])
    need = lsp.attn_key_weights_workspace_bytes(lsp.LSP_BF16, B, S, Hq, Hkv, D, C, L)
    ws = torch.full((need + 4096,), 7, dtype=torch.uint8, device="cuda")
    got = lsp.attn_key_weights_layers(table, P.cuda(), N.cuda(), w.cuda(), workspace=ws[:need])
    assert (ws[need:] == 7).all()
    for l in (0, 31, 32):
        _close(got[l], serving.key_weights(q[l], k[l], c[l], P, N, w[l]), w[l], P, N, C)
