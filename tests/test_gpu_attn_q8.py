"""lsp_attn_step_q8 against the definition in 64 bits."""
import math

import pytest
import torch

from oracle import eight_bits

pytestmark = pytest.mark.gpu
POISON = -768.0


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


def _cache(shape, g, scales=(110, 125)):
    """Random values of a cache: bytes of all sizes, their sum of squares that of a few units."""
    val = (torch.randn(shape, generator=g) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
    return val, torch.randint(*scales, (*shape[:-3], shape[-2], -(-shape[-3] // 32)), generator=g, dtype=torch.uint8)


def _operands(B, S, Hq, H, D, C, P, N, seed, layers=1, poison=True, size=1.0):
    g = torch.Generator().manual_seed(seed)
    q = (torch.randn((layers, B, S, Hq, D), generator=g) * size).to(torch.bfloat16)
    ks, vs = (torch.randn((layers, B, S, H, D), generator=g).to(torch.bfloat16) for _ in range(2))
    (kc, ke), (vc, ve) = (_cache((layers, B, C, H, D), g, (119, 122)) for _ in range(2))
    if poison:      # what is not there is NaN, with scales that are none
        for b in range(B):
            p, n = min(max(P[b], 0), C), min(max(N[b], 0), S)
            for c, e in ((kc, ke), (vc, ve)):
                c.view(torch.uint8)[:, b, p:] = 0x7f
                e[:, b, :, -(-p // 32):] = 255
            for x in (q, ks, vs):
                x[:, b, n:] = math.nan
    return q, ks, vs, kc, vc, ke, ve


def _close(got, want, mass, N, S):
    """Each probability is rounded to bf16, 2^-8 of it at most, which adds up to that much of the sum of |v|; the scores' own errors (sums of up to 128
    products in fp32, a few units of 2^-24 of a score of up to about 50) and the sum's stay below 2^-12; and the result is rounded."""
    got = got.cpu().double()
    for b in range(got.shape[0]):
        n = min(max(int(N[b]), 0), S)
        tol = (2.0 ** -8 + 2.0 ** -12) * mass[b, :n] + 2.0 ** -8 * want[b, :n].abs()
        err = (got[b, :n] - want[b, :n]).abs()
        assert not got[b, :n].isnan().any()
        assert (err <= tol).all(), ((err / tol).max(), b)
        assert (got[b, n:] == POISON).all()


CASES = [   # B, S, Hq, Hkv, D, C, prefix, suffix
    (1, 1, 1, 1, 64, 1, [0], [1]), (1, 1, 4, 4, 128, 40, [33], [1]), (2, 3, 4, 2, 64, 17, [17, 0], [3, 2]), (1, 64, 4, 4, 64, 200, [128], [64]),
    (3, 70, 8, 2, 128, 300, [129, 0, 300], [70, 33, 1]), (2, 33, 7, 1, 128, 100, [31, 64], [32, 33]), (1, 200, 2, 2, 64, 700, [513], [200]),
    (4, 17, 28, 4, 128, 90, [63, 65, 1, 32], [17, 0, 16, 1]), (1, 129, 3, 3, 128, 1300, [1025], [129]), (1, 5, 2, 1, 128, 5000, [4999], [5]),
    (2, 257, 4, 4, 128, 400, [255, 397], [257, 256]), (16, 21, 4, 4, 128, 130, [100 + b for b in range(16)], [1 + b for b in range(16)]),
    (3, 7, 2, 2, 64, 70, [-5, 99, 32], [9, 7, -1]), (1, 2, 28, 4, 128, 2500, [2400], [2]), (1, 600, 7, 1, 64, 300, [200], [600]),
    (2, 300, 3, 1, 128, 900, [130, 0], [300, 299]), (1, 1, 2, 2, 64, 8000, [7999], [1]), (3, 40, 8, 8, 64, 1000, [1000, 31, 500], [40, 40, 7]),
    (5, 9, 14, 2, 128, 700, [700, 1, 640, 639, 641], [9, 9, 9, 5, 1]), (2, 512, 8, 8, 128, 600, [600, 577], [512, 100]), (1, 1025, 2, 2, 128, 64, [0], [1025])]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_the_definition(lsp, case):
    B, S, Hq, H, D, C, P, N = CASES[case]
    t = _operands(B, S, Hq, H, D, C, P, N, case)
    one = [x[0] for x in t]
    want, mass = eight_bits.attention(*one[:3], eight_bits.values(one[3], one[5]), eight_bits.values(one[4], one[6]), P, N)
    out = torch.full((B, S, Hq, D), POISON, dtype=torch.bfloat16, device="cuda")
    lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (P, N)]
    d = [x.cuda() for x in one]
    assert lsp.attn_step_q8(*d, *lens, out=out) is out
    _close(out, want, mass, N, S)
    again = torch.full_like(out, POISON)
    lsp.attn_step_q8(*d, *lens, out=again)
    assert torch.equal(out, again)


def test_layers_strides_and_scale(lsp, marshalled):
    """Three layers in one call, operands that are parts of larger buffers, a scale of the caller's."""
    B, S, Hq, H, D, C, L = 2, 50, 6, 2, 64, 120, 3
    g = torch.Generator().manual_seed(1)
    P, N = [70, 11], [50, 37]
    qkv = torch.randn((L, B, S, Hq + 2 * H, D), generator=g).to(torch.bfloat16).cuda()
    val, e = zip(*[_cache((L, B, C + 3, H + 1, D), g, (119, 122)) for _ in range(2)])
    dev = [v.cuda()[:, :, 2:2 + C, 1:] for v in val]
    sc = [torch.randint(119, 122, (L, B, H, 4), generator=g, dtype=torch.uint8) for _ in range(2)]
    buf = torch.full((L, B, S + 1, Hq + 1, D), POISON, dtype=torch.bfloat16, device="cuda")
    q, k, v, out = qkv[..., :Hq, :], qkv[..., Hq:Hq + H, :], qkv[..., Hq + H:, :], buf[:, :, 1:, 1:]
    un = lambda t: list(t.unbind(0))       # noqa: E731
    dsc = [s.cuda() for s in sc]
    table = lsp.Q8LayerTable(un(k), un(v), un(dev[0]), un(dev[1]), un(dsc[0]), un(dsc[1]), q=un(q), out=un(out))
    lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (P, N)]
    assert lsp.attn_step_q8_layers(table, *lens, scale=0.2) is table.out
    for l in range(L):
        kv = [eight_bits.values(val[i][l, :, 2:2 + C, 1:].contiguous(), sc[i][l]) for i in range(2)]
        want, mass = eight_bits.attention(q[l].cpu(), k[l].cpu(), v[l].cpu(), *kv, P, N, scale=0.2)
        _close(out[l], want, mass, N, S)
        one = torch.full((B, S, Hq, D), POISON, dtype=torch.bfloat16, device="cuda")
        lsp.attn_step_q8(q[l], k[l], v[l], dev[0][l], dev[1][l], dsc[0][l], dsc[1][l], *lens, scale=0.2, out=one)
        _close(one, want, mass, N, S)
    assert (buf[:, :, 0] == POISON).all() and (buf[:, :, :, 0] == POISON).all()


def test_more_layers_than_one_launch_takes(lsp):
    B, S, Hq, H, D, C, P, N, L = 2, 6, 4, 2, 128, 80, [70, 3], [6, 2], 35
    t = [x.cuda() for x in _operands(B, S, Hq, H, D, C, P, N, 3, layers=L)]
    lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (P, N)]
    out = torch.full((L, B, S, Hq, D), POISON, dtype=torch.bfloat16, device="cuda")
    un = lambda x: list(x.unbind(0))       # noqa: E731
    lsp.attn_step_q8_layers(lsp.Q8LayerTable(*[un(x) for x in t[1:]], q=un(t[0]), out=un(out)), *lens)
    for l in (0, 17, 31, 32, 34):
        one = [x[l].cpu() for x in t]
        want, mass = eight_bits.attention(*one[:3], eight_bits.values(one[3], one[5]), eight_bits.values(one[4], one[6]), P, N)
        _close(out[l], want, mass, N, S)


@pytest.mark.parametrize("S, N", [(3, 3), (40, 2), (300, 300)])
def test_scores_far_apart_and_references_that_move(lsp, S, N):
    """Scores of hundreds, keys that come late and outweigh all before, and rows for which they are the least."""
    B, Hq, H, D, C, P = 1, 4, 2, 128, 700, 650
    t = _operands(B, S, Hq, H, D, C, [P], [N], 9, size=8.0)
    one = [x[0] for x in t]
    one[0][0, :N, 0] = one[0][0, :N, 0].abs()
    one[3].view(torch.uint8)[0, 600, 0] = 0x70        # a key of 128s
    want, mass = eight_bits.attention(*one[:3], eight_bits.values(one[3], one[5]), eight_bits.values(one[4], one[6]), [P], [N])
    out = torch.full((B, S, Hq, D), POISON, dtype=torch.bfloat16, device="cuda")
    lens = [torch.tensor([x], dtype=torch.int32, device="cuda") for x in (P, N)]
    lsp.attn_step_q8(*[x.cuda() for x in one], *lens, out=out)
    got = out.cpu().double()[0, :N]
    # scores of up to 2000 in fp32: sums of 128 products of up to 16 each, 2^-24 of 2000 per rounding, 128 of them at most in a key's score
    tol = (2.0 ** -8 + 2.0 ** -12 + 128 * 2000 * 2.0 ** -24) * mass[0, :N] + 2.0 ** -8 * want[0, :N].abs()
    assert ((got - want[0, :N]).abs() <= tol).all()


def test_infinities_and_nan_reach_only_their_rows(lsp):
    """A NaN among one head's cached keys makes that head's rows NaN, and no others; one in a suffix value that element's column."""
    B, S, Hq, H, D, C, P, N = 2, 20, 4, 2, 64, 100, [90, 64], [20, 20]
    t = [x[0] for x in _operands(B, S, Hq, H, D, C, P, N, 4)]
    t[3].view(torch.uint8)[0, 40, 1, 3] = 0x7f
    t[2][1, 7, 0, 5] = math.nan
    out = torch.zeros((B, S, Hq, D), dtype=torch.bfloat16, device="cuda")
    lsp.attn_step_q8(*[x.cuda() for x in t], *[torch.tensor(x, dtype=torch.int32, device="cuda") for x in (P, N)], out=out)
    bad = out.isnan().cpu()
    assert bad[0, :, 2:].all() and not bad[0, :, :2].any()
    assert bad[1, :, :2, 5].all() and bad[1].sum() == 20 * 2


def test_offsets_beyond_32_bits(lsp):
    """The last rows of a cache of more than 2^31 bytes, against the same rows at the front of a small one."""
    B, S, H, D, C, P = 2, 4, 32, 128, 300000, 299999
    g = torch.Generator(device="cuda").manual_seed(2)
    q, ks, vs = (torch.randn((B, S, H, D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    val = torch.randint(0, 100, (B, C, H, D), generator=g, device="cuda", dtype=torch.uint8)
    kc = val.view(torch.float8_e4m3fn)
    sc = torch.full((B, H, C // 32), 118, dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(q)
    lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([P] * B, [S] * B)]
    lsp.attn_step_q8(q, ks, vs, kc, kc, sc, sc, *lens, out=out)
    for b in range(B):
        for h in (0, 31):
            k = torch.cat([kc[b, :P, h].double() * 2.0 ** -9, ks[b, :, h].double()])
            v = torch.cat([kc[b, :P, h].double() * 2.0 ** -9, vs[b, :, h].double()])
            p = torch.softmax(q[b, :, h].double() @ k.T.contiguous() / math.sqrt(D), dim=1)
            want, mass = p @ v, p @ v.abs()
            tol = (2.0 ** -8 + 2.0 ** -12) * mass + 2.0 ** -8 * want.abs()
            assert ((out[b, :, h].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("S, N", [(8, [8, 3]), (140, [140, 9])])
def test_streams_workspaces_and_graphs(lsp, marshalled, S, N):
    """Calls on two streams at once, and two captured graphs that replay in turn with eager calls in between."""
    B, Hq, H, D, C = 2, 8, 2, 128, 1500
    sets = []
    for seed in range(2):
        P = [1400 - 100 * seed, 31]
        t = [x[0].cuda() for x in _operands(B, S, Hq, H, D, C, P, N, seed)]
        lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (P, N)]
        want = torch.full((B, S, Hq, D), POISON, dtype=torch.bfloat16, device="cuda")
        lsp.attn_step_q8(*t, *lens, out=want)
        sets.append((t, lens, want, torch.full_like(want, POISON)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        for (t, lens, want, out), s in zip(sets, streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                out.fill_(POISON)
                lsp.attn_step_q8(*t, *lens, out=out)
        torch.cuda.synchronize()
        for t, lens, want, out in sets:
            assert torch.equal(out, want)
    ws = torch.empty(max(16, lsp.attn_q8_workspace_bytes(B, S, Hq, H, D, C)), dtype=torch.uint8, device="cuda")     # one for both: replays are in order
    graphs = []
    for t, lens, want, out in sets:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            lsp.attn_step_q8(*t, *lens, out=out, workspace=ws)
    for _ in range(3):
        for gr, (t, lens, want, out) in zip(graphs, sets):
            out.fill_(POISON)
            gr.replay()
            got = out.clone()
            lsp.attn_step_q8(*t, *lens, out=out)
            assert torch.equal(got, want) and torch.equal(out, want)


def test_a_workspace_that_will_not_do(lsp, marshalled):
    B, S, Hq, H, D, C, P, N = 1, 2, 4, 1, 128, 4000, [3999], [2]
    t = [x[0] for x in _operands(B, S, Hq, H, D, C, P, N, 6)]
    want, mass = eight_bits.attention(*t[:3], eight_bits.values(t[3], t[5]), eight_bits.values(t[4], t[6]), P, N)
    lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (P, N)]
    d = [x.cuda() for x in t]
    for ws in (None, torch.empty(8, dtype=torch.uint8, device="cuda"), torch.empty(1 << 22, dtype=torch.uint8, device="cuda")[1:], torch.empty(1 << 22, dtype=torch.uint8)):
        out = torch.full((B, S, Hq, D), POISON, dtype=torch.bfloat16, device="cuda")
        lsp.attn_step_q8(*d, *lens, out=out, workspace=ws)
        _close(out, want, mass, N, S)


def _run(lsp, B, S, Hq, H, D, C, P, N, seed, copies=1):
    """A call whose layers are the same operands `copies` times, against the definition and each other."""
    t = [x[0] for x in _operands(B, S, Hq, H, D, C, P, N, seed)]
    want, mass = eight_bits.attention(*t[:3], eight_bits.values(t[3], t[5]), eight_bits.values(t[4], t[6]), P, N)
    lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (P, N)]
    q, *rest = [x.cuda() for x in t]
    out = torch.full((copies, B, S, Hq, D), POISON, dtype=torch.bfloat16, device="cuda")
    table = lsp.Q8LayerTable(*[[x] * copies for x in rest], q=[q] * copies, out=list(out.unbind(0)))
    lsp.attn_step_q8_layers(table, *lens)
    _close(out[0], want, mass, N, S)
    assert all(torch.equal(o, out[0]) for o in out[1:])


EDGES = [15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 513]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("turn", [0, 7])
def test_every_tile_in_one_batch(lsp, D, turn):
    """Rows at the edges of the tiles, on prefixes at the edges of blocks and steps."""
    P = [0, 1, 31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 128, 129, 300, 5]
    _run(lsp, 16, 520, 2, 2, D, 300, P[turn:] + P[:turn], EDGES, 50 + turn)


WHOLE = [   # ..., copies: work enough that a workgroup has several heads; keys that are divided among workgroups, in each kind of tile; more than 64 sequences
    (9, 5, 8, 4, 128, 2300, [2300 - b for b in range(9)], [5, 4, 0, 3, 2, 1, 5, 5, 5], 32), (9, 6, 12, 6, 64, 2300, [2299] * 9, [3] * 9, 24),
    (9, 33, 4, 4, 128, 1100, [1100] * 9, [33, 17, 32, 33, 1, 33, 33, 16, 33], 12), (5, 3, 5, 5, 128, 2300, [2300, 1, 2200, 2111, 2300], [3] * 5, 32),
    (1, 20, 8, 8, 128, 66000, [65990], [20], 1), (1, 33, 6, 6, 64, 66000, [65999], [33], 1), (1, 4, 3, 3, 128, 66000, [65999], [3], 2),
    (1, 100, 2, 2, 128, 6000, [5950], [100], 1), (1, 100, 2, 2, 64, 6000, [5950], [100], 1), (1, 300, 2, 2, 128, 6000, [6000], [300], 1),
    (2, 300, 4, 2, 128, 4000, [3990, 10], [130, 300], 1), (5, 300, 16, 16, 128, 9000, [9000, 8999, 9000, 100, 8970], [17, 3, 33, 300, 16], 1),
    (130, 9, 3, 3, 64, 50, [(7 * b) % 51 for b in range(130)], [b % 10 for b in range(130)], 1),
    (70, 12, 4, 2, 128, 2100, [(301 * b) % 2101 for b in range(70)], [b % 13 for b in range(70)], 1)]


@pytest.mark.parametrize("case", range(len(WHOLE)))
def test_work_is_dealt_out_whole(lsp, case):
    *shape, copies = WHOLE[case]
    _run(lsp, *shape, 70 + case, copies)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S, Hq, P, first", [(40, 2, 0, 32), (64, 2, 70, 33), (140, 2, 0, 64), (140, 2, 33, 96), (300, 2, 0, 32), (3, 8, 0, 1), (40, 2, 2100, 40)])
def test_scores_of_minus_infinity_weigh_nothing(lsp, D, S, Hq, P, first):
    """The first suffix keys' scores are -infinity: a whole block's, a step's, all that a wave meets."""
    B, H = 2, 2
    t = [x[0] for x in _operands(B, S, Hq, H, D, P + 20, [P, P], [S, S - 1], 6)]
    t[0][..., 0] = t[0][..., 0].abs() + 0.5
    t[1][:, :first, :, 0] = -math.inf
    if P == 0 and first >= S - 1:
        t[1][:, S - 1:, :, 0] = 0.0
    N = [S, S - 1]
    want, mass = eight_bits.attention(*t[:3], eight_bits.values(t[3], t[5]), eight_bits.values(t[4], t[6]), [P, P], N)
    assert not want[0].isnan().any()
    out = torch.full((B, S, Hq, D), POISON, dtype=torch.bfloat16, device="cuda")
    lsp.attn_step_q8(*[x.cuda() for x in t], *[torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([P, P], N)], out=out)
    _close(out, want, mass, N, S)


@pytest.mark.parametrize("B, H, L, P", [(8, 32, 1, 1900), (1, 32, 16, 1000), (3, 16, 8, 1300), (2, 20, 9, 1500)])
def test_few_heads_beside_each_other(lsp, B, H, L, P):
    """Work enough for heads beside each other, but not for all workgroups: fewer heads to each."""
    N = [4 - b % 3 for b in range(B)]
    _run(lsp, B, 4, H, H, 64, P + 10, [P - b for b in range(B)], N, 90 + H, L)
