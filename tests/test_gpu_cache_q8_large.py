"""lsp_kv_append_q8 and lsp_kv_read_q8 where a launch has fewer workgroups than there is work: each takes several blocks of rows, four of them at once when it
reads, and past the last cache's 256 MB both go by nontemporal accesses.  Against the definition, value by value."""
import pytest
import torch

from oracle import eight_bits

pytestmark = pytest.mark.gpu
GROUPS = 4096       # workgroups of a launch, where there is work for them
LAST_CACHE = 256 << 20


@pytest.fixture(scope="module")
def lsp():
    import paper_2603_05454_amd as m
    assert torch.cuda.is_available()
    return m


def _same(a, b):
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


def _groups(layers, B, most):
    return max(1, min(-(-GROUPS // (2 * layers * B)), most))


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _rows(shape, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * torch.exp(torch.randn((*shape[:-1], 1), generator=g))).to(dtype)


def _e4m3(shape, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(0, 127, shape, generator=g, dtype=torch.uint8) | torch.randint(0, 2, shape, generator=g, dtype=torch.uint8) << 7


def _near(kv, e, suf, n, P):
    """Every committed row stands for what was written, to half a step of e4m3: 2^-4 of a normal value, 2^-10 units below.  (All heads; the definition,
    number by number, is compared with for some.)"""
    C = kv.shape[1]
    unit = torch.exp2(e.double() - 127).repeat_interleave(32, dim=2)[:, :, :C].transpose(1, 2).unsqueeze(-1)
    got = kv.double() * unit
    for b in range(kv.shape[0]):
        x, at = suf[b, :n[b]].double(), slice(P[b] - n[b], P[b])
        assert ((got[b, at] - x).abs() <= torch.maximum(x.abs() / 16, unit[b, at] * 2.0 ** -10)).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_of_more_blocks_than_waves(lsp, dtype, D):
    """Eight layers of eight sequences: 32 workgroups, 128 waves, and up to 13 blocks of 21 heads for them, so two and three blocks to a wave.  The first
    blocks have rows from before, under larger and smaller scales."""
    L, B, S, H, C = 8, 8, 400, 21, 450
    assert _groups(L, B, -(-(-(-(S + 32) // 32) * H) // 4)) * 4 < 12 * H
    n = [400, 399, 369, 33, 1, 0, 385, 400]
    P = [450, 400, 400, 64, 33, 40, 418, 433]
    suf = [_rows((B, S, H, D), dtype, s) for s in (1, 2)]
    val = [_e4m3((B, C, H, D), s) for s in (3, 4)]
    sc = [torch.randint(112, 130, (B, H, -(-C // 32)), generator=torch.Generator().manual_seed(s), dtype=torch.uint8) for s in (5, 6)]
    kv = [v.cuda().expand(L, *v.shape).contiguous().view(torch.float8_e4m3fn) for v in val]
    e = [s.cuda().expand(L, *s.shape).contiguous() for s in sc]
    un = lambda t: list(t.unbind(0))       # noqa: E731
    table = lsp.Q8LayerTable([suf[0].cuda()] * L, [suf[1].cuda()] * L, un(kv[0]), un(kv[1]), un(e[0]), un(e[1]))
    lsp.kv_append_q8(table, _i32(n), _i32(P))
    heads = [0, 9, H - 1]
    for i in range(2):
        raw = kv[i].view(torch.uint8)
        assert (raw == raw[:1]).all() and (e[i] == e[i][:1]).all()
        _near(kv[i][0], e[i][0], suf[i].cuda(), n, P)
        want, E = eight_bits.append(suf[i][:, :, heads], val[i][:, :, heads].view(torch.float8_e4m3fn), sc[i][:, heads], n, P)
        assert _same(kv[i][0][:, :, heads].cpu().double(), want) and torch.equal(e[i][0][:, heads].cpu().to(torch.int64), E)


@pytest.mark.parametrize("more", range(5))
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_read_of_more_rows_than_threads(lsp, dtype, D, more):
    """Eight layers of eight sequences: 32 workgroups read 32 x 4096 / D rows of heads at a time, four such steps at once and what is left singly.  The
    sequences' rows are one to ten steps, none to three of them left over, whole ones and such that end inside a step."""
    L, B, H = 8, 8, 5
    step = 32 * (256 * 16 // D)
    assert _groups(L, B, 1 << 20) == 32
    steps = [1 + more, 2 + more, 3 + more, 4 + more, 5 + more, 4, 8, 9]
    count = [max(1, -(-k * step // H) - (i % 3)) for i, k in enumerate(steps)]
    C = max(count) + 40
    val = _e4m3((B, C, H, D), 7).cuda()
    sc = torch.randint(100, 140, (B, H, -(-C // 32)), generator=torch.Generator().manual_seed(8), dtype=torch.uint8).cuda()
    kc = val.view(torch.float8_e4m3fn)
    first = [(5 * b) % 33 for b in range(B)]
    suf = torch.zeros((B, 1, H, D), dtype=dtype, device="cuda")
    table = lsp.Q8LayerTable([suf] * L, [suf] * L, [kc] * L, [kc] * L, [sc] * L, [sc] * L)
    R = max(count) + 3
    out = torch.full((2, L, B, R, H, D), 7.0, dtype=dtype, device="cuda")
    un = lambda t: list(t.unbind(0))       # noqa: E731
    lsp.kv_read_q8(table, _i32(first), _i32([a + c for a, c in zip(first, count)]), un(out[0]), un(out[1]))
    want = torch.full((B, R, H, D), 7.0, dtype=torch.float64)
    values = eight_bits.values(kc.cpu(), sc.cpu())
    for b in range(B):
        want[b, :count[b]] = values[b, first[b]:first[b] + count[b]]
    assert torch.equal(out[0, 0].cpu().double(), want)       # (these scales' values are exact in both types)
    assert (out == out[:1, :1]).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_buffers_beyond_the_last_cache(lsp, dtype, D):
    """One layer's operands, as every layer's: 32 layers' buffers count as more than 256 MB."""
    L, B, S, H, C = 32, 3, 1030, 24, 1100
    assert 2 * L * B * S * H * D * (4 if dtype == torch.float32 else 2) > LAST_CACHE
    n, P = [1030, 700, 1], [1100, 1051, 65]
    suf = [_rows((B, S, H, D), dtype, s) for s in (11, 12)]
    val = [_e4m3((B, C, H, D), s) for s in (13, 14)]
    sc = [torch.randint(112, 130, (B, H, -(-C // 32)), generator=torch.Generator().manual_seed(s), dtype=torch.uint8) for s in (15, 16)]
    kv = [v.cuda().expand(L, *v.shape).contiguous().view(torch.float8_e4m3fn) for v in val]
    e = [s.cuda().expand(L, *s.shape).contiguous() for s in sc]
    un = lambda t: list(t.unbind(0))       # noqa: E731
    table = lsp.Q8LayerTable([suf[0].cuda()] * L, [suf[1].cuda()] * L, un(kv[0]), un(kv[1]), un(e[0]), un(e[1]))
    lsp.kv_append_q8(table, _i32(n), _i32(P))
    out = [torch.full((L, B, S, H, D), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    first, end = [70, 31, 0], [1100, 1051, 65]
    lsp.kv_read_q8(table, _i32(first), _i32(end), un(out[0]), un(out[1]))
    heads = [0, 5, H - 1]
    for i in range(2):
        raw = kv[i].view(torch.uint8)
        assert (raw == raw[:1]).all() and (e[i] == e[i][:1]).all() and (out[i] == out[i][:1]).all()
        _near(kv[i][0], e[i][0], suf[i].cuda(), n, P)
        want, E = eight_bits.append(suf[i][:, :, heads], val[i][:, :, heads].view(torch.float8_e4m3fn), sc[i][:, heads], n, P)
        assert _same(kv[i][0][:, :, heads].cpu().double(), want) and torch.equal(e[i][0][:, heads].cpu().to(torch.int64), E)
        read = torch.full((B, S, len(heads), D), 7.0, dtype=torch.float64)
        values = eight_bits.values(want, E)
        for b in range(B):
            m = min(end[b] - first[b], S)
            read[b, :m] = values[b, first[b]:first[b] + m]
        assert torch.equal(out[i][0][:, :, heads].cpu().double(), read)
