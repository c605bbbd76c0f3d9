"""lsp_kv_append_q8 and lsp_kv_read_q8 against the definition: every value has to be equal."""
import math

import pytest
import torch

from oracle import eight_bits

pytestmark = pytest.mark.gpu
POISON = 0x55


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


def _same(a, b):
    a, b = a.double(), b.double()
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


def _start(layers, B, C, H, D, filled, g):
    """Caches of bytes that are all numbers, with scales near 1; beyond `filled` rows they hold the poison."""
    kv = [torch.randint(0, 127, (layers, B, C, H, D), generator=g, dtype=torch.uint8) | torch.randint(0, 2, (layers, B, C, H, D), generator=g, dtype=torch.uint8) << 7
          for _ in range(2)]
    sc = [torch.randint(115, 130, (layers, B, H, -(-C // 32)), generator=g, dtype=torch.uint8) for _ in range(2)]
    for t, s in zip(kv, sc):
        for b in range(B):
            t[:, b, filled[b]:] = POISON
            s[:, b, :, -(-filled[b] // 32):] = POISON
    return kv, sc


def _check(lsp, dtype, layers, B, S, H, D, C, P, n, seed=0, size=1.0, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    P, n = torch.tensor(P, dtype=torch.int32), torch.tensor(n, dtype=torch.int32)
    before = [min(max(int(p), 0), C) - min(max(int(k), 0), S, min(max(int(p), 0), C)) for p, k in zip(P, n)]
    kv, sc = _start(layers, B, C, H, D, before, g)
    suf = [(torch.randn((layers, B, S, H, D), generator=g) * size * torch.exp(spread * torch.randn((layers, B, S, H, 1), generator=g))).to(dtype) for _ in range(2)]
    dkv = [t.cuda().view(torch.float8_e4m3fn) for t in kv]
    dsc, dsuf = [t.cuda() for t in sc], [t.cuda() for t in suf]
    table = lsp.Q8LayerTable(*[list(t.unbind(0)) for t in (*dsuf, *dkv, *dsc)])
    for _ in range(2):      # the second call changes nothing
        lsp.kv_append_q8(table, n.cuda(), P.cuda())
        for i in range(2):
            for l in range(layers):
                val, E = eight_bits.append(suf[i][l], kv[i][l].view(torch.float8_e4m3fn), sc[i][l], n, P)
                assert torch.equal(dsc[i][l].cpu().to(torch.int64), E)
                got = dkv[i][l].cpu()
                assert _same(got, val)
                for b in range(B):
                    p = min(max(int(P[b]), 0), C)
                    assert (got.view(torch.uint8)[b, p:] == POISON).all()
                    full = before[b] // 32 * 32       # whole blocks of rows from before: the same bytes
                    assert torch.equal(got.view(torch.uint8)[b, :full], kv[i][l][b, :full])
    return dkv, dsc


CASES = [   # B, S, H, D, C, P (with the new rows), new rows
    (1, 1, 1, 64, 1, [1], [1]), (1, 4, 2, 128, 40, [1], [1]), (2, 40, 3, 64, 70, [31, 32], [31, 32]), (2, 40, 1, 128, 70, [33, 70], [33, 40]),
    (3, 64, 2, 64, 100, [64, 65, 40], [1, 33, 0]), (1, 200, 4, 128, 333, [333], [200]), (4, 5, 5, 64, 64, [0, 64, 32, 33], [3, 5, 5, 2]),
    (2, 7, 2, 64, 50, [-3, 99], [4, 9]), (1, 6, 2, 128, 33, [3], [6]), (2, 31, 7, 64, 63, [62, 63], [31, 30])]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_append(lsp, marshalled, dtype, case):
    B, S, H, D, C, P, n = CASES[case]
    _check(lsp, dtype, 1 + case % 2, B, S, H, D, C, P, n, seed=case)


@pytest.mark.parametrize("size", [0.0, 1e-39, 1e-30, 1e-3, 1e3, 1e30, 1e37])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_of_any_size(lsp, dtype, size):
    """Rows that are all zero, far below and far above what the block holds so far."""
    _check(lsp, dtype, 1, 2, 40, 2, 64, 90, [50, 81], [21, 40], seed=3, size=size, spread=3.0 if size < 1e36 else 0.2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_of_what_is_not_finite(lsp, dtype):
    g = torch.Generator().manual_seed(5)
    x = torch.randn((1, 40, 2, 64), generator=g)
    x[0, 3, 0, 5], x[0, 4, 0, 6], x[0, 5, 1, 7], x[0, 33, 1] = math.nan, math.inf, -math.inf, math.nan
    x[0, 9, 1, 0] = 3.3e38
    x = x.to(dtype)
    kc, vc, ke, ve = lsp.q8_cache(1, 64, 2, 64)
    table = lsp.Q8LayerTable([x.cuda()], [x.cuda()], [kc], [vc], [ke], [ve])
    n = torch.tensor([40], dtype=torch.int32)
    lsp.kv_append_q8(table, n.cuda(), n.cuda())
    val, E = eight_bits.append(x, torch.zeros(1, 64, 2, 64).to(torch.float8_e4m3fn), torch.ones(1, 2, 2, dtype=torch.uint8), n, n)
    assert val.isnan().sum() == 3 + 64
    for c, s in ((kc, ke), (vc, ve)):
        assert _same(c.cpu(), val) and torch.equal(s.cpu().to(torch.int64), E)
    out = [torch.zeros((1, 40, 2, 64), device="cuda") for _ in range(2)]
    lsp.kv_read_q8(table, torch.zeros(1, dtype=torch.int32, device="cuda"), n.cuda(), [out[0]], [out[1]])
    assert _same(out[0].cpu(), eight_bits.values(val, E)[:, :40]) and _same(out[1].cpu(), eight_bits.values(val, E)[:, :40])


def test_rows_one_at_a_time(lsp):
    """Forty steps of one row: a block's exponent only grows, and every value is within half a step of e4m3 of what was written (a second
    rounding, under a larger exponent, is of what fell below its normal range alone)."""
    g = torch.Generator().manual_seed(7)
    x = (torch.randn((40, 1, 1, 2, 64), generator=g) * torch.exp2(torch.arange(40).view(40, 1, 1, 1, 1) % 7)).to(torch.bfloat16)
    kc, vc, ke, ve = lsp.q8_cache(1, 70, 2, 64)
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    for t in range(40):
        table = lsp.Q8LayerTable([x[t].cuda()], [x[t].cuda()], [kc], [vc], [ke], [ve])
        lsp.kv_append_q8(table, one, one * (t + 1))
        E = ke[0, :, t // 32]
        assert t % 32 == 0 or (E >= last).all()
        last = E.clone()
    out = [torch.zeros((1, 40, 2, 64), device="cuda") for _ in range(2)]
    lsp.kv_read_q8(table, one * 0, one * 40, [out[0]], [out[1]])
    want = x[:, 0, 0].double()
    unit = torch.pow(2.0, eight_bits.BLOCK * 0 + ke[0].cpu().double() - 127).repeat_interleave(32, dim=1)[:, :40].T.unsqueeze(-1)
    # half a step of a normal value, 2^-4 of it; below 2^-6 units, half a step there and once more for the second rounding
    assert ((out[0][0].cpu().double() - want).abs() <= torch.maximum(want.abs() * 2.0 ** -4, unit * 2.0 ** -10 * 2)).all()
    assert torch.equal(out[0], out[1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_read_every_byte_under_every_scale(lsp, marshalled, dtype):
    codes = torch.arange(256, dtype=torch.uint8).view(4, 64)
    C = 246 * 32
    cache = codes.repeat(C // 4, 1).view(1, C, 1, 64).contiguous()
    scale = torch.arange(1, 247, dtype=torch.uint8).view(1, 1, 246)
    k = cache.cuda().view(torch.float8_e4m3fn)
    suf = torch.zeros((1, 1, 1, 64), dtype=dtype, device="cuda")
    table = lsp.Q8LayerTable([suf], [suf], [k], [k], [scale.cuda()], [scale.cuda()])
    out = [torch.full((1, C + 3, 1, 64), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    at = lambda x: torch.tensor([x], dtype=torch.int32, device="cuda")      # noqa: E731
    lsp.kv_read_q8(table, at(0), at(C), [out[0]], [out[1]])
    want = eight_bits.values(cache.view(torch.float8_e4m3fn), scale)
    for o in out:
        got = o.cpu().double()
        assert (got[:, C:] == 7).all()
        first = 0 if dtype == torch.float32 else 9 * 32
        assert _same(got[:, first:C], want[:, first:])
        # bf16's subnormal numbers are 2^-133 apart
        assert ((got[:, :C] - want).abs().nan_to_num(0) <= (0 if dtype == torch.float32 else 2.0 ** -134)).all()


@pytest.mark.parametrize("rows", [([0, 5, 33], [1, 70, 33]), ([31, -4, 64], [33, 200, 20]), ([69, 1, 0], [70, 1, 64])])
def test_read_ranges_strides_and_layers(lsp, marshalled, rows):
    """35 layers in two launches, caches and outputs that are parts of larger buffers; rows that are not read are left as they are."""
    g = torch.Generator().manual_seed(11)
    B, C, H, D, R, L = 3, 70, 2, 64, 37, 35
    raw = torch.randint(0, 127, (2, L, B, C + 5, H + 1, D), generator=g, dtype=torch.uint8)
    sc = torch.randint(100, 140, (2, L, B, H, 3), generator=g, dtype=torch.uint8)
    d = raw.cuda().view(torch.float8_e4m3fn)[:, :, :, 3:3 + C, 1:]
    out = torch.full((2, L, B, R + 1, H + 2, D), 7.0, device="cuda")
    o = out[:, :, :, 1:, 2:]
    suf = [torch.zeros((B, 1, H, D), device="cuda")] * L
    un = lambda t: list(t.unbind(0))       # noqa: E731
    dsc = sc.cuda()
    table = lsp.Q8LayerTable(suf, suf, un(d[0]), un(d[1]), un(dsc[0]), un(dsc[1]))
    first, end = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in rows)
    lsp.kv_read_q8(table, first, end, un(o[0]), un(o[1]))
    got = out.cpu()
    want = torch.full_like(got, 7.0)
    for i in range(2):
        for l in range(0, L, 17):
            val = eight_bits.values(raw[i, l, :, 3:3 + C, 1:].contiguous().view(torch.float8_e4m3fn), sc[i, l])
            for b, (a, z) in enumerate(zip(*rows)):
                a = min(max(a, 0), C)
                n = min(max(min(z, C) - a, 0), R)
                want[i, l, b, 1:1 + n, 2:] = val[b, a:a + n].float()
            assert torch.equal(got[i, l], want[i, l])


def test_append_strided_and_many_layers(lsp, marshalled):
    """Keys and values as parts of one projection's output, caches as parts of larger ones, more layers than one launch takes."""
    g = torch.Generator().manual_seed(13)
    B, S, C, H, D, L = 2, 12, 50, 2, 128, 34
    qkv = torch.randn((L, B, S, 4 + 2 * H, D), generator=g).to(torch.bfloat16)
    raw = torch.full((2, L, B, C + 2, H + 1, D), POISON, dtype=torch.uint8)
    sc = torch.full((2, L, B, H, 2), POISON, dtype=torch.uint8)
    x, d, s = qkv.cuda(), raw.cuda(), sc.cuda()
    c = d.view(torch.float8_e4m3fn)[:, :, :, 1:1 + C, :H]
    un = lambda t: list(t.unbind(0))       # noqa: E731
    table = lsp.Q8LayerTable(un(x[..., 4:4 + H, :]), un(x[..., 4 + H:, :]), un(c[0]), un(c[1]), un(s[0]), un(s[1]))
    n = torch.tensor([12, 7], dtype=torch.int32)
    lsp.kv_append_q8(table, n.cuda(), n.cuda())
    for i, a in ((0, 4), (1, 4 + H)):
        for l in range(0, L, 11):
            val, E = eight_bits.append(qkv[l, :, :, a:a + H], raw[i, l, :, 1:1 + C, :H].contiguous().view(torch.float8_e4m3fn), sc[i, l], n, n)
            assert _same(c[i, l].cpu(), val) and torch.equal(s[i, l].cpu().to(torch.int64), E)
    assert (d[:, :, :, [0, -1]] == POISON).all() and (d[..., H, :] == POISON).all()


def test_offsets_beyond_32_bits(lsp):
    """The last rows of caches of more than 2^31 bytes."""
    B, C, H, D = 2, 300001, 32, 128
    g = torch.Generator(device="cuda").manual_seed(17)
    kc, vc = (torch.zeros((B, C, H, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    ke, ve = (torch.ones((B, H, -(-C // 32)), dtype=torch.uint8, device="cuda") for _ in range(2))
    x = torch.randn((B, 40, H, D), generator=g, device="cuda").to(torch.bfloat16)
    table = lsp.Q8LayerTable([x], [-x], [kc], [vc], [ke], [ve])
    at = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")      # noqa: E731
    lsp.kv_append_q8(table, at(40, 33), at(C, C - 1))
    out = [torch.zeros((B, 40, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lsp.kv_read_q8(table, at(C - 40, C - 34), at(C, C - 1), [out[0]], [out[1]])
    for b, n in ((0, 40), (1, 33)):
        want = x[b, :n].float()
        assert ((out[0][b, :n].float() - want).abs() <= torch.maximum(want.abs() / 16, torch.tensor(2.0 ** -8, device="cuda"))).all() and want.abs().max() > 3
        assert torch.equal(out[0][b, :n], -out[1][b, :n])
        p = C - 40 if b == 0 else C - 34
        assert int(kc.view(torch.uint8)[b, p - 100:p].max()) == 0 and int(kc.view(torch.uint8)[b, p:p + n].max()) > 0
    assert int(kc.view(torch.uint8)[1, C - 1].max()) == 0 and int(kc.view(torch.uint8)[1, :1000].max()) == 0


def test_streams_and_graphs(lsp):
    """Captured with the step's own length buffers, replayed over other contents, on a stream of its own."""
    g = torch.Generator(device="cuda").manual_seed(19)
    x = torch.randn((2, 20, 3, 64), generator=g, device="cuda").to(torch.bfloat16)
    kc, vc, ke, ve = lsp.q8_cache(2, 90, 3, 64)
    table = lsp.Q8LayerTable([x], [x], [kc], [vc], [ke], [ve])
    n, P = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([20, 3], [20, 3]))
    out = [torch.zeros((2, 90, 3, 64), device="cuda") for _ in range(2)]
    zero = torch.zeros(2, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lsp.kv_append_q8(table, n, P)
        lsp.kv_read_q8(table, zero, P, [out[0]], [out[1]])
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        lsp.kv_append_q8(table, n, P)
        lsp.kv_read_q8(table, zero, P, [out[0]], [out[1]])
    val, E = torch.zeros(2, 90, 3, 64).to(torch.float8_e4m3fn), torch.ones(2, 3, 3, dtype=torch.uint8)
    v, E = eight_bits.append(x.cpu(), val, E, n.cpu(), P.cpu())
    for step in range(3):
        x.normal_(std=2.0 ** step)
        n.copy_(torch.tensor([7 + step, 18], dtype=torch.int32))
        P.add_(n)
        graph.replay()
        torch.cuda.synchronize()
        v, E = eight_bits.append(x.cpu(), v.float().to(torch.float8_e4m3fn), E.to(torch.uint8), n.cpu(), P.cpu())
        want = eight_bits.values(v, E)
        for b in range(2):
            assert torch.equal(out[0][b, :P[b]].cpu().double(), want[b, :P[b]]) and torch.equal(out[1], out[0])
