"""lsp_attn_step_q8 finds every key once, whatever workgroup, wave, step and block it falls to.

Key t belongs to one of D groups and, by its value, to one of D elements.  A query asks for one group: its keys' scores are 200 octaves above all others',
whose weights are 0.  The result is then, element by element, how many of the group's keys have that element, over the group's size: with a few keys to each pair a key
that is lost, met twice, taken from another place or read under another block's scale changes a result by more than a twentieth of it, where sums over random keys
would hide it.  Keys and values are powers of two under scales that differ from block to block; what is not there is NaN."""
import ctypes
import math

import pytest
import torch

from oracle import eight_bits

pytestmark = pytest.mark.gpu
OCTAVES, SIZE = 200.0, 16.0


@pytest.fixture(scope="module")
def lsp():
    import paper_2603_05454_amd as m
    assert torch.cuda.is_available()
    return m


def _codes(t, b, h, D):
    """Group and element of keys t [n,1] of sequence b's heads h [1,H]."""
    return (t + 5 * h + 11 * b) % D, (13 * (t // D) + 5 * (t // (D * D)) + 3 * h + 7 * b) % D


def _one_hot(cache, scale, b, rows, at, g):
    """Rows of a cache: at element at[t,h] the number 1, as a power of two under the block's scale."""
    H, blocks = scale.shape[1:]
    k = torch.randint(-6, 9, (H, blocks), generator=g, device="cuda", dtype=torch.int32)
    used = -(-rows // 32)
    scale[b, :, :used] = (127 - k[:, :used]).to(torch.uint8)
    byte = ((k + 7) << 3).to(torch.uint8)             # e4m3: 2^k has the exponent k + 7
    of = byte.repeat_interleave(32, dim=1)[:, :rows].T
    cache[b, :rows] = 0
    cache[b, :rows].scatter_(2, at.unsqueeze(-1), of.unsqueeze(-1).contiguous())


def _keys(B, S, H, D, C, P, N, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kc, vc = (torch.full((B, C, H, D), 0x7f, dtype=torch.uint8, device="cuda") for _ in range(2))
    ke, ve = (torch.full((B, H, -(-C // 32)), 255, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((B, S, H, D), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cells = torch.zeros((B, H, D, D), dtype=torch.float64, device="cuda")     # of a group, of an element
    head = torch.arange(H, device="cuda").unsqueeze(0)
    for b in range(B):
        t = torch.arange(P[b] + N[b], device="cuda").unsqueeze(1)
        group, element = _codes(t, b, head, D)
        if P[b] > 0:
            _one_hot(kc, ke, b, P[b], group[:P[b]], g)
            _one_hot(vc, ve, b, P[b], element[:P[b]], g)
        for x, at in ((ks, group), (vs, element)):
            x[b, :N[b]] = torch.nn.functional.one_hot(at[P[b]:], D).to(torch.bfloat16)
        cell = (head * D + group) * D + element
        cells[b] = torch.bincount(cell.flatten(), minlength=H * D * D).view(H, D, D).double()
    e4m3 = torch.float8_e4m3fn
    return ks, vs, kc.view(e4m3), vc.view(e4m3), ke, ve, cells


def _attend(lsp, q, keys, lens, scale, out, copies, workspace):
    if workspace:
        table = lsp.Q8LayerTable(*[[t] * copies for t in keys], q=[q] * copies, out=list(out.unbind(0)))
        lsp.attn_step_q8_layers(table, *lens, scale=scale)
        return
    B, S, Hq, D = q.shape
    d = lsp.AttnDesc(dtype=lsp.LSP_BF16, B=B, S=S, Hq=Hq, Hkv=keys[0].shape[2], D=D, C=keys[2].shape[1], scale=scale)
    lists = [(ctypes.c_void_p * copies)(*[t.data_ptr() for t in ts]) for ts in ([q] * copies, *[[t] * copies for t in keys], out.unbind(0))]
    rc = lsp.lib().lsp_attn_step_q8_layers(ctypes.byref(d), copies, *lists[:7], *[ctypes.c_void_p(t.data_ptr()) for t in lens], lists[7], None,
                                           ctypes.c_size_t(0), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert rc == 0, lsp.lib().lsp_last_error()


def _every_key_is_found(lsp, B, S, Hq, H, D, C, P, N, copies=1, workspace=True):
    assert all(p + n >= D for p, n in zip(P, N) if n > 0)       # no group is empty
    *keys, cells = _keys(B, S, H, D, C, P, N)
    rep = Hq // H
    lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (P, N)]
    want = cells / cells.sum(-1, keepdim=True)                  # [B,H,group,element]
    few = min(n for n in N if n > 0) * rep
    entry = torch.arange(S, device="cuda").view(S, 1) * rep + torch.arange(Hq, device="cuda") % rep      # of a unit
    head = torch.arange(Hq, device="cuda") // rep
    for first in range(0, D, few):
        group = (entry + first) % D                             # [S,Hq]
        q = (SIZE * torch.nn.functional.one_hot(group, D)).to(torch.bfloat16).expand(B, S, Hq, D).contiguous()
        for b in range(B):
            q[b, N[b]:] = math.nan
        out = torch.full((copies, B, S, Hq, D), -768.0, dtype=torch.bfloat16, device="cuda")
        _attend(lsp, q, keys, lens, OCTAVES / (SIZE * math.log2(math.e)), out, copies, workspace)
        assert (out == out[:1]).all()
        for b in range(B):
            w = want[b][head.expand(N[b], Hq), group[:N[b]]]
            # a weight's exponent is off by half a step of 2^-16 at 200, which the sum of weights has, their rounding to bf16 takes away, and the result is rounded
            err, tol = (out[0, b, :N[b]].double() - w).abs(), (2.0 ** -8 + 2.0 ** -16) * w
            assert (err <= tol).all(), (b, first, (err > tol).nonzero()[:4].tolist())
            assert (out[0, b, N[b]:] == -768.0).all()


CASES = [   # B, S, Hq, Hkv, D, C, prefix, suffix, copies
    # short tiles: one row, sixteen and more entries, heads beside each other, keys divided in many parts
    (1, 1, 1, 1, 64, 8000, [7999], [1], 1), (1, 1, 28, 4, 128, 800, [700], [1], 1), (1, 5, 2, 1, 128, 5000, [4999], [5], 1), (1, 4, 3, 3, 128, 66000, [65999], [3], 2),
    (1, 20, 8, 8, 128, 66000, [65990], [20], 1), (1, 33, 6, 6, 64, 66000, [65999], [33], 1), (1, 64, 1, 1, 128, 3001, [3001], [64], 1),
    (9, 5, 8, 4, 128, 2300, [2300 - b for b in range(9)], [5, 4, 0, 3, 2, 1, 5, 5, 5], 32), (9, 6, 12, 6, 64, 2300, [2299] * 9, [3] * 9, 24),
    (8, 4, 32, 32, 64, 1910, [1900 - b for b in range(8)], [4 - b % 3 for b in range(8)], 1),
    (70, 12, 4, 2, 128, 2100, [(301 * b) % 1951 + 130 for b in range(70)], [b % 13 for b in range(70)], 1),
    # tall tiles of four waves
    (1, 100, 2, 2, 128, 6000, [5950], [100], 1), (1, 100, 2, 2, 64, 6000, [5983], [97], 1), (1, 300, 2, 2, 64, 6000, [6000], [300], 1), (3, 70, 8, 2, 64, 300, [129, 40, 300], [70, 33, 1], 1),
    (9, 65, 4, 4, 128, 1100, [1100 - 7 * b for b in range(9)], [65 + b % 2 - 1 for b in range(9)], 12),
    # tall tiles of eight waves
    (1, 300, 2, 2, 128, 6000, [6000], [300], 1), (2, 300, 4, 2, 128, 4000, [3990, 10], [130, 300], 1), (1, 1025, 2, 2, 128, 64, [0], [1025], 1),
    (5, 300, 16, 16, 128, 9000, [9000, 8999, 9000, 120, 8970], [17, 3, 33, 300, 16], 1), (4, 257, 7, 1, 128, 1030, [1021, 31, 64, 95], [257, 250, 129, 256], 1),
    (2, 512, 8, 8, 128, 600, [600, 577], [512, 130], 8)]


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_every_key_is_found(lsp, case, workspace):
    *shape, copies = CASES[case]
    _every_key_is_found(lsp, *shape, copies=copies, workspace=workspace)


@pytest.mark.parametrize("S, N", [(4, [2, 4]), (150, [3, 150])])
def test_every_key_beyond_32_bits_is_found(lsp, S, N):
    """Caches of 2.4 GB each, keys and values in buffers of their own: their rows on both sides of 2^31 bytes, under the scales of their own blocks."""
    _every_key_is_found(lsp, 2, S, 32, 32, 128, 300001, [300001, 299999], N)


# ---- scales far apart, NaN, in every kind of tile -------------------------------------
TILES = [   # S, Hq, Hkv, prefix, suffix
    (3, 4, 2, [700, 33], [3, 2]), (16, 4, 4, [3000, 64], [16, 9]), (40, 2, 2, [700, 95], [40, 33]), (100, 2, 2, [700, 31], [100, 66]), (300, 2, 2, [700, 129], [300, 258])]


def _random(B, S, Hq, H, D, C, k_scales, v_scales, seed):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((B, S, Hq, D), generator=g).to(torch.bfloat16)
    ks, vs = (torch.randn((B, S, H, D), generator=g).to(torch.bfloat16) for _ in range(2))
    kc, vc = ((torch.randn((B, C, H, D), generator=g) * 100).clamp(-448, 448).to(torch.float8_e4m3fn) for _ in range(2))
    ke, ve = (torch.randint(a, z, (B, H, -(-C // 32)), generator=g, dtype=torch.uint8) for a, z in (k_scales, v_scales))
    return q, ks, vs, kc, vc, ke, ve


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tile", range(len(TILES)))
def test_neighbouring_scales_far_apart(lsp, D, tile):
    """Keys' scales from 2^-67 to 2^-6, values' from 2^-27 to 2^13, each block's its own."""
    S, Hq, H, P, N = TILES[tile]
    C = max(P) + 20
    t = _random(2, S, Hq, H, D, C, (60, 122), (100, 141), tile)
    want, mass = eight_bits.attention(*t[:3], eight_bits.values(t[3], t[5]), eight_bits.values(t[4], t[6]), P, N)
    out = torch.full(t[0].shape, -768.0, dtype=torch.bfloat16, device="cuda")
    lsp.attn_step_q8(*[x.cuda() for x in t], *[torch.tensor(x, dtype=torch.int32, device="cuda") for x in (P, N)], out=out)
    got = out.cpu().double()
    for b, n in enumerate(N):
        # probabilities' rounding to bf16, 2^-8 of the sum of |v| at most; scores (sums of up to 128 products in fp32, of a score of up to about 50) and
        # sums below 2^-12 of it; the result's rounding
        assert ((got[b, :n] - want[b, :n]).abs() <= (2.0 ** -8 + 2.0 ** -12) * mass[b, :n] + 2.0 ** -8 * want[b, :n].abs()).all()
        assert (got[b, n:] == -768.0).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tile", range(len(TILES)))
def test_nan_reaches_only_its_rows(lsp, D, tile):
    """A NaN among one head's cached keys makes that head's rows NaN, and no others; one among the cached or the suffix's values its element's column."""
    S, Hq, H, P, N = TILES[tile]
    rep = Hq // H
    t = _random(2, S, Hq, H, D, max(P) + 20, (119, 122), (119, 122), 20 + tile)
    t[3].view(torch.uint8)[0, P[0] - 3, 1, 3] = 0x7f
    t[4].view(torch.uint8)[1, P[1] - 1, 0, 9] = 0xff
    t[2][1, N[1] - 1, 1, 5] = math.nan
    out = torch.zeros(t[0].shape, dtype=torch.bfloat16, device="cuda")
    lsp.attn_step_q8(*[x.cuda() for x in t], *[torch.tensor(x, dtype=torch.int32, device="cuda") for x in (P, N)], out=out)
    want = torch.zeros(out.shape, dtype=torch.bool)
    want[0, :N[0], rep:2 * rep] = True
    want[1, :N[1], :rep, 9] = True
    want[1, :N[1], rep:2 * rep, 5] = True
    assert torch.equal(out.isnan().cpu(), want)
