"""lsp_qk_norm_rope where a workgroup takes several rows, and at the most rows that it takes."""
import ctypes

import pytest
import torch

from oracle import eight_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsp():
    import paper_2603_05454_amd as m
    assert torch.cuda.is_available()
    return m


def _freq(R):
    return (10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)).float()


@pytest.mark.parametrize("S", [(1 << 24) - 1, 1 << 24])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_most_rows(lsp, dtype, S):
    """Heads that are work for all threads of a workgroup, and as many rows as the call takes: 2^32 threads, were a workgroup to have one row.  The
    buffers hold the active rows alone, which are all that is read and written."""
    Hq, H, D, N = 32, 32, 128, 3
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k = (torch.randn((1, N, h, D), generator=g, device="cuda").to(dtype) for h in (Hq, H))
    f, w = _freq(D).cuda(), torch.randn(D, generator=g, device="cuda")
    want = lsp.qk_norm_rope(q, k, f, w, w)
    out = [torch.zeros_like(x) for x in (q, k)]
    n = torch.tensor([N], dtype=torch.int32, device="cuda")
    d = lsp.QkNormRopeDesc(dtype=lsp.LSP_F32 if dtype == torch.float32 else lsp.LSP_BF16, B=1, S=S, Hq=Hq, Hkv=H, D=D, R=D, eps=1e-6)
    at = lambda t: ctypes.c_void_p(t.data_ptr())      # noqa: E731
    rc = lsp.lib().lsp_qk_norm_rope(ctypes.byref(d), at(q), at(k), at(w), at(w), at(f), None, at(n), None, at(out[0]), at(out[1]),
                                    ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert rc == 0, lsp.lib().lsp_last_error()
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    # (what both are compared with is itself held to the definition: a row of it here)
    (y, size), _ = eight_bits.norm_rope(q.cpu(), k.cpu(), f.cpu(), w.cpu(), w.cpu())
    # 21 roundings of 2^-24 and the rounding to the type, as in the call's own test
    tol = 21 * 2.0 ** -24 * size + (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24) * y.abs() + 1e-30
    assert ((want[0].cpu().double() - y).abs() <= tol).all()


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("R", [16, 48, "D"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_four_rows_to_a_workgroup(lsp, dtype, D, R, interleaved, given):
    """More than 2048 rows of few heads, every kind of pair, positions by length and given; lengths that leave one to four rows to the last workgroup."""
    B, S, Hq, H = 5, 701, 5, 2
    R = D if R == "D" else R
    g = torch.Generator().manual_seed(D + R)
    q, k = ((torch.randn((B, S, h, D), generator=g) * torch.exp(torch.randn((B, S, h, 1), generator=g))).to(dtype) for h in (Hq, H))
    w = [torch.randn(D, generator=g) for _ in range(2)] if R != 48 else [None, None]
    N, P = torch.tensor([701, 700, 3, 698, -1], dtype=torch.int32), torch.tensor([0, 4093, 100003, 17, 5], dtype=torch.int32)
    pos = torch.randint(0, 1 << 30, (B, S), generator=g, dtype=torch.int32) if given else None
    f = _freq(R)
    want = eight_bits.norm_rope(q, k, f, *w, eps=1e-5, prefix_len=P, suffix_len=N, positions=pos, interleaved=interleaved)
    dev = lambda t: None if t is None else t.cuda()      # noqa: E731
    out = [torch.full_like(x, 7.0).cuda() for x in (q, k)]
    lsp.qk_norm_rope(q.cuda(), k.cuda(), f.cuda(), dev(w[0]), dev(w[1]), 1e-5, P.cuda(), N.cuda(), dev(pos), interleaved, out)
    for o, (y, size) in zip(out, want):
        got = o.cpu().double()
        for b in range(B):
            n = max(int(N[b]), 0)
            # as above
            tol = 21 * 2.0 ** -24 * size[b, :n] + (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24) * y[b, :n].abs() + 1e-30
            assert ((got[b, :n] - y[b, :n]).abs() <= tol).all() and (got[b, n:] == 7).all()
