"""lsp_token_scores of rows whose logits are far from 0, of either sign: any finite row is in its range."""
import math

import pytest
import torch

from oracle import serving

pytestmark = pytest.mark.gpu
FAR = [2.0 ** 25, 2.0 ** 26, 1e8, 5e9, 1e10, 1e15, 1e30, 3e38]


@pytest.fixture(scope="module")
def lsp():
    import paper_2603_05454_amd as m
    assert torch.cuda.is_available()
    return m


def _rows(V, far, dtype):
    """Of magnitude `far`: all equal; one entry a step above; spread over a thousandth; both signs; ordinary entries among masked ones; one far entry among ordinary ones."""
    g = torch.Generator().manual_seed(V)
    one = torch.full((V,), far)
    step = one.clone()
    step[V // 2] = far * (1 + 2.0 ** -7)
    spread = far * (1 - 0.001 * torch.rand(V, generator=g))
    signs = torch.where(torch.arange(V) % 3 == 0, far, -far)
    masked = torch.where(torch.arange(V) % 4 == 1, torch.randn(V, generator=g), -far)
    single = torch.randn(V, generator=g)
    single[V // 3] = far
    return torch.stack([one, -one, step, -step, spread, -spread, signs, masked, single, -single]).clamp(-3.38e38, 3.38e38).to(dtype)


def _check(got, want, V, K):
    """Sums as in the tests of ordinary rows: chains of V / 64 terms of half a step, exponents up to 30 with two roundings, a dozen joins.  A difference from the maximum,
    and the logarithm's subtraction, are off by half a step of the result each, and results are as large as the rows."""
    lp, h, ids, alt = [t.cpu() for t in got]
    sums = (min(V, V / 64 + 64) + 60 + 2 + 12) * 2.0 ** -24

    def close(x, y, tol):
        y = y.float().double()      # (differences beyond fp32's range: -inf)
        x, fine = x.double(), torch.isfinite(y)
        assert torch.equal(x[~fine], y[~fine])
        assert ((x - y).abs()[fine] <= (tol + y.abs() * 2 * 2.0 ** -24)[fine]).all(), (x, y)
    close(lp, want[0], sums + 240 * 2.0 ** -24)
    close(h, want[1], sums * (2 + math.log(V + 1) + want[1].abs()))
    assert torch.equal(ids, want[2])
    close(alt, want[3], sums + 240 * 2.0 ** -24)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 9, 1000, 20001, 50001, 130001])
@pytest.mark.parametrize("cut", [True, False])
def test_rows_far_from_zero(lsp, dtype, V, cut):
    """cut: rows that several workgroups may share; more sequences than lengths are counted of, else."""
    z = torch.cat([_rows(V, f, dtype) for f in FAR])
    R = z.shape[0]
    ids = (torch.arange(R) * 7 % V).to(torch.int32)[None]
    want = serving.token_scores(z[None], ids, None, 5)
    if cut:
        got = lsp.token_scores(z[None].cuda(), ids.cuda(), num_alt=5)
    else:
        B = max(R, 257)
        lens = (torch.arange(B) < R).to(torch.int32)[:, None]
        zb = torch.zeros((B, 1, V), dtype=dtype, device="cuda")
        zb[:R, 0] = z.cuda()
        tid = torch.zeros((B, 1), dtype=torch.int32, device="cuda")
        tid[:R, 0] = ids[0].cuda()
        got = [t[:R].transpose(0, 1) for t in lsp.token_scores(zb, tid, lens[:, 0].cuda(), num_alt=5)]
    torch.cuda.synchronize()
    _check(got, want, V, 5)
