"""lsp_confidence of rows whose logits are far from 0, of either sign, and of vocabularies masked with large finite numbers: any finite maximum is in its range."""
import pytest
import torch

pytestmark = pytest.mark.gpu
FAR = [2.0 ** 25, 2.0 ** 26, 1e8, 5e9, 1e10, 1e15, 1e30, 3e38]


@pytest.fixture(scope="module")
def lsp():
    import paper_2603_05454_amd as m
    assert torch.cuda.is_available()
    return m


def _rows(V, far, dtype):
    """All equal; one entry a step above; spread over a thousandth; both signs; ordinary entries among masked ones, alternating and behind
    the first ninth (so that whole lanes hold nothing else); one far entry among ordinary ones."""
    g = torch.Generator().manual_seed(V)
    one = torch.full((V,), far)
    step = one.clone()
    step[V // 2] = far * (1 + 2.0 ** -7)
    spread = far * (1 - 0.001 * torch.rand(V, generator=g))
    signs = torch.where(torch.arange(V) % 3 == 0, far, -far)
    noise = torch.randn(V, generator=g)
    masked = torch.where(torch.arange(V) % 4 == 1, noise, -far)
    behind = torch.where(torch.arange(V) <= V // 9, noise, -far)
    single = noise.clone()
    single[V // 3] = far
    return torch.stack([one, -one, step, -step, spread, -spread, signs, masked, behind, single, -single]).clamp(-3.38e38, 3.38e38).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [2, 9, 1000, 4099, 20001, 50001, 130001])
@pytest.mark.parametrize("call", ["cut", "whole", "static"])
def test_rows_far_from_zero(lsp, dtype, V, call):
    z = torch.cat([_rows(V, f, dtype) for f in FAR])
    R = z.shape[0]
    x = z.double()
    top = x.max(-1, keepdim=True)
    first = torch.where(x == top.values, torch.arange(V), V).min(-1).values.to(torch.int32)
    prob = 1 / (x - top.values).exp().sum(-1)
    two = z.float().topk(2, -1).values
    if call == "whole":     # more sequences than lengths are counted of: a workgroup to a row
        B = max(R, 257)
        zb = torch.zeros((B, 1, V), dtype=dtype, device="cuda")
        zb[:R, 0] = z.cuda()
        ids, p, margin = [t[:R, 0].cpu() for t in lsp.confidence(zb, (torch.arange(B) < R).to(torch.int32).cuda())]
    else:
        zg = z[None].cuda()
        if call == "cut":
            got = lsp.confidence(zg)
        else:
            got = lsp.confidence_static(zg, None, (torch.zeros((1, R), dtype=torch.int32, device="cuda"), torch.zeros((1, R), device="cuda"), torch.zeros((1, R), device="cuda")))
        ids, p, margin = [t[0].cpu() for t in got]
    assert torch.equal(ids, first) and torch.equal(margin, two[:, 0] - two[:, 1])
    # chains of at most V / 64 terms of half a step, exponents up to 60 (32 octaves behind the maximum) with two roundings, a dozen joins, the exponential and the quotient
    tol = (min(V, V / 64 + 64) + 120 + 2 + 12 + 2) * 2.0 ** -24
    assert ((p.double() - prob).abs() <= tol * prob).all(), (p, prob)
