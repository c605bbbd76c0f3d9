"""The plain form of the attention over caches in 8 bits: pinned to torch's own attention in 64 bits, and to results known by hand."""
import math

import pytest
import torch

from oracle import eight_bits as o


@pytest.mark.parametrize("scale", [0.0, 0.3])
@pytest.mark.parametrize("B, S, Hq, H, D, C, P, N", [(1, 1, 1, 1, 64, 1, [0], [1]), (2, 5, 4, 2, 64, 40, [33, 0], [5, 2]), (2, 9, 6, 1, 128, 70, [70, 31], [1, 9]),
                                                    (3, 3, 3, 3, 64, 10, [-2, 99, 4], [7, 3, 0])])
def test_it_is_torchs_attention(B, S, Hq, H, D, C, P, N, scale):
    g = torch.Generator().manual_seed(B + S)
    q = torch.randn(B, S, Hq, D, generator=g).bfloat16()
    ks, vs = (torch.randn(B, S, H, D, generator=g).bfloat16() for _ in range(2))
    cached = [o.values((torch.randn(B, C, H, D, generator=g) * 50).to(torch.float8_e4m3fn), torch.randint(119, 123, (B, H, -(-C // 32)), generator=g, dtype=torch.uint8))
              for _ in range(2)]
    out, mass = o.attention(q, ks, vs, *cached, P, N, scale=scale)
    for b in range(B):
        p, n = min(max(P[b], 0), C), min(max(N[b], 0), S)
        assert out[b, n:].isnan().all() and mass[b, n:].isnan().all()
        if n == 0:
            continue
        k, v = (torch.cat([c[b, :p], x[b, :n].double()]).transpose(0, 1).repeat_interleave(Hq // H, dim=0) for c, x in zip(cached, (ks, vs)))
        heads = q[b, :n].double().transpose(0, 1)
        for got, values in ((out, v), (mass, v.abs())):
            want = torch.nn.functional.scaled_dot_product_attention(heads, k, values, scale=scale or None).transpose(0, 1)
            # both are sums of some hundred terms in 64 bits, each with a few roundings of 2^-53: below 2^-40 of the sum of magnitudes
            assert ((got[b, :n] - want).abs() <= 2.0 ** -40 * mass[b, :n]).all()


def test_results_known_by_hand():
    """Equal scores weigh alike; scores log 3 apart weigh three to one."""
    q = torch.zeros(1, 1, 1, 64)
    q[..., 0] = 1.0
    ks, vs = torch.zeros(1, 1, 1, 64), torch.full((1, 1, 1, 64), -8.0)
    kc, vc = torch.zeros(1, 3, 1, 64, dtype=torch.float64), torch.tensor([2.0, 4.0, 1000.0], dtype=torch.float64).view(1, 3, 1, 1).expand(1, 3, 1, 64)
    out, mass = o.attention(q, ks, vs, kc, vc, [2], [1], scale=1.0)
    assert torch.allclose(out, torch.full_like(out, (2 + 4 - 8) / 3)) and torch.allclose(mass, torch.full_like(mass, 14 / 3))
    kc[0, 1, 0, 0] = math.log(3.0)
    out, mass = o.attention(q, ks, vs, kc, vc, [2], [1], scale=1.0)
    assert torch.allclose(out, torch.full_like(out, (2 + 3 * 4 - 8) / 5)) and torch.allclose(mass, torch.full_like(mass, (2 + 3 * 4 + 8) / 5))
