"""The plain forms of a cache in 8 bits: pinned to torch's own e4m3 conversion, to tiny cases by hand and to each other."""
import math

import pytest
import torch

from oracle import eight_bits as o


def test_nearest_is_torchs_conversion():
    x = torch.cat([torch.arange(-448, 449).double() / 3, torch.randn(2000, dtype=torch.float64, generator=torch.Generator().manual_seed(0)) * 0.02,
                   torch.tensor([0.0, 448.0, -448.0, 17.0, 18.0, 19.0, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, 2.5 * 2.0 ** -9])])
    assert torch.equal(o.nearest(x), x.float().to(torch.float8_e4m3fn).double())
    assert o.nearest(torch.tensor([1e9]))[0] == 448 and o.nearest(torch.tensor([math.inf]))[0].isnan()


@pytest.mark.parametrize("most, E", [(448.0, 127), (449.0, 128), (224.0, 126), (1.0, 119), (0.0, 1), (1e-40, 1), (3.39e38, 246), (1.75 * 2.0 ** 127, 246)])
def test_exponent(most, E):
    assert o.exponent(torch.tensor([0.0, -most, math.nan, math.inf])) == E


def test_append_by_hand():
    """Rows of 1 in a block, then a row of 1000 in the same block: 1000 <= 448 * 4 moves the exponent, and what was there is rounded under it."""
    suf = torch.ones(1, 4, 1, 64)
    cache, scale = torch.zeros(1, 40, 1, 64).to(torch.float8_e4m3fn), torch.ones(1, 1, 2, dtype=torch.uint8)
    val, E = o.append(suf, cache, scale, [3], [3])
    assert E[0, 0].tolist() == [119, 1] and (val[0, :3] == 256).all() and (val[0, 3:] == 0).all()
    val, E = o.append(suf * 1000, val.to(torch.float8_e4m3fn), E, [1], [4])
    assert E[0, 0, 0] == 129 and (val[0, :3] == 0.25).all() and (val[0, 3] == 256).all()      # 250 lies between 240 and 256
    assert (o.values(val, E)[0, :4, 0, 0] == torch.tensor([1, 1, 1, 1024])).all()


def test_rotation_is_a_rotation():
    g = torch.Generator().manual_seed(1)
    q, k = torch.randn(2, 3, 4, 64, generator=g), torch.randn(2, 3, 2, 64, generator=g)
    f = torch.rand(16, generator=g)
    for inter in (False, True):
        (a, _), (b, _) = o.norm_rope(q, k, f, interleaved=inter, prefix_len=torch.tensor([5, 1000]))
        assert torch.allclose(a.norm(dim=-1), q.double().norm(dim=-1)) and torch.equal(a[..., 32:], q[..., 32:].double())
        (c, _), _ = o.norm_rope(a, k, -f, interleaved=inter, prefix_len=torch.tensor([5, 1000]))
        assert torch.allclose(c, q.double())
        # products go by distances alone
        (d, _), (e, _) = o.norm_rope(q, k, f, interleaved=inter, prefix_len=torch.tensor([17, 1012]))
        assert torch.allclose((a[:, :, 0] * b[:, :, 0]).sum(-1), (d[:, :, 0] * e[:, :, 0]).sum(-1))


def test_attention_of_a_cache_that_holds_its_rows_exactly():
    from oracle import serving
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(1, 3, 2, 64, generator=g) for _ in range(3))
    c = torch.randn(1, 9, 2, 64, generator=g)
    out, mass = o.attention(q, k, v, c.double(), c.double(), [7], [2])
    assert out[0, 2].isnan().all() and (mass[0, :2] >= out[0, :2].abs()).all()
    w = serving.key_weights(q, k, c, torch.tensor([7]), torch.tensor([2]), torch.zeros(1, 2, 9))
    assert torch.allclose(w.sum(-1), torch.full((1, 2), 2.0, dtype=torch.float64))
