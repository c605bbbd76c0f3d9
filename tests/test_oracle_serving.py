"""The 64-bit forms that the GPU tests of token scores, key weights and eviction compare with, against closed forms and brute force."""
import itertools
import math

import torch

from oracle import serving


def test_scores_of_known_distributions():
    z = torch.tensor([[[0.0, 0.0, 0.0, 0.0], [math.log(8), math.log(4), -math.inf, math.log(4)], [-math.inf] * 4]])
    lp, h, ids, alt = serving.token_scores(z, torch.tensor([[2, 1, 0]], dtype=torch.int32), None, 5)
    assert torch.allclose(lp[0, :2], torch.tensor([-math.log(4), -math.log(4)]).double()) and lp[0, 2] == -math.inf
    assert torch.allclose(h[0], torch.tensor([math.log(4), 1.5 * math.log(2), 0.0]).double())
    assert ids[0].tolist() == [[0, 1, 2, 3, -1], [0, 1, 3, 2, -1], [0, 1, 2, 3, -1]]
    assert torch.allclose(alt[0, 1].exp(), torch.tensor([0.5, 0.25, 0.25, 0, 0]).double()) and alt[0, 1, 4] == -math.inf


def test_ids_outside_the_vocabulary_and_inactive_rows():
    z = torch.randn(2, 3, 7)
    lp, h, ids, alt = serving.token_scores(z, torch.tensor([[7, -1, 0], [0, 0, 0]], dtype=torch.int32), torch.tensor([3, 1]), 1)
    assert lp[0, :2].tolist() == [-math.inf, -math.inf] and torch.isfinite(lp[0, 2])
    assert torch.isnan(h[1, 1:]).all() and (ids[1, 1:] == -2).all()


def test_mass_adds_up_to_the_number_of_rows():
    g = torch.Generator().manual_seed(1)
    q, k, c = (torch.randn(s, generator=g) for s in ((2, 5, 4, 8), (2, 5, 2, 8), (2, 9, 2, 8)))
    w = torch.rand(2, 2, 16, generator=g)[..., :9].clone()
    P, N = torch.tensor([4, 0]), torch.tensor([5, 3])
    got = serving.key_weights(q, k, c, P, N, w, decay=0.0)
    assert torch.allclose(got[0].sum(-1), torch.full((2,), 10.0).double())          # 5 rows of 2 heads, 4 + 5 keys
    assert torch.allclose(got[1, :, :3].sum(-1), torch.full((2,), 6.0).double()) and torch.equal(got[1, :, 3:], w[1, :, 3:].double())
    assert torch.allclose(serving.key_weights(q, k, c, P, N, w, decay=0.5)[0, :, :4], got[0, :, :4] + 0.5 * w[0, :, :4])
    assert torch.equal(serving.key_weights(q, k, c, P, torch.tensor([0, 0]), w), w.double())


def test_one_key_takes_all_and_equal_keys_share():
    q, k = torch.ones(1, 2, 1, 4), torch.ones(1, 2, 1, 4)
    c = torch.zeros(1, 3, 1, 4)
    got = serving.key_weights(q, k, c, torch.tensor([1]), torch.tensor([2]), torch.zeros(1, 1, 3), scale=100.0)
    assert torch.allclose(got, torch.tensor([[[0.0, 1.0, 1.0]]]).double())


def test_eviction_against_all_subsets():
    """Of all sets that hold the protected rows, the one kept has the largest sum, and the first rows among equal sums."""
    for seed in range(20):
        g = torch.Generator().manual_seed(seed)
        w = (torch.rand(1, 1, 1, 8, generator=g) * 3).floor()
        P, keep, first, recent = 7, 4, seed % 2, seed % 3
        cache = torch.arange(8.0).view(1, 1, 8, 1, 1).clone()
        new, length, index = serving.evict(w, torch.tensor([P]), keep, first=first, recent=recent, caches=[cache])
        must = set(range(first)) | set(range(P - recent, P))
        best = max((s for s in itertools.combinations(range(P), keep) if must <= set(s)), key=lambda s: (sum(w[0, 0, 0, t].item() for t in s), [-t for t in s]))
        assert sorted(index[0, 0, 0].tolist()) == list(best) and length.tolist() == [keep]
        assert cache[0, 0, :keep, 0, 0].tolist() == index[0, 0, 0].tolist() and new[0, 0, 0, :keep].tolist() == w[0, 0, 0, index[0, 0, 0].long()].tolist()
        assert all(t == j for j, t in enumerate(index[0, 0, 0].tolist()) if t < keep)       # rows below `keep` that stay do not move


def test_short_sequences_are_left_alone():
    w = torch.tensor([3.0, 1, 2, 0, 5, 4]).view(1, 1, 1, 6)
    new, length, index = serving.evict(w.expand(1, 3, 1, 6).contiguous(), torch.tensor([2, 5, 6]), 3, high=5)
    assert length.tolist() == [2, 5, 3] and index[0, :, 0].tolist() == [[0, 1, -1], [0, 1, 2], [0, 4, 5]]
    assert new[0, 2, 0].tolist() == [3, 5, 4, 0, 5, 4]
