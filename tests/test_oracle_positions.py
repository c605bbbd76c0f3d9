"""The plain form of eviction again and again, by positions: rows carry their tokens' positions as labels."""
import pytest
import torch

from oracle import serving


def _steps(keep, high, first, recent, aged, per_step=(2, 5, 1), P0=(30, 41, 12), steps=40, seed=0):
    """Every step appends rows of low weight and cuts back.  Yields tokens so far, length, labels of the cached rows, positions, the weights before and after."""
    g = torch.Generator().manual_seed(seed)
    B, H, C = len(P0), 2, 100
    label = torch.arange(C).float().expand(1, B, H, C).transpose(2, 3).unsqueeze(-1).contiguous()       # [L,B,C,H,1]
    w = torch.rand((1, B, H, C), generator=g) + 1
    tokens = torch.tensor(P0, dtype=torch.int32)
    length, positions = tokens.clone(), torch.full((1, B, H, C), serving.BY_PLACE, dtype=torch.int32)
    for _ in range(steps):
        for b in range(B):
            for _ in range(per_step[b]):
                label[0, b, length[b]], w[0, b, :, length[b]] = float(tokens[b]), torch.rand(H, generator=g) * 1e-3
                length[b] += 1
                tokens[b] += 1
        kw = dict(positions=positions, token_len=tokens) if aged else {}
        w, length, _ = serving.evict(w, length, keep, high, first, recent, caches=[label], **kw)
        yield tokens, length, label[0, ..., 0], positions[0], w


@pytest.mark.parametrize("keep,high,first,recent", [(20, None, 2, 8), (20, 26, 0, 20), (20, 22, 3, 10), (20, None, 20, 0), (1, None, 0, 1)])
def test_the_newest_rows_stay_and_positions_follow_them(keep, high, first, recent):
    for tokens, length, label, positions, _ in _steps(keep, high, first, recent, aged=True):
        for b, (T, n) in enumerate(zip(tokens.tolist(), length.tolist())):
            assert n <= (high or keep)
            for h in range(2):
                held = [int(x) for x in label[b, :n, h]]
                assert len(set(held)) == n and set(held) >= set(range(T - min(recent, T), T)) | set(range(min(first, n)))
                assert [T - (n - t) if p == serving.BY_PLACE else p for t, p in enumerate(positions[b, h, :n].tolist())] == held
                assert (positions[b, h, n:] == serving.BY_PLACE).all()


def test_the_last_places_are_not_the_newest_rows():
    """Why positions are kept: by place, from the second eviction on, fewer than `recent` of the newest rows are held."""
    held = [sum(int(x) >= T - 8 for x in label[0, :n, 0])
            for tokens, length, label, _, _ in _steps(20, None, 2, 8, aged=False) for T, n in [(int(tokens[0]), int(length[0]))]]
    assert held[0] == 8 and held[-1] == 2       # two rows were appended at the last step


def test_a_first_eviction_goes_by_place_either_way():
    g = torch.Generator().manual_seed(3)
    w = torch.rand((2, 3, 2, 60), generator=g)
    P = torch.tensor([60, 33, 41], dtype=torch.int32)
    caches = [torch.rand((2, 3, 60, 2, 4), generator=g) for _ in range(2)]
    caches[1].copy_(caches[0])
    a = serving.evict(w, P, 30, 40, 2, 9, caches=caches[:1])
    for T in (P, P + 1000):
        positions = torch.full((2, 3, 2, 60), serving.BY_PLACE, dtype=torch.int32)
        c = caches[1].clone()
        b = serving.evict(w, P, 30, 40, 2, 9, caches=[c], positions=positions, token_len=T)
        assert all(torch.equal(x, y) for x, y in zip(a, b)) and torch.equal(c, caches[0])
        assert torch.equal(positions[:, 0, :, :30], a[2][:, 0] + (T[0] - P[0])) and (positions[:, 1] == serving.BY_PLACE).all()


def test_positions_that_make_no_sense_leave_the_last_places():
    w = torch.rand((1, 1, 1, 30), generator=torch.Generator().manual_seed(1))
    same = torch.full((1, 1, 1, 30), 29, dtype=torch.int32)
    a = serving.evict(w, torch.tensor([30]), 10, first=1, recent=4)
    b = serving.evict(w, torch.tensor([30]), 10, first=1, recent=4, positions=same, token_len=torch.tensor([30]))
    assert all(torch.equal(x, y) for x, y in zip(a, b))
