"""Buffers of the decode loop's options are looked at before the first step (no GPU needed)."""
import types

import pytest
import torch

import paper_2603_05454_amd as m
from paper_2603_05454_amd.loop import _Budget, _Scores


def test_scores_are_where_the_tokens_are():
    """A buffer elsewhere was met behind the first step's commit, which had changed the caller's state."""
    tokens = torch.zeros((2, 9), dtype=torch.int32, device="meta")
    f = torch.zeros((2, 9))
    with pytest.raises(m.LspError, match="logprob.*cpu.*meta"):
        _Scores(dict(logprob=f), tokens, 100)
    with pytest.raises(m.LspError, match="alt_id"):
        _Scores(dict(alt_id=torch.zeros((2, 9, 3), dtype=torch.int32), alt_logprob=torch.zeros((2, 9, 3), device="meta")), tokens, 100)
    assert _Scores(dict(logprob=f), torch.zeros((2, 9), dtype=torch.int32), 100).K == 0


@pytest.mark.parametrize("which", ["weights", "positions", "cache_len"])
def test_a_budgets_buffers_are_where_the_lengths_are(which):
    """Positions elsewhere were met behind the first step's commit and append."""
    table = types.SimpleNamespace(n=1, B=2, Hkv=1, C=20)
    i = dict(dtype=torch.int32)
    make = dict(weights=lambda **k: torch.zeros((1, 2, 1, 20), **k), positions=lambda **k: torch.zeros((1, 2, 1, 20), **i, **k),
                cache_len=lambda **k: torch.zeros(2, **i, **k))
    prefix_len, suffix_len = torch.zeros(2, **i), torch.ones(2, **i)
    with pytest.raises(m.LspError, match=f"{which}.*meta.*cpu"):
        _Budget(keep=4, recent=2, **{which: make[which](device="meta")}).start(table, prefix_len, suffix_len)
    _Budget(keep=4, recent=2, **{which: make[which]()}).start(table, prefix_len, suffix_len)
