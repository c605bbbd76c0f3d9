"""Strides of 0 stand for a dense tensor in the C calls, so a tensor that is broadcast in the dimensions they are of would be read, or written, past its end:
the binding refuses it (no GPU needed: nothing is launched)."""
import pytest
import torch

import paper_2603_05454_amd as m


@pytest.fixture
def host(monkeypatch):
    """Host tensors stand in for device tensors: a call that got past the checks would reach the library, which is not there."""
    monkeypatch.setattr(m, "_here", lambda *ts: None)
    monkeypatch.setattr(m, "_dev", lambda *ts: None)
    monkeypatch.setattr(m, "lib", lambda: pytest.fail("the call reached the library"))
    monkeypatch.setattr(m, "_attn_workspace", lambda d, given: (None, 0))
    for name in ("_nat", "_nat_addresses", "_nat_attn_table", "_nat_layer_table"):
        monkeypatch.setattr(m, name, None)


def _row(n, heads, dim=64):
    """[2, n, heads, dim] of one row of one head."""
    return torch.zeros(dim).expand(2, n, heads, dim)


@pytest.mark.parametrize("which", ["q", "suffix", "cache", "out"])
def test_attention_operands(host, which):
    q, k, c = torch.zeros(2, 4, 4, 64), torch.zeros(2, 4, 2, 64), torch.zeros(2, 16, 2, 64)
    out, i = q.clone(), torch.zeros(2, dtype=torch.int32)
    if which == "q":
        q = _row(4, 4)
    elif which == "suffix":
        k = _row(4, 2)
    elif which == "cache":
        c = _row(16, 2)
    else:
        out = _row(4, 4)
    for call in (lambda: m.AttnLayerTable([q], [k], [k], [c], [c], [out]), lambda: m.attn_step(q, k, k, c, c, i, i, out=out),
                 lambda: m.attn_step(q, k, k, c, c, i, i, out=out, cache_row_index=torch.zeros((2, 16), dtype=torch.int32))):
        with pytest.raises(m.LspError, match="broadcast"):
            call()


@pytest.mark.gpu
def test_the_native_path_refuses_them_too():
    q, k, c = torch.zeros(2, 4, 4, 64).cuda(), torch.zeros(2, 4, 2, 64).cuda(), torch.zeros(2, 16, 2, 64).cuda()
    i = torch.zeros(2, dtype=torch.int32).cuda()
    m.lib()
    assert m._nat is not None
    for bad in (dict(q=q.new_zeros(64).expand(2, 4, 4, 64)), dict(k=k.new_zeros(64).expand(2, 4, 2, 64)),
                dict(c=c.new_zeros(64).expand(2, 16, 2, 64)), dict(out=q.new_zeros(64).expand(2, 4, 4, 64))):
        a = {**dict(q=q, k=k, c=c, out=q.clone()), **bad}
        with pytest.raises(m.LspError, match="broadcast"):
            m.AttnLayerTable([a["q"]], [a["k"]], [a["k"]], [a["c"]], [a["c"]], [a["out"]])
        with pytest.raises(m.LspError, match="broadcast"):
            m.attn_step(a["q"], a["k"], a["k"], a["c"], a["c"], i, i, out=a["out"])


@pytest.mark.parametrize("which", ["suffix", "cache"])
def test_rows_that_are_committed(host, which):
    """Caches and suffix buffers of a layer table, which commits, appends and evictions go by."""
    k, c = torch.zeros(2, 4, 2, 64), torch.zeros(2, 16, 2, 64)
    if which == "suffix":
        k = k[:1].expand(2, 4, 2, 64)
    else:
        c = c[:1].expand(2, 16, 2, 64)
    with pytest.raises(m.LspError, match="broadcast"):
        m.LayerTable([k], [k], [c], [c])
    one = m.LayerTable([k[:1]], [k[:1]], [c[:1]], [c[:1]])      # (one sequence's stride is of no use)
    assert one.B == 1 and one.C == 16


@pytest.mark.gpu
def test_the_native_table_refuses_them_too():
    k, c = torch.zeros(2, 4, 2, 64).cuda(), torch.zeros(2, 16, 2, 64).cuda()
    m.lib()
    assert m._nat_layer_table is not None
    for a in ([k[:1].expand(2, 4, 2, 64), c], [k, c[:1].expand(2, 16, 2, 64)]):
        with pytest.raises(m.LspError, match="broadcast"):
            m.LayerTable([a[0]], [a[0]], [a[1]], [a[1]])


def test_keys_and_values_of_a_table_are_laid_out_alike(host):
    """One batch stride is handed over for both."""
    k, c = torch.zeros(2, 4, 2, 64), torch.zeros(2, 16, 2, 64)
    wide = torch.zeros(2, 20, 2, 64)
    for a in ((k, wide[:, :4], c, c), (wide[:, :4], k, c, c), (k, k, c, wide[:, :16]), (k, k, wide[:, :16], c), (k, k[:, :3], c, c), (k, k, c[:, :9], c)):
        with pytest.raises(m.LspError, match="share"):
            m.LayerTable(*[[t] for t in a])
    m.LayerTable([k], [k], [wide[:, :16]], [wide[:, 4:]])
    m.LayerTable([k[:1]], [wide[:1, :4]], [c[:1]], [wide[:1, :16]])      # (one sequence's stride is of no use)


@pytest.mark.parametrize("S", [1, 5])
def test_logits_hidden_states_and_weights(host, S):
    """(All but one of size 1 is a tensor that a stride of 0 says nothing about.)"""
    i = torch.zeros((2, S), dtype=torch.int32)
    out = (i, i.float(), i.float())
    z = torch.zeros(8)
    for bad in (z.expand(2, S, 8), torch.zeros(1, S, 8).expand(2, S, 8), torch.zeros(2, 1, 8).expand(2, 5, 8)):
        o = tuple(torch.zeros(bad.shape[:2], dtype=t.dtype) for t in out)
        for call in (lambda: m.confidence(bad), lambda: m.confidence(bad, out=o), lambda: m.confidence_static(bad, None, o),
                     lambda: m.lm_head_confidence(bad, torch.zeros(16, 8)), lambda: m.lm_head_confidence(bad, torch.zeros(16, 8), out=o)):
            with pytest.raises(m.LspError, match="broadcast"):
                call()
    with pytest.raises(m.LspError, match="broadcast"):
        m.lm_head_confidence(torch.zeros(2, S, 8), z.expand(16, 8))


@pytest.mark.gpu
def test_the_native_reductions_refuse_them_too():
    z, w = torch.zeros(2, 5, 64).cuda().bfloat16(), torch.zeros(32, 64).cuda().bfloat16()
    f = torch.zeros(2, 5).cuda()
    out = (f.int(), f, f.clone())
    for bad in (z[:1].expand(2, 5, 64), z[:, :1].expand(2, 5, 64)):
        for call in (lambda: m.confidence(bad), lambda: m.lm_head_confidence(bad, w, out=out, workspace=torch.zeros(1 << 20, dtype=torch.uint8).cuda()),
                     lambda: m.token_scores(bad, out=(None, f, None, None))):
            with pytest.raises(m.LspError, match="broadcast"):
                call()
    with pytest.raises(m.LspError, match="broadcast"):
        m.lm_head_confidence(z, w[:1].expand(32, 64), out=out, workspace=torch.zeros(1 << 20, dtype=torch.uint8).cuda())
