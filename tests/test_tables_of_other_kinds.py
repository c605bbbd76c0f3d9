"""A call takes the table that is its own: another kind's lists of addresses are in another order, and their caches of another size (no GPU needed:
nothing is launched)."""
import pytest
import torch

import paper_2603_05454_amd as m

B, S, HQ, H, D, C = 2, 5, 4, 2, 64, 70


@pytest.fixture(params=["native", "general"])
def no_device(request, monkeypatch):
    """Host tensors stand in for device tensors; a call that got past the checks would reach the library.  The native module takes six lists of addresses
    for lsp_attn_step_layers, and answers None (the general path looks) where there are others."""
    m.lib()
    real = m.lib()
    native = m._nat
    for name in ("_here", "_dev", "_table_here"):
        monkeypatch.setattr(m, name, lambda *ts: None)
    monkeypatch.setattr(m, "_nat", None)
    for name in ("_nat_attn_table", "_nat_layer_table"):
        monkeypatch.setattr(m, name, None)
    monkeypatch.setattr(m, "_addresses", lambda lst: None)
    tables = _tables()
    if request.param == "native":
        if native is None:
            pytest.skip("the native module is not built")
        monkeypatch.setattr(m, "_nat", native)

    class Refusing:
        def __getattr__(self, n):
            if n.endswith("_workspace_bytes"):
                return lambda *a: 0
            return lambda *a: pytest.fail(f"the call reached {n}")
    monkeypatch.setattr(m, "lib", lambda: Refusing())
    assert real is not None
    return tables


def _tables():
    bf = dict(dtype=torch.bfloat16)
    kc, vc, ke, ve = m.q8_cache(B, C, H, D, device="cpu")
    q, out = (torch.zeros(B, S, HQ, D, **bf) for _ in range(2))
    ks, vs = (torch.zeros(B, S, H, D, **bf) for _ in range(2))
    kc16, vc16 = (torch.zeros(B, C, H, D, **bf) for _ in range(2))
    return dict(q8=m.Q8LayerTable([ks], [vs], [kc], [vc], [ke], [ve], q=[q], out=[out]), q8_without=m.Q8LayerTable([ks], [vs], [kc], [vc], [ke], [ve]),
                attn=m.AttnLayerTable([q], [ks], [vs], [kc16], [vc16], [out]), layers=m.LayerTable([ks], [vs], [kc16], [vc16]))


@pytest.mark.parametrize("kind", ["q8", "q8_without", "layers"])
def test_attention_over_caches_of_16_bits(no_device, kind):
    n = torch.ones(B, dtype=torch.int32)
    with pytest.raises(m.LspError, match="AttnLayerTable"):
        m.attn_step_layers(no_device[kind], n, n)
    with pytest.raises(m.LspError, match="AttnLayerTable"):
        m.attn_key_weights_layers(no_device[kind], n, n, torch.zeros(1, B, H, C))


@pytest.mark.parametrize("kind", ["attn", "layers"])
def test_caches_of_8_bits(no_device, kind):
    n, out = torch.ones(B, dtype=torch.int32), [torch.zeros(B, S, H, D)]
    with pytest.raises(m.LspError, match="Q8LayerTable"):
        m.attn_step_q8_layers(no_device[kind], n, n)
    with pytest.raises(m.LspError, match="Q8LayerTable"):
        m.kv_append_q8(no_device[kind], n, n)
    with pytest.raises(m.LspError, match="Q8LayerTable"):
        m.kv_read_q8(no_device[kind], n, n, out, out)
