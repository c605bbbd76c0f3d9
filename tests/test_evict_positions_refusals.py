"""Eviction by positions refuses on the host what its kernel would misread (no GPU needed: nothing is launched)."""
import ctypes

import pytest
import torch

import paper_2603_05454_amd as m

BUF = (ctypes.c_int32 * 256)()


def _p(off=0):
    return ctypes.c_void_p(((ctypes.addressof(BUF) + 15) & ~15) + off)


def test_entry_point():
    L, p = m.lib(), _p()
    one = (ctypes.c_void_p * 1)(p.value)

    def call(at=p, T=_p(512), nl=p, **kw):
        d = m.EvictDesc(**{**dict(kv_dtype=1, B=2, Hkv=2, D=64, C=40, num_layers=1, keep=20, high=20, first=1, recent=4), **kw})
        return L.lsp_kv_evict_positions(ctypes.byref(d), p, at, T, p, one, one, p, nl, None, p, ctypes.c_size_t(1 << 20), None)
    for kw, word in ((dict(at=None), b"null"), (dict(T=None), b"null"), (dict(T=p), b"new_len"), (dict(T=_p(4)), b"new_len"), (dict(nl=_p(516)), b"new_len"),
                     (dict(keep=41, high=41), b"keep"), (dict(first=10, recent=11), b"first")):
        assert call(**kw) == -1 and word in L.lsp_last_error(), (kw, L.lsp_last_error())
    assert L.lsp_kv_evict_positions(None, p, p, _p(512), p, one, one, p, p, None, p, ctypes.c_size_t(0), None) == -1 and b"null descriptor" in L.lsp_last_error()


def test_the_binding_refuses_wrong_tensors(monkeypatch):
    """Host tensors stand in for device tensors: a call that got past the checks would reach the library, which is not there."""
    monkeypatch.setattr(m, "_here", lambda *ts: None)
    monkeypatch.setattr(m, "_dev", lambda *ts: None)
    monkeypatch.setattr(m, "lib", lambda: pytest.fail("the call reached the library"))
    for name in ("_nat", "_nat_addresses", "_nat_attn_table", "_nat_layer_table"):
        monkeypatch.setattr(m, name, None)
    k, c = torch.zeros(2, 4, 2, 64), torch.zeros(2, 16, 2, 64)
    lay, w, P = m.LayerTable([k], [k], [c], [c]), torch.zeros(1, 2, 2, 16), torch.zeros(2, dtype=torch.int32)
    at = torch.zeros((1, 2, 2, 16), dtype=torch.int32)
    for text, kw in (("together", dict(positions=at)), ("together", dict(token_len=P)), ("positions must be torch.int32", dict(positions=at.float(), token_len=P)),
                     ("positions must have shape", dict(positions=at[:, :1], token_len=P)), ("token_len must have shape", dict(positions=at, token_len=P[:1])),
                     ("token_len must be torch.int32", dict(positions=at, token_len=P.long()))):
        with pytest.raises(m.LspError, match=text):
            m.kv_evict(w, P, lay, 8, **kw)
