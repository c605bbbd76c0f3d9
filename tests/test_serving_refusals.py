"""Token scores, key weights and eviction refuse on the host what their kernels would misread (no GPU needed: nothing is launched)."""
import ctypes

import pytest
import torch

import paper_2603_05454_amd as m


def _p(buf, off=0):
    return ctypes.c_void_p(((ctypes.addressof(buf) + 15) & ~15) + off)


BUF = (ctypes.c_int32 * 64)()


def test_token_scores_entry_point():
    L, p, i64 = m.lib(), _p(BUF), ctypes.c_int64

    def call(dtype=1, z=p, B=1, S=4, V=8, row=0, batch=0, ids=p, K=2, lp=p, h=p, ai=p, al=p):
        return L.lsp_token_scores(dtype, z, B, S, V, i64(row), i64(batch), None, ids, K, lp, h, ai, al, None, ctypes.c_size_t(0), None)
    for kw, word in ((dict(dtype=2), b"dtype"), (dict(z=None), b"null"), (dict(h=None), b"null"), (dict(V=0), b"V>0"), (dict(B=70000), b"65535"),
                     (dict(K=-1), b"num_alt"), (dict(K=33), b"num_alt"), (dict(ai=None), b"alt_id"), (dict(al=None), b"alt_id"),
                     (dict(lp=None), b"together"), (dict(ids=None), b"together"), (dict(row=7), b"strides"), (dict(batch=-8), b"strides"),
                     (dict(z=_p(BUF, 1)), b"misaligned")):
        assert call(**kw) == -1 and word in L.lsp_last_error(), kw
    assert L.lsp_token_scores_workspace_bytes(0, 4, 8, 0) == 0


def test_key_weights_entry_point():
    L, p = m.lib(), _p(BUF)
    one = (ctypes.c_void_p * 1)(p.value)

    def call(d, n=1, q=one, ks=one, kc=one, P=p, N=p, decay=1.0, w=p, ws=p, wsb=1 << 20):
        return L.lsp_attn_key_weights(ctypes.byref(d), n, q, ks, kc, P, N, ctypes.c_float(decay), w, ws, ctypes.c_size_t(wsb), None)
    d = lambda **kw: m.AttnDesc(**{**dict(dtype=1, B=1, S=4, Hq=4, Hkv=2, D=128, C=8), **kw})      # noqa: E731
    for desc, kw, rc, word in ((d(Hq=3), {}, -1, b"multiple"), (d(S=0), {}, -1, b"dimension"), (d(dtype=3), {}, -1, b"dtype"), (d(D=96), {}, -2, b"head_dim"),
                               (d(), dict(n=0), -1, b"num_layers"), (d(), dict(q=None), -1, b"null"), (d(), dict(w=None), -1, b"null"),
                               (d(), dict(decay=1.5), -1, b"decay"), (d(), dict(decay=float("nan")), -1, b"decay"), (d(), dict(ws=None), -3, b"workspace"),
                               (d(), dict(wsb=8), -3, b"workspace"), (d(), dict(ws=_p(BUF, 4)), -3, b"workspace"),
                               (d(), dict(kc=(ctypes.c_void_p * 1)(0)), -1, b"layer 0"), (d(), dict(q=(ctypes.c_void_p * 1)(p.value + 2)), -1, b"aligned")):
        assert call(desc, **kw) == rc and word in L.lsp_last_error(), (kw, L.lsp_last_error())
    assert L.lsp_attn_key_weights_workspace_bytes(None, 1) == 0 and L.lsp_attn_key_weights_workspace_bytes(ctypes.byref(d()), 0) == 0


def test_evict_entry_point():
    L, p = m.lib(), _p(BUF)
    one = (ctypes.c_void_p * 1)(p.value)

    def call(kc=one, vc=one, w=p, P=p, nw=p, nl=p, ws=p, wsb=1 << 20, **kw):
        d = m.EvictDesc(**{**dict(kv_dtype=1, B=1, Hkv=2, D=64, C=40, num_layers=1, keep=20, high=20, first=1, recent=4), **kw})
        return L.lsp_kv_evict(ctypes.byref(d), w, P, kc, vc, nw, nl, None, ws, ctypes.c_size_t(wsb), None)
    for kw, rc, word in ((dict(kv_dtype=5), -1, b"kv_dtype"), (dict(B=0), -1, b"dimension"), (dict(num_layers=0), -1, b"dimension"), (dict(keep=0), -1, b"keep"),
                         (dict(keep=41, high=41), -1, b"keep"), (dict(high=19), -1, b"high"), (dict(first=-1), -1, b"first"),
                         (dict(first=10, recent=11), -1, b"first"), (dict(first=2 ** 31 - 1, recent=2 ** 31 - 1), -1, b"first"), (dict(D=4), -1, b"multiple of 16"),
                         (dict(cache_batch_stride=100), -1, b"stride"), (dict(w=None), -1, b"null"), (dict(nl=None), -1, b"null"),
                         (dict(kc=(ctypes.c_void_p * 1)(0)), -1, b"layer 0"), (dict(vc=(ctypes.c_void_p * 1)(p.value + 8)), -1, b"aligned"),
                         (dict(C=9000, ws=None), -3, b"workspace"), (dict(C=9000, wsb=8), -3, b"workspace"), (dict(D=1 << 17), -1, b"65536"),
                         (dict(C=1 << 30), -1, b"2^30"), (dict(B=65535, Hkv=65535), -1, b"many heads")):
        assert call(**kw) == rc and word in L.lsp_last_error(), (kw, L.lsp_last_error())
    assert L.lsp_kv_evict_workspace_bytes(None) == 0


def test_sizes_beyond_what_is_counted_in_32_bits():
    L, p, i64 = m.lib(), _p(BUF), ctypes.c_int64
    assert L.lsp_token_scores(1, p, 1, 1, (1 << 30) + 1, i64(0), i64(0), None, None, 0, None, p, None, None, None, ctypes.c_size_t(0), None) == -1
    assert b"2^30" in L.lsp_last_error()
    one = (ctypes.c_void_p * 1)(p.value)
    for size in (dict(C=(1 << 30) - 3), dict(S=(1 << 30) - 7), dict(S=1 << 28, Hq=32, Hkv=4), dict(C=2 ** 31 - 1, S=2 ** 31 - 1)):
        d = m.AttnDesc(**{**dict(dtype=1, B=1, S=4, Hq=4, Hkv=4, D=128, C=8), **size})
        assert L.lsp_attn_key_weights(ctypes.byref(d), 1, one, one, one, p, p, ctypes.c_float(1), p, p, ctypes.c_size_t(1 << 62), None) == -1, size
        assert b"2^30" in L.lsp_last_error(), size


def test_the_binding_refuses_wrong_tensors(monkeypatch):
    """Host tensors stand in for device tensors: a call that got past the checks would reach the library, which is not there."""
    monkeypatch.setattr(m, "_here", lambda *ts: None)
    monkeypatch.setattr(m, "_dev", lambda *ts: None)
    monkeypatch.setattr(m, "lib", lambda: pytest.fail("the call reached the library"))
    monkeypatch.setattr(m, "_nat", None)
    for name in ("_nat_addresses", "_nat_attn_table", "_nat_layer_table"):
        monkeypatch.setattr(m, name, None)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)     # noqa: E731
    f32 = lambda *s: torch.zeros(s)                        # noqa: E731
    z = f32(2, 4, 64)
    q, k, c = f32(2, 4, 4, 64), f32(2, 4, 2, 64), f32(2, 16, 2, 64)
    lay = m.LayerTable([k], [k], [c], [c])
    tab = m.AttnLayerTable([q], [k], [k], [c], [c], [q])
    out = (f32(2, 4), f32(2, 4), i32(2, 4, 3), f32(2, 4, 3))
    cases = [
        ("token_id must be torch.int32", lambda: m.token_scores(z, i32(2, 4).long())),
        ("token_id must have shape", lambda: m.token_scores(z, i32(2, 5))),
        ("suffix_len must be torch.int32", lambda: m.token_scores(z, None, i32(2).long())),
        ("num_alt", lambda: m.token_scores(z, num_alt=33)),
        ("contiguous rows", lambda: m.token_scores(z.transpose(1, 2))),
        ("out must be", lambda: m.token_scores(z, i32(2, 4), out=out[:3])),
        ("alt_id", lambda: m.token_scores(z, i32(2, 4), num_alt=2, out=out)),
        ("needs token_id", lambda: m.token_scores(z, None, num_alt=3, out=out)),
        ("logprob", lambda: m.token_scores(z, i32(2, 4), num_alt=3, out=(None, *out[1:]))),
        ("k_suf must be", lambda: m.attn_key_weights(q, k.bfloat16(), c, i32(2), i32(2), f32(2, 2, 16))),
        ("k_cache must be", lambda: m.attn_key_weights(q, k, c[:, :, :1], i32(2), i32(2), f32(2, 2, 16))),
        ("weights must have shape", lambda: m.attn_key_weights(q, k, c, i32(2), i32(2), f32(2, 2, 15))),
        ("weights must be torch.float32", lambda: m.attn_key_weights(q, k, c, i32(2), i32(2), f32(2, 2, 16).double())),
        ("prefix_len must be", lambda: m.attn_key_weights(q, k, c, i32(2).long(), i32(2), f32(2, 2, 16))),
        ("weights must have shape", lambda: m.attn_key_weights_layers(tab, i32(2), i32(2), f32(2, 2, 16))),
        ("weights must have shape", lambda: m.kv_evict(f32(2, 2, 16), i32(2), lay, 8)),
        ("new_weights must", lambda: m.kv_evict(f32(1, 2, 2, 16), i32(2), lay, 8, new_weights=f32(1, 2, 2, 8))),
        ("new_len must", lambda: m.kv_evict(f32(1, 2, 2, 16), i32(2), lay, 8, new_len=i32(3))),
        ("broadcast", lambda: m.token_scores(f32(1, 1, 64).expand(2, 4, 64), i32(2, 4))),
        ("broadcast", lambda: m.attn_key_weights(f32(1, 1, 1, 64).expand(2, 4, 4, 64), k, c, i32(2), i32(2), f32(2, 2, 16))),
        ("broadcast", lambda: m.kv_evict(f32(1, 2, 2, 16), i32(2), m.LayerTable([k], [k], [c[:1].expand(2, 16, 2, 64)], [c[:1].expand(2, 16, 2, 64)]), 8)),
        ("kept_index must", lambda: m.kv_evict(f32(1, 2, 2, 16), i32(2), lay, 8, kept_index=i32(1, 2, 2, 9))),
    ]
    for text, call in cases:
        with pytest.raises(m.LspError, match=text):
            call()


def test_host_tensors_are_refused():
    z = torch.zeros(1, 2, 8)
    with pytest.raises(m.LspError, match="device tensors only"):
        m.token_scores(z)
    with pytest.raises(m.LspError, match="device tensors only"):
        m.attn_key_weights(z[None], z[None], z[None], z, z, z)
