"""The calls of caches in 8 bits refuse on the host what their kernels would misread (no GPU needed: nothing is launched)."""
import ctypes
import os
import re

import pytest
import torch

import paper_2603_05454_amd as m

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BUF = (ctypes.c_int32 * 64)()


def _p(off=0):
    return ctypes.c_void_p(((ctypes.addressof(BUF) + 15) & ~15) + off)


def test_every_declared_name_is_exported():
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "lsp.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(lsp_\w+)\s*\(", src))
    assert names == set(m.EXPORTS) | set(m.EXPORTS_Q8)
    for n in names:
        assert hasattr(m.lib(), n), n


def _desc(**kw):
    return m.AttnDesc(**{**dict(dtype=1, B=1, S=4, Hq=4, Hkv=2, D=128, C=40), **kw})


def _strides(*s):
    return (ctypes.c_int64 * 3)(*s)


ONE = (ctypes.c_void_p * 1)(_p().value)
NULL, ODD = (ctypes.c_void_p * 1)(0), (ctypes.c_void_p * 1)(_p().value + 8)
COMMON = [   # descriptor, arguments, status, word
    (dict(S=0), {}, -1, b"dimension"), (dict(dtype=3), {}, -1, b"dtype"), (dict(D=96), {}, -2, b"head_dim"), (dict(D=256), {}, -2, b"head_dim"),
    (dict(B=70000), {}, -1, b"65535"), (dict(cache_stride=_strides(40 * 256 + 8, 256, 128)), {}, -1, b"16 bytes"),
    (dict(cache_stride=_strides(1 << 30, (1 << 24) + 16, 128)), {}, -1, b"row strides"), (dict(cache_stride=_strides(40 * 256, 256, 64)), {}, -1, b"bad strides"),
    (dict(C=(1 << 30) + 1), {}, -1, b"2^30"), (dict(S=(1 << 30) + 1), {}, -1, b"2^30"), ({}, dict(n=0), -1, b"num_layers"),
    ({}, dict(kc=None), -1, b"null"), ({}, dict(ke=None), -1, b"null"), ({}, dict(x=None), -1, b"null"), ({}, dict(y=None), -1, b"null"),
    ({}, dict(kc=NULL), -1, b"layer 0"), ({}, dict(ke=NULL), -1, b"layer 0"), ({}, dict(kc=ODD), -1, b"aligned")]


@pytest.mark.parametrize("desc, kw, rc, word", COMMON + [
    (dict(B=2, cache_stride=_strides(0, 256, 128)), {}, -1, b"shared"), ({}, dict(ks=NULL), -1, b"layer 0"), ({}, dict(ks=ODD), -1, b"aligned"),
    (dict(S=1 << 30, Hkv=65535, Hq=65535), {}, -1, b"2^31")])
def test_append(desc, kw, rc, word):
    def call(d, n=1, ks=ONE, vs=ONE, kc=ONE, vc=ONE, ke=ONE, ve=ONE, x=_p(), y=_p()):
        return m.lib().lsp_kv_append_q8(ctypes.byref(d), n, ks, vs, kc, vc, ke, ve, x, y, None)
    assert call(_desc(**desc), **kw) == rc and word in m.lib().lsp_last_error(), m.lib().lsp_last_error()


@pytest.mark.parametrize("desc, kw, rc, word", COMMON + [
    (dict(B=2, kv_suf_stride=_strides(0, 256, 128)), {}, -1, b"shared"), ({}, dict(ko=NULL), -1, b"layer 0"), ({}, dict(vo=ODD), -1, b"aligned")])
def test_read(desc, kw, rc, word):
    def call(d, n=1, kc=ONE, vc=ONE, ke=ONE, ve=ONE, x=_p(), y=_p(), ko=ONE, vo=ONE):
        return m.lib().lsp_kv_read_q8(ctypes.byref(d), n, kc, vc, ke, ve, x, y, ko, vo, None)
    assert call(_desc(**desc), **kw) == rc and word in m.lib().lsp_last_error(), m.lib().lsp_last_error()


@pytest.mark.parametrize("desc, kw, rc, word", COMMON + [
    (dict(dtype=0), {}, -2, b"bf16"), (dict(Hq=3), {}, -1, b"multiple"), (dict(scale=-1.0), {}, -1, b"scale"),
    (dict(B=2, o_stride=_strides(0, 512, 128)), {}, -1, b"shared"), (dict(S=1 << 27, Hq=32, Hkv=1), {}, -1, b"2^30"), (dict(B=65535, Hq=2048, Hkv=2048), {}, -1, b"2^23"),
    ({}, dict(q=NULL), -1, b"layer 0"), ({}, dict(out=ODD), -1, b"aligned")])
def test_attention(desc, kw, rc, word):
    def call(d, n=1, q=ONE, ks=ONE, vs=ONE, kc=ONE, vc=ONE, ke=ONE, ve=ONE, x=_p(), y=_p(), out=ONE):
        return m.lib().lsp_attn_step_q8_layers(ctypes.byref(d), n, q, ks, vs, kc, vc, ke, ve, x, y, out, None, ctypes.c_size_t(0), None)
    assert call(_desc(**desc), **kw) == rc and word in m.lib().lsp_last_error(), m.lib().lsp_last_error()
    if not kw:
        assert m.lib().lsp_attn_q8_workspace_bytes(ctypes.byref(_desc(**desc)), 1) == 0


@pytest.mark.parametrize("desc, kw, rc, word", [
    (dict(dtype=2), {}, -1, b"dtype"), (dict(B=0), {}, -1, b"dimension"), (dict(S=(1 << 24) + 1), {}, -1, b"2^24"), (dict(D=80), {}, -2, b"head_dim"),
    (dict(R=24), {}, -1, b"R must"), (dict(R=144), {}, -1, b"R must"), (dict(R=-16), {}, -1, b"R must"), (dict(eps=-1.0), {}, -1, b"eps"),
    (dict(eps=float("nan")), {}, -1, b"eps"), ({}, dict(q=None), -1, b"null"), ({}, dict(f=None), -1, b"null"), ({}, dict(ko=None), -1, b"null"),
    ({}, dict(qw=_p()), -1, b"together"), ({}, dict(kw=_p()), -1, b"together"), ({}, dict(q=_p(8)), -1, b"aligned"),
    (dict(q_stride=_strides(4096, 512, 64)), {}, -1, b"strides"), (dict(k_stride=_strides(4096, 260, 130)), {}, -1, b"strides"),
    (dict(B=2, q_out_stride=_strides(0, 512, 128)), {}, -1, b"shared")])
def test_norm_rope(desc, kw, rc, word):
    d = m.QkNormRopeDesc(**{**dict(dtype=1, B=1, S=4, Hq=4, Hkv=2, D=128, R=128, eps=1e-6), **desc})

    def call(q=_p(), k=_p(), qw=None, kw=None, f=_p(), qo=_p(), ko=_p()):
        return m.lib().lsp_qk_norm_rope(ctypes.byref(d), q, k, qw, kw, f, None, None, None, qo, ko, None)
    assert call(**kw) == rc and word in m.lib().lsp_last_error(), m.lib().lsp_last_error()


@pytest.fixture
def no_device(monkeypatch):
    """Host tensors stand in for device tensors: a call that got past the checks would reach the library, which is not there."""
    monkeypatch.setattr(m, "_here", lambda *ts: None)
    monkeypatch.setattr(m, "_dev", lambda *ts: None)
    monkeypatch.setattr(m, "_nat", None)
    m.lib()
    return monkeypatch


B, S, HQ, H, D, C = 2, 5, 6, 2, 64, 70


def _tensors(**kw):
    bf = dict(dtype=torch.bfloat16)
    kc, vc, ke, ve = m.q8_cache(B, C, H, D, device="cpu")
    t = dict(q=torch.zeros(B, S, HQ, D, **bf), k_suf=torch.zeros(B, S, H, D, **bf), v_suf=torch.zeros(B, S, H, D, **bf), k_cache=kc, v_cache=vc, k_scale=ke,
             v_scale=ve, out=torch.zeros(B, S, HQ, D, **bf))
    t.update(kw)
    return t


WRONG = [dict(v_suf=torch.zeros(B, S, H, D)), dict(k_cache=torch.zeros(B, C, H, D, dtype=torch.uint8)), dict(k_cache=torch.zeros(B, C, H, D).to(torch.float8_e4m3fn)[:, ::2]),
         dict(k_scale=torch.zeros(B, H, 2, dtype=torch.uint8)), dict(v_scale=torch.zeros(B, H, 3)), dict(k_scale=torch.zeros(B, 3, H, dtype=torch.uint8).transpose(1, 2)),
         dict(v_cache=torch.zeros(B, C + 1, H, D).to(torch.float8_e4m3fn)[:, 1:]), dict(q=torch.zeros(B, S, HQ, D)), dict(q=torch.zeros(B, S + 1, HQ, D, dtype=torch.bfloat16)),
         dict(out=torch.zeros(B, S, HQ, D)), dict(out=torch.zeros(1, S, HQ, D, dtype=torch.bfloat16).expand(B, S, HQ, D)),
         dict(k_suf=torch.zeros(B, S, 1, D, dtype=torch.bfloat16).expand(B, S, H, D), v_suf=torch.zeros(B, S, 1, D, dtype=torch.bfloat16).expand(B, S, H, D))]


@pytest.mark.parametrize("wrong", range(len(WRONG)))
def test_the_binding_refuses_wrong_tensors(no_device, wrong):
    no_device.setattr(m, "lib", lambda: None)
    t = _tensors(**WRONG[wrong])
    names = ("q", "k_suf", "v_suf", "k_cache", "v_cache", "k_scale", "v_scale")
    n = torch.ones(B, dtype=torch.int32)
    with pytest.raises(m.LspError):
        m.attn_step_q8(*[t[x] for x in names], n, n, out=t["out"])
    with pytest.raises(m.LspError):
        m.Q8LayerTable(*[[t[x]] for x in names[1:]], q=[t["q"]], out=[t["out"]])


def test_tables_and_lengths(no_device):
    t = _tensors()
    lists = [[t[x]] for x in ("k_suf", "v_suf", "k_cache", "v_cache", "k_scale", "v_scale")]
    for bad in (dict(q=[t["q"]]), dict(q=[t["q"]] * 2, out=[t["out"]] * 2)):
        with pytest.raises(m.LspError):
            m.Q8LayerTable(*lists, **bad)
    with pytest.raises(m.LspError):
        m.Q8LayerTable(*[[]] * 6)
    table = m.Q8LayerTable(*lists)
    no_device.setattr(m, "_table_here", lambda t: None)
    real = m.lib()

    class Refusing:
        lsp_attn_q8_workspace_bytes = staticmethod(lambda *a: 0)

        def __getattr__(self, n):
            pytest.fail("the call reached the library")
    no_device.setattr(m, "lib", lambda: Refusing())
    good, short, wide = torch.ones(B, dtype=torch.int32), torch.ones(B - 1, dtype=torch.int32), torch.ones(B, dtype=torch.int64)
    for bad in (short, wide):
        for a in ((bad, good), (good, bad)):
            with pytest.raises(m.LspError):
                m.kv_append_q8(table, *a)
            with pytest.raises(m.LspError):
                m.kv_read_q8(table, *a, [torch.zeros(B, 3, H, D)], [torch.zeros(B, 3, H, D)])
            with pytest.raises(m.LspError):
                m.attn_step_q8(*[t[x] for x in ("q", "k_suf", "v_suf", "k_cache", "v_cache", "k_scale", "v_scale")], *a)
    out = torch.zeros(B, 3, H, D)
    for k, v in (([out], [out.half()]), ([out, out], [out, out]), ([torch.zeros(B, 3, H, 32)], [torch.zeros(B, 3, H, 32)]), ([out], [torch.zeros(B, 4, H, D)]),
                 ([out.half()], [out.half()]), ([torch.zeros(1, 3, H, D).expand(B, 3, H, D)],) * 2):
        with pytest.raises(m.LspError):
            m.kv_read_q8(table, good, good, k, v)
    with pytest.raises(m.LspError):
        m.attn_step_q8_layers(table, good, good)      # a table without q and out
    assert real is not None


@pytest.mark.parametrize("wrong", [dict(k=torch.zeros(B, S, H, D)), dict(k=torch.zeros(B, S, H, 32, dtype=torch.bfloat16)), dict(inv_freq=torch.zeros(33)),
                                   dict(inv_freq=torch.zeros(8, 4)), dict(inv_freq=torch.zeros(8).double()), dict(q_weight=torch.zeros(D, dtype=torch.bfloat16)),
                                   dict(k_weight=torch.zeros(D - 1)), dict(prefix_len=torch.zeros(B)), dict(suffix_len=torch.zeros(B + 1, dtype=torch.int32)),
                                   dict(positions=torch.zeros(B, S)), dict(positions=torch.zeros(S, dtype=torch.int32)), dict(out=(torch.zeros(B, S, HQ, D),)),
                                   dict(out=(torch.zeros(B, S, HQ, D), torch.zeros(B, S, H, D))), dict(q=torch.zeros(B, S, HQ, D, dtype=torch.float16)),
                                   dict(q=torch.zeros(1, S, HQ, D, dtype=torch.bfloat16).expand(B, S, HQ, D))])
def test_norm_rope_refuses_wrong_tensors(no_device, wrong):
    no_device.setattr(m, "lib", lambda: pytest.fail("the call reached the library"))
    t = dict(q=torch.zeros(B, S, HQ, D, dtype=torch.bfloat16), k=torch.zeros(B, S, H, D, dtype=torch.bfloat16), inv_freq=torch.zeros(32))
    t.update(wrong)
    with pytest.raises(m.LspError):
        m.qk_norm_rope(t.pop("q"), t.pop("k"), t.pop("inv_freq"), **t)


@pytest.mark.parametrize("S, C, word", [(1 << 20, 1 << 21, b"2^30"), (1 << 21, 1 << 20, b"2^30"), ((1 << 20) - 1, 1 << 21, b"layer 0"), (1 << 21, (1 << 20) - 1, b"layer 0")])
def test_read_counts_rows_of_heads_in_32_bits(S, C, word):
    d = _desc(S=S, C=C, Hq=1024, Hkv=1024, D=64)
    assert m.lib().lsp_kv_read_q8(ctypes.byref(d), 1, ONE, ONE, ONE, ONE, _p(), _p(), ONE, NULL, None) == -1
    assert word in m.lib().lsp_last_error(), m.lib().lsp_last_error()
