"""Refusals of the decode-step entry points and the sizes they ask for: checked
before any device work, so no GPU is needed (the pointers are never followed)."""
import ctypes

import numpy as np
import pytest

from paper_2607_17154_amd import ordermoe as om

P = 1 << 20            # a 16-byte aligned address that nothing reads


def _cache(**kw):
    a = dict(format=om.CACHE_INT8, n_kv=2, head_dim=128, page_size=16, n_pages=4, k_codes=P, v_codes=P, k_scale=P, v_scale=P)
    a.update(kw)
    return om.Cache(**a)


def _heads(**kw):
    a = dict(dtype=om.BF16, n_q=4, rotary_dim=128, interleaved=0, max_pos=10, eps=1e-6, q_norm=P, k_norm=P, cos_sin=P)
    a.update(kw)
    return om.Heads(**a)


def _write(cache, heads, q=P, qs=512, k=P, ks=256, v=P, vs=256, T=3, pos=P, slots=P, out=P):
    return om.lib().ordermoe_cache_write(ctypes.byref(cache) if cache else None, ctypes.byref(heads) if heads else None, q, qs, k,
                                         ks, v, vs, T, pos, slots, out, None)


CACHE_BAD = [dict(format=2), dict(n_kv=0), dict(n_kv=1025), dict(head_dim=96), dict(head_dim=0), dict(page_size=8),
             dict(page_size=48), dict(page_size=2048), dict(n_pages=0), dict(n_pages=1 << 31), dict(k_codes=0), dict(v_codes=P + 8),
             dict(k_scale=P + 4), dict(v_scale=None)]


@pytest.mark.parametrize("kw", CACHE_BAD)
def test_a_bad_cache_is_refused_everywhere(kw):
    c = _cache(**kw)
    want = om.EDTYPE if "format" in kw else om.EINVAL
    assert _write(c, _heads()) == want and om.last_error()
    assert om.lib().ordermoe_cache_read(ctypes.byref(c), om.F32, P, 1, P, P, None) == want
    assert om.lib().ordermoe_draft_attention_workspace_size(ctypes.byref(c), om.BF16, 4, 1, 1) == 0
    assert _attend(c) == want


@pytest.mark.parametrize("heads,args", [
    (dict(dtype=5), {}), (dict(n_q=3), {}), (dict(n_q=0), {}), (dict(n_q=1026), {}), (dict(rotary_dim=8), {}),
    (dict(rotary_dim=144), {}), (dict(rotary_dim=-16), {}), (dict(interleaved=2), {}), (dict(eps=-1.0), {}),
    (dict(eps=float("nan")), {}), (dict(eps=float("inf")), {}), (dict(max_pos=0), {}), (dict(cos_sin=None), {}), (dict(q_norm=P + 2), {}),
    (dict(cos_sin=P + 4), {}),
    ({}, dict(T=-1)), ({}, dict(T=1 << 29)), ({}, dict(q=0)), ({}, dict(k=0)), ({}, dict(v=0)), ({}, dict(pos=0)),
    ({}, dict(slots=0)), ({}, dict(out=0)), ({}, dict(q=P + 8)), ({}, dict(out=P + 4)), ({}, dict(qs=504)), ({}, dict(ks=260)),
    ({}, dict(vs=0)), (dict(dtype=om.F32), dict(ks=258)),
])
def test_write_refusals(heads, args):
    assert _write(_cache(), _heads(**heads), **args) == (om.EDTYPE if heads.get("dtype") == 5 else om.EINVAL)
    assert "cache_write" in om.last_error()


def test_null_structs_are_refused():
    assert _write(None, _heads()) == om.EINVAL
    assert _write(_cache(), None) == om.EINVAL


def _attend(cache, dtype=om.BF16, n_q=4, q=P, T=3, B=2, max_q=2, qs=P, ctx=P, table=P, max_pages=4, tree=None, scale=0.1,
            out=P, lse=None, ws=P, ws_bytes=1 << 40):
    return om.lib().ordermoe_draft_attention(ctypes.byref(cache), dtype, n_q, q, T, B, max_q, qs, ctx, table, max_pages, tree,
                                             scale, out, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), om.EDTYPE), (dict(n_q=3), om.EINVAL), (dict(n_q=0), om.EINVAL), (dict(n_q=2048), om.EINVAL),
    (dict(B=-1), om.EINVAL), (dict(B=65536), om.EINVAL), (dict(max_q=0), om.EINVAL), (dict(max_q=65), om.EINVAL),
    (dict(T=-1), om.EINVAL), (dict(T=1 << 31), om.EINVAL), (dict(max_pages=0), om.EINVAL), (dict(max_pages=1 << 27), om.EINVAL),
    (dict(scale=float("nan")), om.EINVAL), (dict(scale=float("inf")), om.EINVAL), (dict(q=0), om.EINVAL), (dict(q=P + 8), om.EINVAL),
    (dict(qs=0), om.EINVAL), (dict(ctx=0), om.EINVAL), (dict(table=0), om.EINVAL), (dict(out=0), om.EINVAL),
    (dict(out=P + 2), om.EINVAL), (dict(ws=0), om.EWORKSPACE), (dict(ws_bytes=100), om.EWORKSPACE),
])
def test_attention_refusals(kw, code):
    assert _attend(_cache(), **kw) == code
    assert "draft_attention" in om.last_error()


def test_attention_of_nothing_is_fine():
    assert _attend(_cache(), T=0) == om.OK
    assert _attend(_cache(), B=0) == om.OK
    assert om.last_error() == ""


def test_read_refusals():
    c, L = _cache(), om.lib()
    f = lambda dt=om.F32, slots=P, n=5, k=P, v=P: L.ordermoe_cache_read(ctypes.byref(c), dt, slots, n, k, v, None)  # noqa: E731
    assert f(dt=3) == om.EDTYPE
    for kw in (dict(slots=0), dict(n=-1), dict(n=1 << 30), dict(k=0), dict(v=0), dict(k=P + 4)):
        assert f(**kw) == om.EINVAL, kw
    assert f(n=0, slots=0, k=0, v=0) == om.OK


def test_attention_workspace_grows_with_the_batch_and_the_drafts():
    c, L = _cache(n_kv=8), om.lib()
    size = lambda B, n: L.ordermoe_draft_attention_workspace_size(ctypes.byref(c), om.BF16, 32, B, n)  # noqa: E731
    assert 0 < size(1, 1) < size(8, 1) < size(8, 64)
    # every sequence's rows at least once
    assert size(8, 64) >= 8 * 64 * 32 * 128 * 4


def test_rotary_table():
    t = om.rotary_table(5, 8, 100.0)
    assert t.shape == (5, 8) and t.dtype == np.float32
    np.testing.assert_allclose(t[3], np.concatenate([np.cos(3 * 100.0 ** (-np.arange(4) / 4)), np.sin(3 * 100.0 ** (-np.arange(4) / 4))]),
                               rtol=1e-6)
    assert om.rotary_table(4, 0).shape == (4, 0)


def _few_structs(layer=None, experts=None):
    ids = np.array([0, 3], np.int32)
    la = dict(dtype=om.BF16, d=256, E=8, k=2, M=2, gmax=3, pin_local_exact=1, allow_sub=1, renorm=1, Qbar=0.25, omega_Q=0.5,
              w_router=P, t1_k=P, t1_q=P, t1_n=P, srvmask=P, S=P)
    ea = dict(dtype=om.BF16, d=256, f=128, E=8, n_local=2, n_shared=1, local_experts=ids.ctypes.data, w_gate_up=P, w_down=P,
              w_shared_gate_up=P, w_shared_down=P)
    la.update(layer or {})
    ea.update(experts or {})
    e = om.Experts(**ea)
    e._ids = ids
    return om.Layer(**la), e, om.RouteOut(**{n: P for n, _ in om.RouteOut._fields_})


def _few(L, E, out, x=P, T=4, loc=P, qhat=P, server=0, y=P, ws=P, ws_bytes=1 << 40):
    r = ctypes.byref
    return om.lib().ordermoe_few_moe_layer(r(L) if L else None, r(E) if E else None, x, T, loc, qhat, server, r(out) if out else None,
                                           y, ws, ws_bytes, None)


@pytest.mark.parametrize("layer,experts,args,code", [
    (dict(dtype=7), {}, {}, om.EINVAL), ({}, dict(dtype=7), {}, om.EDTYPE), (dict(d=512), {}, {}, om.EINVAL),
    (dict(E=9), {}, {}, om.EINVAL), (dict(dtype=om.F32), {}, {}, om.EINVAL), (dict(d=100), dict(d=100), {}, om.EINVAL),
    ({}, dict(f=100), {}, om.EINVAL), ({}, dict(n_local=9), {}, om.EINVAL), ({}, dict(w_gate_up=P + 8), {}, om.EINVAL),
    (dict(k=9), {}, {}, om.EINVAL), (dict(M=0), {}, {}, om.EINVAL), (dict(gmax=16), {}, {}, om.EINVAL), (dict(S=None), {}, {}, om.EINVAL),
    (dict(w_router=P + 2), {}, {}, om.EINVAL), ({}, {}, dict(T=-1), om.EINVAL), ({}, {}, dict(T=17), om.EINVAL),
    ({}, {}, dict(x=0), om.EINVAL), ({}, {}, dict(x=P + 8), om.EINVAL), ({}, {}, dict(loc=0), om.EINVAL),
    ({}, {}, dict(qhat=0), om.EINVAL), ({}, {}, dict(y=0), om.EINVAL), ({}, {}, dict(y=P + 4), om.EINVAL),
    ({}, {}, dict(server=32), om.EINVAL), ({}, {}, dict(server=-1), om.EINVAL), ({}, {}, dict(ws=0), om.EWORKSPACE),
    ({}, {}, dict(ws_bytes=64), om.EWORKSPACE),
])
def test_few_layer_refusals(layer, experts, args, code):
    L, E, out = _few_structs(layer, experts)
    assert _few(L, E, out, **args) == code
    assert om.last_error()


def test_few_layer_null_structs_and_sizes():
    L, E, out = _few_structs()
    assert _few(None, E, out) == om.EINVAL and _few(L, None, out) == om.EINVAL and _few(L, E, None) == om.EINVAL
    size = lambda T: om.lib().ordermoe_few_workspace_size(ctypes.byref(L), ctypes.byref(E), T)  # noqa: E731
    assert size(1) > 0 and size(16) > 0 and size(17) == 0 and size(-1) == 0
