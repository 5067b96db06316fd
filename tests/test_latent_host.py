"""Refusals of the latent and prompt attention's entry points and of the eviction,
and the sizes they ask for: checked before any device work, so no GPU is needed
(the pointers are never followed)."""
import ctypes

import numpy as np
import pytest

from oracle import latent as ol
from paper_2607_17154_amd import ordermoe as om

P = 1 << 20            # a 16-byte aligned address that nothing reads
NAN, INF = float("nan"), float("inf")
ref = lambda s: ctypes.byref(s) if s else None  # noqa: E731


def _cache(**kw):
    a = dict(dtype=om.BF16, rank=512, rotary_dim=64, page_size=16, n_pages=4, rows=P)
    a.update(kw)
    return om.LatentCache(**a)


def _heads(**kw):
    a = dict(n_q=4, head_dim=128, interleaved=0, max_pos=10, eps=1e-6, norm=P, cos_sin=P, w_k=P, w_v=P)
    a.update(kw)
    return om.LatentHeads(**a)


def _write(c, h, q=P, qs=4 * 192, kv=P, kvs=576, T=3, pos=P, slots=P, absorb=1, out=P):
    return om.lib().ordermoe_latent_write(ref(c), ref(h), q, qs, kv, kvs, T, pos, slots, absorb, out, None)


def _attend(c, h, q=P, T=3, B=2, max_q=2, qs=P, ctx=P, table=P, max_pages=4, tree=None, scale=0.1, out=P, lse=None, mass=None,
            mass_out=None, stride=0, decay=1.0, ws=P, ws_bytes=1 << 40):
    return om.lib().ordermoe_latent_attention(ref(c), ref(h), q, T, B, max_q, qs, ctx, table, max_pages, tree, scale, out, lse, mass,
                                              mass_out, stride, decay, ws, ws_bytes, None)


def _expand(c, h, slots=P, n=5, k=P, r=P, v=P):
    return om.lib().ordermoe_latent_expand(ref(c), ref(h), slots, n, k, r, v, None)


def _prompt(dtype=om.BF16, n_q=8, n_kv=2, D=128, rot=64, q=P, T=5, k=P, r=P, v=P, L=7, B=2, qs=P, ks=P, scale=0.1, out=P, lse=None,
            ws=P, ws_bytes=1 << 40):
    return om.lib().ordermoe_prompt_attention(dtype, n_q, n_kv, D, rot, q, T, k, r, v, L, B, qs, ks, scale, out, lse, ws, ws_bytes, None)


def _evict(c, B=2, ctx=P, seq=P, table=P, max_pages=4, keep=10, first=1, recent=2, mass=P, pos=P, stride=64, kept=P, len_out=P,
           mass_out=P, pos_out=P, ws=P, ws_bytes=1 << 40):
    return om.lib().ordermoe_latent_evict(ref(c), B, ctx, seq, table, max_pages, keep, first, recent, mass, pos, stride, kept, len_out,
                                          mass_out, pos_out, ws, ws_bytes, None)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(rank=64), dict(rank=0), dict(rank=384), dict(rotary_dim=0), dict(rotary_dim=48),
                                dict(page_size=8), dict(page_size=48), dict(page_size=2048), dict(n_pages=0), dict(n_pages=1 << 31),
                                dict(rows=None), dict(rows=P + 8)])
def test_a_bad_cache_is_refused_everywhere(kw):
    c, h = _cache(**kw), _heads()
    want = om.EDTYPE if "dtype" in kw else om.EINVAL
    assert _write(c, h) == want and "latent_write" in om.last_error()
    assert _attend(c, h) == want and "latent_attention" in om.last_error()
    assert _expand(c, h) == want and "latent_expand" in om.last_error()
    assert _evict(c) == want and "latent_evict" in om.last_error()
    assert om.lib().ordermoe_latent_attention_workspace_size(ref(c), ref(h), 1, 1, 4, 0) == 0
    assert om.lib().ordermoe_latent_evict_workspace_size(ref(c), 1, 4, 10) == 0


@pytest.mark.parametrize("kw", [dict(n_q=0), dict(n_q=129), dict(head_dim=32), dict(head_dim=256), dict(w_k=None), dict(w_v=None),
                                dict(w_k=P + 2), dict(w_v=P + 8)])
def test_bad_heads_are_refused_everywhere(kw):
    c, h = _cache(), _heads(**kw)
    assert _write(c, h) == om.EINVAL and _attend(c, h) == om.EINVAL and _expand(c, h) == om.EINVAL
    assert _write(None, _heads()) == om.EINVAL and _write(c, None) == om.EINVAL
    assert _attend(None, _heads()) == om.EINVAL and _expand(c, None) == om.EINVAL and _evict(None) == om.EINVAL


@pytest.mark.parametrize("heads,args", [
    (dict(interleaved=2), {}), (dict(eps=-1.0), {}), (dict(eps=NAN), {}), (dict(eps=INF), {}), (dict(norm=P + 4), {}),
    (dict(cos_sin=P + 4), {}), (dict(max_pos=0), {}), ({}, dict(absorb=2)), ({}, dict(absorb=-1)), ({}, dict(T=-1)),
    ({}, dict(T=1 << 29)), ({}, dict(kv=0)), ({}, dict(kv=P + 8)), ({}, dict(q=P + 8)), ({}, dict(out=0)), ({}, dict(out=P + 2)),
    ({}, dict(slots=0)), ({}, dict(pos=0)), ({}, dict(qs=4 * 192 - 8)), ({}, dict(qs=4 * 192 + 4)), ({}, dict(kvs=568)),
    ({}, dict(kvs=580)),
])
def test_write_refusals(heads, args):
    assert _write(_cache(), _heads(**heads), **args) == om.EINVAL
    assert "latent_write" in om.last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), om.EINVAL), (dict(B=65536), om.EINVAL), (dict(max_q=0), om.EINVAL), (dict(max_q=65), om.EINVAL),
    (dict(T=-1), om.EINVAL), (dict(T=1 << 29), om.EINVAL), (dict(max_pages=0), om.EINVAL), (dict(max_pages=1 << 27), om.EINVAL),
    (dict(scale=NAN), om.EINVAL), (dict(scale=INF), om.EINVAL), (dict(decay=NAN), om.EINVAL), (dict(decay=-INF), om.EINVAL),
    (dict(q=0), om.EINVAL), (dict(q=P + 8), om.EINVAL), (dict(qs=0), om.EINVAL), (dict(ctx=0), om.EINVAL), (dict(table=0), om.EINVAL),
    (dict(out=0), om.EINVAL), (dict(out=P + 2), om.EINVAL), (dict(mass=P), om.EINVAL), (dict(mass_out=P), om.EINVAL),
    (dict(mass_out=P, stride=-3), om.EINVAL), (dict(mass_out=P, stride=1 << 41), om.EINVAL), (dict(ws=0), om.EWORKSPACE),
    (dict(ws_bytes=100), om.EWORKSPACE),
])
def test_attention_refusals(kw, code):
    assert _attend(_cache(), _heads(), **kw) == code
    assert "latent_attention" in om.last_error()


def test_attention_that_weighs_needs_room_for_its_scores():
    c, h = _cache(), _heads()
    size = lambda B, n, w: om.lib().ordermoe_latent_attention_workspace_size(ref(c), ref(h), B, n, 8, w)  # noqa: E731
    assert 0 < size(1, 1, 0) < size(8, 1, 0)
    assert size(8, 64, 1) >= size(8, 64, 0) + 8 * 64 * 4 * 8 * 16 * 4
    assert _attend(c, h, B=8, max_q=64, max_pages=8, ws_bytes=size(8, 64, 0), mass_out=P, stride=128) == om.EWORKSPACE
    # every sequence's rows at least once
    assert size(8, 64, 0) >= 8 * 64 * 4 * 512 * 4


def test_expand_refusals():
    for kw in (dict(n=-1), dict(n=1 << 29), dict(slots=0), dict(k=0), dict(r=0), dict(v=0), dict(k=P + 4), dict(r=P + 8), dict(v=P + 2)):
        assert _expand(_cache(), _heads(), **kw) == om.EINVAL, kw


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), om.EDTYPE), (dict(n_q=0), om.EINVAL), (dict(n_kv=0), om.EINVAL), (dict(n_q=9), om.EINVAL), (dict(n_q=1026), om.EINVAL),
    (dict(D=96), om.EINVAL), (dict(D=256), om.EINVAL), (dict(rot=16), om.EINVAL), (dict(rot=128), om.EINVAL), (dict(T=-1), om.EINVAL),
    (dict(T=1 << 28), om.EINVAL), (dict(L=-1), om.EINVAL), (dict(L=1 << 31), om.EINVAL), (dict(B=-1), om.EINVAL), (dict(B=65536), om.EINVAL),
    (dict(scale=NAN), om.EINVAL), (dict(q=0), om.EINVAL), (dict(q=P + 8), om.EINVAL), (dict(k=0), om.EINVAL), (dict(k=P + 4), om.EINVAL),
    (dict(v=0), om.EINVAL), (dict(r=0), om.EINVAL), (dict(out=0), om.EINVAL), (dict(out=P + 8), om.EINVAL), (dict(qs=0), om.EINVAL),
    (dict(ks=0), om.EINVAL),
])
def test_prompt_refusals(kw, code):
    assert _prompt(**kw) == code
    assert "prompt_attention" in om.last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), om.EINVAL), (dict(B=65536), om.EINVAL), (dict(max_pages=0), om.EINVAL), (dict(max_pages=1 << 27), om.EINVAL),
    (dict(keep=0), om.EINVAL), (dict(first=-1), om.EINVAL), (dict(recent=-1), om.EINVAL), (dict(first=5, recent=6), om.EINVAL),
    (dict(first=(1 << 31) - 1, recent=(1 << 31) - 1), om.EINVAL), (dict(stride=0), om.EINVAL), (dict(stride=1 << 41), om.EINVAL),
    (dict(ctx=0), om.EINVAL), (dict(seq=0), om.EINVAL), (dict(table=0), om.EINVAL), (dict(mass=0), om.EINVAL), (dict(pos=0), om.EINVAL),
    (dict(kept=0), om.EINVAL), (dict(len_out=0), om.EINVAL), (dict(mass_out=0), om.EINVAL), (dict(pos_out=0), om.EINVAL),
    (dict(ws=0), om.EWORKSPACE), (dict(ws_bytes=8), om.EWORKSPACE),
])
def test_evict_refusals(kw, code):
    assert _evict(_cache(), **kw) == code
    assert "latent_evict" in om.last_error()


def test_calls_of_nothing_are_fine():
    c, h = _cache(), _heads()
    assert _write(c, h, T=0, q=0, kv=0, pos=0, slots=0, out=0) == om.OK
    assert _attend(c, h, T=0, q=0) == om.OK and _attend(c, h, B=0, q=0) == om.OK
    assert _expand(c, h, n=0, slots=0, k=0, r=0, v=0) == om.OK
    assert _prompt(T=0, q=0) == om.OK and _prompt(B=0, q=0) == om.OK
    assert _evict(c, B=0, ctx=0) == om.OK
    assert om.last_error() == ""


def test_oracle_forms_agree():
    """Absorbed and expanded attention are the same function; eviction by hand."""
    rng = np.random.default_rng(3)
    n, ctx, h, D, R, rot = 3, 5, 2, 4, 6, 2
    rows, q = rng.normal(size=(ctx + n, R + rot)), rng.normal(size=(n, h, D + rot))
    wk, wv = rng.normal(size=(2, h, D, R))
    seen = ol.tree_seen(n, ctx, [(2 << i) - 1 for i in range(n)], ctx + n)
    qa, _ = ol.absorbed(q, wk, None, None, False)
    a = ol.latent_attention(qa, rows, seen, wv, 0.3)
    b = ol.prompt_attention(q, ol.expanded(rows[:, :R], wk)[0], ol.expanded(rows[:, :R], wv)[0], rows[:, R:], 0.3)
    np.testing.assert_allclose(a["out"], b["out"], rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(a["lse"], b["lse"], rtol=1e-12)
    np.testing.assert_allclose(a["mass"].sum(), n * h, rtol=1e-12)
    # nine tokens to five: place 0 and the last two are protected, then masses 9, 8 and the lower of the two 7s
    mass, pos = np.array([0, 7, 9, 1, 7, 8, 2, 0, np.nan]), np.arange(9)
    assert ol.evict(9, 9, 6, 1, 2, mass, pos).tolist() == [0, 1, 2, 7, 8, 5]
    assert ol.evict(4, 9, 6, 1, 2, mass, pos).tolist() == [0, 1, 2, 3, -1, -1]


@pytest.mark.parametrize("L", [(1 << 31) - 127, (1 << 31) - 64, (1 << 31) - 1])
def test_positions_up_to_two_tiles_below_32_bits(L):
    """The loop over tiles looks two of them ahead in 32 bits: so many positions have no room for that."""
    assert _prompt(L=L) == om.EINVAL and "prompt_attention" in om.last_error()
    assert _prompt(L=L, T=0, q=0) == om.EINVAL


def _grows(size, grid):
    """size over a grid of arguments: as large as at any arguments of which none is larger."""
    s = np.array([[[size(x, y, z) for z in grid[2]] for y in grid[1]] for x in grid[0]], np.int64)
    assert (s > 0).any()
    for axis in range(3):
        assert (np.diff(s, axis=axis) >= 0).all(), axis


@pytest.mark.parametrize("dtype", [om.BF16, om.F32])
@pytest.mark.parametrize("n_q,rank", [(1, 128), (3, 512), (16, 512), (40, 256), (128, 128)])
@pytest.mark.parametrize("weighs", [0, 1])
def test_attention_s_workspace_serves_every_smaller_call(dtype, n_q, rank, weighs):
    c, h = _cache(dtype=dtype, rank=rank, page_size=64), _heads(n_q=n_q)
    f = om.lib().ordermoe_latent_attention_workspace_size
    _grows(lambda B, n, pages: f(ref(c), ref(h), B, n, pages, weighs),
           ([1, 2, 3, 17, 64, 1000], list(range(1, 65)), [1, 2, 7, 40, 100, 3000, 1 << 20]))
    assert f(ref(c), ref(h), 5, 9, 100, 1) >= f(ref(c), ref(h), 5, 9, 100, 0)


@pytest.mark.parametrize("n_q,n_kv,D", [(1, 1, 128), (32, 8, 128), (16, 16, 64), (128, 1, 64), (128, 128, 128), (160, 160, 64), (1024, 16, 64)])
def test_prompts_workspace_serves_every_smaller_call(n_q, n_kv, D):
    f = om.lib().ordermoe_prompt_attention_workspace_size
    T = sorted({1, 2, 3, 5, 16, 31, 32, 33, 64, 100, 127, 128, 129, 130, 250, 257, 300, 512, 600, 1000, 2049, 4000, 8000, 100000})
    s = np.array([[f(om.BF16, n_q, n_kv, D, 0, t, B) for B in (1, 2, 3, 16, 100, 65535)] for t in [0] + T], np.int64)
    assert (np.diff(s, axis=0) >= 0).all() and (np.diff(s, axis=1) >= 0).all()
    assert s.max() <= 512 * 128 * (D + 2) * 4 + 512          # what 512 workgroups' rows take


def test_eviction_s_workspace_serves_every_smaller_call():
    c = _cache(page_size=64)
    f = om.lib().ordermoe_latent_evict_workspace_size
    _grows(lambda B, pages, keep: f(ref(c), B, pages, keep),
           ([1, 2, 9, 500], [1, 2, 50, 100, 127, 128, 129, 200, 5000],
            [1, 10, 64, 127, 129, 1000, 3199, 3200, 3201, 4000, 6000, 6399, 6400, 9000, 1 << 20, (1 << 31) - 1]))


@pytest.mark.parametrize("scale", [2.4e38, -3.4e38])
def test_scales_whose_scores_in_units_of_log_2_have_no_factor(scale):
    """scale * log2(e) is no finite number there: a score of 0 would be none either."""
    assert _attend(_cache(), _heads(), scale=scale) == om.EINVAL and "latent_attention" in om.last_error()
    assert _prompt(scale=scale) == om.EINVAL and "prompt_attention" in om.last_error()
