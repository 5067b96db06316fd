"""Heads made for one size used with a cache of another: refused before any pointer is
handed on (the norm weights have as many elements as the size they were made for)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2607_17154_amd import ordermoe as om  # noqa: E402


class _OnDevice(torch.Tensor):
    is_cuda = True


def test_heads_of_another_size_are_refused():
    P = 1 << 20
    cache = om.Cache(format=om.CACHE_INT8, n_kv=1, head_dim=128, page_size=16, n_pages=1, k_codes=P, v_codes=P, k_scale=P, v_scale=P)
    dev = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt).as_subclass(_OnDevice)  # noqa: E731
    w = dev(64)
    heads = om.make_heads(om.F32, 1, 64, w, w)
    rows = dev(0, 1, 128)                                       # no tokens: nothing is launched
    call = lambda h: om.ordermoe_cache_write(cache, h, rows, rows, rows, None, dev(0, dt=torch.int64), dev(0, 1, 128), 1)  # noqa: E731
    with pytest.raises(ValueError, match="heads of 64, the cache of 128"):
        call(heads)
    call(om.make_heads(om.F32, 1, 128, dev(128), dev(128)))
    # a struct filled in by hand has no size of its own
    call(om.Heads(dtype=om.F32, n_q=1))
