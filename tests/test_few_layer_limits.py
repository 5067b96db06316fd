"""A router whose weights span 2^31 bytes is refused by the layer for a few tokens, which
addresses them with 31 bits (no GPU: refused before any device work)."""
import ctypes

import pytest

from paper_2607_17154_amd import ordermoe as om

from .test_decode_host import _few, _few_structs


@pytest.mark.parametrize("d,fits", [(1 << 21, False), ((1 << 21) - 64, True), (1 << 22, False)])
def test_router_weights_span_31_bits(d, fits):
    L, E, out = _few_structs(dict(dtype=om.F32, d=d, E=256), dict(dtype=om.F32, d=d, E=256, f=32))
    size = om.lib().ordermoe_few_workspace_size(ctypes.byref(L), ctypes.byref(E), 4)
    assert (size > 0) == fits
    assert _few(L, E, out, ws_bytes=64) == (om.EWORKSPACE if fits else om.EINVAL)
    assert "few_moe_layer" in om.last_error()
