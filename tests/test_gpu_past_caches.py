"""The variants that large calls take: the layer for a few tokens with weights read past the
caches, reads whose outputs are stored past them, writes of many rows of few bytes."""
import numpy as np
import pytest

import workloads as wl

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2607_17154_amd import ordermoe as om  # noqa: E402

from ._pipeline import DeviceLayer, build_case, host, library_tables  # noqa: E402
from .test_gpu_cache_attention import CODE, DT, _Cache, _dev  # noqa: E402
from .test_gpu_few_moe import _check_route, _check_y, _few  # noqa: E402

MIB = 1 << 20


@pytest.mark.parametrize("k,M,n_shared", [(6, 8, 2), (2, 4, 0)])
def test_layer_of_64_mib_of_gate_and_up_weights(k, M, n_shared):
    """(Tolerances: those of the smaller layers, which do not depend on the size.)"""
    cfg = wl.C4.with_(T=16, d=2048, f=1024, T_cal=2048, k=k, M=M, capacity=wl._cap(M, 64 // M), n_shared=n_shared)
    case = build_case(cfg)
    dl = DeviceLayer(case, library_tables(case))
    assert dl.w_gu.numel() * 2 >= 64 * MIB
    for T in (16, 3, 1):
        case.X, case.loc, case.qhat = case.X[:T], case.loc[:T], case.qhat[:T]
        x, loc, qh = dl.inputs()
        out, y = _few(dl, x, loc, qh, T)
        _check_route(dl, out, dl.route(x, loc, qh, T), T)
        _check_y(case, out, y, T, cfg.m0)
        _, again = _few(dl, x, loc, qh, T)
        np.testing.assert_array_equal(host(again), host(y))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("hkv,D,page", [(8, 64, 16), (3, 128, 64), (2, 256, 32)])
def test_reads_of_64_mib_and_of_parts_of_it(dtype, fmt, hkv, D, page):
    size = 2 if dtype == "bf16" else 4
    n = 66 * MIB // (2 * hkv * D * size) + 5
    rng = np.random.default_rng(D + hkv)
    ca = _Cache(fmt, 40, hkv, page, D)
    ca.fill(np.arange(40 * page), rng)
    at = _dev(rng.integers(-3, 40 * page + 3, n))
    whole, parts = (([torch.full((n, hkv, D), 7.0, dtype=DT[dtype], device="cuda") for _ in range(2)]) for _ in range(2))
    om.ordermoe_cache_read(ca.c, at, *whole)
    for i in range(0, n, 1000):
        om.ordermoe_cache_read(ca.c, at[i:i + 1000], *(t[i:i + 1000] for t in parts))
    for a, b in zip(whole, parts):
        assert torch.equal(a, b)
    # and some rows against the values themselves
    some = rng.integers(0, n, 200)
    slots = host(at)[some]
    inside = (slots >= 0) & (slots < 40 * page)
    for got, want in zip(whole, ca.rows(np.where(inside, slots, 0))):
        want = torch.from_numpy((want * inside[:, None, None]).astype(np.float32)).to(DT[dtype])
        np.testing.assert_array_equal(host(got[torch.from_numpy(some).cuda()]), host(want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("hq,hkv,D", [(1, 1, 64), (2, 1, 128), (4, 2, 64)])
def test_writes_of_many_rows_of_few_bytes(dtype, fmt, hq, hkv, D):
    """65536 head rows and more, with queries below 32 MiB: the same bits as in parts of fewer."""
    heads = hq + 2 * hkv
    T = 65536 // heads + 77
    assert T * heads >= 65536 and T * hq * D * 4 < 32 * MIB
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    q, k, v = torch.randn((T, heads, D), generator=g, device="cuda").to(DT[dtype]).split([hq, hkv, hkv], 1)
    page, pages = 32, -(-T // 32)
    w = [(1 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(DT[dtype]) for _ in range(2)]
    h = om.make_heads(CODE[dtype], hq, D, *w, _dev(om.rotary_table(T, D // 2)), 1)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:T]
    res = []
    for step in (T, 301):
        ca, out = _Cache(fmt, pages, hkv, page, D), torch.empty((T, hq, D), dtype=DT[dtype], device="cuda")
        for i in range(0, T, step):
            c = slice(i, i + step)
            om.ordermoe_cache_write(ca.c, h, q[c], k[c], v[c], pos[c], slots[c], out[c])
        res.append([out] + ca.codes + [s.nan_to_num(-1.0) for s in ca.scale])
    for a, b in zip(*res):
        assert torch.equal(a, b)
