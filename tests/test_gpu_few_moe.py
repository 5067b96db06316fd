"""The whole layer for a few tokens (ordermoe_few_moe_layer) through the C ABI.

Routing outputs: those of ordermoe_route_select, bit for bit in bf16 (the same
partial sums in the same order), on unflagged tokens in fp32; they are themselves
checked against the oracle elsewhere.  Layer output, from these decisions in fp64:
  bf16: the weighted activation is rounded to bf16 (2^-8 of it) and the output too
    (2^-8): 2^-8 of sum |W_down| |w act| and of |y|, a fifth more for the fp32 sums and the
    hardware's exp and reciprocal, and 1e-6;
  fp32: 1e-4 of the token's largest output (the layer's own bar)."""
import numpy as np
import pytest

import workloads as wl

from ._pipeline import DeviceLayer, build_case, host, library_tables, oracle_decisions
from ._random_layers import N_RANDOM, qhat_scale, random_layer

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2607_17154_amd import ordermoe as om  # noqa: E402

PER_TOKEN = ("idx", "w", "margin", "flag", "exec_k", "exec_m", "cls", "qhat_out", "loc_out")


def _few(dl, x, loc, qh, T, stream=None, out=None, ws=None, y=None, server=None):
    cfg = dl.cfg
    out = out or om.alloc_route_out(T, cfg.k, cfg.M, "cuda")
    need = om.ordermoe_few_workspace_size(dl.layer, dl.experts, T)
    assert need > 0
    if ws is None:
        ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")     # NaNs and large counts
    if y is None:
        y = torch.full((T, cfg.d), 7.0, dtype=x.dtype, device="cuda")
    om.ordermoe_few_moe_layer(dl.layer, dl.experts, x, T, loc, qh, cfg.m0 if server is None else server, out, y, ws, stream=stream)
    return out, y


def _expected(case, out, T, server):
    """y and the size of its terms (fp64) from the device's decisions."""
    cfg = case.cfg
    ek, em, w = (host(out[n]) for n in ("exec_k", "exec_m", "w"))
    y, mag = np.zeros((T, cfg.d)), np.zeros((T, cfg.d))

    def add(t, weights, gate):
        Wg, Wu, Wd = (np.asarray(m, np.float64) for m in weights)
        g, u = Wg @ case.X[t].astype(np.float64), Wu @ case.X[t].astype(np.float64)
        a = gate * g / (1 + np.exp(-g)) * u
        y[t] += Wd @ a
        mag[t] += np.abs(Wd) @ np.abs(a)

    for t in range(T):
        for s in range(cfg.k):
            if em[t, s] == server:
                add(t, case.expert(int(ek[t, s])), float(w[t, s]))
        if case.loc[t] == server:
            for sh in case.shared():
                add(t, sh, 1.0)
    return y, mag


def _check_y(case, out, y, T, server):
    want, mag = _expected(case, out, T, server)
    got = host(y).astype(np.float64)
    if case.cfg.dtype == "bf16":
        tol = 1.2 * 2.0 ** -8 * mag + 2.0 ** -8 * np.abs(want) + 1e-6
    else:
        tol = 1e-4 * np.abs(want).max(1, keepdims=True)
    over = np.abs(got - want) - tol
    assert (over <= 0).all(), over.max()
    empty = (mag == 0).all(1)
    assert (got[empty] == 0).all()


def _check_route(dl, out, ref, T, exact=True, ok=None):
    cfg = dl.cfg
    ok = np.ones(T, bool) if ok is None else ok
    for n in PER_TOKEN:
        a, b = host(out[n]), host(ref[n])
        if exact:
            np.testing.assert_array_equal(a, b, err_msg=n)
        elif a.dtype.kind == "f":
            np.testing.assert_allclose(a[ok], b[ok], rtol=1e-5, atol=1e-6, err_msg=n)
        else:
            np.testing.assert_array_equal(a[ok], b[ok], err_msg=n)
    if exact or ok.all():
        for n in ("dst_count", "counters"):
            np.testing.assert_array_equal(host(out[n]), host(ref[n]), err_msg=n)
        n_remote = int(host(ref["counters"])[om.CNT_REMOTE_SLOTS])
        np.testing.assert_array_equal(host(out["dispatch"])[:n_remote], host(ref["dispatch"])[:n_remote])
        assert (host(out["dispatch"])[n_remote:T * cfg.k] == -1).all()


TS = (1, 2, 3, 5, 8, 13, 16)


@pytest.mark.parametrize("i", range(N_RANDOM))
def test_random_layers(i):
    T = TS[i % len(TS)]
    cfg = random_layer(i).with_(T=T)
    print("few: %s T=%d n_shared=%d m0=%d" % (cfg.name, T, cfg.n_shared, cfg.m0), flush=True)
    case = build_case(cfg, qhat_scale=qhat_scale(i))
    dl = DeviceLayer(case, library_tables(case))
    x, loc, qh = dl.inputs()
    out, y = _few(dl, x, loc, qh, T)
    ref = dl.route(x, loc, qh, T)
    torch.cuda.synchronize()
    bf = cfg.dtype == "bf16"
    _check_route(dl, out, ref, T, exact=bf, ok=host(ref["margin"]) >= 1e-4)
    _check_y(case, out, y, T, cfg.m0)
    # the same bits again
    out2, y2 = _few(dl, x, loc, qh, T)
    np.testing.assert_array_equal(host(y2), host(y))


@pytest.mark.parametrize("cfg", [wl.C1, wl.C3.with_(d=512, f=256, T_cal=2048), wl.C4.with_(d=512, f=256, T_cal=2048),
                                 wl.C2.with_(d=512, f=2048, T_cal=2048)], ids=["C1", "C3", "C4", "C2"])
@pytest.mark.parametrize("T", [1, 4, 16])
def test_workload_shapes_agree_with_the_oracle(cfg, T):
    case = build_case(cfg.with_(T=T))
    dl = DeviceLayer(case, library_tables(case))
    x, loc, qh = dl.inputs()
    out, y = _few(dl, x, loc, qh, T)
    dec = oracle_decisions(case)
    ok = (dec["margin"] >= 1e-4) & (host(out["margin"]) >= 1e-4)
    for n in ("idx", "exec_k", "exec_m", "cls"):
        np.testing.assert_array_equal(host(out[n])[ok], dec[n][ok], err_msg=n)
    _check_y(case, out, y, T, cfg.m0)


def _layer(T=16, **kw):
    cfg = wl.C4.with_(T=T, d=256, f=128, T_cal=2048, **kw)
    case = build_case(cfg)
    return case, DeviceLayer(case, library_tables(case))


def test_no_tokens():
    case, dl = _layer()
    out = om.alloc_route_out(1, dl.cfg.k, dl.cfg.M, "cuda")
    for v in out.values():
        v.fill_(9)
    x, loc, qh = dl.inputs()
    _few(dl, x, loc, qh, 0, out=out)
    torch.cuda.synchronize()
    assert (host(out["counters"]) == 0).all() and (host(out["dst_count"]) == 0).all()
    assert (host(out["idx"]) == 9).all() and (host(out["dispatch"]) == 9).all()


def test_tokens_off_the_servers_and_servers_without_rows():
    case, dl = _layer()
    loc = np.zeros(16, np.uint8)
    loc[[2, 5]] = 200, dl.cfg.M
    case.loc = loc
    x, l, qh = dl.inputs()
    out, y = _few(dl, x, l, qh, 16)
    ref = dl.route(x, l, qh, 16)
    _check_route(dl, out, ref, 16)
    assert int(host(out["counters"])[om.CNT_INVALID]) == 2 and (host(out["exec_k"])[[2, 5]] == -1).all()
    _check_y(case, out, y, 16, 0)
    assert (host(y)[[2, 5]] == 0).all()
    # a server that no slot runs on: zeros everywhere
    out, y = _few(dl, x, l, qh, 16, server=31)
    assert (host(y) == 0).all()


def test_a_server_without_routed_experts():
    case, dl = _layer(n_shared=2)
    dl.experts = om.make_experts(dl.code, dl.cfg.d, dl.cfg.f, dl.cfg.E, [], None, None, 2, dl.w_sh_gu, dl.w_sh_dn)
    x, loc, qh = dl.inputs()
    out, y = _few(dl, x, loc, qh, 16)
    ref = dl.route(x, loc, qh, 16)
    _check_route(dl, out, ref, 16)
    for n in ("exec_k", "exec_m"):
        out[n].fill_(255 if n == "exec_m" else -1)              # only the shared experts run here
    _check_y(case, out, y, 16, 0)


def test_a_token_that_is_no_number_leaves_the_others_alone():
    case, dl = _layer(n_shared=1)
    x, loc, qh = dl.inputs()
    x[3, 7] = float("nan")
    x[9, 1] = float("inf")
    out, y = _few(dl, x, loc, qh, 16)
    torch.cuda.synchronize()
    want, mag = _expected(case, out, 16, 0)
    keep = np.setdiff1d(np.arange(16), [3, 9])
    tol = 1.2 * 2.0 ** -8 * mag + 2.0 ** -8 * np.abs(want) + 1e-6
    assert (np.abs(host(y) - want) <= tol)[keep].all()
    assert np.isnan(host(y)[3]).all()


@pytest.mark.parametrize("k,M,allow_sub,renorm", [(8, 8, 1, 1), (3, 8, 2, 0), (8, 16, 1, 1), (1, 2, 0, 0)])
def test_tables_at_any_address(k, M, allow_sub, renorm):
    """Tables that 16-byte reads cannot take, and costs too large to be kept on the chip
    (16 servers x 16 x 64 experts), give the decisions of the routing."""
    case, dl = _layer(k=k, M=M, capacity=wl._cap(M, max(8, 64 // M)), allow_sub=allow_sub, renorm=renorm)
    x, loc, qh = dl.inputs()
    cfg = dl.cfg
    ref = dl.route(x, loc, qh, 16)
    first, y = _few(dl, x, loc, qh, 16)
    _check_route(dl, first, ref, 16)
    moved = {}
    for n, v in dl.tabs_dev.items():
        room = torch.empty(v.numel() + 1, dtype=v.dtype, device="cuda")
        room[1:] = v.reshape(-1)
        moved[n] = room[1:]
        assert moved[n].data_ptr() % 16 == 4
    dl.layer = om.make_layer(dl.code, cfg.d, cfg.E, cfg.k, cfg.M, 15, dl.w_router, moved, dl.Qbar, cfg.omega_Q, cfg.pin_local_exact,
                             cfg.allow_sub, cfg.renorm)
    out, y2 = _few(dl, x, loc, qh, 16)
    _check_route(dl, out, ref, 16)
    np.testing.assert_array_equal(host(y2), host(y))


def test_two_streams_and_shared_weights():
    case, dl = _layer(n_shared=2)
    x, loc, qh = dl.inputs()
    xs = [x, x.flip(0).contiguous()]
    want = [_few(dl, v, loc, qh, 16) for v in xs]
    torch.cuda.synchronize()
    need = om.ordermoe_few_workspace_size(dl.layer, dl.experts, 16)
    bufs = [(om.alloc_route_out(16, dl.cfg.k, dl.cfg.M, "cuda"), torch.empty(need, dtype=torch.uint8, device="cuda"),
             torch.zeros_like(x)) for _ in xs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for v, (o, ws, y), s in zip(xs, bufs, streams):
            _few(dl, v, loc, qh, 16, stream=s, out=o, ws=ws, y=y)
    torch.cuda.synchronize()
    for (o, _, y), (wo, wy) in zip(bufs, want):
        np.testing.assert_array_equal(host(y), host(wy))
        for n in PER_TOKEN:
            np.testing.assert_array_equal(host(o[n]), host(wo[n]), err_msg=n)


def test_captured_layer_follows_its_tokens():
    case, dl = _layer(n_shared=1)
    x, loc, qh = dl.inputs()
    need = om.ordermoe_few_workspace_size(dl.layer, dl.experts, 16)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out, y = om.alloc_route_out(16, dl.cfg.k, dl.cfg.M, "cuda"), torch.zeros_like(x)
    _few(dl, x, loc, qh, 16, out=out, ws=ws, y=y)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _few(dl, x, loc, qh, 16, out=out, ws=ws, y=y)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    for _ in range(4):
        x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        g.replay()
        torch.cuda.synchronize()
        got = {n: host(out[n]).copy() for n in PER_TOKEN + ("counters",)}, host(y).copy()
        o2, y2 = _few(dl, x, loc, qh, 16)
        torch.cuda.synchronize()
        np.testing.assert_array_equal(got[1], host(y2))
        for n in got[0]:
            np.testing.assert_array_equal(got[0][n], host(o2[n]), err_msg=n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_workgroups_than_the_chip_holds(dtype):
    """Six calls of 256 workgroups at once, one of which fills a compute unit: some
    start when others of their call have long begun to wait."""
    cfg = wl.C4.with_(T=16, d=1024, f=512, T_cal=2048, n_shared=1, dtype=dtype)
    case = build_case(cfg)
    dl = DeviceLayer(case, library_tables(case))
    x, loc, qh = dl.inputs()
    xs = [x.roll(i, 0).contiguous() for i in range(6)]
    want = [_few(dl, v, loc, qh, 16) for v in xs]
    need = om.ordermoe_few_workspace_size(dl.layer, dl.experts, 16)
    bufs = [(om.alloc_route_out(16, cfg.k, cfg.M, "cuda"), torch.empty(need, dtype=torch.uint8, device="cuda"),
             torch.zeros_like(x)) for _ in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for _ in range(8):
        for v, (o, ws, y), s in zip(xs, bufs, streams):
            _few(dl, v, loc, qh, 16, stream=s, out=o, ws=ws, y=y)
    torch.cuda.synchronize()
    for (o, _, y), (wo, wy) in zip(bufs, want):
        np.testing.assert_array_equal(host(y), host(wy))
        for n in PER_TOKEN:
            np.testing.assert_array_equal(host(o[n]), host(wo[n]), err_msg=n)
    _check_y(case, want[0][0], want[0][1], 16, cfg.m0)
