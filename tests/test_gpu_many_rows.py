"""Calls near the largest that the cache's entry points take: more than 2^32 threads, which no
launch has along one axis.  (The largest holds 138 GB of outputs; skipped where they do not fit.)"""
import numpy as np
import pytest

from oracle import attention as oa

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2607_17154_amd import ordermoe as om  # noqa: E402

THREADS = 1 << 32


@pytest.fixture(autouse=True)
def _memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def _room(gb):
    if torch.cuda.mem_get_info()[0] < gb * 1.1e9:
        pytest.skip("needs %d GB of free memory" % gb)


def _cache(n_kv, page, D, rng):
    """One page of int8 rows, and their values as fp32 [page, n_kv, D]."""
    parts, vals = [], []
    for _ in range(2):
        codes, scale = oa.quantise(rng.normal(size=(1, n_kv, page, D)).astype(np.float32), oa.INT8)
        parts.append([torch.from_numpy(codes).cuda(), torch.from_numpy(scale).cuda()])
        vals.append(torch.from_numpy(codes.view(np.int8)[0].astype(np.float32) * scale[0][..., None]).cuda().transpose(0, 1).contiguous())
    return om.make_cache(om.CACHE_INT8, parts[0][0], parts[1][0], parts[0][1], parts[1][1]), vals


def test_read():
    n_kv, D, page = 1024, 64, 16
    n = (1 << 19) + 16
    assert 2 * n * n_kv * 4 > THREADS                           # 16 lanes take four rows
    _room(140)
    cache, vals = _cache(n_kv, page, D, np.random.default_rng(0))
    slots = torch.arange(n, device="cuda") % page
    slots[-1] = -1
    ko, vo = (torch.empty((n, n_kv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    om.ordermoe_cache_read(cache, slots, ko, vo)
    for got, v in zip((ko, vo), vals):
        want = v.to(torch.bfloat16)
        assert (got[-1] == 0).all() and torch.equal(got[-page:-1], want[:-1])
        for part in got[:-page].view(-1, page, n_kv, D).split(1024):
            assert (part == want).all()


def test_write():
    D, page, base = 64, 16, 4096
    T = 87392 * base
    assert 3 * T * 4 > THREADS
    _room(100)
    rng = np.random.default_rng(1)
    rows = torch.from_numpy(rng.normal(size=(base, 1, D)).astype(np.float32)).cuda().to(torch.bfloat16)
    x = torch.empty((T, 1, D), dtype=torch.bfloat16, device="cuda")
    x.view(-1, base, 1, D)[:] = rows
    cache, _ = _cache(1, page, D, rng)
    slots = torch.full((T,), -1, dtype=torch.int64, device="cuda")
    at = torch.tensor([0, T // 2 + 5, T - 2, T - 1], device="cuda")
    slots[at] = torch.arange(4, device="cuda")
    q = torch.empty_like(x)
    om.ordermoe_cache_write(cache, om.make_heads(om.BF16, 1, D), x, x, x, None, slots, q)
    for part in q.view(-1, base, 1, D).split(1024):
        assert (part == rows).all()
    ko, vo = (torch.empty((4, 1, D), device="cuda") for _ in range(2))
    om.ordermoe_cache_read(cache, torch.arange(4, device="cuda"), ko, vo)
    codes, scale = oa.quantise(x[at].float().cpu().numpy(), oa.INT8)
    want = oa.code_values(oa.INT8).astype(np.float32)[codes] * scale[..., None]
    np.testing.assert_array_equal(ko.cpu().numpy(), want)
    np.testing.assert_array_equal(vo.cpu().numpy(), want)


def test_attention():
    """Tolerance: the output's and the weights' rounding to bf16, 2^-8 each of sum_p weight |v_p|, and 1e-4."""
    B, n_kv, D, page = 16400, 1024, 64, 16
    assert B * n_kv * 256 > THREADS
    _room(16)
    cache, (k, v) = _cache(n_kv, page, D, np.random.default_rng(2))
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    q = torch.randn((B, n_kv, D), generator=g, device="cuda").to(torch.bfloat16)
    ctx = torch.arange(B, dtype=torch.int32, device="cuda") % page
    start = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    table = torch.zeros((B, 1), dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    ws = torch.empty(om.ordermoe_draft_attention_workspace_size(cache, om.BF16, n_kv, B, 1), dtype=torch.uint8, device="cuda")
    om.ordermoe_draft_attention(cache, q, start, ctx, table, 1, D ** -0.5, out, ws)
    p = torch.arange(page, device="cuda")
    for i in range(0, B, 2050):
        s = (q[i:i + 2050, None].float() * k).sum(-1) * D ** -0.5                   # [n, page, n_kv]
        w = torch.softmax(s.masked_fill((p > ctx[i:i + 2050, None])[..., None], float("-inf")), 1)
        want, mag = ((w[..., None] * t).sum(1) for t in (v, v.abs()))
        assert ((out[i:i + 2050].float() - want).abs() <= (2.0 ** -7 + 1e-4) * mag).all()
        del s, w, want, mag
