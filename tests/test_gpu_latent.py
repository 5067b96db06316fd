"""The latent cache's operators, the prompts' attention and the eviction against the
oracle, through the C ABI.

Tolerances, fixed beforehand (u = 2^-24, an fp32 rounding; a bf16 rounding is at most 2^-8 of the value):
  a sum of n products: n + 1 roundings relative to the sum of the products' magnitudes;
  rows: a norm is a scaling, 40 u of the value (its sum of squares: 8 additions in a chain and 6 in a
    tree; a square root, two divisions, two products); a turned element 4 u of |a| + |b|;
  a score: (width + 4) u of its products' magnitudes, e; a softmax weight then 2 e, and 8 u for exp2 and
    the changes of its reference, relative; its sum over n places n u;
  outputs: sum_p weight |v_p| times the weights' error, 2^-8 more where they are rounded to bf16 (2^-16
    in two parts); what goes through W_v likewise, 2^-16 for its operand in two parts; then the output's rounding;
  lse: e, 8 u, n u, and 2 u of its size;  mass: the weights' error and rows * u, relative, and 4 u."""
import numpy as np
import pytest

from oracle import latent as ol

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2607_17154_amd import ordermoe as om  # noqa: E402

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": 0.0}        # the output's rounding (fp32: among the sums' roundings)


def _dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _host(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _weights(rng, h, D, R, dtype):
    return [_dev(rng.normal(size=(h, D, R)) * R ** -0.5, DT[dtype]) for _ in range(2)]


def _within(got, want, tol, what):
    with np.errstate(invalid="ignore"):
        bad = ~(np.abs(got - want) <= tol)
    bad &= ~((got == want) | (np.isnan(got) & np.isnan(want)))
    assert not bad.any(), "%s: %d of %d off, worst %.3g of its tolerance" % (
        what, bad.sum(), bad.size, np.nanmax((np.abs(got - want) / np.maximum(tol, 1e-300))[bad]))


# ------------------------------------------------------------------ write
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,h,D,R,rot,absorb,inter,norm,packed", [
    (1, 1, 64, 128, 32, 1, 0, 1, 0), (7, 5, 128, 512, 64, 1, 1, 1, 1), (65, 2, 64, 256, 64, 1, 0, 0, 1), (130, 4, 128, 128, 32, 1, 1, 1, 0),
    (1, 3, 128, 512, 64, 0, 1, 1, 1), (33, 8, 64, 256, 32, 0, 0, 1, 0), (200, 1, 128, 512, 32, 0, 1, 0, 1), (17, 128, 64, 128, 64, 0, 0, 1, 0),
])
def test_rows_and_queries(dtype, T, h, D, R, rot, absorb, inter, norm, packed):
    rng = np.random.default_rng(T + D + R)
    max_pos, page = 5000, 16
    x = rng.normal(size=(T, h * (D + rot) + R + rot)) * np.exp(rng.normal(size=(T, 1)))
    x = _dev(x, DT[dtype])
    q, kv = x[:, :h * (D + rot)].unflatten(1, (h, D + rot)), x[:, h * (D + rot):]
    if not packed:
        q, kv = q.contiguous(), kv.contiguous()
    n_pages = -(-T // page) + 2
    rows = torch.full((n_pages, page, R + rot), 7.0, dtype=DT[dtype], device="cuda")
    cache = om.make_latent_cache(rows, R)
    table = om.rotary_table(max_pos, rot)
    w = _dev(1 + 0.2 * rng.normal(size=R), DT[dtype]) if norm else None
    wk, wv = _weights(rng, h, D, R, dtype)
    heads = om.make_latent_heads(cache, wk, wv, w, _dev(table), inter, 1e-5)
    pos = rng.integers(0, max_pos, T).astype(np.int32)
    pos[0] = max_pos - 1
    slots = rng.permutation(n_pages * page)[:T].astype(np.int64)
    out = torch.empty((T, h, (R if absorb else D) + rot), dtype=DT[dtype], device="cuda")
    om.ordermoe_latent_write(cache, heads, q, kv, _dev(pos), _dev(slots), out, absorb)
    hq, hkv = _host(q), _host(kv)
    want = ol.token_rows(hkv, R, None if w is None else _host(w), 1e-5, table, pos, bool(inter))
    got = _host(rows.flatten(0, 1))
    pair = np.abs(hkv[:, R:]).max(-1, keepdims=True) * 2
    tol = np.concatenate([40 * U * np.abs(want[:, :R]), 4 * U * np.broadcast_to(pair, (T, rot))], 1)
    _within(got[slots], want, tol + HALF[dtype] * np.abs(want), "rows")
    left = np.ones(n_pages * page, bool)
    left[slots] = False
    assert (got[left] == 7).all()
    pair = np.abs(hq[..., D:]).max(-1, keepdims=True) * 2
    turned = 4 * U * np.broadcast_to(pair, (T, h, rot))
    if absorb:
        want, size = ol.absorbed(hq, _host(wk), table, pos, bool(inter))
        tol = np.concatenate([(D + 1) * U * size[..., :R], turned], 2)
    else:
        one = np.broadcast_to(np.eye(D), (h, D, D))
        want, _ = ol.absorbed(hq, one, table, pos, bool(inter))
        tol = np.concatenate([np.zeros((T, h, D)), turned], 2)
        np.testing.assert_array_equal(_host(out)[..., :D], hq[..., :D])
    _within(_host(out), want, tol + HALF[dtype] * np.abs(want), "queries")


def test_rows_without_a_slot_a_position_a_rotation_or_queries():
    T, h, D, R, rot, page = 6, 2, 64, 128, 32, 16
    rng = np.random.default_rng(1)
    q, kv = _dev(rng.normal(size=(T, h, D + rot)), torch.float32), _dev(rng.normal(size=(T, R + rot)), torch.float32)
    wk, wv = _weights(rng, h, D, R, "f32")
    slots = np.array([-1, 16, 2, 3, 1 << 50, 5], np.int64)
    pos = np.array([0, 1, -1, 9, 3, 10], np.int32)
    new = lambda: torch.full((1, page, R + rot), 7.0, device="cuda")  # noqa: E731
    rows = new()
    cache = om.make_latent_cache(rows, R)
    heads = om.make_latent_heads(cache, wk, wv, None, _dev(om.rotary_table(10, rot)))
    out = torch.empty((T, h, D + rot), device="cuda")
    om.ordermoe_latent_write(cache, heads, q, kv, _dev(pos), _dev(slots), out, 0)
    got, o = _host(rows)[0], _host(out)
    assert (np.delete(got, [2, 3, 5], 0) == 7).all() and np.isfinite(got[3]).all()
    for s, t in ((2, 2), (5, 5)):                            # positions -1 and 10 of 10
        np.testing.assert_array_equal(got[s, :R], _host(kv)[t, :R])
        assert np.isnan(got[s, R:]).all() and np.isnan(o[t, :, D:]).all() and np.isfinite(o[t, :, :D]).all()
    # no table: nothing is turned; no queries: rows only
    rows = new()
    cache = om.make_latent_cache(rows, R)
    om.ordermoe_latent_write(cache, om.make_latent_heads(cache, wk, wv), None, kv, None, _dev(slots), None, 1)
    np.testing.assert_array_equal(_host(rows)[0, [2, 3, 5]], _host(kv)[[2, 3, 5]])


# ------------------------------------------------------------------ expand
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,h,D,R,rot,page", [(1, 1, 64, 128, 32, 16), (63, 3, 64, 256, 64, 32), (130, 2, 128, 512, 32, 16), (300, 40, 128, 128, 64, 16),
                                              (4200, 1, 64, 128, 32, 64), (8200, 8, 64, 128, 32, 1024), (1100, 127, 64, 128, 32, 64), (4400, 30, 128, 512, 64, 64),
                                              (16500, 8, 64, 256, 64, 16)])
def test_expanded_rows(dtype, n, h, D, R, rot, page):
    rng = np.random.default_rng(n)
    n_pages = max(2, -(-n // page) // 2)
    rows = _dev(rng.normal(size=(n_pages, page, R + rot)), DT[dtype])
    cache = om.make_latent_cache(rows, R)
    wk, wv = _weights(rng, h, D, R, dtype)
    slots = rng.integers(0, n_pages * page, n).astype(np.int64)
    if n > 2:
        slots[[1, n // 2, n - 1]] = -1, n_pages * page, -(1 << 40)
        rows[0, 0, 0] = float("nan")                         # read in their place, and left out
        slots[slots == 0] = 1
    k, v = (torch.full((n, h, D), 7.0, dtype=DT[dtype], device="cuda") for _ in range(2))
    r = torch.full((n, rot), 7.0, dtype=DT[dtype], device="cuda")
    om.ordermoe_latent_expand(cache, om.make_latent_heads(cache, wk, wv), _dev(slots), k, r, v)
    inside = (slots >= 0) & (slots < n_pages * page)
    x = np.zeros((n, R + rot))
    x[inside] = _host(rows.flatten(0, 1))[slots[inside]]
    np.testing.assert_array_equal(_host(r), x[:, R:])
    some = np.unique(np.concatenate([np.arange(min(n, 200)), np.arange(max(0, n - 200), n)]))
    for got, w in ((k, wk), (v, wv)):
        want, size = ol.expanded(x[some, :R], _host(w))
        _within(_host(got)[some], want, (R + 1) * U * size + HALF[dtype] * np.abs(want), "values")


# ------------------------------------------------------------------ attention
class _Batch:
    """Ragged sequences in a paged latent cache whose other memory is NaN."""

    def __init__(self, rng, dtype, ctx, n, h, D, R, rot, page, spread=1.0):
        self.dtype, self.ctx, self.n, self.page, self.R = dtype, np.asarray(ctx), np.asarray(n), page, R
        L = self.ctx + self.n
        pages = -(-L // page)
        total = int(pages.sum()) + 1
        order = rng.permutation(total).astype(np.int32)
        self.table = np.full((len(L), max(1, int(pages.max()))), -1, np.int32)
        at = 0
        for b in range(len(L)):
            self.table[b, :pages[b]] = order[at:at + pages[b]]
            at += pages[b]
        self.rows = torch.full((total, page, R + rot), float("nan"), dtype=DT[dtype], device="cuda")
        for b in range(len(L)):
            p = np.arange(L[b])
            self.rows[_dev(self.table[b, p // page].astype(np.int64)), _dev(p % page)] = _dev(rng.normal(size=(L[b], R + rot)), DT[dtype])
        self.cache = om.make_latent_cache(self.rows, R)
        self.wk, self.wv = _weights(rng, h, D, R, dtype)
        self.heads = om.make_latent_heads(self.cache, self.wk, self.wv)
        self.T = int(self.n.sum()) + 2                       # two tokens behind the last sequence
        self.q = _dev(rng.normal(size=(self.T, h, R + rot)) * spread * 2 * (D + rot) ** 0.5 / (R + rot) ** 0.5, DT[dtype])
        self.start = np.concatenate([[0], np.cumsum(self.n)]).astype(np.int32)
        self.scale = (D + rot) ** -0.5
        self.h, self.D = h, D

    def cached(self, b, length):
        p = np.arange(length)
        return _host(self.rows[_dev(self.table[b, p // self.page].astype(np.int64)), _dev(p % self.page)])

    def run(self, max_q, tree=None, mass=None, decay=1.0, fill=7.0, stride=None, ws=None, stream=None):
        B, d = len(self.n), DT[self.dtype]
        out = torch.full((self.T, self.h, self.D), fill, dtype=d, device="cuda")
        lse = torch.full((self.T, self.h), fill, device="cuda")
        mo = None if stride is None else torch.full((B, stride), fill, device="cuda")
        if ws is None:
            size = om.ordermoe_latent_attention_workspace_size(self.cache, self.heads, B, max_q, self.table.shape[1], int(mo is not None))
            ws = torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda")
        om.ordermoe_latent_attention(self.cache, self.heads, self.q, _dev(self.start), _dev(self.ctx.astype(np.int32)), _dev(self.table),
                                     max_q, self.scale, out, ws, tree=tree, lse=lse, mass=mass, mass_out=mo, decay=decay)
        return out, lse, mo

    def check(self, got, max_q, words=None, mass=None, decay=1.0):
        out, lse, mo = got
        o, ls = _host(out), _host(lse)
        width = self.rows.shape[2]
        fine = self.dtype == "bf16" and max_q * self.h <= 32
        written = np.zeros(self.T, bool)
        for b in range(len(self.n)):
            n, s0 = min(int(self.n[b]), max_q), self.start[b]
            L = int(self.ctx[b]) + n
            w = [(2 << i) - 1 for i in range(n)] if words is None else words[s0:s0 + n]
            e = ol.latent_attention(_host(self.q)[s0:s0 + n], self.cached(b, L), ol.tree_seen(n, int(self.ctx[b]), w, L), _host(self.wv), self.scale)
            t = np.arange(s0, s0 + n)
            written[t] = True
            es = e["score"] * (width + 4) * U
            ew = 2 * es + (8 + L) * U + (0 if self.dtype == "f32" else 2.0 ** -16 if fine else 2.0 ** -8)
            tol = ew * e["size"] + (2.0 ** -16 + (self.R + 1) * U) * e["through"] + HALF[self.dtype] * np.abs(e["out"])
            _within(o[t], e["out"], tol, "out of sequence %d" % b)
            if n:
                with np.errstate(invalid="ignore"):
                    _within(ls[t], e["lse"], es + (8 + L) * U + 2 * U * np.abs(np.where(np.isfinite(e["lse"]), e["lse"], 0)), "lse of %d" % b)
            if mo is not None:
                m, want = _host(mo)[b], e["mass"].copy()
                k = min(L, mo.shape[1]) if n else 0
                add = np.zeros(L)
                if mass is not None:
                    c = min(int(self.ctx[b]), mass.shape[1])
                    add[:c] = decay * _host(mass)[b][:c]
                want = want + add
                # (exp2 has no results below fp32's smallest normal number, 2^-126: a weight under it counts as 0)
                tol = (2 * es + (8 + L + n * self.h) * U) * e["mass"] + 4 * U * np.abs(want) + n * self.h * 2.0 ** -126
                _within(m[:k], want[:k], tol[:k], "mass of %d" % b)
                assert (m[k:] == 7).all()
        assert (o[~written] == 7).all() and (ls[~written] == 7).all()


def _trees(rng, n):
    """Words of trees; some places are padded and see the context alone."""
    words = []
    for c in n:
        w = []
        for i in range(c):
            up = int(rng.integers(0, i + 1))
            w.append((w[up - 1] if up else 0) | 1 << i)
        if c > 4:
            w[int(rng.integers(1, c))] = 0
        words += w
    return words


def _tree_tensor(words, T):
    w = np.zeros(T, np.uint64)
    w[:len(words)] = words
    return _dev(w.view(np.int64))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h,D,R,rot,page,max_q,tree,weighs", [
    (1, 64, 128, 32, 16, 1, 0, 1), (16, 128, 512, 64, 64, 1, 0, 0), (5, 128, 512, 64, 16, 3, 1, 1), (8, 64, 512, 32, 32, 5, 1, 0),
    (32, 128, 512, 64, 16, 2, 0, 1), (10, 64, 256, 64, 64, 11, 1, 1), (128, 128, 256, 32, 16, 2, 0, 0), (4, 64, 128, 64, 128, 64, 1, 1),
    (20, 128, 512, 64, 32, 33, 1, 1), (2, 64, 256, 32, 16, 8, 0, 0),
])
def test_ragged_batches(dtype, h, D, R, rot, page, max_q, tree, weighs):
    rng = np.random.default_rng(h + R + max_q)
    ctx = [0, 1, 0, 15, 16, 33, 200, 0, 700, 64]
    n = [max_q, 1, 0, max_q, 1, (max_q + 1) // 2, max_q, 1, 1, max_q + 2]     # the last has more than are attended to
    ba = _Batch(rng, dtype, ctx, n, h, D, R, rot, page)
    words = _trees(rng, np.minimum(n, 64)) if tree else None
    if words and max_q + 2 > 64:
        words += [0] * (ba.T - len(words))
    t = _tree_tensor(words, ba.T) if tree else None
    mass = _dev(rng.random((len(n), 500)), torch.float32) if weighs else None
    got = ba.run(max_q, t, mass, 0.75, stride=500 if weighs else None)
    ba.check(got, max_q, words, mass, 0.75)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h,max_q", [(16, 1), (3, 4), (40, 1), (16, 4), (16, 20)])
def test_long_sequences_are_split_and_joined(dtype, h, max_q):
    rng = np.random.default_rng(h)
    ba = _Batch(rng, dtype, [5003, 40, 2500], [max_q, 1, max_q], h, 64, 256, 32, 16)
    first = ba.run(max_q, stride=5100)
    ba.check(first, max_q)
    for _ in range(3):                                       # the same bits every time
        again = ba.run(max_q, stride=5100)
        for x, y in zip(first, again):
            assert torch.equal(x, y)


def test_a_large_batch():
    """More sequences than a wave plans at a time, and more tokens than a workgroup of the last product takes."""
    rng = np.random.default_rng(11)
    n = rng.integers(0, 3, 150)
    ba = _Batch(rng, "bf16", rng.integers(0, 300, 150), n, 8, 128, 128, 32, 16)
    ba.check(ba.run(2, stride=310), 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h,max_q", [(2, 6), (4, 6), (10, 6), (30, 6)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_what_a_token_does_not_see_has_no_effect(dtype, h, max_q, value):
    rng = np.random.default_rng(5)
    ba = _Batch(rng, dtype, [37, 90], [6, 6], h, 64, 128, 64, 16)
    words = [(2 << i) - 1 for i in range(6)] + [1, 3, 5, 0, 17, 32]
    t = _tree_tensor(words, ba.T)
    want = ba.run(max_q, t)
    at = 90 + 2                                              # seen by the second sequence's third token alone
    keep = ba.rows[int(ba.table[1, at // 16]), at % 16].clone()
    ba.rows[int(ba.table[1, at // 16]), at % 16, 3] = value
    got = ba.run(max_q, t)
    sees = np.zeros(ba.T, bool)
    sees[6 + 2] = True
    for x, y in zip(want[:2], got[:2]):
        np.testing.assert_array_equal(_host(x)[~sees], _host(y)[~sees])
    assert not np.isfinite(_host(got[0])[sees]).any()
    ba.rows[int(ba.table[1, at // 16]), at % 16] = keep
    # a page outside the cache: its places are unseen
    ba.table[0, 1] = 10 ** 6
    o, _, _ = ba.run(max_q, t)
    assert torch.isfinite(o[:12].float()).all()
    rows = ba.cached(0, 16)
    rows = np.concatenate([rows, ba_rows(ba, 0, 32, 37 + 6)])
    seen = np.concatenate([np.ones((6, 16 + 5), bool), np.tril(np.ones((6, 6), bool))], 1)
    e = ol.latent_attention(_host(ba.q)[:6], rows, seen, _host(ba.wv), ba.scale)
    _within(_host(o)[:6], e["out"], (2.0 ** -7) * e["size"] + 2.0 ** -8 * np.abs(e["out"]), "out")


def ba_rows(ba, b, lo, hi):
    p = np.arange(lo, hi)
    return _host(ba.rows[_dev(ba.table[b, p // ba.page].astype(np.int64)), _dev(p % ba.page)])


def test_tokens_that_see_nothing():
    rng = np.random.default_rng(6)
    ba = _Batch(rng, "bf16", [0, 20], [4, 4], 16, 64, 128, 32, 16)
    words = [0, 2, 0, 15, 0, 1, 0, 0]
    out, lse, mass = ba.run(4, _tree_tensor(words, ba.T), stride=30)
    o, ls = _host(out), _host(lse)
    assert (o[[0, 2]] == 0).all() and np.isneginf(ls[[0, 2]]).all() and np.isfinite(ls[[1, 3, 4, 5, 6, 7]]).all()
    ba.check((out, lse, mass), 4, words)


def test_large_scores_and_a_negative_scale():
    rng = np.random.default_rng(7)
    for scale in (1.0, -1.0):
        ba = _Batch(rng, "f32", [300], [2], 4, 64, 128, 32, 16, spread=20.0)
        ba.scale *= scale
        ba.check(ba.run(2, stride=310), 2)


# ------------------------------------------------------------------ prompts
def _prompt(rng, dtype, n, ctx, h, g, D, rot, scale=None, spread=1.5):
    n, L = np.asarray(n), np.asarray(n) + np.asarray(ctx)
    L = np.maximum(L, 0)
    T, Lt = int(n.sum()) + 2, int(L.sum()) + 3
    q = _dev(rng.normal(size=(T, h, D + rot)) * spread, DT[dtype])
    k, v = (_dev(rng.normal(size=(Lt, g, D)), DT[dtype]) for _ in range(2))
    r = _dev(rng.normal(size=(Lt, rot)), DT[dtype]) if rot else None
    at = lambda a: np.concatenate([[0], np.cumsum(a)]).astype(np.int32)  # noqa: E731
    return dict(q=q, k=k, v=v, r=r, qs=at(n), ks=at(L), scale=scale or (D + rot) ** -0.5, dtype=dtype)


def _run_prompt(p, fill=7.0):
    T, h, _ = p["q"].shape
    D, g = p["k"].shape[2], p["k"].shape[1]
    rot = 0 if p["r"] is None else p["r"].shape[1]
    out = torch.full((T, h, D), fill, dtype=p["q"].dtype, device="cuda")
    lse = torch.full((T, h), fill, device="cuda")
    size = om.ordermoe_prompt_attention_workspace_size(om.BF16 if p["dtype"] == "bf16" else om.F32, h, g, D, rot, T, len(p["qs"]) - 1)
    ws = torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda")
    om.ordermoe_prompt_attention(p["q"], p["k"], p["v"], _dev(p["qs"]), _dev(p["ks"]), p["scale"], out, ws, k_shared=p["r"], lse=lse)
    return out, lse


def _check_prompt(p, got):
    o, ls = _host(got[0]), _host(got[1])
    q, k, v, r = (None if p[n] is None else _host(p[n]) for n in "qkvr")
    qs, ks = p["qs"], p["ks"]
    for b in range(len(qs) - 1):
        t, kk = slice(qs[b], qs[b + 1]), slice(ks[b], ks[b + 1])
        if t.start == t.stop:
            continue
        e = ol.prompt_attention(q[t], k[kk], v[kk], None if r is None else r[kk], p["scale"])
        L = kk.stop - kk.start
        es = e["score"] * (q.shape[2] + 4) * U
        ew = 2 * es + (8 + L) * U + (2.0 ** -8 if p["dtype"] == "bf16" else 0)
        _within(o[t], e["out"], ew * e["size"] + 2 * U * np.abs(e["out"]) + HALF[p["dtype"]] * np.abs(e["out"]), "out of %d" % b)
        _within(ls[t], e["lse"], es + (8 + L) * U + 2 * U * np.abs(np.where(np.isfinite(e["lse"]), e["lse"], 0)), "lse of %d" % b)
    assert (o[qs[-1]:] == 7).all() and (ls[qs[-1]:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h,g,D,rot", [(2, 2, 128, 64), (3, 3, 64, 32), (4, 1, 128, 0), (8, 2, 64, 0), (5, 5, 64, 64), (1, 1, 128, 32),
                                       (24, 8, 64, 0), (16, 1, 128, 0)])
def test_ragged_prompts(dtype, h, g, D, rot):
    rng = np.random.default_rng(h + D + rot)
    p = _prompt(rng, dtype, [1, 0, 31, 33, 129, 64, 300, 5, 128], [0, 3, 0, 70, 1, 64, 0, 200, 0], h, g, D, rot)
    _check_prompt(p, _run_prompt(p))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_queries_than_positions(dtype):
    rng = np.random.default_rng(2)
    p = _prompt(rng, dtype, [5, 200, 40, 7], [-2, -130, -40, 0], 2, 2, 64, 32)
    got = _run_prompt(p)
    _check_prompt(p, got)
    assert np.isneginf(_host(got[1])[[0, 1]]).all() and (_host(got[0])[[0, 1]] == 0).all()


def test_a_long_prompt_and_a_long_context():
    rng = np.random.default_rng(3)
    p = _prompt(rng, "bf16", [1500, 3], [0, 3000], 4, 4, 128, 64)
    first = _run_prompt(p)
    _check_prompt(p, first)
    for _ in range(3):
        for x, y in zip(first, _run_prompt(p)):
            assert torch.equal(x, y)
    p = _prompt(rng, "f32", [400], [600], 4, 2, 64, 0, scale=-0.2, spread=4.0)
    _check_prompt(p, _run_prompt(p))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("what", ["k", "v", "r"])
def test_a_prompt_s_later_positions_have_no_effect(dtype, value, what):
    rng = np.random.default_rng(4)
    p = _prompt(rng, dtype, [150, 40], [10, 0], 2, 2, 64, 32)
    want = _run_prompt(p)
    at = 10 + 77                                             # token 77's own position: tokens 0 .. 76 do not see it
    if what == "r":
        p["r"][at, 5] = value
    else:
        p[what][at, 1, 5] = value
    p[what][p["ks"][-1]:] = float("nan")                     # behind the last sequence
    got = _run_prompt(p)
    for x, y in zip(want, got):
        np.testing.assert_array_equal(_host(x)[:77], _host(y)[:77])
        np.testing.assert_array_equal(_host(x)[150:], _host(y)[150:])
        if what != "r":
            np.testing.assert_array_equal(_host(x)[:, 0], _host(y)[:, 0])
    if what == "v":
        assert not np.isfinite(_host(got[0])[77:150, 1, 5]).any()


# ------------------------------------------------------------------ eviction
def _evict(rng, n, seq, keep, first, recent, mass, pos, dtype="bf16", page=16, R=128, rot=32, in_place=False, bad_page=None):
    B, stride = mass.shape
    pages = -(-stride // page)
    rows = _dev(rng.normal(size=(B * pages + 1, page, R + rot)), DT[dtype])
    before = _host(rows)
    cache = om.make_latent_cache(rows, R)
    table = rng.permutation(B * pages + 1)[:B * pages].reshape(B, pages).astype(np.int32)
    if bad_page is not None:
        table[0, bad_page] = -5
    i32 = torch.int32
    d = dict(ctx=_dev(np.asarray(n, np.int32)), mass=_dev(mass.astype(np.float32)), pos=_dev(pos.astype(np.int32)))
    kept = torch.full((B, keep), 99, dtype=i32, device="cuda")
    lo = d["ctx"] if in_place else torch.full((B,), 99, dtype=i32, device="cuda")
    mo = d["mass"] if in_place else torch.full((B, stride), 99.0, device="cuda")
    po = d["pos"] if in_place else torch.full((B, stride), 99, dtype=i32, device="cuda")
    ws = torch.full((om.ordermoe_latent_evict_workspace_size(cache, B, pages, keep),), 0x7F, dtype=torch.uint8, device="cuda")
    om.ordermoe_latent_evict(cache, d["ctx"], _dev(np.asarray(seq, np.int32)), _dev(table), keep, first, recent, d["mass"], d["pos"], kept, lo,
                             mo, po, ws)
    after, kept, lo, mo, po = _host(rows), _host(kept), _host(lo), _host(mo), _host(po)
    flat = before.reshape(-1, R + rot)
    want_rows = flat.copy()
    slot = lambda b, p: table[b, p // page].astype(np.int64) * page + p % page  # noqa: E731
    for b in range(B):
        nb = min(int(n[b]), stride)
        want = ol.evict(nb, int(seq[b]), keep, first, recent, mass[b], pos[b])
        np.testing.assert_array_equal(kept[b], want)
        new = min(nb, keep)
        assert lo[b] == new
        np.testing.assert_array_equal(mo[b, :new], mass[b, want[:new]].astype(np.float32))
        np.testing.assert_array_equal(po[b, :new], pos[b, want[:new]])
        if in_place:
            np.testing.assert_array_equal(mo[b, new:], mass[b, new:].astype(np.float32))
        else:
            assert (mo[b, new:] == 99).all() and (po[b, new:] == 99).all()
        for i in np.flatnonzero(want[:new] != np.arange(new)):
            src, dst = slot(b, want[i]), slot(b, i)
            if dst >= 0:
                want_rows[dst] = flat[src] if src >= 0 else 0
    np.testing.assert_array_equal(after.reshape(-1, R + rot), want_rows)


@pytest.mark.parametrize("dtype,in_place", [("bf16", False), ("f32", True)])
@pytest.mark.parametrize("keep,first,recent", [(1, 0, 0), (20, 4, 16), (100, 0, 30), (257, 2, 0), (1000, 4, 64)])
def test_evicted_sequences(dtype, in_place, keep, first, recent):
    rng = np.random.default_rng(keep)
    B, stride = 7, 1100
    n = np.array([0, 1, keep, min(stride, keep + 1), 700, 1100, 999])
    mass = rng.random((B, stride)) ** 6 * 40
    mass[:, ::5] = 0.25                                      # ties
    mass[5, 3::7] = np.nan
    mass[5, 4] = -1.0
    mass[6, 10:14] = np.inf, -np.inf, 0.0, -0.0
    pos = np.stack([rng.permutation(2000)[:stride] for _ in range(B)])
    _evict(rng, n, np.full(B, 2000), keep, first, recent, mass, pos, dtype, in_place=in_place)


def test_evict_ties_and_sequences_longer_than_the_registers_hold():
    rng = np.random.default_rng(9)
    stride = 70001
    mass = np.stack([np.zeros(stride), np.round(rng.random(stride) * 50) / 8, rng.random(stride)])
    pos = np.tile(np.arange(stride), (3, 1))
    _evict(rng, [stride, 65537, 40000], [stride, 65537, 40000], 33000, 4, 500, mass, pos, page=1024)


def test_evict_past_the_table_and_with_a_page_outside_the_cache():
    rng = np.random.default_rng(10)
    mass, pos = rng.random((2, 100)), np.tile(np.arange(100), (2, 1))
    _evict(rng, [500, 100], [100, 100], 40, 0, 5, mass, pos)                       # more tokens than places
    _evict(rng, [96, 90], [100, 100], 40, 2, 5, mass, pos, bad_page=1)             # rows into it are dropped
    _evict(rng, [96, 90], [100, 100], 40, 2, 5, mass, pos, bad_page=4, in_place=True)   # rows from it are zeros


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("n,ctx,h,g,D,rot", [([150, 40], [10, 0], 2, 2, 64, 32), ([16, 5], [2500, 700], 8, 2, 128, 0), ([300], [0], 4, 1, 128, 64)])
def test_a_value_that_is_no_number_reaches_its_own_element_alone(dtype, value, n, ctx, h, g, D, rot):
    """Of the tokens that see it, in tiles that all of a workgroup's tokens see and in others; the sums of the weights stay."""
    rng = np.random.default_rng(n[0] + D)
    p = _prompt(rng, dtype, n, ctx, h, g, D, rot)
    want = _run_prompt(p)
    hit = {(c, g - 1, e) for c, e in ((0, 3), (ctx[0] // 2, 9), (ctx[0] + 2, 5), (ctx[0] + 7, 5), (ctx[0] + 7, 6), (ctx[0] + n[0] - 1, D - 1))}
    for at, kh, e in hit:                                    # positions of the first sequence
        p["v"][at, kh, e] = value
    got = _run_prompt(p)
    assert torch.equal(want[1], got[1])
    spoilt = np.zeros(got[0].shape, bool)
    for at, kh, e in hit:
        spoilt[max(0, at - ctx[0]):n[0], kh * (h // g):(kh + 1) * (h // g), e] = True
    np.testing.assert_array_equal(_host(want[0])[~spoilt], _host(got[0])[~spoilt])
    assert not np.isfinite(_host(got[0])[spoilt]).any()


# ------------------------------------------------------------------ keys that are no numbers
def _by_scores(got, e, lse, score, width, L, rounding, dtype, extra=0.0):
    """out [n, h, D] and lse [n, h] against the oracle's, where a score of +infinity or NaN makes a row NaN whole, and one of
    -infinity is as a place that is not seen."""
    out, ls = got
    spoilt = ~np.isfinite(e["out"]).all(-1)
    assert np.isnan(out[spoilt]).all() and np.isnan(ls[spoilt]).all()
    es = score * (width + 4) * U
    tol = (2 * es + (8 + L) * U + rounding) * e["size"] + extra + (2 * U + HALF[dtype]) * np.abs(e["out"])
    _within(out[~spoilt], e["out"][~spoilt], tol[~spoilt], "out")
    fine = ~spoilt & np.isfinite(lse)
    _within(ls[fine], lse[fine], es + (8 + L) * U + 2 * U * np.abs(lse[fine]), "lse")
    nothing = ~spoilt & np.isneginf(lse)
    assert np.isneginf(ls[nothing]).all() and (out[nothing] == 0).all()
    return spoilt, nothing


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("n,ctx,h,g,D,rot,scale", [(150, 10, 2, 2, 64, 32, 0.1), (16, 2500, 8, 2, 128, 0, -0.08), (300, 0, 4, 1, 128, 64, 0.07)])
def test_a_key_that_is_no_number_acts_through_its_score(dtype, value, n, ctx, h, g, D, rot, scale):
    rng = np.random.default_rng(n + D)
    p = _prompt(rng, dtype, [n], [ctx], h, g, D, rot, scale)
    clean = ol.prompt_attention(*(None if p[c] is None else _host(p[c])[:k] for c, k in (("q", n), ("k", n + ctx), ("v", n + ctx), ("r", n + ctx))),
                                scale)
    # seen by the first token alone of all that it sees (or of a few), in tiles that all rows see, and late
    for what, at in [("k", 0), ("k", ctx + 3), ("k", ctx + n - 2)] + ([("r", 0), ("r", ctx + 7)] if rot else []):
        t = p[what]
        keep = t[at].clone()
        if what == "k":
            t[at, g - 1, 5] = value
        else:
            t[at, 6] = value
        q, k, v, r = (None if p[c] is None else _host(p[c]) for c in "qkvr")
        L = n + ctx
        with np.errstate(invalid="ignore"):
            e = ol.prompt_attention(q[:n], k[:L], v[:L], None if r is None else r[:L], scale)
        got = _run_prompt(p)
        spoilt, _ = _by_scores((_host(got[0])[:n], _host(got[1])[:n]), e, e["lse"], clean["score"], D + rot, L,
                               2.0 ** -8 if dtype == "bf16" else 0.0, dtype)
        sees = np.arange(n)[:, None] + ctx >= at
        x = q[:n, :, 5] if what == "k" else q[:n, :, D + 6]
        reads = np.arange(h)[None, :] >= (h - h // g if what == "k" else 0)
        want = sees & reads & (np.ones_like(x, bool) if np.isnan(value) else x * scale * value > 0)
        np.testing.assert_array_equal(spoilt, want)
        t[at] = keep


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("h,n", [(2, 1), (3, 6), (8, 4), (10, 6)])
def test_a_cached_row_that_is_no_number(dtype, value, h, n):
    """In its rotary part it acts through its score; in its latent part, which is the value too, it spoils the tokens that see it."""
    rng = np.random.default_rng(h + n)
    D, R, rot, ctx = 64, 128, 32, 130
    ba = _Batch(rng, dtype, [ctx], [n], h, D, R, rot, 16)
    words = [(2 << i) - 1 for i in range(n)]
    seen = ol.tree_seen(n, ctx, words, ctx + n)
    clean = ol.latent_attention(_host(ba.q)[:n], ba.cached(0, ctx + n), seen, _host(ba.wv), ba.scale)
    for at in (3, ctx - 1, ctx + n - 1):                     # in a tile that all see; beside places that some do not
        slot = ba.rows[int(ba.table[0, at // 16]), at % 16]
        keep = slot.clone()
        slot[R + 5] = value
        with np.errstate(invalid="ignore"):
            e = ol.latent_attention(_host(ba.q)[:n], ba.cached(0, ctx + n), seen, _host(ba.wv), ba.scale)
        out, lse, mass = ba.run(n, stride=ctx + n)
        rounding = 0.0 if dtype == "f32" else 2.0 ** -16 if n * h <= 32 else 2.0 ** -8
        spoilt, _ = _by_scores((_host(out)[:n], _host(lse)[:n]), e, e["lse"], clean["score"], R + rot, ctx + n, rounding, dtype,
                               (2.0 ** -16 + (R + 1) * U) * e["through"])
        x = _host(ba.q)[:n, :, R + 5]
        np.testing.assert_array_equal(spoilt, seen[:, None, at] & (np.ones_like(x, bool) if np.isnan(value) else x * value > 0))
        if not spoilt.any():
            assert torch.isfinite(mass).all() and float(mass[0, at]) == 0
        slot.copy_(keep)
        slot[7] = value
        out, _, _ = ba.run(n, stride=ctx + n)
        np.testing.assert_array_equal(np.isnan(_host(out)[:n]).all((1, 2)), seen[:, at])
        assert np.isfinite(_host(out)[:n][~seen[:, at]]).all()
        slot.copy_(keep)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_whose_every_score_is_minus_infinity(dtype):
    """As tokens that see nothing."""
    rng = np.random.default_rng(14)
    p = _prompt(rng, dtype, [3, 70], [0, 0], 2, 2, 64, 0)
    p["q"] = p["q"].abs()
    p["k"][0, 1, 9] = -float("inf")                          # the only position of the first token
    p["k"][3:73, 0, 9] = -float("inf")
    out, lse = _run_prompt(p)
    assert (out[0, 1] == 0).all() and torch.isneginf(lse[0, 1]) and torch.isfinite(lse[0, 0]) and torch.isfinite(lse[1:3]).all()
    assert (out[3:73, 0] == 0).all() and torch.isneginf(lse[3:73, 0]).all() and torch.isfinite(lse[3:73, 1]).all()
    ba = _Batch(rng, dtype, [0, 40], [1, 2], 3, 64, 128, 32, 16)
    ba.q.abs_()
    ba.rows[int(ba.table[0, 0]), 0, 128] = -float("inf")
    out, lse, mass = ba.run(2, stride=50)
    assert (out[0] == 0).all() and torch.isneginf(lse[0]).all() and torch.isfinite(lse[1:3]).all() and float(mass[0, 0]) == 0


def test_long_sums_in_fp32_keep_their_bits():
    """Outputs' error against 64 bits, of their size.  A sum of n products of varying sign, in one sum, is off by u sqrt(n / 6) of its
    size (partial sums grow with the square root of their terms, each rounding is u / sqrt(3) of one); in four sums by half of that.
    A score's error is its weight's: with scores of size 2, 2 * u sqrt(544 / 6) / 2; then the last product's, u sqrt(512 / 6) / 2; half as much
    again for the weights' sums and exponentials."""
    rng = np.random.default_rng(20)
    R, rot, h, D = 512, 32, 20, 128
    ba = _Batch(rng, "f32", np.linspace(85, 686, 8).astype(int), [1] * 8, h, D, R, rot, 16)
    out, _, _ = ba.run(1)
    off = size = 0.0
    for b in range(8):
        L = int(ba.ctx[b]) + 1
        e = ol.latent_attention(_host(ba.q)[b:b + 1], ba.cached(b, L), np.ones((1, L), bool), _host(ba.wv), ba.scale)["out"]
        off, size = off + ((_host(out)[b] - e[0]) ** 2).sum(), size + (e ** 2).sum()
    assert (off / size) ** 0.5 <= 1.5 * U * np.hypot((R + rot) ** 0.5, R ** 0.5 / 2) / 6 ** 0.5
