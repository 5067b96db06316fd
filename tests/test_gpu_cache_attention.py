"""The quantised cache and the drafted tokens' attention against the oracle,
through the C ABI.

Tolerances, fixed beforehand:
  codes and scales of rows that are neither normed nor turned: the same bits (the
    definition is in fp32 steps that round the same everywhere);
  normed and turned rows: fp32 arithmetic of at most 16 additions in a chain and
    4 in a tree, a square root, a division and about 8 products: 32 roundings of 2^-24 each,
    relative to the row's largest magnitude; then half a code step for codes, 2^-8 of
    the value (bf16's rounding) for queries;
  attention, bf16: each weight is rounded to bf16 (8 significant bits: 2^-8) and so is
    the output (2^-8): 2^-7 of sum_p weight |v_p|, and 1e-4 of it for the fp32 sums;
    lse: 2e-6 + 2e-6 |lse|;
  attention, fp32: scores of up to 256 products, each rounded 2^-24 relative to
    terms that sum to at most about 40 here: an error of a score below 2e-5 (that of a
    weight), and as much again for the sums: 4e-5 of sum_p weight |v_p|; lse 2e-5."""
import numpy as np
import pytest

from oracle import attention as oa

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2607_17154_amd import ordermoe as om  # noqa: E402

FMT = {"int8": om.CACHE_INT8, "fp8": om.CACHE_FP8}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
CODE = {"bf16": om.BF16, "f32": om.F32}


def _dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _host(t):
    return t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


class _Cache:
    """A cache whose memory starts as nothing a writer makes: NaN codes, NaN scales."""

    def __init__(self, fmt, n_pages, n_kv, page, D):
        self.fmt, self.page = FMT[fmt], page
        self.codes = [torch.full((n_pages, n_kv, page, D), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(2)]
        self.scale = [torch.full((n_pages, n_kv, page), float("nan"), device="cuda") for _ in range(2)]
        self.c = om.make_cache(self.fmt, *self.codes, *self.scale)

    def fill(self, slots, rng, spread=1.0):
        """Random rows at the slots, straight into the memory."""
        n, kv, D = len(slots), self.codes[0].shape[1], self.codes[0].shape[3]
        p, o = _dev(slots // self.page), _dev(slots % self.page)
        for i in range(2):
            codes, scale = oa.quantise((rng.normal(size=(n, kv, D)) * spread).astype(np.float32), self.fmt)
            self.codes[i][p, :, o] = _dev(codes)
            self.scale[i][p, :, o] = _dev(scale)

    def rows(self, slots):
        return [oa.cache_rows(_host(c), _host(s), slots, self.fmt) for c, s in zip(self.codes, self.scale)]


# ------------------------------------------------------------------ write and read
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("T,hq,hkv,D,page", [(1, 1, 1, 64, 16), (37, 6, 2, 128, 32), (130, 4, 4, 256, 16), (5, 32, 8, 128, 1024)])
def test_plain_rows_have_the_oracle_s_bits(dtype, fmt, T, hq, hkv, D, page):
    rng = np.random.default_rng(T + D)
    ca = _Cache(fmt, 2 * -(-T // page) + 1, hkv, page, D)
    x = _dev(rng.normal(size=(T, hq + 2 * hkv, D)) * np.exp(rng.normal(size=(T, hq + 2 * hkv, 1)) * 3), DT[dtype])
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]      # one array of QKV rows
    slots = rng.permutation(ca.codes[0].shape[0] * page)[:T].astype(np.int64)
    q_out = torch.empty((T, hq, D), dtype=DT[dtype], device="cuda")
    om.ordermoe_cache_write(ca.c, om.make_heads(CODE[dtype], hq, D), q, k, v, None, _dev(slots), q_out)
    np.testing.assert_array_equal(_host(q_out), _host(q))
    for i, src in enumerate((k, v)):
        codes, scale = oa.quantise(_host(src), FMT[fmt])
        np.testing.assert_array_equal(_host(ca.codes[i])[slots // page, :, slots % page], codes)
        np.testing.assert_array_equal(_host(ca.scale[i])[slots // page, :, slots % page], scale)
    # every other slot is as it was
    left = np.ones(ca.codes[0].shape[0] * page, bool)
    left[slots] = False
    for i in range(2):
        assert (_host(ca.codes[i].transpose(1, 2).reshape(-1, hkv, D))[left] == 0x7F).all()
    # read back, any order, repeats and slots outside: the values, rounded once
    at = np.concatenate([slots[::-1], slots[:1], [-1, ca.codes[0].shape[0] * page, -(1 << 40)]]).astype(np.int64)
    inside = np.arange(len(at)) <= T
    for out_dt in (torch.float32, torch.bfloat16):
        ko, vo = (torch.full((len(at), hkv, D), 7.0, dtype=out_dt, device="cuda") for _ in range(2))
        om.ordermoe_cache_read(ca.c, _dev(at), ko, vo)
        for got, want in zip((ko, vo), ca.rows(at[inside])):
            exp = torch.from_numpy(want.astype(np.float32)).to(out_dt)
            np.testing.assert_array_equal(_host(got)[inside], _host(exp))
            assert (_host(got)[~inside] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("D,rot,inter,norm", [(64, 64, 0, "qk"), (64, 8, 1, "k"), (128, 128, 1, "qk"), (128, 48, 0, "q"),
                                              (256, 256, 0, "qk"), (256, 96, 1, ""), (128, 0, 0, "qk")])
def test_normed_and_turned_rows(dtype, fmt, D, rot, inter, norm):
    T, hq, hkv, page, max_pos = 29, 4, 2, 16, 5000
    rng = np.random.default_rng(D + rot)
    ca = _Cache(fmt, 4, hkv, page, D)
    parts = [_dev(rng.normal(size=(T, h, D)) * 2, DT[dtype]) for h in (hq, hkv, hkv)]
    w = [_dev(1 + 0.2 * rng.normal(size=D), DT[dtype]) if n in norm else None for n in "qk"]
    table = om.rotary_table(max_pos, rot)
    pos = rng.integers(0, max_pos, T).astype(np.int32)
    pos[:2] = 0, max_pos - 1
    slots = rng.permutation(4 * page)[:T].astype(np.int64)
    heads = om.make_heads(CODE[dtype], hq, D, *w, _dev(table) if rot else None, inter, 1e-5)
    q_out = torch.empty((T, hq, D), dtype=DT[dtype], device="cuda")
    om.ordermoe_cache_write(ca.c, heads, *parts, _dev(pos), _dev(slots), q_out)
    h = lambda t: None if t is None else _host(t)  # noqa: E731
    q, k = (oa.head_rows(_host(x), h(ww), 1e-5, table if rot else None, pos, bool(inter)) for x, ww in zip(parts, w))
    fp = 32 * 2.0 ** -24
    big = lambda x: np.abs(x).max(-1, keepdims=True)  # noqa: E731
    assert (np.abs(_host(q_out) - q) <= fp * big(q) + (2.0 ** -8 * np.abs(q) if dtype == "bf16" else 0)).all()
    kv, _ = ca.rows(slots)
    half = big(k) / 254 if fmt == "int8" else np.maximum(np.abs(k) / 16, big(k) / 448 * 2.0 ** -10)
    assert (np.abs(kv - k) <= half * 1.0001 + fp * big(k)).all()
    # the values are untouched by norm and rotation
    codes, scale = oa.quantise(_host(parts[2]), FMT[fmt])
    np.testing.assert_array_equal(_host(ca.codes[1])[slots // page, :, slots % page], codes)


def test_rows_without_a_slot_or_a_position_and_rows_that_are_no_numbers():
    T, hq, hkv, D, page = 8, 2, 1, 128, 16
    rng = np.random.default_rng(0)
    ca = _Cache("fp8", 1, hkv, page, D)
    x = rng.normal(size=(T, hq + 2 * hkv, D)).astype(np.float32)
    x[3, hq, 5] = np.inf                  # a key
    x[4, hq + 1, 6] = np.nan              # a value
    x[5, hq + 1] = 0
    x[6, hq + 1] = 1e-35
    x = _dev(x)
    slots = np.array([-1, 16, 2, 3, 4, 5, 6, 1 << 50], np.int64)
    pos = np.array([0, 1, 9, 3, 4, 5, -1, 7], np.int32)          # tokens 2 and 6: outside the table of 9
    q_out = torch.zeros((T, hq, D), device="cuda")
    om.ordermoe_cache_write(ca.c, om.make_heads(om.F32, hq, D, None, None, _dev(om.rotary_table(9, 64))), x[:, :hq],
                            x[:, hq:hq + hkv], x[:, hq + hkv:], _dev(pos), _dev(slots), q_out)
    codes, scale = [_host(c)[0, 0] for c in ca.codes], [_host(s)[0, 0] for s in ca.scale]
    for i in range(2):                    # slots that no token has
        keep = np.setdiff1d(np.arange(page), [2, 3, 4, 5, 6])
        assert (codes[i][keep] == 0x7F).all() and np.isnan(scale[i][keep]).all()
    q = _host(q_out)
    out = np.isin(np.arange(T), [2, 6])
    assert np.isnan(q[out][:, :, :64]).all() and np.isfinite(q[~out]).all() and np.isfinite(q[out][:, :, 64:]).all()
    assert np.isnan(scale[0][[2, 3, 6]]).all() and (codes[0][[2, 3, 6]] == 0).all()
    assert np.isnan(scale[1][4]) and (codes[1][4] == 0).all()
    assert (scale[1][[5, 6]] == 0).all() and (codes[1][[5, 6]] == 0).all()
    assert np.isfinite(scale[0][[4, 5]]).all() and (codes[0] != 0x7F)[[2, 3, 4, 5, 6]].all()


@pytest.mark.parametrize("dtype,D,hq,hkv,T", [("bf16", 128, 32, 8, 4201), ("f32", 64, 48, 4, 2801), ("bf16", 64, 64, 8, 4203)])
def test_a_prompt_in_one_call_and_in_parts(dtype, D, hq, hkv, T):
    """Rows of over 32 MiB go past the caches; the same rows in parts of a few hundred tokens have the same bits."""
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    qkv = torch.randn((T, hq + 2 * hkv, D), generator=g, device="cuda").to(DT[dtype])
    q, k, v = qkv.split([hq, hkv, hkv], 1)
    assert q.numel() * q.element_size() > 32 << 20
    page, pages = 64, -(-T // 64)
    w = [(1 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(DT[dtype]) for _ in range(2)]
    heads = om.make_heads(CODE[dtype], hq, D, *w, _dev(om.rotary_table(T, D)), 0)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:T]
    res = []
    for step in (T, 401):
        ca, out = _Cache("int8", pages, hkv, page, D), torch.empty((T, hq, D), dtype=DT[dtype], device="cuda")
        for i in range(0, T, step):
            c = slice(i, i + step)
            om.ordermoe_cache_write(ca.c, heads, q[c], k[c], v[c], pos[c], slots[c], out[c])
        torch.cuda.synchronize()
        res.append([out] + ca.codes + [s.nan_to_num(-1.0) for s in ca.scale])
    for a, b in zip(*res):
        assert torch.equal(a, b)


def test_slots_past_2_31_bytes():
    """A slot whose codes lie more than 2^31 bytes into the cache, written, read and attended."""
    n_kv, page, D = 16, 128, 256
    n_pages = (1 << 31) // (n_kv * page * D) + 2
    codes = [torch.empty((n_pages, n_kv, page, D), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scale = [torch.empty((n_pages, n_kv, page), device="cuda") for _ in range(2)]
    c = om.make_cache(om.CACHE_INT8, *codes, *scale)
    rng = np.random.default_rng(5)
    x = _dev(rng.normal(size=(3, 3 * n_kv, D)), torch.bfloat16)
    slots = _dev(np.array([(n_pages - 1) * page, (n_pages - 1) * page + 1, (n_pages - 1) * page + 2], np.int64))
    q = torch.empty((3, n_kv, D), dtype=torch.bfloat16, device="cuda")
    om.ordermoe_cache_write(c, om.make_heads(om.BF16, n_kv, D), x[:, :n_kv], x[:, n_kv:2 * n_kv], x[:, 2 * n_kv:], None, slots, q)
    ko, vo = (torch.empty((3, n_kv, D), device="cuda") for _ in range(2))
    om.ordermoe_cache_read(c, slots, ko, vo)
    for got, src in ((ko, x[:, n_kv:2 * n_kv]), (vo, x[:, 2 * n_kv:])):
        cd, sc = oa.quantise(_host(src), oa.INT8)
        np.testing.assert_array_equal(_host(got), oa.code_values(oa.INT8).astype(np.float32)[cd] * sc[..., None])
    out = torch.empty_like(q)
    ws = torch.empty(om.ordermoe_draft_attention_workspace_size(c, om.BF16, n_kv, 1, 3), dtype=torch.uint8, device="cuda")
    om.ordermoe_draft_attention(c, q, _dev(np.array([0, 3], np.int32)), _dev(np.array([0], np.int32)),
                                _dev(np.array([[n_pages - 1]], np.int32)), 3, D ** -0.5, out, ws)
    want, _, mag = oa.draft_attention(_host(q), _host(ko).astype(np.float64), _host(vo).astype(np.float64), 0, oa.chain(3), D ** -0.5)
    assert (np.abs(_host(out) - want) <= (2.0 ** -7 + 1e-4) * mag).all()


# ------------------------------------------------------------------ attention
def _trees(rng, n, empty):
    """Words of a random tree of n drafted tokens; `empty` of them see no token of it."""
    words = []
    for i in range(n):
        up = int(rng.integers(0, i + 1))
        words.append((words[up - 1] if up else 0) | (1 << i))
    for i in rng.permutation(n)[:empty]:
        words[i] = 0
    return words


class _Batch:
    def __init__(self, rng, fmt, dtype, ctx, n, hq, hkv, D, page, tree, spread=1.0):
        self.hq, self.D, self.n, self.ctx, self.dtype = hq, D, n, ctx, dtype
        L = [c + m if m else 0 for c, m in zip(ctx, n)]
        pages = [-(-v // page) for v in L]
        self.ca = _Cache(fmt, sum(pages) + 2, hkv, page, D)
        order = rng.permutation(sum(pages) + 2)
        table = np.full((len(n), max(pages + [0]) + 1), 1 << 30, np.int32)       # unused entries: no page of the cache
        self.slots, at = [], 0
        for b, p in enumerate(pages):
            table[b, :p] = order[at:at + p]
            at += p
            pos = np.arange(L[b])
            self.slots.append(table[b, pos // page].astype(np.int64) * page + pos % page)
        self.ca.fill(np.concatenate(self.slots), rng, spread)
        T = sum(n)
        self.q = _dev(rng.normal(size=(T, hq, D)) * spread, DT[dtype])
        self.words = [_trees(rng, m, m // 4) if tree else oa.chain(m) for m in n]
        flat = np.array([w for ws in self.words for w in ws], np.uint64).view(np.int64)
        self.tree = _dev(flat) if tree else None
        self.start, self.ctx_d, self.table = (_dev(np.asarray(a, np.int32)) for a in (np.concatenate([[0], np.cumsum(n)]), ctx, table))
        self.scale = D ** -0.5

    def run(self, max_q=None, lse=True, stream=None):
        max_q = max_q or max(self.n + [1])
        out = torch.full_like(self.q, 77.0)
        ls = torch.full(self.q.shape[:2], 77.0, device="cuda") if lse else None
        need = om.ordermoe_draft_attention_workspace_size(self.ca.c, CODE[self.dtype], self.hq, len(self.n), max_q)
        ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")          # NaNs wherever it is read unwritten
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        om.ordermoe_draft_attention(self.ca.c, self.q, self.start, self.ctx_d, self.table, max_q, self.scale, out, ws, tree=self.tree,
                                    lse=ls, stream=stream)
        torch.cuda.synchronize()
        return _host(out), (_host(ls) if lse else None)

    def want(self):
        t, res = 0, []
        for b, m in enumerate(self.n):
            k, v = self.ca.rows(self.slots[b])
            res.append(oa.draft_attention(_host(self.q[t:t + m]), k, v, self.ctx[b], self.words[b], self.scale))
            t += m
        return [np.concatenate(x) for x in zip(*res)]

    def check(self, got):
        out, lse = got
        w_out, w_lse, mag = self.want()
        tol = (2.0 ** -7 + 1e-4) if self.dtype == "bf16" else 4e-5
        over = np.abs(out - w_out) - tol * mag
        assert (over <= 0).all(), over.max()
        if lse is not None:
            empty = np.isneginf(w_lse)
            np.testing.assert_array_equal(np.isneginf(lse), empty)
            assert (out[empty] == 0).all()
            e = 2e-6 if self.dtype == "bf16" else 2e-5
            assert (np.abs(lse[~empty] - w_lse[~empty]) <= e + 2e-6 * np.abs(w_lse[~empty])).all()


SHAPES = [  # ctx, n, hq, hkv, D, page, tree
    ([0], [1], 1, 1, 128, 16, False),                       # one token alone
    ([0], [1], 4, 1, 64, 16, True),                         # which may see nothing at all
    ([5, 0, 700, 31], [1, 1, 1, 1], 8, 2, 128, 32, False),
    ([16, 15, 17, 32, 33, 127, 128, 129], [1] * 8, 4, 4, 64, 16, False),
    ([0, 3, 64, 1], [7, 0, 16, 1], 6, 2, 128, 16, True),    # a sequence without drafts between others
    ([40, 0], [64, 64], 2, 2, 128, 64, True),
    ([9, 300], [64, 33], 16, 2, 128, 32, True),             # several row blocks
    ([77], [64], 8, 1, 256, 128, True),
    ([10, 1000], [5, 9], 3, 1, 256, 16, True),
    ([2600, 3, 1500], [2, 3, 1], 4, 2, 128, 64, True),      # split over workgroups, and not
    ([5000], [1], 2, 1, 64, 16, False),
    ([4111], [40], 4, 2, 64, 1024, False),
    ([600] * 70, [1] * 70, 2, 1, 64, 32, False),            # more sequences than lanes
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attention(dtype, fmt, shape):
    ctx, n, hq, hkv, D, page, tree = SHAPES[shape]
    b = _Batch(np.random.default_rng(shape), fmt, dtype, ctx, n, hq, hkv, D, page, tree)
    got = b.run()
    b.check(got)
    # again, on another stream, with a larger bound and without lse: the same bits where nothing else is split
    s = torch.cuda.Stream()
    again, _ = b.run(lse=False, stream=s)
    np.testing.assert_array_equal(again, got[0])
    b.check(b.run(max_q=64))


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("ctx,n,hq,hkv,D,page", [
    ([777, 3, 2600], [1, 1, 1], 32, 8, 128, 64), ([5000], [4], 4, 1, 64, 16), ([900, 31], [5, 1], 6, 2, 256, 32)])
def test_few_rows_keep_the_weights_bits(fmt, ctx, n, hq, hkv, D, page):
    """Up to 16 rows a head (or heads of 256): the output's rounding, 2^-8 of it, and of the terms'
    sum 2^-17 for the weights in two parts and 2^-24 D |score| (|score| < 5) for the scores."""
    b = _Batch(np.random.default_rng(21), fmt, "bf16", ctx, n, hq, hkv, D, page, False)
    out, _ = b.run()
    want, _, mag = b.want()
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -17 + 5 * D * 2.0 ** -24 + 2e-6) * mag
    over = np.abs(out - want) - tol
    assert (over <= 0).all(), over.max()


@pytest.mark.parametrize("spread", [0.0, 1e-3, 12.0])
def test_scores_from_all_equal_to_far_apart(spread):
    """Weights that are all 1/len, and ones where a few keys take everything (the
    running maximum then moves by more than its allowance, several times)."""
    b = _Batch(np.random.default_rng(3), "int8", "bf16", [900, 2100], [3, 5], 4, 2, 128, 16, True, spread)
    out, lse = b.run()
    w_out, w_lse, mag = b.want()
    # scores up to 12 * 12 * sqrt(128) * 3: fp32 holds them to 2^-24 of their terms' sum
    e = 2e-6 if spread < 2 else 5e-3
    np.testing.assert_allclose(lse, w_lse, atol=e, rtol=2e-6)
    assert (np.abs(out - w_out) <= (2.0 ** -7 + 1e-4 + 2 * e) * mag + 1e-30).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_rising_score_on_every_token(dtype):
    """Keys whose scores grow along the sequence: every tile has a new maximum."""
    rng = np.random.default_rng(4)
    b = _Batch(rng, "int8", dtype, [1300], [4], 2, 1, 64, 16, False)
    p, o = _dev(b.slots[0] // 16), _dev(b.slots[0] % 16)
    b.q.abs_()
    b.ca.codes[0][p, :, o] = _dev(np.full((1304, 1, 64), 100, np.uint8))
    b.ca.scale[0][p, 0, o] = _dev((np.arange(1304) * (1e-4 if dtype == "bf16" else 4e-5) + 1e-4).astype(np.float32))
    b.check(b.run())


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_what_is_not_seen_has_no_effect(fmt, bad):
    """Drafted tokens whose rows are no numbers change nothing for tokens that do not
    see them, and make those that do NaN (NaN value rows: the whole row of the output)."""
    rng = np.random.default_rng(6)
    b = _Batch(rng, fmt, "bf16", [50, 900], [12, 20], 4, 2, 128, 16, True)
    clean = b.run()
    b.check(clean)
    t = 0
    for s, m in enumerate(b.n):
        j = m // 2                                          # drafted token j: its key and its value
        slot = int(b.slots[s][b.ctx[s] + j])
        for sc in b.ca.scale:
            sc[slot // 16, :, slot % 16] = float(bad)
        sees = np.array([(w >> j) & 1 for w in b.words[s]], bool)
        assert sees.any() and not sees.all()
        out, lse = b.run()
        np.testing.assert_array_equal(out[t:t + m][~sees], clean[0][t:t + m][~sees])
        np.testing.assert_array_equal(lse[t:t + m][~sees], clean[1][t:t + m][~sees])
        assert np.isnan(out[t:t + m][sees]).any(-1).all()
        t += m


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("hq,D", [(4, 128), (2, 64), (8, 256)])
def test_drafted_places_that_nothing_was_written_to(dtype, fmt, hq, D):
    """A padded place of a tree has no row in the cache; no token sees it, and whatever
    its slot holds (codes that are no numbers, a scale that is none) changes nothing."""
    rng = np.random.default_rng(12)
    b = _Batch(rng, fmt, dtype, [50, 0, 900], [12, 3, 33], hq, 2, D, 16, True)
    pads = [(s, int(j)) for s, m in enumerate(b.n) for j in rng.permutation(m)[:1 + m // 6]]
    for s, j in pads:
        b.words[s] = [w & ~(1 << j) for w in b.words[s]]
    b.tree = _dev(np.array([w for ws in b.words for w in ws], np.uint64).view(np.int64))
    clean = b.run()
    b.check(clean)
    for s, j in pads:
        slot = int(b.slots[s][b.ctx[s] + j])
        for codes, scale in zip(b.ca.codes, b.ca.scale):
            codes[slot // 16, :, slot % 16] = 0x7F if j % 2 else 0xFF
            scale[slot // 16, :, slot % 16] = float("nan")
    for got, want in zip(b.run(), clean):
        np.testing.assert_array_equal(got, want)


def test_pages_outside_the_cache_and_positions_past_the_table_are_unseen():
    rng = np.random.default_rng(7)
    b = _Batch(rng, "int8", "bf16", [100, 40], [2, 3], 2, 1, 64, 16, False)
    want = []
    for s, hole in ((0, 2), (1, 0)):                        # positions 32 .. 47 of the first, 0 .. 15 of the second
        b.table[s, hole] = (-5, 1 << 29)[s]
        L = b.ctx[s] + b.n[s]
        keep = np.array([p for p in range(L) if p // 16 != hole])
        k, v = b.ca.rows(b.slots[s][keep])
        t = sum(b.n[:s])
        want.append(oa.draft_attention(_host(b.q[t:t + b.n[s]]), k, v, b.ctx[s] - 16, b.words[s], b.scale))
    out, lse = b.run()
    w_out, w_lse, mag = (np.concatenate(x) for x in zip(*want))
    assert (np.abs(out - w_out) <= (2.0 ** -7 + 1e-4) * mag).all()
    np.testing.assert_allclose(lse, w_lse, atol=2e-6, rtol=2e-6)
    # a table that ends before the sequences do
    b = _Batch(rng, "int8", "bf16", [100], [2], 2, 1, 64, 16, False)
    b.table = b.table[:, :3].contiguous()
    k, v = b.ca.rows(b.slots[0][:48])
    w_out, w_lse, mag = oa.draft_attention(_host(b.q), k, v, 48, [0, 0], b.scale)
    out, lse = b.run()
    assert (np.abs(out - w_out) <= (2.0 ** -7 + 1e-4) * mag).all()
    np.testing.assert_allclose(lse, w_lse, atol=2e-6, rtol=2e-6)


def test_rows_of_no_sequence_and_past_max_q_are_not_written():
    rng = np.random.default_rng(8)
    b = _Batch(rng, "fp8", "bf16", [20, 30], [3, 6], 2, 1, 64, 16, False)
    full = b.run()
    out, lse = b.run(max_q=4)
    # the second sequence's first four tokens see the same cache: the rows past them are left alone
    assert (out[7:] == 77).all() and (lse[7:] == 77).all()
    np.testing.assert_array_equal(out[:3], full[0][:3])
    np.testing.assert_array_equal(out[3:7], full[0][3:7])
    b.start = _dev(np.array([2, 3, 9], np.int32))
    out, _ = b.run(max_q=6)
    assert (out[:2] == 77).all() and (out[2:] != 77).all()


def test_written_then_attended_equals_the_oracle_on_the_same_rows():
    """The two operators together: prompt rows written, a drafted tree written and attended."""
    rng = np.random.default_rng(9)
    ctx, n, hq, hkv, D, page = 45, 6, 4, 2, 128, 16
    ca = _Cache("fp8", 5, hkv, page, D)
    table = np.array([[3, 0, 4, 1]], np.int32)
    words = _trees(rng, n, 0)
    depth = [bin(w).count("1") - 1 for w in words]
    pos = np.concatenate([np.arange(ctx), ctx + np.array(depth)]).astype(np.int32)
    slots = np.array([table[0, p // page] * page + p % page for p in range(ctx + n)], np.int64)
    x = _dev(rng.normal(size=(ctx + n, hq + 2 * hkv, D)), torch.bfloat16)
    q = torch.empty((ctx + n, hq, D), dtype=torch.bfloat16, device="cuda")
    heads = om.make_heads(om.BF16, hq, D, *(_dev(np.ones(D), torch.bfloat16) for _ in range(2)), _dev(om.rotary_table(100, D)))
    om.ordermoe_cache_write(ca.c, heads, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], _dev(pos), _dev(slots), q)
    qd = q[ctx:].contiguous()
    out = torch.empty_like(qd)
    ws = torch.empty(om.ordermoe_draft_attention_workspace_size(ca.c, om.BF16, hq, 1, n), dtype=torch.uint8, device="cuda")
    om.ordermoe_draft_attention(ca.c, qd, _dev(np.array([0, n], np.int32)), _dev(np.array([ctx], np.int32)), _dev(table), n,
                                D ** -0.5, out, ws, tree=_dev(np.array(words, np.int64)))
    k, v = ca.rows(slots)
    want, _, mag = oa.draft_attention(_host(qd), k, v, ctx, words, D ** -0.5)
    assert (np.abs(_host(out) - want) <= (2.0 ** -7 + 1e-4) * mag).all()


def test_captured_calls_follow_their_lengths():
    """A HIP graph of write and attention, replayed as the sequence grows by a token."""
    rng = np.random.default_rng(10)
    hq, hkv, D, page, start = 4, 2, 64, 16, 20
    ca = _Cache("int8", 4, hkv, page, D)
    table = _dev(np.array([[2, 0, 3, 1]], np.int32))
    slot_of = [int([2, 0, 3, 1][p // page] * page + p % page) for p in range(64)]
    ca.fill(np.array(slot_of[:start]), rng)
    x = torch.zeros((1, hq + 2 * hkv, D), dtype=torch.bfloat16, device="cuda")
    pos, slots, ctx = (torch.zeros(1, dtype=d, device="cuda") for d in (torch.int32, torch.int64, torch.int32))
    q_start = _dev(np.array([0, 1], np.int32))
    q, out = (torch.zeros((1, hq, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = torch.empty(om.ordermoe_draft_attention_workspace_size(ca.c, om.BF16, hq, 1, 1), dtype=torch.uint8, device="cuda")
    heads = om.make_heads(om.BF16, hq, D, None, None, _dev(om.rotary_table(64, D)))

    def step():
        om.ordermoe_cache_write(ca.c, heads, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], pos, slots, q)
        om.ordermoe_draft_attention(ca.c, q, q_start, ctx, table, 1, D ** -0.5, out, ws)

    slots.fill_(-1)
    step()                                                   # (a first run outside the capture)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for p in range(start, start + 5):
        x.copy_(_dev(rng.normal(size=tuple(x.shape)), torch.bfloat16))
        for t, v in ((pos, p), (slots, slot_of[p]), (ctx, p)):
            t.fill_(v)
        g.replay()
        torch.cuda.synchronize()
        k, v = ca.rows(np.array(slot_of[:p + 1]))
        want, _, mag = oa.draft_attention(_host(q), k, v, p, [1], D ** -0.5)
        assert (np.abs(_host(out) - want) <= (2.0 ** -7 + 1e-4) * mag).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ctx,n,hq,hkv,D,page", [
    ([20000], [1], 4, 2, 64, 16),                           # some eighty pieces of four rows
    ([3000, 40, 1500], [40, 2, 7], 16, 2, 128, 32),         # a few pieces of some thousand rows
    ([2500] + [3] * 39, [1] * 40, 8, 2, 64, 16),            # a long sequence among many short ones
    ([400], [33], 8, 8, 128, 64),                           # short tables: in one piece
    ([500], [1], 2, 2, 256, 16),
    ([900, 20], [2, 1], 4, 1, 128, 32),
    ([1000] * 40, [1] * 40, 8, 8, 64, 16),
])
def test_sequences_split_into_few_and_many_pieces(dtype, ctx, n, hq, hkv, D, page):
    b = _Batch(np.random.default_rng(len(ctx) + D), "fp8", dtype, ctx, n, hq, hkv, D, page, False)
    got = b.run()
    b.check(got)
    again, _ = b.run()
    np.testing.assert_array_equal(again, got[0])
    b.check(b.run(max_q=64))
