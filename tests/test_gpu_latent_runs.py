"""The latent cache's operators together, as a server runs them: prompts, steps, evictions; in
graphs, on streams beside one another, and in caches past 32-bit offsets.

Tolerances as in test_gpu_latent.  Where the expanded and the absorbed way meet, one formula from the queries
and the cached rows is the measure of both; bf16 keys, values and absorbed queries are rounded once on
the way (2^-8 of their value at most): scores are off by up to 2^-8 of their products' magnitudes, e, weights
by 2 e, values by 2^-8."""
import numpy as np
import pytest

from oracle import latent as ol
from tests.test_gpu_latent import DT, HALF, U, _Batch, _dev, _host, _prompt, _run_prompt, _weights, _within, om, torch

pytestmark = pytest.mark.gpu


class _Server:
    """B sequences of one layer: cache, weights and what a step needs, on the device."""

    def __init__(self, seed, dtype, B=3, h=4, D=64, R=128, rot=32, page=16, places=160, keep=40):
        rng = self.rng = np.random.default_rng(seed)
        self.dtype, self.B, self.h, self.D, self.R, self.rot, self.page, self.keep = dtype, B, h, D, R, rot, page, keep
        self.stride, self.pages = places, places // page
        order = rng.permutation(B * self.pages + 2)[:B * self.pages]
        self.table = order.reshape(B, self.pages).astype(np.int32)
        d = DT[dtype]
        self.rows = torch.zeros((B * self.pages + 2, page, R + rot), dtype=d, device="cuda")
        self.cache = om.make_latent_cache(self.rows, R)
        self.angles = om.rotary_table(1000, rot)
        self.wk, self.wv = _weights(rng, h, D, R, dtype)
        self.norm = _dev(1 + 0.1 * rng.normal(size=R), d)
        self.heads = om.make_latent_heads(self.cache, self.wk, self.wv, self.norm, _dev(self.angles), 1)
        self.d_table = _dev(self.table)
        self.scale = (D + rot) ** -0.5
        self.mass = torch.zeros((B, places), device="cuda")
        self.pos = torch.zeros((B, places), dtype=torch.int32, device="cuda")
        self.ctx = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.kept = torch.zeros((B, keep), dtype=torch.int32, device="cuda")
        self.ws = torch.full((max(om.ordermoe_latent_attention_workspace_size(self.cache, self.heads, B, 1, self.pages, 1),
                                  om.ordermoe_latent_evict_workspace_size(self.cache, B, self.pages, keep)),),
                             0x7F, dtype=torch.uint8, device="cuda")

    def slot(self, b, p):
        return self.table[b, p // self.page].astype(np.int64) * self.page + p % self.page

    def tokens(self, T):
        d = DT[self.dtype]
        return (_dev(2 * self.rng.normal(size=(T, self.h, self.D + self.rot)), d), _dev(self.rng.normal(size=(T, self.R + self.rot)), d))

    def cached(self, b, n):
        return _host(self.rows.flatten(0, 1)[_dev(self.slot(b, np.arange(n)))])

    def step(self, q, kv, at, slots, starts, qa, out, lse):
        """One token of each sequence, then the eviction."""
        om.ordermoe_latent_write(self.cache, self.heads, q, kv, at, slots, qa, 1)
        om.ordermoe_latent_attention(self.cache, self.heads, qa, starts, self.ctx, self.d_table, 1, self.scale, out, self.ws, lse=lse,
                                     mass=self.mass, mass_out=self.mass, decay=0.9)

    def evict(self, seq):
        om.ordermoe_latent_evict(self.cache, self.ctx, seq, self.d_table, self.keep, 2, 8, self.mass, self.pos, self.kept, self.ctx,
                                 self.mass, self.pos, self.ws)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompts_steps_and_evictions(dtype):
    s = _Server(1, dtype)
    n = np.array([50, 17, 64])
    T, qs = int(n.sum()), np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    q, kv = s.tokens(T)
    at = np.concatenate([np.arange(c) for c in n]).astype(np.int32)
    slots = np.concatenate([s.slot(b, np.arange(c)) for b, c in enumerate(n)])
    d = DT[dtype]
    qp = torch.empty((T, s.h, s.D + s.rot), dtype=d, device="cuda")
    qa = torch.empty((T, s.h, s.R + s.rot), dtype=d, device="cuda")
    om.ordermoe_latent_write(s.cache, s.heads, q, kv, _dev(at), _dev(slots), qp, 0)
    first = s.rows.clone()
    om.ordermoe_latent_write(s.cache, s.heads, q, kv, _dev(at), _dev(slots), qa, 1)
    assert torch.equal(first, s.rows) and torch.equal(qp[..., s.D:], qa[..., s.R:])
    # both ways over the same rows
    k, v = (torch.empty((T, s.h, s.D), dtype=d, device="cuda") for _ in range(2))
    r = torch.empty((T, s.rot), dtype=d, device="cuda")
    om.ordermoe_latent_expand(s.cache, s.heads, _dev(slots), k, r, v)
    p = dict(q=qp, k=k, v=v, r=r, qs=qs, ks=qs, scale=s.scale, dtype=dtype)
    o1, l1 = _run_prompt(p)
    o2, l2 = torch.empty_like(o1), torch.empty_like(l1)
    ws = torch.empty(om.ordermoe_latent_attention_workspace_size(s.cache, s.heads, s.B, 64, s.pages), dtype=torch.uint8, device="cuda")
    om.ordermoe_latent_attention(s.cache, s.heads, qa, _dev(qs), s.ctx, s.d_table, 64, s.scale, o2, ws, lse=l2)
    step = 2.0 ** -8 if dtype == "bf16" else 0.0
    for b in range(s.B):
        t, c = slice(qs[b], qs[b + 1]), s.cached(b, n[b])
        keys, values = ol.expanded(c[:, :s.R], _host(s.wk))[0], ol.expanded(c[:, :s.R], _host(s.wv))[0]
        e = ol.prompt_attention(_host(qp)[t], keys, values, c[:, s.R:], s.scale)
        qabs, qsize = ol.absorbed(_host(qp)[t], _host(s.wk), None, at[t], True)
        qabs = np.maximum(np.abs(qabs), qsize)               # magnitudes on either way, the larger ones
        es = (step + (s.D + s.R + s.rot + 8) * U) * s.scale * np.einsum("nhr,pr->nhp", qabs, np.abs(c)).max()
        ew = 2 * es + step + (8 + n[b]) * U
        size = np.broadcast_to(ol.expanded(np.abs(c[:, :s.R]), np.abs(_host(s.wv)))[0].max(0)[None], e["out"].shape)
        for o, ls in ((o1, l1), (o2, l2)):
            _within(_host(o)[t], e["out"], (ew + step + (s.R + 8) * U) * size + HALF[dtype] * np.abs(e["out"]), "out of %d" % b)
            _within(_host(ls)[t], e["lse"], es + (8 + n[b]) * U + 2 * U * np.abs(e["lse"]), "lse of %d" % b)
    # steps, an eviction after every third
    s.ctx.copy_(_dev(n.astype(np.int32)))
    for b in range(s.B):
        s.pos[b, :n[b]] = torch.arange(int(n[b]), dtype=torch.int32, device="cuda")
        s.mass[b, :n[b]] = torch.rand(int(n[b]), device="cuda")
    ctx, seq = n.copy(), n.copy()
    starts = _dev(np.arange(s.B + 1, dtype=np.int32))
    out = torch.empty((s.B, s.h, s.D), dtype=d, device="cuda")
    lse = torch.empty((s.B, s.h), device="cuda")
    qa = torch.empty((s.B, s.h, s.R + s.rot), dtype=d, device="cuda")
    for i in range(7):
        q, kv = s.tokens(s.B)
        slots = np.array([s.slot(b, ctx[b]) for b in range(s.B)])
        was = _host(s.mass)
        s.step(q, kv, _dev(seq.astype(np.int32)), _dev(slots), starts, qa, out, lse)
        for b in range(s.B):
            c, L = s.cached(b, ctx[b] + 1), int(ctx[b]) + 1
            e = ol.latent_attention(_host(qa)[b:b + 1], c, np.ones((1, L), bool), _host(s.wv), s.scale)
            es = e["score"] * (s.R + s.rot + 4) * U
            ew = 2 * es + (8 + L) * U + (2.0 ** -16 if dtype == "bf16" else 0)
            _within(_host(out)[b:b + 1], e["out"], ew * e["size"] + (2.0 ** -16 + (s.R + 1) * U) * e["through"] + HALF[dtype] * np.abs(e["out"]),
                    "out of %d, step %d" % (b, i))
            want = e["mass"] + np.concatenate([0.9 * was[b, :L - 1], [0.0]])
            _within(_host(s.mass)[b, :L], want, (2 * es + (8 + L + s.h) * U) * e["mass"] + 4 * U * want + s.h * 2.0 ** -126, "mass")
            s.pos[b, int(ctx[b])] = int(seq[b])
        s.ctx += 1
        ctx, seq = ctx + 1, seq + 1
        if i % 3 == 2:
            mass, pos, rows = _host(s.mass), _host(s.pos), [s.cached(b, ctx[b]) for b in range(s.B)]
            s.evict(_dev(seq.astype(np.int32)))
            for b in range(s.B):
                kept = ol.evict(int(ctx[b]), int(seq[b]), s.keep, 2, 8, mass[b], pos[b])
                np.testing.assert_array_equal(_host(s.kept)[b], kept)
                ctx[b] = min(ctx[b], s.keep)
                np.testing.assert_array_equal(s.cached(b, ctx[b]), rows[b][kept[:ctx[b]]])
            np.testing.assert_array_equal(_host(s.ctx), ctx)


def test_a_captured_step_goes_on_as_an_eager_one():
    """Write, attention with weights and eviction in one graph, replayed over a state that changes, with eager
    work between the replays: the same bits as the eager calls."""
    a, b = _Server(2, "bf16", keep=24), _Server(2, "bf16", keep=24)
    rng = np.random.default_rng(3)
    fixed = []
    for s in (a, b):
        s.ctx.fill_(24)
        s.pos[:, :24] = torch.arange(24, dtype=torch.int32, device="cuda")
        fixed.append(dict(q=torch.empty((s.B, s.h, s.D + s.rot), dtype=torch.bfloat16, device="cuda"),
                          kv=torch.empty((s.B, s.R + s.rot), dtype=torch.bfloat16, device="cuda"),
                          at=torch.full((s.B,), 24, dtype=torch.int32, device="cuda"),
                          slots=_dev(np.array([s.slot(i, 24) for i in range(s.B)])), starts=_dev(np.arange(s.B + 1, dtype=np.int32)),
                          qa=torch.zeros((s.B, s.h, s.R + s.rot), dtype=torch.bfloat16, device="cuda"),
                          out=torch.zeros((s.B, s.h, s.D), dtype=torch.bfloat16, device="cuda"), lse=torch.zeros((s.B, s.h), device="cuda")))
    start = rng.normal(size=(a.B, 24, a.R + a.rot))
    for s in (a, b):
        for i in range(s.B):
            s.rows.flatten(0, 1)[_dev(s.slot(i, np.arange(24)))] = _dev(start[i], torch.bfloat16)

    def run(s, f):
        s.step(**f)
        s.pos[:, 24] = f["at"]
        s.ctx += 1
        f["at"] += 1
        s.evict(f["at"])

    def feed(f, i):
        g = np.random.default_rng(100 + i)
        f["q"].copy_(_dev(2 * g.normal(size=f["q"].shape), torch.bfloat16))
        f["kv"].copy_(_dev(g.normal(size=f["kv"].shape), torch.bfloat16))

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for s, f in ((a, fixed[0]), (b, fixed[1])):          # an eager step of both first
            feed(f, 0)
            run(s, f)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(a, fixed[0])
    for i in range(1, 7):
        for f in fixed:
            feed(f, i)
        graph.replay()
        run(b, fixed[1])
        torch.cuda.synchronize()
        for x, y in ((a.rows, b.rows), (a.mass[:, :24], b.mass[:, :24]), (a.pos[:, :24], b.pos[:, :24]), (a.ctx, b.ctx), (a.kept, b.kept),
                     (fixed[0]["out"], fixed[1]["out"]), (fixed[0]["lse"], fixed[1]["lse"]), (fixed[0]["qa"], fixed[1]["qa"])):
            assert torch.equal(x, y), i


def test_calls_beside_one_another():
    """Each operator on two streams at once, each call with its own workspace, beside other work: the same bits as alone."""
    rng = np.random.default_rng(4)
    batches = [_Batch(rng, "bf16", [3000, 40, 900], [m, 1, m], 16, 64, 256, 32, 16) for m in (1, 20)]
    prompts = [_prompt(rng, "bf16", [40, 3], [1500, 2100], 4, 2, 128, 0), _prompt(rng, "bf16", [700, 200], [0, 100], 8, 8, 128, 64)]
    wk, wv = batches[0].wk, batches[0].wv

    def all_of(i):
        ba, m = batches[i], (1, 20)[i]
        o = list(ba.run(m, stride=3100)) + list(_run_prompt(prompts[i]))
        slots = _dev(np.arange(4000 + 300 * i, dtype=np.int64) % (ba.rows.shape[0] * ba.page - 16))
        k, v = (torch.empty((slots.numel(), 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        r = torch.empty((slots.numel(), 32), dtype=torch.bfloat16, device="cuda")
        om.ordermoe_latent_expand(ba.cache, om.make_latent_heads(ba.cache, wk, wv), slots, k, r, v)
        return o + [k, v, r]

    want = [all_of(0), all_of(1)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = [None, None]
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                got[i] = all_of(i)
        torch.cuda.synchronize()
        for x, y in zip(want[0] + want[1], got[0] + got[1]):
            assert torch.equal(x.nan_to_num(9), y.nan_to_num(9))


def test_a_captured_prompt_in_pieces():
    rng = np.random.default_rng(5)
    p = _prompt(rng, "bf16", [16, 2], [2500, 700], 8, 2, 128, 0)
    want = _run_prompt(p)
    out, lse = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    qs, ks = _dev(p["qs"]), _dev(p["ks"])
    ws = torch.zeros(om.ordermoe_prompt_attention_workspace_size(om.BF16, 8, 2, 128, 0, 20, 2), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        om.ordermoe_prompt_attention(p["q"], p["k"], p["v"], qs, ks, p["scale"], out, ws, lse=lse)
    for i in range(3):
        out.fill_(7.0)
        lse.fill_(7.0)
        ws.fill_(0x7F)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        assert torch.equal(_run_prompt(p)[0], want[0])


def test_a_cache_past_32_bit_offsets():
    """4.6 GB of rows, the last pages in use: written, attended to, expanded, evicted."""
    rng = np.random.default_rng(6)
    h, D, R, rot, page, L = 2, 64, 512, 64, 1024, 1500
    pages = 4000
    rows = torch.empty((pages, page, R + rot), dtype=torch.bfloat16, device="cuda")
    cache = om.make_latent_cache(rows, R)
    wk, wv = _weights(rng, h, D, R, "bf16")
    heads = om.make_latent_heads(cache, wk, wv)
    table = np.array([[pages - 1, pages - 3]], np.int32)
    place = np.arange(L)
    slots = table[0, place // page].astype(np.int64) * page + place % page
    kv = _dev(rng.normal(size=(L, R + rot)), torch.bfloat16)
    om.ordermoe_latent_write(cache, heads, None, kv, None, _dev(slots), None, 0)
    assert torch.equal(rows.flatten(0, 1)[_dev(slots)], kv)
    q = _dev(rng.normal(size=(1, h, R + rot)), torch.bfloat16)
    out = torch.empty((1, h, D), dtype=torch.bfloat16, device="cuda")
    mass = torch.zeros((1, L), device="cuda")
    ws = torch.empty(om.ordermoe_latent_attention_workspace_size(cache, heads, 1, 1, 2, 1), dtype=torch.uint8, device="cuda")
    one = lambda *a: _dev(np.array(a, np.int32))  # noqa: E731
    om.ordermoe_latent_attention(cache, heads, q, one(0, 1), one(L - 1), _dev(table), 1, 0.05, out, ws, mass_out=mass)
    e = ol.latent_attention(_host(q), _host(kv), np.ones((1, L), bool), _host(wv), 0.05)
    ew = 2 * e["score"] * (R + rot + 4) * U + (8 + L) * U + 2.0 ** -16
    _within(_host(out), e["out"], ew * e["size"] + (2.0 ** -16 + (R + 1) * U) * e["through"] + 2.0 ** -8 * np.abs(e["out"]), "out")
    k, v = (torch.empty((L, h, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    r = torch.empty((L, rot), dtype=torch.bfloat16, device="cuda")
    om.ordermoe_latent_expand(cache, heads, _dev(slots), k, r, v)
    assert torch.equal(r, kv[:, R:])
    want, size = ol.expanded(_host(kv)[:, :R], _host(wv))
    _within(_host(v), want, (R + 1) * U * size + 2.0 ** -8 * np.abs(want), "values")
    keep = 1100
    kept = torch.empty((1, keep), dtype=torch.int32, device="cuda")
    pos = _dev(place.astype(np.int32)[None])
    ln, m2, p2 = one(0), torch.zeros_like(mass), torch.zeros_like(pos)
    ws = torch.empty(om.ordermoe_latent_evict_workspace_size(cache, 1, 2, keep), dtype=torch.uint8, device="cuda")
    om.ordermoe_latent_evict(cache, one(L), one(L), _dev(table), keep, 4, 100, mass, pos, kept, ln, m2, p2, ws)
    moved = ol.evict(L, L, keep, 4, 100, _host(mass)[0], place)
    np.testing.assert_array_equal(_host(kept)[0], moved)
    assert torch.equal(rows.flatten(0, 1)[_dev(slots[:keep])], kv[_dev(moved)])


def test_keys_and_values_past_32_bit_offsets():
    rng = np.random.default_rng(7)
    L, g, D, n, n0 = 280000, 64, 128, 70, 300
    k, v = (torch.empty((L, g, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for x in (k, v):
        x[L - n0:] = _dev(rng.normal(size=(n0, g, D)), torch.bfloat16)
    q = _dev(rng.normal(size=(n, g, D)), torch.bfloat16)
    out, lse = torch.empty((n, g, D), dtype=torch.bfloat16, device="cuda"), torch.empty((n, g), device="cuda")
    ws = torch.empty(om.ordermoe_prompt_attention_workspace_size(om.BF16, g, g, D, 0, n, 1), dtype=torch.uint8, device="cuda")
    one = lambda *a: _dev(np.array(a, np.int32))  # noqa: E731
    om.ordermoe_prompt_attention(q, k, v, one(0, n), one(L - n0, L), 0.09, out, ws, lse=lse)
    e = ol.prompt_attention(_host(q), _host(k[L - n0:]), _host(v[L - n0:]), None, 0.09)
    ew = 2 * e["score"] * (D + 4) * U + (8 + n0) * U + 2.0 ** -8
    _within(_host(out), e["out"], ew * e["size"] + (2.0 ** -8 + 2 * U) * np.abs(e["out"]), "out")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,h,g,rot", [(150, 4, 4, 32), (100, 2, 1, 0), (70, 40, 5, 0)])
def test_many_prompts_with_gaps_between_them(dtype, B, h, g, rot):
    """More sequences than a wave looks through at a time, in one piece and in several; tokens before the first."""
    rng = np.random.default_rng(B)
    n = rng.integers(0, 9, B)
    n[rng.integers(0, B, 5)] = 0
    n[B // 2] = 140
    p = _prompt(rng, dtype, n, rng.integers(0, 40, B), h, g, 64, rot)
    d = DT[dtype]
    # the same sequences, five tokens and seven positions later
    ahead = lambda x, c: torch.cat([torch.full((c,) + x.shape[1:], float("nan"), dtype=d, device="cuda"), x])  # noqa: E731
    want = _run_prompt(p)
    later = dict(p, q=ahead(p["q"], 5), k=ahead(p["k"], 7), v=ahead(p["v"], 7), r=None if p["r"] is None else ahead(p["r"], 7),
                 qs=p["qs"] + 5, ks=p["ks"] + 7)
    got = _run_prompt(later)
    for x, y in zip(want, got):
        assert torch.equal(x, y[5:]) and (y[:5] == 7).all()
    q, k, v, r = (None if p[c] is None else _host(p[c]) for c in "qkvr")
    qs, ks = p["qs"], p["ks"]
    for b in range(B):
        t, kk = slice(qs[b], qs[b + 1]), slice(ks[b], ks[b + 1])
        if t.start == t.stop:
            continue
        e = ol.prompt_attention(q[t], k[kk], v[kk], None if r is None else r[kk], p["scale"])
        es = e["score"] * (64 + rot + 4) * U
        ew = 2 * es + (8 + kk.stop - kk.start) * U + (2.0 ** -8 if dtype == "bf16" else 0)
        _within(_host(want[0])[t], e["out"], ew * e["size"] + (2 * U + HALF[dtype]) * np.abs(e["out"]), "out of %d" % b)


def test_prompts_without_positions_and_a_scale_of_nothing():
    rng = np.random.default_rng(8)
    p = _prompt(rng, "bf16", [3, 70], [-3, -70], 4, 2, 64, 0)
    p["k"], p["v"] = p["k"][:0], p["v"][:0]
    out, lse = _run_prompt(p)
    assert (out[:73] == 0).all() and torch.isneginf(lse[:73]).all() and (out[73:] == 7).all()
    p = _prompt(rng, "f32", [5, 66], [2, 0], 2, 2, 64, 32)
    p["scale"] = 0.0                                         # the mean of what a token sees
    out, lse = _run_prompt(p)
    v = _host(p["v"])
    for t, (lo, seen) in {0: (0, 3), 4: (0, 7), 5: (7, 1), 70: (7, 66)}.items():
        some = v[lo:lo + seen]
        _within(_host(out)[t], some.mean(0), (8 + seen) * U * np.abs(some).mean(0), "mean of %d" % seen)
        _within(_host(lse)[t], np.full(2, np.log(seen)), (8 + seen) * U * (1 + np.log(seen)), "lse")


def test_a_thousand_short_sequences():
    rng = np.random.default_rng(9)
    n = rng.integers(0, 3, 1000)
    ba = _Batch(rng, "bf16", rng.integers(0, 40, 1000), n, 4, 64, 128, 32, 16)
    got = ba.run(2, stride=50)
    ba.check(got, 2)
    stays = _host(got[2])[n == 0]                            # entries of sequences without tokens
    assert (stays == 7).all()


def test_evictions_of_few_and_of_many_rows_and_one_after_another():
    """Tables whose rows move in the kernel that finds them, or in one of their own; the second cut starts from the first."""
    rng = np.random.default_rng(10)
    for places, keep, first, recent in ((288, 40, 4, 8), (288, 30, 30, 0), (320, 200, 0, 200), (16, 15, 0, 0), (544, 280, 3, 7)):
        s = _Server(11, "bf16", B=5, places=places, keep=keep)
        n = np.array([0, places, keep, min(places, keep + 1), places - 3])
        s.ctx.copy_(_dev(n.astype(np.int32)))
        s.rows.copy_(_dev(rng.normal(size=s.rows.shape), torch.bfloat16))
        s.mass.copy_(_dev(np.round(rng.random((5, places)) * 9) / 4, torch.float32))
        s.pos.copy_(_dev(np.stack([rng.permutation(places) for _ in range(5)]).astype(np.int32)))
        seq, ctx = np.full(5, places), n
        for cut in (keep, max(1, keep // 2)):
            f, r = min(first, cut), min(recent, cut - min(first, cut))
            mass, pos, rows = _host(s.mass), _host(s.pos), [s.cached(b, ctx[b]) for b in range(5)]
            kept = torch.full((5, cut), 99, dtype=torch.int32, device="cuda")
            ws = torch.full((om.ordermoe_latent_evict_workspace_size(s.cache, 5, s.pages, cut),), 0x7F, dtype=torch.uint8, device="cuda")
            om.ordermoe_latent_evict(s.cache, s.ctx, _dev(seq.astype(np.int32)), s.d_table, cut, f, r, s.mass, s.pos, kept, s.ctx, s.mass,
                                     s.pos, ws)
            for b in range(5):
                want = ol.evict(int(ctx[b]), int(seq[b]), cut, f, r, mass[b], pos[b])
                np.testing.assert_array_equal(_host(kept)[b], want)
                new = min(int(ctx[b]), cut)
                np.testing.assert_array_equal(s.cached(b, new), rows[b][want[:new]])
                np.testing.assert_array_equal(_host(s.mass)[b, :new], mass[b][want[:new]])
                np.testing.assert_array_equal(_host(s.pos)[b, :new], pos[b][want[:new]])
            ctx = np.minimum(ctx, cut)
            np.testing.assert_array_equal(_host(s.ctx), ctx)


@pytest.mark.parametrize("n,h,D,R", [(4400, 120, 64, 128), (6500, 127, 64, 256), (16500, 128, 64, 128), (16640, 64, 128, 512)])
def test_large_expansions(n, h, D, R):
    """Several weight tiles of a workgroup one after the other: all of them whole, the last one not, few tokens in the last tile."""
    rng = np.random.default_rng(n)
    page, rot = 64, 32
    rows = _dev(rng.normal(size=(n // page // 2, page, R + rot)), torch.bfloat16)
    cache = om.make_latent_cache(rows, R)
    wk, wv = _weights(rng, h, D, R, "bf16")
    slots = rng.integers(0, rows.shape[0] * page, n).astype(np.int64)
    slots[[0, 300, n - 1]] = -1
    k, v = (torch.full((n, h, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    r = torch.full((n, rot), 7.0, dtype=torch.bfloat16, device="cuda")
    heads, d_slots = om.make_latent_heads(cache, wk, wv), _dev(slots)
    om.ordermoe_latent_expand(cache, heads, d_slots, k, r, v)
    x = torch.where(d_slots[:, None] >= 0, rows.flatten(0, 1)[d_slots.clamp(min=0)], torch.zeros((), dtype=torch.bfloat16, device="cuda"))
    assert torch.equal(r, x[:, R:])
    x = x[:, :R].float()
    for got, w in ((k, wk), (v, wv)):
        for lo in range(0, h, 32):                           # every output, in fp32 (its own error: as the kernel's sums')
            w32 = w[lo:lo + 32].float().flatten(0, 1).t().contiguous()
            want, size = x @ w32, x.abs() @ w32.abs()
            off = (got[:, lo:lo + 32].flatten(1).float() - want).abs() > 2 * (R + 1) * U * size + 2.0 ** -8 * want.abs()
            assert not off.any(), (lo, int(off.sum()))
    again = [torch.empty_like(t) for t in (k, r, v)]
    for _ in range(3):
        om.ordermoe_latent_expand(cache, heads, d_slots, *again)
        for a, b in zip((k, r, v), again):
            assert torch.equal(a, b)


def test_rows_alone_of_more_tokens_than_one_row_of_the_grid_takes():
    """No queries, and more than 2^22 workgroups: the launch has some that find nothing to do."""
    T, R, rot, page = (1 << 24) + 4, 128, 32, 1024
    pages = -(-T // page)
    kv = torch.empty((T, R + rot), dtype=torch.bfloat16, device="cuda")
    kv.view(torch.int16).random_(0, 0x7000)                  # (finite numbers)
    rows = torch.zeros((pages, page, R + rot), dtype=torch.bfloat16, device="cuda")
    cache = om.make_latent_cache(rows, R)
    wk, wv = _weights(np.random.default_rng(12), 1, 64, R, "bf16")
    slots = torch.arange(T - 1, -1, -1, dtype=torch.int64, device="cuda")
    for absorb in (0, 1):
        rows.zero_()
        om.ordermoe_latent_write(cache, om.make_latent_heads(cache, wk, wv), None, kv, None, slots, None, absorb)
        flat = rows.flatten(0, 1)
        assert torch.equal(flat[:T].view(torch.int16), kv.flip(0).view(torch.int16)) and not flat[T:].view(torch.int16).any()


@pytest.mark.parametrize("places", [160, 8320])              # tables that one kernel goes through, and longer ones
def test_a_budget_of_the_largest_number(places):
    keep = (1 << 31) - 1
    s = _Server(13, "bf16", B=1, places=places, keep=1)
    n = places - 3
    s.ctx.fill_(n)
    s.mass.copy_(_dev(s.rng.random((1, places)), torch.float32))
    rows, mass = s.rows.clone(), s.mass.clone()
    kept = torch.full((1, keep), 99, dtype=torch.int32, device="cuda")
    ws = torch.full((om.ordermoe_latent_evict_workspace_size(s.cache, 1, s.pages, keep),), 0x7F, dtype=torch.uint8, device="cuda")
    om.ordermoe_latent_evict(s.cache, s.ctx, s.ctx.clone(), s.d_table, keep, 5, keep - 5, s.mass, s.pos, kept, s.ctx, s.mass, s.pos, ws)
    assert int(s.ctx) == n and torch.equal(s.rows, rows) and torch.equal(s.mass, mass)
    assert torch.equal(kept[0, :n], torch.arange(n, dtype=torch.int32, device="cuda")) and bool((kept[0, n:] == -1).all())


def _guarded(size):
    """A workspace of this size, and the bytes behind it, which no call may touch."""
    both = torch.full((size + 4096,), 0x7F, dtype=torch.uint8, device="cuda")
    return both[:size], both[size:]


def test_one_workspace_serves_smaller_calls():
    rng = np.random.default_rng(15)
    ba = _Batch(rng, "bf16", [3000, 40, 900, 7], [20, 1, 9, 17], 16, 64, 256, 32, 16)
    ws, behind = _guarded(om.ordermoe_latent_attention_workspace_size(ba.cache, ba.heads, 4, 20, ba.table.shape[1], 1))
    for max_q in (20, 17, 16, 9, 8, 3, 2, 1):
        ws.fill_(0x7F)
        got = ba.run(max_q, stride=3100, ws=ws)
        ba.check(got, max_q)
        for x, y in zip(got, ba.run(max_q, stride=3100)):
            assert torch.equal(x, y)
        ba.run(max_q, ws=ws)
    assert (behind == 0x7F).all()
    h, g, D = 8, 2, 128
    ws, behind = _guarded(om.ordermoe_prompt_attention_workspace_size(om.BF16, h, g, D, 0, 2002, 5))
    for n, ctx in (([2000], [0]), ([600], [100]), ([300, 7], [900, 4000]), ([127], [3000]), ([16, 16, 1], [2500, 1, 700]), ([33], [9000]), ([1], [5000])):
        p = _prompt(rng, "bf16", n, ctx, h, g, D, 0)
        want = _run_prompt(p)
        out, lse = torch.full_like(want[0], 7.0), torch.full_like(want[1], 7.0)
        ws.fill_(0x7F)
        om.ordermoe_prompt_attention(p["q"], p["k"], p["v"], _dev(p["qs"]), _dev(p["ks"]), p["scale"], out, ws, lse=lse)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert (behind == 0x7F).all()
    s = _Server(16, "bf16", B=5, places=9600, keep=1)
    ws, behind = _guarded(om.ordermoe_latent_evict_workspace_size(s.cache, 5, s.pages, 9000))
    for keep in (9000, 5000, 4800, 100):
        n = np.array([9600, 4801, keep, 7000, 9599])
        s.ctx.copy_(_dev(n.astype(np.int32)))
        mass = s.rng.random((5, 9600)).astype(np.float32)
        s.mass.copy_(_dev(mass))
        pos = np.tile(np.arange(9600, dtype=np.int32), (5, 1))
        s.pos.copy_(_dev(pos))
        kept = torch.full((5, keep), 99, dtype=torch.int32, device="cuda")
        ws.fill_(0x7F)
        om.ordermoe_latent_evict(s.cache, s.ctx, _dev(n.astype(np.int32)), s.d_table, keep, 2, 8, s.mass, s.pos, kept, s.ctx, s.mass, s.pos, ws)
        for b in range(5):
            np.testing.assert_array_equal(_host(kept)[b], ol.evict(int(n[b]), int(n[b]), keep, 2, 8, mass[b], pos[b]))
    assert (behind == 0x7F).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,h,max_q", [(20, 8, 1), (64, 8, 1), (17, 32, 3)])
def test_one_long_sequence_among_short_ones(dtype, B, h, max_q):
    """Its pieces are far more than a sequence of the batch has on average."""
    rng = np.random.default_rng(B)
    ctx, n = rng.integers(0, 11, B), rng.integers(1, max_q + 1, B)
    ctx[B // 2], n[B // 2] = 30011, max_q
    ba = _Batch(rng, dtype, ctx, n, h, 64, 128, 32, 64)
    first = ba.run(max_q, stride=100)
    ba.check(first, max_q)
    for _ in range(2):
        for x, y in zip(first, ba.run(max_q, stride=100)):
            assert torch.equal(x, y)
