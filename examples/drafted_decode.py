"""Drafted decoding of a few users through a small MoE model on one server.

    python examples/drafted_decode.py [--dtype bf16|f32] [--format int8|fp8] [--tokens N]

Each layer is attention over a quantised paged cache, then the MoE layer:

    cache_write      norms, rotation and the new rows into the cache
    draft_attention  the new tokens over the cache: a chain of a prompt's
                     tokens, one token, or a tree of drafted tokens
    few_moe_layer    the MoE layer for up to 16 tokens (longer chunks of a
                     prompt: route_select, then local_moe_forward)

A step drafts a tree for every user (what followed the latest earlier places of
the user's last token), runs all trees through the model at once and keeps the longest path that
the model itself would have taken, plus the token after it.  The weights are
random; plain decoding, one token a step, gives the same tokens, which the
program checks.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

from paper_2607_17154_amd import ordermoe as om  # noqa: E402

DEV = "cuda"
CLOSE = 0.05          # a greedy choice nearer to a tie may differ between two orders of summation


class Model:
    """`n_layers` layers of hidden size d: n_q / n_kv heads of D, E experts of f (top-k) and one shared expert."""

    def __init__(self, dtype="bf16", vocab=64, n_layers=2, d=512, n_q=4, n_kv=2, D=128, E=16, f=256, k=2, max_pos=4096, seed=0):
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.code = om.BF16 if dtype == "bf16" else om.F32
        self.d, self.n_q, self.n_kv, self.D, self.E, self.k, self.vocab = d, n_q, n_kv, D, E, k, vocab
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)

        def rand(*shape):
            return (torch.randn(shape, generator=g, device=DEV) * shape[-1] ** -0.5).to(self.dtype)

        self.embed = rand(vocab, d) * d ** 0.5
        self.head = rand(vocab, d) * 4
        self.cos_sin = torch.from_numpy(om.rotary_table(max_pos, D)).to(DEV)
        # every expert is deployed on the one server, so that nothing is sent anywhere
        self.tables = dict(t1_k=torch.full((E, 1), -1, dtype=torch.int32, device=DEV),
                           t1_q=torch.zeros((E, 1), device=DEV), t1_n=torch.zeros(E, dtype=torch.int32, device=DEV),
                           srvmask=torch.ones(E, dtype=torch.int32, device=DEV), S=torch.zeros((1, 1, E), device=DEV))
        self.layers = []
        for _ in range(n_layers):
            w = dict(qkv=rand((n_q + 2 * n_kv) * D, d), o=rand(d, n_q * D), router=rand(E, d) * 4,
                     q_norm=torch.ones(D, dtype=self.dtype, device=DEV), k_norm=torch.ones(D, dtype=self.dtype, device=DEV))
            for name, n in (("", E), ("sh_", 1)):
                w[name + "gu"], w[name + "dn"] = rand(n, 2 * f, d), rand(n, d, f)
                om.ordermoe_pack_gate_up(rand(n, f, d), rand(n, f, d), w[name + "gu"])
                om.ordermoe_pack_down(rand(n, d, f), w[name + "dn"])
            w["heads"] = om.make_heads(self.code, n_q, D, w["q_norm"], w["k_norm"], self.cos_sin)
            w["layer"] = om.make_layer(self.code, d, E, k, 1, 1, w["router"], self.tables, 0.0, 0.5)
            w["experts"] = om.make_experts(self.code, d, f, E, np.arange(E, dtype=np.int32), w["gu"], w["dn"], 1, w["sh_gu"],
                                           w["sh_dn"])
            self.layers.append(w)

    def moe(self, w, x):
        T = x.shape[0]
        loc, qhat = torch.zeros(T, dtype=torch.uint8, device=DEV), torch.zeros(T, device=DEV)
        out, y = om.alloc_route_out(T, self.k, 1, DEV), torch.empty_like(x)
        if T <= om.MAX_FEW:
            ws = torch.empty(om.ordermoe_few_workspace_size(w["layer"], w["experts"], T), dtype=torch.uint8, device=DEV)
            om.ordermoe_few_moe_layer(w["layer"], w["experts"], x, T, loc, qhat, 0, out, y, ws)
            return y
        ws = torch.empty(om.ordermoe_route_workspace_size(T, self.k, 1), dtype=torch.uint8, device=DEV)
        om.ordermoe_route_select(w["layer"], x, T, loc, qhat, out, ws)
        rows = torch.empty(self.E + 2, dtype=torch.int32, device=DEV)
        ws = torch.empty(om.ordermoe_forward_workspace_size(w["experts"], T, self.k), dtype=torch.uint8, device=DEV)
        om.ordermoe_local_moe_forward(w["experts"], x, T, self.k, out["w"], out["exec_k"], out["exec_m"], loc, 0, y, rows, ws)
        return y


def _norm(x):
    return torch.nn.functional.rms_norm(x, x.shape[-1:], eps=1e-6)


class Session:
    """Users' sequences and their caches, one cache per layer over one page table."""

    def __init__(self, model: Model, users: int, fmt: str, max_len: int, page: int = 16):
        self.m, self.page = model, page
        pages = -(-max_len // page)
        rng = np.random.RandomState(0)
        self.table = rng.permutation(users * pages).astype(np.int32).reshape(users, pages)
        self.table_dev = torch.from_numpy(self.table).to(DEV)
        self.caches = [om.alloc_cache(om.CACHE_INT8 if fmt == "int8" else om.CACHE_FP8, users * pages, model.n_kv, page, model.D, DEV)
                       for _ in model.layers]
        self.len = np.zeros(users, np.int64)            # tokens of each user in the cache

    def slots(self, user, pos):
        return self.table[user, pos // self.page].astype(np.int64) * self.page + pos % self.page

    def forward(self, tokens, depths=None, words=None):
        """Logits (float32, on the host) of new tokens after the users' cached ones: `tokens` a list per user.
        Trees: `depths` their depths below the context, `words` which tokens each sees."""
        m, n = self.m, [len(t) for t in tokens]
        depths = depths or [list(range(c)) for c in n]
        pos = np.concatenate([self.len[u] + np.asarray(depths[u], np.int64) for u in range(len(n))])
        slots = np.concatenate([self.slots(u, self.len[u] + np.arange(n[u])) for u in range(len(n))])
        dev = lambda a, t: torch.from_numpy(np.asarray(a).astype(t)).to(DEV)  # noqa: E731
        pos, slots, start, ctx = (dev(pos, np.int32), dev(slots, np.int64), dev(np.concatenate([[0], np.cumsum(n)]), np.int32),
                                  dev(self.len, np.int32))
        tree = dev(np.array([w for ws in words for w in ws], np.uint64).view(np.int64), np.int64) if words else None
        T, max_q = sum(n), max(n)
        x = m.embed[dev([t for ts in tokens for t in ts], np.int64)]
        q_out = torch.empty((T, m.n_q, m.D), dtype=m.dtype, device=DEV)
        attended = torch.empty_like(q_out)
        for w, cache in zip(m.layers, self.caches):
            qkv = (_norm(x) @ w["qkv"].t()).view(T, m.n_q + 2 * m.n_kv, m.D)
            om.ordermoe_cache_write(cache, w["heads"], *qkv.split([m.n_q, m.n_kv, m.n_kv], 1), pos, slots, q_out)
            ws = torch.empty(om.ordermoe_draft_attention_workspace_size(cache, m.code, m.n_q, len(n), max_q), dtype=torch.uint8,
                             device=DEV)
            om.ordermoe_draft_attention(cache, q_out, start, ctx, self.table_dev, max_q, m.D ** -0.5, attended, ws, tree=tree)
            x = x + attended.view(T, -1) @ w["o"].t()
            x = x + m.moe(w, _norm(x).contiguous())
        return (_norm(x) @ m.head.t()).float().cpu().numpy()

    def prompt(self, prompts):
        """Logits of each user's last prompt token; chunks of MAX_DRAFT tokens, a user at a time."""
        last = []
        for u, p in enumerate(prompts):
            for at in range(0, len(p), om.MAX_DRAFT):
                part = p[at:at + om.MAX_DRAFT]
                out = self.forward([part if v == u else [] for v in range(len(prompts))])
                self.len[u] += len(part)
            last.append(out[-1])
        return last

    def keep(self, user, path):
        """The accepted drafted tokens move up to follow the context; the rest is given up."""
        src, dst = (self.slots(user, self.len[user] + np.asarray(p, np.int64)) for p in (path, range(len(path))))
        (sp, so), (dp, do) = ((torch.from_numpy(s // self.page).to(DEV), torch.from_numpy(s % self.page).to(DEV)) for s in (src, dst))
        for cache in self.caches:
            for t in cache._tensors:
                t[dp, :, do] = t[sp, :, so]
        self.len[user] += len(path)


def draft(history, branches=3, length=4):
    """A tree below the last token of `history`: (tokens, parents); parent -1 is the context.  The root is the token
    to come, known already; the branches are what followed the latest earlier places of that token."""
    tokens, parents = [history[-1]], [-1]
    places = [i for i in range(len(history) - 2, -1, -1) if history[i] == history[-1]][:branches]
    for i in places:
        at = 0
        for t in history[i + 1:i + 1 + length]:
            known = [j for j, p in enumerate(parents) if p == at and tokens[j] == t]
            if known:
                at = known[0]
                continue
            tokens.append(t)
            parents.append(at)
            at = len(tokens) - 1
    return tokens, parents


def drafted(model, prompts, n_tokens, fmt):
    """(tokens, gap of the two largest logits at each) of every user, and the steps taken."""
    s = Session(model, len(prompts), fmt, max(map(len, prompts)) + n_tokens + 64)
    texts = [list(p) for p in prompts]
    gaps = [[] for _ in prompts]

    def take(u, logits):
        top = np.sort(logits)
        texts[u].append(int(logits.argmax()))
        gaps[u].append(float(top[-1] - top[-2]))

    for u, logits in enumerate(s.prompt(prompts)):
        take(u, logits)
    steps = 0
    while min(len(t) - len(p) for t, p in zip(texts, prompts)) < n_tokens:
        # a user that has its tokens drafts no more: its row of the page table ends soon after them
        trees = [draft(t) if len(t) - len(p) < n_tokens else ([], []) for t, p in zip(texts, prompts)]
        depths, words = [], []
        for tokens, parents in trees:
            d, w = [], []
            for i, p in enumerate(parents):
                d.append(d[p] + 1 if p >= 0 else 0)
                w.append((w[p] if p >= 0 else 0) | 1 << i)
            depths.append(d)
            words.append(w)
        logits = s.forward([t for t, _ in trees], depths, words)
        first = 0
        for u, (tokens, parents) in enumerate(trees):
            if not tokens:
                continue
            path = [0]
            while True:
                take(u, logits[first + path[-1]])
                nxt = [j for j, p in enumerate(parents) if p == path[-1] and tokens[j] == texts[u][-1]]
                if not nxt:
                    break
                path.append(nxt[0])
            s.keep(u, path)
            first += len(tokens)
        steps += 1
    return [(t[len(p):][:n_tokens], g[:n_tokens]) for t, p, g in zip(texts, prompts, gaps)], steps


def plain(model, prompts, n_tokens, fmt):
    """The same, one token of every user a step."""
    s = Session(model, len(prompts), fmt, max(map(len, prompts)) + n_tokens + 64)
    logits, out = s.prompt(prompts), [([], []) for _ in prompts]
    for i in range(n_tokens):
        for (tokens, gaps), x in zip(out, logits):
            top = np.sort(x)
            tokens.append(int(x.argmax()))
            gaps.append(float(top[-1] - top[-2]))
        if i + 1 < n_tokens:
            logits = s.forward([[t[-1]] for t, _ in out])
            s.len += 1
    return out


def agree(a, b):
    """Tokens that two decodings share; False at a difference that is no near tie."""
    n = 0
    for (ta, ga), (tb, gb) in zip(a, b):
        for x, y, g, h in zip(ta, tb, ga, gb):
            if x != y:
                if min(g, h) > CLOSE:
                    return False, n
                break
            n += 1
    return True, n


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--dtype", choices=["bf16", "f32"], default="bf16")
    ap.add_argument("--format", choices=["int8", "fp8"], default="int8")
    ap.add_argument("--tokens", type=int, default=48, help="tokens to decode for each user")
    a = ap.parse_args(argv)
    model = Model(a.dtype)
    rng = np.random.RandomState(1)
    prompts = [list(map(int, np.tile(rng.randint(0, model.vocab, 7), 20)[:n])) for n in (5, 100, 37)]
    got, steps = drafted(model, prompts, a.tokens, a.format)
    want = plain(model, prompts, a.tokens, a.format)
    ok, same = agree(got, want)
    for u, (t, _) in enumerate(got):
        print("user %d (%d tokens of prompt): %s" % (u, len(prompts[u]), " ".join(map(str, t))))
    print("%d steps for %d tokens of each user; %d of %d tokens as in plain decoding%s" % (
        steps, a.tokens, same, a.tokens * len(prompts), "" if ok else ", which differs clear of a tie"))
    return 0 if ok else 1


if __name__ == "__main__":
    sys.exit(main())
