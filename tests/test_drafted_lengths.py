"""The example's drafted decoding on the host: users whose drafts are taken far more often
than others' stay inside their rows of the page table."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))
import drafted_decode as dd  # noqa: E402

CYCLE = 4


def _follower(token):
    """Tokens below CYCLE go round, every other one is followed by the next number."""
    return (token + 1) % CYCLE if token < CYCLE else token + 1


class _Model:
    layers = ()


def _forward(session, tokens, depths=None, words=None):
    n = [len(t) for t in tokens]
    assert max(n) > 0 and max(n) <= dd.om.MAX_DRAFT
    for u in range(len(n)):
        session.slots(u, session.len[u] + np.arange(n[u]))          # every new token has a place
    flat = [t for ts in tokens for t in ts]
    logits = np.zeros((len(flat), 4096), np.float32)
    logits[np.arange(len(flat)), [_follower(t) for t in flat]] = 1
    return logits


@pytest.mark.parametrize("n_tokens", [1, 2, 5, 48, 200])
def test_users_of_different_speeds(monkeypatch, n_tokens):
    monkeypatch.setattr(dd, "DEV", "cpu")
    monkeypatch.setattr(dd.Session, "forward", _forward)
    prompts = [[i % CYCLE for i in range(100)], [CYCLE + 10, CYCLE + 11, CYCLE + 12], [3]]
    got, steps = dd.drafted(_Model(), prompts, n_tokens, "int8")
    for (tokens, gaps), p in zip(got, prompts):
        want = [_follower(p[-1])]
        while len(want) < n_tokens:
            want.append(_follower(want[-1]))
        assert tokens == want and len(gaps) == n_tokens
    # the user that never repeats itself takes one token a step after its prompt's
    assert steps == n_tokens - 1
