"""The example's drafts: what followed earlier places of the last token, as a tree."""
import os
import sys

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))
import drafted_decode as dd  # noqa: E402


def test_branches_share_their_beginnings():
    tokens, parents = dd.draft([7, 1, 2, 3, 7, 1, 5, 7])
    assert tokens == [7, 1, 5, 7, 2, 3, 7] or tokens == [7, 1, 5, 7, 2, 3]
    assert parents[:4] == [-1, 0, 1, 2] and parents[4:6] == [1, 4]


def test_a_token_without_history_stands_alone():
    assert dd.draft([1, 2, 3]) == ([3], [-1])


def test_agreement_stops_at_a_near_tie_only():
    a, b = [([1, 2, 3], [1.0, 1.0, 1.0])], [([1, 4, 3], [1.0, 0.01, 1.0])]
    assert dd.agree(a, a) == (True, 3)
    assert dd.agree(a, b) == (True, 1)
    assert dd.agree(a, [([1, 4, 3], [1.0, 1.0, 1.0])]) == (False, 1)
