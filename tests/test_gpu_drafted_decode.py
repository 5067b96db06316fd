"""The drafted-decoding example: the cache, the attention and the MoE layer for a few
tokens together give the tokens that plain decoding gives."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))
import drafted_decode as dd  # noqa: E402


@pytest.mark.parametrize("dtype,fmt", [("bf16", "int8"), ("bf16", "fp8"), ("f32", "int8"), ("f32", "fp8")])
def test_drafted_and_plain_decoding_agree(dtype, fmt):
    model = dd.Model(dtype, seed=3)
    prompts = [[1, 2, 3], [5, 6, 7, 8] * 20, [9], list(range(40, 60))]
    got, steps = dd.drafted(model, prompts, 24, fmt)
    want = dd.plain(model, prompts, 24, fmt)
    ok, same = dd.agree(got, want)
    assert ok and same > 0
    assert all(len(t) == 24 for t, _ in got) and steps <= 23


def test_the_program(capsys):
    assert dd.main(["--tokens", "16"]) == 0
    assert "steps for 16 tokens" in capsys.readouterr().out
