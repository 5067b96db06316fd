"""The bits of a token's weights do not go with how many tokens its neighbours have drafted."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from .test_gpu_cache_attention import _Batch  # noqa: E402


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("ctx,n,hq,hkv,D,page", [
    ([777, 900, 3], [1, 33, 2], 32, 8, 128, 64), ([100, 2600], [4, 64], 8, 2, 64, 16), ([40, 31, 2], [1, 20, 16], 2, 2, 128, 32)])
def test_few_rows_beside_many(fmt, ctx, n, hq, hkv, D, page):
    """Sequences of up to 16 rows a head in a batch with one of more: the output's rounding, 2^-8 of
    it, and of the terms' sum 2^-17 for the weights in two parts and 2^-24 D |score| (|score| < 5)
    for the scores, as without the neighbour."""
    b = _Batch(np.random.default_rng(41), fmt, "bf16", ctx, n, hq, hkv, D, page, False)
    out, _ = b.run()
    want, _, mag = b.want()
    few = np.repeat([m * hq // hkv <= 16 for m in n], n)
    assert few.any() and not few.all()
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -17 + 5 * D * 2.0 ** -24 + 2e-6) * mag
    over = (np.abs(out - want) - tol)[few]
    assert (over <= 0).all(), over.max()
