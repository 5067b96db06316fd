"""Drafted places that were never written and that only some tokens of the sequence see."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from .test_gpu_cache_attention import _Batch  # noqa: E402


def _unwritten(b, s, j):
    """Drafted place j of sequence s as memory that nothing was written to may be; who sees it."""
    slot = int(b.slots[s][b.ctx[s] + j])
    for codes, scale in zip(b.ca.codes, b.ca.scale):
        codes[slot // b.ca.page, :, slot % b.ca.page] = 0x7F if j % 2 else 0xFF
        scale[slot // b.ca.page, :, slot % b.ca.page] = float("nan")
    return np.array([(w >> j) & 1 for w in b.words[s]], bool)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("hq,D,tree", [(4, 128, False), (2, 64, True), (8, 256, False), (16, 128, True)])
def test_who_does_not_see_an_unwritten_place_is_not_changed(dtype, fmt, hq, D, tree):
    """The last places of a chain that only pads the batch have no row in the cache; their own
    tokens see them (and are no numbers), the tokens before them do not."""
    rng = np.random.default_rng(31)
    b = _Batch(rng, fmt, dtype, [50, 0, 900], [12, 3, 33], hq, 2, D, 16, tree)
    clean = b.run()
    b.check(clean)
    sees = [np.zeros(m, bool) for m in b.n]
    for s, m in enumerate(b.n):
        for j in range(m - 1 - m // 6, m):
            if tree and b.words[s][j] == 0:
                continue
            sees[s] |= _unwritten(b, s, j)
    sees = np.concatenate(sees)
    assert sees.any() and not sees.all()
    out, lse = b.run()
    np.testing.assert_array_equal(out[~sees], clean[0][~sees])
    np.testing.assert_array_equal(lse[~sees], clean[1][~sees])
    assert np.isnan(out[sees]).all() and np.isnan(lse[sees]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,D", [(4, 128), (2, 64), (8, 256)])
def test_value_codes_that_are_no_numbers(dtype, hq, D):
    """One e4m3 code of a drafted value row that is a NaN, with every scale and key in
    order: only the outputs of the tokens that see it are no numbers, and no lse."""
    b = _Batch(np.random.default_rng(32), "fp8", dtype, [40, 7], [9, 20], hq, 2, D, 16, True)
    clean = b.run()
    t = 0
    for s, m in enumerate(b.n):
        j = next(j for j in range(m) if b.words[s][j] and not all((w >> j) & 1 for w in b.words[s]))
        slot = int(b.slots[s][b.ctx[s] + j])
        b.ca.codes[1][slot // 16, :, slot % 16, 5 + 3 * s] = (0x7F, 0xFF)[s]
        sees = np.array([(w >> j) & 1 for w in b.words[s]], bool)
        out, lse = b.run()
        np.testing.assert_array_equal(out[t:t + m][~sees], clean[0][t:t + m][~sees])
        np.testing.assert_array_equal(lse[t:t + m], clean[1][t:t + m])
        assert np.isnan(out[t:t + m][sees][..., 5 + 3 * s]).all()
        t += m
