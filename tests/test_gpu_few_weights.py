"""Weights that are no numbers in the whole layer for a few tokens (ordermoe_few_moe_layer)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from ._pipeline import host  # noqa: E402
from .test_gpu_few_moe import _few, _layer  # noqa: E402


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", ["inf", "nan"])
@pytest.mark.parametrize("n_shared", [0, 1])
def test_weights_that_are_no_numbers_reach_their_expert_s_tokens_only(dtype, bad, n_shared):
    """As where every expert runs its own rows alone: down weights of a routed expert, then of the
    shared one, change nothing for the tokens that it does not serve."""
    case, dl = _layer(n_shared=n_shared, dtype=dtype)
    case.loc = np.array([0, 1] * 8, np.uint8)
    x, loc, qh = dl.inputs()
    out, y = _few(dl, x, loc, qh, 16)
    torch.cuda.synchronize()
    before, ek, em = host(y), host(out["exec_k"]), host(out["exec_m"])
    uses = [((ek == e) & (em == 0)).any(1) for e in case.local]
    i = int(np.argmax([u.any() and not u.all() for u in uses]))
    assert uses[i].any() and not uses[i].all()
    kept = dl.w_dn[i].clone()
    dl.w_dn[i] = float(bad)
    _, y = _few(dl, x, loc, qh, 16)
    np.testing.assert_array_equal(host(y)[~uses[i]], before[~uses[i]])
    assert not np.isfinite(host(y)[uses[i]]).any()
    dl.w_dn[i] = kept
    if n_shared:
        dl.w_sh_dn[:] = float(bad)
        _, y = _few(dl, x, loc, qh, 16)
        np.testing.assert_array_equal(host(y)[case.loc == 1], before[case.loc == 1])
        assert not np.isfinite(host(y)[case.loc == 0]).any()
