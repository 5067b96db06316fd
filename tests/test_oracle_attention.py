"""The oracle's cache and attention against what is known of them otherwise:
torch's e4m3 type, rotations as 2 x 2 matrices, softmax term by term."""
import numpy as np
import pytest
import torch

from oracle import attention as oa


def test_e4m3_values_are_torch_s():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(oa.code_values(oa.FP8), want)


def test_int8_values_are_two_s_complement():
    np.testing.assert_array_equal(oa.code_values(oa.INT8), np.arange(256).astype(np.uint8).view(np.int8).astype(np.float64))


def test_nearest_e4m3_code_is_torch_s_cast():
    rng = np.random.default_rng(0)
    v = oa.code_values(oa.FP8)[:127]
    y = np.concatenate([v, (v[1:] + v[:-1]) / 2, rng.uniform(-448, 448, 4000), rng.normal(size=4000) * 0.02]).astype(np.float32)
    y = np.concatenate([y, -y])
    want = torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(oa.nearest_codes(y, oa.FP8), want)


@pytest.mark.parametrize("fmt", [oa.INT8, oa.FP8])
def test_rows_that_are_zero_tiny_or_no_numbers(fmt):
    x = np.ones((5, 8), np.float32)
    x[0] = 0
    x[1] = 1e-31
    x[2, 3] = np.inf
    x[3, 0] = np.nan
    codes, scale = oa.quantise(x, fmt)
    assert (codes[:4] == 0).all() and (scale[:2] == 0).all() and np.isnan(scale[2:4]).all()
    assert scale[4] == np.float32(1) / oa.CODE_MAX[fmt]
    assert (oa.code_values(fmt)[codes[4]] == oa.CODE_MAX[fmt]).all()


def test_quantised_values_lie_within_half_a_step():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(50, 64)).astype(np.float32)
    codes, scale = oa.quantise(x, oa.INT8)
    assert np.abs(oa.code_values(oa.INT8)[codes] * scale[:, None].astype(np.float64) - x).max() <= scale.max() * 0.5001


@pytest.mark.parametrize("inter", [False, True])
def test_rotation_is_a_rotation_by_the_table_s_angle(inter):
    rng = np.random.default_rng(2)
    x = rng.normal(size=(3, 2, 16))
    ang = rng.uniform(0, 6, size=(7, 4))
    cs = np.concatenate([np.cos(ang), np.sin(ang)], 1)
    pos = np.array([6, 0, 3])
    got = oa.head_rows(x, None, 0.0, cs, pos, inter)
    for t in range(3):
        for i in range(4):
            a, b = (2 * i, 2 * i + 1) if inter else (i, i + 4)
            th = ang[pos[t], i]
            rot = np.array([[np.cos(th), -np.sin(th)], [np.sin(th), np.cos(th)]])
            np.testing.assert_allclose(got[t][:, [a, b]], x[t][:, [a, b]] @ rot.T, atol=1e-12)
    np.testing.assert_array_equal(got[:, :, 8:], x[:, :, 8:])


def test_attention_term_by_term_and_empty_rows():
    rng = np.random.default_rng(3)
    k, v = rng.normal(size=(2, 5, 1, 4))
    q = rng.normal(size=(2, 2, 4))
    out, lse, mag = oa.draft_attention(q, k, v, 3, [0b01, 0b11], 0.5)
    for i, seen in enumerate(([0, 1, 2, 3], [0, 1, 2, 3, 4])):
        for h in range(2):
            e = [np.exp(0.5 * float(q[i, h] @ k[p, 0])) for p in seen]
            np.testing.assert_allclose(lse[i, h], np.log(sum(e)), rtol=1e-12)
            np.testing.assert_allclose(out[i, h], sum(w * v[p, 0] for w, p in zip(e, seen)) / sum(e), rtol=1e-12)
    out, lse, _ = oa.draft_attention(q, k[3:], v[3:], 0, [0, 0b10], 0.5)
    assert (out[0] == 0).all() and np.isneginf(lse[0]).all()
    np.testing.assert_allclose(out[1], np.broadcast_to(v[4], out[1].shape), rtol=1e-12)
    assert (mag >= np.abs(out[1]) * 0).all()
