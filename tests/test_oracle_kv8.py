"""Pins of the oracle's 8-bit cache, head norms and attention with hidden rows: torch's own e4m3, closed forms, brute force."""
import numpy as np
import pytest
import torch

from oracle import reference as R
from paper_2505_22179_amd import inputs as I


def test_e4m3_numbers_and_rounding_are_torchs():
    codes = np.arange(256, dtype=np.uint8)
    theirs = torch.from_numpy(codes).view(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(R.e4m3_table(), theirs)
    y = np.arange(0x7C00, dtype=np.uint16).view(np.float16).astype(np.float64)   # every fp16 magnitude
    y = np.concatenate([y[y <= 448], -y[y <= 448]])
    theirs = torch.from_numpy(y.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(R._nearest_e4m3(y), theirs)


@pytest.mark.parametrize("fmt", [R.INT8, R.E4M3])
def test_every_magnitude_of_a_head_reads_back_as_fp16_within_half_a_step(fmt):
    amax = np.arange(0x7C00, dtype=np.uint16).view(np.float16)
    x = np.stack([amax, -(amax * np.float16(0.5)), amax * np.float16(0.3), amax * np.float16(0.011)], -1)
    codes, scales = R.kv8_quantise(x, fmt)
    y = R.kv8_values(codes, scales, fmt)
    np.testing.assert_array_equal(y, y.astype(np.float16).astype(np.float64))
    s, big = scales.astype(np.float64), amax.astype(np.float64)
    err = np.abs(y - x.astype(np.float64))
    if fmt == R.INT8:
        assert (127 * s >= np.minimum(big, 65024)).all()
        # rounded up by less than one unit of four bits, an eighth at most, or of 2^-24
        assert (s < np.maximum(big / 127 * 9 / 8, big / 127 + 2.0 ** -24) * (1 + 1e-12)).all()
        assert (err <= np.where(big > 65024, 480, s / 2)[:, None]).all()
    else:
        assert (s * 448 >= np.minimum(big, 57344)).all() and (np.log2(s) == np.rint(np.log2(s))).all()
        assert (err <= np.maximum(2.0 ** -4 * np.abs(x.astype(np.float64)), (s * 2.0 ** -10)[:, None])).all()


@pytest.mark.parametrize("fmt", [R.INT8, R.E4M3])
def test_zero_and_not_finite_heads(fmt):
    x = np.zeros((3, 2, 8), dtype=np.float16)
    x[1, 0, 3], x[2, 1, 7] = np.inf, np.nan
    x[1, 1] = whole = 127 / 64 if fmt == R.INT8 else 1.75   # a scale of 2^-6 and 2^-8: held exactly
    codes, scales = R.kv8_quantise(x, fmt)
    y = R.kv8_values(codes, scales, fmt)
    assert np.isnan(y[1, 0]).all() and np.isnan(y[2, 1]).all() and (codes[1, 0] == 0).all() and (codes[2, 1] == 0).all()
    assert (y[0] == 0).all() and (y[1, 1] == whole).all() and (y[2, 0] == 0).all()


def test_head_norm_of_a_constant_head_and_rotation_by_nothing():
    M, Hq, Hkv, D = 3, 2, 1, 8
    qkv = np.repeat(np.array([2.0, -3.0, 5.0, 7.0], dtype=np.float16), D)[None].repeat(M, 0)
    one, zero = np.ones((4, D // 2), dtype=np.float32), np.zeros((4, D // 2), dtype=np.float32)
    gq, gk = np.full(D, 3.0, dtype=np.float16), np.full(D, 0.5, dtype=np.float16)
    cache = np.zeros((M + 2, Hkv, D), dtype=np.float16)
    q, k, v = R.rope_append_qk_norm(qkv, gq, gk, 0.0, np.arange(M), one, zero, cache, cache, 2, Hq, Hkv, D)
    np.testing.assert_allclose(q[:, 0], 3.0), np.testing.assert_allclose(q[:, 1], -3.0)
    np.testing.assert_allclose(k[2:], 0.5), np.testing.assert_allclose(v[2:], 7.0)
    assert (k[:2] == 0).all()
    # unit gammas and a head of unit mean square: the plain rotation
    rng = np.random.default_rng(5)
    x = rng.standard_normal((M, 4, D))
    x /= np.sqrt((x * x).mean(-1, keepdims=True))
    cos, sin = I.make_rope_tables(16, D)
    a = R.rope_append_qk_norm(x.reshape(M, -1), np.ones(D), np.ones(D), 0.0, [1, 5, 9], cos, sin, cache, cache, 1, Hq, Hkv, D)
    b = R.rope_append(x.reshape(M, -1), [1, 5, 9], cos, sin, cache, cache, 1, Hq, Hkv, D)
    np.testing.assert_allclose(a[0], b[0], atol=1e-14)


def test_attention_with_hidden_rows():
    a = I.make_attn(77, 9, 20, 8, 2, 128)
    want, _ = R.tree_verify_attn(a.q, a.k, a.v, a.mask, a.scale)
    got, spread = R.tree_verify_attn_seen(a.q, a.k, a.v, a.mask, a.scale)
    np.testing.assert_allclose(got, want, atol=1e-12)
    assert (spread >= np.abs(got) - 1e-12).all()
    k, v, mask = a.k[20:].copy(), a.v[20:].copy(), a.mask.copy()
    mask[4], mask[:, 7] = 0, 0
    k[7], v[7] = np.nan, np.inf
    got, _ = R.tree_verify_attn_seen(a.q, k, v, mask, a.scale)
    assert np.isfinite(got).all() and (got[4] == 0).all()
