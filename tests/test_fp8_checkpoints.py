"""Weights that come as codes and scales, widened and quantized again, by the oracle."""
import numpy as np

import oracle


def widened(rng, N, K, most):
    """Codes up to `most` in every block of 128 x 128, scales, and the numbers they stand for in binary32."""
    finite = np.flatnonzero(np.abs(np.nan_to_num(oracle.E4M3, nan=1e9)) <= most).astype(np.uint8)
    codes = rng.choice(finite, (N, K))
    largest = int(finite[np.argmax(oracle.E4M3[finite])])
    codes[::128, ::128] = largest
    scales = np.exp(rng.standard_normal((-(-N // 128), -(-K // 128)))).astype(np.float32) * np.float32(1e-4)
    spread = scales[np.arange(N) // 128][:, np.arange(K) // 128]
    return codes, scales, oracle.e4m3_values(codes).astype(np.float32) * spread


def test_blocks_that_hold_the_largest_code_keep_their_codes():
    codes, scales, W = widened(np.random.default_rng(1), 300, 517, 448.0)
    again, s = oracle.quant_weight_fp8(W)
    assert np.array_equal(np.where(again == 0x80, 0, again), np.where(codes == 0x80, 0, codes))
    assert np.all(np.abs(s.view(np.int32) - scales.view(np.int32)) <= 1)


def test_other_blocks_are_rounded_once_more():
    codes, scales, W = widened(np.random.default_rng(2), 140, 200, 416.0)
    again, s = oracle.quant_weight_fp8(W)
    assert np.any(again != codes)
    back = oracle.e4m3_values(again) * s[np.arange(140) // 128][:, np.arange(200) // 128].astype(np.float64)
    step = s.max() * 2.0 ** -9   # of the smallest codes; half of it, or half of 2^-3 of a value
    assert np.all(np.abs(back - W) <= np.maximum(np.abs(W) * 2.0 ** -4, step / 2) * (1 + 2.0 ** -20))
