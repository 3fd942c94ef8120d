"""CPU checks of the block-of-128 oracle: codes are the nearest values, the SwiGLU gradient is the
differences of SwiGLU, odd shapes and blocks without a finite maximum."""
import numpy as np
import pytest

from oracle import fp8, mx


def test_codes_are_the_nearest_values():
    g = np.random.default_rng(0)
    x = (g.standard_normal((7, 300)) * np.exp(g.uniform(-8, 8, (7, 1)))).astype(np.float32)
    codes, scales = fp8.quantize(x)
    assert codes.shape == (7, 384) and scales.shape == (7, 3) and not codes[:, 300:].any()
    table = mx.fmt_values(mx.E4M3)
    table = np.concatenate([-table[::-1], table])
    q = x.astype(np.float64) / np.repeat(scales.astype(np.float64), 128, 1)[:, :300]
    got = mx.decode(codes, mx.E4M3)[:, :300]
    nearest = np.abs(q[..., None] - table).min(-1)
    assert np.all(np.abs(got - q) <= nearest + 2.0 ** -23 * np.abs(q))
    # each block's maximum is coded as 448
    full = np.zeros((7, 384))
    full[:, :300] = got
    assert np.all(np.abs(full).reshape(7, 3, 128).max(-1) == 448)


def test_tiles_share_one_scale_and_transpose():
    g = np.random.default_rng(1)
    x = g.standard_normal((200, 260)).astype(np.float32)
    codes, scales = fp8.quantize(x, 128)
    assert scales.shape == (2, 3)
    ct, st = fp8.quantize(np.ascontiguousarray(x.T), 128)
    assert np.array_equal(st, scales.T) and np.array_equal(ct[:260, :200], codes[:, :260].T)


def test_blocks_without_a_finite_maximum():
    x = np.zeros((4, 256), dtype=np.float32)
    x[0, 5], x[1, 200], x[2] = np.inf, np.nan, 1e-30
    codes, scales = fp8.quantize(x)
    assert np.isnan(scales[0, 0]) and np.isnan(scales[1, 1]) and np.isfinite(scales[0, 1]) and np.isfinite(scales[1, 0])
    assert not codes[:2].any() and not codes[2].any()          # far below the smallest scale's step
    assert np.all(scales[3] == np.float32(2.0 ** -60) / np.float32(448))


@pytest.mark.parametrize("rows,I", [(3, 4), (1, 7)])
def test_swiglu_gradient_is_its_differences(rows, I):
    g = np.random.default_rng(2)
    gu, dh, h = 2 * g.standard_normal((rows, 2 * I)), g.standard_normal((rows, I)), 1e-6
    d, val, mag = fp8.swiglu_backward(gu, dh)
    assert np.allclose(val, fp8.swiglu(gu), rtol=1e-14) and np.all(np.abs(d) <= mag * (1 + 1e-12))
    for c in range(2 * I):
        step = np.zeros_like(gu)
        step[:, c] = h
        want = ((fp8.swiglu(gu + step) - fp8.swiglu(gu - step)) * dh).sum(1) / (2 * h)
        assert np.allclose(d[:, c], want, atol=1e-7)
