"""The numpy definitions that the microscaled GPU tests compare with, against
the formats' published values and by hand (CPU)."""
import numpy as np
import pytest

import mx_ref


def test_grids():
    """e2m1 and e4m3 as published: the largest values, the smallest steps."""
    assert mx_ref.FP4.tolist() == [0, .5, 1, 1.5, 2, 3, 4, 6]
    assert mx_ref.FP8[-1] == 448 and mx_ref.FP8[1] == 2.0 ** -9 and mx_ref.FP8[8] == 2.0 ** -6
    assert np.all(np.diff(mx_ref.FP8) > 0)


@pytest.mark.parametrize("bits, grid", [(4, mx_ref.FP4), (8, mx_ref.FP8)])
def test_ties_go_to_the_even_code(bits, grid):
    mid = (grid[:-1] + grid[1:]) / 2
    got = mx_ref.nearest(mid, grid)
    assert np.all(got % 2 == 0) and np.all(np.abs(got - np.arange(len(mid)) - 0.5) == 0.5)


@pytest.mark.parametrize("bits", [4, 8])
def test_quantise_by_hand(bits):
    x = np.zeros((3, 33), np.float32)
    x[0, :4] = [1.0, -0.5, 0.3, 6.0]          # largest 6: exponent 2
    x[0, 32] = 2.0 ** -140                    # an fp32 denormal: the least scale
    x[1, 5] = np.inf
    x[2, 32] = 7.9                            # above the largest value's share of its binade
    r = mx_ref.quantise(x, bits)
    nb, cb = 2, 4 * bits
    assert r.shape == (3, mx_ref.record_bytes(33, bits))
    s = 2 if bits == 4 else 8
    assert r[0, nb * cb:nb * cb + 2].tolist() == [129 - s, 0]
    assert r[1, nb * cb] == 255 and r[2, nb * cb + 1] == 129 - s
    v = mx_ref.values(r, 33, bits)
    # scale 1: 0.3 is nearest to 0.5; scale 2^-6: 0.3 is 19.2 of them, nearest to 20 (steps of 2)
    assert v[0, :4].tolist() == ([1.0, -0.5, 0.5, 6.0] if bits == 4 else [1.0, -0.5, 20 / 64, 6.0])
    assert np.isnan(v[1, :32]).all() and v[1, 32] == 0
    assert v[2, 32] == (6.0 if bits == 4 else 7.0)
    assert np.all(r[:, nb * (cb + 1):] == 0)


def test_largest_scales_stay_finite():
    x = np.full((1, 32), np.finfo(np.float32).max, np.float32)
    for bits in (4, 8):
        v = mx_ref.values(mx_ref.quantise(x, bits), 32, bits)
        assert np.isfinite(v.astype(np.float32)).all() and v[0, 0] > 2e38


def test_distill_gradient_is_the_loss_s_difference():
    rng = np.random.default_rng(3)
    n, C, k = 4, 7, 3
    z = rng.normal(size=(n, C))
    top, cls = rng.normal(size=(n, k)), rng.integers(-1, C, size=(n, k))
    cls[1] = -1
    cls[2] = 4                                # one class three times
    labels = np.array([2, -1, 0, 6])
    for alpha, T in [(0.5, 2.0), (1.0, 1.0), (0.0, 3.0)]:
        _, grad, _ = mx_ref.distill(z, top, cls, labels, alpha, T)
        for i in range(n):
            for c in range(C):
                h = 1e-5
                a, b = z.copy(), z.copy()
                a[i, c] += h
                b[i, c] -= h
                d = (mx_ref.distill(a, top, cls, labels, alpha, T)[0].mean()
                     - mx_ref.distill(b, top, cls, labels, alpha, T)[0].mean()) / (2 * h)
                assert abs(d - grad[i, c]) < 1e-8
