"""The norm's adjoint where its sums, or what it computes on the way, leave binary32 although the gradients do not.

Bounds.  As in rows of ordinary size: (130 + d / 512) U of the sum over the terms' magnitudes, a rounding, and where binary32 ends 10^-37; a gradient beyond
binary32's largest number is an infinity."""
import numpy as np
import pytest

from oracle import token_oracle as to
from token_util import HALF, U, dev, host, near, space

pytestmark = pytest.mark.gpu
TINY = 1e-37
LARGEST = float(np.finfo(np.float32).max)
#        each number of lanes to a row, and rows in two passes (bfloat16 from 16 385 on, binary32 from 12 289 on)
WIDTHS = [40, 96, 200, 500, 1000, 1500, 4096, 7000, 11000, 13000, 17001]


def check(dy, h, w, eps, dtype="f32", d_h=None, neighbours=()):
    """All gradients against 64 bits; rows `neighbours` have the bits that they have without the others."""
    import torch
    from paper_2602_17681_amd import binding as ae
    rows, d = h.shape
    dy, h = host(dev(dy, dtype)), host(dev(h, dtype))
    w32 = None if w is None else dev(w)
    a = None if d_h is None else dev(d_h, dtype)
    dx, dw = torch.empty((rows, d), dtype=dev(h[:1], dtype).dtype, device="cuda"), torch.empty(d, device="cuda")
    ws = space(ae.model_rms_norm_backward_workspace(rows, d, ae.DTYPES[dtype]))
    ae.model_rms_norm_backward(dev(dy, dtype), dev(h, dtype), rows, d, w32, eps, dx, dw, ws, d_h=a)
    weight = None if w is None else w.astype(np.float64)
    eps = float(np.float32(eps))
    want, d_w, mag, mag_w = to.rms_norm_backward(dy, h, weight, eps, None if d_h is None else host(a))
    tol = (130 + d / 512) * U * mag + (HALF[dtype] if dtype == "bf16" else U) * np.abs(want) + TINY
    over = np.abs(want) > LARGEST * 1.01
    assert not np.any((np.abs(want) + tol > LARGEST) & ~over), "the inputs leave the outcome to the rounding"
    near(host(dx), np.where(over, np.sign(want) * np.inf, want), tol)
    tol_w = (rows + 45 + d / 2048) * U * mag_w + TINY
    fine = np.abs(d_w) + tol_w < LARGEST
    near(host(dw)[fine], d_w[fine], tol_w[fine])
    neighbours = list(neighbours)
    if neighbours:
        alone = torch.empty((len(neighbours), d), dtype=dx.dtype, device="cuda")
        ae.model_rms_norm_backward(dev(dy[neighbours], dtype), dev(h[neighbours], dtype), len(neighbours), d, w32, eps, alone, None, ws, d_h=None if a is None else a[neighbours].contiguous())
        assert torch.equal(dx[neighbours], alone)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rms,spread", [(0.5, 0.5), (0.02, 0.5), (1e-3, 2.0 ** -7)])
@pytest.mark.parametrize("d", WIDTHS)
def test_the_sum_of_products_just_inside_the_range(d, rms, spread, dtype):
    """Gradients along h: their sum of products with h is 0.8 of binary32's largest number or less, and 1 / rms times it is beyond; the gradient of h is not."""
    rng = np.random.default_rng(d)
    h = rng.standard_normal((7, d))
    dy = rng.standard_normal((7, d))
    for i in (1, 4, 5):
        h[i] = rms * np.sign(h[i]) * (1 + spread * rng.uniform(-1, 1, d))
        dy[i] = np.sign(h[i]) * (0.8 * LARGEST / np.abs(h[i]).sum())
        h[i, d // 2] = dy[i, d // 2] = 0.0
    # dx is linear in dy: what would leave the range is scaled down, to 0.9 of its end
    dx = to.rms_norm_backward(dy, h, None, 1e-9)[0]
    dy *= np.minimum(1.0, 0.9 * LARGEST / np.maximum(np.abs(dx), np.abs(dy)).max(1, keepdims=True))
    check(dy.astype(np.float32), h.astype(np.float32), None, 1e-9, dtype, neighbours=(0, 2, 3, 6))


@pytest.mark.parametrize("d", [2, 64] + WIDTHS)
def test_large_gradients_of_large_rows(d):
    """One element of 2^64, gradients of 2^90 elsewhere: the gradient of h is 2^26 sqrt(d)."""
    h, dy = np.zeros((3, d), np.float32), np.ones((3, d), np.float32)
    h[0, 0] = h[2, d - 1] = 2.0 ** 64
    h[1] = 1.0
    dy[0, 1] = 2.0 ** 90
    dy[2, 0] = -2.0 ** 120
    check(dy, h, None, 1e-6, neighbours=(1,))


@pytest.mark.parametrize("d", WIDTHS)
def test_small_gradients_beside_large_ones(d):
    """Where the sum of products leaves the range, columns with h = 0 keep gradients of 10^-20 and 10^-30."""
    rng = np.random.default_rng(d)
    h = rng.standard_normal((6, d)).astype(np.float32)
    dy = rng.standard_normal((6, d)).astype(np.float32)
    for i in (0, 3):
        h[i] = np.sign(h[i]) * (0.5 + np.abs(h[i]))
        dy[i] = np.sign(h[i]) * np.float32(2e38 / d * 8)
        h[i, 1:3] = 0
        dy[i, 1], dy[i, 2] = 1e-20, -1e-30
    check(dy, h, None, 1e-6, neighbours=(1, 2, 4, 5))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_rows_of_large_and_small_elements(d, dtype):
    """Rows beyond the range of squares with elements of 10^-15 in them, and gradients of every size; the weight's gradient of the small ones."""
    rng = np.random.default_rng(d)
    h = rng.standard_normal((5, d))
    dy = rng.standard_normal((5, d))
    h[1] *= 1e-15
    h[1, 0] = 2.0 ** 65
    h[2, : d // 2] *= 1e20
    dy[2] *= 1e10
    h[4] *= 1e-10
    h[4, d - 1] = 3e38
    dy[4] *= 1e25
    dy[[0, 3]] = 0                              # the weight's gradient is that of these rows
    check(dy.astype(np.float32), h.astype(np.float32), (1 + 0.2 * rng.standard_normal(d)).astype(np.float32), 1e-6, dtype, d_h=(rng.standard_normal((5, d)) * (rng.random((5, d)) < 0.5)).astype(np.float32), neighbours=(0, 3))


@pytest.mark.parametrize("d", WIDTHS)
def test_products_with_the_weight_beyond_the_range(d):
    """dy times weight beyond binary32, whose product with 1 / rms is not; beside h = 0, too."""
    rng = np.random.default_rng(d)
    h = (rng.standard_normal((4, d)) * 1e12).astype(np.float32)
    dy = rng.standard_normal((4, d)).astype(np.float32)
    w = np.full(d, 1e6, np.float32)
    dy[1] *= np.float32(1e34)
    dy[2, 3] = 1e37
    h[2, 3] = 0
    check(dy, h, w, 1e-6, neighbours=(0, 3))


@pytest.mark.parametrize("d", WIDTHS)
def test_differences_near_the_largest_number(d):
    """The largest gradients against a part along h of the other sign, rms 10: their difference is beyond binary32, a tenth of it is not."""
    rng = np.random.default_rng(d)
    h = (10 * np.sign(rng.standard_normal((3, d)))).astype(np.float32)
    dy = rng.standard_normal((3, d)).astype(np.float32)
    dy[1] = np.sign(h[1]) * np.float32(3.3e38)
    dy[1, 0] *= -1
    check(dy, h, None, 1e-6, neighbours=(0, 2))


@pytest.mark.parametrize("size", [1e-21, 1e-24, 1e-27])
@pytest.mark.parametrize("d", WIDTHS)
def test_products_below_the_range(d, size):
    """h, gradients and eps so small that the products of h and the gradients are subnormal or zero, while gradient over rms is ordinary."""
    rng = np.random.default_rng(d)
    h = (rng.standard_normal((6, d)) * 1e-19).astype(np.float32)
    dy = (rng.standard_normal((6, d)) * size).astype(np.float32)
    dy[2] = np.sign(h[2]) * np.float32(10 * size)
    h[3] = 0
    h[4], dy[4] = np.abs(h[4, 0]), 0                       # large products that cancel
    dy[4, 0], dy[4, 1] = 1e20, -1e20
    h[4, 2], dy[4, 2] = 0, 1e10
    dy[5] = np.abs(dy[5]) * np.sign(h[5])
    h[5, ::3] = np.abs(h[5, ::3])
    dy[5, ::3] = 0                                         # nothing but the part along h there
    check(dy, h, None, 2.0 ** -125)


@pytest.mark.parametrize("size", [1e-21, 1e-24, 1e-27])
@pytest.mark.parametrize("d", WIDTHS)
def test_products_below_the_range_of_rows_far_below_eps(d, size):
    """h so far below the root of eps that u times mean(g u) is subnormal, too, though 1 / rms times it is ordinary; gradients in every second column."""
    rng = np.random.default_rng(d)
    h = (rng.standard_normal((4, d)) * 1e-26).astype(np.float32)
    dy = (rng.standard_normal((4, d)) * size).astype(np.float32)
    dy[1] = np.sign(h[1]) * np.float32(size)
    dy[:, 1::2] = 0
    dy[2, 1] = 1e-5
    check(dy, h, None, 2.0 ** -125)
