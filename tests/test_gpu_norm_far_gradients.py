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
