"""Norms of rows that hold large and small elements together, so that the sum of squares leaves binary32 while other elements are ordinary or tiny.

Bounds.  y is h times a number that is rounded once or as in rows of ordinary size, then times the weight: (36 + d / 2048) U as there.
Where u = h / rms is subnormal it is off by up to 2^-150 before it is multiplied by w, and the product by up to 2^-150 again: 2^-150 (1 + |w|) besides."""
import numpy as np
import pytest

from oracle import fp8_oracle as fo
from oracle import token_oracle as to
from token_util import HALF, U, dev, host, near

pytestmark = pytest.mark.gpu
#        each number of lanes to a row, and rows that are read twice
WIDTHS = [2, 40, 96, 200, 500, 1000, 1500, 3000, 7000, 11000, 15000, 17001]


def mixed(rng, d, dtype):
    """Ordinary rows; rows with one element, or a half, whose squares leave binary32 beside elements of 10^-15, 1 and 10^-30; the largest numbers beside 10^-5."""
    x = rng.standard_normal((9, d)).astype(np.float32)
    half = max(1, d // 2)
    small = np.sign(x) * np.exp(rng.uniform(np.log(1e-18), np.log(1e-10), x.shape))
    x[1] = small[1]
    x[1, 0] = 2.0 ** 65
    x[3, half:] = small[3, half:]
    x[3, :half] *= np.float32(1e20)
    x[4, d - 1] = -2.0 ** 64.5
    x[6] = np.sign(x[6]) * np.float32(1e-5)
    x[6, :half] = np.float32(3e38) * np.sign(x[6, :half])
    x[7] *= np.float32(1e-15)
    x[7, d // 3] = 1e25
    return host(dev(x, dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_small_elements_of_large_rows(d, dtype):
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(d)
    x = mixed(rng, d, dtype)
    w = (1 + 0.2 * rng.standard_normal(d)).astype(np.float32)
    r = np.zeros_like(x)                       # a residual that leaves the sum what it is
    rows = len(x)
    y, h = torch.empty((rows, d), device="cuda", dtype={"f32": torch.float32, "bf16": torch.bfloat16}[dtype]), None
    q, s = torch.empty((rows, -(-d // 16) * 16), dtype=torch.uint8, device="cuda"), torch.empty((-(-d // 128), rows), device="cuda")
    rel = (36 + d / 2048) * U
    for residual in (None, dev(r, dtype)):
        h = None if residual is None else torch.empty_like(y)
        ae.model_rms_norm(dev(x, dtype), rows, d, dev(w), 1e-6, h=h, y=y, q=q[:, :d], scale=s, residual=residual)
        hs, want = to.rms_norm(x, None, w, 1e-6)
        sub = 2.0 ** -150 * (1 + np.abs(w.astype(np.float64))) * 1.001 + (2.0 ** -134 if dtype == "bf16" else 0)
        near(host(y), want, (rel + (HALF["bf16"] if dtype == "bf16" else 0)) * np.abs(want) + sub)
        assert h is None or np.array_equal(host(h), hs)
        # each code is the nearest to y / scale, but for the rounding of y and of the scale: blocks of nothing but small elements have their own scale
        blocks = -(-d // 128)
        amax = np.stack([np.abs(want[:, c * 128:(c + 1) * 128]).max(1) for c in range(blocks)])
        scale = host(s)
        near(scale, np.maximum(amax / 448, 2.0 ** -126), (rel + 2 * U) * amax / 448 + 2.0 ** -149)
        per = scale[np.arange(d) // 128].T
        near(fo.VALUES[q[:, :d].cpu().numpy()] * per, want, 2.0 ** -4 * (1 + 2.0 ** -10) * np.abs(want) + per * 2.0 ** -10)
        if dtype == "f32":
            codes, scales = fo.quantize(y.cpu().numpy())
            assert np.array_equal(q[:, :d].cpu().numpy(), codes) and np.array_equal(scale, scales)


@pytest.mark.parametrize("d", WIDTHS)
def test_other_rows_are_not_affected(d):
    """The rows beside those have the same bits as without them."""
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(d)
    x = mixed(rng, d, "f32")
    w = dev((1 + 0.2 * rng.standard_normal(d)).astype(np.float32))
    plain = [0, 2, 5, 8]
    both, alone = torch.empty((9, d), device="cuda"), torch.empty((4, d), device="cuda")
    ae.model_rms_norm(dev(x), 9, d, w, 1e-6, y=both)
    ae.model_rms_norm(dev(x[plain]), 4, d, w, 1e-6, y=alone)
    assert torch.equal(both[plain], alone)
