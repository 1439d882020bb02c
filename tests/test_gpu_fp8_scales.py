"""Products of scales at the ends of binary32's range: one binary32 product each, in every form of the kernels, and without
effect on other rows and columns."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("blocks", ["rows", "tiles"])
@pytest.mark.parametrize("m,n", [(5, 300), (40, 300), (100, 300), (300, 1000), (1100, 1100), (2100, 2100), (4100, 4100)])
def test_scales_far_apart(m, n, blocks, dtype):
    import torch
    from paper_2602_17681_amd import binding as ae
    k, kb = 256, 2
    rng = np.random.default_rng(m)
    room = lambda r: torch.empty((r, k), dtype=torch.uint8, device="cuda")      # noqa: E731
    av, bv = rng.choice([-1.0, 1.0], (m, k)), rng.choice([-1.0, 1.0], (n, k))
    av[2] = 0.0                                            # a block sum of 0 everywhere
    code = lambda v: torch.from_numpy(np.where(v == 0, 0, np.where(v > 0, 0x38, 0xB8)).astype(np.uint8)).cuda()      # noqa: E731
    a, b = room(m), room(n)
    a.copy_(code(av))
    b.copy_(code(bv))
    sa = np.full((kb, m), 1.0, np.float32)
    sb = np.full((kb, n) if blocks == "rows" else (-(-n // 128), kb), 1.0, np.float32)
    big, small = np.float32(2.0 ** 100), np.float32(2.0 ** -100)
    sa[0, 0], sa[0, 1], sa[0, 2], sa[1, 3], sa[:, 4] = big, small, big, 2.0 ** 27, small
    if blocks == "rows":
        sb[0, 7], sb[0, 9], sb[1, n - 1] = big, small, 2.0 ** 100
    else:
        sb[0, 0], sb[1, 0], sb[-1, 0] = big, 2.0 ** 100, small
    y = torch.full((m, n), -7.0, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    ae.model_fp8_matmul(a, torch.from_numpy(sa).cuda(), b, torch.from_numpy(sb).cuda(), blocks, None, m, n, k, y)
    # block sums are whole numbers below 2^8; in binary32, as the call does it
    want = np.zeros((m, n), np.float32)
    with np.errstate(all="ignore"):
        for c in range(kb):
            s = slice(128 * c, 128 * c + 128)
            col = sb[c] if blocks == "rows" else sb[np.arange(n) // 128, c]
            want = (want.astype(np.float64) + (av[:, s] @ bv[:, s].T) * (sa[c][:, None] * col[None, :]).astype(np.float64)).astype(np.float32)
    got, want = y.float().cpu().numpy(), torch.from_numpy(want).to(y.dtype).float().numpy()
    assert np.isnan(want).any() and np.isinf(want).any()   # 0 times an infinite product, and others
    assert np.array_equal(got, want, equal_nan=True)
