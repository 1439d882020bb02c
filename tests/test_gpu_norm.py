"""Root-mean-square norm with the residual's addition and its adjoint against the oracle in 64 bits.

Bounds.  A sum of n positive squares, added by chains of at most k additions, is off by (k + 1) U relative; the inverse root
halves that.  k: up to 32 in a thread's registers (d / 1 024 + 8 in the pass that reads rows twice), 6 over a wavefront, 5 over the
others.  With the rounding of h (twice), quotient, sum, root, reciprocal and two products: (26 + d / 2 048 + 9) U, taken as
(36 + d / 2048) U.  A rounding to bfloat16 adds 2^-8 of the result."""
import numpy as np
import pytest

from oracle import fp8_oracle as fo
from oracle import token_oracle as to
from token_util import HALF, U, Room, dev, host, near, replayed, space

pytestmark = pytest.mark.gpu
EPS = 1e-5
TINY = 1e-37                     # where binary32 ends

#        rows, d: one piece, parts of one, each number of wavefronts to a row, its borders, rows that are read twice
SIZES = [(1, 1), (3, 7), (37, 8), (70, 57), (33, 64), (34, 65), (5, 128), (4, 511), (7, 513), (1, 1024), (33, 1003), (9, 2047), (2, 2049), (1, 4096), (130, 4096), (3, 4100), (3, 8192), (2, 8200),
         (3, 12288), (2, 12291), (2, 16384), (3, 16386), (3, 20001), (2, 32768), (2, 32776), (1, 70001)]
#        more rows than teams of the launch
MANY = [(40000, 50), (33001, 64), (9001, 130), (8200, 1000), (2500, 1100), (2300, 4096), (1100, 5000), (600, 9000), (560, 13001), (600, 17000), (530, 33000)]


def rel(d):
    return (36 + d / 2048) * U


def inputs(rows, d, dtype, seed):
    rng = np.random.default_rng(seed)
    gain = np.where(rng.random(d) < 0.02, 20.0, 1.0)
    x, r = (host(dev((rng.standard_normal((rows, d)) * gain).astype(np.float32), dtype)) for _ in range(2))
    return rng, x, r, (1 + 0.2 * rng.standard_normal(d)).astype(np.float32).astype(np.float64)


def check_codes(q, scale, y, d):
    """Each code is the nearest to y / scale, but for the rounding of y and of the scale; each scale that of its block."""
    codes = q.contiguous().view(__import__("torch").uint8).cpu().numpy()
    s = scale.double().cpu().numpy()
    blocks = -(-d // 128)
    amax = np.stack([np.abs(y[:, c * 128:(c + 1) * 128]).max(1) for c in range(blocks)])
    near(s, np.maximum(amax / 448, 2.0 ** -126), (rel(d) + 2 * U) * amax / 448)
    per = s[np.arange(d) // 128].T
    v = fo.VALUES[codes] * per
    near(v, y, 2.0 ** -4 * (1 + 2.0 ** -10) * np.abs(y) + per * 2.0 ** -10)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("rows,d", SIZES)
def test_forward(rows, d, residual, dtype):
    import torch
    from paper_2602_17681_amd import binding as ae
    rng, x, r, w = inputs(rows, d, dtype, rows + d)
    xm, rm = Room(rows, d, dtype, 3, 1, dev(x)), Room(rows, d, dtype, 0, 5, dev(r))
    hm, ym = Room(rows, d, dtype, 5, 3), Room(rows, d, dtype, 1, 0)
    q = torch.full((rows + 1, -(-d // 16) * 16 + 16), 0x55, dtype=torch.uint8, device="cuda")
    scale = torch.full((-(-d // 128) * rows + 3,), 9.0, device="cuda")
    ae.model_rms_norm(xm.m, rows, d, dev(w), EPS, hm.m, ym.m, q[:rows, :d], scale[:-3].view(-1, rows), residual=rm.m if residual else None)
    h, y = to.rms_norm(x, r if residual else None, w, EPS)
    near(host(hm.m), h, HALF[dtype] * np.abs(h) + TINY * 1e-6)
    near(host(ym.m), y, (rel(d) + (HALF[dtype] if dtype == "bf16" else 0)) * np.abs(y) + TINY)
    check_codes(q[:rows, :d], scale[:-3].view(-1, rows), y, d)
    assert hm.whole() and ym.whole() and xm.whole() and bool((q[rows:] == 0x55).all()) and bool((q[:, d:] == 0x55).all()) and bool((scale[-3:] == 9).all())
    if dtype == "f32":           # the codes of exactly the y that is returned
        codes, s = fo.quantize(ym.m.cpu().numpy())
        assert np.array_equal(q[:rows, :d].cpu().numpy(), codes) and np.array_equal(scale[:-3].view(-1, rows).cpu().numpy(), s)
    # each output alone gives the same bits
    h2, y2 = Room(rows, d, dtype), Room(rows, d, dtype)
    q2, s2 = torch.zeros_like(q), torch.zeros_like(scale)
    res = rm.m if residual else None
    ae.model_rms_norm(xm.m, rows, d, dev(w), EPS, h=h2.m, residual=res)
    ae.model_rms_norm(xm.m, rows, d, dev(w), EPS, y=y2.m, residual=res)
    ae.model_rms_norm(xm.m, rows, d, dev(w), EPS, q=q2[:rows, :d], scale=s2[:-3].view(-1, rows), residual=res)
    assert torch.equal(h2.m, hm.m) and torch.equal(y2.m, ym.m) and torch.equal(q2[:rows, :d], q[:rows, :d]) and torch.equal(s2[:-3], scale[:-3])
    # without a weight: ones
    ae.model_rms_norm(xm.m, rows, d, None, EPS, y=y2.m, residual=res)
    ae.model_rms_norm(xm.m, rows, d, torch.ones(d, device="cuda"), EPS, y=ym.m, residual=res)
    assert torch.equal(y2.m, ym.m)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d", MANY)
def test_many_rows_in_place(rows, d, dtype):
    """h in the residual's place and y in x's place; as many rows as the launch takes in more than one round."""
    import torch
    from paper_2602_17681_amd import binding as ae
    rng, x, r, w = inputs(rows, d, dtype, rows)
    xm, rm = Room(rows, d, dtype, 0, 0, dev(x)), Room(rows, d, dtype, 2, 1, dev(r))
    q, s = torch.empty((rows, -(-d // 16) * 16), dtype=torch.float8_e4m3fn, device="cuda")[:, :d], torch.empty((-(-d // 128), rows), device="cuda")
    ae.model_rms_norm(xm.m, rows, d, dev(w), EPS, h=rm.m, y=xm.m, q=q, scale=s, residual=rm.m)
    h, y = to.rms_norm(x, r, w, EPS)
    near(host(rm.m), h, HALF[dtype] * np.abs(h))
    near(host(xm.m), y, (rel(d) + (HALF[dtype] if dtype == "bf16" else 0)) * np.abs(y) + TINY)
    check_codes(q, s, y, d)
    assert xm.whole() and rm.whole()


@pytest.mark.parametrize("d", [40, 96, 3000, 9000, 40000])
def test_unusual_rows(d):
    """Zeros, one number alone, magnitudes whose squares leave binary32, the largest numbers, tiny ones, infinities, NaN; neighbours are not affected."""
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(d)
    x = rng.standard_normal((12, d)).astype(np.float32)
    x[1] = 0
    x[2] = 0
    x[2, d // 2] = 3.0
    x[3] *= np.float32(1e30)
    x[4] = np.float32(3.4e38) * np.sign(x[4])
    x[5] *= np.float32(1e-25)
    x[6, 0] = np.inf
    x[7, d - 1] = np.nan
    x[8] *= np.float32(1e19)
    x[10] *= np.float32(1e-38)
    w = (1 + 0.2 * rng.standard_normal(d)).astype(np.float32)
    q, s = torch.empty((12, -(-d // 16) * 16), dtype=torch.uint8, device="cuda"), torch.empty((-(-d // 128), 12), device="cuda")
    y = torch.empty((12, d), device="cuda")
    for eps in (1e-6, 2.0 ** -120):
        ae.model_rms_norm(dev(x), 12, d, dev(w), eps, y=y, q=q[:, :d], scale=s)
        _, want = to.rms_norm(np.where(np.isfinite(x), x, 0), None, w, eps)
        fine = [i for i in range(12) if i not in (6, 7)]
        # squares of 10^-38 times a mean's 1/d lie among binary32's subnormals: their sum is off by up to d halves of 2^-149, which eps outweighs
        sub = d * 2.0 ** -150 / d / eps
        near(host(y)[fine], want[fine], (rel(d) + sub) * np.abs(want[fine]) + 2.0 ** -149)
        got = host(y)
        assert np.isnan(got[6, 0]) and np.all(got[6, 1:] == 0) and np.all(np.isnan(got[7]))
        codes, scales = fo.quantize(y.cpu().numpy())
        c = q[:, :d].cpu().numpy()
        assert np.array_equal(fo.VALUES[c], fo.VALUES[codes], equal_nan=True) and np.array_equal(s.cpu().numpy(), scales)
    # a weight whose products overflow: saturated codes beside the infinities of y
    ae.model_rms_norm(dev(x), 12, d, dev(np.full(d, 3e38, np.float32)), 1e-6, y=y, q=q[:, :d], scale=s)
    codes, scales = fo.quantize(y.cpu().numpy())
    assert np.isinf(host(y)[0]).any() and np.array_equal(fo.VALUES[q[:, :d].cpu().numpy()], fo.VALUES[codes], equal_nan=True) and np.array_equal(s.cpu().numpy(), scales)


def grad_bound(dx, mag, d, dtype):
    """A signed sum of n terms is off by (k + 1) U of the sum over magnitudes, k as above, and each term by the rounding of its factors: r (36 + d / 2048 U),
    two products, u; 2 (36 + d / 2048) + 45 + d / 1024 + 6 of `mag` in all."""
    return (130 + d / 512) * U * mag + (HALF[dtype] if dtype == "bf16" else U) * np.abs(dx) + TINY


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("rows,d", SIZES)
def test_backward(rows, d, residual, dtype):
    import torch
    from paper_2602_17681_amd import binding as ae
    rng, x, r, w = inputs(rows, d, dtype, rows + d)
    dy, add = (host(dev(1e-3 * rng.standard_normal((rows, d)).astype(np.float32), dtype)) for _ in range(2))
    hm, gm, am, dm = Room(rows, d, dtype, 3, 1, dev(x)), Room(rows, d, dtype, 0, 3, dev(dy)), Room(rows, d, dtype, 2, 2, dev(add)), Room(rows, d, dtype, 5, 1)
    ws = space(ae.model_rms_norm_backward_workspace(rows, d, ae.DTYPES[dtype]))
    dw = torch.full((d + 2,), 7.0, device="cuda")
    a = am.m if residual else None
    ae.model_rms_norm_backward(gm.m, hm.m, rows, d, dev(w), EPS, dm.m, dw[:d], ws, d_h=a)
    dx, d_w, mag, mag_w = to.rms_norm_backward(dy, x, w, EPS, add if residual else None)
    near(host(dm.m), dx, grad_bound(dx, mag, d, dtype))
    near(host(dw[:d]), d_w, (rows + 45 + d / 2048) * U * mag_w + TINY)
    assert dm.whole() and hm.whole() and bool((dw[d:] == 7).all())
    # one output alone, no weight
    d2, dw2 = Room(rows, d, dtype), torch.empty(d, device="cuda")
    ae.model_rms_norm_backward(gm.m, hm.m, rows, d, dev(w), EPS, d2.m, None, ws, d_h=a)
    ae.model_rms_norm_backward(gm.m, hm.m, rows, d, dev(w), EPS, None, dw2, ws, d_h=a)
    assert torch.equal(d2.m, dm.m) and torch.equal(dw2, dw[:d])
    ae.model_rms_norm_backward(gm.m, hm.m, rows, d, None, EPS, d2.m, dw2, ws, d_h=a)
    dx, d_w, mag, mag_w = to.rms_norm_backward(dy, x, None, EPS, add if residual else None)
    near(host(d2.m), dx, grad_bound(dx, mag, d, dtype))


@pytest.mark.parametrize("place", ["dy", "h", "d_h"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d", MANY)
def test_backward_many_rows_in_place(rows, d, dtype, place):
    import torch
    from paper_2602_17681_amd import binding as ae
    rng, x, r, w = inputs(rows, d, dtype, rows)
    dy, add = (host(dev(1e-3 * rng.standard_normal((rows, d)).astype(np.float32), dtype)) for _ in range(2))
    m = dict(h=dev(x, dtype), dy=dev(dy, dtype), d_h=dev(add, dtype))
    ws, dw = space(ae.model_rms_norm_backward_workspace(rows, d, ae.DTYPES[dtype])), torch.empty(d, device="cuda")
    ae.model_rms_norm_backward(m["dy"], m["h"], rows, d, dev(w), EPS, m[place], dw, ws, d_h=m["d_h"])
    dx, d_w, mag, mag_w = to.rms_norm_backward(dy, x, w, EPS, add)
    near(host(m[place]), dx, grad_bound(dx, mag, d, dtype))
    near(host(dw), d_w, (rows + 45 + d / 2048) * U * mag_w)


@pytest.mark.parametrize("d", [40, 96, 3000, 9000, 40000])
def test_backward_of_unusual_rows(d):
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(d)
    x = rng.standard_normal((8, d)).astype(np.float32)
    x[1] = 0
    x[2] *= np.float32(1e30)
    x[3] *= np.float32(3e37)
    x[4] *= np.float32(1e-30)
    x[5] *= np.float32(1e19)
    dy = rng.standard_normal((8, d)).astype(np.float32)
    dy[5] *= np.float32(1e22)
    ws, dx, dw = space(ae.model_rms_norm_backward_workspace(8, d, ae.AE_F32)), torch.empty((8, d), device="cuda"), torch.empty(d, device="cuda")
    ae.model_rms_norm_backward(dev(dy), dev(x), 8, d, None, 1e-6, dx, dw, ws)
    want, d_w, mag, mag_w = to.rms_norm_backward(dy, x, None, 1e-6)
    near(host(dx), want, grad_bound(want, mag, d, "f32") + 2.0 ** -149)
    near(host(dw), d_w, (8 + 45 + d / 2048) * U * mag_w + TINY)
    x[6, 1], x[7, 0] = np.nan, np.inf          # their own rows only, and the weight's gradient
    ae.model_rms_norm_backward(dev(dy), dev(x), 8, d, None, 1e-6, dx, dw, ws)
    near(host(dx)[:6], want[:6], grad_bound(want, mag, d, "f32")[:6] + 2.0 ** -149)
    assert np.all(np.isnan(host(dx)[6]))


@pytest.mark.parametrize("d", [48, 96, 200, 3000, 9000])
def test_backward_where_only_the_sum_of_products_leaves_the_range(d):
    """Gradients along h whose products with it add up beyond binary32, at ordinary, small (eps as large as the mean) and large h; other rows of the
    same wavefront are not affected, nor is the weight's gradient by an infinite or NaN gradient of another column."""
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(d)
    h = rng.standard_normal((9, d)).astype(np.float32)
    dy = rng.standard_normal((9, d)).astype(np.float32)
    h[2] *= np.float32(1e-3)
    h[4] *= np.float32(1e20)
    big = np.float32(3e38 / d * 4)
    dy[0] = np.sign(h[0]) * big
    dy[2] = np.sign(h[2]) * np.float32(1e35)
    h[2, :8] = np.float32(1e5)                       # the products here leave the range, the mean is far above eps
    dy[4] *= np.float32(1e25)
    dy[6] = np.sign(h[6]) * big
    ws, dx, dw = space(ae.model_rms_norm_backward_workspace(9, d, ae.AE_F32)), torch.empty((9, d), device="cuda"), torch.empty(d, device="cuda")
    ae.model_rms_norm_backward(dev(dy), dev(h), 9, d, None, 1e-6, dx, dw, ws)
    want, d_w, mag, mag_w = to.rms_norm_backward(dy, h, None, 1e-6)
    near(host(dx), want, grad_bound(want, mag, d, "f32"))
    near(host(dw), d_w, (9 + 45 + d / 2048) * U * mag_w + TINY)
    # an infinity and a NaN among gradients of rows whose mean of squares is as small as eps
    h = (rng.standard_normal((9, d)) * 1e-3).astype(np.float32)
    dy = rng.standard_normal((9, d)).astype(np.float32)
    _, d_w, _, mag_w = to.rms_norm_backward(dy, h, None, 1e-6)
    dy[3, 5], dy[7, d - 1] = np.inf, np.nan
    ae.model_rms_norm_backward(dev(dy), dev(h), 9, d, None, 1e-6, dx, dw, ws)
    other = np.ones(d, bool)
    other[[5, d - 1]] = False
    near(host(dw)[other], d_w[other], (9 + 45 + d / 2048) * U * mag_w[other] + TINY)
    assert np.isinf(host(dw)[5]) and np.isnan(host(dw)[d - 1])
    fine = [0, 1, 2, 4, 5, 6, 8]
    want, _, mag, _ = to.rms_norm_backward(dy[fine], h[fine], None, 1e-6)
    near(host(dx)[fine], want, grad_bound(want, mag, d, "f32"))


def test_backward_against_differences_of_the_forward_pass():
    """In binary32: differences over 2^-4, whose error is of third order in it and the forward pass's rounding over it."""
    import torch
    from paper_2602_17681_amd import binding as ae
    rows, d, t = 3, 40, 2.0 ** -4
    rng, x, r, w = inputs(rows, d, "f32", 5)
    dy = rng.standard_normal((rows, d))
    ws, dx, dw = space(ae.model_rms_norm_backward_workspace(rows, d, ae.AE_F32)), torch.empty((rows, d), device="cuda"), torch.empty(d, device="cuda")
    ae.model_rms_norm_backward(dev(dy.astype(np.float32)), dev(x), rows, d, dev(w), EPS, dx, dw, ws)

    def loss(x, w):
        y = torch.empty((rows, d), device="cuda")
        ae.model_rms_norm(dev(x.astype(np.float32)), rows, d, dev(w.astype(np.float32)), EPS, y=y)
        return (host(y) * dy.astype(np.float32)).sum()
    for i in [(0, 0), (1, 17), (2, 39)]:
        e = np.zeros((rows, d))
        e[i] = t
        # a row's rms is 1 to 4 here: third derivatives of y stay below 3 sum |dy| / rms^3
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * t) - host(dx)[i]) <= t * t / 6 * 3 * np.abs(dy[i[0]]).sum() + 100 * U * np.abs(dy).sum() * 20 / t
    for j in (0, 31):
        e = np.zeros(d)
        e[j] = t
        assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * t) - host(dw)[j]) <= 100 * U * np.abs(dy).sum() * 20 / t


def test_no_rows():
    import torch
    from paper_2602_17681_amd import binding as ae
    x = torch.empty((0, 50), device="cuda")
    ae.model_rms_norm(x, 0, 50, None, EPS, y=x)
    dw = torch.full((50,), 3.0, device="cuda")
    assert ae.model_rms_norm_backward_workspace(0, 50, ae.AE_F32) == 0
    ae.model_rms_norm_backward(x, x, 0, 50, None, EPS, None, dw, None)
    assert bool((dw == 0).all())


@pytest.mark.parametrize("rows,d", [(300, 1000), (70, 4096), (5, 40000)])
def test_streams_and_graphs(rows, d):
    import torch
    from paper_2602_17681_amd import binding as ae
    sets = [inputs(rows, d, "bf16", i) for i in range(3)]
    x, r, w = dev(sets[0][1], "bf16"), dev(sets[0][2], "bf16"), dev(sets[0][3])
    h, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(d, device="cuda")
    q, s = torch.empty((rows, -(-d // 16) * 16), dtype=torch.uint8, device="cuda"), torch.empty((-(-d // 128), rows), device="cuda")
    ws = space(ae.model_rms_norm_backward_workspace(rows, d, ae.AE_BF16))

    def step():
        ae.model_rms_norm(x, rows, d, w, EPS, h=h, q=q[:, :d], scale=s, residual=r)
        ae.model_rms_norm_backward(r, h, rows, d, w, EPS, dx, dw, ws, d_h=x)

    def change(i):
        x.copy_(dev(sets[i][1], "bf16"))
        r.copy_(dev(sets[i][2], "bf16"))
    outs = [h, q, s, dx, dw]
    for i, got in enumerate(replayed(step, outs, change)):
        change(i)
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, outs):
            assert torch.equal(a[:, :d] if a is got[1] else a, b[:, :d] if b is q else b)
