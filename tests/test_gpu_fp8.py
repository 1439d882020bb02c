"""The quantiser to E4M3 codes with a scale for each block of 128, the product of such matrices and the linear layer made
of both, against the oracle: codes and scales equal, products within bounds derived from the number of roundings."""
import numpy as np
import pytest

from oracle import fp8_oracle as fo

pytestmark = pytest.mark.gpu


def dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def room(rows, cols, extra=0):
    """Codes with rows on 16-byte borders in a buffer full of a marker."""
    import torch
    ld = -(-cols // 16) * 16 + 16 * extra
    buf = torch.full((rows, ld), 0x5A, dtype=torch.uint8, device="cuda")
    return buf, buf[:, :cols]


def same_codes(got, want):
    g, w = fo.VALUES[got], fo.VALUES[want]
    return np.array_equal(np.isnan(g), np.isnan(w)) and np.array_equal(got[~np.isnan(w)], want[~np.isnan(w)])


def source(rows, cols, dtype, seed, pad=0, offset=0):
    """(device matrix with a row stride of cols + pad that begins `offset` elements into its buffer, the same numbers in binary32)."""
    import torch
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1)) * 3) * np.where(rng.random(cols) < 0.05, 30, 1)).astype(np.float32)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    buf = torch.full((rows * (cols + pad) + offset,), 1e9, dtype=td, device="cuda")
    t = buf[offset:].view(rows, cols + pad)[:, :cols]
    t.copy_(dev(x))
    return t, t.float().cpu().numpy()


SIZES = [(1, 1), (1, 128), (3, 129), (127, 5), (128, 128), (129, 257), (200, 1003), (33, 16), (260, 384), (7, 2050)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("blocks", ["rows", "tiles"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_quantiser_equals_its_oracle(rows, cols, blocks, dtype):
    import torch
    from paper_2602_17681_amd import binding as ae
    for pad, offset, extra in ((0, 0, 0), (3, 1, 1)):
        x, xh = source(rows, cols, dtype, rows * 7 + cols, pad, offset)
        buf, q = room(rows, cols, extra)
        buft, qt = room(cols, rows, extra)
        shape = lambda r, c: (-(-c // 128), r) if blocks == "rows" else (-(-r // 128), -(-c // 128))      # noqa: E731
        s, st = torch.full(shape(rows, cols), -1.0, device="cuda"), torch.full(shape(cols, rows), -1.0, device="cuda")
        ae.model_fp8_quantize(x, rows, cols, blocks, q, s, qt, st)
        cw, sw = fo.quantize(xh, blocks)
        ct, stw = (cw.T, sw.T) if blocks == "tiles" else fo.quantize(xh.T, "rows")
        assert np.array_equal(s.cpu().numpy(), sw) and same_codes(q.cpu().numpy(), cw)
        assert np.array_equal(st.cpu().numpy(), stw) and same_codes(qt.cpu().numpy(), ct)
        assert bool((buf[:, cols:] == 0x5A).all()) and bool((buft[:, rows:] == 0x5A).all())
        # one orientation at a time
        _, q1 = room(rows, cols)
        _, qt1 = room(cols, rows)
        s1, st1 = torch.empty_like(s), torch.empty_like(st)
        ae.model_fp8_quantize(x, rows, cols, blocks, q1, s1)
        ae.model_fp8_quantize(x, rows, cols, blocks, None, None, qt1, st1)
        assert torch.equal(q1, q) and torch.equal(s1, s) and torch.equal(qt1, qt) and torch.equal(st1, st)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantiser_of_unusual_numbers(dtype):
    """Zeros, subnormals, the largest numbers, infinities and NaN: what is not finite has no part in the scale."""
    import torch
    from paper_2602_17681_amd import binding as ae
    rows, cols = 9, 256
    x = np.random.default_rng(0).standard_normal((rows, cols)).astype(np.float32)
    x[0], x[1], x[2] = 0.0, 1e-40, 3e38
    x[3, 5], x[4, 7], x[5, 9], x[5, 10] = np.inf, -np.inf, np.nan, np.inf
    x[6], x[7, :128] = np.nan, np.inf
    x[8] = -0.0
    t = dev(x, torch.bfloat16 if dtype == "bf16" else torch.float32)
    for blocks in ("rows", "tiles"):
        _, q = room(rows, cols)
        s = torch.empty((2, rows) if blocks == "rows" else (1, 2), device="cuda")
        ae.model_fp8_quantize(t, rows, cols, blocks, q, s)
        cw, sw = fo.quantize(t.float().cpu().numpy(), blocks)
        assert np.array_equal(s.cpu().numpy(), sw) and same_codes(q.cpu().numpy(), cw)


def product_bound(mag, ref, k, dtype):
    """binary32: 128 products of a block summed (at most 2^-23 of the magnitudes each), block sums scaled and added (3 roundings
    and one per block).  bfloat16: the 8-bit instruction cuts each of eight products off 2^-13 below the largest of them, and
    the result is rounded once."""
    kb = -(-k // 128)
    err = mag * ((128 + 4) * 2.0 ** -23 + kb * 2.0 ** -24)
    return err if dtype == "f32" else err + mag * 2.0 ** -10 + 2.0 ** -8 * (np.abs(ref) + mag * 2.0 ** -10)


def operands(m, n, k, b_blocks, seed):
    rng = np.random.default_rng(seed)
    a, sa = fo.quantize((rng.standard_normal((m, k)) * np.where(rng.random(k) < 0.05, 30, 1)).astype(np.float32))
    b, sb = fo.quantize(rng.standard_normal((n, k)).astype(np.float32), b_blocks)
    return a, sa, b, sb, rng.standard_normal(n).astype(np.float32)


def run_product(a, sa, b, sb, b_blocks, bias, dtype, pad=0):
    import torch
    from paper_2602_17681_amd import binding as ae
    (m, k), n = a.shape, b.shape[0]
    bufs = []
    for codes in (a, b):
        buf, q = room(*codes.shape, pad)
        buf.fill_(0x7F)                                    # NaN codes between the rows: never used
        q.copy_(dev(codes))
        bufs.append(q)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    out = torch.full((m + 1, n + 3), 7.0, dtype=td, device="cuda")
    y = out[:m, :n]
    ws = torch.full((max(1, ae.model_fp8_matmul_workspace(m, n, k)),), 0xFF, dtype=torch.uint8, device="cuda")
    ae.model_fp8_matmul(bufs[0], dev(sa), bufs[1], dev(sb), b_blocks, None if bias is None else dev(bias), m, n, k, y, ws)
    assert bool((out[m] == 7.0).all()) and bool((out[:, n:] == 7.0).all())
    return y.double().cpu().numpy()


# few rows and many, sides below, at and above tiles of 16, 64, 128 and 256, K of one block and less, of no whole 16 bytes,
# of many blocks; narrow results with long sums
SHAPES = [(1, 1, 1), (1, 16, 128), (1, 4096, 512), (2, 77, 1000), (5, 300, 4113), (15, 130, 256), (16, 128, 128), (17, 129, 140), (16, 64, 8192),
          (33, 200, 333), (64, 256, 640), (65, 96, 1024), (100, 1500, 257), (128, 128, 384), (129, 384, 129), (255, 257, 300), (256, 256, 256),
          (256, 512, 1024), (300, 130, 2048), (513, 260, 127), (777, 300, 1003), (1024, 1024, 512), (2050, 257, 272), (40, 4000, 1536)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("b_blocks", ["tiles", "rows"])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product_against_64_bits(m, n, k, b_blocks, dtype):
    a, sa, b, sb, bias = operands(m, n, k, b_blocks, m + 3 * n + 7 * k)
    for bi, pad in ((None, 0), (bias, 1)):
        ref, mag = fo.matmul(a, sa, b, sb, b_blocks, bi)
        y = run_product(a, sa, b, sb, b_blocks, bi, dtype, pad)
        assert np.all(np.abs(y - ref) <= product_bound(mag, ref, k, dtype))


@pytest.mark.parametrize("m,n", [(1, 20), (16, 64), (40, 70), (200, 300), (300, 520)])
def test_binary32_results_keep_small_products(m, n):
    """One product of 2^16 among 127 of 1: every sum is an integer below 2^24, so a binary32 result is exact."""
    a = np.full((m, 256), fo.encode(1.0), np.uint8)
    a[:, 5] = a[:, 200] = fo.encode(256.0)
    b = np.full((n, 256), fo.encode(1.0), np.uint8)
    b[:, 5] = b[:, 200] = fo.encode(256.0)
    for b_blocks in ("tiles", "rows"):
        sb = np.ones((-(-n // 128), 2) if b_blocks == "tiles" else (2, n), np.float32)
        y = run_product(a, np.ones((2, m), np.float32), b, sb, b_blocks, None, "f32")
        assert np.all(y == 2 * (65536 + 127))


def test_nan_codes_stay_in_their_rows():
    a, sa, b, sb, _ = operands(70, 90, 300, "tiles", 3)
    a[7, 130] = 0x7F
    b[11, 299] = 0xFF
    for dtype in ("bf16", "f32"):
        y = run_product(a, sa, b, sb, "tiles", None, dtype)
        want = np.zeros((70, 90), bool)
        want[7], want[:, 11] = True, True
        assert np.array_equal(np.isnan(y), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(1, 300, 1003), (1, 512, 4096), (3, 64, 128), (8, 1000, 640), (16, 272, 2064), (17, 500, 384), (31, 129, 200), (130, 260, 300), (600, 256, 512)])
def test_linear_is_quantiser_and_product(m, n, k, dtype):
    import torch
    from paper_2602_17681_amd import binding as ae
    for pad, offset, with_bias in ((0, 0, False), (5, 1, True)):
        x, xh = source(m, k, dtype, m + n + k, pad, offset)
        rng = np.random.default_rng(k)
        w, sw = fo.quantize(rng.standard_normal((n, k)).astype(np.float32) * k ** -0.5, "tiles")
        bias = rng.standard_normal(n).astype(np.float32) if with_bias else None
        _, q = room(n, k)
        q.copy_(dev(w))
        y = torch.empty((m, n), dtype=x.dtype, device="cuda")
        ws = torch.full((ae.model_fp8_linear_workspace(m, n, k) + 16,), 0xFF, dtype=torch.uint8, device="cuda")
        ae.model_fp8_linear(x, q, dev(sw), None if bias is None else dev(bias), m, n, k, y, ws)
        a, sa = fo.quantize(xh)
        ref, mag = fo.matmul(a, sa, w, sw, "tiles", bias)
        assert np.all(np.abs(y.double().cpu().numpy() - ref) <= product_bound(mag, ref, k, dtype))


def test_linear_of_unusual_rows():
    """A row of zeros, one with NaN, one with an infinity among few rows (one launch) and many."""
    import torch
    from paper_2602_17681_amd import binding as ae
    n, k = 96, 300
    rng = np.random.default_rng(9)
    w, sw = fo.quantize(rng.standard_normal((n, k)).astype(np.float32), "tiles")
    _, q = room(n, k)
    q.copy_(dev(w))
    for m in (4, 40):
        xh = rng.standard_normal((m, k)).astype(np.float32)
        xh[0], xh[1, 299], xh[2, 3] = 0, np.nan, np.inf
        x = dev(xh)
        y = torch.empty((m, n), device="cuda")
        ws = torch.empty(ae.model_fp8_linear_workspace(m, n, k) + 16, dtype=torch.uint8, device="cuda")
        ae.model_fp8_linear(x, q, dev(sw), None, m, n, k, y, ws)
        a, sa = fo.quantize(xh)
        ref, mag = fo.matmul(a, sa, w, sw)
        got = y.double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.all(got[0] == 0)
        ok = ~np.isnan(ref)
        assert np.all(np.abs(got - ref)[ok] <= product_bound(mag, ref, k, "f32")[ok])


def test_backward_products_are_the_gradients():
    """With L = sum dY * Y: dX from dY and the transposed codes of W, dW from the transposed codes of dY and X, each against
    the formula in 64 bits and against differences of the forward product (which is linear in either factor)."""
    import torch
    from paper_2602_17681_amd import binding as ae
    m, n, k = 150, 140, 260
    rng = np.random.default_rng(12)
    x, w, dy = (rng.standard_normal(s).astype(np.float32) for s in ((m, k), (n, k), (m, n)))
    shape = lambda r, c: torch.empty((-(-c // 128), r), device="cuda")      # noqa: E731
    dq, dqt, xt = room(m, n)[1], room(n, m)[1], room(k, m)[1]
    ds, dst, xts = shape(m, n), shape(n, m), shape(k, m)
    ae.model_fp8_quantize(dev(dy), m, n, "rows", dq, ds, dqt, dst)
    ae.model_fp8_quantize(dev(x), m, k, "rows", None, None, xt, xts)
    wq, wt = room(n, k)[1], room(k, n)[1]
    wsc, wtsc = torch.empty((2, 3), device="cuda"), torch.empty((3, 2), device="cuda")
    ae.model_fp8_quantize(dev(w), n, k, "tiles", wq, wsc, wt, wtsc)
    dx, dw = torch.empty((m, k), device="cuda"), torch.empty((n, k), device="cuda")
    ws = torch.empty(max(16, ae.model_fp8_matmul_workspace(m, k, n), ae.model_fp8_matmul_workspace(n, k, m)), dtype=torch.uint8, device="cuda")
    ae.model_fp8_matmul(dq, ds, wt, wtsc, "tiles", None, m, k, n, dx, ws)
    ae.model_fp8_matmul(dqt, dst, xt, xts, "rows", None, n, k, m, dw, ws)
    vdy, vdyt, vxt = fo.values(*fo.quantize(dy)), fo.values(*fo.quantize(dy.T)), fo.values(*fo.quantize(x.T))
    vw = fo.values(*fo.quantize(w, "tiles"), "tiles")
    for got, a, b in ((dx, vdy, vw), (dw, vdyt, vxt.T)):
        ref, mag = a @ b, np.abs(a) @ np.abs(b)
        assert np.all(np.abs(got.double().cpu().numpy() - ref) <= product_bound(mag, ref, max(m, n), "f32"))
    gx, gw = dx.double().cpu().numpy(), dw.double().cpu().numpy()
    for _ in range(3):
        d = rng.standard_normal((m, k))
        diff = ((vdy * ((x + d) @ vw.T)).sum() - (vdy * ((x - d) @ vw.T)).sum()) / 2
        assert abs((gx * d).sum() - diff) <= 1e-4 * np.abs(gx * d).sum()
        d = rng.standard_normal((n, k))
        diff = ((vdyt.T * (vxt.T @ (vw + d).T)).sum() - (vdyt.T * (vxt.T @ (vw - d).T)).sum()) / 2
        assert abs((gw * d).sum() - diff) <= 1e-4 * np.abs(gw * d).sum()


def test_no_work_and_repeatability():
    import torch
    from paper_2602_17681_amd import binding as ae
    e = torch.empty((0, 64), device="cuda")
    ae.model_fp8_linear(e, room(32, 64)[1], torch.ones((1, 1), device="cuda"), None, 0, 32, 64, torch.empty((0, 32), device="cuda"), torch.empty(16, dtype=torch.uint8, device="cuda"))
    ae.model_fp8_quantize(e, 0, 64, "rows", torch.empty((0, 64), dtype=torch.uint8, device="cuda"), torch.empty((1, 0), device="cuda"))
    a, sa, b, sb, bias = operands(16, 96, 5000, "tiles", 1)
    first = run_product(a, sa, b, sb, "tiles", bias, "f32")
    for _ in range(3):
        assert np.array_equal(first, run_product(a, sa, b, sb, "tiles", bias, "f32"))


@pytest.mark.parametrize("m", [1, 64, 700])
def test_other_streams_and_captured_graphs(m):
    """On a stream of the caller's own, and replayed from a captured graph with new inputs: the same bits as eager calls."""
    import torch
    from paper_2602_17681_amd import binding as ae
    n, k = 384, 1024
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    w = torch.randn((n, k), device="cuda", generator=gen)
    q, s = torch.empty((n, k), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((3, 8), device="cuda")
    ae.model_fp8_quantize(w, n, k, "tiles", q, s)
    x = torch.randn((m, k), device="cuda", generator=gen).bfloat16()
    ws = torch.empty(ae.model_fp8_linear_workspace(m, n, k) + 16, dtype=torch.uint8, device="cuda")
    y = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    call = lambda: ae.model_fp8_linear(x, q, s, None, m, n, k, y, ws)      # noqa: E731
    call()
    eager = y.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y.zero_()
        call()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        x.copy_(torch.randn((m, k), device="cuda", generator=gen).bfloat16())
        call()
        eager = y.clone()
        y.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, eager)
