"""Norms and lookups of calls that move more than 96 MB, which read and write as a stream: every number of lanes to a row in both types, widths on
16-byte borders and off them.  The references are torch's operations in 64 bits on the GPU; bounds as in the tests of ordinary sizes."""
import pytest

from token_util import U

pytestmark = pytest.mark.gpu
STREAM = 96 << 20
EPS = 1e-5
TINY = 1e-37
DTYPE = {"f32": "float32", "bf16": "bfloat16"}
WIDTHS = [5, 64, 67, 128, 133, 256, 301, 512, 771, 1024, 1501, 2048, 2500, 4096, 5003, 8192, 9000, 12288, 13001, 16384]


def parts(rows, d):
    step = max(1, (1 << 22) // d)
    return [slice(i, min(i + step, rows)) for i in range(0, rows, step)]


def normal(gen, rows, d, t):
    import torch
    return torch.randn((rows, d), generator=gen, device="cuda").to(t)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_norm(d, dtype):
    import torch
    from paper_2602_17681_amd import binding as ae
    t, es = getattr(torch, DTYPE[dtype]), 4 if dtype == "f32" else 2
    rows = STREAM // (d * (4 * es + 1)) + 333
    gen = torch.Generator(device="cuda").manual_seed(d)
    x, r, w = normal(gen, rows, d, t), normal(gen, rows, d, t), 1 + 0.2 * torch.randn(d, generator=gen, device="cuda")
    y, first = torch.empty_like(x), r.clone()
    q, s = torch.full((rows, -(-d // 16) * 16), 0x55, dtype=torch.uint8, device="cuda"), torch.empty((-(-d // 128), rows), device="cuda")
    ae.model_rms_norm(x, rows, d, w, EPS, h=r, y=y, q=q[:, :d], scale=s, residual=r)          # h in the residual's place
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    column = torch.arange(d, device="cuda") // 128
    for p in parts(rows, d):
        h = x[p].double() + first[p].double()
        want = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * w.double()
        assert bool(((r[p].double() - h).abs() <= (half or U) * h.abs() + 1e-43).all())
        assert bool(((y[p].double() - want).abs() <= ((36 + d / 2048) * U + half) * want.abs() + TINY).all())
        scale = s[:, p].t().double()[:, column]
        assert bool(((q[p, :d].contiguous().view(torch.float8_e4m3fn).double() * scale - want).abs() <= 2.0 ** -4 * (1 + 2.0 ** -10) * want.abs() + scale * 2.0 ** -10).all())
    assert bool((q[:, d:] == 0x55).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_norm_backward(d, dtype):
    import torch
    from paper_2602_17681_amd import binding as ae
    t, es = getattr(torch, DTYPE[dtype]), 4 if dtype == "f32" else 2
    rows = STREAM // (d * 4 * es) + 333
    gen = torch.Generator(device="cuda").manual_seed(d)
    h, dy, add, w = normal(gen, rows, d, t), normal(gen, rows, d, t), normal(gen, rows, d, t), 1 + 0.2 * torch.randn(d, generator=gen, device="cuda")
    dx, dw = torch.empty_like(h), torch.empty(d, device="cuda")
    ws = torch.full((ae.model_rms_norm_backward_workspace(rows, d, ae.DTYPES[dtype]),), 255, dtype=torch.uint8, device="cuda")
    ae.model_rms_norm_backward(dy, h, rows, d, w, EPS, dx, dw, ws, d_h=add)
    half = 2.0 ** -8 if dtype == "bf16" else U
    total, mag = (torch.zeros(d, dtype=torch.float64, device="cuda") for _ in range(2))
    for p in parts(rows, d):
        hh, g = h[p].double(), dy[p].double() * w.double()
        r = torch.rsqrt((hh * hh).mean(1, keepdim=True) + EPS)
        u = hh * r
        want = add[p].double() + r * (g - u * (g * u).mean(1, keepdim=True))
        bound = add[p].double().abs() + r * (g.abs() + u.abs() * (g * u).abs().mean(1, keepdim=True))
        assert bool(((dx[p].double() - want).abs() <= (130 + d / 512) * U * bound + half * want.abs() + TINY).all())
        total += (dy[p].double() * u).sum(0)
        mag += (dy[p].double() * u).abs().sum(0)
    # a workgroup's lanes add up at most rows / 256 rows one after the other, then come up to 31 + 8 + 4 + 4 additions of what they have
    assert bool(((dw.double() - total).abs() <= (rows / 256 + 1 + 47 + 45 + d / 2048) * U * mag).all())


@pytest.mark.parametrize("d", [515, 2056, 3001])
def test_lookup_in_binary32(d):
    import torch
    from paper_2602_17681_amd import binding as ae
    n, vocab = STREAM // (8 * d) + 1100, 700
    gen = torch.Generator(device="cuda").manual_seed(d)
    table = torch.randn((vocab, d), generator=gen, device="cuda")
    ids = torch.randint(-1, vocab + 1, (n,), generator=gen, device="cuda").to(torch.int32)
    out = torch.empty((n, d), device="cuda")
    ae.model_embedding(table, vocab, d, ids, n, out, scale=1.25)
    want = torch.where(((ids >= 0) & (ids < vocab))[:, None], (table * 1.25)[ids.clamp(0, vocab - 1).long()], torch.zeros((), device="cuda"))
    assert torch.equal(out, want)
