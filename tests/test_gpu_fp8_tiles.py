"""Products of many rows, at sizes where each tile shape runs, against 64 bits on the device."""
import pytest

pytestmark = pytest.mark.gpu


def operand(rows, cols, blocks, gen, outliers):
    """(codes on 16-byte rows, scales, values in binary64)."""
    import torch
    ld = -(-cols // 16) * 16
    buf = torch.full((rows, ld), 0x7F, dtype=torch.uint8, device="cuda")         # NaN codes between the rows
    q = buf[:, :cols]
    x = torch.randn((rows, cols), generator=gen, device="cuda") * 60
    if outliers:
        x *= torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.02, 7.0, 1.0)
    q.copy_(x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    rb, cb = -(-rows // 128), -(-cols // 128)
    s = torch.rand((cb, rows) if blocks == "rows" else (rb, cb), generator=gen, device="cuda") + 0.5
    per = s.t() if blocks == "rows" else s.repeat_interleave(128, 0)[:rows]
    v = q.contiguous().view(torch.float8_e4m3fn).double() * per.double().repeat_interleave(128, 1)[:, :cols]
    return q, s, v


# 192 tiles and more of 256 x 256 (bfloat16 and tiles) or 256 x 128 (the others), with edges in both directions, K of one
# block, of less, of no whole 16 bytes, of many blocks; and products that stay with 128 x 128
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("b_blocks", ["tiles", "rows"])
@pytest.mark.parametrize("m,n,k", [(4096, 4096, 256), (3333, 4100, 300), (8200, 1700, 130), (2050, 7000, 97), (3073, 4097, 16), (4001, 4000, 1040), (256 * 192, 200, 144),
                                   (100, 256 * 96, 384), (1024, 1500, 777), (1000, 520, 1001)])
def test_tiles_against_64_bits(m, n, k, b_blocks, dtype):
    import torch
    from paper_2602_17681_amd import binding as ae
    gen = torch.Generator(device="cuda")
    gen.manual_seed(m + n + k)
    a, sa, va = operand(m, k, "rows", gen, True)
    b, sb, vb = operand(n, k, b_blocks, gen, False)
    bias = torch.randn(n, generator=gen, device="cuda")
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    guard = torch.full((m + 1, n), 7.0, dtype=td, device="cuda")
    y = guard[:m]
    ws = torch.empty(max(16, ae.model_fp8_matmul_workspace(m, n, k)), dtype=torch.uint8, device="cuda")
    ae.model_fp8_matmul(a, sa, b, sb, b_blocks, bias, m, n, k, y, ws)
    vbt = vb.t().contiguous()
    ref = va @ vbt + bias.double()
    mag = va.abs() @ vbt.abs() + bias.abs().double()
    # binary32: 128 products of a block (at most 2^-23 of the magnitudes each), block sums scaled and added; bfloat16: the 8-bit
    # instruction cuts each of eight products off 2^-13 below the largest of them, and the result is rounded once
    err = mag * ((128 + 4) * 2.0 ** -23 + -(-k // 128) * 2.0 ** -24)
    if dtype == "bf16":
        err = err + mag * 2.0 ** -10 + 2.0 ** -8 * (ref.abs() + mag * 2.0 ** -10)
    assert bool(((y.double() - ref).abs() <= err).all())
    assert bool((guard[m] == 7.0).all())
