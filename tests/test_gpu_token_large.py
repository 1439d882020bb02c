"""Norms, embeddings, clipping and adjusted logits where a launch does not take all workgroups, and where offsets pass 32 bits.  The references are torch's
operations in 64 bits on the GPU, in parts; bounds as in the tests of each call."""
import pytest

from token_util import U

pytestmark = pytest.mark.gpu


def test_norm_of_more_rows_than_one_round_takes():
    """2^20 workgroups of 32 rows each, rows shorter than a piece."""
    import torch
    from paper_2602_17681_amd import binding as ae
    rows, d = (1 << 25) + 21, 3
    x = torch.randn((rows, d), device="cuda").to(torch.bfloat16)
    y = torch.empty_like(x)
    ae.model_rms_norm(x, rows, d, None, 1e-5, y=y)
    want = x.double() * torch.rsqrt((x.double() ** 2).mean(1, keepdim=True) + 1e-5)
    assert bool(((y.double() - want).abs() <= (2.0 ** -8 + 40 * U) * want.abs() + 1e-37).all())


def test_norm_of_rows_beyond_32_bits():
    """A row to a workgroup, several rounds of them, more than 2^31 elements; the backward pass of the same."""
    import torch
    from paper_2602_17681_amd import binding as ae
    rows, d = (1 << 20) + 300, 2100
    x = torch.randn((rows, d), device="cuda", dtype=torch.bfloat16)
    w = 1 + 0.1 * torch.randn(d, device="cuda")
    y = torch.empty_like(x)
    q, s = torch.empty((rows, 2112), dtype=torch.uint8, device="cuda")[:, :d], torch.empty((17, rows), device="cuda")
    ae.model_rms_norm(x, rows, d, w, 1e-5, y=y, q=q, scale=s)
    for part in (slice(0, 1000), slice(rows // 2, rows // 2 + 1000), slice(rows - 1000, rows)):
        h = x[part].double()
        want = h * torch.rsqrt((h * h).mean(1, keepdim=True) + 1e-5) * w.double()
        assert bool(((y[part].double() - want).abs() <= (2.0 ** -8 + 40 * U) * want.abs() + 1e-37).all())
        scale = s[:, part].t().double()[:, torch.arange(d, device="cuda") // 128]
        assert bool(((q[part].contiguous().view(torch.float8_e4m3fn).double() * scale - want).abs() <= 2.0 ** -4 * 1.001 * want.abs() + scale * 2.0 ** -10).all())
    del q, s
    dw = torch.empty(d, device="cuda")
    ws = torch.empty(ae.model_rms_norm_backward_workspace(rows, d, ae.AE_BF16), dtype=torch.uint8, device="cuda")
    ae.model_rms_norm_backward(x, x, rows, d, w, 1e-5, y, dw, ws)             # the gradient is the input itself
    total, mag = torch.zeros(d, dtype=torch.float64, device="cuda"), torch.zeros(d, dtype=torch.float64, device="cuda")
    for h in x.split(1 << 17):
        h = h.double()
        u = h * torch.rsqrt((h * h).mean(1, keepdim=True) + 1e-5)
        total += (h * u).sum(0)
        mag += (h * u).abs().sum(0)
    # a workgroup adds up to ceil(rows / 512) rows one after the other, then come 8 + 4 + 4 additions of the parts
    assert bool(((dw.double() - total).abs() <= (rows / 512 + 1 + 16 + 45) * U * mag).all())
    h = x[-500:].double()
    r = torch.rsqrt((h * h).mean(1, keepdim=True) + 1e-5)
    g = h * w.double()
    want = r * (g - h * r * (g * h * r).mean(1, keepdim=True))
    bound = r * (g.abs() + (h * r).abs() * (g * h * r).abs().mean(1, keepdim=True))
    assert bool(((y[-500:].double() - want).abs() <= 140 * U * bound + 2.0 ** -8 * want.abs() + 1e-37).all())


def test_embedding_of_more_tokens_than_one_launch_takes():
    import torch
    from paper_2602_17681_amd import binding as ae
    n, vocab = (1 << 28) + 333, 1000
    table = torch.randn((vocab, 1), device="cuda").to(torch.bfloat16)
    ids = torch.randint(-1, vocab + 1, (n,), device="cuda", dtype=torch.int32)
    out = torch.empty((n, 1), dtype=torch.bfloat16, device="cuda")
    ae.model_embedding(table, vocab, 1, ids, n, out)
    for a, b in zip(ids.split(1 << 26), out.split(1 << 26)):
        want = torch.where((a >= 0) & (a < vocab), table[a.clamp(0, vocab - 1).long(), 0], torch.zeros((), dtype=torch.bfloat16, device="cuda"))
        assert torch.equal(b[:, 0], want)


@pytest.mark.parametrize("d", [2056, 3001])
def test_embedding_of_calls_that_write_as_a_stream(d):
    import torch
    from paper_2602_17681_amd import binding as ae
    n, vocab = 20000, 700
    table = torch.randn((vocab, d), device="cuda").to(torch.bfloat16)
    ids = torch.randint(-1, vocab + 1, (n,), device="cuda", dtype=torch.int32)
    out = torch.empty((n, d), dtype=torch.bfloat16, device="cuda")
    ae.model_embedding(table, vocab, d, ids, n, out, scale=1.25)
    want = torch.where(((ids >= 0) & (ids < vocab))[:, None], (table.float() * 1.25).to(torch.bfloat16)[ids.clamp(0, vocab - 1).long()], torch.zeros((), dtype=torch.bfloat16, device="cuda"))
    assert torch.equal(out, want)


def test_embedding_and_gradient_beyond_32_bits():
    import torch
    from paper_2602_17681_amd import binding as ae
    n, vocab, d = 3000, 1 << 20, 2100
    table = torch.randn((vocab, d), device="cuda", dtype=torch.bfloat16)
    ids = torch.randint(0, vocab, (n,), device="cuda", dtype=torch.int32)
    ids[:1000] = vocab - 1 - torch.arange(1000, device="cuda", dtype=torch.int32) % 7
    out = torch.empty((n, d), dtype=torch.bfloat16, device="cuda")
    ae.model_embedding(table, vocab, d, ids, n, out, scale=2.0)
    assert torch.equal(out, table[ids.long()] * 2)
    del table
    grad = torch.full((vocab, d), 1.0, device="cuda")
    ws = torch.empty(ae.model_embedding_backward_workspace(n, vocab, d, ae.AE_BF16), dtype=torch.uint8, device="cuda")
    for accumulate in (True, False):
        ae.model_embedding_backward(out, ids, n, vocab, d, grad, ws, scale=0.5, accumulate=accumulate)
        tokens, at = ids.long().unique(return_inverse=True)
        want = torch.zeros((len(tokens), d), dtype=torch.float64, device="cuda").index_add_(0, at, out.double() * 0.5)
        mag = torch.zeros((len(tokens), d), dtype=torch.float64, device="cuda").index_add_(0, at, out.double().abs() * 0.5)
        count = torch.bincount(at)[:, None]
        base = 1.0 if accumulate else 0.0
        assert bool(((grad[tokens].double() - want - base).abs() <= (count + 3) * U * mag + U * (want.abs() + base)).all())
        other = torch.ones(vocab, dtype=torch.bool, device="cuda")
        other[tokens] = False
        assert all(bool((g[o] == base).all()) for g, o in zip(grad.split(1 << 17), other.split(1 << 17)))


def test_clip_of_a_tensor_beyond_32_bits():
    import torch
    from paper_2602_17681_amd import binding as ae
    n = (1 << 31) + 12345
    g, small = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda"), torch.full((7,), 3.0, device="cuda")
    lst, norm = ae.GradList([small, g], [small, g]), torch.empty(1, device="cuda")
    ws = torch.empty(ae.model_grad_clip_workspace(lst), dtype=torch.uint8, device="cuda")
    exact = (n * 0.25 + 63.0) ** 0.5
    ae.model_grad_clip(lst, exact / 4, norm, ws)
    assert abs(norm.item() - exact) <= 1.001 * U * exact
    assert bool((g == 0.125).all()) and abs(small[6].item() - 0.75) <= 3 * U


def test_logits_of_more_rows_than_one_launch_takes():
    import torch
    from paper_2602_17681_amd import binding as ae
    rows, vocab = (1 << 23) + 77, 4
    z = torch.randn((rows, vocab), device="cuda").to(torch.bfloat16)
    history = torch.randint(-1, vocab + 1, (rows, 1), device="cuda", dtype=torch.int32)
    allowed = torch.randint(0, 16, (rows, 1), device="cuda", dtype=torch.int32)
    out = torch.empty_like(z)
    ae.model_logits_adjust(z, rows, vocab, out, history=history, presence=torch.full((rows,), 0.5, device="cuda"), allowed=allowed)
    at = torch.arange(vocab, device="cuda", dtype=torch.int32)
    want = torch.where(history == at, z.float() - 0.5, z.float()).to(torch.bfloat16)
    want = torch.where(allowed >> at & 1 == 1, want, torch.full((), float("-inf"), dtype=torch.bfloat16, device="cuda"))
    assert torch.equal(out, want)


def test_logits_beyond_32_bits():
    import torch
    from paper_2602_17681_amd import binding as ae
    rows, vocab, ld = 2100, 5000, 1 << 20
    buf = torch.zeros((rows, ld), dtype=torch.bfloat16, device="cuda")
    z = buf[:, :vocab]
    z.copy_(torch.randn((rows, vocab), device="cuda"))
    before = z.clone()
    ids = torch.randint(0, vocab, (rows, 1), device="cuda", dtype=torch.int32)
    ae.model_logits_adjust(z, rows, vocab, z, bias_id=ids, bias=torch.full((rows, 1), 2.0, device="cuda"))
    want = before.float().scatter_add(1, ids.long(), torch.full((rows, 1), 2.0, device="cuda")).to(torch.bfloat16)
    assert torch.equal(z, want) and not bool(buf[:, vocab:vocab + 4096].any())
