"""Calls whose threads are more than one launch takes (2^32 - 1): many short rows, long narrow matrices."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [(1 << 23) + 5, 1 << 24])
def test_log_probabilities_of_many_rows(rows):
    import torch
    from paper_2602_17681_amd import binding as ae
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    z = (torch.randn((rows, 3), generator=gen, device="cuda") * 2).bfloat16()
    tokens = torch.randint(0, 3, (rows, 1), generator=gen, device="cuda", dtype=torch.int32)
    f = lambda *s: torch.full(s, -7.0, device="cuda")      # noqa: E731
    logprob, entropy, lse, top_logit, ids = f(rows, 1), f(rows), f(rows), f(rows, 2), torch.full((rows, 2), -7, dtype=torch.int32, device="cuda")
    ae.model_token_logprobs(z, rows, 3, tokens, 2, logprob, entropy, lse, ids, top_logit, None, None)
    logq = torch.log_softmax(z.double(), 1)
    assert bool(((lse.double() - torch.logsumexp(z.double(), 1)).abs() <= 1e-5).all())
    assert bool(((entropy.double() + (torch.exp(logq) * logq).sum(1)).abs() <= 1e-5).all())
    assert bool(((logprob.double() - logq.gather(1, tokens.long())).abs() <= 1e-5).all())
    s = torch.sort(z.float(), dim=1, descending=True, stable=True)
    assert torch.equal(ids.long(), s.indices[:, :2]) and torch.equal(top_logit, s.values[:, :2])


@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("rows", [(1 << 23) + 5, 1 << 24])
def test_distillation_of_many_rows(rows, grad):
    import torch
    from paper_2602_17681_amd import binding as ae
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    z = (torch.randn((rows, 3), generator=gen, device="cuda") * 2).bfloat16()
    ids = torch.randint(0, 3, (rows, 1), generator=gen, device="cuda", dtype=torch.int32)
    t = torch.zeros((rows, 1), device="cuda")
    ws = torch.empty(ae.model_loss_distill_workspace(rows, 3, ae.AE_BF16), dtype=torch.uint8, device="cuda")
    lr, total, g = torch.full((rows,), -7.0, device="cuda"), torch.full((1,), -7.0, device="cuda"), torch.full_like(z, 3.0)
    ae.model_loss_distill(z, rows, 3, ids, t, lr, total, g if grad else None, ws)
    logq = torch.log_softmax(z.double(), 1)
    want = -logq.gather(1, ids.long())[:, 0]
    assert bool(((lr.double() - want).abs() <= 1e-5).all())
    assert abs(total.item() - want.sum().item()) <= 1e-6 * want.sum().item()
    if grad:
        q = torch.exp(logq).scatter_add_(1, ids.long(), torch.full((rows, 1), -1.0, dtype=torch.float64, device="cuda"))
        assert bool(((g.double() - q).abs() <= 2.0 ** -8 * q.abs() + 1e-6).all())


def test_quantiser_of_a_long_narrow_matrix():
    import torch
    from paper_2602_17681_amd import binding as ae
    rows, cols = (1 << 29) + 37, 3
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    x.normal_(generator=gen)
    q = torch.full((rows, 16), 0x7F, dtype=torch.uint8, device="cuda")
    scale = torch.full((1, rows), -7.0, device="cuda")
    ae.model_fp8_quantize(x, rows, cols, "rows", q[:, :cols], scale)
    for at in (0, 1 << 28, (1 << 29) - 70, rows - 100):
        part = x[at:at + 100].contiguous()
        q1, s1 = torch.empty((100, 16), dtype=torch.uint8, device="cuda"), torch.empty((1, 100), device="cuda")
        ae.model_fp8_quantize(part, 100, cols, "rows", q1[:, :cols], s1)
        assert torch.equal(q[at:at + 100, :cols], q1[:, :cols]) and torch.equal(scale[:, at:at + 100], s1)
    assert bool((scale > 0).all()) and bool((q[:, cols:] == 0x7F).all())


@pytest.mark.parametrize("m,n,linear", [(1, (1 << 27) + 40, False), (17, (1 << 27) + 40, False), (2, (1 << 29) + 72, True)])
def test_products_with_many_columns(m, n, linear):
    """One block of K with codes of 1 and -1: the sums are small whole numbers, exact in bfloat16."""
    import torch
    from paper_2602_17681_amd import binding as ae
    k = 16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    one = 0x38                                             # the code of 1; with the sign's bit -1
    b = torch.randint(0, 2, (n, k), generator=gen, dtype=torch.uint8, device="cuda").mul_(0x80).add_(one)
    bs = torch.exp2(torch.randint(-3, 4, (-(-n // 128), 1), generator=gen, device="cuda").float())
    a = torch.randint(0, 2, (m, k), generator=gen, dtype=torch.uint8, device="cuda").mul_(0x80).add_(one)
    y = torch.full((m, n), -7.0, dtype=torch.bfloat16, device="cuda")
    av = torch.where(a >= 0x80, -1.0, 1.0)
    if linear:
        ae.model_fp8_linear(av.bfloat16(), b, bs, None, m, n, k, y)
    else:
        ae.model_fp8_matmul(a, torch.ones((1, m), device="cuda"), b, bs, "tiles", None, m, n, k, y)
    step = 1 << 22
    for at in range(0, n, step):
        e = min(n, at + step)
        want = (av @ torch.where(b[at:e] >= 0x80, -1.0, 1.0).t()) * bs[at // 128:-(-e // 128), 0].repeat_interleave(128)[:e - at]
        assert torch.equal(y[:, at:e].float(), want), at


def test_tiles_with_many_columns():
    """65 rows: tiles of 256 x 128, over 2^23 of them."""
    import torch
    from paper_2602_17681_amd import binding as ae
    m, n, k = 65, (1 << 30) + 72, 16
    if torch.cuda.mem_get_info()[0] < 180 << 30:
        pytest.skip("a result of 140 GB")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    b = torch.empty((n, k), dtype=torch.uint8, device="cuda").random_(0, 2, generator=gen).mul_(0x80).add_(0x38)
    bs = torch.exp2(torch.arange(n, device="cuda") % 5 - 2.0)[None]
    a = torch.randint(0, 2, (m, k), generator=gen, dtype=torch.uint8, device="cuda").mul_(0x80).add_(0x38)
    y = torch.full((m, n), -7.0, dtype=torch.bfloat16, device="cuda")
    ae.model_fp8_matmul(a, torch.ones((1, m), device="cuda"), b, bs, "rows", None, m, n, k, y)
    av = torch.where(a >= 0x80, -1.0, 1.0)
    step = 1 << 22
    for at in range(0, n, step):
        e = min(n, at + step)
        want = (av @ torch.where(b[at:e] >= 0x80, -1.0, 1.0).t()) * bs[:, at:e]
        assert torch.equal(y[:, at:e].float(), want), at
    del y, b, bs, want
    torch.cuda.empty_cache()
