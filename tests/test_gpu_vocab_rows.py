"""Rows of logits in every form that the kernels take them: pieces of few long rows, rows held in registers by workgroups of
each size, workgroups that go on to further rows, rows that fit no registers; against 64 bits on the device."""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def sum_error(vocab, temperature, spread):
    """Relative error of a row's sum: exponents (their argument is off by 2^-23 of itself, and the terms that count lie within the
    row's spread), the exponential's own last place, and as many additions as a thread makes in turn."""
    return ((spread / temperature + 4) * 4 + vocab / 512 + 40) * U


def make(rows, vocab, dtype, seed, masked, offset=0):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    buf = torch.full((rows * vocab + offset,), float("nan"), dtype=td, device="cuda")
    z = buf[offset:].view(rows, vocab)
    z.copy_(torch.randn((rows, vocab), generator=gen, device="cuda") * 2.5)
    if masked:
        u = torch.rand((rows, vocab), generator=gen, device="cuda")
        z.masked_fill_(u < 0.2, -math.inf)
        z.masked_fill_(u > 0.9, torch.finfo(td).min)
        z[rows // 2] = -math.inf
    return z, gen


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,top,masked", [(1, 65537, 5, False), (3, 70001, 64, True), (5, 131075, 256, False), (63, 66000, 20, True), (64, 66000, 33, False),
                                                   (2, 200003, 1, True), (100, 131072, 40, False), (4, 90001, 0, True)])
def test_logprobs_of_long_rows(rows, vocab, top, masked, dtype):
    import torch
    from paper_2602_17681_amd import binding as ae
    temperature = 0.75
    z, gen = make(rows, vocab, dtype, rows + vocab, masked, offset=1)
    tokens = torch.randint(-1, vocab, (rows, 4), generator=gen, device="cuda", dtype=torch.int32)
    f = lambda *s: torch.full(s, -7.0, device="cuda")      # noqa: E731
    logprob, entropy, lse, top_logit, top_logprob = f(rows, 4), f(rows), f(rows), f(rows, top), f(rows, top)
    ids = torch.full((rows, top), -7, dtype=torch.int32, device="cuda")
    ws = torch.full((max(16, ae.model_token_logprobs_workspace(rows, vocab, top, ae.AE_BF16 if dtype == "bf16" else ae.AE_F32)),), 0xFF, dtype=torch.uint8, device="cuda")
    ae.model_token_logprobs(z, rows, vocab, tokens, top, logprob, entropy, lse, ids, top_logit, top_logprob, ws, temperature=temperature)
    x = z.double() / temperature
    # next to the type's lowest number nothing of a logarithm is left: relative to the maximum
    m = x.amax(1, keepdim=True)
    empty = torch.isinf(m[:, 0])
    d = x - torch.where(torch.isinf(m), 0.0, m)
    log_s = torch.log(torch.exp(d).sum(1))
    ref_lse = torch.where(empty, -math.inf, m[:, 0] + log_s)
    logq = torch.where(empty[:, None], -math.inf, d - log_s[:, None])
    e = sum_error(vocab, temperature, 25.0)
    near = lambda a, b, tol: bool((torch.where(torch.isinf(b), (a.double() == b), (a.double() - b).abs() <= tol)).all())      # noqa: E731
    assert near(lse, ref_lse, e + 6 * U * 40)
    ref_h = -torch.nan_to_num(torch.exp(logq) * logq, nan=0.0).sum(1)
    assert near(entropy, ref_h, (e + 8 * U) * (math.log(vocab) + 2) * 2)
    at = tokens.long()
    ref_t = torch.where(at < 0, 0.0, logq.gather(1, at.clamp(min=0)))
    # a lowest number over a temperature below 1 is -infinity in binary32
    big = torch.finfo(torch.float32).max
    ref_t = torch.where(ref_t < -big, -math.inf, ref_t)
    assert near(logprob, ref_t, e + 8 * U * (torch.nan_to_num(ref_t, neginf=0.0).abs() + 30))
    if top:
        order = torch.sort(z.double(), dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(ids.long(), order)
        assert torch.equal(top_logit.double(), z.double().gather(1, order))
        ref_p = logq.gather(1, order)
        assert near(top_logprob, ref_p, e + 8 * U * (torch.nan_to_num(ref_p, neginf=0.0).abs() + 30))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("edit", ["constant", "two_values", "rising", "falling", "nan", "all_nan"])
def test_top_lists_of_unusual_pieces(edit, dtype):
    """Ties, sorted rows and NaN where a row is cut into pieces: falling logits, equal ones by their index, NaN last."""
    import torch
    from paper_2602_17681_amd import binding as ae
    rows, vocab, top = 3, 70003, 100
    z, gen = make(rows, vocab, dtype, 11, False)
    if edit == "constant":
        z.fill_(1.25)
    elif edit == "two_values":
        z.copy_(torch.where(torch.rand((rows, vocab), generator=gen, device="cuda") < 0.001, 2.0, -1.0))
    elif edit in ("rising", "falling"):
        z.copy_(torch.sort(z.float(), dim=1, descending=edit == "falling").values)
    elif edit == "nan":
        z[torch.rand((rows, vocab), generator=gen, device="cuda") < 0.9995] = float("nan")
    else:
        z.fill_(float("nan"))
    ids = torch.empty((rows, top), dtype=torch.int32, device="cuda")
    ws = torch.empty(ae.model_token_logprobs_workspace(rows, vocab, top, ae.AE_BF16 if dtype == "bf16" else ae.AE_F32), dtype=torch.uint8, device="cuda")
    ae.model_token_logprobs(z, rows, vocab, None, top, None, None, None, ids, None, None, ws)
    key = torch.where(torch.isnan(z), -math.inf, z.double())
    order = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(ids.long(), order)


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("rows,vocab,dtype", [(3, 33000, "f32"), (100, 20001, "bf16"), (130, 9000, "bf16"), (300, 30001, "bf16"), (300, 16001, "f32"), (600, 40001, "bf16"),
                                              (1100, 50021, "bf16"), (700, 33003, "f32"), (520, 70005, "bf16"), (400, 131080, "bf16"), (270, 131072, "bf16"), (300, 65540, "f32"),
                                              (6000, 1501, "bf16"), (257, 7, "f32")])
def test_distill_rows(rows, vocab, dtype, masked):
    import torch
    from paper_2602_17681_amd import binding as ae
    temperature, k = 1.5, min(40, vocab)
    for tail in (False, True):
        z, gen = make(rows, vocab, dtype, rows + vocab, masked, offset=1)
        share = vocab // k
        ids = (torch.rand((rows, k), generator=gen, device="cuda") * share).long().clamp_(max=share - 1) + torch.arange(k, device="cuda") * vocab // k
        z.scatter_(1, ids, (torch.randn((rows, k), generator=gen, device="cuda") * 2 + 5).to(z.dtype))
        t = (torch.randn((rows, k), generator=gen, device="cuda") * 2 + 6).sort(1, descending=True).values
        w = torch.rand(rows, generator=gen, device="cuda") + 0.5
        if masked:
            ids = ids.masked_fill(torch.arange(k, device="cuda") >= torch.randint(0, k + 1, (rows, 1), generator=gen, device="cuda"), -1)
            w[torch.rand(rows, generator=gen, device="cuda") < 0.3] = 0.0
            z[rows // 2] = -math.inf
        there = ids >= 0
        x = torch.where(there, t.double() / temperature, -math.inf)
        norm = torch.nan_to_num(torch.logsumexp(x, 1), neginf=2.0)
        lse = (norm + 0.1 + 0.5 * torch.rand(rows, generator=gen, device="cuda")).float() if tail else None
        # 64 bits
        zs = z.double() / temperature
        m = zs.amax(1, keepdim=True)
        empty = torch.isinf(m[:, 0])
        d = zs - torch.where(torch.isinf(m), 0.0, m)
        ee = torch.exp(d)
        s = ee.sum(1)
        q = torch.where(empty[:, None], 0.0, ee / s[:, None])
        inside = torch.zeros((rows, vocab + 1), dtype=torch.bool, device="cuda").scatter_(1, torch.where(there, ids, vocab), True)[:, :vocab]
        logp = x - (lse.double() if tail else norm)[:, None]
        p = torch.exp(logp)
        q_out = torch.where(inside, 0.0, q).sum(1)
        rest = (1 - p.sum(1)).clamp(min=0) if tail else torch.zeros_like(norm)
        rest = torch.where(q_out > 0, rest, 0.0)
        logq = torch.where(there, d.gather(1, ids.clamp(min=0)) - torch.log(s)[:, None], 0.0)
        loss = torch.where(p > 0, p * (logp - logq), 0.0).sum(1) + torch.where(rest > 0, rest * (torch.log(rest) - torch.log(q_out)), 0.0)
        live = ~empty & (w != 0)
        loss = torch.where(live, loss, 0.0)
        mass = p.sum(1) + rest
        ratio = torch.where(rest > 0, rest / q_out, 0.0)
        grad = torch.where(inside, mass[:, None] * q, (mass - ratio)[:, None] * q)
        grad.scatter_add_(1, ids.clamp(min=0), torch.where(there, -p, 0.0))
        scale = torch.where(live, w.double() / temperature, 0.0)[:, None]
        grad = torch.where(live[:, None], grad * scale, 0.0)
        # the call, into a buffer of its own and in the logits' place
        dt = ae.AE_BF16 if dtype == "bf16" else ae.AE_F32
        ws = torch.full((ae.model_loss_distill_workspace(rows, vocab, dt),), 0xFF, dtype=torch.uint8, device="cuda")
        lr, total, g = torch.full((rows,), -7.0, device="cuda"), torch.full((1,), -7.0, device="cuda"), torch.full_like(z, 3.0)
        i32 = ids.to(torch.int32)
        ae.model_loss_distill(z, rows, vocab, i32, t, lr, total, g, ws, teacher_lse=lse, weight=w, temperature=temperature)
        e = sum_error(vocab, temperature, 30.0)
        assert bool(((lr.double() - loss).abs() <= 3 * e + 8 * U * (loss.abs() + 1)).all())
        want = (loss * w.double()).sum().item()
        assert abs(total.item() - want) <= ((3 * e + 8 * U) * w.sum().item()) + 12 * U * abs(want) + 1e-30
        xs = (-torch.nan_to_num(d, neginf=0.0)).clamp(max=120.0)
        tol = scale * (torch.maximum(torch.ones_like(mass), mass + ratio)[:, None] * q * (3 * e + 4 * U * (xs + 4))) + 4 * U * grad.abs() + 1e-37
        if dtype == "bf16":
            tol = tol + 2.0 ** -8 * grad.abs()
        assert bool(((g.double() - grad).abs() <= tol).all())
        lr2 = torch.empty_like(lr)
        ae.model_loss_distill(z, rows, vocab, i32, t, lr2, None, z, ws, teacher_lse=lse, weight=w, temperature=temperature)
        assert torch.equal(z, g) and torch.equal(lr2, lr)
        torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(5, 20001), (140, 20001), (260, 900), (300, 40001), (140, 131090)])
def test_distill_of_extreme_rows(rows, vocab, dtype):
    """A row of the type's lowest number only, one of numbers near the largest, one of large ones, one whose logits are all
    alike: differences to the maximum are what counts, and they are exact."""
    import torch
    from paper_2602_17681_amd import binding as ae
    z, gen = make(rows, vocab, dtype, 5, False)
    low = torch.finfo(z.dtype).min
    z[0] = low
    z[1] = 2e38
    z[1, ::7] = -2e38
    z[2] *= 1e6
    z[3] = 1.5
    k = 12
    ids = torch.arange(k, device="cuda").repeat(rows, 1) * 7 + 3
    ids[1, :3] = torch.arange(3, device="cuda") * 7
    t = (torch.randn((rows, k), generator=gen, device="cuda") + 3).sort(1, descending=True).values
    t[1, :3] = -math.inf                                   # tokens that the student all but rules out, and the teacher does
    lse = (torch.logsumexp(t.double(), 1) + 0.3).float()
    ws = torch.empty(ae.model_loss_distill_workspace(rows, vocab, ae.AE_BF16 if dtype == "bf16" else ae.AE_F32), dtype=torch.uint8, device="cuda")
    lr, g = torch.empty(rows, device="cuda"), torch.empty_like(z)
    ae.model_loss_distill(z, rows, vocab, ids.to(torch.int32), t, lr, None, g, ws, teacher_lse=lse)
    for r in (0, 1, 2, 3):
        zr, at = z[r].double(), ids[r]
        d = zr - zr.max()
        s = torch.exp(d).sum()
        logq = d - torch.log(s)
        q = torch.exp(logq)
        logp = t[r].double() - lse[r].double()
        p = torch.exp(logp)
        outside = torch.ones(vocab, dtype=torch.bool, device="cuda")
        outside[at] = False
        q_out = q[outside].sum()
        rest = 1 - p.sum() if q_out > 0 else torch.zeros((), dtype=torch.float64, device="cuda")
        loss = torch.where(p > 0, p * (logp - logq[at]), 0.0).sum() + (rest * (torch.log(rest) - torch.log(q_out)) if rest > 0 else 0.0)
        e = sum_error(vocab, 1.0, 30.0)
        # logits of a million: the terms p (z_i - m) of the loss are binary32 products of that size at most
        assert abs(lr[r].item() - loss.item()) <= 3 * e + 8 * U * (abs(loss.item()) + 1)
        mass = p.sum() + rest
        grad = q * (mass - (rest / q_out if rest > 0 else 0.0))
        grad[at] = mass * q[at] - p
        tol = (mass + (rest / q_out if rest > 0 else 0.0)) * q * (3 * e + 16 * U) + 4 * U * grad.abs() + 1e-37
        if dtype == "bf16":
            tol = tol + 2.0 ** -8 * grad.abs()
        assert bool(((g[r].double() - grad).abs() <= tol).all())
