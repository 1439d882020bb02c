"""Distillation from a teacher in which some rows are empty, as the log probabilities' call returns them (top_logit and lse of
-infinity): those rows have neither loss nor gradient, the others are as without them."""
import math

import pytest

from test_gpu_vocab_large import SHAPES, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype,rows,vocab,k", [(d, r, v, 20) for d in SHAPES for r, v in SHAPES[d]] + [("bf16", 300, 4003, 300), ("f32", 5, 40001, 20)])
def test_empty_teacher_rows(dtype, rows, vocab, k, tail):
    import torch
    from paper_2602_17681_amd import binding as ae
    z, ids, t, _ = make(rows, vocab, dtype, k)
    dt = ae.AE_BF16 if dtype == "bf16" else ae.AE_F32
    lse = (torch.logsumexp(t.double(), 1) + 0.3).float() if tail else None

    def run(t, lse, g):
        ws = torch.full((ae.model_loss_distill_workspace(rows, vocab, dt),), 0xFF, dtype=torch.uint8, device="cuda")
        lr, total = torch.full((rows,), -7.0, device="cuda"), torch.full((1,), -7.0, device="cuda")
        ae.model_loss_distill(z, rows, vocab, ids.to(torch.int32), t, lr, total, g, ws, teacher_lse=lse)
        return lr, total.item()
    g0, g1 = torch.full_like(z, 3.0), torch.full_like(z, 3.0)
    lr0, _ = run(t, lse, g0)
    empty = torch.zeros(rows, dtype=torch.bool, device="cuda")
    empty[::3] = True
    t1 = t.masked_fill(empty[:, None], -math.inf)
    lse1 = lse.masked_fill(empty, -math.inf) if tail else None
    lr1, total = run(t1, lse1, g1)
    assert bool((lr1[empty] == 0).all()) and bool((g1[empty] == 0).all())
    assert torch.equal(lr1[~empty], lr0[~empty]) and torch.equal(g1[~empty], g0[~empty])
    want = lr1.double().sum().item()
    assert abs(total - want) <= 2.0 ** -22 * (1 + want)
    lr2, total2 = run(t1, lse1, None)                      # the loss alone
    assert bool((lr2[empty] == 0).all()) and abs(total2 - want) <= 1e-4 * (1 + want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(3, 40001), (270, 3001)])
def test_the_two_calls_joined(rows, vocab, dtype):
    """The list of an empty row, as it is returned, goes on into the loss."""
    import torch
    from paper_2602_17681_amd import binding as ae
    k = 16
    z, _, _, gen = make(rows, vocab, dtype, 20)
    teacher = z + torch.randn((rows, vocab), generator=gen, device="cuda").to(z.dtype)
    teacher[1] = -math.inf
    dt = ae.AE_BF16 if dtype == "bf16" else ae.AE_F32
    ids, tl, lse = torch.empty((rows, k), dtype=torch.int32, device="cuda"), torch.empty((rows, k), device="cuda"), torch.empty(rows, device="cuda")
    ws = torch.empty(max(16, ae.model_token_logprobs_workspace(rows, vocab, k, dt), ae.model_loss_distill_workspace(rows, vocab, dt)), dtype=torch.uint8, device="cuda")
    ae.model_token_logprobs(teacher, rows, vocab, None, k, None, None, lse, ids, tl, None, ws)
    lr, total, g = torch.empty(rows, device="cuda"), torch.empty(1, device="cuda"), torch.empty_like(z)
    ae.model_loss_distill(z, rows, vocab, ids, tl, lr, total, g, ws, teacher_lse=lse)
    assert lr[1].item() == 0 and bool((g[1] == 0).all()) and bool((lr[torch.arange(rows, device="cuda") != 1] > 0).all()) and math.isfinite(total.item())
