"""Distillation of a student's row that holds NaN or an infinity: NaN for that row's loss and gradient, whatever the teacher's list
holds, also where no entry of it counts."""
import math

import pytest

from test_gpu_vocab_large import SHAPES, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("entries", ["none", "some", "one_of_no_probability"])
@pytest.mark.parametrize("dtype,rows,vocab,k", [(d, r, v, 20) for d in SHAPES for r, v in SHAPES[d]] + [("f32", 300, 2003, 300)])
def test_nan_in_the_student(dtype, rows, vocab, k, entries):
    import torch
    from paper_2602_17681_amd import binding as ae
    z, ids, t, _ = make(rows, vocab, dtype, k)
    ids = ids.to(torch.int32)
    z[1, 7], z[2, vocab - 1], z[3, int(ids[3, 2])], z[4, int(ids[4, 0])] = math.nan, math.inf, math.nan, math.inf
    if entries == "none":
        ids[:] = -1
        ids[5:, 0] = vocab
    elif entries == "one_of_no_probability":
        ids[:, 1:] = -1
        t[:, 0] = -math.inf
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
    bad[1:5] = True
    for lse in (None, torch.full((rows,), 9.0, device="cuda")):
        ws = torch.full((ae.model_loss_distill_workspace(rows, vocab, ae.AE_BF16 if dtype == "bf16" else ae.AE_F32),), 0xFF, dtype=torch.uint8, device="cuda")
        for grad in (True, False):
            lr, total, g = torch.full((rows,), -7.0, device="cuda"), torch.full((1,), -7.0, device="cuda"), torch.full_like(z, 3.0)
            ae.model_loss_distill(z, rows, vocab, ids, t, lr, total, g if grad else None, ws, teacher_lse=lse)
            assert torch.equal(torch.isnan(lr), bad) and math.isnan(total.item())
            if grad:
                assert bool(torch.isnan(g[bad]).all()) and bool(torch.isfinite(g[~bad]).all())
