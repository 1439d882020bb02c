"""Top lists of rows of NaN and of rows with fewer numbers than the list is long, in long rows and pieces: every entry is written,
falling logits first, equal ones by their index, NaN last."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("top", [1, 20, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(64, 33000), (4, 50257), (4, 65536), (64, 131072), (63, 1 << 20), (70, 1 << 18), (300, 20001), (3, 70003)])
def test_lists_of_rows_with_nan(rows, vocab, dtype, top):
    import torch
    from paper_2602_17681_amd import binding as ae
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows + vocab)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    nan = float("nan")
    z = (torch.randn((rows, vocab), generator=gen, device="cuda") * 2.5).to(td)
    u = lambda: torch.rand(vocab, generator=gen, device="cuda")      # noqa: E731
    z[0] = nan                                             # nothing but NaN
    z[1, u() < 0.9995] = nan                               # a few numbers
    z[2] = nan
    z[2, ::977] = -math.inf                                # NaN and what cannot occur
    if rows > 3:
        z[3] = nan
        z[3, vocab - 1] = 1.0                              # one number
    if rows > 8:
        z[4] = torch.where(u() < 0.5, nan, -math.inf)
        z[5] = torch.where(u() < 0.999, nan, torch.finfo(td).min)
        z[6, :vocab // 2] = nan                            # numbers in one half only
        z[7, 64:] = nan
        z[8, u() < 0.9] = nan
    # what memory held before: neither the outputs nor the workspace may show through
    ids = torch.full((rows, top), -7, dtype=torch.int32, device="cuda")
    logit, logprob, lse = (torch.full(s, -7.0, device="cuda") for s in ((rows, top), (rows, top), (rows,)))
    ws = torch.full((max(16, ae.model_token_logprobs_workspace(rows, vocab, top, ae.AE_BF16 if dtype == "bf16" else ae.AE_F32)),), 0x7F, dtype=torch.uint8, device="cuda")
    ae.model_token_logprobs(z, rows, vocab, None, top, None, None, lse, ids, logit, logprob, ws)
    for r in list(range(min(rows, 9))) + [rows - 1]:
        key = torch.where(torch.isnan(z[r]), torch.full((), -math.inf, dtype=torch.float64, device="cuda"), z[r].double())
        # numbers before NaN, also where they are -infinity
        order = torch.sort(torch.isnan(z[r]), stable=True).indices
        order = order[torch.sort(torch.where(torch.isnan(z[r][order]), -math.inf, key[order]), descending=True, stable=True).indices][:top]
        assert ids[r].tolist() == order.tolist(), r
        want = z[r][order].float()
        assert torch.equal(torch.isnan(logit[r]), torch.isnan(want)) and torch.equal(torch.nan_to_num(logit[r], nan=5.0), torch.nan_to_num(want, nan=5.0)), r
        if bool(torch.isnan(z[r]).any()):
            assert bool(torch.isnan(logprob[r]).all()) and bool(torch.isnan(lse[r])), r
