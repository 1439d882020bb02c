"""The calibration step of an 8-bit output layer as a whole: folding, quantiser, product, log probabilities, distillation and
both gradients, each against its oracle on what the step before it left."""
import numpy as np
import pytest

from oracle import fp8_oracle as fo
from oracle import vocab_oracle as vo

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,d,vocab,k", [(40, 256, 500, 16), (7, 128, 1001, 64)])
def test_step_against_the_oracles(tokens, d, vocab, k):
    import torch
    import bench
    from paper_2602_17681_amd import binding as ae
    st = bench.build_output_layer(torch, ae, tokens, d, vocab, seed=3, top_k=k)
    h = lambda t: t.detach().double().cpu().numpy() if t.is_floating_point() and t.dtype != torch.float8_e4m3fn else t.view(torch.uint8).cpu().numpy() if t.dtype == torch.float8_e4m3fn else t.cpu().numpy()      # noqa: E731
    n, temp = tokens, st["temperature"]
    teacher = vo.token_logprobs(h(st["teacher"]), None, k, temp)
    bench.output_layer_step(st, ae)
    assert np.array_equal(h(st["top_id"]), teacher["top_id"]) and np.allclose(h(st["teacher_lse"]), teacher["lse"], rtol=1e-5, atol=1e-4)
    # the layer: its logits once more, since the step put the gradient in their place
    logits = torch.empty((n, vocab), dtype=torch.bfloat16, device="cuda")
    ae.model_fp8_linear(st["x"], st["w"], st["w_s"], st["bias"], n, vocab, d, logits, st["ws"])
    a, sa = fo.quantize(st["x"].float().cpu().numpy())
    ref, mag = fo.matmul(a, sa, h(st["w"]), st["w_s"].cpu().numpy(), "tiles", h(st["bias"]))
    assert np.all(np.abs(h(logits) - ref) <= mag * 2.0 ** -9 + 2.0 ** -8 * np.abs(ref))
    z = h(logits)
    lp = vo.token_logprobs(z, h(st["target"]))
    assert np.allclose(h(st["logprob"]), lp["logprob"], atol=1e-4) and np.allclose(h(st["entropy"]), lp["entropy"], atol=1e-4)
    w = np.full(n, 1.0 / n)
    _, loss, grad = vo.distill(z, h(st["top_id"]), h(st["top_logit"]), temp, h(st["teacher_lse"]), w)
    assert abs(st["loss"].item() - loss) <= 1e-4 * (1 + abs(loss)) and 0 < loss < 2     # a layer in 8 bits is near its teacher
    g = h(st["logits"])
    assert np.all(np.abs(g - grad) <= 2.0 ** -8 * np.abs(grad) + 2e-4 / n * (np.abs(grad) * n + 1e-3))
    # the gradients from the rounded gradient of the logits
    gf, xf = g.astype(np.float32), st["x"].float().cpu().numpy()
    (gq, gs), (gt, gts), (xt, xts) = fo.quantize(gf), fo.quantize(gf.T), fo.quantize(xf.T)
    assert np.array_equal(fo.VALUES[h(st["g"])], fo.VALUES[gq]) and np.array_equal(fo.VALUES[h(st["gt"])], fo.VALUES[gt]) and np.array_equal(fo.VALUES[h(st["xt"])], fo.VALUES[xt])
    dx, dx_mag = fo.matmul(gq, gs, h(st["wt"]), st["wt_s"].cpu().numpy(), "tiles")
    assert np.all(np.abs(h(st["dx"]) - dx) <= dx_mag * 2.0 ** -9 + 2.0 ** -8 * np.abs(dx))
    dw, dw_mag = fo.matmul(gt, gts, xt, xts, "rows")
    assert np.all(np.abs(h(st["dw"]) - dw) <= dw_mag * (132 * 2.0 ** -23 + 2.0 ** -24 * 8))
    # and they are near the gradients of the unquantised chain: E4M3 has three fraction bits, 2^-4 of each factor
    wv = fo.values(h(st["w"]), st["w_s"].cpu().numpy(), "tiles")
    assert np.linalg.norm(h(st["dx"]) - g @ wv) <= 0.05 * np.linalg.norm(g @ wv) and np.linalg.norm(h(st["dw"]) - g.T @ xf) <= 0.08 * np.linalg.norm(g.T @ xf)
