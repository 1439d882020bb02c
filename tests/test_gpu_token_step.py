"""Training and decoding steps from tokens to an 8-bit output layer and back, each stage against its oracle on what the stage before it left."""
import numpy as np
import pytest

from oracle import fp8_oracle as fo
from oracle import token_oracle as to
from oracle import vocab_oracle as vo
from token_util import U, host, near

pytestmark = pytest.mark.gpu


def codes(t):
    import torch
    return t.contiguous().view(torch.uint8).cpu().numpy()


@pytest.mark.parametrize("tokens,d,vocab,k", [(40, 256, 500, 16), (7, 136, 1001, 8), (300, 130, 700, 5)])
def test_training_step(tokens, d, vocab, k):
    import torch
    import bench
    from paper_2602_17681_amd import binding as ae
    st = bench.build_token_step(torch, ae, tokens, d, vocab, seed=3, top_k=k, rows=min(4, tokens))
    bench.token_train_step(st, ae, max_norm=float("inf"))
    ids, gain, n = st["ids"].cpu().numpy(), host(st["gain"]), tokens
    scale = float(np.float32(st["embed_scale"]))
    x = to.embedding(host(st["table"]), ids, scale)
    near(host(st["x"][:n]), x, 2.0 ** -8 * 1.001 * np.abs(x))
    hs, y = to.rms_norm(host(st["x"][:n]), host(st["stream"][:n]), gain, st["eps"])
    near(host(st["h"][:n]), hs, 2.0 ** -8 * np.abs(hs) + 1e-40)
    near(host(st["y"][:n]), y, (2.0 ** -8 + 40 * U) * np.abs(y) + 1e-40)
    s = st["q_s"][n].double().cpu().numpy()[np.arange(d) // 128].T
    near(fo.VALUES[codes(st["q"][:n])] * s, y, 2.0 ** -4 * 1.001 * np.abs(y) + s * 2.0 ** -10)
    # loss and its gradient, from the product of what was quantised
    z, mag = fo.matmul(codes(st["q"][:n]), st["q_s"][n].cpu().numpy(), codes(st["w"]), st["w_s"].cpu().numpy(), "tiles")
    _, loss, grad = vo.distill(z, st["top_id"].cpu().numpy(), host(st["top_logit"]), st["temperature"], host(st["teacher_lse"]), host(st["weight"]))
    assert abs(st["loss"].item() - loss) <= 2e-2 * (1 + abs(loss))             # from logits rounded to bfloat16: up to 2^-8 of some tens
    g = host(st["logits"][:n])                                                    # the gradient stands in their place
    assert np.linalg.norm(g - grad) <= 0.05 * np.linalg.norm(grad) and np.all(g[ids < 0] == 0)
    # the gradients, from the rounded ones before them
    gf, yf = g.astype(np.float32), st["y"][:n].float().cpu().numpy()
    (gq, gs), (gt, gts), (yt, yts) = fo.quantize(gf), fo.quantize(gf.T), fo.quantize(yf.T)
    dy, dy_mag = fo.matmul(gq, gs, codes(st["wt"]), st["wt_s"].cpu().numpy(), "tiles")
    near(host(st["dy"]), dy, dy_mag * 2.0 ** -9 + 2.0 ** -8 * np.abs(dy) + 1e-40)
    dx, dg, mx, mg = to.rms_norm_backward(host(st["dy"]), host(st["h"][:n]), gain, st["eps"])
    near(host(st["dx"]), dx, 140 * U * mx + 2.0 ** -8 * np.abs(dx) + 1e-37)
    near(host(st["d_gain"]), dg, (n + 46) * U * mg + 1e-37)
    dw, dw_mag = fo.matmul(gt, gts, yt, yts, "rows")
    de, de_mag, count = to.embedding_backward(host(st["dx"]), ids, vocab, scale)
    near(host(st["d_table"]), dw + de, dw_mag * (132 * 2.0 ** -23 + 2.0 ** -24 * 8) + (count[:, None] + 3) * U * de_mag + U * np.abs(dw + de))
    norm, _ = to.grad_clip([host(st["d_table"]), host(st["d_gain"])], 1.0)
    assert abs(st["norm"].item() - norm) <= 1.001 * U * norm
    # clipped in place: the same step with half of that norm allowed
    table, gain_grad = host(st["d_table"]), host(st["d_gain"])
    bench.token_train_step(st, ae, max_norm=norm / 2)
    half = float(np.float32(norm / 2)) / norm
    near(host(st["d_table"]), table * half, 3 * U * np.abs(table) * half + 1e-44)
    near(host(st["d_gain"]), gain_grad * half, 3 * U * np.abs(gain_grad) * half + 1e-44)


@pytest.mark.parametrize("tokens,d,vocab,rows", [(8, 256, 500, 4), (3, 130, 5003, 7), (1, 4096, 32768, 1)])
def test_decoding_step(tokens, d, vocab, rows):
    """Eager, and as a captured graph that is replayed."""
    import torch
    import bench
    from paper_2602_17681_amd import binding as ae
    st = bench.build_token_step(torch, ae, tokens, d, vocab, seed=5, top_k=4, rows=rows)
    bench.token_decode_step(st, ae)
    x = to.embedding(host(st["table"]), st["last"].cpu().numpy(), float(np.float32(st["embed_scale"])))
    near(host(st["x"][:rows]), x, 2.0 ** -8 * 1.001 * np.abs(x))
    _, y = to.rms_norm(host(st["x"][:rows]), host(st["stream"][:rows]), host(st["gain"]), st["eps"])
    s = st["q_s"][rows].double().cpu().numpy()[np.arange(d) // 128].T
    near(fo.VALUES[codes(st["q"][:rows])] * s, y, 2.0 ** -4 * 1.001 * np.abs(y) + s * 2.0 ** -10)
    z, mag = fo.matmul(codes(st["q"][:rows]), st["q_s"][rows].cpu().numpy(), codes(st["w"]), st["w_s"].cpu().numpy(), "tiles")
    arrays = {k: st[k].cpu().numpy() for k in ("history", "n_prompt", "repetition", "presence", "frequency", "bias_id", "bias")}
    want, terms = to.logits_adjust(z, **arrays, allowed=st["allowed"].cpu().numpy().view(np.uint32))
    got = host(st["logits"][:rows])
    # the product's rounding to bfloat16 and its sums, through a penalty of at most 1.2, then the second rounding
    near(got, want, np.where(np.isfinite(want), 1.2 * (mag * 2.0 ** -9 + 2.0 ** -8 * np.abs(z)) + 2.0 ** -8 * np.abs(np.where(np.isfinite(want), want, 0)) * 1.01 + 6 * U * terms, 0))
    top = vo.token_logprobs(got, None, st["best"].shape[1], 1.0)
    assert np.array_equal(st["best"].cpu().numpy(), top["top_id"])
    first = [st[k].clone() for k in ("best", "best_logprob", "logits")]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        bench.token_decode_step(st, ae)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bench.token_decode_step(st, ae)
    for _ in range(3):
        st["best"].fill_(-5)
        st["logits"][:rows].fill_(7.0)
        torch.ones(100, device="cuda").sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a[:rows], st[k][:rows]) for a, k in zip(first, ("best", "best_logprob", "logits")))


def test_tensors_of_another_device_than_the_current_one_are_refused(monkeypatch):
    import torch
    from paper_2602_17681_amd import binding as ae
    x, ids, w = torch.zeros((4, 64), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda"), torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    lst, y = ae.GradList([x]), torch.full((4, 64), 7.0, device="cuda")
    calls = [lambda: ae.model_rms_norm(x, 4, 64, None, 1e-6, y=y), lambda: ae.model_rms_norm_backward(x, x, 4, 64, None, 1e-6, y, None, w),
             lambda: ae.model_embedding(x, 4, 64, ids, 4, y), lambda: ae.model_embedding_backward(x, ids, 4, 4, 64, y, w),
             lambda: ae.model_grad_clip(lst, 1.0, y[0, :1], w), lambda: ae.model_logits_adjust(x, 4, 64, y)]
    with monkeypatch.context() as m:
        m.setattr(ae, "_current_device", lambda: 1)
        for call in calls:
            with pytest.raises(AssertionError, match="device 0"):
                call()
    torch.cuda.synchronize()
    assert bool((y == 7).all())
    for call in calls:
        call()
