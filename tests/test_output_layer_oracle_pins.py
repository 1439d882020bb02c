"""Pins of the oracles of the 8-bit matrices and of the passes over logits: independent statements of the same things."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as fo
from oracle import vocab_oracle as vo


def test_codes_are_the_types_own():
    """All 256 values, and the nearest code of numbers between, at and around them, as torch's float8_e4m3fn has them."""
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(np.isnan(t), np.isnan(fo.VALUES)) and np.array_equal(t[~np.isnan(t)], fo.VALUES[~np.isnan(t)].astype(np.float32))
    mids = (fo.POSITIVE[1:] + fo.POSITIVE[:-1]) / 2
    y = np.concatenate([fo.POSITIVE, mids, mids * (1 + 1e-6), mids * (1 - 1e-6), np.random.default_rng(0).uniform(0, 448, 5000)])
    y = np.concatenate([y, -y]).astype(np.float32)
    want = torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(fo.encode(y), want)
    assert list(fo.encode(np.float32([500, -1e30, np.inf, np.nan, 0.0]))) == [126, 254, 126, 127, 0]


@pytest.mark.parametrize("blocks", ["rows", "tiles"])
def test_quantised_values_are_near(blocks):
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((130, 300)) * np.exp(rng.standard_normal((130, 1)) * 4)).astype(np.float32)
    x[3] = 0
    q, s = fo.quantize(x, blocks)
    v = fo.values(q, s, blocks)
    # a code is within half a step: 2^-4 of the value, or half the subnormal spacing 2^-10 of the block's scale
    step = s[np.arange(300) // 128].T if blocks == "rows" else s[np.arange(130) // 128][:, np.arange(300) // 128]
    assert np.all(np.abs(v - x) <= np.maximum(np.abs(x) * 2.0 ** -4, step * 2.0 ** -10) * (1 + 1e-6))
    assert np.all(v[3] == 0)
    # the largest of a block comes back as it is
    assert np.allclose(np.abs(v[:128, :128]).max(), np.abs(x[:128, :128]).max(), rtol=1e-6)


def test_product_of_values():
    rng = np.random.default_rng(2)
    a, sa = fo.quantize(rng.standard_normal((5, 200)))
    b, sb = fo.quantize(rng.standard_normal((140, 200)), "tiles")
    y, _ = fo.matmul(a, sa, b, sb)
    i, j = 3, 131
    s = sum(float(fo.VALUES[a[i, k]]) * float(fo.VALUES[b[j, k]]) * float(sa[k // 128, i]) * float(sb[j // 128, k // 128]) for k in range(200))
    assert abs(y[i, j] - s) <= 1e-12 * abs(s) + 1e-12


def test_log_probabilities_against_torch():
    rng = np.random.default_rng(3)
    z = rng.standard_normal((4, 50)) * 5
    z[1, ::3] = -np.inf
    z[2] = -np.inf
    o = vo.token_logprobs(z, np.array([[0, -1], [1, 50], [2, 3], [4, 4]]), 5, 0.7)
    ref = torch.distributions.Categorical(logits=torch.from_numpy(z[[0, 1, 3]] / 0.7))
    assert np.allclose(o["entropy"][[0, 1, 3]], ref.entropy().numpy())
    assert np.allclose(o["logprob"][0, 0], ref.logits[0, 0].item()) and o["logprob"][0, 1] == 0 and o["logprob"][1, 1] == 0
    assert o["entropy"][2] == 0 and o["lse"][2] == -np.inf and np.all(o["logprob"][2] == -np.inf) and list(o["top_id"][2]) == [0, 1, 2, 3, 4]
    assert np.allclose(o["top_logit"][0], np.sort(z[0])[::-1][:5])
    ties = vo.token_logprobs(np.array([[1.0, 3.0, 3.0, np.nan, 2.0, 3.0]]), None, 6)
    assert list(ties["top_id"][0]) == [1, 2, 5, 4, 0, 3]


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("temperature", [0.6, 1.0, 1.5])
def test_distillation_gradient_against_differences(tail, temperature):
    rng = np.random.default_rng(4)
    z = rng.standard_normal((3, 20)) * 2
    ids = np.stack([rng.permutation(20)[:6] for _ in range(3)])
    ids[1, 4:] = -1
    t = np.sort(rng.standard_normal((3, 6)) * 2)[:, ::-1]
    lse = np.log(np.exp(t / temperature).sum(1)) + 0.3 if tail else None
    w = np.array([1.0, 0.5, 2.0])
    _, total, g = vo.distill(z, ids, t, temperature, lse, w)
    num = np.zeros_like(z)
    for r in range(3):
        for j in range(20):
            d = np.zeros_like(z)
            d[r, j] = 1e-5
            num[r, j] = (vo.distill(z + d, ids, t, temperature, lse, w)[1] - vo.distill(z - d, ids, t, temperature, lse, w)[1]) / 2e-5
    assert np.abs(num - g).max() <= 1e-8
    assert np.abs(g.sum(1)).max() <= 1e-12                 # a constant added to a row changes nothing
    assert total > 0


def test_distillation_special_cases():
    rng = np.random.default_rng(5)
    z = rng.standard_normal((2, 9)) * 3
    # the whole vocabulary as a list: the divergence of two softmax distributions, with or without the teacher's own sum
    t = rng.standard_normal((2, 9)) * 3
    ids = np.tile(np.arange(9), (2, 1))
    ref = torch.nn.functional.kl_div(torch.log_softmax(torch.from_numpy(z) / 1.5, 1), torch.log_softmax(torch.from_numpy(t) / 1.5, 1), reduction="none", log_target=True).sum(1).numpy()
    assert np.allclose(vo.distill(z, ids, t, 1.5)[0], ref)
    assert np.allclose(vo.distill(z, ids, t, 1.5, np.log(np.exp(t / 1.5).sum(1)))[0], ref)
    # one token: the cross entropy
    assert np.allclose(vo.distill(z, np.array([[3], [5]]), np.array([[0.2], [7.0]]))[0], [-vo.log_softmax(z[0])[0][3], -vo.log_softmax(z[1])[0][5]])
    # nothing listed: nothing to learn; the teacher's equal distribution: no loss, no gradient
    l, _, g = vo.distill(z, np.full((2, 1), -1), np.zeros((2, 1)), 1.0, np.zeros(2))
    assert np.allclose(l, 0) and np.allclose(g, 0)
    l, _, g = vo.distill(z, ids[:, :4], z[:, :4], 1.0, np.log(np.exp(z).sum(1)))
    assert np.allclose(l, 0) and np.allclose(g, 0)
