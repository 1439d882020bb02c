"""Rows of logits whose maximum over the temperature is large: differences to the maximum are what counts, whichever form of the
kernel takes the row; against 64 bits on the device."""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
LEVELS = [1e5, -1e5, 1e7, -1e9, 1e9, -3e9, 3e9, -1e10, 1e10, -1e12, 1e12, 1e15, -1e20, 1e20, -1e30, 1e30, -2e38]
# rows x columns that each form of the kernel takes: rows in registers of 256, 512 and 1 024 threads, with 4, 8 and 16 vectors,
# pieces, rows read twice (no gradient, long lists)
SHAPES = {"bf16": [(300, 4003), (300, 12005), (300, 30001), (300, 60004), (400, 131072), (60, 30001)],
          "f32": [(300, 2003), (300, 6005), (300, 15001), (300, 30002), (400, 65536), (60, 30001)]}


def sum_error(vocab):
    """Relative error of a row's sum: exponents (off by 2^-23 of themselves, those that count lie within 30), the exponential's own
    last place, and as many additions as a thread makes in turn."""
    return ((30.0 + 4) * 4 + vocab / 512 + 40) * U


def distill_64(z, ids, t, temperature, lse):
    """(loss, gradient, bound of what the gradient's terms are) of every row, a few rows at a time."""
    import torch
    losses, grads, sizes = [], [], []
    for r in range(0, z.shape[0], 50):
        x, at = z[r:r + 50].double(), ids[r:r + 50]
        # relative to the maximum before the division, so that nothing is lost of differences next to a large maximum
        m = x.amax(1, keepdim=True)
        d = (x - m) / temperature
        logq = d - torch.log(torch.exp(d).sum(1, keepdim=True))
        q = torch.exp(logq)
        tt = t[r:r + 50].double()
        if lse is None:
            dt = (tt - tt.amax(1, keepdim=True)) / temperature
            logp = dt - torch.log(torch.exp(dt).sum(1, keepdim=True))
        else:
            logp = tt / temperature - lse[r:r + 50].double()[:, None]
        p = torch.exp(logp)
        outside = torch.ones_like(q, dtype=torch.bool).scatter_(1, at, False)
        log_out = torch.logsumexp(torch.where(outside, logq, -math.inf), 1)
        rest = (1 - p.sum(1)).clamp(min=0) if lse is not None else torch.zeros_like(log_out)
        rest = torch.where(log_out > -700, rest, 0.0)
        loss = torch.where(p > 0, p * (logp - logq.gather(1, at)), 0.0).sum(1) + torch.where(rest > 0, rest * (torch.log(rest) - log_out), 0.0)
        mass = p.sum(1) + rest
        pull = torch.where((rest > 0)[:, None] & outside, rest[:, None] * torch.exp(logq - log_out[:, None]), 0.0)
        g = (mass[:, None] * q - pull).scatter_add_(1, at, -p)
        losses.append(loss)
        grads.append(g / temperature)
        sizes.append((mass[:, None] * q + pull) / temperature)
    return torch.cat(losses), torch.cat(grads), torch.cat(sizes)


def check(z, ids, t, temperature, lse=None, long_list=False):
    """The call in its usual form, in the logits' place, and without a gradient; temperature as the call receives it."""
    import numpy as np
    import torch
    from paper_2602_17681_amd import binding as ae
    temperature = float(np.float32(temperature))
    rows, vocab = z.shape
    dt = ae.AE_BF16 if z.dtype == torch.bfloat16 else ae.AE_F32
    loss, grad, size = distill_64(z, ids, t, temperature, lse)
    ws = torch.full((ae.model_loss_distill_workspace(rows, vocab, dt),), 0xFF, dtype=torch.uint8, device="cuda")
    lr, total, g = torch.full((rows,), -7.0, device="cuda"), torch.full((1,), -7.0, device="cuda"), torch.full_like(z, 3.0)
    i32 = ids.to(torch.int32)
    ae.model_loss_distill(z, rows, vocab, i32, t, lr, total, g, ws, teacher_lse=lse, temperature=temperature)
    e = sum_error(vocab)
    tol = size * (3 * e + 4 * U * 124) + 4 * U * grad.abs() + 1e-37
    if z.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * grad.abs()
    assert bool(((g.double() - grad).abs() <= tol).all())
    near = lambda a: bool(((a.double() - loss).abs() <= 3 * e + 8 * U * (loss.abs() + 1)).all())      # noqa: E731
    assert near(lr)
    want = loss.sum().item()
    if want > torch.finfo(torch.float32).max:              # losses of 1e38 at the lowest temperatures: their sum is no binary32 number
        assert total.item() == math.inf
    else:
        assert abs(total.item() - want) <= rows * 3 * e + 12 * U * (loss.abs().sum().item() + rows)
    lr2 = torch.full_like(lr, -7.0)
    ae.model_loss_distill(z, rows, vocab, i32, t, lr2, None, None, ws, teacher_lse=lse, temperature=temperature)
    assert near(lr2)
    ae.model_loss_distill(z, rows, vocab, i32, t, lr2, None, z, ws, teacher_lse=lse, temperature=temperature)
    assert torch.equal(z, g) and torch.equal(lr2, lr)


def make(rows, vocab, dtype, k, seed=3):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    z = (torch.randn((rows, vocab), generator=gen, device="cuda") * 2.5).to(td)
    share = vocab // k
    ids = (torch.rand((rows, k), generator=gen, device="cuda") * share).long().clamp_(max=share - 1) + torch.arange(k, device="cuda") * vocab // k
    t = (torch.randn((rows, k), generator=gen, device="cuda") * 2 + 6).sort(1, descending=True).values
    return z, ids, t, gen


@pytest.mark.parametrize("temperature", [0.3, 0.7, 1.0, 1.5, 2.0])
@pytest.mark.parametrize("dtype,rows,vocab,k", [(d, r, v, 20) for d in SHAPES for r, v in SHAPES[d]] + [("bf16", 300, 4003, 300), ("f32", 300, 2003, 300)])
def test_distill_of_rows_with_a_large_maximum(dtype, rows, vocab, k, temperature):
    """Rows of one value (all masked with it), rows with a forced token, rows of two values near it."""
    import torch
    z, ids, t, gen = make(rows, vocab, dtype, k)
    n = len(LEVELS)
    for i, v in enumerate(LEVELS):
        z[i] = v
        z[n + i, (7 * i + 5) % vocab] = abs(v)
        z[n + i, ids[n + i]] = abs(v)                      # the teacher's tokens too: the loss stays of the list's size
        z[2 * n + i] = v
        z[2 * n + i, torch.rand(vocab, generator=gen, device="cuda") < 0.3] = v * (1 + 2.0 ** -6) if v < 0 else v * (1 - 2.0 ** -6)
        z[2 * n + i, ids[2 * n + i]] = v
    for tail in (False, True):
        lse = (torch.logsumexp(t.double() / float(torch.tensor(temperature)), 1) + 0.4).float() if tail else None
        check(z.clone(), ids, t, temperature, lse)


@pytest.mark.parametrize("base", [1e10, -1e10, 3e8])
@pytest.mark.parametrize("rows,vocab", SHAPES["f32"])
def test_distill_of_neighbouring_large_logits(rows, vocab, base):
    """Logits a few last places apart, at a temperature at which these differences count."""
    import torch
    z, ids, t, gen = make(rows, vocab, "f32", 20)
    step = abs(base) * 2.0 ** -23
    z.copy_(torch.randint(-16, 17, (rows, vocab), generator=gen, device="cuda") * step + base)
    t *= step
    check(z, ids, t, 2.5 * step)


@pytest.mark.parametrize("temperature", [1.2e-38, 1e-31, 1e-20, 1e-8])
@pytest.mark.parametrize("dtype,rows,vocab", [(d, r, v) for d in SHAPES for r, v in SHAPES[d]])
def test_distill_at_the_lowest_temperatures(dtype, rows, vocab, temperature):
    """All of a row's probability lies with its maximum, or is shared by those that equal it."""
    z, ids, t, _ = make(rows, vocab, dtype, 20)
    z[:, 3], z[::3, vocab - 2] = 12.0, 12.0
    ids[:, 0] = 3
    t[:, 0] = 20.0
    z[1::4] *= -1
    z[1::4, 3] = 15.0
    check(z, ids, t, temperature)
