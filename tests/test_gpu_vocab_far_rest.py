"""Distillation where the student's probability outside the teacher's list is far below what a binary32 number holds next to the
row's maximum: the remaining mass of the teacher still counts, up to a gap of 708 T.  Against 64 bits on the device."""
import math

import pytest

from test_gpu_vocab_large import SHAPES, check, make

pytestmark = pytest.mark.gpu

ALL = [(d, r, v) for d in SHAPES for r, v in SHAPES[d]] + [("bf16", 5, 40001), ("f32", 2, 131077)]


def teacher_lse(t, temperature):
    """The teacher's lse that leaves it a rest of a third."""
    import torch
    return (torch.logsumexp(t.double() / float(torch.tensor(temperature)), 1) + math.log(1.5)).float()


@pytest.mark.parametrize("temperature", [0.25, 1.0, 2.0])
@pytest.mark.parametrize("dtype,rows,vocab", ALL)
def test_list_far_above_the_rest(dtype, rows, vocab, temperature):
    """Gaps from a little over what binary32 sums hold to nearly the largest that counts; between, all but a few of the others masked."""
    import torch
    z, ids, t, gen = make(rows, vocab, dtype, 20)
    gaps = torch.tensor([60.0, 80.0, 86.0, 88.0, 92.0, 100.0, 104.0, 150.0, 300.0, 600.0, 20.0, 28.0], device="cuda")
    gap = (gaps[torch.arange(rows, device="cuda") % len(gaps)] * temperature)[:, None]
    near = torch.rand((rows, 20), generator=gen, device="cuda") * 0.5
    near[::2, 3:] = 0.0                                    # several equal maxima
    z.mul_(0.25)
    if rows > 30:                                          # one other token that can occur at all, or two; in the last column, too
        z[24:30] = -math.inf
        z[24:30, 7], z[26:30, vocab - 1] = 0.5, 0.25
        z[28, :] = torch.finfo(z.dtype).min                # the others by the type's lowest number
        z[28, 11] = 0.0
    z.scatter_(1, ids, (gap + near).to(z.dtype))
    check(z, ids, t, temperature, teacher_lse(t, temperature))


@pytest.mark.parametrize("dtype,rows,vocab", ALL)
def test_list_above_everything_that_counts(dtype, rows, vocab):
    """Others that are masked with -infinity or a low number are none: the teacher's remaining mass is left out."""
    import torch
    z, ids, t, _ = make(rows, vocab, dtype, 20)
    lows = [-math.inf, torch.finfo(z.dtype).min, -1e30, -1e9, -1e4, -2e3]
    for r in range(rows):
        z[r] = lows[r % len(lows)]
    z.scatter_(1, ids, (t * 0.3).to(z.dtype))
    check(z, ids, t, 1.0, teacher_lse(t, 1.0))


@pytest.mark.parametrize("rows,vocab", [(300, 2003), (300, 30002), (40, 30001)])
def test_far_rest_next_to_a_large_maximum(rows, vocab):
    """Both at once: logits of 1e10 a few last places apart, of which those of the list lie 100 T above the others."""
    import torch
    z, ids, t, gen = make(rows, vocab, "f32", 20)
    step = 1024.0
    z.copy_(torch.randint(-3, 4, (rows, vocab), generator=gen, device="cuda") * step + 9.9e9)
    z.scatter_(1, ids, torch.randint(0, 3, (rows, 20), generator=gen, device="cuda") * step + (9.9e9 + 250 * step))
    t *= step
    check(z, ids, t, 2.5 * step, teacher_lse(t, 2.5 * step))


def test_whole_vocabulary_as_list_leaves_no_rest():
    import torch
    z, ids, t, _ = make(300, 40, "f32", 40)
    z, ids = z.contiguous(), torch.arange(40, device="cuda").repeat(300, 1)
    lse = (torch.logsumexp(t.double(), 1) + 0.3).float()
    check(z, ids, t, 1.0, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(40, 30001), (300, 6005)])
def test_long_lists_with_masked_entries(rows, vocab, dtype):
    """More entries than threads, some of them with tokens that neither side holds possible: the others keep their digits."""
    import torch
    k = 1300
    z, ids, t, gen = make(rows, vocab, dtype, k)
    off = torch.rand((rows, k), generator=gen, device="cuda") < 0.5
    at = z.gather(1, ids)
    z.scatter_(1, ids, torch.where(off, torch.full((), torch.finfo(z.dtype).min, dtype=z.dtype, device="cuda"), at))
    t.masked_fill_(off, -math.inf)
    check(z, ids, t, 1.5, teacher_lse(t, 1.5))
    z.scatter_(1, ids, torch.where(off, torch.full((), -math.inf, dtype=z.dtype, device="cuda"), at + 200))
    check(z, ids, t, 1.5, teacher_lse(t, 1.5))
