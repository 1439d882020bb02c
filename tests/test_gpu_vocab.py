"""Log probabilities, entropy and top alternatives, and the distillation loss with its gradient, against the oracle in 64 bits."""
import numpy as np
import pytest

from oracle import vocab_oracle as vo

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def make(rows, vocab, dtype, seed, pad=0, offset=0, scale=2.5, edit=None):
    """(logits on the device with a row stride of vocab + pad, `offset` elements into their buffer; the same in binary64)."""
    import torch
    rng = np.random.default_rng(seed)
    z = (rng.standard_normal((rows, vocab)) * scale).astype(np.float32)
    if edit is not None:
        edit(z, rng)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    buf = torch.full((rows * (vocab + pad) + offset,), float("nan"), dtype=td, device="cuda")
    t = buf[offset:].view(rows, vocab + pad)[:, :vocab]
    t.copy_(torch.from_numpy(z).cuda())
    return t, t.double().cpu().numpy()


def sum_error(vocab, temperature, spread):
    """Relative error of a row's sum: exponents (their argument is off by 2^-23 of itself, and the terms that count lie within the
    row's spread), the exponential's own last place, and as many additions as a thread makes in turn."""
    return ((spread / temperature + 4) * 4 + vocab / 512 + 40) * U


def run_logprobs(z, tokens, k, temperature):
    import torch
    from paper_2602_17681_amd import binding as ae
    rows, vocab = z.shape
    n = 0 if tokens is None else tokens.shape[1]
    f = lambda *s: torch.full(s, -7.0, device="cuda")      # noqa: E731
    out = dict(logprob=f(rows, n), entropy=f(rows), lse=f(rows), top_logit=f(rows, k), top_logprob=f(rows, k))
    out["top_id"] = torch.full((rows, k), -7, dtype=torch.int32, device="cuda")
    need = ae.model_token_logprobs_workspace(rows, vocab, k, ae.AE_BF16 if z.dtype == torch.bfloat16 else ae.AE_F32)
    ws = torch.full((max(16, need),), 0xFF, dtype=torch.uint8, device="cuda")
    ae.model_token_logprobs(z, rows, vocab, None if tokens is None else torch.from_numpy(tokens.astype(np.int32)).cuda(), k, out["logprob"], out["entropy"],
                            out["lse"], out["top_id"], out["top_logit"], out["top_logprob"], ws, temperature=temperature)
    return {n: t.cpu().numpy() for n, t in out.items()}


def near(got, want, tol):
    fine = np.isfinite(want)
    return np.array_equal(fine, np.isfinite(got)) and np.array_equal(np.isnan(got), np.isnan(want)) and \
        np.array_equal(got[np.isinf(want)], want[np.isinf(want)]) and np.all(np.abs(got - want)[fine] <= np.broadcast_to(tol, want.shape)[fine])


def check_logprobs(z, zh, k, temperature, seed=0):
    temperature = float(np.float32(temperature))           # the number that the call receives
    rows, vocab = z.shape
    rng = np.random.default_rng(seed + 1)
    tokens = rng.integers(-1, vocab + 1, (rows, 3))
    got, want = run_logprobs(z, tokens, k, temperature), vo.token_logprobs(zh, tokens, k, temperature)
    assert np.array_equal(got["top_id"], want["top_id"])
    assert np.array_equal(got["top_logit"].astype(np.float64), want["top_logit"], equal_nan=True)
    e = sum_error(vocab, temperature, 25.0)
    fin = np.where(np.isfinite(zh), np.abs(zh), 0).max(1) / temperature
    assert near(got["lse"], want["lse"], e + 6 * U * (fin + np.log(vocab) + 1))
    assert near(got["entropy"], want["entropy"], (e + 8 * U) * (np.log(vocab) + 2) * 2)
    for name in ("logprob", "top_logprob"):
        w = want[name]
        assert near(got[name], w, e + 8 * U * (np.where(np.isfinite(w), np.abs(w), 0) + np.log(vocab) + 1)), name


VOCABS = [1, 2, 7, 8, 63, 129, 511, 1000, 4095, 4096, 4097, 8200, 16391, 33000, 50021]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", VOCABS)
def test_logprobs_sizes(vocab, dtype):
    """One row and a few (pieces of rows that are joined), and enough rows for one workgroup each."""
    for rows, k, temperature, pad, offset in ((1, 5, 1.0, 0, 0), (3, 64, 0.7, 3, 1), (5, 0, 2.0, 0, 0), (260 if vocab < 9000 else 2, 1, 1.5, 1, 0)):
        z, zh = make(rows, vocab, dtype, vocab + rows, pad, offset)
        check_logprobs(z, zh, min(k, vocab), temperature, rows)


@pytest.mark.parametrize("rows", [2, 300])
def test_logprobs_longest_list(rows):
    z, zh = make(rows, 3000, "f32", 5)
    check_logprobs(z, zh, 256, 1.0)
    z, zh = make(rows, 256, "bf16", 6)
    check_logprobs(z, zh, 256, 1.0)                        # the whole vocabulary in order


EDITS = {
    "constant": lambda z, rng: z.__setitem__(slice(None), 1.25),                       # nothing but ties
    "two_values": lambda z, rng: np.copyto(z, np.where(rng.random(z.shape) < 0.3, 2.0, -1.0)),
    "rising": lambda z, rng: np.copyto(z, np.sort(z, 1)),
    "falling": lambda z, rng: np.copyto(z, -np.sort(-z, 1)),
    "zeros_of_both_signs": lambda z, rng: np.copyto(z, np.where(rng.random(z.shape) < 0.5, 0.0, -0.0)),
    "mostly_masked": lambda z, rng: z.__setitem__(rng.random(z.shape) < 0.999, -np.inf),
    "all_masked": lambda z, rng: z.__setitem__(slice(None), -np.inf),
    "one_left": lambda z, rng: (z.__setitem__(slice(None), -np.inf), z.__setitem__((slice(None), z.shape[1] // 2), 3.0)),
    "lowest": lambda z, rng: z.__setitem__(rng.random(z.shape) < 0.5, -3.3e38),
    "all_lowest": lambda z, rng: z.__setitem__(slice(None), -3.3e38),
    "lowest_then_one": lambda z, rng: (z.__setitem__(slice(None), -3.3e38), z.__setitem__((slice(None), -1), 3.0)),
    "large": lambda z, rng: np.multiply(z, 1e4, out=z),
    "peak_at_the_end": lambda z, rng: z.__setitem__((slice(None), -1), 80.0),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("edit", sorted(EDITS))
def test_logprobs_of_unusual_rows(edit, dtype):
    for rows, vocab in ((2, 9000), (257, 3001)):
        z, zh = make(rows, vocab, dtype, 8, edit=EDITS[edit])
        check_logprobs(z, zh, 40, 1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(4, 10000), (300, 700)])
def test_logprobs_nan_and_infinity_stay_in_their_row(rows, vocab, dtype):
    clean, ch = make(rows, vocab, dtype, 3)
    base = run_logprobs(clean, None, 10, 1.0)
    z = clean.clone()
    z[1, 17] = float("nan")
    z[2, vocab - 1] = float("inf")
    z[3, :] = float("nan")
    got = run_logprobs(z, np.tile([[3, 5]], (rows, 1)), 10, 1.0)
    keep = np.ones(rows, bool)
    keep[1:4] = False
    for n in ("entropy", "lse", "top_id", "top_logit", "top_logprob"):
        assert np.array_equal(got[n][keep], base[n][keep]), n
    for n in ("entropy", "lse", "logprob"):
        assert np.all(np.isnan(got[n][1:4])), n
    zh = z[1:4].double().cpu().numpy()
    assert np.array_equal(got["top_id"][1:4], vo.token_logprobs(zh, None, 10)["top_id"])


def test_logprobs_outputs_can_be_left_out():
    import torch
    from paper_2602_17681_amd import binding as ae
    z, zh = make(300, 500, "f32", 2)
    lse, ids = torch.empty(300, device="cuda"), torch.empty((300, 4), dtype=torch.int32, device="cuda")
    ae.model_token_logprobs(z, 300, 500, None, 4, None, None, lse, ids, None, None, None)
    full = run_logprobs(z, None, 4, 1.0)
    assert np.array_equal(ids.cpu().numpy(), full["top_id"]) and np.array_equal(lse.cpu().numpy(), full["lse"])
    ae.model_token_logprobs(z[:0], 0, 500, None, 4, None, None, lse[:0], None, None, None, None)


# ---- distillation ------------------------------------------------------------------------------------------------
def teacher(rng, rows, vocab, k, temperature, tail, short=False):
    ids = np.stack([rng.permutation(vocab)[:k] for _ in range(rows)]).astype(np.int32)
    t = -np.sort(-(rng.standard_normal((rows, k)) * 2 + 3), 1).astype(np.float32)
    if short:
        ids[np.arange(k)[None, :] >= rng.integers(0, k + 1, (rows, 1))] = -1
    lse = None
    if tail:
        x = np.where(ids >= 0, t.astype(np.float64) / temperature, -np.inf)
        with np.errstate(divide="ignore"):
            lse = np.log(np.exp(x).sum(1)) + rng.uniform(0.1, 0.7, rows)
        lse = np.where(np.isfinite(lse), lse, 2.0).astype(np.float32)
    return ids, t, lse


def run_distill(z, ids, t, temperature, lse=None, weight=None, in_place=False, pad=0):
    import torch
    from paper_2602_17681_amd import binding as ae
    rows, vocab = z.shape
    d = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()      # noqa: E731
    buf = torch.full((rows, vocab + pad), 5.0, dtype=z.dtype, device="cuda")
    g = z if in_place else buf[:, :vocab]
    loss_rows, loss = torch.full((rows,), -7.0, device="cuda"), torch.full((1,), -7.0, device="cuda")
    ws = torch.full((max(16, ae.model_loss_distill_workspace(rows, vocab, ae.AE_BF16 if z.dtype == torch.bfloat16 else ae.AE_F32)),), 0xFF, dtype=torch.uint8, device="cuda")
    ae.model_loss_distill(z, rows, vocab, d(ids), d(t), loss_rows, loss, g, ws, teacher_lse=d(lse), weight=d(weight), temperature=temperature)
    assert in_place or bool((buf[:, vocab:] == 5.0).all())
    return loss_rows.cpu().numpy(), loss.item(), g


def check_distill(z, zh, ids, t, temperature, lse, weight, in_place=False, pad=0):
    import torch
    temperature = float(np.float32(temperature))           # the number that the call receives
    dtype = z.dtype
    rows, vocab = z.shape
    w_rows, w_loss, w_grad = vo.distill(zh, ids, t, temperature, lse, weight)
    l_rows, l, g = run_distill(z, ids, t, temperature, lse, weight, in_place, pad)
    e = sum_error(vocab, temperature, 30.0)
    big = np.where(np.isfinite(zh), np.abs(zh), 0).max(1)
    assert near(l_rows, w_rows, 3 * e + 8 * U * (big * 0 + np.where(np.isfinite(w_rows), np.abs(w_rows), 0) + 1))
    w = np.ones(rows) if weight is None else weight.astype(np.float64)
    assert near(np.array([l]), np.array([w_loss]), ((3 * e + 8 * U) * np.abs(w)).sum() + 12 * U * np.abs(w_rows * w)[w != 0].sum() + 1e-30)
    # q is off by the sums' error and by its own exponent's, and so is what the rest of the teacher's mass is divided by
    gh = g.double().cpu().numpy()
    q = np.exp(np.stack([vo.log_softmax(r, temperature)[0] for r in zh]))
    x = np.minimum(np.where(np.isfinite(zh), zh.max(1, keepdims=True, initial=-3e38) - zh, 0) / temperature, 120.0)
    with np.errstate(all="ignore"):
        # the factor of the entries outside, up to a rounding of the tail's quotient
        f = np.abs(w)[:, None] / temperature * np.maximum(1.0, tail_factor(zh, ids, t, temperature, lse))[:, None]
        tol = f * np.nan_to_num(q) * (3 * e + 4 * U * (x + 4)) + 4 * U * np.abs(w_grad) + 1e-37
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * np.abs(w_grad)
    assert near(gh, w_grad, tol)


def tail_factor(zh, ids, t, temperature, lse):
    """P + p_r / q_r of each row: how far the gradient outside the list magnifies an error of q."""
    out = np.ones(len(zh))
    for r in range(len(zh)):
        there = (ids[r] >= 0) & (ids[r] < zh.shape[1])
        if lse is None:
            continue
        p = np.exp(t[r][there].astype(np.float64) / temperature - float(lse[r]))
        q = np.exp(vo.log_softmax(zh[r], temperature)[0])
        q[ids[r][there]] = 0
        rest = max(0.0, 1 - p.sum())
        out[r] = p.sum() + rest + (rest / q.sum() if q.sum() > 0 else 0)
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("vocab", [1, 2, 9, 64, 130, 1001, 4096, 4104, 9999, 33000, 50021])
def test_distill_sizes(vocab, tail, dtype):
    for rows, k, temperature, pad, offset in ((1, 1, 1.0, 0, 0), (3, 20, 1.5, 3, 1), (260 if vocab < 5000 else 4, 64, 0.7, 1, 0)):
        k = min(k, vocab)
        rng = np.random.default_rng(vocab + rows)
        ids, t, lse = teacher(rng, rows, vocab, k, temperature, tail)
        z, zh = make(rows, vocab, dtype, vocab + rows + 1, pad, offset)
        weight = None if rows == 1 else rng.uniform(0.2, 2.0, rows).astype(np.float32)
        check_distill(z, zh, ids, t, temperature, lse, weight, pad=pad)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(3, 20000), (300, 1200)])
def test_distill_short_lists_weights_and_masks(rows, vocab, dtype):
    """Lists of different lengths down to none, rows without weight that hold NaN, empty rows, masked logits outside the list."""
    rng = np.random.default_rng(vocab)
    for tail in (False, True):
        ids, t, lse = teacher(rng, rows, vocab, 24, 1.5, tail, short=True)
        keep = np.zeros((rows, vocab), bool)
        for r in range(rows):
            keep[r, ids[r][ids[r] >= 0]] = True

        def edit(z, g):
            z[(g.random(z.shape) < 0.3) & ~keep] = -np.inf
            z[(g.random(z.shape) < 0.1) & ~keep] = -3.3e38
            z[1] = -np.inf
        z, zh = make(rows, vocab, dtype, 4, edit=edit)
        weight = rng.uniform(0.5, 1.5, rows).astype(np.float32)
        weight[2::5] = 0
        z[2, 5] = float("nan")
        check_distill(z, zh, ids, t, 1.5, lse, weight)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(2, 30000), (270, 900)])
def test_distill_gradient_in_the_logits_place(rows, vocab, dtype):
    rng = np.random.default_rng(6)
    ids, t, lse = teacher(rng, rows, vocab, 40, 1.0, True)
    ids[0, :6] = [0, 1, 2, 7, 8, vocab - 1]
    ids[0, 6:] = np.setdiff1d(rng.permutation(vocab), ids[0, :6])[:34]
    z, zh = make(rows, vocab, dtype, 9)
    _, _, g = run_distill(z.clone(), ids, t, 1.0, lse)
    z2 = z.clone()
    _, _, g2 = run_distill(z2, ids, t, 1.0, lse, in_place=True)
    assert g2 is z2 and np.array_equal(g.float().cpu().numpy(), g2.float().cpu().numpy())
    check_distill(z, zh, ids, t, 1.0, lse, None, in_place=True)


@pytest.mark.parametrize("tail", [False, True])
def test_distill_whole_vocabulary_as_list(tail):
    """The full divergence: no tail is left, whatever rounding makes of 1 - sum p."""
    rng = np.random.default_rng(2)
    for rows, vocab in ((2, 5000), (256, 300)):
        ids = np.stack([rng.permutation(vocab) for _ in range(rows)]).astype(np.int32)
        t = (rng.standard_normal((rows, vocab)) * 2).astype(np.float32)
        lse = np.log(np.exp(t.astype(np.float64)).sum(1)).astype(np.float32) if tail else None
        z, zh = make(rows, vocab, "f32", 1)
        check_distill(z, zh, ids, t, 1.0, lse, None)


def test_distill_infinite_loss_and_nan():
    """The student rules out what the teacher holds possible; a NaN, an infinity: in their own rows only."""
    rng = np.random.default_rng(3)
    rows, vocab = 260, 400
    ids, t, lse = teacher(rng, rows, vocab, 8, 1.0, True)
    z, zh = make(rows, vocab, "f32", 1)
    clean_rows, _, clean = run_distill(z, ids, t, 1.0, lse)
    z2 = z.clone()
    z2[0, int(ids[0, 0])] = -float("inf")
    z2[1, 7], z2[2, 9] = float("nan"), float("inf")
    l, _, g = run_distill(z2, ids, t, 1.0, lse)
    assert l[0] == np.inf and np.isfinite(g[0].cpu().numpy()).all()
    assert np.isnan(l[1:3]).all() and np.isnan(g[1:3].cpu().numpy()).all()
    assert np.array_equal(l[3:], clean_rows[3:]) and bool((g[3:] == clean[3:]).all())


@pytest.mark.parametrize("rows", [2, 260])
def test_distill_gradient_against_differences(rows):
    """Central differences of the loss: their own error is of the step's square, 0.05^2 / 6 of a third derivative below 1 / T^3."""
    rng = np.random.default_rng(5)
    vocab, temperature, h = 600, 1.3, 0.05
    ids, t, lse = teacher(rng, rows, vocab, 12, temperature, True)
    z, _ = make(rows, vocab, "f32", 2, scale=1.0)
    _, _, g = run_distill(z, ids, t, temperature, lse)
    for j in [0, 5, 599] + [int(i) for i in ids[0, :4]]:
        up, down = z.clone(), z.clone()
        up[:, j] += h
        down[:, j] -= h
        num = (run_distill(up, ids, t, temperature, lse)[0].astype(np.float64) - run_distill(down, ids, t, temperature, lse)[0]) / (2 * h)
        # binary32 losses of about 5 that differ by 2 h g
        assert np.all(np.abs(num - g[:, j].double().cpu().numpy()) <= h * h / 6 / temperature ** 3 + 2 * 8 * U * 8 / (2 * h))


def test_distill_outputs_can_be_left_out():
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(7)
    for rows, vocab in ((3, 9000), (300, 200)):
        ids, t, _ = teacher(rng, rows, vocab, 5, 1.0, False)
        z, _ = make(rows, vocab, "bf16", 3)
        l, total, g = run_distill(z, ids, t, 1.0)
        di, dt = torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda()
        ws = torch.empty(ae.model_loss_distill_workspace(rows, vocab, ae.AE_BF16), dtype=torch.uint8, device="cuda")
        one = torch.empty(1, device="cuda")
        ae.model_loss_distill(z, rows, vocab, di, dt, None, one, None, ws)
        assert one.item() == total
        g2 = torch.empty_like(g)
        ae.model_loss_distill(z, rows, vocab, di, dt, None, None, g2, ws)
        assert torch.equal(g2, g)
    zero = torch.full((1,), 3.0, device="cuda")
    ae.model_loss_distill(z[:0], 0, 200, di[:0], dt[:0], None, zero, None, ws)
    assert zero.item() == 0.0


def test_largest_vocabulary():
    """2^20 columns: pieces of one row, and whole rows with the marks of the whole vocabulary in LDS."""
    import torch
    from paper_2602_17681_amd import binding as ae
    vocab = 1 << 20
    for rows in (1, 256):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(rows)
        z = (torch.randn((rows, vocab), device="cuda", generator=gen) * 2).bfloat16()
        ids = torch.tensor([[0, 5, vocab - 1, 70000]], dtype=torch.int32, device="cuda").repeat(rows, 1)
        t = torch.tensor([[4.0, 3.0, 2.0, 1.0]], device="cuda").repeat(rows, 1)
        loss_rows, g = torch.empty(rows, device="cuda"), torch.empty_like(z)
        ws = torch.empty(ae.model_loss_distill_workspace(rows, vocab, ae.AE_BF16), dtype=torch.uint8, device="cuda")
        ae.model_loss_distill(z, rows, vocab, ids, t, loss_rows, None, g, ws)
        lse, top = torch.empty(rows, device="cuda"), torch.empty((rows, 3), dtype=torch.int32, device="cuda")
        w2 = torch.empty(max(16, ae.model_token_logprobs_workspace(rows, vocab, 3, ae.AE_BF16)), dtype=torch.uint8, device="cuda")
        ae.model_token_logprobs(z, rows, vocab, None, 3, None, None, lse, top, None, None, w2)
        for r in (0, rows - 1):
            zr = z[r].double()
            ref = torch.logsumexp(zr, 0)
            assert abs(lse[r].item() - ref.item()) <= sum_error(vocab, 1.0, 25.0) + 8 * U * 20
            p = torch.softmax(t[r].double(), 0)
            want = (p * (torch.log(p) - (zr[ids[r].long()] - ref))).sum()
            assert abs(loss_rows[r].item() - want.item()) <= 3 * sum_error(vocab, 1.0, 25.0) + 8 * U * 20
            q = torch.exp(zr - ref)
            q[ids[r].long()] -= p
            assert bool(((g[r].double() - q).abs() <= 2.0 ** -8 * q.abs() + q.abs() * 1e-3 + 1e-37 + 4 * U * (ids.shape[1] and 1)).all())
            best = torch.sort(zr, descending=True, stable=True).indices[:3]
            assert top[r].tolist() == best.tolist()


@pytest.mark.parametrize("rows", [3, 300])
def test_other_streams_and_captured_graphs(rows):
    import torch
    from paper_2602_17681_amd import binding as ae
    vocab, k = 9000 if rows == 3 else 1111, 12
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    z = torch.randn((rows, vocab), device="cuda", generator=gen).bfloat16()
    f = lambda *s: torch.empty(s, device="cuda")      # noqa: E731
    lse, ent, tl, tp, lr, l = f(rows), f(rows), f(rows, k), f(rows, k), f(rows), f(1)
    ids, g = torch.empty((rows, k), dtype=torch.int32, device="cuda"), torch.empty_like(z)
    ws = torch.empty(max(16, ae.model_token_logprobs_workspace(rows, vocab, k, ae.AE_BF16), ae.model_loss_distill_workspace(rows, vocab, ae.AE_BF16)), dtype=torch.uint8, device="cuda")

    def call():
        ae.model_token_logprobs(z, rows, vocab, None, k, None, ent, lse, ids, tl, tp, ws, temperature=1.5)
        ae.model_loss_distill(z, rows, vocab, ids, tl, lr, l, g, ws, teacher_lse=lse, temperature=1.5)
    outs = (lse, ent, tl, tp, lr, l, ids, g)
    call()
    assert float(lr.abs().max()) <= 1e-4                   # a teacher that is the student
    eager = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for o in outs:
            o.zero_()
        call()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(outs, eager))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        z.copy_(torch.randn((rows, vocab), device="cuda", generator=gen).bfloat16())
        call()
        eager = [o.clone() for o in outs]
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager))
