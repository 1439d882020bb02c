"""The operators behind the calibration and the evaluation of a quantised output layer, as cases of known size.

  linear       y = x W^T + b with E4M3 codes on both sides and a scale for each block of 128: x is quantised in the call
  linear_grad  the backward pass of the same layer: dX = dY W and dW = dY^T X, both as products of E4M3 codes
  logprobs     log probabilities of given tokens, entropy, log-sum-exp and the top alternatives of every row of logits
  distill      the KL divergence from a teacher's top logits at a temperature, with the gradient of the student's logits

A case is a dict of plain values; `prepare` makes what a program holds before the call, `run` is one pass, in elementary
torch operations in binary32 (`own` false) or through the library's entry points (`own` true).
"""
import math

import torch

own = False

BLOCK = 128                      # elements that share a scale
E4M3_MAX = 448.0                 # largest magnitude of the codes
SCALE_MIN = 2.0 ** -126          # smallest normal binary32: the scale of a block of zeros
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- the cases ---------------------------------------------------------------------------------------------------
def listed():
    return [
        # one token through a square projection, as in single-sequence decoding: the weights are read for one row
        dict(name="linear_token", op="linear", m=1, n=4096, k=4096, dtype="bf16", bias=False),
        # a decoding batch of 16 sequences through a widening projection with a folded bias
        dict(name="linear_batch", op="linear", m=16, n=8192, k=4096, dtype="bf16", bias=True),
        # a user's own sizes: no side a multiple of a tile, rows of x on no 16-byte border, binary32 results
        dict(name="linear_ragged", op="linear", m=777, n=1500, k=1003, dtype="f32", bias=True),
        # a calibration batch of 16 sequences of 1 024 tokens through a square projection
        dict(name="linear_prompt", op="linear", m=16384, n=4096, k=4096, dtype="bf16", bias=True),
        # the backward pass of a training step on 4 sequences of 1 024 tokens
        dict(name="linear_train", op="linear_grad", m=4096, n=4096, k=4096, dtype="bf16"),
        # the backward pass of a small layer on a batch whose token count is odd
        dict(name="linear_train_ragged", op="linear_grad", m=1001, n=520, k=1000, dtype="f32"),
        # a decoding step: four sequences, the sampled token's log probability and eight alternatives
        dict(name="logprobs_decode", op="logprobs", rows=4, vocab=131072, dtype="bf16", tokens=1, top=8, temperature=0.8, masked=False),
        # scoring answers: three candidate tokens per position, odd vocabulary, constrained rows, binary32 logits
        dict(name="logprobs_ragged", op="logprobs", rows=333, vocab=50021, dtype="f32", tokens=3, top=20, temperature=1.0, masked=True),
        # the teacher's pass over two calibration sequences of 1 024 tokens: its 64 top logits are kept
        dict(name="logprobs_teacher", op="logprobs", rows=2048, vocab=131072, dtype="bf16", tokens=1, top=64, temperature=1.5, masked=False),
        # one short answer, renormalised over the teacher's list
        dict(name="distill_small", op="distill", rows=4, vocab=32768, dtype="f32", top=16, temperature=1.0, tail=False, masked=False),
        # odd vocabulary, lists of different lengths, rows without weight, the teacher's remaining mass as one more outcome
        dict(name="distill_ragged", op="distill", rows=257, vocab=50021, dtype="f32", top=20, temperature=2.0, tail=True, masked=True),
        # a calibration step on 8 sequences of 1 024 tokens at the paper's temperature
        dict(name="distill_step", op="distill", rows=8192, vocab=131072, dtype="bf16", top=64, temperature=1.5, tail=True, masked=False),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear_grad", "logprobs", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("linear", "linear_grad"):
        m = _log_uniform(rng, 1 if op == "linear" else 64, 16384)
        n, k = _log_uniform(rng, 64, 16384), _log_uniform(rng, 64, 16384)
        if rng.random() < 0.5:                       # widths of whole blocks, as most layers have them
            n, k = max(BLOCK, n // BLOCK * BLOCK), max(BLOCK, k // BLOCK * BLOCK)
        most = (1 if op == "linear" else 0.5) * 16384 * 4096 * 4096
        while m * n * k > most:
            m = max(1, m // 2)
        return dict(op=op, m=m, n=n, k=k, dtype=dtype, **({"bias": rng.random() < 0.5} if op == "linear" else {}))
    vocab = _log_uniform(rng, 1000, 200000)
    if rng.random() < 0.5:
        vocab = vocab // 64 * 64
    rows = min(_log_uniform(rng, 1, 8192), (8192 if op == "distill" else 2048) * 131072 // vocab)
    if dtype == "f32":
        rows = max(1, rows // 2)
    c = dict(op=op, rows=rows, vocab=vocab, dtype=dtype, temperature=rng.choice([0.7, 1.0, 1.5, 2.0]), masked=rng.random() < 0.4)
    if op == "logprobs":
        return dict(c, tokens=rng.randint(1, 4), top=rng.choice([0, 1, 5, 20, rng.randint(2, 128)]))
    return dict(c, top=_log_uniform(rng, 1, 256), tail=rng.random() < 0.5)


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] in ("linear", "linear_grad"):
        m, n, k = case["m"], case["n"], case["k"]
        w = n * k + 4 * -(-n // BLOCK) * -(-k // BLOCK)
        if case["op"] == "linear":
            return {"bytes": m * k * e + w + m * n * e + (4 * n if case["bias"] else 0), "flops": 2.0 * m * n * k}
        return {"bytes": m * n * e + m * k * e + w + m * k * e + n * k * 4, "flops": 4.0 * m * n * k}
    rows, vocab, k = case["rows"], case["vocab"], case["top"]
    if case["op"] == "logprobs":
        # each logit: its difference to the maximum, an exponential, the sum and the entropy's sum
        return {"bytes": rows * (vocab * e + case["tokens"] * 8 + 8 + k * 12), "flops": 6.0 * rows * vocab}
    # each logit: difference, exponential and sum; the same again and two products for its gradient
    return {"bytes": rows * (2 * vocab * e + 8 * k + 12), "flops": 8.0 * rows * vocab}


# ---- the inputs --------------------------------------------------------------------------------------------------
def _pad16(n):
    return -(-n // 16) * 16


def _codes(rows, cols):
    """Room for rows x cols codes whose rows begin on 16-byte borders."""
    return torch.empty((rows, _pad16(cols)), dtype=torch.float8_e4m3fn, device="cuda")[:, :cols]


def _activations(gen, rows, cols, dtype):
    """Roughly Gaussian, with a few features that are many times larger than the rest, as hidden states have."""
    x = torch.randn((rows, cols), generator=gen, device="cuda")
    gain = torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.01, 20.0, 1.0)
    return x.mul_(gain).to(dtype)


def _logits(gen, rows, vocab, dtype, masked):
    z = torch.randn((rows, vocab), generator=gen, device="cuda").mul_(2.5)
    if masked:      # constrained decoding: tokens that are not allowed, by -inf or by the type's lowest value; one row allows nothing
        u = torch.rand((rows, vocab), generator=gen, device="cuda")
        z.masked_fill_(u < 0.1, -math.inf)
        z.masked_fill_(u > 0.95, torch.finfo(dtype).min)
        if rows > 2:
            z[rows // 2] = -math.inf
    return z.to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = DTYPE[case["dtype"]]
    s = dict(case=case)
    if case["op"] in ("linear", "linear_grad"):
        m, n, k = case["m"], case["n"], case["k"]
        w = torch.randn((n, k), generator=gen, device="cuda").mul_(k ** -0.5)
        codes, scales = _quantize(w, tiles=True)
        s["x"] = _activations(gen, m, k, dt)
        if case["op"] == "linear":
            s["w"], s["w_scale"] = _codes(n, k), scales.contiguous()
            s["w"].copy_(codes)
            s["bias"] = torch.randn(n, generator=gen, device="cuda") if case["bias"] else None
            s["y"] = torch.empty((m, n), dtype=dt, device="cuda")
        else:
            # the layer keeps the transposed codes for its backward pass: the same codes and the same scales
            s["wt"], s["wt_scale"] = _codes(k, n), scales.t().contiguous()
            s["wt"].copy_(codes.t())
            s["dy"] = torch.randn((m, n), generator=gen, device="cuda").mul_(1e-3).to(dt)
            s["dx"] = torch.empty((m, k), dtype=dt, device="cuda")
            s["dw"] = torch.empty((n, k), dtype=torch.float32, device="cuda")
            mb, nb = -(-m // BLOCK), -(-n // BLOCK)
            s["dy_q"], s["dy_s"] = _codes(m, n), torch.empty((nb, m), device="cuda")
            s["dyt_q"], s["dyt_s"] = _codes(n, m), torch.empty((mb, n), device="cuda")
            s["xt_q"], s["xt_s"] = _codes(k, m), torch.empty((mb, k), device="cuda")
        return s
    rows, vocab, top = case["rows"], case["vocab"], case["top"]
    s["logits"] = _logits(gen, rows, vocab, dt, case["masked"])
    if case["op"] == "logprobs":
        s["tokens"] = torch.randint(0, vocab, (rows, case["tokens"]), generator=gen, device="cuda", dtype=torch.int32)
        if case["masked"]:      # the scored tokens are allowed ones, but for the row that allows nothing; some positions are not scored
            z = torch.randn(vocab, generator=gen, device="cuda").mul_(2.5).to(dt)[s["tokens"].long()]
            if rows > 2:
                z[rows // 2] = -math.inf
            s["logits"].scatter_(1, s["tokens"].long(), z)
            s["tokens"].masked_fill_(torch.rand((rows, case["tokens"]), generator=gen, device="cuda") < 0.1, -1)
        f = lambda *shape: torch.empty(shape, device="cuda")  # noqa: E731
        s.update(logprob=f(rows, case["tokens"]), entropy=f(rows), lse=f(rows), top_logit=f(rows, top), top_logprob=f(rows, top),
                 top_id=torch.empty((rows, top), dtype=torch.int32, device="cuda"))
        return s
    # distinct tokens in the teacher's lists, in the order of its logits; the student has learned some of it already
    share = vocab // top
    ids = (torch.rand((rows, top), generator=gen, device="cuda") * share).long().clamp_(max=share - 1) + torch.arange(top, device="cuda") * vocab // top
    ids = ids.gather(1, torch.rand((rows, top), generator=gen, device="cuda").argsort(1))
    s["logits"].scatter_(1, ids, (torch.randn((rows, top), generator=gen, device="cuda") * 2 + 6).to(dt))
    t = (torch.randn((rows, top), generator=gen, device="cuda") * 2 + 8).sort(1, descending=True).values
    s["teacher_lse"] = torch.logsumexp(t / case["temperature"], 1) + 0.05 + 0.6 * torch.rand(rows, generator=gen, device="cuda") if case["tail"] else None
    s["weight"] = torch.rand(rows, generator=gen, device="cuda") + 0.5
    if case["masked"]:          # shorter lists, and rows that do not count
        ids.masked_fill_(torch.arange(top, device="cuda") >= torch.randint(1, top + 1, (rows, 1), generator=gen, device="cuda"), -1)
        s["weight"].masked_fill_(torch.rand(rows, generator=gen, device="cuda") < 0.2, 0.0)
        if rows > 2:
            s["logits"][rows // 2] = -math.inf
    s["top_id"], s["top_logit"] = ids.to(torch.int32), t
    s["loss_rows"], s["loss"] = torch.empty(rows, device="cuda"), torch.empty(1, device="cuda")
    s["d_logits"] = torch.empty_like(s["logits"])
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------
def _quantize(x, tiles=False):
    """E4M3 codes of x and their scales: [block of columns][row], or [block of rows][block of columns] for tiles."""
    rows, cols = x.shape
    cb = -(-cols // BLOCK)
    x = torch.nn.functional.pad(x.float(), (0, cb * BLOCK - cols))
    amax = x.abs().view(rows, cb, BLOCK).amax(2)
    if tiles:
        rb = -(-rows // BLOCK)
        amax = torch.nn.functional.pad(amax, (0, 0, 0, rb * BLOCK - rows)).view(rb, BLOCK, cb).amax(1)
    s = (amax / torch.full_like(amax, E4M3_MAX)).clamp(min=SCALE_MIN)      # quotients of tensors: correctly rounded
    inv = torch.ones_like(s) / s
    if tiles:
        inv = inv.repeat_interleave(BLOCK, 0)[:rows]
    q = (x.view(rows, cb, BLOCK) * inv[:, :, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return q.view(rows, cb * BLOCK)[:, :cols], s if tiles else s.t()


def _values(q, s, tiles=False):
    """The values that codes and scales stand for."""
    rows, cols = q.shape
    s = s.repeat_interleave(BLOCK, 0)[:rows] if tiles else s.t()
    return q.float() * s.repeat_interleave(BLOCK, 1)[:, :cols]


def _plain_linear(s):
    y = _values(*_quantize(s["x"])) @ _values(s["w"], s["w_scale"], tiles=True).t()
    if s["bias"] is not None:
        y = y + s["bias"]
    return {"y": y.to(s["x"].dtype)}


def _plain_linear_grad(s):
    dy, x = s["dy"], s["x"]
    dx = _values(*_quantize(dy)) @ _values(s["wt"], s["wt_scale"], tiles=True).t()
    dw = _values(*_quantize(dy.t())) @ _values(*_quantize(x.t())).t()
    return {"dx": dx.to(x.dtype), "dw": dw}


def _scaled(z, temperature):
    """(z - max z) / T of every row, the maximum, and whether the row has any entry above -inf."""
    top = z.amax(1, keepdim=True)
    some = top > -math.inf
    top = torch.where(some, top, torch.zeros_like(top))
    return (z - top) / temperature, top, some[:, 0]


def _plain_logprobs(s):
    c, z = s["case"], s["logits"].float()
    d, top, some = _scaled(z, c["temperature"])
    e = torch.exp(d)
    total = e.sum(1)
    log_total = torch.log(total)
    inf = torch.full_like(total, -math.inf)
    entropy = torch.where(some, log_total - torch.where(e > 0, e * d, torch.zeros_like(e)).sum(1) / total, torch.zeros_like(total))
    lse = torch.where(some, top[:, 0] / c["temperature"] + log_total, inf)
    norm = torch.where(some, log_total, torch.zeros_like(total))[:, None]        # a row without entries: -inf - 0
    ids = s["tokens"].long()
    logprob = torch.where(ids >= 0, d.gather(1, ids.clamp(min=0)) - norm, torch.zeros((), device="cuda"))
    out = {"logprob": logprob, "entropy": entropy, "lse": lse}
    if c["top"]:
        # equal logits in the order of their index: the order of the bits, then of the index
        bits = (z + 0.0).view(torch.int32)
        bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        index = torch.arange(c["vocab"], device="cuda")
        best = torch.topk((bits << 32) + (0xFFFFFFFF - index), c["top"], 1).values
        at = 0xFFFFFFFF - (best & 0xFFFFFFFF)
        out.update(top_id=at.to(torch.int32), top_logit=z.gather(1, at), top_logprob=d.gather(1, at) - norm)
    return out


def _plain_distill(s):
    c, z, temp = s["case"], s["logits"].float(), s["case"]["temperature"]
    d, _, some = _scaled(z, temp)
    zero = torch.zeros((), device="cuda")
    live = some & (s["weight"] != 0)
    ids, there = s["top_id"].long().clamp(min=0), s["top_id"] >= 0
    t = torch.where(there, s["top_logit"] / temp, torch.full((), -math.inf, device="cuda"))
    e = torch.exp(d)
    # the sums inside and outside the list
    inside = torch.zeros_like(e, dtype=torch.bool).scatter_(1, torch.where(there, ids, ids[:, :1]), True)
    e_out = torch.where(inside, zero, e).sum(1)
    total = e_out + torch.where(inside, e, zero).sum(1)
    log_q = torch.where(there, d.gather(1, ids) - torch.log(total)[:, None], zero)
    if c["tail"]:
        p = torch.exp(t - s["teacher_lse"][:, None])
        rest = (1.0 - p.sum(1)).clamp(min=0.0)
        rest = torch.where(e_out > 0, rest, zero)
    else:
        p = torch.softmax(t, 1)
        rest = torch.zeros_like(total)
    q_out = e_out / total
    term = torch.where(p > 0, p * (torch.log(p) - log_q), zero).sum(1)
    term = term + torch.where(rest > 0, rest * (torch.log(rest) - torch.log(q_out)), zero)
    loss_rows = torch.where(live, term, zero)
    mass = p.sum(1) + rest
    factor = torch.where(live, s["weight"] / (temp * total), zero)
    outside = mass - torch.where(rest > 0, rest / q_out, zero)
    grad = torch.where(inside, mass[:, None], outside[:, None]) * e
    grad.scatter_add_(1, ids, torch.where(there, -p * total[:, None], zero))
    grad = torch.where(live[:, None], grad * factor[:, None], zero)
    return {"loss": (loss_rows * s["weight"]).sum().reshape(1), "loss_rows": loss_rows, "d_logits": grad.to(s["logits"].dtype)}


# ---- the library's calls -----------------------------------------------------------------------------------------
def _room(ae, s, nbytes):
    """The workspace, which a program keeps from call to call."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(max(16, nbytes()), dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _run_own(s):
    from paper_2602_17681_amd import binding as ae
    c = s["case"]
    dt = ae.DTYPES[c["dtype"]]
    if c["op"] == "linear":
        m, n, k = c["m"], c["n"], c["k"]
        ws = _room(ae, s, lambda: ae.model_fp8_linear_workspace(m, n, k))
        ae.model_fp8_linear(s["x"], s["w"], s["w_scale"], s["bias"], m, n, k, s["y"], ws)
        return {"y": s["y"]}
    if c["op"] == "linear_grad":
        m, n, k = c["m"], c["n"], c["k"]
        ws = _room(ae, s, lambda: max(ae.model_fp8_matmul_workspace(m, k, n), ae.model_fp8_matmul_workspace(n, k, m)))
        ae.model_fp8_quantize(s["dy"], m, n, "rows", s["dy_q"], s["dy_s"], s["dyt_q"], s["dyt_s"])
        ae.model_fp8_quantize(s["x"], m, k, "rows", None, None, s["xt_q"], s["xt_s"])
        ae.model_fp8_matmul(s["dy_q"], s["dy_s"], s["wt"], s["wt_scale"], "tiles", None, m, k, n, s["dx"], ws)
        ae.model_fp8_matmul(s["dyt_q"], s["dyt_s"], s["xt_q"], s["xt_s"], "rows", None, n, k, m, s["dw"], ws)
        return {"dx": s["dx"], "dw": s["dw"]}
    rows, vocab, top = c["rows"], c["vocab"], c["top"]
    if c["op"] == "logprobs":
        ws = _room(ae, s, lambda: ae.model_token_logprobs_workspace(rows, vocab, top, dt))
        ae.model_token_logprobs(s["logits"], rows, vocab, s["tokens"], top, s["logprob"], s["entropy"], s["lse"], s["top_id"],
                                s["top_logit"], s["top_logprob"], ws, temperature=c["temperature"])
        out = {n: s[n] for n in ("logprob", "entropy", "lse")}
        return dict(out, **{n: s[n] for n in ("top_id", "top_logit", "top_logprob")}) if top else out
    ws = _room(ae, s, lambda: ae.model_loss_distill_workspace(rows, vocab, dt))
    ae.model_loss_distill(s["logits"], rows, vocab, s["top_id"], s["top_logit"], s["loss_rows"], s["loss"], s["d_logits"], ws,
                          teacher_lse=s["teacher_lse"], weight=s["weight"], temperature=c["temperature"])
    return {n: s[n] for n in ("loss", "loss_rows", "d_logits")}


def run(state):
    if own:
        return _run_own(state)
    return {"linear": _plain_linear, "linear_grad": _plain_linear_grad, "logprobs": _plain_logprobs, "distill": _plain_distill}[state["case"]["op"]](state)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------
def _exact_codes(x, tiles=False):
    """The values that x has after quantisation, block by block; scale and scaled element are binary32 numbers by definition."""
    x = x.double()
    out = torch.empty_like(x)
    for c in range(0, x.shape[1], BLOCK):
        b = x[:, c:c + BLOCK]
        big = b.abs().amax(1, keepdim=True)
        if tiles:
            big = torch.cat([r.amax().expand(r.shape[0], 1) for r in big.split(BLOCK)])
        s = (big / 448).float().double().clamp(min=2.0 ** -126)
        y = (b * (1 / s).float().double()).float().double().clamp(-448, 448)
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)        # three fraction bits, subnormals below 2^-6
        out[:, c:c + BLOCK] = torch.round(y / step) * step * s
    return out


def _exact_values(q, s):
    """Codes with a scale for each 128 x 128 tile, as numbers."""
    r = torch.arange(q.shape[0], device="cuda") // BLOCK
    c = torch.arange(q.shape[1], device="cuda") // BLOCK
    return q.float().double() * s.double()[r][:, c]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        y = torch.matmul(_exact_codes(s["x"]), _exact_values(s["w"], s["w_scale"]).t())
        return {"y": y if s["bias"] is None else y + s["bias"].double()}
    if case["op"] == "linear_grad":
        dyt, xt = _exact_codes(s["dy"].t().contiguous()), _exact_codes(s["x"].t().contiguous())
        return {"dx": torch.matmul(_exact_codes(s["dy"]), _exact_values(s["wt"], s["wt_scale"]).t()), "dw": torch.matmul(dyt, xt.t())}
    temp, n = case["temperature"], case["rows"]
    z = s["logits"].double() / temp
    lse = torch.logsumexp(z, 1)
    empty = torch.isinf(lse)
    if case["op"] == "logprobs":
        logp = torch.where(empty[:, None], z, z - lse[:, None])
        tokens = s["tokens"].long()
        res = {"lse": lse, "entropy": -torch.nan_to_num(torch.exp(logp) * logp, nan=0.0).sum(1),
               "logprob": torch.where(tokens < 0, 0.0, logp.gather(1, tokens.clamp(min=0)))}
        if case["top"]:
            # the order of equal logits: a stable sort by descending value
            order = torch.cat([torch.sort(r, dim=1, descending=True, stable=True).indices[:, :case["top"]] for r in z.split(max(1, 2 ** 27 // z.shape[1]))])
            res.update(top_id=order.to(torch.int32), top_logit=s["logits"].gather(1, order).double(), top_logprob=logp.gather(1, order))
        return res
    loss_rows = torch.zeros(n, dtype=torch.float64, device="cuda")
    grad = torch.zeros_like(z)
    live = ~empty & (s["weight"] != 0)
    w = s["weight"].double()
    at = s["top_id"].long()
    listed_ = at >= 0
    at = torch.where(listed_, at, at[:, :1])                    # an entry that is there, in the place of one that is not
    t = s["top_logit"].double() / temp
    t = torch.where(listed_, t, -math.inf)
    logp = t - (s["teacher_lse"].double()[:, None] if case["tail"] else torch.logsumexp(t, 1, keepdim=True))
    p = torch.exp(logp)
    others = z.scatter(1, at, -math.inf)
    log_rest = torch.logsumexp(others, 1) - lse                 # of the student's mass outside the list
    p_rest = (1 - p.sum(1)).clamp(min=0) if case["tail"] else torch.zeros_like(lse)
    p_rest = torch.where(torch.isinf(log_rest), 0.0, p_rest)
    logq = z.gather(1, at) - lse[:, None]
    terms = torch.where(p > 0, p * (logp - logq), 0.0).sum(1) + torch.where(p_rest > 0, p_rest * (torch.log(p_rest) - log_rest), 0.0)
    loss_rows[live] = terms[live]
    mass = p.sum(1) + p_rest
    tail = torch.where(p_rest > 0, p_rest * torch.exp(-log_rest), 0.0)
    grad[live] = torch.exp(others[live] - lse[live, None]) * (mass - tail)[live, None]
    pulled = torch.exp(logq) * mass[:, None] - p
    grad.scatter_(1, at, torch.where(live[:, None], pulled[:, :1], 0.0).expand_as(at).contiguous())     # the entry that stands in for missing ones
    rows = torch.arange(n, device="cuda")[:, None].expand_as(at)
    ok = listed_ & live[:, None]
    grad[rows[ok], at[ok]] = pulled[ok]
    grad *= (w / temp)[:, None]
    return {"loss": (loss_rows * w).sum().reshape(1), "loss_rows": loss_rows, "d_logits": grad}
