"""The operators between tokens and an 8-bit output layer, and between its gradient and the optimiser, as cases of known size.

  norm        h = x + residual, y = h / sqrt(mean h^2 + eps) * weight, y as E4M3 codes with a scale for each block of 128
              elements of a row (what an 8-bit product takes), in the inputs' type, or both
  norm_grad   the gradients of h (with what arrives on the residual path added) and of the weight
  embed       rows of a table picked by tokens, times a number
  embed_grad  the gradient of that table: the rows of equal tokens added up
  clip        the norm of all gradients together, and the gradients scaled down to a largest norm
  logits      penalties for tokens that occurred, biases of given tokens, and a mask of allowed tokens, on rows of logits

A case is a dict of plain values; `prepare` makes what a program holds before the call, `run` is one pass, in elementary
torch operations in binary32 (`own` false) or through the library's entry points (`own` true).
"""
import math

import torch

own = False

BLOCK = 128                      # elements that share a scale
E4M3_MAX = 448.0                 # largest magnitude of the codes
SCALE_MIN = 2.0 ** -126          # smallest normal binary32: the scale of a block of zeros
EPS = 1e-6
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- the cases ---------------------------------------------------------------------------------------------------
def listed():
    return [
        # one token of one sequence in decoding: the norm before an 8-bit projection, with the residual's addition
        dict(name="norm_token", op="norm", rows=1, d=4096, dtype="bf16", residual=True, codes=True, y=False),
        # the same before the projections of a calibration batch of 16 sequences of 1 024 tokens
        dict(name="norm_prompt", op="norm", rows=16384, d=4096, dtype="bf16", residual=True, codes=True, y=False),
        # the backward pass of a training step on 4 sequences of 1 024 tokens, with the residual path's gradient
        dict(name="norm_train", op="norm_grad", rows=4096, d=4096, dtype="bf16", residual=True),
        # a small model in binary32: an odd number of tokens, rows on no 16-byte border, no residual path
        dict(name="norm_train_ragged", op="norm_grad", rows=1001, d=1003, dtype="f32", residual=False),
        # a decoding step of 16 sequences, embeddings scaled by sqrt(d)
        dict(name="embed_decode", op="embed", tokens=16, vocab=32768, d=4096, dtype="bf16", padded=False),
        # a padded calibration batch of 16 sequences of 1 024 tokens from a large table
        dict(name="embed_prompt", op="embed", tokens=16384, vocab=131072, d=4096, dtype="bf16", padded=True),
        # the embedding's part of a training step on 16 sequences of 1 024 tokens
        dict(name="embed_train", op="embed_grad", tokens=16384, vocab=32768, d=4096, dtype="bf16", padded=False),
        # a small model in binary32 with padded sequences: odd sizes throughout
        dict(name="embed_train_ragged", op="embed_grad", tokens=4097, vocab=8009, d=515, dtype="f32", padded=True),
        # the LU parameters of 32 transformations of the head dimension 128: many small tensors
        dict(name="clip_heads", op="clip", layers=32, d=128, dtype="f32", max_norm=1.0),
        # the LU parameters of four transformations of width 4 096
        dict(name="clip_layers", op="clip", layers=4, d=4096, dtype="f32", max_norm=1.0),
        # a decoding step of four sequences with a grammar: 2 048 tokens each so far, 16 biases
        dict(name="logits_decode", op="logits", rows=4, vocab=131072, dtype="bf16", history=2048, biases=16, masked=True),
        # a large decoding batch of binary32 logits over an odd vocabulary, histories of different lengths, one row allows nothing
        dict(name="logits_batch", op="logits", rows=333, vocab=50021, dtype="f32", history=777, biases=5, masked=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "embed", "embed_grad", "clip", "logits"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    d = _log_uniform(rng, 64, 16384)
    if rng.random() < 0.5:                           # widths of whole blocks, as most layers have them
        d = max(BLOCK, d // BLOCK * BLOCK)
    if op in ("norm", "norm_grad"):
        rows = _log_uniform(rng, 1 if op == "norm" else 16, 16384)
        rows = max(1, min(rows, (16384 if op == "norm" else 4096) * 4096 // (d * (1 if dtype == "bf16" else 2))))
        c = dict(op=op, rows=rows, d=d, dtype=dtype, residual=rng.random() < 0.7)
        return c if op == "norm_grad" else dict(c, **rng.choice([dict(codes=True, y=False), dict(codes=True, y=True), dict(codes=False, y=True)]))
    if op in ("embed", "embed_grad"):
        tokens, vocab = _log_uniform(rng, 1 if op == "embed" else 64, 32768), _log_uniform(rng, 1000, 131072)
        while tokens * d * (1 if dtype == "bf16" else 2) > 16384 * 4096:
            tokens = max(1, tokens // 2)
        while vocab * d > (131072 if op == "embed" else 24576) * 4096:
            vocab = vocab // 2
        return dict(op=op, tokens=tokens, vocab=vocab, d=d, dtype=dtype, padded=rng.random() < 0.5)
    if op == "clip":
        d = _log_uniform(rng, 32, 4096)
        layers = min(_log_uniform(rng, 1, 64), max(1, 4 * 4096 * 4096 // (d * d)))
        return dict(op=op, layers=layers, d=d, dtype=dtype, max_norm=rng.choice([0.1, 1.0, 1.0, 1e6]))
    vocab = _log_uniform(rng, 1000, 200000)
    if rng.random() < 0.5:
        vocab = vocab // 64 * 64
    rows = min(_log_uniform(rng, 1, 512), 333 * 50021 // vocab)
    return dict(op=op, rows=max(1, rows), vocab=vocab, dtype=dtype, history=rng.choice([0, _log_uniform(rng, 1, 8192), _log_uniform(rng, 1, 8192)]),
                biases=rng.choice([0, _log_uniform(rng, 1, 300)]), masked=rng.random() < 0.6)


def _shapes(case):
    """The parameters of one transformation: two triangular factors, its scales and its shift."""
    d = case["d"]
    return [(d, d), (d, d)], [(d,), (d,)]


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    op = case["op"]
    if op == "norm":
        n, rows = case["rows"] * case["d"], case["rows"]
        out = (e * n if case["residual"] else 0) + (e * n if case["y"] else 0) + (n + 4 * rows * -(-case["d"] // BLOCK) if case["codes"] else 0)
        # each element: the sum, its square and the sum of those, two products; its magnitude and the product with the scale
        return {"bytes": n * e * (2 if case["residual"] else 1) + 4 * case["d"] + out, "flops": 7.0 * n}
    if op == "norm_grad":
        n = case["rows"] * case["d"]
        return {"bytes": n * e * (4 if case["residual"] else 3) + 8 * case["d"], "flops": 12.0 * n}
    if op == "embed":
        return {"bytes": case["tokens"] * (4 + 2 * e * case["d"]), "flops": 1.0 * case["tokens"] * case["d"]}
    if op == "embed_grad":
        return {"bytes": case["tokens"] * (4 + e * case["d"]) + 4 * case["vocab"] * case["d"], "flops": 1.0 * (case["tokens"] + case["vocab"]) * case["d"]}
    if op == "clip":
        big, small = (case["layers"] * sum(math.prod(s) for s in g) for g in _shapes(case))
        return {"bytes": 2 * (e * big + 4 * small) + 4, "flops": 3.0 * (big + small)}
    n = case["rows"] * case["vocab"]
    return {"bytes": 2 * e * n + (n // 8 if case["masked"] else 0) + case["rows"] * (4 * case["history"] + 8 * case["biases"] + 16), "flops": 4.0 * n}


# ---- the inputs --------------------------------------------------------------------------------------------------
def _codes(rows, cols):
    """Room for rows x cols codes whose rows begin on 16-byte borders."""
    return torch.empty((rows, -(-cols // 16) * 16), dtype=torch.float8_e4m3fn, device="cuda")[:, :cols]


def _activations(gen, rows, cols, dtype):
    """Roughly Gaussian, with a few features that are many times larger than the rest, as hidden states have."""
    x = torch.randn((rows, cols), generator=gen, device="cuda")
    gain = torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.01, 20.0, 1.0)
    return x.mul_(gain).to(dtype)


def _text(gen, n, vocab):
    """Tokens whose frequency falls with their rank, as in text: the most frequent are one in ten to twenty; ranks lie all over the vocabulary."""
    rank = torch.exp(torch.rand(n, generator=gen, device="cuda", dtype=torch.float64) * math.log(vocab)).long() - 1
    return ((rank.clamp(0, vocab - 1) * 7919 + 13) % vocab).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, op = DTYPE[case["dtype"]], case["op"]
    s = dict(case=case)
    if op in ("norm", "norm_grad"):
        rows, d = case["rows"], case["d"]
        s["weight"] = 1.0 + 0.2 * torch.randn(d, generator=gen, device="cuda")
        x = _activations(gen, rows, d, dt)
        if op == "norm":
            s["x"] = x
            s["residual"] = _activations(gen, rows, d, dt) if case["residual"] else None
            s["h"] = torch.empty_like(x) if case["residual"] else None
            s["y"] = torch.empty_like(x) if case["y"] else None
            s["q"] = _codes(rows, d) if case["codes"] else None
            s["scale"] = torch.empty((-(-d // BLOCK), rows), device="cuda") if case["codes"] else None
        else:
            s["h"] = x
            s["dy"] = torch.randn((rows, d), generator=gen, device="cuda").mul_(1e-3).to(dt)
            s["d_h"] = torch.randn((rows, d), generator=gen, device="cuda").mul_(1e-3).to(dt) if case["residual"] else None
            s["dx"], s["d_weight"] = torch.empty_like(x), torch.empty(d, device="cuda")
    elif op in ("embed", "embed_grad"):
        n, vocab, d = case["tokens"], case["vocab"], case["d"]
        s["scale"] = math.sqrt(d)
        s["ids"] = _text(gen, n, vocab)
        if case["padded"]:      # sequences of different lengths, padded with -1
            length = -(-n // 16)
            ends = (torch.rand(16, generator=gen, device="cuda") * 0.7 + 0.3) * length
            at = torch.arange(n, device="cuda")
            s["ids"].masked_fill_(at % length >= ends[at // length], -1)
        if op == "embed":
            s["table"] = torch.randn((vocab, d), generator=gen, device="cuda").mul_(d ** -0.5).to(dt)
            s["out"] = torch.empty((n, d), dtype=dt, device="cuda")
        else:
            s["d_out"] = torch.randn((n, d), generator=gen, device="cuda").mul_(1e-3).to(dt)
            s["d_table"] = torch.empty((vocab, d), device="cuda")
    elif op == "clip":
        # two buffers, of the matrices' and of the vectors' gradients, which the tensors are parts of
        for name, group, t in zip(("matrices", "vectors"), _shapes(case), (dt, torch.float32)):
            size = [math.prod(g) for g in group] * case["layers"]
            flat = torch.randn(sum(size), generator=gen, device="cuda").mul_(0.05).to(t)
            s[name], s[name + "_out"] = flat, torch.empty_like(flat)
            s[name + "_parts"] = list(flat.split(size))
            s[name + "_out_parts"] = list(s[name + "_out"].split(size))
        s["norm"] = torch.empty(1, device="cuda")
    else:
        rows, vocab, n, nb = case["rows"], case["vocab"], case["history"], case["biases"]
        z = torch.randn((rows, vocab), generator=gen, device="cuda").mul_(2.5)
        z.masked_fill_(torch.rand((rows, vocab), generator=gen, device="cuda") < 0.01, -math.inf)      # tokens that the model never gives
        s["logits"] = z.to(dt)
        s["out"] = torch.empty_like(s["logits"])
        f = lambda lo, hi: torch.rand(rows, generator=gen, device="cuda") * (hi - lo) + lo      # noqa: E731
        s["history"] = s["n_prompt"] = s["bias_id"] = s["bias"] = s["allowed"] = None
        s["repetition"], s["presence"], s["frequency"] = f(1.0, 1.5), f(0.0, 1.0), f(0.0, 0.5)
        if n:           # prompt, then answer, then nothing
            length = ((torch.rand(rows, generator=gen, device="cuda") * 0.5 + 0.5) * n).long().clamp(min=1)
            s["history"] = _text(gen, rows * n, vocab).view(rows, n).masked_fill_(torch.arange(n, device="cuda") >= length[:, None], -1)
            s["n_prompt"] = (length * torch.rand(rows, generator=gen, device="cuda")).to(torch.int32)
        if nb:          # distinct tokens in no order; some lists are shorter
            share = vocab // nb
            ids = (torch.rand((rows, nb), generator=gen, device="cuda") * share).long().clamp_(max=share - 1) + torch.arange(nb, device="cuda") * share
            ids = ids.gather(1, torch.rand((rows, nb), generator=gen, device="cuda").argsort(1))
            s["bias_id"] = ids.masked_fill_(torch.rand((rows, nb), generator=gen, device="cuda") < 0.1, -1).to(torch.int32)
            s["bias"] = torch.randn((rows, nb), generator=gen, device="cuda") * 5
        if case["masked"]:      # a third of each row's words of 32 tokens is forbidden as a whole, and some of the other tokens
            words = -(-vocab // 32)
            bits = torch.randint(-2 ** 31, 2 ** 31, (rows, words), generator=gen, device="cuda") | torch.randint(-2 ** 31, 2 ** 31, (rows, words), generator=gen, device="cuda")
            bits.masked_fill_(torch.rand((rows, words), generator=gen, device="cuda") < 0.33, 0)
            if rows > 2:
                bits[rows // 2] = 0
            s["allowed"] = bits.to(torch.int32)
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------
def _quantize(x):
    """E4M3 codes of x and their scales, [block of columns][row]."""
    rows, cols = x.shape
    cb = -(-cols // BLOCK)
    x = torch.nn.functional.pad(x, (0, cb * BLOCK - cols)).view(rows, cb, BLOCK)
    amax = x.abs().amax(2)
    s = (amax / torch.full_like(amax, E4M3_MAX)).clamp(min=SCALE_MIN)      # quotients of tensors: correctly rounded
    inv = torch.ones_like(s) / s
    q = (x * inv[:, :, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return q.view(rows, cb * BLOCK)[:, :cols], s.t().contiguous()


def _plain_norm(s):
    c, x = s["case"], s["x"].float()
    h = x + s["residual"].float() if c["residual"] else x
    rstd = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    y = h * rstd * s["weight"]
    out = {"h": h.to(s["x"].dtype)} if c["residual"] else {}
    if c["y"]:
        out["y"] = y.to(s["x"].dtype)
    if c["codes"]:
        out["q"], out["scale"] = _quantize(y)
    return out


def _plain_norm_grad(s):
    h, dy = s["h"].float(), s["dy"].float()
    rstd = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    unit = h * rstd
    g = dy * s["weight"]
    dx = (g - unit * (g * unit).mean(1, keepdim=True)) * rstd
    if s["d_h"] is not None:
        dx = dx + s["d_h"].float()
    return {"dx": dx.to(s["h"].dtype), "d_weight": (dy * unit).sum(0)}


def _plain_embed(s):
    ids = s["ids"].long()
    rows = s["table"][ids.clamp(min=0)].float() * s["scale"]
    return {"out": torch.where((ids >= 0)[:, None], rows, torch.zeros((), device="cuda")).to(s["table"].dtype)}


def _plain_embed_grad(s):
    ids = s["ids"].long()
    rows = torch.where((ids >= 0)[:, None], s["d_out"].float() * s["scale"], torch.zeros((), device="cuda"))
    return {"d_table": torch.zeros_like(s["d_table"]).index_add_(0, ids.clamp(min=0), rows)}


def _plain_clip(s):
    a, b = s["matrices"].float(), s["vectors"]
    norm = torch.sqrt((a * a).sum(dtype=torch.float64) + (b * b).sum(dtype=torch.float64)).float()
    factor = (s["case"]["max_norm"] / norm).clamp(max=1.0)
    return {"norm": norm.reshape(1), "matrices": (a * factor).to(s["matrices"].dtype), "vectors": b * factor}


def _plain_logits(s):
    z = s["logits"].float()
    rows, vocab = z.shape
    col = lambda t: t[:, None]      # noqa: E731
    if s["history"] is not None:
        ids = s["history"].long()
        there = ids >= 0
        answered = there & (torch.arange(ids.shape[1], device="cuda") >= col(s["n_prompt"]))
        count = torch.zeros_like(z).scatter_add_(1, ids.clamp(min=0), answered.float())
        seen = torch.zeros_like(z).scatter_add_(1, ids.clamp(min=0), there.float()) > 0
        z = torch.where(seen, torch.where(z > 0, z / col(s["repetition"]), z * col(s["repetition"])), z)
        z = z - col(s["frequency"]) * count
        z = torch.where(count > 0, z - col(s["presence"]), z)
    if s["bias_id"] is not None:
        ids = s["bias_id"].long()
        z = z + torch.zeros_like(z).scatter_add_(1, ids.clamp(min=0), torch.where(ids >= 0, s["bias"], torch.zeros((), device="cuda")))
    if s["allowed"] is not None:
        at = torch.arange(vocab, device="cuda")
        ok = (s["allowed"][:, at // 32] >> (at % 32).to(torch.int32)) & 1
        z = torch.where(ok != 0, z, torch.full((), -math.inf, device="cuda"))
    return {"out": z.to(s["logits"].dtype)}


# ---- the library's calls -----------------------------------------------------------------------------------------
def _room(s, nbytes):
    """The workspace, which a program keeps from call to call."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(max(16, nbytes()), dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _run_own(s):
    from paper_2602_17681_amd import binding as ae
    c = s["case"]
    op = c["op"]
    if op == "norm":
        ae.model_rms_norm(s["x"], c["rows"], c["d"], s["weight"], EPS, s["h"], s["y"], s["q"], s["scale"], residual=s["residual"])
        return {n: s[n] for n in ("h", "y", "q", "scale") if s[n] is not None}
    if op == "norm_grad":
        ws = _room(s, lambda: ae.model_rms_norm_backward_workspace(c["rows"], c["d"], ae.DTYPES[c["dtype"]]))
        ae.model_rms_norm_backward(s["dy"], s["h"], c["rows"], c["d"], s["weight"], EPS, s["dx"], s["d_weight"], ws, d_h=s["d_h"])
        return {n: s[n] for n in ("dx", "d_weight")}
    if op == "embed":
        ae.model_embedding(s["table"], c["vocab"], c["d"], s["ids"], c["tokens"], s["out"], scale=s["scale"])
        return {"out": s["out"]}
    if op == "embed_grad":
        ws = _room(s, lambda: ae.model_embedding_backward_workspace(c["tokens"], c["vocab"], c["d"], ae.DTYPES[c["dtype"]]))
        ae.model_embedding_backward(s["d_out"], s["ids"], c["tokens"], c["vocab"], c["d"], s["d_table"], ws, scale=s["scale"])
        return {"d_table": s["d_table"]}
    if op == "clip":
        if "grads" not in s:        # the lists of a program's gradients and of where the clipped ones go: the same for every step
            s["grads"] = ae.GradList(s["matrices_parts"] + s["vectors_parts"], s["matrices_out_parts"] + s["vectors_out_parts"])
        ae.model_grad_clip(s["grads"], c["max_norm"], s["norm"], _room(s, lambda: ae.model_grad_clip_workspace(s["grads"])))
        return {"norm": s["norm"], "matrices": s["matrices_out"], "vectors": s["vectors_out"]}
    ae.model_logits_adjust(s["logits"], c["rows"], c["vocab"], s["out"], history=s["history"], n_prompt=s["n_prompt"], repetition=s["repetition"],
                           presence=s["presence"], frequency=s["frequency"], bias_id=s["bias_id"], bias=s["bias"], allowed=s["allowed"])
    return {"out": s["out"]}


def run(state):
    if own:
        return _run_own(state)
    return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "embed": _plain_embed, "embed_grad": _plain_embed_grad, "clip": _plain_clip,
            "logits": _plain_logits}[state["case"]["op"]](state)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        h = s["x"].double()
        out = {}
        if case["residual"]:
            h += s["residual"].double()
            out["h"] = h
        y = h / (torch.linalg.vector_norm(h, dim=1, keepdim=True) ** 2 / case["d"] + EPS) ** 0.5 * s["weight"].double()
        if case["y"]:
            out["y"] = y
        if case["codes"]:       # a scale and a scaled element are binary32 numbers by definition; three fraction bits, subnormals below 2^-6
            code, scale = torch.empty_like(y), []
            for c in range(0, case["d"], BLOCK):
                b = y[:, c:c + BLOCK]
                t = (b.abs().amax(1) / 448).float().double().clamp(min=2.0 ** -126)
                u = (b * (1 / t).float().double()[:, None]).float().double().clamp(-448, 448)
                step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) - 3)
                code[:, c:c + BLOCK] = torch.round(u / step) * step
                scale.append(t)
            out["q"], out["scale"] = code, torch.stack(scale)
        return out
    if op == "norm_grad":
        h, dy, w = s["h"].double(), s["dy"].double(), s["weight"].double()
        var = h.pow(2).sum(1) / case["d"] + EPS
        dot = (dy * w * h).sum(1)
        dx = dy * w * var.rsqrt()[:, None] - h * (dot / (case["d"] * var * var.sqrt()))[:, None]
        return {"dx": dx if s["d_h"] is None else dx + s["d_h"].double(), "d_weight": torch.mv((dy * h).t().contiguous(), var.rsqrt())}
    if op == "embed":
        out = torch.zeros((case["tokens"], case["d"]), dtype=torch.float64, device="cuda")
        some = s["ids"] >= 0
        out[some] = torch.index_select(s["table"], 0, s["ids"][some]).double() * s["scale"]
        return {"out": out}
    if op == "embed_grad":
        some = s["ids"] >= 0
        out = torch.zeros((case["vocab"], case["d"]), dtype=torch.float64, device="cuda")
        out.index_put_((s["ids"][some].long(),), s["d_out"][some].double(), accumulate=True)
        return {"d_table": out.mul_(s["scale"])}
    if op == "clip":
        parts = [p.double() for p in s["matrices_parts"] + s["vectors_parts"]]
        norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(p) for p in parts]))
        k = 1.0 if float(norm) <= case["max_norm"] else case["max_norm"] / float(norm)
        n = len(s["matrices_parts"])
        return {"norm": norm.reshape(1), "matrices": torch.cat(parts[:n]).mul_(k), "vectors": torch.cat(parts[n:]).mul_(k)}
    z = s["logits"].double()
    row = torch.arange(case["rows"], device="cuda")[:, None]
    if case["history"]:
        ids = s["history"].long()
        place = torch.arange(case["history"], device="cuda")[None, :]
        prompt = place < s["n_prompt"][:, None]
        at = (row * case["vocab"] + ids)
        seen = torch.bincount(at[ids >= 0], minlength=z.numel()).view_as(z) > 0
        count = torch.bincount(at[(ids >= 0) & ~prompt], minlength=z.numel()).view_as(z).double()
        r = s["repetition"].double()[:, None].expand_as(z)
        z[seen] = torch.where(z[seen] > 0, z[seen] / r[seen], z[seen] * r[seen])
        z = z - count * s["frequency"].double()[:, None] - count.clamp(max=1) * s["presence"].double()[:, None]
    if case["biases"]:
        real = s["bias_id"] >= 0
        z[row.expand_as(real)[real], s["bias_id"][real].long()] += s["bias"].double()[real]
    if case["masked"]:
        bits = (s["allowed"].long()[:, :, None] >> torch.arange(32, device="cuda")) & 1
        z[bits.flatten(1)[:, :case["vocab"]] == 0] = -math.inf
    return {"out": z}
