"""Adjusted logits against the oracle in 64 bits.  Penalty, count times frequency, two differences and the bias's sum are each rounded to binary32 once: 5 U of
the sum over magnitudes; a result in bfloat16 is off by 2^-8 of itself more.  Tokens that nothing names keep their bits."""
import numpy as np
import pytest

from oracle import token_oracle as to
from token_util import U, Room, dev, host, ints, near, replayed

pytestmark = pytest.mark.gpu


def lists(rng, rows, vocab, nh, nb, mask):
    s = dict(history=None, n_prompt=None, bias_id=None, bias=None, allowed=None)
    s.update({k: rng.uniform(lo, hi, rows).astype(np.float32) for k, lo, hi in (("repetition", 0.8, 1.6), ("presence", -0.5, 1.0), ("frequency", -0.2, 0.7))})
    if nh:
        s["history"] = np.where(rng.random((rows, nh)) < 0.5, rng.integers(0, min(vocab, 7), (rows, nh)), rng.integers(-2, vocab + 2, (rows, nh)))
        s["n_prompt"] = rng.integers(-1, nh + 2, rows)
        s["history"][0, 0] = -2 ** 31
    if nb:
        s["bias_id"] = rng.integers(-1, vocab + 1, (rows, nb))                 # also tokens that are listed twice
        s["bias"] = (4 * rng.standard_normal((rows, nb))).astype(np.float32)
    if mask:
        words = -(-vocab // 32)
        s["allowed"] = rng.integers(0, 2 ** 32, (rows, words), dtype=np.uint64) | rng.integers(0, 2 ** 32, (rows, words), dtype=np.uint64)
        s["allowed"][:, rng.integers(0, words)] = 0
        if rows > 1:
            s["allowed"][rows // 2] = 0                                        # a row that allows nothing
            s["allowed"][0] = 2 ** 32 - 1
    return s


def device(s):
    f = dict(history=ints, n_prompt=ints, bias_id=ints, allowed=lambda a: ints(a.astype(np.uint32).view(np.int32)))
    return {k: None if v is None else f.get(k, dev)(v) for k, v in s.items()}


def check(z, s, got, dtype):
    want, mag = to.logits_adjust(z, **s)
    with np.errstate(all="ignore"):
        near(got, want, np.where(np.isfinite(mag), 5 * U * mag, 0) + (2.0 ** -8 if dtype == "bf16" else 0) * np.abs(np.where(np.isfinite(want), want, 0)))
    same = (want == z) | np.isneginf(want)
    assert np.array_equal(got[same], want[same])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,nh,nb,mask", [(1, 1, 1, 1, True), (3, 7, 20, 3, True), (1, 33, 0, 0, True), (2, 100, 0, 0, False), (5, 1000, 50, 0, False), (4, 2048, 0, 9, False),
                                                   (4, 2049, 300, 9, True), (3, 5003, 0, 0, True), (3, 8192, 1, 300, False), (2, 50021, 777, 5, True), (1, 131072, 5000, 2047, True),
                                                   (400, 4099, 60, 4, True), (70, 30011, 200, 40, False), (1100, 900, 33, 2, True), (1, 1 << 20, 999, 20, True)])
def test_adjust(rows, vocab, nh, nb, mask, dtype):
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(rows + vocab)
    x = 3 * rng.standard_normal((rows, vocab))
    x[rng.random((rows, vocab)) < 0.05] = -np.inf
    x[rng.random((rows, vocab)) < 0.02] = 0.0
    zm, om = Room(rows, vocab, dtype, 3, 1, dev(x.astype(np.float32))), Room(rows, vocab, dtype, 1, 5)
    z = host(zm.m)
    s = lists(rng, rows, vocab, nh, nb, mask)
    d = device(s)
    ae.model_logits_adjust(zm.m, rows, vocab, om.m, **d)
    check(z, s, host(om.m), dtype)
    assert om.whole() and np.array_equal(host(zm.m), z)
    ae.model_logits_adjust(zm.m, rows, vocab, zm.m, **d)          # in place
    assert torch.equal(zm.m, om.m) and zm.whole()


@pytest.mark.parametrize("left_out", ["n_prompt", "repetition", "presence", "frequency", "all three"])
def test_arguments_that_may_be_missing(left_out):
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(2)
    z = host(dev(3 * rng.standard_normal((6, 3001)).astype(np.float32)))
    s = lists(rng, 6, 3001, 90, 3, False)
    for k in ("repetition", "presence", "frequency") if left_out == "all three" else (left_out,):
        s[k] = None
    out = torch.empty((6, 3001), device="cuda")
    ae.model_logits_adjust(dev(z), 6, 3001, out, **device(s))
    check(z, s, host(out), "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_unusual_logits(dtype):
    """NaN, infinities and the type's lowest number under every rule; what is forbidden is -infinity whatever it was."""
    import torch
    from paper_2602_17681_amd import binding as ae
    vocab = 70
    low = float(torch.finfo(torch.float32 if dtype == "f32" else torch.bfloat16).min)
    z = np.zeros((1, vocab))
    z[0, ::5], z[0, 1::5], z[0, 2::5], z[0, 3::5], z[0, 4::5] = np.nan, np.inf, -np.inf, low, -low
    t = dev(z.astype(np.float32), dtype)
    word = [0xFFFF0000, 0xFFFFFFFF, 0xFFFFFFFF]
    s = dict(history=np.arange(40, 60)[None], n_prompt=np.array([10]), repetition=np.array([0.5], np.float32), presence=np.array([1.0], np.float32),
             frequency=np.array([0.5], np.float32), bias_id=np.arange(50, 70)[None], bias=np.ones((1, 20), np.float32), allowed=np.array([word], np.uint64))
    out = torch.empty_like(t)
    ae.model_logits_adjust(t, 1, vocab, out, **device(s))
    want, _ = to.logits_adjust(host(t), **s)
    want = np.where(want > 3.4029e38, np.inf, np.where(want < -3.4029e38, -np.inf, want))       # beyond the types' range
    got = host(out)
    assert np.all(np.isneginf(got[0, :16])) and np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
    fine = np.isfinite(want)
    near(got[fine], want[fine], 2.0 ** (-8 if dtype == "bf16" else -22) * np.abs(want[fine]))


def test_long_history_and_counts():
    """One token a hundred thousand times: counts are whole numbers, whatever the order they are taken in."""
    import torch
    from paper_2602_17681_amd import binding as ae
    n = (1 << 20) - 1
    hist = np.full((1, n), 5)
    hist[0, 1000:2000] = 9
    z = np.ones((1, 50), np.float32)
    s = dict(history=hist, n_prompt=np.array([500]), repetition=np.array([2.0], np.float32), presence=np.array([0.0], np.float32), frequency=np.array([2.0 ** -10], np.float32))
    out = torch.empty((1, 50), device="cuda")
    ae.model_logits_adjust(dev(z), 1, 50, out, **{k: (ints if v.dtype != np.float32 else dev)(v) for k, v in s.items()})
    want = np.ones((1, 50))
    want[0, 5], want[0, 9] = 0.5 - (n - 1500) / 1024, 0.5 - 1000 / 1024
    near(host(out), want, 4 * U * np.abs(want) + 2 * U)


def test_rows_beyond_one_slice_border_and_log_probabilities():
    """The adjusted rows as model_token_logprobs takes them: forbidden tokens have probability 0, an empty row has no outcome."""
    import torch
    from oracle import vocab_oracle as vo
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(6)
    rows, vocab, k = 9, 9001, 12
    t = dev(3 * rng.standard_normal((rows, vocab)).astype(np.float32), "bf16")
    s = lists(rng, rows, vocab, 300, 8, True)
    ae.model_logits_adjust(t, rows, vocab, t, **device(s))
    lse, ids, top = torch.empty(rows, device="cuda"), torch.empty((rows, k), dtype=torch.int32, device="cuda"), torch.empty((rows, k), device="cuda")
    ws = torch.empty(max(16, ae.model_token_logprobs_workspace(rows, vocab, k, ae.AE_BF16)), dtype=torch.uint8, device="cuda")
    ae.model_token_logprobs(t, rows, vocab, None, k, None, None, lse, ids, None, top, ws)
    want = vo.token_logprobs(host(t), None, k, 1.0)
    assert np.array_equal(ids.cpu().numpy(), want["top_id"]) and np.isneginf(host(lse)[rows // 2])
    near(host(lse), want["lse"], 1e-4)
    ok = np.array([[int(s["allowed"][r][j // 32]) >> (j % 32) & 1 for j in ids[r].tolist()] for r in range(rows)])
    assert np.all(ok[np.isfinite(host(top))] == 1)


def test_no_rows():
    import torch
    from paper_2602_17681_amd import binding as ae
    z = torch.empty((0, 50), device="cuda")
    ae.model_logits_adjust(z, 0, 50, z)


def test_streams_and_graphs():
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(12)
    rows, vocab = 7, 20001
    sets = [(3 * rng.standard_normal((rows, vocab)).astype(np.float32), device(lists(rng, rows, vocab, 128, 6, True))) for _ in range(3)]
    z, out = dev(sets[0][0]), torch.empty((rows, vocab), device="cuda")
    d = {k: v.clone() for k, v in sets[0][1].items()}

    def change(i):
        z.copy_(dev(sets[i][0]))
        for k in d:
            d[k].copy_(sets[i][1][k])
    for i, got in enumerate(replayed(lambda: ae.model_logits_adjust(z, rows, vocab, out, **d), [out], change)):
        change(i)
        ae.model_logits_adjust(z, rows, vocab, out, **d)
        torch.cuda.synchronize()
        assert torch.equal(got[0], out)
