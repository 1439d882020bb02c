"""Embeddings bit for bit, and their gradient against the oracle in 64 bits: a sum of n terms is off by n U of the sum over magnitudes, the product with the
scale by one U more and what is added to an existing gradient by another."""
import numpy as np
import pytest

from oracle import token_oracle as to
from token_util import U, Room, dev, host, ints, near, replayed, space, td

pytestmark = pytest.mark.gpu


def tokens(rng, n, vocab, kind):
    if kind == "text":
        ids = np.minimum(np.exp(rng.random(n) * np.log(vocab + 1)).astype(np.int64) - 1, vocab - 1) * 7919 % vocab
    elif kind == "one":
        ids = np.full(n, vocab // 2)
    elif kind == "none":
        ids = np.full(n, -1)
    elif kind == "ends":
        ids = np.where(rng.random(n) < 0.5, 0, vocab - 1)
    elif kind == "rising":
        ids = np.arange(n) % vocab
    else:                        # anything, the outside too
        ids = rng.integers(-3, vocab + 3, n)
        if n > 4:
            ids[:4] = (-2 ** 31, 2 ** 31 - 1, vocab, -1)
    return ids.astype(np.int64)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,d,scale", [(1, 1, 1, 1.0), (1, 50, 4096, 0.3), (5, 7, 3, 2.0), (16, 1000, 4096, 64.0), (33, 100, 128, 1.7), (300, 77, 515, 0.1),
                                             (1027, 500, 1003, -1.3), (4100, 3000, 2056, 1.0), (20000, 10, 64, 0.5), (1500, 9, 5000, 3.3), (2, 5, 300000, 1.1)])
def test_forward(n, vocab, d, scale, dtype):
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(n + d)
    t, o = Room(vocab, d, dtype, 3, 1, dev(rng.standard_normal((vocab, d)).astype(np.float32))), Room(n, d, dtype, 1, 3)
    ids = tokens(rng, n, vocab, "any")
    ae.model_embedding(t.m, vocab, d, ints(ids), n, o.m, scale=scale)
    ok = torch.from_numpy((ids >= 0) & (ids < vocab)).cuda()
    rows = t.m.float()[torch.from_numpy(np.clip(ids, 0, vocab - 1)).cuda()] * torch.full((1,), scale, device="cuda")
    assert torch.equal(o.m, torch.where(ok[:, None], rows, torch.zeros((), device="cuda")).to(td(dtype))) and o.whole() and t.whole()
    near(host(o.m), to.embedding(host(t.m), ids, float(np.float32(scale))), 2.0 ** (-8 if dtype == "bf16" else -24) * 1.001 * np.abs(host(rows)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["text", "one", "none", "ends", "rising", "any"])
@pytest.mark.parametrize("n,vocab,d", [(1, 1, 1), (1, 300, 130), (15, 4, 9), (16, 16, 64), (17, 1000, 515), (64, 5, 8), (1000, 700, 33), (4097, 8009, 40), (5000, 3, 2051),
                                       (33000, 20011, 12), (40000, 257, 5)])
def test_gradient(n, vocab, d, kind, dtype):
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(n + vocab)
    ids = tokens(rng, n, vocab, kind)
    g = Room(n, d, dtype, 2, 1, dev(rng.standard_normal((n, d)).astype(np.float32)))
    scale = 1.7
    want, mag, count = to.embedding_backward(host(g.m), ids, vocab, float(np.float32(scale)))
    t = Room(vocab, d, "f32", 3, 1)
    ws = space(ae.model_embedding_backward_workspace(n, vocab, d, ae.DTYPES[dtype]))
    ae.model_embedding_backward(g.m, ints(ids), n, vocab, d, t.m, ws, scale=scale)
    tol = (count[:, None] + 2) * U * mag
    near(host(t.m), want, tol)
    assert t.whole() and g.whole()
    first = t.m.clone()
    if ws is not None:           # the workspace's contents do not matter, and the same call gives the same bits
        ws.zero_()
    ae.model_embedding_backward(g.m, ints(ids), n, vocab, d, t.m, ws, scale=scale)
    assert torch.equal(t.m, first)
    # added to what is there; rows without a token stay as they are
    there = rng.standard_normal((vocab, d)).astype(np.float32)
    a = Room(vocab, d, "f32", 1, 2, dev(there))
    ae.model_embedding_backward(g.m, ints(ids), n, vocab, d, a.m, ws, scale=scale, accumulate=True)
    near(host(a.m), want + there, tol + U * (np.abs(want) + np.abs(there)) * 1.001)
    assert a.whole() and np.array_equal(a.m.cpu().numpy()[count == 0], there[count == 0])


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("kind", ["text", "one", "none", "any"])
@pytest.mark.parametrize("n,vocab,d,dtype", [(511, 40, 515, "f32"), (512, 40, 515, "bf16"), (513, 40, 515, "bf16"), (300, 90, 2051, "f32"), (500, 5000, 3, "bf16"), (512, 3, 300, "f32"),
                                             (129, 1, 4, "f32"), (64, 17, 256, "bf16"), (65, 16, 257, "f32"), (513, 1000, 512, "f32")])
def test_gradient_on_both_sides_of_the_rule_for_few_places(n, vocab, d, dtype, kind, accumulate):
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(n + d)
    ids = tokens(rng, n, vocab, kind)
    g, t = Room(n, d, dtype, 1, 3, dev(rng.standard_normal((n, d)).astype(np.float32))), Room(vocab, d, "f32", 2, 1)
    there = host(t.m) if accumulate else 0.0
    want, mag, count = to.embedding_backward(host(g.m), ids, vocab, -0.75)
    ws = space(ae.model_embedding_backward_workspace(n, vocab, d, ae.DTYPES[dtype]))
    assert (ws is None) == (n <= 512)
    ae.model_embedding_backward(g.m, ints(ids), n, vocab, d, t.m, ws, scale=-0.75, accumulate=accumulate)
    near(host(t.m), want + there, (count[:, None] + 2) * U * mag + accumulate * U * (np.abs(want) + np.abs(there)) * 1.001)
    assert t.whole() and (not accumulate or np.array_equal(host(t.m)[count == 0], there[count == 0]))


def test_gradient_of_long_lists():
    """A frequent token in hundreds of thousands of places, in binary32 partial sums of a run's length each."""
    import torch
    from paper_2602_17681_amd import binding as ae
    n, vocab, d = 700001, 1000, 16
    rng = np.random.default_rng(3)
    ids = np.where(rng.random(n) < 0.6, 17, rng.integers(0, vocab, n))
    g = dev(rng.standard_normal((n, d)).astype(np.float32))
    t, ws = torch.empty((vocab, d), device="cuda"), space(ae.model_embedding_backward_workspace(n, vocab, d, ae.AE_F32))
    ae.model_embedding_backward(g, ints(ids), n, vocab, d, t, ws)
    i64 = torch.from_numpy(ids).cuda()
    want = torch.zeros((vocab, d), dtype=torch.float64, device="cuda").index_add_(0, i64, g.double())
    mag = torch.zeros((vocab, d), dtype=torch.float64, device="cuda").index_add_(0, i64, g.double().abs())
    # chains: up to ceil(n / 2 048) = 342 rows of a run, then the runs, at most 2 048
    near(host(t), host(want), (342 + 2048 + 2) * U * host(mag))


def test_gradient_is_the_adjoint_of_the_lookup():
    """<embedding(table), d> = <table, embedding_backward(d)>, in 64 bits from binary32 results."""
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(9)
    n, vocab, d = 400, 90, 72
    ids = tokens(rng, n, vocab, "any")
    table, g = dev(rng.standard_normal((vocab, d)).astype(np.float32)), dev(rng.standard_normal((n, d)).astype(np.float32))
    o, t = torch.empty_like(g), torch.empty_like(table)
    ae.model_embedding(table, vocab, d, ints(ids), n, o, scale=3.0)
    ae.model_embedding_backward(g, ints(ids), n, vocab, d, t, space(ae.model_embedding_backward_workspace(n, vocab, d, ae.AE_F32)), scale=3.0)
    a, b = (host(o) * host(g)).sum(), (host(table) * host(t)).sum()
    count = np.bincount(ids[(ids >= 0) & (ids < vocab)], minlength=vocab).max()
    assert abs(a - b) <= (count + 3) * U * 3 * np.abs(host(o) * host(g)).sum() + (count + 3) * U * np.abs(host(table)).max() * 3 * np.abs(host(g)).sum()


def test_no_tokens():
    import torch
    from paper_2602_17681_amd import binding as ae
    e = torch.empty((0, 70), device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    t = Room(5000, 70, "f32", 3, 1)
    ae.model_embedding(t.m, 5000, 70, none, 0, e)
    assert ae.model_embedding_backward_workspace(0, 5000, 70, ae.AE_F32) == 0
    ae.model_embedding_backward(e, none, 0, 5000, 70, t.m, None, accumulate=True)
    assert bool((t.m == 123).all())
    ae.model_embedding_backward(e, none, 0, 5000, 70, t.m, None)
    assert bool((t.m == 0).all()) and t.whole()


def test_infinities_stay_in_their_rows():
    import torch
    from paper_2602_17681_amd import binding as ae
    ids = np.array([3, 5, 3, -1, 7] * 20)
    g = np.ones((100, 24), np.float32)
    g[0, 1], g[1, 2], g[3, :] = np.inf, np.nan, np.nan
    t = torch.empty((9, 24), device="cuda")
    ae.model_embedding_backward(dev(g), ints(ids), 100, 9, 24, t, space(ae.model_embedding_backward_workspace(100, 9, 24, ae.AE_F32)))
    want = np.zeros((9, 24))
    want[3], want[5], want[7] = 40, 20, 20
    want[3, 1], want[5, 2] = np.inf, np.nan
    near(host(t), want, 0.0)


def test_streams_and_graphs():
    import torch
    from paper_2602_17681_amd import binding as ae
    n, vocab, d = 3000, 400, 200
    rng = np.random.default_rng(4)
    sets = [(tokens(rng, n, vocab, k), rng.standard_normal((n, d)).astype(np.float32)) for k in ("text", "any", "one")]
    ids, g, table = ints(sets[0][0]), dev(sets[0][1], "bf16"), dev(rng.standard_normal((vocab, d)).astype(np.float32), "bf16")
    o, t = torch.empty_like(g), torch.empty((vocab, d), device="cuda")
    ws = space(ae.model_embedding_backward_workspace(n, vocab, d, ae.AE_BF16))

    def step():
        ae.model_embedding(table, vocab, d, ids, n, o, scale=2.5)
        ae.model_embedding_backward(g, ids, n, vocab, d, t, ws, scale=2.5)

    def change(i):
        ids.copy_(ints(sets[i][0]))
        g.copy_(dev(sets[i][1], "bf16"))
    for i, got in enumerate(replayed(step, [o, t], change)):
        change(i)
        step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], o) and torch.equal(got[1], t)
