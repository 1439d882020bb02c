"""Clipping by norms that binary32 does not hold, by factors that it does not, and lists at the border of a launch.

Bounds.  The factor is a quotient in binary64, the product is rounded to binary32 once: U, and 2^-150 where it is subnormal; to bfloat16 from there: 2^-8."""
import numpy as np
import pytest

from oracle import token_oracle as to
from token_util import HALF, U, dev, host, near, space, td

pytestmark = pytest.mark.gpu
ONCE = U * (1 + 2.0 ** -20)


def run(ae, grads, max_norm, out):
    import torch
    lst, norm = ae.GradList(grads, out), torch.full((1,), 5.0, device="cuda")
    ae.model_grad_clip(lst, max_norm, norm, space(ae.model_grad_clip_workspace(lst)))
    return norm.item()


def bound(want, dtype):
    return (ONCE if dtype == "f32" else HALF["bf16"] + U) * np.abs(want) + (2.0 ** -150 if dtype == "f32" else 2.0 ** -134) * 1.001


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("size,max_norm", [(3e38, 1e-3), (3e38, 1.0), (1e38, 1e-37), (1e30, 1e-10), (1e25, 1e-20), (1e10, 1e-30), (3e38, 3e38)])
def test_factors_below_binary32(size, max_norm, in_place, dtype):
    """max_norm / norm is subnormal or less; clipped gradients are as exact as any.  A norm beyond binary32 reads as infinity and clips all the same."""
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(3)
    g = [host(dev((size * rng.uniform(-1, 1, n)).astype(np.float32), dtype)) for n in (1, 1000, 9001)]
    g[0][0] = host(dev(np.float32([size]), dtype))[0]
    norm, want = to.grad_clip(g, float(np.float32(max_norm)))
    ts = [dev(v, dtype) for v in g]
    out = ts if in_place else [torch.empty_like(t) for t in ts]
    got = run(ae, ts, max_norm, out)
    assert abs(got - norm) <= 1.001 * U * norm if norm < 3.4e38 else got == np.inf
    for o, w in zip(out, want):
        near(host(o), w, bound(w, dtype))
    assert abs(host(out[1])).max() > 0 or max_norm < 1e-36


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_rounding(dtype):
    """Factor and product are not rounded to binary32 one after the other."""
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(7)
    g = host(dev(rng.standard_normal(200000).astype(np.float32), dtype))
    norm, (want,) = to.grad_clip([g], float(np.float32(0.7)))
    out = torch.empty(200000, dtype=td(dtype), device="cuda")
    run(ae, [dev(g, dtype)], 0.7, [out])
    near(host(out), want, bound(want, dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norms_next_to_the_largest(dtype):
    """Lists clipped to a norm just below their own, by factors within 2^-25 of one and further off: elsewhere and in place alike."""
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(11)
    g = [host(dev((2.0 ** np.arange(-20, 20).repeat(50) * (1 + rng.integers(0, 2 ** 23, 2000) * 2.0 ** -23)).astype(np.float32), dtype))]
    norm, _ = to.grad_clip(g, 1.0)
    for steps in (1, 2, 3, 8, 1000):
        limit = float(np.float32(norm))
        for _ in range(steps):
            limit = float(np.nextafter(np.float32(limit), np.float32(0)))
        _, (want,) = to.grad_clip(g, limit)
        a, out = dev(g[0], dtype), torch.empty(2000, dtype=td(dtype), device="cuda")
        run(ae, [a], limit, [out])
        near(host(out), want, bound(want, dtype))
        run(ae, [a], limit, [a])
        assert torch.equal(a, out)


@pytest.mark.parametrize("kind", ["f32", "bf16", "both"])
@pytest.mark.parametrize("full", [127, 128, 129, 256, 257, 1000])
def test_lists_at_the_border_of_a_launch(full, kind):
    """As many tensors as a launch takes, and one more or less, with tensors of no elements before, at and behind the border."""
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(full)
    for empty_at in ((), (0,), (full,), (127, 128), (126, 127, 128, 129, full)):
        sizes, at = [], 0
        for i in range(full + 1):
            sizes += [0] * empty_at.count(i)
            if i < full:
                sizes.append(int(rng.integers(1, 40)) if i != full - 1 else 8193)
        dtypes = [("f32", "bf16")[i % 2] if kind == "both" else kind for i in range(len(sizes))]
        bufs = {t: torch.full((sum(sizes) + 64 * len(sizes),), 77.0, device="cuda").to(td(t)) for t in ("f32", "bf16")}
        g = [host(dev(rng.standard_normal(n).astype(np.float32), t)) for n, t in zip(sizes, dtypes)]
        ts, out, inside = [], [], {t: torch.zeros(b.shape, dtype=torch.bool, device="cuda") for t, b in bufs.items()}
        for v, n, t in zip(g, sizes, dtypes):
            ts.append(dev(v, t))
            out.append(bufs[t][at:at + n])
            inside[t][at:at + n] = True
            at += n + int(rng.integers(0, 5))
        norm, want = to.grad_clip(g, 1.0)
        assert abs(run(ae, ts, 1.0, None) - norm) <= 1.001 * U * norm
        assert abs(run(ae, ts, 1.0, out) - norm) <= 1.001 * U * norm
        for o, w, t in zip(out, want, dtypes):
            near(host(o), w, bound(w, t))
        assert all(bool((b[~inside[t]] == 77).all()) for t, b in bufs.items())
        assert abs(run(ae, ts, 1.0, ts) - norm) <= 1.001 * U * norm
        assert all(torch.equal(a, b) for a, b in zip(ts, out))


@pytest.mark.parametrize("count", [500, 640, 641, 1000, 5000])
def test_long_lists(count):
    """Dozens of launches, whose shares of the sum are added up once; replayed as a graph, too."""
    import torch
    from paper_2602_17681_amd import binding as ae
    from token_util import replayed
    rng = np.random.default_rng(5)
    sizes = [int(n) for n in rng.integers(1, 30, count - 1)] + [20000]
    g = [rng.standard_normal(n).astype(np.float32) for n in sizes]
    flat = dev(np.concatenate(g))
    ts, res = list(flat.split(sizes)), torch.empty_like(flat)
    out = list(res.split(sizes))
    norm, want = to.grad_clip(g, 2.0)
    assert abs(run(ae, ts, 2.0, out) - norm) <= 1.001 * U * norm
    near(host(res), np.concatenate(want), bound(np.concatenate(want), "f32"))
    lst, n = ae.GradList(ts, out), torch.empty(1, device="cuda")
    ws = space(ae.model_grad_clip_workspace(lst))
    first = flat.clone()
    for i, got in enumerate(replayed(lambda: ae.model_grad_clip(lst, 2.0, n, ws), [n, res], lambda i: flat.copy_(first * (i + 1)))):
        flat.copy_(first * (i + 1))
        ae.model_grad_clip(lst, 2.0, n, ws)
        torch.cuda.synchronize()
        assert torch.equal(got[0], n) and torch.equal(got[1], res)


@pytest.mark.parametrize("in_place", [False, True])
def test_a_kept_list_follows_its_tensors(in_place):
    """Gradients, and places of the clipped ones, that are given other memory between two calls: the old memory stays as it is."""
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(2)
    ts = [dev(rng.standard_normal(n).astype(np.float32)) for n in (5000, 3, 9000)]
    out = ts if in_place else [torch.empty_like(t) for t in ts]
    lst, norm = ae.GradList(ts, out), torch.empty(1, device="cuda")
    ws = space(ae.model_grad_clip_workspace(lst))
    for step in range(4):
        if step:
            old = [t.detach() for t in ts] + [o.detach() for o in out]
            kept = [o.clone() for o in old]
            g = [rng.standard_normal(t.numel()).astype(np.float32) for t in ts]
            for k, t in enumerate(ts):
                if step == 3 or k == step:
                    t.data = dev(g[k])
                else:
                    t.copy_(dev(g[k]))
            if not in_place and step == 2:
                out[1].data = torch.full_like(out[1], 9.0)
        h = [host(t) for t in ts]
        want_norm, want = to.grad_clip(h, 1.0)
        ae.model_grad_clip(lst, 1.0, norm, ws)
        assert abs(norm.item() - want_norm) <= 1.001 * U * want_norm
        for o, w in zip(out, want):
            near(host(o), w, bound(w, "f32"))
        if step == 3:
            assert all(torch.equal(a, b) for a, b in zip(old[:3], kept[:3]))
