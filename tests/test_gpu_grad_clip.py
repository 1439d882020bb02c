"""The norm of many gradients and the clipped gradients against 64 bits: sums are binary64 (the norm is one rounding to binary32, and n 2^-53, away), the factor
is rounded once and the product once more: 2 U relative, and 2^-8 for bfloat16."""
import numpy as np
import pytest

from oracle import token_oracle as to
from token_util import HALF, U, dev, host, near, replayed, space, td

pytestmark = pytest.mark.gpu


def gradients(rng, sizes, dtypes, scale=1.0):
    """Views into one buffer for each type, at odd places."""
    import torch
    out = []
    for n, t in zip(sizes, dtypes):
        buf = torch.full((n + 8,), 77.0, device="cuda").to(td(t))
        off = int(rng.integers(0, 5))
        m = buf[off:off + n]
        m.copy_(dev((scale * rng.standard_normal(n)).astype(np.float32)))
        out.append((buf, m))
    return [b for b, _ in out], [m for _, m in out]


def run(ae, ms, max_norm, out):
    import torch
    lst = ae.GradList(ms, out)
    norm = torch.full((3,), 5.0, device="cuda")
    ae.model_grad_clip(lst, max_norm, norm[1:2], space(ae.model_grad_clip_workspace(lst)))
    assert float(norm[0]) == 5 and float(norm[2]) == 5
    return float(norm[1])


LISTS = {"one": [1], "none": [], "empty": [0, 0], "small": [1, 2, 3, 7, 8, 9, 0, 100], "mixed": [5000, 1, 8192, 8193, 0, 16385, 3, 100000], "hundreds": [17 + 31 * (i % 50) for i in range(500)],
         "border": [8] * 112, "behind": [8] * 113, "large": [12000001, 5, 3000000]}


@pytest.mark.parametrize("types", ["f32", "bf16", "both"])
@pytest.mark.parametrize("name", list(LISTS))
def test_lists(name, types):
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(len(name))
    sizes = LISTS[name]
    dtypes = [("f32", "bf16")[i % 2] if types == "both" else types for i in range(len(sizes))]
    bufs, ms = gradients(rng, sizes, dtypes)
    h = [host(m) for m in ms]
    norm, _ = to.grad_clip(h, 1.0)
    assert abs(run(ae, ms, 1.0, None) - norm) <= 1.001 * U * norm                 # the norm alone: nothing is written
    assert all(np.array_equal(host(m), v) for m, v in zip(ms, h))
    for max_norm in (0.5 * norm + 1e-3, 2 * norm + 1, float("inf")):
        obufs, out = gradients(rng, sizes, dtypes)
        assert abs(run(ae, ms, max_norm, out) - norm) <= 1.001 * U * norm
        _, want = to.grad_clip(h, float(np.float32(max_norm)))
        for m, o, v, w, t, b in zip(ms, out, h, want, dtypes, obufs):
            near(host(o), w, (2.001 * U + (HALF["bf16"] if t == "bf16" else 0)) * np.abs(w) + 2.0 ** -134 * (t == "bf16"))
            assert np.array_equal(host(m), v) and int((b.float() == 77).sum()) == 8
            if max_norm > norm:
                assert torch.equal(o, m)
    # in place: first left alone, then clipped, and the norm is the largest norm afterwards
    assert abs(run(ae, ms, 2 * norm + 1, ms) - norm) <= 1.001 * U * norm and all(np.array_equal(host(m), v) for m, v in zip(ms, h))
    if norm:
        run(ae, ms, 0.25 * norm, ms)
        _, want = to.grad_clip(h, float(np.float32(0.25 * norm)))
        for m, w, t, b in zip(ms, want, dtypes, bufs):
            near(host(m), w, (2.001 * U + (HALF["bf16"] if t == "bf16" else 0)) * np.abs(w) + 2.0 ** -134 * (t == "bf16"))
            assert int((b.float() == 77).sum()) == 8
        assert abs(run(ae, ms, 1.0, None) - 0.25 * norm) <= 2.0 ** -8 * 0.25 * norm


def test_some_in_place_some_not():
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(8)
    _, ms = gradients(rng, [9000, 50, 300], ["f32", "bf16", "f32"])
    h = [host(m) for m in ms]
    other = torch.empty_like(ms[1])
    run(ae, ms, 3.0, [ms[0], other, ms[2]])
    _, want = to.grad_clip(h, 3.0)
    near(host(ms[0]), want[0], 2.001 * U * np.abs(want[0]))
    near(host(other), want[1], 2.0 ** -8 * 1.001 * np.abs(want[1]))
    near(host(ms[2]), want[2], 2.001 * U * np.abs(want[2]))
    assert np.array_equal(host(ms[1]), h[1])


@pytest.mark.parametrize("value", [3e38, 1e-38, 1e-44, 0.0])
def test_extreme_magnitudes(value):
    """Squares that binary32 does not hold; norms beyond binary32 are infinite as a number and right as a factor."""
    import torch
    from paper_2602_17681_amd import binding as ae
    x = dev(np.full(1000, value, np.float32))
    exact = float(np.float32(value)) * np.sqrt(1000.0)
    out = torch.empty_like(x)
    limit = 1.0 if value > 1 else 1e-38
    got = run(ae, [x], limit, [out])
    assert got == np.float32(exact) or abs(got - exact) <= 1.001 * U * exact + 2.0 ** -150
    lim = float(np.float32(limit))
    want = float(np.float32(value)) * min(1.0, lim / exact if exact else 1.0)
    # the factor may be a subnormal number, 2^-149 apart, and so may the product
    near(host(out), np.full(1000, want), 2.001 * U * want + 2.0 ** -150 * 1.001 + float(np.float32(value)) * 2.0 ** -150)


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_a_norm_that_is_no_number_scales_nothing(bad):
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(8)
    _, ms = gradients(rng, [9000, 50], ["f32", "bf16"])
    ms[0][8999] = float(bad)
    out = [torch.empty_like(m) for m in ms]
    norm = run(ae, ms, 1.0, out)
    assert (np.isnan(norm) if np.isnan(bad) else norm == np.inf)
    assert torch.equal(out[0][:-1], ms[0][:-1]) and torch.equal(out[1], ms[1]) and np.array_equal(host(out[0][-1:]), [bad], equal_nan=True)
    before = ms[1].clone()
    run(ae, ms, 1.0, ms)
    assert torch.equal(ms[1], before)


def test_streams_and_graphs():
    """The captured call keeps the addresses; more tensors than one launch takes."""
    import torch
    from paper_2602_17681_amd import binding as ae
    rng = np.random.default_rng(3)
    sizes = [50 + i for i in range(230)]
    sets = [gradients(rng, sizes, ["f32"] * 230, s)[1] for s in (1.0, 1e-3, 50.0)]
    _, ms = gradients(rng, sizes, ["f32"] * 230)
    out = [torch.empty_like(m) for m in ms]
    lst, norm = ae.GradList(ms, out), torch.empty(1, device="cuda")
    ws = space(ae.model_grad_clip_workspace(lst))

    def change(i):
        for m, v in zip(ms, sets[i]):
            m.copy_(v)
    for i, got in enumerate(replayed(lambda: ae.model_grad_clip(lst, 2.0, norm, ws), [norm] + out, change)):
        change(i)
        ae.model_grad_clip(lst, 2.0, norm, ws)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, [norm] + out))
