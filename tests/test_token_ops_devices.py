"""Every tensor of a call has to be on the current device, and a list of gradients is of where they lie now; on the host, before any call into the library."""
import pytest
import torch


class Elsewhere(torch.Tensor):
    """A tensor that says of itself that it lies on a device."""
    at = 0
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.at

    def is_contiguous(self, *a, **k):
        return True


def on(device, *shape, dtype=torch.float32):
    with torch._C.DisableTorchFunctionSubclass():
        t = torch.zeros(shape, dtype=dtype).as_subclass(Elsewhere)
    t.at = device
    return t


class Library:
    """Stands in for the library's calls on the device: none may be reached; queries of sizes go through."""

    def __init__(self, lib):
        self.lib, self.calls = lib, []

    def __getattr__(self, name):
        if name.endswith("_workspace"):
            return getattr(self.lib, name)

        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def ae(monkeypatch):
    from paper_2602_17681_amd import binding
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    monkeypatch.setattr(binding, "_stream_of", lambda device: 0)
    monkeypatch.setattr(binding, "lib", Library(binding.lib))
    return binding


R, D, V, N = 4, 64, 100, 600          # N: more tokens than the form without a workspace takes
i32 = torch.int32


def calls(ae, at):
    """Each call with the device that `at` gives to each of its tensors."""
    m = lambda name, *shape, dtype=torch.float32: on(at(name), *shape, dtype=dtype)      # noqa: E731
    room = lambda n: m("workspace", max(16, n), dtype=torch.uint8)      # noqa: E731
    yield "rms_norm", lambda: ae.model_rms_norm(m("x", R, D), R, D, m("weight", D), 1e-6, m("h", R, D), m("y", R, D), m("q", R, D, dtype=torch.uint8), m("scale", 1, R), residual=m("residual", R, D))
    yield "rms_norm_backward", lambda: ae.model_rms_norm_backward(m("dy", R, D), m("h", R, D), R, D, m("weight", D), 1e-6, m("dx", R, D), m("d_weight", D),
                                                                  room(ae.model_rms_norm_backward_workspace(R, D, 0)), d_h=m("d_h", R, D))
    yield "embedding", lambda: ae.model_embedding(m("table", V, D), V, D, m("ids", N, dtype=i32), N, m("out", N, D))
    yield "embedding_backward", lambda: ae.model_embedding_backward(m("d_out", N, D), m("ids", N, dtype=i32), N, V, D, m("d_table", V, D), room(ae.model_embedding_backward_workspace(N, V, D, 0)))
    yield "grad_clip", lambda: ae.model_grad_clip(ae.GradList([on(0, D)], [on(0, D)]), 1.0, m("norm", 1), room(64))
    yield "logits_adjust", lambda: ae.model_logits_adjust(m("logits", R, V), R, V, m("out", R, V), history=m("history", R, 3, dtype=i32), n_prompt=m("n_prompt", R, dtype=i32),
                                                          repetition=m("repetition", R), presence=m("presence", R), frequency=m("frequency", R), bias_id=m("bias_id", R, 2, dtype=i32),
                                                          bias=m("bias", R, 2), allowed=m("allowed", R, 4, dtype=i32))


TENSORS = {"rms_norm": ["x", "weight", "h", "y", "q", "scale", "residual"], "rms_norm_backward": ["dy", "h", "weight", "dx", "d_weight", "workspace", "d_h"], "embedding": ["table", "ids", "out"],
           "embedding_backward": ["d_out", "ids", "d_table", "workspace"], "grad_clip": ["norm", "workspace"],
           "logits_adjust": ["logits", "out", "history", "n_prompt", "repetition", "presence", "frequency", "bias_id", "bias", "allowed"]}


def test_calls_on_the_current_device_go_through(ae):
    for name, call in calls(ae, lambda tensor: 0):
        call()
        assert ae.lib.calls.pop()[0] == "model_" + name


@pytest.mark.parametrize("name,tensor", [(n, t) for n, ts in TENSORS.items() for t in ts])
def test_a_tensor_of_another_device_is_refused(ae, name, tensor):
    call = dict(calls(ae, lambda t: 1 if t == tensor else 0))[name]
    with pytest.raises(AssertionError, match="device 1"):
        call()
    assert not ae.lib.calls


def test_a_list_of_another_device_is_refused(ae):
    lst = ae.GradList([on(1, D)])
    with pytest.raises(AssertionError, match="device 1"):
        ae.model_grad_clip(lst, 1.0, on(0, 1), on(0, 64, dtype=torch.uint8))
    with pytest.raises(AssertionError):
        ae.GradList([on(0, D), on(1, D)])
    assert not ae.lib.calls


def addresses(call):
    return [None if call[1][i] is None else list(call[1][i]) for i in (0, 6)], list(call[1][1])


def test_a_list_follows_its_tensors(ae):
    """Tensors that were given other memory since the list was made: the call takes what they are now, or refuses it."""
    g, o = [on(0, D), on(0, 8)], [on(0, D), on(0, 8)]
    lst, norm, ws = ae.GradList(g, o), on(0, 1), on(0, 64, dtype=torch.uint8)
    ae.model_grad_clip(lst, 1.0, norm, ws)
    where = lambda ts: [t.data_ptr() for t in ts]      # noqa: E731
    assert addresses(ae.lib.calls.pop()) == ([where(g), where(o)], [D, 8])
    for k, ts in enumerate((g, o)):
        before = ts[1].data_ptr()
        ts[1].data = torch.ones(8)
        assert ts[1].data_ptr() != before
        ae.model_grad_clip(lst, 1.0, norm, ws)
        assert addresses(ae.lib.calls.pop()) == ([where(g), where(o)], [D, 8])
    for t in (g[0], o[0]):
        t.data = torch.zeros(2 * D)
    ae.model_grad_clip(lst, 1.0, norm, ws)
    assert addresses(ae.lib.calls.pop()) == ([where(g), where(o)], [2 * D, 8])
    g[0].data = torch.zeros(3 * D)                       # no longer of its output's size
    with pytest.raises(AssertionError):
        ae.model_grad_clip(lst, 1.0, norm, ws)
    alone = ae.GradList(g)
    g[1].data = torch.zeros(8)
    ae.model_grad_clip(alone, 1.0, norm, ws)
    assert addresses(ae.lib.calls.pop()) == ([where(g), None], [3 * D, 8])


def test_a_list_in_place_follows_its_tensors(ae):
    g = [on(0, D), on(0, 8)]
    lst, norm, ws = ae.GradList(g, g), on(0, 1), on(0, 64, dtype=torch.uint8)
    g[0].data = torch.zeros(D)
    ae.model_grad_clip(lst, 1.0, norm, ws)
    where = [t.data_ptr() for t in g]
    assert addresses(ae.lib.calls.pop()) == ([where, where], [D, 8])
