"""Matrices with room between and around their rows, and what the tests of norms, embeddings, clipping and logits share."""
import numpy as np

U = 2.0 ** -24                   # half a step of binary32, relative
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
MARK = 123.0                     # what lies in the room; exact in every type


def td(dtype):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]


class Room:
    """A device matrix [rows][cols] inside a larger buffer: `pad` elements behind each row, `off` before the first, two rows' room behind the last."""

    def __init__(self, rows, cols, dtype, pad=0, off=0, data=None):
        import torch
        self.t = dtype if isinstance(dtype, torch.dtype) else td(dtype)
        self.ld = cols + pad
        self.buf = torch.full((off + (rows + 2) * self.ld + 8,), MARK, dtype=torch.float32, device="cuda").to(self.t)
        self.m = torch.as_strided(self.buf, (rows, cols), (self.ld, 1), off)
        self.inside = torch.zeros(self.buf.shape, dtype=torch.bool, device="cuda")
        torch.as_strided(self.inside, (rows, cols), (self.ld, 1), off).fill_(True)
        if data is not None:
            self.m.copy_(data if isinstance(data, torch.Tensor) else torch.from_numpy(np.ascontiguousarray(data)))

    def whole(self):
        """Whether everything outside the matrix is as it was."""
        return bool((self.buf.float()[~self.inside] == MARK).all())


def dev(a, dtype="f32"):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(td(dtype))


def ints(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def host(t):
    """In 64 bits."""
    return t.detach().double().cpu().numpy()


def space(nbytes):
    """A workspace of exactly these bytes (or none), full of NaN patterns."""
    import torch
    return torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda") if nbytes else None


def near(got, want, tol):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[np.isinf(want)], want[np.isinf(want)]) and np.all(np.isfinite(got[fine]))
    off = np.abs(got - np.where(fine, want, 0.0)) - np.broadcast_to(tol, want.shape)
    assert not np.any(off[fine] > 0), "worst excess %g at %s" % (off[fine].max(), np.unravel_index(np.argmax(np.where(fine, off, -1)), off.shape))


def replayed(call, outputs, change):
    """The call captured and replayed three times, with eager work between and inputs changed by change(i): what each replay wrote."""
    import torch
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    got = []
    for i in range(3):
        change(i)
        for o in outputs:
            o.view(torch.uint8).fill_(0xA5)
        torch.ones(1000, device="cuda").sum().item()
        g.replay()
        torch.cuda.synchronize()
        got.append([o.clone() for o in outputs])
    return got
