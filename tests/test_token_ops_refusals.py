"""Arguments that norms, embeddings, clipping and adjusted logits refuse, on the host, before any GPU call."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def ae():
    from paper_2602_17681_amd import binding
    return binding


P, P2, P3 = C.c_void_p(4096), C.c_void_p(1 << 30), C.c_void_p(1 << 31)            # never read: every call below is refused first
ODD = C.c_void_p(4097)


def refused(ae, rc, word):
    assert rc == -1 and word in ae.model_last_error(), (rc, ae.model_last_error())


def test_rms_norm(ae):
    def call(x=P, ldx=64, r=None, ldr=64, w=P, rows=4, d=64, eps=1e-6, dt=0, h=None, ldh=64, y=P2, ldy=64, q=None, ldq=64, s=None):
        return ae.lib.model_rms_norm(x, ldx, r, ldr, w, rows, d, eps, dt, h, ldh, y, ldy, q, ldq, s, None)
    refused(ae, call(dt=2), "dtype")
    for rows in (-1, (1 << 31) - 512):
        refused(ae, call(rows=rows), "rows")
    for d in (0, (1 << 20) + 1):
        refused(ae, call(d=d, ldx=1 << 21, ldy=1 << 21), "d must be")
    for eps in (0.0, -1.0, 1e-39, 2.0 ** 61, float("nan"), float("inf")):
        refused(ae, call(eps=eps), "eps")
    refused(ae, call(y=None), "no output")
    refused(ae, call(q=P), "together")
    refused(ae, call(s=P), "together")
    refused(ae, call(x=None), "null")
    for bad in (dict(ldx=63), dict(r=P, ldr=63), dict(h=P3, ldh=63), dict(ldy=63), dict(x=ODD), dict(y=ODD), dict(ldx=1 << 40)):
        refused(ae, call(**bad), "rows must not overlap")
    refused(ae, call(w=ODD), "misaligned")
    for bad in (dict(q=ODD, s=P), dict(q=P3, s=P, ldq=72), dict(q=P3, s=P, ldq=48)):
        refused(ae, call(**bad), "16-byte")
    refused(ae, call(h=P, ldx=128, ldh=64), "stride")
    refused(ae, call(y=P, ldx=128, ldy=64), "stride")
    refused(ae, call(r=P3, ldr=128, h=P3, ldh=64), "stride")
    refused(ae, call(h=P2, y=P2), "places of their own")
    assert call(rows=0, x=None) == 0


def test_rms_norm_backward(ae):
    def call(dy=P, ldy=64, h=P, ldh=64, w=P, dh=None, ldg=64, rows=4, d=64, eps=1e-6, dt=0, dx=P2, ldd=64, dw=P, ws=P3):
        return ae.lib.model_rms_norm_backward(dy, ldy, h, ldh, w, dh, ldg, rows, d, eps, dt, dx, ldd, dw, ws, None)
    refused(ae, call(dt=5), "dtype")
    refused(ae, call(rows=-1), "rows")
    refused(ae, call(d=0), "d must be")
    refused(ae, call(eps=0.0), "eps")
    refused(ae, call(dx=None, dw=None), "no output")
    refused(ae, call(dy=None), "null")
    refused(ae, call(h=None), "null")
    refused(ae, call(ws=None), "workspace")
    refused(ae, call(ws=C.c_void_p(8)), "workspace")
    for bad in (dict(ldy=63), dict(ldh=63), dict(dh=P, ldg=63), dict(ldd=63), dict(dy=ODD), dict(dx=ODD)):
        refused(ae, call(**bad), "rows must not overlap")
    refused(ae, call(w=ODD), "misaligned")
    refused(ae, call(dw=ODD), "misaligned")
    refused(ae, call(dx=P, ldy=128, ldd=64), "stride")
    n = C.c_int64()
    refused(ae, ae.lib.model_rms_norm_backward_workspace(4, 64, 0, None), "null")
    refused(ae, ae.lib.model_rms_norm_backward_workspace(4, 0, 0, C.byref(n)), "d must be")
    assert ae.lib.model_rms_norm_backward_workspace(4, 64, 0, C.byref(n)) == 0 and n.value >= 64 * 4


def test_embedding(ae):
    def call(t=P, ldt=64, vocab=100, d=64, ids=P, n=4, dt=0, out=P2, ldo=64):
        return ae.lib.model_embedding(t, ldt, vocab, d, ids, n, 1.0, dt, out, ldo, None)
    refused(ae, call(dt=2), "dtype")
    refused(ae, call(n=-1), "tokens")
    refused(ae, call(n=(1 << 30) + 1), "tokens")
    refused(ae, call(vocab=0), "vocab")
    refused(ae, call(vocab=(1 << 20) + 1), "vocab")
    refused(ae, call(d=0), "d must be")
    refused(ae, call(ldt=63), "overlap")
    refused(ae, call(ldo=63), "overlap")
    for bad in (dict(t=None), dict(ids=None), dict(out=None)):
        refused(ae, call(**bad), "null")
    for bad in (dict(t=ODD), dict(ids=ODD), dict(out=ODD)):
        refused(ae, call(**bad), "misaligned")
    refused(ae, call(out=P), "place")
    assert call(n=0, t=None) == 0


def test_embedding_backward(ae):
    def call(g=P, ldo=64, ids=P, n=4, vocab=100, d=64, dt=0, t=P2, ldt=64, acc=0, ws=P3):
        return ae.lib.model_embedding_backward(g, ldo, ids, n, vocab, d, 1.0, dt, t, ldt, acc, ws, None)
    refused(ae, call(dt=2), "dtype")
    refused(ae, call(n=-1), "tokens")
    refused(ae, call(vocab=0), "vocab")
    refused(ae, call(d=(1 << 20) + 1, ldo=1 << 21, ldt=1 << 21), "d must be")
    refused(ae, call(ldo=63), "overlap")
    refused(ae, call(ldt=63), "overlap")
    refused(ae, call(t=None), "null")
    refused(ae, call(t=ODD), "misaligned")
    for bad in (dict(g=None), dict(ids=None)):
        refused(ae, call(**bad), "null")
    for bad in (dict(g=ODD), dict(ids=ODD)):
        refused(ae, call(**bad), "misaligned")
    refused(ae, call(n=600, ws=None), "workspace")
    refused(ae, call(n=600, ws=C.c_void_p(8)), "workspace")
    assert call(n=0, acc=1, g=None, ids=None, ws=None) == 0        # nothing to add
    n = C.c_int64()
    refused(ae, ae.lib.model_embedding_backward_workspace(4, 100, 64, 0, None), "null")
    refused(ae, ae.lib.model_embedding_backward_workspace(4, 0, 64, 0, C.byref(n)), "vocab")
    assert ae.lib.model_embedding_backward_workspace(600, 100, 64, 0, C.byref(n)) == 0 and n.value >= 101 * 4 + 2 * 64 * 4


def test_grad_clip(ae):
    def call(grads=(1 << 20, 1 << 21), sizes=(100, 50), dtypes=(0, 1), count=None, mx=1.0, norm=P, out=(1 << 22, 1 << 23), ws=P3):
        a = lambda t, v: None if v is None else (t * max(1, len(v)))(*v)      # noqa: E731
        return ae.lib.model_grad_clip(a(C.c_void_p, grads), a(C.c_int64, sizes), a(C.c_int, dtypes), len(sizes or ()) if count is None else count, mx, norm,
                                      a(C.c_void_p, out), ws, None)
    refused(ae, call(count=-1), "count")
    refused(ae, call(sizes=None, count=2), "count")
    refused(ae, call(sizes=(100, -1)), "sizes")
    refused(ae, call(sizes=(100, (1 << 40) + 1)), "sizes")
    refused(ae, call(norm=None, out=None), "no output")
    refused(ae, call(norm=ODD), "misaligned")
    for mx in (0.0, -1.0, float("nan")):
        refused(ae, call(mx=mx), "max_norm")
    refused(ae, call(grads=None), "null")
    refused(ae, call(dtypes=None), "null")
    refused(ae, call(dtypes=(0, 3)), "dtype of tensor 1")
    refused(ae, call(grads=(1 << 20, None)), "tensor 1 is null")
    refused(ae, call(out=(1 << 22, None)), "tensor 1 is null")
    refused(ae, call(grads=((1 << 20) + 2, 1 << 21)), "tensor 0 is misaligned")
    refused(ae, call(out=(1 << 22, (1 << 23) + 1)), "tensor 1 is misaligned")
    refused(ae, call(ws=None), "workspace")
    refused(ae, call(ws=C.c_void_p(8)), "workspace")
    # outputs that overlap: one twice, partly, another's gradient, the own gradient shifted; in either order of addresses
    for out in ((1 << 22, 1 << 22), (1 << 22, (1 << 22) + 396), ((1 << 22) + 96, 1 << 22), (1 << 22, 1 << 20), (1 << 22, (1 << 21) + 2), ((1 << 20) + 4, 1 << 23)):
        refused(ae, call(out=out), "overlaps")
    refused(ae, call(grads=(1 << 20, 1 << 20), out=(1 << 20, 1 << 20)), "overlaps")
    n = C.c_int64()
    refused(ae, ae.lib.model_grad_clip_workspace((C.c_int64 * 1)(5), 1, None), "null")
    assert ae.lib.model_grad_clip_workspace((C.c_int64 * 3)(5, 0, 1 << 30), 3, C.byref(n)) == 0 and n.value >= 16
    assert ae.lib.model_grad_clip_workspace(None, 0, C.byref(n)) == 0 and n.value == 0


def test_logits_adjust(ae):
    def call(z=P, rows=4, vocab=100, ld=100, dt=0, hist=P, nh=5, npr=P, rep=P, pre=P, fre=P, bid=P, b=P, nb=3, ok=P, out=P2, ldo=100):
        return ae.lib.model_logits_adjust(z, rows, vocab, ld, dt, hist, nh, npr, rep, pre, fre, bid, b, nb, ok, out, ldo, None)
    refused(ae, call(dt=2), "dtype")
    refused(ae, call(rows=-1), "rows")
    refused(ae, call(rows=(1 << 24) + 1), "rows")
    refused(ae, call(vocab=0), "vocab")
    refused(ae, call(vocab=(1 << 20) + 1, ld=1 << 21, ldo=1 << 21), "vocab")
    refused(ae, call(ld=99), "overlap")
    refused(ae, call(ldo=99), "overlap")
    refused(ae, call(nh=-1), "n_history")
    refused(ae, call(nh=1 << 20), "n_history")
    refused(ae, call(nb=-1), "n_bias")
    refused(ae, call(nb=2048), "n_bias")
    for bad in (dict(z=None), dict(out=None), dict(hist=None), dict(bid=None), dict(b=None)):
        refused(ae, call(**bad), "null")
    refused(ae, call(z=ODD), "misaligned logits")
    refused(ae, call(out=ODD), "misaligned logits")
    for name in ("hist", "npr", "rep", "pre", "fre", "bid", "b", "ok"):
        refused(ae, call(**{name: ODD}), "misaligned list")
    refused(ae, call(out=P, ld=128), "stride")
    assert call(rows=0, z=None) == 0


def test_binding_refuses_wrong_tensors(ae):
    """The binding's own checks, on CPU tensors: none of them reaches the library."""
    import torch
    x, ids = torch.zeros((4, 64)), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: ae.model_rms_norm(x, 4, 64, None, 1e-6, y=x), lambda: ae.model_rms_norm_backward(x, x, 4, 64, None, 1e-6, x, None, None),
                 lambda: ae.model_embedding(x, 4, 64, ids, 4, x), lambda: ae.model_embedding_backward(x, ids, 4, 4, 64, x, None),
                 lambda: ae.GradList([x]), lambda: ae.model_logits_adjust(x, 4, 64, x)):
        with pytest.raises(AssertionError):
            call()
