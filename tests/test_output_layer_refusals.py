"""Arguments that the 8-bit products and the passes over logits refuse, on the host, before any GPU call."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def ae():
    from paper_2602_17681_amd import binding
    return binding


P = C.c_void_p(4096)            # never read: every call below is refused first
ODD = C.c_void_p(4097)


def refused(ae, rc, word):
    assert rc == -1 and word in ae.model_last_error(), (rc, ae.model_last_error())


def test_quantize(ae):
    q = ae.lib.model_fp8_quantize
    refused(ae, q(P, 4, 64, 64, 7, 0, P, 64, P, None, 0, None, None), "dtype")
    refused(ae, q(P, 4, 64, 64, 0, 2, P, 64, P, None, 0, None, None), "blocks")
    refused(ae, q(P, -1, 64, 64, 0, 0, P, 64, P, None, 0, None, None), "size")
    refused(ae, q(P, 4, 64, 63, 0, 0, P, 64, P, None, 0, None, None), "size")
    refused(ae, q(P, 4, 64, 64, 0, 0, None, 64, None, None, 0, None, None), "no output")
    refused(ae, q(P, 4, 64, 64, 0, 0, P, 64, None, None, 0, None, None), "together")
    refused(ae, q(None, 4, 64, 64, 0, 0, P, 64, P, None, 0, None, None), "null")
    refused(ae, q(ODD, 4, 64, 64, 1, 0, P, 64, P, None, 0, None, None), "border")
    refused(ae, q(P, 4, 60, 64, 0, 0, P, 60, P, None, 0, None, None), "16-byte")
    refused(ae, q(P, 4, 64, 64, 0, 0, P, 48, P, None, 0, None, None), "16-byte")
    refused(ae, q(P, 40, 64, 64, 0, 0, None, 0, None, P, 32, P, None), "16-byte")
    refused(ae, q(P, 4, 64, 64, 0, 0, P, 64, ODD, None, 0, None, None), "scales")
    assert q(None, 0, 64, 64, 0, 0, P, 64, P, None, 0, None, None) == 0 and q(None, 5, 0, 0, 0, 0, P, 0, P, None, 0, None, None) == 0


def test_matmul(ae):
    mm = lambda a=P, lda=64, sa=P, b=P, ldb=64, sb=P, bl=0, bias=None, m=4, n=8, k=64, dt=0, y=P, ldy=8: \
        ae.lib.model_fp8_matmul(a, lda, sa, b, ldb, sb, bl, bias, m, n, k, dt, y, ldy, None, None)      # noqa: E731
    refused(ae, mm(dt=3), "dtype")
    refused(ae, mm(bl=5), "b_blocks")
    for bad in (dict(m=-1), dict(n=-1), dict(k=0), dict(m=1 << 31), dict(k=1 << 40)):
        refused(ae, mm(**bad), "size")
    for bad in (dict(a=None), dict(sa=None), dict(b=None), dict(sb=None), dict(y=None)):
        refused(ae, mm(**bad), "null")
    for bad in (dict(lda=48), dict(lda=72), dict(ldb=63), dict(a=ODD), dict(b=ODD)):
        refused(ae, mm(**bad), "16-byte")
    refused(ae, mm(sa=ODD), "misaligned")
    refused(ae, mm(bias=ODD), "misaligned")
    refused(ae, mm(ldy=7), "bad y")
    refused(ae, mm(y=ODD), "bad y")
    assert mm(m=0, a=None) == 0 and mm(n=0, b=None) == 0
    n = C.c_int64()
    refused(ae, ae.lib.model_fp8_matmul_workspace(4, 4, 0, C.byref(n)), "bad argument")
    refused(ae, ae.lib.model_fp8_matmul_workspace(4, 4, 4, None), "bad argument")


def test_linear(ae):
    lin = lambda x=P, ldx=64, w=P, ldw=64, ws=P, m=400, n=8, k=64, dt=0, y=P, room=P: \
        ae.lib.model_fp8_linear(x, ldx, w, ldw, ws, None, m, n, k, dt, y, n, room, None)      # noqa: E731
    refused(ae, lin(room=None), "workspace")
    refused(ae, lin(room=C.c_void_p(8)), "workspace")
    refused(ae, lin(dt=9), "dtype")
    refused(ae, lin(k=0), "size")
    refused(ae, lin(ldx=63), "size")
    refused(ae, lin(x=None), "null")
    refused(ae, lin(m=1, x=None), "null")
    refused(ae, lin(x=ODD), "border")
    refused(ae, lin(m=1, ldw=40), "16-byte")
    refused(ae, lin(m=1, w=None), "null")
    refused(ae, lin(m=1, ws=None), "null")
    refused(ae, lin(m=1, y=None), "null")
    assert lin(m=0, x=None, room=None) == 0
    n = C.c_int64()
    assert ae.lib.model_fp8_linear_workspace(400, 8, 64, C.byref(n)) == 0 and n.value >= 400 * 64 + 400 * 4


def test_token_logprobs(ae):
    def call(z=P, rows=4, vocab=100, ld=100, dt=0, temp=1.0, tok=P, nt=1, k=5, lp=P, room=P):
        return ae.lib.model_token_logprobs(z, rows, vocab, ld, dt, temp, tok, nt, k, lp, P, P, P, P, P, room, None)
    refused(ae, call(dt=2), "dtype")
    refused(ae, call(rows=-1), "rows")
    refused(ae, call(rows=(1 << 24) + 1), "rows")
    refused(ae, call(vocab=0), "vocab")
    refused(ae, call(vocab=(1 << 20) + 1, ld=1 << 21), "vocab")
    refused(ae, call(ld=99), "overlap")
    for t in (0.0, -1.0, float("nan"), float("inf")):
        refused(ae, call(temp=t), "temperature")
    refused(ae, call(nt=-1), "n_tokens")
    refused(ae, call(nt=1025), "n_tokens")
    refused(ae, call(k=-1), "top_k")
    refused(ae, call(k=101), "top_k")
    refused(ae, call(k=257, vocab=1000, ld=1000), "top_k")
    refused(ae, call(z=None), "null")
    refused(ae, call(tok=None), "null")
    refused(ae, call(lp=None), "null")
    refused(ae, call(z=ODD), "misaligned")
    refused(ae, call(vocab=50000, ld=50000, room=None), "workspace")
    assert call(rows=0, z=None) == 0
    n = C.c_int64()
    assert ae.lib.model_token_logprobs_workspace(4, 50000, 5, 0, C.byref(n)) == 0 and n.value > 0
    refused(ae, ae.lib.model_token_logprobs_workspace(4, 50000, 5, 0, None), "null")


def test_loss_distill(ae):
    def call(z=P, rows=4, vocab=100, ld=100, dt=0, temp=1.0, ids=P, t=P, k=5, lr=P, l=P, g=P, ldd=100, room=P):
        return ae.lib.model_loss_distill(z, rows, vocab, ld, dt, temp, ids, t, k, None, None, lr, l, g, ldd, room, None)
    refused(ae, call(dt=2), "dtype")
    refused(ae, call(rows=-1), "rows")
    refused(ae, call(vocab=0), "vocab")
    refused(ae, call(ld=99), "overlap")
    refused(ae, call(ldd=99), "overlap")
    refused(ae, call(temp=0.0), "temperature")
    refused(ae, call(k=0), "top_k")
    refused(ae, call(k=101), "top_k")
    refused(ae, call(lr=None, l=None, g=None), "no output")
    for bad in (dict(z=None), dict(ids=None), dict(t=None)):
        refused(ae, call(**bad), "null")
    refused(ae, call(z=ODD), "misaligned")
    refused(ae, call(ld=128, ldd=100), "stride")
    refused(ae, call(g=C.c_void_p(8192), room=None), "workspace")
    n = C.c_int64()
    assert ae.lib.model_loss_distill_workspace(4, 50000, 1, C.byref(n)) == 0 and n.value >= 16


def test_binding_refuses_wrong_tensors(ae):
    """The binding's own checks, on CPU tensors: none of them reaches the library."""
    import torch
    x = torch.zeros((4, 64))
    with pytest.raises(AssertionError):
        ae.model_fp8_quantize(x, 4, 64, "rows", None, None)
    with pytest.raises(AssertionError):
        ae.model_token_logprobs(x, 4, 64, None, 0, None, None, None, None, None, None, None)
    with pytest.raises(AssertionError):
        ae.model_loss_distill(x, 4, 64, torch.zeros((4, 1), dtype=torch.int32), torch.zeros((4, 1)), None, None, None, None)


@pytest.mark.parametrize("temp", [1e-39, float.fromhex("0x1.fffffcp-127"), -1.0, float("nan"), float("inf")])
def test_temperature_is_a_positive_normal_number(ae, temp):
    refused(ae, ae.lib.model_token_logprobs(P, 4, 64, 64, ae.AE_BF16, temp, None, 0, 1, None, P, P, P, P, P, P, None), "temperature")
    refused(ae, ae.lib.model_loss_distill(P, 4, 64, 64, ae.AE_BF16, temp, P, P, 4, None, None, P, P, None, 0, P, None), "temperature")


def test_sizes_end_below_the_largest_int(ae):
    room = C.c_int64()
    assert ae.lib.model_fp8_matmul_workspace((1 << 31) - 513, 1, 1, C.byref(room)) == 0 and room.value == 0
    refused(ae, ae.lib.model_fp8_matmul_workspace((1 << 31) - 512, 1, 1, C.byref(room)), "bad argument")
    refused(ae, ae.lib.model_fp8_matmul_workspace(1, (1 << 31) - 512, 1, C.byref(room)), "bad argument")
    refused(ae, ae.lib.model_fp8_linear_workspace(1, 1, (1 << 31) - 512, C.byref(room)), "bad argument")
