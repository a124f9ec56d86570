"""Refusals of the calls of the layers around the step: the binding's layout checks
(CPU tensors, nothing reaches a device), the C entry points' own, and the size
queries."""
import pytest
import torch

from paper_2002_09018_amd import binding as B

BF16, F32 = torch.bfloat16, torch.float32


def _raises(fn, match):
    with pytest.raises(ValueError, match=match):
        fn()


def _i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def _bytes(n):
    return torch.zeros(n, dtype=torch.uint8)


def _room(n):
    return _bytes(max(n, 1))


def test_sizes():
    f, g = B.shampoo_vocab_logprobs_workspace_bytes, B.shampoo_vocab_logprobs_grad_workspace_bytes
    assert f(0, 8, 8, F32) == 0 and f(-1, 8, 8, F32) == 0 and f(8, 0, 8, F32) == 0 and f(8, 8, 0, F32) == 0
    assert f(8, (1 << 20) + 1, 8, F32) == 0 and f(8, 8, (1 << 30) + 1, F32) == 0 and f(8, 8, 8, 7) == 0
    assert f(1 << 31, 8, 8, F32) == 0 and f((1 << 31) - 1, 8, 8, BF16) > 0
    assert g(8, 8, 8, F32, 7) == 0 and g(0, 8, 8, F32, F32) == 0
    w, x = B.shampoo_gated_ffn_workspace_bytes, B.shampoo_gated_ffn_grad_workspace_bytes
    assert w(0, 8, 8, BF16) == 0 and w(8, 8, (1 << 19) + 1, BF16) == 0 and w(8, 8, 1 << 19, BF16) > 0
    assert x(8, 8, 8, BF16, 9) == 0 and x(8, 8, 8, BF16, BF16) > 0
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        f(8, 8, 8, torch.float16)


def test_the_logits_are_not_kept():
    """The workspace grows with a piece of the logits, not with all of them."""
    rows, dim = 8192, 1024
    for vocab in (131072, 1 << 20):
        logits = 2 * rows * vocab
        assert B.shampoo_vocab_logprobs_workspace_bytes(rows, dim, vocab, BF16) < logits / 4
        assert B.shampoo_vocab_logprobs_grad_workspace_bytes(rows, dim, vocab, BF16, BF16) < (1 << 30)


def test_vocab_checks():
    n, d, v = 4, 6, 10
    room = _room(B.shampoo_vocab_logprobs_workspace_bytes(n, d, v, F32))

    def call(**o):
        a = dict(X=torch.zeros(n, d), W=torch.zeros(v, d), targets=_i32(n), logp=torch.zeros(n), lse=torch.zeros(n),
                 workspace=room)
        a.update(o)
        return lambda: B.shampoo_vocab_logprobs(None, **a)
    _raises(call(), "expected a GPU tensor")
    _raises(call(X=torch.zeros(n, d + 3)[:, :d]), "expected a GPU tensor")
    _raises(call(X=torch.zeros(n, d, dtype=BF16)), "dtype")
    _raises(call(X=torch.zeros(n, d, dtype=torch.float16), W=torch.zeros(v, d, dtype=torch.float16)), "float32 or bfloat16")
    _raises(call(W=torch.zeros(v, d + 1)), "expected")
    _raises(call(W=torch.zeros(d, v).t()), "adjacent")
    _raises(call(X=torch.zeros(1, d).expand(n, d)), "row stride")
    _raises(call(targets=None), "go together")
    _raises(call(logp=None), "go together")
    _raises(call(targets=torch.zeros(n, dtype=torch.int64)), "int32")
    _raises(call(lse=None), "required")
    _raises(call(lse=torch.zeros(n + 1)), "expected")
    _raises(call(logp=torch.zeros(n, dtype=torch.float64)), "float32")
    _raises(call(workspace=None), "needed")
    _raises(call(workspace=room[:-1]), "at least")
    _raises(call(workspace=torch.zeros(1 << 20)), "uint8")


def test_vocab_grad_checks():
    n, d, v = 4, 6, 10
    room = _room(B.shampoo_vocab_logprobs_grad_workspace_bytes(n, d, v, F32, F32))

    def call(**o):
        a = dict(X=torch.zeros(n, d), W=torch.zeros(v, d), targets=_i32(n), lse=torch.zeros(n), dX=torch.zeros(n, d),
                 dW=torch.zeros(v, d), g_logp=torch.zeros(n), g_lse=torch.zeros(n), workspace=room)
        a.update(o)
        return lambda: B.shampoo_vocab_logprobs_grad(None, **a)
    _raises(call(), "expected a GPU tensor")
    _raises(call(dX=None), "expected a GPU tensor")
    _raises(call(dW=torch.zeros(v, d, dtype=BF16)), "expected a GPU tensor")
    _raises(call(dX=None, dW=None), "required")
    _raises(call(targets=None), "needs targets")
    _raises(call(dX=torch.zeros(n, d, dtype=BF16)), "dtype")
    _raises(call(dX=torch.zeros(n, d + 1)), "expected")
    _raises(call(dW=torch.zeros(v + 1, d)), "expected")
    x = torch.zeros(n, d)
    _raises(call(X=x, dX=x), "overlap")
    w = torch.zeros(v, d)
    _raises(call(W=w, dW=w), "overlap")
    big = torch.zeros(n * d + v * d - 1)
    _raises(call(dX=big[:n * d].view(n, d), dW=big[n * d - 1:].view(v, d)), "overlap")
    _raises(call(g_lse=torch.zeros(n, 1)), "expected")
    _raises(call(workspace=room[:-1]), "at least")


def test_ffn_checks():
    n, d, w = 5, 6, 7
    room = _room(B.shampoo_gated_ffn_workspace_bytes(n, d, w, F32))
    grad_room = _room(B.shampoo_gated_ffn_grad_workspace_bytes(n, d, w, F32, F32))
    z = torch.zeros

    def fwd(**o):
        a = dict(X=z(n, d), Wg=z(d, w), Wu=z(d, w), H=z(n, w), G=z(n, w), U=z(n, w), workspace=room)
        a.update(o)
        return lambda: B.shampoo_gated_ffn(None, **a)

    def bwd(**o):
        a = dict(X=z(n, d), Wg=z(d, w), Wu=z(d, w), dH=z(n, w), G=z(n, w), U=z(n, w), dX=z(n, d), dWg=z(d, w),
                 dWu=z(d, w), workspace=grad_room)
        a.update(o)
        return lambda: B.shampoo_gated_ffn_grad(None, **a)
    _raises(fwd(), "expected a GPU tensor")
    _raises(fwd(G=None, U=None), "expected a GPU tensor")
    _raises(fwd(G=None), "go together")
    _raises(fwd(H=None), "required")
    _raises(fwd(Wu=z(d, w, dtype=BF16)), "dtype")
    _raises(fwd(Wu=z(d, w + 1)), "expected")
    _raises(fwd(Wg=z(d + 1, w)), "expected")
    _raises(fwd(H=z(w, n).t()), "adjacent")
    h = z(n, w)
    _raises(fwd(H=h, G=h), "overlap")
    _raises(fwd(workspace=room[:-1]), "at least")
    both = z(n, 2 * w)
    _raises(fwd(G=both[:, :w], U=both[:, w:]), "expected a GPU tensor")  # ranges of one buffer are apart
    _raises(bwd(), "expected a GPU tensor")
    _raises(bwd(dX=None), "expected a GPU tensor")
    _raises(bwd(dWg=None, dWu=None), "expected a GPU tensor")
    _raises(bwd(dWg=None), "go together")
    _raises(bwd(dX=None, dWg=None, dWu=None), "required")
    _raises(bwd(U=None), "go together")
    _raises(bwd(dH=None), "required")
    _raises(bwd(dWu=z(d, w, dtype=BF16)), "dtype")
    _raises(bwd(dWg=z(d, w, dtype=BF16), dWu=z(d, w, dtype=BF16)), "expected a GPU tensor")
    g = z(n, w)
    _raises(bwd(dH=g, G=g), "expected a GPU tensor")                     # both are read only
    dw = z(d, w)
    _raises(bwd(dWg=dw, dWu=dw), "overlap")
    _raises(bwd(Wg=dw, dWg=dw), "overlap")
    _raises(bwd(workspace=grad_room[:-1]), "at least")


def test_dropout_checks():
    n, c = 5, 7
    x, y, r = torch.zeros(n, c), torch.zeros(n, c), torch.zeros(n, c)

    def call(X=x, Y=y, rate=0.1, seed=1, **kw):
        return lambda: B.shampoo_dropout(None, X, Y, rate, seed, **kw)
    _raises(call(), "expected a GPU tensor")
    _raises(call(Y=x, R=r), "expected a GPU tensor")
    _raises(call(Y=r, R=r), "expected a GPU tensor")
    _raises(call(Y=torch.zeros(n, c, dtype=BF16)), "dtype")
    _raises(call(R=torch.zeros(n, c + 1)), "expected")
    _raises(call(X=x.half()), "float32 or bfloat16")
    _raises(call(seed=-1), "outside")
    _raises(call(seed=1 << 64), "outside")
    _raises(call(offset=1 << 64), "outside")
    buf = torch.zeros(n * c + 1)
    _raises(call(X=buf[:-1].view(n, c), Y=buf[1:].view(n, c)), "overlap")
    _raises(call(R=buf[:-1].view(n, c), Y=buf[1:].view(n, c)), "overlap")


def test_null_handle_is_refused():
    lib = B._lib
    assert lib.shampoo_vocab_logprobs(None, None, None, 0, 1, 1, 1, 1, 1, None, None, None, None, 0, None) == B.SHAMPOO_EINVAL
    assert lib.shampoo_vocab_logprobs_grad(None, None, None, 0, 1, 1, 1, 1, 1, None, None, None, None, None, 1, None, 0, 1,
                                           0.0, None, 0, None) == B.SHAMPOO_EINVAL
    assert lib.shampoo_gated_ffn(None, None, None, None, 0, 1, 1, 1, 1, 1, 1, 0, None, 1, None, 1, None, 1, None, 0,
                                 None) == B.SHAMPOO_EINVAL
    assert lib.shampoo_gated_ffn_grad(None, None, None, None, 0, 1, 1, 1, 1, 1, 1, 0, None, 1, None, 1, None, 1, None, 1,
                                      None, 1, None, 1, 0, 0.0, None, 0, None) == B.SHAMPOO_EINVAL
    assert lib.shampoo_dropout(None, None, None, None, 0, 1, 1, 1, 1, 1, 0.5, 0, 0, None) == B.SHAMPOO_EINVAL
