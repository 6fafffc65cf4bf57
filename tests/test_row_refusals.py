"""What the calls on rows of logits refuse, without a GPU: every check comes before anything is enqueued."""
import ctypes as C

import pytest
import torch

E_ARG, E_CAPACITY = -1, -4


def _lib():
    from paper_2505_19201_b200 import api, build
    build.build()
    return api.lib()


P = C.c_void_p(1 << 20)                                      # an address nobody looks at
Q = C.c_void_p(1 << 40)


def sample(logits=P, dtype=0, rows=4, vocab=100, ld=100, uniforms=Q, tokens=Q):
    return _lib().dream_sample(logits, dtype, rows, vocab, ld, None, None, None, None, uniforms, tokens, None, None, None)


def truncate(logits=P, dtype=0, rows=4, vocab=100, ld=100, out=Q, out_ld=100):
    return _lib().dream_truncate_logits(logits, dtype, rows, vocab, ld, None, None, None, None, out, out_ld, None, None)


def loss(logits=P, dtype=0, rows=4, vocab=100, ld=100, ids=Q, top_logits=Q, top=8, tl=None, tau=1.0, loss=Q, lse=Q, rest=None, grad=None, grad_ld=0):
    return _lib().dream_distill_loss(logits, dtype, rows, vocab, ld, ids, top_logits, top, tl, tau, loss, lse, rest, None, grad, grad_ld, None)


def grad(logits=P, dtype=0, rows=4, vocab=100, ld=100, ids=Q, top_logits=Q, top=8, tl=None, tau=1.0, lse=Q, rest=None, grad=Q, grad_ld=100):
    return _lib().dream_distill_grad(logits, dtype, rows, vocab, ld, ids, top_logits, top, tl, tau, lse, rest, None, grad, grad_ld, None)


@pytest.mark.parametrize("call", [sample, truncate, loss, grad])
@pytest.mark.parametrize("bad,code", [(dict(logits=None), E_ARG), (dict(dtype=2), E_ARG), (dict(rows=0), E_ARG), (dict(rows=-1), E_ARG),
                                      (dict(vocab=0), E_ARG), (dict(ld=99), E_ARG), (dict(ld=0), E_ARG), (dict(logits=C.c_void_p((1 << 20) + 2)), E_ARG),
                                      (dict(vocab=262145, ld=262145), E_CAPACITY), (dict(rows=(1 << 24) + 1), E_CAPACITY)])
def test_matrix(call, bad, code):
    kw = dict(bad)
    if "ld" in kw and kw["ld"] > 100 and call in (truncate, grad):
        kw["out_ld" if call is truncate else "grad_ld"] = kw["ld"]
    assert call(**kw) == code
    assert _lib().dream_last_error(None)


@pytest.mark.parametrize("call,bad", [
    (sample, dict(uniforms=None)), (sample, dict(tokens=None)),
    (truncate, dict(out=None)), (truncate, dict(out_ld=50)), (truncate, dict(out=C.c_void_p((1 << 40) + 1))),
    (loss, dict(ids=None)), (loss, dict(top_logits=None)), (loss, dict(loss=None)), (loss, dict(lse=None)), (loss, dict(top=0)), (loss, dict(top=129)),
    (loss, dict(tau=0.0)), (loss, dict(tau=-1.0)), (loss, dict(tau=float("nan"))), (loss, dict(tau=float("inf"))), (loss, dict(tau=1e-30)), (grad, dict(tau=1e30)),
    (loss, dict(tl=Q)), (loss, dict(rest=Q)), (loss, dict(grad=Q, grad_ld=99)),
    (grad, dict(grad=None)), (grad, dict(lse=None)), (grad, dict(tl=Q)), (grad, dict(rest=Q)), (grad, dict(top=129)), (grad, dict(tau=0.0)),
])
def test_the_other_arguments(call, bad):
    assert call(**bad) == E_ARG


@pytest.mark.parametrize("call,out,out_ld", [(truncate, "out", "out_ld"), (grad, "grad", "grad_ld"), (loss, "grad", "grad_ld")])
def test_matrices_that_overlap(call, out, out_ld):
    at = lambda elements: C.c_void_p((1 << 20) + 4 * elements)  # noqa: E731
    for where, ld, old in ((0, 100, 120), (1, 100, 100), (50, 100, 100), (-50, 100, 100), (399, 100, 100), (250, 300, 300)):
        assert call(**{"ld": ld, out: at(where), out_ld: old}) == E_ARG, where
    assert "overlap" in _lib().dream_last_error(None).decode()


def test_wrappers_check_types_shapes_and_devices():
    from paper_2505_19201_b200 import api
    _lib()
    x, i32 = torch.zeros(3, 10), lambda *n: torch.zeros(*n, dtype=torch.int32)
    u, n = torch.zeros(3), i32(3)
    with pytest.raises(api.DreamError) as e:
        api.dream_sample(x, u, n)                            # not on a GPU
    assert e.value.code == E_ARG and "CUDA" in str(e.value)
    for bad in (x.double(), x[0], torch.zeros(3, 20)[:, ::2], x.int()):
        for call in (lambda t: api.dream_sample(t, u, n), lambda t: api.dream_truncate_logits(t, t),
                     lambda t: api.dream_distill_loss(t, i32(3, 2), torch.zeros(3, 2), u, u),
                     lambda t: api.dream_distill_grad(t, i32(3, 2), torch.zeros(3, 2), u, t)):
            with pytest.raises(api.DreamError) as e:
                call(bad)
            assert e.value.code == E_ARG
