"""What the Python calls on rows of logits say about arguments that are missing, without a GPU."""
import pytest
import torch

X, U, N = torch.zeros(3, 10), torch.zeros(3), torch.zeros(3, dtype=torch.int32)
IDS, TOP = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2)


@pytest.mark.parametrize("call,args,name", [
    ("dream_sample", (None, U, N), "logits"), ("dream_sample", (X, None, N), "uniforms"), ("dream_sample", (X, U, None), "tokens"),
    ("dream_truncate_logits", (None, X), "logits"),
    ("dream_distill_loss", (None, IDS, TOP, U, U), "logits"), ("dream_distill_loss", (X, None, TOP, U, U), "teacher_ids"),
    ("dream_distill_loss", (X, IDS, None, U, U), "teacher_logits"), ("dream_distill_loss", (X, IDS[:, 0], TOP, U, U), "teacher_ids"),
    ("dream_distill_loss", (X, torch.tensor(1), TOP, U, U), "teacher_ids"),
    ("dream_distill_grad", (None, IDS, TOP, U, X), "logits"), ("dream_distill_grad", (X, None, TOP, U, X), "teacher_ids"),
    ("dream_distill_grad", (X, IDS, None, U, X), "teacher_logits"), ("dream_distill_grad", (X, torch.tensor(1), TOP, U, X), "teacher_ids"),
])
def test_what_is_missing_is_named(call, args, name):
    from paper_2505_19201_b200 import api
    with pytest.raises(api.DreamError) as e:
        getattr(api, call)(*args)
    assert e.value.code == -1 and name in str(e.value)


@pytest.mark.parametrize("bad", [dict(uniform=U.double()), dict(uniform=U[:0]), dict(uniform=U.to("meta")), dict(first_token=U), dict(logprob=N),
                                 dict(logprob=U.to("meta"))])
def test_first_token_checks_its_tensors(bad):
    from types import SimpleNamespace
    from paper_2505_19201_b200 import api
    ctx = SimpleNamespace(h=None, arena=U)
    with pytest.raises(api.DreamError) as e:
        api.Context.dream_sample_first(ctx, 0, **{"uniform": U, **bad})
    assert e.value.code == -1 and next(iter(bad)) in str(e.value)


@pytest.mark.gpu
@pytest.mark.parametrize("call", ["dream_truncate_logits", "dream_distill_loss", "dream_distill_grad"])
def test_missing_outputs(call):
    from paper_2505_19201_b200 import api
    x, u, ids, top = X.cuda(), U.cuda(), IDS.cuda(), TOP.cuda()
    for args in {"dream_truncate_logits": [(x, None)], "dream_distill_loss": [(x, ids, top, None, u), (x, ids, top, u, None)],
                 "dream_distill_grad": [(x, ids, top, None, x), (x, ids, top, u, None)]}[call]:
        with pytest.raises(api.DreamError) as e:
            getattr(api, call)(*args)
        assert e.value.code == -1


@pytest.mark.gpu
def test_no_rows():
    from paper_2505_19201_b200 import api
    x, u, n, ids, top = X.cuda()[:0], U.cuda()[:0], N.cuda()[:0], IDS.cuda()[:0], TOP.cuda()[:0]
    for call in (lambda: api.dream_sample(x, u, n), lambda: api.dream_truncate_logits(x, x), lambda: api.dream_distill_loss(x, ids, top, u, u),
                 lambda: api.dream_distill_grad(x, ids, top, u, x)):
        with pytest.raises(api.DreamError) as e:
            call()
        assert e.value.code == -1
