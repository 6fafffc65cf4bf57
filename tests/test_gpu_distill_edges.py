"""Rows at which the distillation could go wrong: masks by a large finite number, sure students, infinities, against closed forms in float64.
Tolerances are those that tests/test_gpu_distill.py derives, where nothing else is said."""
import pytest
import torch

from tests.test_gpu_distill import close_grad, close_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("mask", [-1e8, -1e9, None])
@pytest.mark.parametrize("V,K", [(5, 2), (700, 9), (40000, 31)])
@pytest.mark.parametrize("tau", [1.0, 0.7, 2.6733145])
def test_all_but_the_listed_ids_masked_by_a_number(tau, V, K, mask, dtype):
    """The teacher leaves q_r to ids that the student masks, all alike: p of a listed id is its softmax among the listed, q_r / p_r p_i is q_r over the
    number of the others.  From a saved log_rest, which is a float, the others' gradient is 0."""
    from paper_2505_19201_b200 import api
    R = 6
    mask = torch.finfo(dtype).min if mask is None else mask
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.full((R, V), mask, dtype=dtype, device="cuda")
    ids = torch.stack([torch.randperm(V, device="cuda", generator=g)[:K] for _ in range(R)])
    z = torch.randn(R, K, device="cuda", generator=g).to(dtype)
    x.scatter_(1, ids, z)
    top = torch.randn(R, K, device="cuda", generator=g)
    tau = float(torch.tensor(tau))
    tl = (torch.logsumexp(top.double() / tau, 1) + 0.8).float()
    scale = torch.rand(R, device="cuda", generator=g) + 0.5
    loss, lse, rest = (torch.zeros(R, device="cuda") for _ in range(3))
    step, back = torch.full_like(x, 3.0), torch.full_like(x, 3.0)
    api.dream_distill_loss(x, ids.int(), top, loss, lse, teacher_lse=tl, log_rest=rest, temperature=tau, row_scale=scale, grad=step)
    api.dream_distill_grad(x, ids.int(), top, lse, back, teacher_lse=tl, log_rest=rest, temperature=tau, row_scale=scale)
    q = torch.exp(top.double() / tau - tl.double()[:, None])
    qr = 1 - q.sum(1, keepdim=True)
    p = torch.softmax(z.double() / tau, 1)
    others = -qr / (V - K) / tau
    want = others.expand(R, V).clone().scatter_(1, ids, (p - q) / tau).cpu()
    size = others.abs().expand(R, V).clone().scatter_(1, ids, p / tau).cpu()
    close_grad(step, want, size, scale, dtype)
    listed = torch.zeros(R, V, dtype=torch.bool).scatter_(1, ids.cpu(), True)
    assert not bool(back.cpu()[~listed].any())
    p = torch.exp(z.double() / tau - lse.double()[:, None])
    want = torch.zeros(R, V, dtype=torch.float64, device="cuda").scatter_(1, ids, (p - q) / tau).cpu()
    close_grad(back, want, torch.where(listed, size, 0.0), scale, dtype)
    close_rows(lse, torch.logsumexp(z.double() / tau, 1).cpu(), "lse")
    assert bool((loss > 1e7).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("mask", [-1e8, -1e9, None])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V", [5, 700, 40000])
def test_every_logit_masked_by_a_number(V, tail, mask, dtype):
    """The student is uniform; from a saved lse, which is a float, the row has gradient 0."""
    from paper_2505_19201_b200 import api
    R, K, tau = 4, 3, 0.7
    mask = torch.finfo(dtype).min if mask is None else mask
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.full((R, V), mask, dtype=dtype, device="cuda")
    ids = torch.stack([torch.randperm(V, device="cuda", generator=g)[:K] for _ in range(R)])
    top = torch.randn(R, K, device="cuda", generator=g)
    tau = float(torch.tensor(tau))
    tl = (torch.logsumexp(top.double() / tau, 1) + 0.8).float() if tail else None
    scale = torch.rand(R, device="cuda", generator=g) + 0.5
    loss, lse = (torch.zeros(R, device="cuda") for _ in range(2))
    rest = torch.zeros(R, device="cuda") if tail else None
    step, back = torch.full_like(x, 3.0), torch.full_like(x, 3.0)
    api.dream_distill_loss(x, ids.int(), top, loss, lse, teacher_lse=tl, log_rest=rest, temperature=tau, row_scale=scale, grad=step)
    api.dream_distill_grad(x, ids.int(), top, lse, back, teacher_lse=tl, log_rest=rest, temperature=tau, row_scale=scale)
    q = torch.exp(top.double() / tau - tl.double()[:, None]) if tail else torch.softmax(top.double() / tau, 1)
    qr = 1 - q.sum(1, keepdim=True) if tail else torch.zeros(R, 1, dtype=torch.float64, device="cuda")
    others = (1.0 / V - qr / (V - K)) / tau
    size = ((1.0 / V + qr / (V - K)) / tau).expand(R, V).clone().scatter_(1, ids, torch.full((R, K), 1.0 / V / tau, dtype=torch.float64, device="cuda"))
    close_grad(step, others.expand(R, V).clone().scatter_(1, ids, (1.0 / V - q) / tau).cpu(), size.cpu(), scale, dtype)
    assert not bool(back.any())
    if tail:
        close_rows(rest, torch.log(torch.full((R,), (V - K) / V, dtype=torch.float64)), "log_rest")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,gap,spot", [(1, 0, 0), (2, 40, 1), (5000, 30, 7), (5000, 90, 4999), (150000, 40, 77777)])
def test_a_student_that_is_sure(V, gap, spot, dtype):
    """One logit holds the row and the teacher lists it alone: loss = log1p((V - 1) e^-gap).  In the kernel the sum is 1, to which terms below 2^-25
    are lost within a thread or added by the others: the loss is off by no more than they all are, (V - 1) e^-gap (1 + 2^-20), and the rounding of a sum
    at 1 in float (2^-24 for each of a warp's five steps, were any of the terms above 2^-25, which none is)."""
    from paper_2505_19201_b200 import api
    x = torch.full((3, V), 2.0 - gap, dtype=dtype, device="cuda")
    x[:, spot] = 2.0
    ids, top = torch.full((3, 1), spot, dtype=torch.int32, device="cuda"), torch.full((3, 1), 1.0, device="cuda")
    loss, lse, grad = torch.zeros(3, device="cuda"), torch.zeros(3, device="cuda"), torch.zeros_like(x)
    rest = (V - 1) * float(torch.exp(torch.tensor(-float(gap), dtype=torch.float64)))
    for g in (None, grad):
        api.dream_distill_loss(x, ids, top, loss, lse, grad=g)
        assert float((loss.double() - rest).abs().max()) <= rest * (1 + 2 ** -20), loss.tolist()
        assert bool(((lse.double() - 2.0 - rest).abs() <= rest + 2 ** -23).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V", [60, 20000, 200000])
def test_rows_with_nan_or_infinity(V, tail, bad, dtype):
    """They have loss, lse and gradient NaN, wherever the logit stands; the rows beside them are as without them."""
    from paper_2505_19201_b200 import api
    from tests.test_gpu_distill import make
    x, ids, top, tl, scale = make(6, V, 7, dtype, seed=30, tail=tail)
    outs = []
    for hurt in (False, True):
        if hurt:
            x[1, V - 1] = bad
            x[3, ids[3, 2].long()] = bad
            x[4, 0] = bad
        loss, lse = torch.zeros(6, device="cuda"), torch.zeros(6, device="cuda")
        rest = torch.zeros(6, device="cuda") if tail else None
        step, back = torch.full_like(x, 3.0), torch.full_like(x, 3.0)
        api.dream_distill_loss(x, ids, top, loss, lse, teacher_lse=tl, log_rest=rest, row_scale=scale, grad=step)
        api.dream_distill_grad(x, ids, top, lse, back, teacher_lse=tl, log_rest=rest, row_scale=scale)
        outs.append((loss, lse, step, back))
    for a, b in zip(*outs):
        assert torch.equal(a[[0, 2, 5]], b[[0, 2, 5]])
        assert bool(torch.isnan(b[[1, 3, 4]]).all())
