"""dream_distill_loss and dream_distill_grad against the formulas in float64.

Tolerances.  An exponential of the kernel, 2^y with y = (l - max) log2(e) / tau, is off by 2^-22 (ex2.approx) and, through y, by
ln 2 * |y| * 2^-23 relative (two roundings of half a step each); terms beyond |y| = 20 hold less than 2^-20 * 2^18 of the largest term
in the widest row, so a sum of them is off by at most 2^-22 + 20 * 0.7 * 2^-23 = 1.9e-6, and adding a thread's terms (up to 128, two
roundings of 2^-24 each at worst beside the exponentials) by 1.5e-5.  lse, loss (a sum of q lse with q adding up to 1) and log_rest carry that as
an absolute error, 1.7e-5, plus half a step of their own rounding (2^-24).  A gradient's p_i is off by that, by its own exponential
(2^-22 + ln 2 |y| 2^-23 with |y| up to 40: 3.6e-6) and by roundings of its factors (three of 2^-24): 2.1e-5 relative, and the result by half
a step of its type.  A listed id's q is a float before it is taken from Q p: half a step of q, which is Q p minus the gradient, so at most
2^-24 (Q p + |gradient|) more; where an id comes k times, k such roundings and k - 1 of their sums: 3 for twice, 23 for the twelve times of one test."""
import pytest
import torch

pytestmark = pytest.mark.gpu
NEG = float("-inf")


def make(R, V, K, dtype=torch.float32, seed=0, pad=0, shift=0, tau=1.0, tail=False):
    g = torch.Generator(device="cuda").manual_seed(seed + V + K)
    t = torch.randn(R, V, device="cuda", generator=g) * 2
    t += (torch.rand(R, V, device="cuda", generator=g) < 0.01) * torch.rand(R, V, device="cuda", generator=g) * 12
    full = torch.full((R, V + pad + shift), 90.0, dtype=dtype, device="cuda")
    full[:, shift:shift + V] = t * 0.9 + torch.randn(R, V, device="cuda", generator=g) * 0.7
    top, ids = torch.topk(t, K, dim=1)
    lse = torch.logsumexp(t.double() / tau, 1).float() if tail else None
    return full[:, shift:shift + V], ids.int(), top.contiguous(), lse, torch.rand(R, device="cuda", generator=g) + 0.5


def formula(s, ids, top, teacher_lse, tau, V, lse=None, log_rest=None):
    """loss, lse, log_rest, gradient at row_scale 1; everything float64 on the CPU.  lse, log_rest: saved values to start from."""
    s, top, ids = s.double().cpu(), top.double().cpu(), ids.long().cpu()
    z = s / tau
    valid = (ids >= 0) & (ids < V)
    at = torch.where(valid, ids, 0)
    t = torch.where(valid, top / tau, NEG)
    tail = teacher_lse is not None
    if tail:
        q = torch.exp(t - teacher_lse.double().cpu()[:, None])
    else:
        m = t.amax(1, keepdim=True)
        q = torch.where(valid, torch.exp(t - torch.where(m > NEG, m, 0.0)), 0.0)
        q = q / torch.where(q.sum(1, keepdim=True) > 0, q.sum(1, keepdim=True), 1.0)
    any_ = q.sum(1) > 0
    qr = torch.where(any_, (1 - q.sum(1)).clamp(min=0.0), 0.0) if tail else torch.zeros(s.shape[0], dtype=torch.float64)
    listed = torch.zeros(s.shape, dtype=torch.float64).scatter_add_(1, at, valid.double()) > 0
    target = torch.zeros(s.shape, dtype=torch.float64).scatter_add_(1, at, torch.where(valid, q, 0.0))
    if lse is None:
        lse = torch.logsumexp(z, 1)
        log_rest = torch.logsumexp(torch.where(listed, NEG, z), 1) - lse
    else:
        lse, log_rest = lse.double().cpu(), None if log_rest is None else log_rest.double().cpu()
    p = torch.exp(z - lse[:, None])
    zt = torch.gather(z, 1, at)
    loss = torch.where(q > 0, q * (torch.log(q.clamp(min=1e-300)) - zt + lse[:, None]), 0.0).sum(1)
    total = q.sum(1) + qr
    bucket = torch.zeros_like(p)                             # q_r p_i / p_r
    if tail:
        loss = loss + torch.where(qr > 0, qr * (torch.log(qr.clamp(min=1e-300)) - log_rest), 0.0)
        bucket = torch.where((qr > 0)[:, None] & (z > NEG), qr[:, None] * torch.exp(z - (lse + log_rest)[:, None]), 0.0)
    grad = torch.where(listed, total[:, None] * p - target, total[:, None] * p - bucket) / tau
    # what an error of 1 in every p (relative) makes of it
    size = torch.where(listed, total[:, None] * p, total[:, None] * p + bucket) / tau
    return loss, lse, log_rest, grad, size


def close_rows(got, want, what):
    got, want = got.double().cpu(), want
    ok = (got == want) | ((got - want).abs() <= 1.7e-5 + want.abs() * 2 ** -24)
    assert bool(ok.all()), f"{what}: {got[~ok][:4].tolist()} {want[~ok][:4].tolist()}"


def close_grad(got, want, size, scale, dtype, q_roundings=3):
    want, size = want * scale.double().cpu()[:, None], size * scale.double().cpu()[:, None].abs()
    err = (got.double().cpu() - want).abs()
    room = 2.1e-5 * size + torch.finfo(dtype).eps / 2 * (want.abs() + 2.1e-5 * size) + q_roundings * 2 ** -24 * (size + want.abs()) + 2 ** -126
    assert bool((err <= room).all()), f"worst {float((err / room).max())} of the room"


def run_all(x, ids, top, teacher_lse, scale, tau=1.0, q_roundings=3):
    """Forward alone, forward with gradient, backward alone, the last in place; each against the formula."""
    from paper_2505_19201_b200 import api
    R, V = x.shape
    new = lambda: torch.full((R,), 5.0, device="cuda")  # noqa: E731
    rest = lambda: new() if teacher_lse is not None else None  # noqa: E731
    loss, lse, lr = new(), new(), rest()
    api.dream_distill_loss(x, ids, top, loss, lse, teacher_lse=teacher_lse, log_rest=lr, temperature=tau)
    loss2, lse2, lr2, g = new(), new(), rest(), torch.full_like(x, 3.0)
    api.dream_distill_loss(x, ids, top, loss2, lse2, teacher_lse=teacher_lse, log_rest=lr2, temperature=tau, row_scale=scale, grad=g)
    g2 = x.clone()
    api.dream_distill_grad(g2, ids, top, lse, g2, teacher_lse=teacher_lse, log_rest=lr, temperature=tau, row_scale=scale)
    g3 = x.clone()
    api.dream_distill_loss(g3, ids, top, new(), new(), teacher_lse=teacher_lse, log_rest=rest(), temperature=tau, row_scale=scale, grad=g3)
    torch.cuda.synchronize()
    a, b, c, d, size = formula(x, ids, top, teacher_lse, tau, V)
    for x1, x2, x3 in ((loss, lse, lr), (loss2, lse2, lr2)):  # the two may share a row differently among blocks
        close_rows(x1, a, "loss")
        close_rows(x2, b, "lse")
        if lr is not None:
            close_rows(x3, c, "log_rest")
    close_grad(g, d, size, scale, x.dtype, q_roundings)
    close_grad(g3, d, size, scale, x.dtype, q_roundings)
    _, _, _, d, size = formula(x, ids, top, teacher_lse, tau, V, lse, lr)
    close_grad(g2, d, size, scale, x.dtype, q_roundings)
    return loss, g, g2


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V,K", [(1, 1), (2, 1), (33, 16), (500, 128), (1024, 5), (4097, 31), (32000, 16), (32769, 128), (49155, 33)])
def test_sizes(V, K, tail, dtype):
    x, ids, top, tl, scale = make(5, V, K, dtype, seed=1, tail=tail, tau=1.0)
    run_all(x, ids, top, tl, scale)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,K,tau", [(131072, 64, 2.0), (200003, 100, 0.7), (262144, 16, 4.0)])
def test_wide_rows(V, K, tau, dtype):
    x, ids, top, tl, scale = make(3, V, K, dtype, seed=2, tail=True, tau=tau)
    run_all(x, ids, top, tl, scale, tau)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,V,K,pad,tail", [(1500, 777, 40, 0, True), (1500, 1024, 7, 0, False), (1337, 3001, 128, 3, True), (700, 20000, 16, 0, True)])
def test_more_rows_than_blocks(R, V, K, pad, tail, dtype):
    """Each block then walks several rows, the next one's copies behind the present one's; entries that are none, or come twice, among them."""
    x, ids, top, tl, scale = make(R, V, K, dtype, seed=11, pad=pad, tail=tail)
    ids[::5, -1] = ids[::5, 0]
    ids[::7, : K // 2] = -1
    ids[::11] = -1
    scale[::13] = 0.0
    if tail:
        tl += 0.7                                            # an id counted twice keeps the shares below one together
    run_all(x, ids, top, tl, scale)


@pytest.mark.parametrize("dtype,R,V", [(torch.float32, 150, 150001), (torch.float32, 130, 100000), (torch.bfloat16, 150, 200008)])
def test_more_wide_rows_than_clusters(dtype, R, V):
    x, ids, top, tl, scale = make(R, V, 32, dtype, seed=12, tail=True, tau=1.3)
    ids[::3, 5] = ids[::3, 9]
    tl += 0.7
    run_all(x, ids, top, tl, scale, 1.3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad,shift", [(1, 0), (0, 5), (8, 8), (13, 2)])
def test_strides_and_alignment(pad, shift, dtype):
    from paper_2505_19201_b200 import api
    x, ids, top, tl, scale = make(7, 5001, 20, dtype, seed=3, pad=pad, shift=shift, tail=True, tau=1.5)
    run_all(x, ids, top, tl, scale, 1.5)
    full = torch.full((7, 5020), 9.0, dtype=dtype, device="cuda")
    lse, rest = torch.zeros(7, device="cuda"), torch.zeros(7, device="cuda")
    api.dream_distill_loss(x, ids, top, torch.zeros(7, device="cuda"), lse, teacher_lse=tl, log_rest=rest, temperature=1.5, grad=full[:, 3:5004])
    assert bool((full[:, :3] == 9.0).all()) and bool((full[:, 5004:] == 9.0).all())
    full.fill_(9.0)
    api.dream_distill_grad(x, ids, top, lse, full[:, 3:5004], teacher_lse=tl, log_rest=rest, temperature=1.5)
    assert bool((full[:, :3] == 9.0).all()) and bool((full[:, 5004:] == 9.0).all())


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V", [300, 40000])
def test_entries_that_are_none_or_come_twice(V, tail):
    x, ids, top, tl, scale = make(6, V, 12, seed=4, tail=tail)
    ids[0, 3:] = -1                                          # a short list
    ids[1, ::2] = V                                          # ids outside the vocabulary
    ids[2] = -1                                              # nothing: loss 0, gradient 0
    ids[3, 5] = ids[3, 0]                                    # one id twice
    ids[4, :] = ids[4, 0]                                    # one id in every place
    if tail:
        top[4] = top[4, 0] - 2.5                             # twelve shares of one id, less than one together
    top[5, 2:7] = NEG                                        # entries without mass
    loss, g, g2 = run_all(x, ids, top, tl, scale, q_roundings=23)
    assert float(loss[2]) == 0.0 and not bool(g[2].any()) and not bool(g2[2].any())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masked_logits_and_padding_rows(dtype):
    from paper_2505_19201_b200 import api
    V = 9001
    x, ids, top, tl, scale = make(6, V, 8, dtype, seed=5, tail=True)
    keep = torch.zeros(6, V, dtype=torch.bool, device="cuda").scatter_(1, ids.long(), True)
    x[0] = torch.where(keep[0] | (torch.arange(V, device="cuda") % 3 == 0), x[0], NEG)      # masked logits, none of them listed
    x[1] = torch.where(keep[1] | (torch.arange(V, device="cuda") % 5 == 0), x[1], torch.finfo(dtype).min)
    run_all(x[:2], ids[:2], top[:2], tl[:2], scale[:2])
    x[2] = NEG                                               # nothing finite
    x[3] = float("nan")                                      # rows of padding: whatever they hold
    x[4, ::2] = float("inf")
    scale[3:] = 0.0
    loss, lse, lr, g = (torch.zeros(6, device="cuda") for _ in range(3)), None, None, torch.full_like(x, 2.0)
    loss, lse, lr = loss
    api.dream_distill_loss(x, ids, top, loss, lse, teacher_lse=tl, log_rest=lr, row_scale=scale, grad=g)
    g2 = torch.full_like(x, 2.0)
    api.dream_distill_grad(x, ids, top, lse, g2, teacher_lse=tl, log_rest=lr, row_scale=scale)
    torch.cuda.synchronize()
    assert float(loss[2]) == float("inf") and float(lse[2]) == NEG
    assert bool(torch.isnan(loss[3]))
    for t in (g, g2):
        assert bool((t[2:] == 0).all())
        assert bool(torch.isfinite(t[:2].float()).all())


def test_a_listed_id_that_the_student_masks():
    """Where the student gives a listed id no mass the loss is infinite; without weight on it, it is not."""
    x, ids, top, _, scale = make(2, 700, 6, seed=6)
    x[0, ids[0, 1].long()] = NEG
    x[1, ids[1, 1].long()] = NEG
    top[1, 1] = NEG
    loss, g, g2 = run_all(x, ids, top, None, scale)
    assert float(loss[0]) == float("inf") and float(loss[1]) < 100


def test_everything_listed():
    """All of a small vocabulary in the list: nothing is left for the rest."""
    x, ids, top, tl, scale = make(4, 40, 40, seed=7, tail=True)
    from paper_2505_19201_b200 import api
    tl = tl - 1e-3                                           # the shares add up to a little over one: q_r is 0
    loss, lse, lr, g = torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros_like(x)
    api.dream_distill_loss(x, ids, top, loss, lse, teacher_lse=tl, log_rest=lr, row_scale=scale, grad=g)
    a, b, c, d, size = formula(x, ids, top, tl, 1.0, 40)
    close_rows(loss, a, "loss")
    assert bool((lr == NEG).all())
    close_grad(g, d, size, scale, x.dtype)


def test_a_sure_student_keeps_the_rest_exact():
    """Listed ids with all but 1e-9 of the mass: the rest is a sum of its own, not a difference."""
    x, ids, top, tl, scale = make(3, 20000, 4, seed=8, tail=True)
    x.scatter_(1, ids.long(), 35.0)
    run_all(x, ids, top, tl, scale)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,tau", [(5000, 1.0), (5000, 0.01), (150001, 0.3)])
@pytest.mark.parametrize("gap", [-3000.0, -95.0, 40.0, 95.0, 400.0, 3000.0])
def test_listed_ids_far_from_the_others(gap, V, tau, dtype):
    """Between the listed ids and the others lie `gap` units of the temperature, more than a float's exponential reaches.  The loss may be off by
    more than elsewhere: the student's 1 / tau is a float's, off by 2^-24, which changes it by 2^-24 of |sum (p - q) z / tau|, at most
    loss + 2 ln V (loss = sum q ln q + H(p) + sum (p - q) z / tau): 2^-24 (|loss| + 25), beside the 1.7e-5 and half a step of its own.
    A gradient's p_i are off by as much as elsewhere, each group's being taken relative to its own largest; ids that are `gap` below the
    other group have next to no p (2^-24 * 95 = 5.7e-6 of e^-95)."""
    from paper_2505_19201_b200 import api
    R, K = 3, 8
    g = torch.Generator(device="cuda").manual_seed(5)
    x = (torch.randn(R, V, device="cuda", generator=g) * tau).to(dtype)
    ids = torch.stack([torch.randperm(V, device="cuda", generator=g)[:K] for _ in range(R)]).int()
    x.scatter_add_(1, ids.long(), torch.full((R, K), gap * tau, device="cuda").to(dtype))
    top = torch.randn(R, K, device="cuda", generator=g) * tau
    tl = (torch.logsumexp(top.double() / tau, 1) + torch.tensor([0.3, 1.0, 3.0], device="cuda", dtype=torch.float64)).float()
    scale = torch.rand(R, device="cuda", generator=g) + 0.5
    out = [torch.full((R,), 5.0, device="cuda") for _ in range(3)]
    grad = torch.full_like(x, 3.0)
    api.dream_distill_loss(x, ids, top, out[0], out[1], teacher_lse=tl, log_rest=out[2], temperature=tau, row_scale=scale, grad=grad)
    back = torch.full_like(x, 3.0)
    api.dream_distill_grad(x, ids, top, out[1], back, teacher_lse=tl, log_rest=out[2], temperature=tau, row_scale=scale)
    tau = float(torch.tensor(tau, dtype=torch.float32))      # as the call has it
    loss, lse, log_rest, want, size = formula(x, ids, top, tl, tau, V)
    assert bool(((out[0].double().cpu() - loss).abs() <= 1.7e-5 + 2 ** -24 * (2 * loss.abs() + 25)).all())
    close_rows(out[1], lse, "lse")
    close_rows(out[2], log_rest, "log_rest")
    close_grad(grad, want, size, scale, dtype)
    # the separate call starts from the rounded lse and log_rest
    _, _, _, want, size = formula(x, ids, top, tl, tau, V, out[1], out[2])
    close_grad(back, want, size, scale, dtype)


@pytest.mark.parametrize("tail", [False, True])
def test_gradient_against_differences(tail):
    """Central differences of the kernel's own loss.  Step h = 0.05: the third derivative of the loss in one logit is below 0.2 where q_r / p_r
    is below 2, so the truncation is below h^2 / 6 * 0.2 = 9e-5; the loss's error on either side, 1.7e-5 of which all but the changed
    logit's own share is the same on both sides, gives at most 2 * 1.7e-5 / (2 h) = 3.4e-4."""
    from paper_2505_19201_b200 import api
    V, K, h = 400, 6, 0.05
    x, ids, top, tl, _ = make(1, V, K, seed=9, tail=tail)
    x = (x * 0.3).contiguous()
    pick = ids[0].tolist() + [i for i in (0, 1, 50, 399) if i not in ids[0].tolist()]
    many = x.repeat(2 * len(pick), 1)
    for i, t in enumerate(pick):
        many[2 * i, t] += h
        many[2 * i + 1, t] -= h
    n = many.shape[0]
    new = lambda k: torch.zeros(k, device="cuda")  # noqa: E731
    rep = lambda v: None if v is None else v.repeat(n, *([1] * (v.dim() - 1)))  # noqa: E731
    loss, g = new(n), torch.zeros_like(x)
    api.dream_distill_loss(many, rep(ids), rep(top), loss, new(n), teacher_lse=rep(tl), log_rest=new(n) if tail else None)
    api.dream_distill_loss(x, ids, top, new(1), new(1), teacher_lse=tl, log_rest=new(1) if tail else None, grad=g)
    for i, t in enumerate(pick):
        step = float(many[2 * i, t] - many[2 * i + 1, t])
        slope = float(loss[2 * i].double() - loss[2 * i + 1].double()) / step
        assert abs(slope - float(g[0, t])) <= 9e-5 + 3.4e-4, (t, slope, float(g[0, t]))


def test_same_bits_in_a_graph_and_on_two_streams():
    from paper_2505_19201_b200 import api
    x, ids, top, tl, scale = make(30, 70001, 40, torch.bfloat16, seed=10, tail=True)
    ids[:, 7] = ids[:, 3]

    def go():
        o = [torch.zeros(30, device="cuda") for _ in range(3)] + [torch.zeros_like(x)]
        return o, lambda: api.dream_distill_loss(x, ids, top, o[0], o[1], teacher_lse=tl, log_rest=o[2], row_scale=scale, grad=o[3])
    first, call = go()
    call()
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        o, call = go()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            call()
        graphs.append(gr)
        outs.append(o)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        for s, gr in zip(streams, graphs):
            with torch.cuda.stream(s):
                gr.replay()
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(a, b) for a, b in zip(first, o))


def test_teacher_from_the_top_k_call_trains_a_row():
    """dream_topk_lse_static makes the teacher's side, dream_distill_loss the gradient; a student that takes steps along it comes to agree
    with the teacher's listed probabilities: its gradient goes to zero where the formula says it does (p = q)."""
    from paper_2505_19201_b200 import api
    V, K, R = 2000, 16, 9
    g = torch.Generator(device="cuda").manual_seed(3)
    t = torch.randn(R, V, device="cuda", generator=g) * 2
    t[:, :30] += torch.rand(R, 30, device="cuda", generator=g) * 8
    tv, ti, tl = torch.zeros(R, K, device="cuda"), torch.zeros(R, K, dtype=torch.int32, device="cuda"), torch.zeros(R, device="cuda")
    api.dream_topk_lse_static(t, K, tv, ti, tl)
    loss, lse, lr, grad = (torch.zeros(R, device="cuda") for _ in range(3)), None, None, torch.ones(R, V, device="cuda")
    loss, lse, lr = loss
    api.dream_distill_loss(t, ti, tv, loss, lse, teacher_lse=tl, log_rest=lr, grad=grad)
    assert float(loss.abs().max()) <= 1.7e-5 + 1e-5          # the student is the teacher; dream_topk_lse_static's lse is good to some 1e-5
    assert float(grad.abs().max()) <= 4e-5
