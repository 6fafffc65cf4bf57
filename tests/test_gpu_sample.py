"""dream_sample and dream_truncate_logits against the definition in float64: tokens, kept counts and kept sets are equal, not close.
A token could only differ where a uniform number, or top_p, falls within some 1e-11 of a border of the running sum (what weights good to
3e-13 and a unit of 2^-44 leave), which none of these fixed inputs does.  logprob is a float: half a step of its own rounding, plus the
same 1e-11."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
NEG = float("-inf")


def kept_ids(x, t, k, p, mp):
    """Kept ids in the order (logit descending, id ascending), weights of all tokens; x: float64 [V]."""
    V = x.numel()
    if not t > 0:
        t, k = 1.0, 1
    ok = x > NEG
    if not bool(ok.any()):
        return torch.empty(0, dtype=torch.long), torch.zeros(V, dtype=torch.float64)
    m = x[ok].max()
    w = torch.where(x == m, 1.0, torch.exp((x - m) / t) if m < math.inf else 0.0)
    w = torch.where(ok, w, 0.0).double()
    order = torch.sort(torch.where(ok, x, NEG), descending=True, stable=True).indices[:int(ok.sum())]
    if 0 < k < V:
        order = order[:k]
    n = order.numel()
    if p < 1:
        run = torch.cumsum(w[order], 0)
        n = min(n, int((run - w[order] < p * run[-1]).sum()))
    if mp > 0:
        n = min(n, int((w[order] >= mp).sum()))
    return order[:max(n, 1)], w


def reference(x, u, t, k, p, mp):
    ids, w = kept_ids(x, t, k, p, mp)
    if ids.numel() == 0:
        return -1, NEG, 0, ids
    s = torch.sort(ids).values
    run = torch.cumsum(w[s], 0)
    i = min(int((run <= u * run[-1]).sum()), s.numel() - 1)
    while i > 0 and w[s[i]] == 0:
        i -= 1
    return int(s[i]), float(torch.log(w[s[i]] / run[-1])), ids.numel(), ids


def check(x, u, t=None, k=None, p=None, mp=None, sample=True, truncate=True):
    """x: CUDA [R, V]; the settings are lists by row, or None."""
    from paper_2505_19201_b200 import api
    R, V = x.shape
    dev = x.device
    f = lambda v: None if v is None else torch.tensor(v, dtype=torch.float32, device=dev)  # noqa: E731
    st = dict(temperature=f(t), top_k=None if k is None else torch.tensor(k, dtype=torch.int32, device=dev), top_p=f(p), min_p=f(mp))
    uni = torch.tensor(u, dtype=torch.float32, device=dev)
    tok, lp = torch.full((R,), -9, dtype=torch.int32, device=dev), torch.full((R,), 9.0, device=dev)
    n1, n2 = torch.full((R,), -9, dtype=torch.int32, device=dev), torch.full((R,), -9, dtype=torch.int32, device=dev)
    out = torch.full_like(x, 7.0)
    api.dream_sample(x, uni, tok, logprob=lp, kept=n1, **st)
    api.dream_truncate_logits(x, out, kept=n2, **st)
    torch.cuda.synchronize()
    at = lambda name, r, off: off if st[name] is None else st[name][r].item()  # noqa: E731
    xc, oc = x.float().cpu().double(), out.float().cpu().double()
    for r in range(R):
        token, logprob, kept, ids = reference(xc[r], float(uni[r]), at("temperature", r, 1.0), at("top_k", r, 0), at("top_p", r, 1.0),
                                              at("min_p", r, 0.0))
        assert (int(n1[r]), int(n2[r])) == (kept, kept), f"row {r}: kept"
        assert int(tok[r]) == token, f"row {r}: token"
        got = float(lp[r])
        assert got == logprob or abs(got - logprob) <= abs(logprob) * 2 ** -24 + 1e-10, f"row {r}: logprob {got} {logprob}"
        want = torch.full((V,), NEG, dtype=torch.float64)
        want[ids] = xc[r][ids]
        assert torch.equal(oc[r], want), f"row {r}: truncated row"


def rows(R, V, dtype=torch.float32, seed=0, pad=0, sigma=2.0, shift=0):
    g = torch.Generator(device="cuda").manual_seed(seed + V)
    x = torch.randn(R, V, device="cuda", generator=g) * sigma
    x += (torch.rand(R, V, device="cuda", generator=g) < 0.003) * torch.rand(R, V, device="cuda", generator=g) * 14
    full = torch.full((R, V + pad + shift), 50.0, dtype=dtype, device="cuda")       # what lies between rows would win if it were read
    full[:, shift:shift + V] = x
    return full[:, shift:shift + V]


U = [0.0, 0.137, 0.5, 0.9, 0.99999994]
SETTINGS = {
    "plain": {},
    "temperature": dict(t=[0.3, 0.7, 1.0, 1.5, 4.0]),
    "top_k": dict(k=[1, 2, 7, 50, 300]),
    "top_p": dict(p=[0.1, 0.5, 0.9, 0.95, 0.999]),
    "min_p": dict(mp=[0.001, 0.05, 0.3, 1.0, 2.0]),
    "all": dict(t=[0.6, 0.8, 1.0, 1.2, 0.0], k=[20, 50, 1000, 5, 40], p=[0.9, 0.95, 0.8, 0.5, 0.9], mp=[0.02, 0.0, 0.01, 0.1, 0.05]),
}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 31, 127, 500, 1024, 4097, 32000, 32769, 65536])
@pytest.mark.parametrize("name", SETTINGS)
def test_settings_and_sizes(name, V, dtype):
    check(rows(5, V, dtype, seed=3), U, **SETTINGS[name])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [131072, 200001, 262144])
@pytest.mark.parametrize("name", ["temperature", "top_p", "all"])
def test_wide_rows(name, V, dtype):
    check(rows(5, V, dtype, seed=4), U, **SETTINGS[name])


@pytest.mark.parametrize("name", ["top_k", "top_p"])
@pytest.mark.parametrize("V", [9000, 150000])
def test_many_kept(name, V):
    """Cuts deep in the bulk of the row, where bins are full."""
    k = [V - 1, V // 2, V, V + 5, 5000]
    check(rows(5, V, seed=5, sigma=1.0), U, **(dict(k=k) if name == "top_k" else dict(p=[0.99, 0.7, 0.999, 0.3, 0.9999], k=k)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad,shift", [(1, 0), (0, 3), (8, 8), (37, 1)])
def test_strides_and_alignment(pad, shift, dtype):
    check(rows(5, 4100, dtype, seed=6, pad=pad, shift=shift), U, **SETTINGS["all"])


@pytest.mark.parametrize("V", [64, 5000, 70000])
def test_ties_take_the_lower_id(V):
    x = torch.randint(-2, 3, (5, V), device="cuda", generator=torch.Generator(device="cuda").manual_seed(V)).float()
    x[1] = 0.0
    x[1, ::3] = -0.0
    x[2] = -7.25
    check(x, U, k=[3, 17, 40, 50, 60])
    check(x, U, p=[0.3, 0.5, 0.25, 0.75, 0.9])
    check(x, U, k=[V - 3, V // 2, V - 1, 33, 20], p=[0.5, 0.5, 0.5, 0.5, 0.999])
    check(x, U)


@pytest.mark.parametrize("V", [40, 33000])
def test_masked_rows(V):
    """-inf, NaN, the type's lowest value and +inf in a row; a row that masks leave empty; one token left."""
    x = rows(8, V, seed=8).clone()
    low = torch.finfo(torch.float32).min
    x[0, ::2] = NEG
    x[1, 1::2] = low
    x[2, ::3] = float("nan")
    x[3] = NEG
    x[4] = NEG
    x[4, V - 1] = -3.0
    x[5, 7] = x[5, V - 2] = float("inf")
    x[6] = low
    x[7] = float("nan")
    u = [0.1, 0.5, 0.999, 0.5, 0.5, 0.6, 0.3, 0.5]
    check(x, u)
    check(x, u, k=[9] * 8, p=[0.8] * 8)
    check(x, u, p=[0.8] * 8)
    check(x, u, mp=[0.1] * 8)
    check(x, u, t=[0.0] * 8)


def test_extreme_settings():
    x = rows(8, 3001, seed=9)
    u = [0.2, 0.4, 0.6, 0.8, 0.1, 0.3, 0.5, 0.7]
    nan, inf = float("nan"), float("inf")
    check(x, u, t=[1e-30, 1e-3, 1e3, 1e30, inf, -1.0, 1e-45, 3e38])
    check(x, u, p=[0.0, -1.0, 1.0, 2.0, 1e-9, 0.5, 0.5, 0.99], k=[0, -5, 2 ** 31 - 1, 3001, 3000, 1, 2, 10])
    # NaN reads as off, as temperature 0 for a temperature; uniforms outside [0, 1) go to the nearer end
    check(x, [0.0, 0.0, 0.99999994, 0.5, 0.5, 0.5, 0.5, 0.5], mp=[1e-30, 1e30, 0.5, 0.1, -1.0, 0.0, 1.0, 0.9])
    from paper_2505_19201_b200 import api
    t = torch.tensor([nan] + [1.0] * 7, device="cuda")
    uu = torch.tensor([0.3, -1.0, nan, 1.0, 7.0, 0.5, 0.5, 0.5], device="cuda")
    off = torch.full((8,), nan, device="cuda")
    tok = torch.zeros(8, dtype=torch.int32, device="cuda")
    api.dream_sample(x, uu, tok, temperature=t, top_p=off, min_p=off)
    want = [reference(x[r].cpu().double(), v, 0.0 if r == 0 else 1.0, 0, 1.0, 0.0)[0]
            for r, v in enumerate([0.3, 0.0, 0.0, 1.0, 1.0, 0.5, 0.5, 0.5])]
    assert tok.tolist() == want


def test_draws_follow_the_distribution():
    """20000 draws from one row: each kept token's share within 4.5 standard deviations, no other token."""
    from paper_2505_19201_b200 import api
    n, V = 20000, 1000
    g = torch.Generator(device="cuda").manual_seed(1)
    x = rows(1, V, seed=10, sigma=1.5)
    many = x.expand(n, V).contiguous()
    tok = torch.zeros(n, dtype=torch.int32, device="cuda")
    api.dream_sample(many, torch.rand(n, device="cuda", generator=g), tok, top_k=torch.full((n,), 12, dtype=torch.int32, device="cuda"))
    ids, w = kept_ids(x[0].cpu().double(), 1.0, 12, 1.0, 0.0)
    prob = w[ids] / w[ids].sum()
    share = torch.bincount(tok.cpu().long(), minlength=V).double() / n
    assert float(share[ids].sum()) == pytest.approx(1.0, abs=1e-12)
    assert bool(((share[ids] - prob).abs() <= 4.5 * torch.sqrt(prob * (1 - prob) / n)).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_truncate_in_place_and_between_rows(dtype):
    from paper_2505_19201_b200 import api
    x = rows(6, 5003, dtype, seed=11, pad=5)
    full = x._base if x._base is not None else x
    k = torch.full((6,), 33, dtype=torch.int32, device="cuda")
    out = torch.full((6, 5010), 9.0, dtype=dtype, device="cuda")
    api.dream_truncate_logits(x, out[:, 2:5005], top_k=k)
    assert bool((out[:, :2] == 9.0).all()) and bool((out[:, 5005:] == 9.0).all())
    api.dream_truncate_logits(x, x, top_k=k)
    assert torch.equal(x, out[:, 2:5005])
    assert int((x > NEG).sum()) == 6 * 33
    assert bool((full[:, 5003:] == 50.0).all())


def test_same_bits_at_every_run_and_in_a_graph():
    from paper_2505_19201_b200 import api
    x = rows(40, 40000, torch.bfloat16, seed=12)
    u = torch.rand(40, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    p, t = torch.full((40,), 0.97, device="cuda"), torch.full((40,), 0.9, device="cuda")

    def go():
        tok, lp, n = torch.zeros(40, dtype=torch.int32, device="cuda"), torch.zeros(40, device="cuda"), torch.zeros(40, dtype=torch.int32, device="cuda")
        return (tok, lp, n), lambda: api.dream_sample(x, u, tok, temperature=t, top_p=p, logprob=lp, kept=n)
    first, call = go()
    call()
    torch.cuda.synchronize()
    # two graphs on streams of their own, replayed together
    graphs, outs = [], []
    for _ in range(2):
        o, call = go()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            call()
        graphs.append(gr)
        outs.append(o)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, gr in zip(streams, graphs):
            with torch.cuda.stream(s):
                gr.replay()
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(a, b) for a, b in zip(first, o))
    # new numbers in the same buffers: the graph sees them
    u.fill_(0.0)
    graphs[0].replay()
    torch.cuda.synchronize()
    ref, call = go()
    call()
    torch.cuda.synchronize()
    assert torch.equal(ref[0], outs[0][0])


def test_on_a_stream_behind_its_inputs():
    """The call waits for the work that makes its inputs on the stream it is given, and nothing else."""
    from paper_2505_19201_b200 import api
    s = torch.cuda.Stream()
    src = rows(16, 20000, seed=13)
    x = torch.zeros_like(src)
    tok, u = torch.zeros(16, dtype=torch.int32, device="cuda"), torch.full((16,), 0.4, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(20):
            x.copy_(src * 0.5 + src * 0.5)
        api.dream_sample(x, u, tok)
        again = tok.clone()
    s.synchronize()
    assert again.tolist() == [reference(src[r].cpu().double(), float(u[0]), 1.0, 0, 1.0, 0.0)[0] for r in range(16)]
