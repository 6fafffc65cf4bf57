"""Rows and settings at which dream_sample and dream_truncate_logits could go wrong by a rounding, against the definition in float64.  Tokens,
kept counts and kept sets are equal, not close; logprob within what tests/test_gpu_sample.py derives."""
import decimal
import fractions
import math

import pytest
import torch

from tests.test_gpu_sample import U, check, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V,t,sigma", [(262144, 1.3, 2.0), (131072, 1.2, 1.0), (200000, 0.7, 0.7), (262144, 1.5, 2.0), (131072, 1.3, 1.0)])
def test_depths_that_round_up_to_a_bins_edge(V, t, sigma):
    """(max - l) * 128 / T, rounded, is an integer that the exact product does not reach: a token on the edge of a bin too full to be listed.  The cut
    falls behind it in that bin, so counting it twice or not at all would move the cut."""
    x, scale, k = None, torch.tensor(128.0) / torch.tensor(t), []
    for seed in range(40):
        one = torch.randn(V, generator=torch.Generator().manual_seed(seed)) * sigma
        d = one.max() - one
        rounded, product = d * scale, d.double() * scale.double()
        count = torch.bincount(rounded.floor().clamp(max=2047).long(), minlength=2048)
        edge = (rounded.floor().double() > product.floor()) & (rounded < 2047)
        k = [int(count[:b].sum() + count[b] // 2) for b in rounded[edge].floor().long().tolist() if count[b] > 412]
        x = one if k else x
        if k:
            break
    assert k
    k = k[:5]
    check(x.cuda().expand(len(k), V).contiguous(), U[:len(k)], t=[t] * len(k), k=k)


@pytest.mark.parametrize("t", [0.7, 1.3, 1.5])
@pytest.mark.parametrize("V", [131072, 262144])
def test_many_kept_at_a_temperature(V, t):
    g = torch.Generator().manual_seed(V)
    for seed in range(4):
        check(rows(8, V, seed=seed, sigma=1.0), [0.05, 0.3, 0.5, 0.6, 0.7, 0.8, 0.9, 0.99], t=[t] * 8,
              k=torch.randint(300, V * 3 // 4, (8,), generator=g).tolist())


@pytest.mark.parametrize("t", [1e-4, 1e-6, 2e-9, 1e-10, 1e-12, 1e-15])
@pytest.mark.parametrize("m", [3.7, 20.0, 3000.0, -3.7, 1e6])
def test_neighbouring_floats_at_low_temperatures(m, t):
    """A step of a float below the largest logit may be a thousand temperatures and more."""
    V = 20000
    x = torch.minimum(rows(5, V, seed=20), torch.tensor(m - 1.0, device="cuda")).contiguous()
    top = torch.tensor(m)
    next_ = torch.nextafter(top, torch.tensor(-1e9))
    for i, at in enumerate((3, 700, 9000, 15000, 19999)):
        x[:, at] = next_ if i % 2 == 0 else top
        x[i, at] = top if i < 3 else next_
    x[3, 4000:4600] = next_
    for s in ({}, dict(k=[1, 2, 3, 50, 4]), dict(k=[300, 1000, 5000, 400, 19000]), dict(p=[0.1, 0.4, 0.7, 0.9, 0.999]), dict(mp=[0.9, 0.5, 0.1, 0.01, 1e-6])):
        check(x, [0.05, 0.3, 0.6, 0.85, 0.99], t=[t] * 5, **s)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [400, 1074, 3704, 20000, 70002, 200000])
@pytest.mark.parametrize("min_p", [None, 0.2])
@pytest.mark.parametrize("mirrored", [False, True])
def test_goal_on_a_border(mirrored, min_p, V, dtype):
    """Rows of two halves with the same weights and u = 1 / 2: the goal is the border between them to a rounding, so the token is the last of the first
    half or the first of the second; it is written, and the same at every run."""
    from paper_2505_19201_b200 import api
    R, h = 96, V // 2
    g = torch.Generator().manual_seed(V)
    half = torch.where(torch.rand(R, h, generator=g) < torch.rand(R, 1, generator=g) * 0.3, torch.rand(R, h, generator=g) * -3.0, float("-inf"))
    half[:, h // 2:] = float("-inf")                          # whole warps without a token between the halves
    half[:, 0] = 0.0
    x = torch.cat([half, half.flip(1) if mirrored else half], 1).to(dtype).cuda()
    u = torch.full((R,), 0.5, device="cuda")
    mp = None if min_p is None else torch.full((R,), min_p, device="cuda")
    out = []
    for _ in range(2):
        tok, lp = torch.full((R,), -9, dtype=torch.int32, device="cuda"), torch.full((R,), 9.0, device="cuda")
        api.dream_sample(x, u, tok, min_p=mp, logprob=lp)
        out.append((tok.tolist(), lp.tolist()))
    assert out[0] == out[1]
    w = torch.exp(x.cpu().double())
    w = torch.where(w >= (min_p or 0.0), w, 0.0)
    for r in range(R):
        ids = w[r].nonzero()[:, 0]
        at = ids.numel() // 2
        tok, lp = out[0][0][r], out[0][1][r]
        assert tok in (int(ids[at - 1]), int(ids[at])), (r, tok)
        want = float(torch.log(w[r, tok] / w[r].sum()))
        assert abs(lp - want) <= abs(want) * 2 ** -24 + 1e-10


def test_cut_at_the_first_of_the_finer_bins():
    """Hundreds of thousands of ties whose approximate mass falls short by a token's weight, a few tokens just in front of a bin's edge, one behind it in
    which the cut falls, and a full bin after: the first look takes the bin after, and the finer bins' first is where the cut is."""
    import numpy as np
    V, step = 262144, np.float32(-1.0 / 128.0)
    tie = np.float32(-0.78850514)                              # 100.93 bins below the largest: there 2^-17 rounds down the most, by 3.8e-6
    x, p = np.full((9, V), -np.inf, np.float32), []
    for r in range(9):
        n = (240000, 255000, 261000)[r // 3]
        row = np.concatenate([[0.0], np.full(n, tie), [step * (128 - 0.0004 - 0.00005 * j) for j in range(10)], [step * 128.0005],
                              [step * (129.1 + 0.003 * j) for j in range(200)]]).astype(np.float32)
        w = np.exp(row.astype(np.float64))
        p.append((w[:n + 11].sum() + (0.2, 0.5, 0.8)[r % 3] * w[n + 11]) / w.sum())
        x[r, :row.size] = np.roll(row, 1000 * r)
    check(torch.from_numpy(x).cuda(), [0.0, 0.3, 0.5, 0.9, 0.99, 0.1, 0.2, 0.7, 0.8], p=p)


def _exp(x):
    """e^x as a fraction, to 60 digits."""
    with decimal.localcontext() as c:
        c.prec = 60
        return fractions.Fraction(decimal.Decimal(x).exp())


@pytest.mark.parametrize("V", [131072, 200001, 262144])
@pytest.mark.parametrize("gap,p", [(22, 0.99999), (25, 0.999999), (25, 0.99999994), (19, 0.9999)])
def test_cut_in_a_far_tail(gap, p, V):
    """One logit and V - 1 ties far below it that hold little of the mass: r tokens stay where 1 + (r - 2) w < p Z <= 1 + (r - 1) w, all of it in
    fractions.  The kernel's p Z - 1 may be off by 2e-12 of the mass (half of the borders' room below)."""
    from paper_2505_19201_b200 import api
    p = float(torch.tensor(p))
    w, P = _exp(-gap), fractions.Fraction(p)
    Z = 1 + (V - 1) * w
    room = fractions.Fraction(4, 10 ** 12) * Z / w
    at = (P * Z - 1) / w
    kept = 1 + max(0, math.ceil(at))
    assert 1 < kept < V
    x = torch.zeros(2, V, device="cuda")
    x[0, V // 3] = x[1, V - 1] = float(gap)
    n, out, n2 = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros_like(x), torch.zeros(2, dtype=torch.int32, device="cuda")
    tok = torch.zeros(2, dtype=torch.int32, device="cuda")
    top_p = torch.full((2,), p, device="cuda")
    api.dream_sample(x, torch.full((2,), 0.5, device="cuda"), tok, top_p=top_p, kept=n)
    api.dream_truncate_logits(x, out, top_p=top_p, kept=n2)
    assert n.tolist() == n2.tolist() and tok.tolist() == [V // 3, V - 1]
    for r in range(2):
        assert abs(int(n[r]) - kept) <= math.ceil(room), (int(n[r]), kept)
        ids = (out[r] > float("-inf")).nonzero()[:, 0].tolist()
        big = tok.tolist()[r]
        assert ids == sorted([big] + [i for i in range(int(n[r])) if i != big][:int(n[r]) - 1])


@pytest.mark.parametrize("k", [None, 200000])
@pytest.mark.parametrize("gap,u", [(32, 1e-9), (32, 3e-9), (28, 1e-9), (40, 5e-13), (60, 1e-21)])
def test_draw_from_a_far_tail(gap, u, k):
    """The largest logit is the last id, so a small enough u falls among the ties in front of it: token floor(u Z / w).  (Where
    fewer stay than that, the goal lies in the last one's own weight.)  Sums in double of at most
    2^18 terms, a thread's 128 in turn: the token's place is good to 1e-12 of itself for the weights and 2^-53 (128 + 16 + 5 + 16) for the sums."""
    from paper_2505_19201_b200 import api
    V = 262144
    u = float(torch.tensor(u))
    n = (k or V) - 1                                           # ties that stay: the first of them
    w = _exp(-gap)
    place = fractions.Fraction(u) * (1 + n * w) / w
    want = math.floor(place) if place < n else V - 1
    assert 1e-6 < place % 1 < 1 - 1e-6
    x = torch.zeros(3, V, device="cuda")
    x[:, V - 1] = float(gap)
    tok = torch.zeros(3, dtype=torch.int32, device="cuda")
    tk = None if k is None else torch.full((3,), k, dtype=torch.int32, device="cuda")
    api.dream_sample(x, torch.full((3,), u, device="cuda"), tok, top_k=tk)
    assert tok.tolist() == [want] * 3


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [40, 33000])
def test_min_p_at_an_infinite_temperature(V, dtype):
    """Every finite logit weighs 1 there, so min_p up to 1 cuts nothing; beside +inf nothing weighs anything."""
    x = rows(6, V, dtype, seed=21).clone()
    x[3, ::2] = float("-inf")
    x[4] = float("-inf")
    x[5, 3] = float("inf")
    inf = float("inf")
    for s in ({}, dict(k=[30, 300, 10, 0, 5, 9]), dict(p=[0.3, 0.9, 0.999, 0.5, 0.5, 0.5])):
        check(x, [0.1, 0.4, 0.8, 0.5, 0.3, 0.7], t=[inf] * 6, mp=[1.0, 0.3, 1.0, 1.0, 1.0, 1.0], **s)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [40, 33000])
def test_the_smallest_draw_beside_infinities(V, dtype):
    """u = 0 takes the first token with mass, which finite logits have none of where one is +inf, the type's largest value and any temperature included."""
    inf = float("inf")
    x = rows(5, V, dtype, seed=22).clone()
    x[:, 1] = torch.finfo(dtype).max
    x[:, V // 2] = x[:, V - 1] = inf
    for s in ({}, dict(k=[1, 2, 5, 30, 300]), dict(k=[10] * 5, mp=[0.5] * 5), dict(p=[0.4, 0.5, 0.6, 0.9, 0.999])):
        check(x, [0.0] * 5, t=[1.0, 1e30, 1e36, 3e38, inf], **s)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [300, 32000, 131072])
def test_top_k_on_both_sides_of_the_short_list(V, dtype):
    k = [1, 111, 112, 113, 127, 128, 129, 255, 256, 257]
    x, u = rows(10, V, dtype, seed=23), [0.05, 0.2, 0.3, 0.4, 0.5, 0.6, 0.7, 0.8, 0.9, 0.97]
    check(x, u, k=k)
    check(x, u, k=k, t=[0.7] * 10, p=[0.9] * 10, mp=[0.01] * 10)
