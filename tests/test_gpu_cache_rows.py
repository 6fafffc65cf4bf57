"""Appending to a paged cache of the caller's own, its bounds, and the pages that are selected by them."""
import random

import pytest
import torch

from .util_cache import HALF, NAN, TYPES, Pages, pools

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def angles(n, rot, theta=10000.0):
    p = torch.arange(n, dtype=torch.float64, device="cuda")[:, None]
    return p * theta ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device="cuda") / rot)


def table(n, rot, theta=10000.0):
    from paper_2505_19201_b200 import api
    t = torch.full((n, rot // 2, 2), NAN, device="cuda")
    api.dream_rope_table(t, theta)
    return t


def turned(x, pos, rot, interleaved, theta=10000.0):
    """In 64 bits, and what a rounding of the factors and of three operations in 32 bits may do."""
    x = x.double().clone()
    if not rot:
        return x, torch.zeros_like(x)
    a = angles(max(pos) + 1, rot, theta)[torch.tensor(pos, device="cuda")][:, None]
    one, two = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    p, q = x[..., one].clone(), x[..., two].clone()
    x[..., one], x[..., two] = p * torch.cos(a) - q * torch.sin(a), q * torch.cos(a) + p * torch.sin(a)
    slack = torch.zeros_like(x)
    slack[..., one] = slack[..., two] = 2.0 ** -20 * (p.abs() + q.abs())
    return x, slack


def near(got, want, slack, dtype):
    err = (got.double() - want).abs()
    assert (err <= HALF[dtype] * want.abs() * (1 + 1e-6) + slack * (1 + HALF[dtype]) + torch.finfo(TYPES[dtype]).tiny).all()


@pytest.mark.parametrize("n,rot,theta", [(1, 16, 1e4), (5, 64, 1e4), (1000, 128, 5e5), (131072, 128, 1e4), (70, 256, 1e6), (40, 48, 1e4)])
def test_rope_table(n, rot, theta):
    t, a = table(n, rot, theta).double(), angles(n, rot, theta)
    # the reduced angle, up to pi, is rounded to 32 bits (2^-23 of itself at most) and sine and cosine are good to two units in the last place
    assert (t[..., 0] - torch.cos(a)).abs().max() < 2.0 ** -20 and (t[..., 1] - torch.sin(a)).abs().max() < 2.0 ** -20


@pytest.mark.parametrize("heads,hkv,d,pt,dtype,layout,rot,interleaved", [
    (4, 4, 128, 64, "bf16", "hnd", 128, False), (8, 2, 64, 16, "f16", "nhd", 64, True), (6, 3, 256, 32, "bf16", "room", 128, False),
    (0, 2, 128, 256, "bf16", "heads", 128, False), (1, 1, 64, 128, "f16", "hnd", 16, True), (40, 40, 128, 64, "bf16", "hnd", 0, False),
    (7, 1, 256, 16, "bf16", "nhd", 256, True), (33, 11, 64, 64, "bf16", "hnd", 48, False)])
@pytest.mark.parametrize("in_place", [False, True])
def test_append(heads, hkv, d, pt, dtype, layout, rot, interleaved, in_place):
    from paper_2505_19201_b200 import api
    rng = random.Random(heads + d)
    k, v = pools(40, hkv, pt, d, dtype, layout)
    tab = torch.tensor(rng.sample(range(40), 36), dtype=torch.int32, device="cuda").view(3, 12)
    bounds = torch.full((40, hkv, 2, d), NAN, dtype=k.dtype, device="cuda")
    cache = api.Cache(k, v, tab, bounds)
    # ranges of three sequences, rows shuffled among one another, two of padding
    rows = [(0, s) for s in range(0, 2 * pt + 3)] + [(1, s) for s in range(pt - 1, pt + 1)] + [(2, 12 * pt - 1)]
    rng.shuffle(rows)
    rows[3:3] = [(-1, 5)]
    rows += [(-1, -9)]
    R = len(rows)
    pos = [max(0, s) + 3 * (i % 2) for i, (_, s) in enumerate(rows)]
    g = torch.Generator(device="cuda").manual_seed(d)
    fused = torch.randn(R, heads + 2 * hkv, d, generator=g, device="cuda").to(k.dtype)
    q, kn, vn = fused[:, :heads].clone() if heads else None, fused[:, heads:heads + hkv], fused[:, heads + hkv:]
    q_in = q.clone() if heads else None
    q_out = None if not heads else q if in_place else torch.full_like(q, 9.0)
    # sequence 1 has tokens in the page that row (1, pt - 1) fills
    old = torch.randn(hkv, pt - 1, d, generator=g, device="cuda").to(k.dtype)
    k[int(tab[1, 0]), :, :pt - 1] = old
    status = i32([0, 0])
    api.dream_cache_append(cache, q, kn, vn, i32([s for s, _ in rows]), i32([t for _, t in rows]), q_out, positions=i32(pos),
                           rope=table(max(pos) + 1, rot) if rot else None, interleaved=interleaved, status=status)
    assert status.tolist() == [0, 0]
    real = torch.tensor([s >= 0 for s, _ in rows], device="cuda")
    if heads:
        want, slack = turned(q_in, pos, rot, interleaved)
        near(q_out[real], want[real], slack[real], dtype)
        assert torch.equal(q_out[~real], (q_in if in_place else torch.full_like(q, 9.0))[~real])
    want, slack = turned(kn, pos, rot, interleaved)
    written = torch.zeros(40, pt, dtype=torch.bool, device="cuda")
    written[int(tab[1, 0]), :pt - 1] = True
    for r, (s, t) in enumerate(rows):
        if s < 0:
            continue
        page = int(tab[s, t // pt])
        near(k[page, :, t % pt], want[r], slack[r], dtype)
        assert torch.equal(v[page, :, t % pt], vn[r])
        written[page, t % pt] = True
    assert torch.isnan(k.permute(0, 2, 1, 3)[~written]).all()                # nothing else was touched
    assert torch.equal(k[int(tab[1, 0]), :, :pt - 1], old)
    full = {int(tab[s, t // pt]) for s, t in rows if s >= 0 and t % pt == pt - 1}
    for page in range(40):
        if page in full and page != int(tab[2, 11]):
            assert torch.equal(bounds[page], torch.stack((k[page].amin(1), k[page].amax(1)), 1))
        elif page not in full:
            assert torch.isnan(bounds[page]).all()


def test_bounds_follow_a_page_that_is_rewritten():
    """Tokens that are refused leave nothing behind in the bounds."""
    from paper_2505_19201_b200 import api
    k, v = pools(2, 1, 16, 64, "bf16")
    bounds = torch.zeros(2, 1, 2, 64, dtype=torch.bfloat16, device="cuda")
    cache = api.Cache(k, v, i32([[1, 0]]), bounds)
    x = torch.randn(40, 1, 64, device="cuda").bfloat16()
    push = lambda a, b, rows: api.dream_cache_append(cache, None, rows, rows, i32([0] * (b - a)), i32(list(range(a, b))), None)  # noqa: E731
    push(0, 16, 100 * x[:16])
    push(10, 16, x[:6])                                         # the tail again
    assert torch.equal(bounds[1], torch.stack((k[1].amin(1), k[1].amax(1)), 1))
    push(0, 10, x[6:16])
    push(10, 16, x[:6])
    assert torch.equal(bounds[1], torch.stack((k[1].amin(1), k[1].amax(1)), 1)) and bounds[1].abs().max() < 10
    assert (bounds[0] == 0).all()


def test_append_numbers_out_of_range():
    from paper_2505_19201_b200 import api
    for rows, pos, bad in (([(0, 0), (3, 1), (0, 2)], None, 1), ([(0, 0), (0, 64), (0, 2)], None, 1), ([(0, 0), (0, -1), (0, 2)], None, 1),
                           ([(0, 0), (0, 1), (0, 2)], [0, 70, 2], 1), ([(0, 0), (1, 1), (0, 2)], None, 1)):
        k, v = pools(4, 2, 16, 64, "bf16")
        cache = api.Cache(k, v, i32([[0, 1, 2, 3], [9, 9, 9, 9]]))
        x = torch.randn(3, 2, 64, device="cuda").bfloat16()
        q_out, status = torch.zeros_like(x), i32([0, 0])
        api.dream_cache_append(cache, x, x, x, i32([s for s, _ in rows]), i32([t for _, t in rows]), q_out, positions=None if pos is None else i32(pos),
                               rope=table(64, 64), status=status)
        assert status[0] == 2
        assert torch.isnan(k[0, :, 1]).all() and torch.isnan(k[1:]).all() and not torch.isnan(k[0, :, [0, 2]]).any()
        assert torch.equal(v[0, :, 0], x[0]) and torch.equal(v[0, :, 2], x[2])


# ---------------------------------------------------------------------------------- selection

def wanted(pg, bounds, q, row_seq, row_pos, budget, first, last):
    R, H, d = q.shape
    ids = torch.full((R, pg.hkv, budget), -1, dtype=torch.int32)
    for r in range(R):
        if row_seq[r] < 0 or row_pos[r] < 0:
            continue
        n = row_pos[r] // pg.pt + 1
        b = bounds[pg.table[row_seq[r], :n].long()].double()                 # [n, hkv, 2, d]
        for h in range(pg.hkv):
            x = q[r, h * H // pg.hkv:(h + 1) * H // pg.hkv].double()
            s = torch.maximum(x[:, None] * b[None, :, h, 0], x[:, None] * b[None, :, h, 1]).sum(2).amax(0).float().cpu()
            s[:first] = s[max(0, n - last):] = float("inf")
            some = sorted(torch.sort(s, descending=True, stable=True).indices[:budget].tolist())
            ids[r, h, :len(some)] = torch.tensor(some, dtype=torch.int32)
    return ids


def selected(pg, bounds, q, row_seq, row_pos, budget, first=1, last=1):
    from paper_2505_19201_b200 import api
    cache = api.Cache(pg.k, pg.v, pg.table, bounds)
    ids, status = torch.full((len(row_seq), pg.hkv, budget), 99, dtype=torch.int32, device="cuda"), i32([0, 0])
    w = torch.full((api.dream_cache_select_bytes(cache, len(row_seq)),), 255, dtype=torch.uint8, device="cuda")
    api.dream_cache_select(cache, q, i32(row_seq), i32(row_pos), ids, w, keep_first=first, keep_last=last, status=status)
    assert status.tolist() == [0, 0]
    return ids.cpu()


def bounds_of(pg):
    """Of full pages; NaN elsewhere (a page that is not full has none)."""
    return torch.stack((pg.k.contiguous().amin(2), pg.k.contiguous().amax(2)), 2)


@pytest.mark.parametrize("heads,hkv,d", [(1, 1, 64), (4, 4, 128), (8, 2, 128), (6, 2, 64), (14, 2, 128), (4, 2, 256), (16, 1, 128), (100, 1, 64), (18, 1, 256)])
@pytest.mark.parametrize("dtype,pt,budget,first,last", [("bf16", 16, 7, 1, 1), ("f16", 32, 5, 0, 2), ("bf16", 64, 3, 2, 1), ("bf16", 16, 40, 4, 3), ("f16", 16, 1, 0, 1)])
def test_selection(heads, hkv, d, dtype, pt, budget, first, last):
    pg = Pages([1, 20 * pt + 5, 130 * pt, 9 * pt + 1], hkv, d, pt, dtype, seed=heads + budget)
    seqs, pos = [0, 1, 1, 2, -1, 3, 3, 2], [0, 20 * pt + 4, 20 * pt - 1, 130 * pt - 1, 3, 9 * pt, -1, 64 * pt]
    q = pg.queries(len(seqs), heads)
    b = bounds_of(pg)
    assert torch.equal(selected(pg, b, q, seqs, pos, budget, first, last), wanted(pg, b, q, seqs, pos, budget, first, last))


def test_selection_ties_go_to_the_lower_page():
    pg = Pages([100 * 16], 2, 64, 16)
    b = bounds_of(pg)
    b[:] = b[int(pg.table[0, 3])]
    q = pg.queries(3, 4)
    got = selected(pg, b, q, [0, 0, 0], [1599, 1000, 17], 8, 1, 2)
    assert got[0, 0].tolist() == [0, 1, 2, 3, 4, 5, 98, 99] and got[1, 1].tolist() == [0, 1, 2, 3, 4, 5, 61, 62] and got[2, 0].tolist() == [0, 1] + [-1] * 6
    q.zero_()
    q[:, :, ::2] = -0.0
    assert torch.equal(selected(pg, bounds_of(pg), q, [0, 0, 0], [1599, 1000, 17], 8, 1, 2), got)      # every score is a zero of some sign


def test_selection_in_a_long_context():
    pg = Pages([16 * 9001 + 3], 1, 64, 16)
    q, b = pg.queries(2, 2), bounds_of(pg)
    for budget in (2, 300, 4096):
        assert torch.equal(selected(pg, b, q, [0, 0], [16 * 9001 + 2, 16 * 5000], budget), wanted(pg, b, q, [0, 0], [16 * 9001 + 2, 16 * 5000], budget, 1, 1))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_selection_with_numbers_of_all_sizes(dtype):
    """Subnormal and very large values: sums in 64 bits hold them all."""
    pg = Pages([200 * 16], 1, 64, 16, dtype)
    b = bounds_of(pg).float()
    g = torch.Generator(device="cuda").manual_seed(1)
    span = 20 if dtype == "bf16" else 12
    b *= 2.0 ** torch.randint(-span, span // 3, b.shape, generator=g, device="cuda")
    b[::3] *= 2.0 ** -(100 if dtype == "bf16" else 8)
    lo, hi = torch.minimum(b[:, :, 0], b[:, :, 1]), torch.maximum(b[:, :, 0], b[:, :, 1])
    b = torch.stack((lo, hi), 2).to(TYPES[dtype])
    q = pg.queries(3, 3)
    q[1] *= 2.0 ** -(60 if dtype == "bf16" else 6)
    q[2, 0] = 0
    for budget in (2, 50, 199):
        assert torch.equal(selected(pg, b, q, [0] * 3, [3199] * 3, budget), wanted(pg, b, q, [0] * 3, [3199] * 3, budget, 1, 1))


def test_selection_numbers_out_of_range():
    from paper_2505_19201_b200 import api
    pg = Pages([20 * 16], 1, 64, 16)
    b = bounds_of(pg)
    pg.table[0, 5] = 777                                        # a page without bounds comes last
    q = pg.queries(1, 1)
    cache = api.Cache(pg.k, pg.v, pg.table, b)
    w = torch.empty(api.dream_cache_select_bytes(cache, 1), dtype=torch.uint8, device="cuda")
    ids, status = i32([[[0] * 19]]), i32([0, 0])
    api.dream_cache_select(cache, q, i32([0]), i32([319]), ids, w, status=status)
    assert status[0] == 2 and ids[0, 0].tolist() == [j for j in range(20) if j != 5]
    for seq, pos in ((1, 5), (0, 10 ** 6)):
        status.zero_()
        api.dream_cache_select(cache, q, i32([seq]), i32([pos]), ids, w, status=status)
        assert status[0] == 2 and (ids == -1).all()
