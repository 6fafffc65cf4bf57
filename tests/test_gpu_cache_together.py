"""The calls on a paged cache as a program uses them: one behind the other over the steps of a batch, on streams, in graphs, and far out in memory."""
import random

import pytest
import torch

from .test_gpu_cache_rows import angles, i32, near, table
from .util_cache import NAN, TYPES, Pages, attend, close, close_lse, dense_reference, pages_reference

pytestmark = pytest.mark.gpu
SPREAD = 16.0          # sum |q k| scale of normal numbers: 0.64 sqrt(256) = 10, rarely twice that (close counts 8 of it by itself)


def room(n):
    return torch.full((n,), 255, dtype=torch.uint8, device="cuda")


def turn(x, pos, rot, interleaved):
    """Rotated in 64 bits; x [rows, heads, d], pos [rows]."""
    x = x.double().clone()
    a = angles(int(pos.max()) + 1, rot)[pos.long()][:, None]
    one, two = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    p, q = x[..., one].clone(), x[..., two].clone()
    x[..., one], x[..., two] = p * torch.cos(a) - q * torch.sin(a), q * torch.cos(a) + p * torch.sin(a)
    slack = torch.zeros_like(x)
    slack[..., one] = slack[..., two] = 2.0 ** -20 * (p.abs() + q.abs())
    return x, slack


def best_pages(cache, table_row, q, pos, budget, first, last):
    """The selection of one row, by the definition: [hkv, budget] page numbers."""
    hkv, pt = cache.heads, cache.k.shape[2]
    own = pos // pt
    n = own + 1
    must = set(range(min(first, n))) | set(range(max(0, n - last), n))
    lo, hi = (cache.bounds[table_row[:n].long(), :, i].double() for i in (0, 1))           # [n, hkv, d]
    ids = torch.full((hkv, budget), -1, dtype=torch.int32)
    G = q.shape[0] // hkv
    for h in range(hkv):
        if n <= budget:
            keep = list(range(n))
        else:
            x = q[h * G:(h + 1) * G].double()
            scores = torch.maximum(x[:, None] * lo[None, :, h], x[:, None] * hi[None, :, h]).sum(2).amax(0).float()
            rest = [p for p in torch.sort(-scores, stable=True)[1].tolist() if p not in must]
            keep = sorted(must | set(rest[:budget - len(must)]))
        ids[h, :len(keep)] = torch.tensor(keep, dtype=torch.int32)
    return ids


@pytest.mark.parametrize("heads,hkv,d,pt,dtype,interleaved", [(8, 2, 128, 16, "bf16", False), (4, 4, 64, 32, "f16", True), (4, 2, 256, 16, "bf16", False)])
def test_steps_of_a_batch(heads, hkv, d, pt, dtype, interleaved):
    """Prompts behind a common prefix, then token by token: append, attend to everything, select, attend to the selected."""
    from paper_2505_19201_b200 import api
    g = torch.Generator(device="cuda").manual_seed(d)
    prefix, prompts, steps, budget = 5 * pt, [3, 2 * pt + 1, pt - 1], pt + 2, 6
    B, rot = len(prompts), d
    lengths = [prefix + p for p in prompts]
    pg = Pages([n + steps for n in lengths], hkv, d, pt, dtype, shared=prefix // pt, extra_entries=2)
    pg.k.fill_(NAN), pg.v.fill_(NAN)
    bounds = torch.full((pg.k.shape[0], hkv, 2, d), NAN, dtype=TYPES[dtype], device="cuda")
    cache = pg.cache = api.Cache(pg.k, pg.v, pg.table, bounds)
    rope, status = table(max(lengths) + steps, rot), i32([0, 0])
    most = sum(prompts) + prefix + 3
    work = room(max(api.dream_cache_attn_bytes(cache, most, heads), api.dream_cache_select_bytes(cache, B + 1)))
    said = {}                                                 # (sequence, token): its key and value as they were given

    def append(rows):
        """Rows (sequence, token), in this order; returns the rotated queries."""
        n = len(rows)
        x = torch.randn(n, heads + 2 * hkv, d, generator=g, device="cuda").to(TYPES[dtype])
        q, kn, vn = x[:, :heads], x[:, heads:heads + hkv], x[:, heads + hkv:]
        out = torch.zeros(n, heads, d, dtype=x.dtype, device="cuda")
        seq, slot = i32([s for s, _ in rows]), i32([t for _, t in rows])
        api.dream_cache_append(cache, q, kn, vn, seq, slot, out, rope=rope, interleaved=interleaved, status=status)
        pos = slot.clamp(min=0)
        real = seq >= 0
        want, slack = turn(q, pos, rot, interleaved)
        near(out[real], want[real], slack[real], dtype)
        want, slack = turn(kn, pos, rot, interleaved)
        page = pg.table[seq.clamp(min=0).long(), (pos // pt).long()].long()
        near(pg.k[page, :, (pos % pt).long()][real], want[real], slack[real], dtype)
        assert torch.equal(pg.v[page, :, (pos % pt).long()][real], vn[real])
        return out

    append([(0, t) for t in range(prefix)])                   # everybody's pages, written once
    now = list(lengths)
    pg.lengths = now
    start = [0]
    for p in prompts:
        start.append(start[-1] + p)
    q = append([(b, prefix + t) for b in range(B) for t in range(prompts[b])] + [(-1, 0)] * 2)

    def attend_all(q, start):
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
        api.dream_cache_attn(cache, q, i32(start), i32(now), out, work, shared_pages=prefix // pt, lse=lse, status=status)
        want, wl, size = dense_reference(pg, q, start)
        n = start[-1]
        close(out[:n], want, size, dtype, spread=SPREAD)
        close_lse(lse[:n], wl, spread=SPREAD)
        assert (out[n:] == 7.0).all() and (lse[n:] == 7.0).all()
        return out

    attend_all(q, start)
    for step in range(steps):
        q = append([(b, now[b]) for b in range(B)] + [(-1, 0)])
        for b in range(B):
            now[b] += 1
        out = attend_all(q, list(range(B + 1)))
        pos = [n - 1 for n in now] + [0]
        ids = torch.full((B + 1, hkv, budget), 99, dtype=torch.int32, device="cuda")
        seq = i32(list(range(B)) + [-1])
        api.dream_cache_select(cache, q, seq, i32(pos), ids, work, keep_first=1, keep_last=2, status=status)
        for b in range(B):
            assert torch.equal(ids[b].cpu(), best_pages(cache, pg.table[b], q[b], pos[b], budget, 1, 2))
        assert (ids[B] == -1).all()
        few = torch.full_like(q, 7.0)
        api.dream_cache_attn_pages(cache, q, seq, i32(pos), ids, few, work, status=status)
        want, _, size = pages_reference(pg, q[:B], list(range(B)), pos[:B], ids[:B])
        close(few[:B], want, size, dtype, spread=SPREAD)
        assert (few[B] == 7.0).all()
        if step == 0:                                         # pages enough for all of a short context: the same attention
            wide = torch.full((B + 1, hkv, 64), 99, dtype=torch.int32, device="cuda")
            room_ = room(api.dream_cache_select_bytes(cache, B + 1))
            api.dream_cache_select(cache, q, seq, i32(pos), wide, room_, keep_first=1, keep_last=2, status=status)
            every = torch.full_like(q, 7.0)
            api.dream_cache_attn_pages(cache, q, seq, i32(pos), wide, every, work, status=status)
            want, _, size = dense_reference(pg, q, list(range(B + 1)))
            close(every[:B], want, size, dtype, spread=SPREAD)
            close(out[:B], want, size, dtype, spread=SPREAD)
    assert status.tolist() == [0, 0]


@pytest.mark.parametrize("rows,heads,hkv,d,dtype,rot,interleaved,bounds", [
    (3001, 10, 2, 256, "bf16", 128, True, True), (6007, 21, 3, 64, "f16", 64, False, True), (6401, 6, 3, 128, "bf16", 96, False, False), (5003, 0, 9, 128, "f16", 128, True, True)])
def test_append_of_many_rows(rows, heads, hkv, d, dtype, rot, interleaved, bounds):
    from paper_2505_19201_b200 import api
    g = torch.Generator(device="cuda").manual_seed(rows)
    pt, seqs = 32, 3
    per = (rows + seqs - 1) // seqs
    width = per // pt + 2
    k, v = (torch.full((seqs * width, hkv, pt, d), NAN, dtype=TYPES[dtype], device="cuda") for _ in range(2))
    tab = torch.randperm(seqs * width, generator=g, device="cuda").int().view(seqs, width)
    b = torch.full((seqs * width, hkv, 2, d), NAN, dtype=TYPES[dtype], device="cuda") if bounds else None
    cache = api.Cache(k, v, tab, b)
    r = torch.arange(rows, device="cuda")
    seq, slot = (r // per).int(), (r % per).int()
    seq[rows // 2] = -1                                       # padding in the middle: a page that does not become full
    q = torch.randn(rows, heads, d, generator=g, device="cuda").to(TYPES[dtype]) if heads else None
    kn, vn = (torch.randn(rows, hkv, d, generator=g, device="cuda").to(TYPES[dtype]) for _ in range(2))
    out = torch.full((rows, heads, d), 5.0, dtype=TYPES[dtype], device="cuda") if heads else None
    status = i32([0, 0])
    api.dream_cache_append(cache, q, kn, vn, seq, slot, out, rope=table(per, rot), interleaved=interleaved, status=status)
    real = seq >= 0
    page, at = tab[seq.clamp(min=0).long(), (slot // pt).long()].long(), (slot % pt).long()
    want, slack = turn(kn, slot, rot, interleaved)
    near(k[page, :, at][real], want[real], slack[real], dtype)
    assert torch.equal(v[page, :, at][real], vn[real])
    if heads:
        want, slack = turn(q, slot, rot, interleaved)
        near(out[real], want[real], slack[real], dtype)
        assert (out[~real] == 5.0).all()
    written = torch.zeros(seqs * width, pt, dtype=torch.bool, device="cuda")
    written[page[real], at[real]] = True
    assert torch.isnan(k.permute(0, 2, 1, 3)[~written]).all() and torch.isnan(v.permute(0, 2, 1, 3)[~written]).all()
    if bounds:
        whole = written.all(1)
        assert torch.equal(b[whole], torch.stack((k[whole].amin(2), k[whole].amax(2)), 2))
        untouched = ~written[:, pt - 1]                       # no last token: no bounds
        assert torch.isnan(b[untouched]).all()
    assert status.tolist() == [0, 0]


@pytest.mark.parametrize("n_seqs,T,heads,hkv,d", [(300, 1, 4, 2, 64), (700, 1, 2, 2, 64), (700, 17, 1, 1, 64), (1500, 2, 4, 1, 64)])
def test_more_sequences_than_threads(n_seqs, T, heads, hkv, d):
    """Sequences of T to T + 12 tokens, a few of them without rows in this call; 64-bit references batched by length."""
    from paper_2505_19201_b200 import api
    rng = random.Random(n_seqs + T)
    g = torch.Generator(device="cuda").manual_seed(n_seqs)
    pt, width = 16, 3
    lens = [rng.randint(T, T + 12) for _ in range(n_seqs)]
    n_rows = [0 if rng.random() < 0.05 else T for _ in range(n_seqs)]
    start = [0]
    for n in n_rows:
        start.append(start[-1] + n)
    k, v = (torch.full((n_seqs * width, hkv, pt, d), NAN, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    tab = torch.randperm(n_seqs * width, generator=g, device="cuda").int().view(n_seqs, width)
    most = T + 12
    kk, vv = (torch.randn(n_seqs, hkv, most, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    live = torch.arange(most, device="cuda")[None] < torch.tensor(lens, device="cuda")[:, None]
    s, t = live.nonzero(as_tuple=True)
    k[tab[s, t // pt].long(), :, t % pt] = kk[s, :, t]
    v[tab[s, t // pt].long(), :, t % pt] = vv[s, :, t]
    cache = api.Cache(k, v, tab)
    rows = start[-1]
    q = torch.randn(rows, heads, d, generator=g, device="cuda").bfloat16()
    out, lse, status = torch.full_like(q, 7.0), torch.full((rows, heads), 7.0, device="cuda"), i32([0, 0])
    api.dream_cache_attn(cache, q, i32(start), i32(lens), out, room(api.dream_cache_attn_bytes(cache, rows, heads)), lse=lse, status=status)
    assert status.tolist() == [0, 0]
    on = torch.tensor([n > 0 for n in n_rows], device="cuda")
    G, n_on = heads // hkv, int(on.sum())
    x = q.view(n_on, T, hkv, G, d).double()
    scores = torch.einsum("bthgd,bhmd->bthgm", x, kk[on].double()) * d ** -0.5
    last = torch.tensor(lens, device="cuda")[on][:, None] - T + torch.arange(T, device="cuda")[None]
    scores = scores.masked_fill(torch.arange(most, device="cuda")[None, None, None, None] > last[:, :, None, None, None], -float("inf"))
    p = torch.softmax(scores, 4)
    want, size = (torch.einsum("bthgm,bhmd->bthgd", p, y).reshape(rows, heads, d) for y in (vv[on].double(), vv[on].double().abs()))
    close(out, want, size, "bf16")
    close_lse(lse, torch.logsumexp(scores, 4).reshape(rows, heads))


def test_graphs_and_streams():
    """Two captured graphs with a workspace each and changing lengths, replayed on two streams while eager calls run on a third."""
    from paper_2505_19201_b200 import api
    pg = [Pages([700 + 300 * i, 90, 1300], 2, 128, 64, seed=i, shared=1) for i in range(3)]
    heads, start = 8, [0, 1, 2, 3]
    streams = [torch.cuda.Stream() for _ in range(3)]
    q = [p.queries(3, heads) for p in pg]
    out = [torch.zeros_like(x) for x in q]
    lens = [i32(p.lengths) for p in pg]
    starts = i32(start)
    status = i32([0, 0])
    spaces = [room(api.dream_cache_attn_bytes(p.cache, 3, heads)) for p in pg]
    torch.cuda.synchronize()

    def call(i, stream=None):
        api.dream_cache_attn(pg[i].cache, q[i], starts, lens[i], out[i], spaces[i], shared_pages=1, status=status, stream=stream)

    graphs = []
    for i in range(2):
        with torch.cuda.stream(streams[i]):
            call(i)
            streams[i].synchronize()
            gr = torch.cuda.CUDAGraph()
            with torch.cuda.graph(gr, stream=streams[i]):
                call(i)
            graphs.append(gr)
    for cut in (0, 65, 1):
        now = [[max(1, n - cut) for n in p.lengths] for p in pg]
        for i in range(3):
            lens[i].copy_(i32(now[i]))
            out[i].fill_(7.0)
        torch.cuda.synchronize()
        for _ in range(4):
            for i in range(2):
                with torch.cuda.stream(streams[i]):
                    graphs[i].replay()
            call(2, streams[2])
        torch.cuda.synchronize()
        for i in range(3):
            whole = pg[i].lengths
            pg[i].lengths = now[i]
            want, _, size = dense_reference(pg[i], q[i], start)
            pg[i].lengths = whole
            close(out[i], want, size, "bf16")
    assert status.tolist() == [0, 0]


def test_offsets_past_32_bits():
    """Pages of K and V in one pool of more than 2^32 elements, the ones in use at its end."""
    from paper_2505_19201_b200 import api
    hkv, pt, d, heads = 1, 256, 256, 4
    per = 2 * hkv * pt * d
    n_pages = (1 << 32) // per + 40
    if torch.cuda.mem_get_info()[0] < 2 * n_pages * per + (2 << 30):
        pytest.skip("needs 11 GB")
    pool = torch.empty(n_pages, 2, hkv, pt, d, dtype=torch.bfloat16, device="cuda")
    k, v = pool[:, 0], pool[:, 1]
    g = torch.Generator(device="cuda").manual_seed(1)
    used = 36
    tab = (n_pages - 1 - torch.randperm(used, generator=g, device="cuda")).int().view(2, used // 2)
    pool[n_pages - used:].fill_(NAN)
    bounds = torch.full((n_pages, hkv, 2, d), NAN, dtype=torch.bfloat16, device="cuda")
    cache = api.Cache(k, v, tab, bounds)
    lens, status = [18 * pt - 3, 5 * pt + 1], i32([0, 0])
    rows = [(s, t) for s in range(2) for t in range(lens[s])]
    R = len(rows)
    seq, slot = i32([s for s, _ in rows]), i32([t for _, t in rows])
    kn, vn = (torch.randn(R, hkv, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    api.dream_cache_append(cache, None, kn, vn, seq, slot, None, status=status)
    page, at = tab[seq.long(), (slot // pt).long()].long(), (slot % pt).long()
    assert torch.equal(k[page, :, at], kn) and torch.equal(v[page, :, at], vn)
    q = torch.randn(2, heads, d, generator=g, device="cuda").bfloat16()
    out = torch.zeros_like(q)
    space = room(max(api.dream_cache_attn_bytes(cache, 2, heads), api.dream_cache_select_bytes(cache, 2)))
    api.dream_cache_attn(cache, q, i32([0, 1, 2]), i32(lens), out, space, status=status)
    pos = [n - 1 for n in lens]
    ids = torch.zeros(2, hkv, 4, dtype=torch.int32, device="cuda")
    api.dream_cache_select(cache, q, i32([0, 1]), i32(pos), ids, space, keep_first=0, keep_last=1, status=status)
    few = torch.zeros_like(q)
    api.dream_cache_attn_pages(cache, q, i32([0, 1]), i32(pos), ids, few, space, status=status)
    for s in range(2):
        mine = seq == s
        kk, vv = (x[mine].transpose(0, 1).double() for x in (kn, vn))
        want, _, size = attend(q[s:s + 1], kk, vv, torch.ones(1, lens[s], dtype=torch.bool, device="cuda"), d ** -0.5)
        close(out[s:s + 1], want, size, "bf16")
        assert torch.equal(ids[s].cpu(), best_pages(cache, tab[s], q[s], pos[s], 4, 0, 1))
        seen = torch.zeros(1, lens[s], dtype=torch.bool, device="cuda")
        for i in ids[s, 0].tolist():
            seen[0, i * pt:(i + 1) * pt] = True
        want, _, size = attend(q[s:s + 1], kk, vv, seen, d ** -0.5)
        close(few[s:s + 1], want, size, "bf16")
    assert status.tolist() == [0, 0]


def test_a_group_wider_than_a_small_tile_in_pages_and_alone():
    """40 query heads of one KV head: tiles of three rows in the dense call, of one listed row in the other."""
    from paper_2505_19201_b200 import api
    pg = Pages([1000, 1, 77], 1, 128, 32, seed=5)
    heads, budget = 40, 3
    q = pg.queries(3, heads)
    pos, ids = [999, 0, 70], i32([[[2, 17, 31]], [[0, -1, -1]], [[0, 1, 2]]])
    out = torch.zeros_like(q)
    api.dream_cache_attn_pages(pg.cache, q, i32([0, 1, 2]), i32(pos), ids, out, room(api.dream_cache_attn_bytes(pg.cache, 3, heads)))
    want, _, size = pages_reference(pg, q, [0, 1, 2], pos, ids)
    close(out, want, size, "bf16")


def test_wrappers_refuse_what_does_not_fit():
    from paper_2505_19201_b200 import api
    pg = Pages([40, 20], 2, 64, 16)
    q, n = pg.queries(2, 4), i32([40, 20])
    out, space, start = torch.zeros_like(q), room(api.dream_cache_attn_bytes(pg.cache, 2, 4)), i32([0, 1, 2])
    good = dict(cache=pg.cache, q=q, q_start=start, kv_len=n, out=out, workspace=space)
    api.dream_cache_attn(**good)
    for bad in (dict(q=q.half()), dict(q=q.cpu()), dict(q=q[:, :, :32]), dict(q=q[:, ::2]), dict(q=None), dict(q=q[0]), dict(out=out[:1]), dict(out=out[:, :2]),
                dict(q_start=start[:2]), dict(q_start=start.long()), dict(q_start=None), dict(kv_len=n[:1]), dict(kv_len=None), dict(workspace=space[:-256]),
                dict(workspace=None), dict(tree_mask=torch.zeros(2, 3, dtype=torch.int32, device="cuda")), dict(lse=torch.zeros(2, 3, device="cuda")), dict(scale=0.0),
                dict(scale=float("nan")), dict(shared_pages=99), dict(q=q[:0], out=out[:0]), dict(cache=None)):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            api.dream_cache_attn(**dict(good, **bad))
    seq, pos = i32([0, 1]), i32([39, 19])
    ids = i32([[[0, 1]] * 2] * 2)
    good = dict(cache=pg.cache, q=q, row_seq=seq, row_pos=pos, ids=ids, out=out, workspace=space)
    api.dream_cache_attn_pages(**good)
    for bad in (dict(ids=ids[:, :1]), dict(ids=ids.long()), dict(ids=None), dict(row_seq=seq[:1]), dict(row_pos=None), dict(ids=ids[:, :, :0])):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            api.dream_cache_attn_pages(**dict(good, **bad))
    with pytest.raises((ValueError, TypeError, RuntimeError)):                    # a cache without bounds
        api.dream_cache_select(pg.cache, q, seq, pos, ids, space)
    torch.cuda.synchronize()


@pytest.mark.parametrize("heads,hkv,d,dtype", [(4, 2, 128, "bf16"), (24, 2, 64, "f16"), (1, 1, 256, "bf16"), (9, 1, 128, "f16")])
def test_selection_with_infinite_bounds(heads, hkv, d, dtype):
    """A channel that is unbounded on the side that a query does not ask about says nothing; on the other side the page comes first."""
    from paper_2505_19201_b200 import api
    g = torch.Generator(device="cuda").manual_seed(d + heads)
    n, pt, budget = 300, 16, 40
    k = torch.randn(n, hkv, pt, d, generator=g, device="cuda").to(TYPES[dtype])
    bounds = torch.stack((k.amin(2), k.amax(2)), 2).contiguous()
    at = torch.randperm(n, generator=g, device="cuda")[:60]
    bounds[at[:30], :, 0, 3] = -float("inf")
    bounds[at[30:45], :, 1, 5] = float("inf")
    tab = torch.randperm(n, generator=g, device="cuda").int().view(1, n)
    cache = api.Cache(k, torch.zeros_like(k), tab, bounds)
    q = torch.randn(3, heads, d, generator=g, device="cuda").to(TYPES[dtype])
    q[q == 0] = 1.0
    q[0, :, 3], q[0, :, 5] = q[0, :, 3].abs(), -q[0, :, 5].abs()                 # row 0: nothing unbounded counts
    pos, seq = [n * pt - 1, 290 * pt, 200 * pt + 3], i32([0, 0, 0])
    ids, status = torch.full((3, hkv, budget), 99, dtype=torch.int32, device="cuda"), i32([0, 0])
    api.dream_cache_select(cache, q, seq, i32(pos), ids, room(api.dream_cache_select_bytes(cache, 3)), keep_first=1, keep_last=1, status=status)
    for r in range(3):
        assert torch.equal(ids[r].cpu(), best_pages(cache, tab[0], q[r], pos[r], budget, 1, 1))
    assert status.tolist() == [0, 0]
