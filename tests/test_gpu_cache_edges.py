"""Calls on a paged cache at the edges of what they allow."""
import random

import pytest
import torch

from .test_gpu_cache_attn import dense
from .test_gpu_cache_rows import i32, table
from .util_cache import NAN, Pages, close, close_lse, dense_reference, pools, tree_words

pytestmark = pytest.mark.gpu


def chain(n, junk):
    """Words of a path of n nodes; with junk, every bit past the n-th set."""
    words = tree_words([i - 1 for i in range(n)])
    if junk:
        for row in words:
            for w in range(4):
                bits = sum(1 << j for j in range(32) if 32 * w + j >= n)
                row[w] = (row[w] & 0xffffffff) | bits
                row[w] -= (row[w] >> 31) << 32
    return words


# (heads, kv heads, rows of each sequence): a call of up to four entries, tiles of up to 128, several of them
FORMS = [(1, 1, [1, 2]), (4, 2, [1]), (8, 2, [1, 2]), (4, 4, [3, 40]), (16, 1, [30, 9])]


@pytest.mark.parametrize("heads,hkv,T", FORMS)
@pytest.mark.parametrize("d,pt,shared,lengths", [(64, 64, 1, [40, 40]), (128, 64, 3, [70, 41]), (256, 16, 9, [50, 63]), (128, 256, 2, [300, 41])])
@pytest.mark.parametrize("tree", [False, True])
def test_nobody_fills_the_shared_pages(heads, hkv, T, d, pt, shared, lengths, tree):
    """What lies behind everybody's last token is NaN, and entries of the table behind it are no pages."""
    lengths = lengths[:len(T)]
    pg = Pages(lengths, hkv, d, pt, shared=shared, seed=heads)
    pg.table[:, (max(lengths) + pt - 1) // pt:] = -1
    dense(pg, T, heads, tree=sum((chain(n, False) for n in T), []) if tree else None)


@pytest.mark.parametrize("heads,hkv,T", FORMS)
@pytest.mark.parametrize("d,pt,shared,lengths", [(128, 64, 2, [128, 90]), (64, 16, 8, [127, 100]), (256, 64, 2, [140, 100])])
def test_bits_of_nodes_that_are_not_there(heads, hkv, T, d, pt, shared, lengths):
    """A tree inside the shared pages, in front of tokens that are another sequence's: bits past its last node say nothing."""
    T, lengths = T[::-1], lengths[::-1][:len(T)]
    pg = Pages([max(lengths)] + lengths, hkv, d, pt, shared=shared, seed=heads)
    dense(pg, [1] + T, heads, tree=chain(1, True) + sum((chain(n, True) for n in T), []))


@pytest.mark.parametrize("hkv,d,pt,dtype,rot,more", [(2, 128, 64, "bf16", 128, 0), (1, 64, 16, "f16", 0, 0), (3, 256, 32, "bf16", 96, 0), (8, 128, 256, "bf16", 128, 0), (8, 128, 32, "f16", 64, 3000)])
def test_bounds_of_a_page_that_several_sequences_write(hkv, d, pt, dtype, rot, more):
    """Rows of three sequences that name one page, at places of their own in it and at entries of their own in the table, in any order; `more` rows of a fourth."""
    from paper_2505_19201_b200 import api
    rng = random.Random(pt)
    n_pages = 8 + more // pt + 1
    k, v = pools(n_pages, hkv, pt, d, dtype)
    tab = torch.full((4, n_pages), -1, dtype=torch.int32)
    tab[0, 0], tab[1, 2], tab[2, 1] = 5, 5, 5
    tab[3, :n_pages - 8] = torch.arange(8, n_pages)
    bounds = torch.full((n_pages, hkv, 2, d), NAN, dtype=k.dtype, device="cuda")
    cache = api.Cache(k, v, tab.cuda(), bounds)
    rope = table(3 * pt + more, rot) if rot else None
    g = torch.Generator(device="cuda").manual_seed(pt)
    for turn in range(8):
        owner = [rng.choice([0, 1, 2, None]) for _ in range(pt)]                # None: it stays as it is, which the first time is nothing
        owner[-1] = turn % 3
        rows = [(s, (0, 2 * pt, pt)[s] + t) for t, s in enumerate(owner) if s is not None] + [(3, t) for t in range(more)]
        if turn % 2:
            rng.shuffle(rows)
        x = (8.0 - turn) * torch.randn(len(rows), hkv, d, generator=g, device="cuda")
        x, status = x.to(k.dtype), i32([0, 0])
        api.dream_cache_append(cache, None, x, x, i32([s for s, _ in rows]), i32([t for _, t in rows]), None, rope=rope, status=status)
        assert status.tolist() == [0, 0]
        page = k[5].float().nan_to_num(nan=0.0)
        there = ~torch.isnan(k[5]).any(2).any(0)
        assert torch.equal(bounds[5].float(), torch.stack((page[:, there].amin(1), page[:, there].amax(1)), 1))


@pytest.mark.parametrize("order", [1, -1])
def test_bounds_hold_what_a_refused_row_leaves(order):
    """A row whose position is out of range is not written: the page's bounds count the token that is there."""
    from paper_2505_19201_b200 import api
    k, v = pools(1, 2, 16, 64, "bf16")
    bounds = torch.full((1, 2, 2, 64), NAN, dtype=torch.bfloat16, device="cuda")
    cache = api.Cache(k, v, i32([[0]]), bounds)
    rope, slots = table(20, 64), list(range(16))[::order]
    old = 50 * torch.randn(16, 2, 64, device="cuda").bfloat16()
    api.dream_cache_append(cache, None, old, old, i32([0] * 16), i32(slots), None, rope=rope)
    was, new, status = k[0, :, 6].clone(), torch.randn(16, 2, 64, device="cuda").bfloat16(), i32([0, 0])
    api.dream_cache_append(cache, None, new, new, i32([0] * 16), i32(slots), None, positions=i32([20 if t == 6 else t for t in slots]), rope=rope, status=status)
    assert status[0] == 2 and torch.equal(k[0, :, 6], was)
    assert torch.equal(bounds[0], torch.stack((k[0].amin(1), k[0].amax(1)), 1))


@pytest.mark.parametrize("n_seqs,busy,T", [(4096, [3, 700, 701, 2500, 4095], [1, 1, 1, 1, 1]), (4096, [0, 1999, 4094], [20, 3, 130]), (65, [64], [1]), (33, [0, 32], [2, 40]), (640, [31, 32, 639], [1, 7, 1])])
@pytest.mark.parametrize("shared", [0, 2])
def test_slots_without_rows(n_seqs, busy, T, shared):
    """Slots of a batch of which few have rows in a call, at any distance from each other."""
    lengths, rows = [0] * n_seqs, [0] * n_seqs
    for i, (b, t) in enumerate(zip(busy, T)):
        lengths[b], rows[b] = 32 + t + 150 * i, t
    pg = Pages(lengths, 2, 64, 16, shared=shared, seed=n_seqs)
    pg.table[:, :shared] = pg.table[busy[0], :shared]
    dense(pg, rows, 4)


MIXED = [[1] * 7 + [40], [40, 0, 1, 0, 2, 0, 0, 3, 0, 0, 0, 0], [0] * 30 + [33, 1], [5, 0, 4, 0, 3, 0, 2, 0, 1, 0, 0, 0, 0, 0, 0, 0], [9] + [0] * 8, [4, 1, 0, 1], [200] + [1] * 60 + [0] * 200]


@pytest.mark.parametrize("heads,hkv,d", [(2, 2, 64), (4, 2, 128), (3, 1, 256), (4, 1, 64), (8, 2, 128)])
@pytest.mark.parametrize("T", MIXED)
@pytest.mark.parametrize("shared", [0, 2])
def test_prompts_beside_single_tokens(heads, hkv, d, T, shared):
    lengths = [(0 if t == 0 and b % 2 else 32 + t + 37 * (b % 5)) for b, t in enumerate(T)]
    pg = Pages(lengths, hkv, d, 16, shared=shared, seed=len(T))
    pg.table[:, :shared] = pg.table[0, :shared]
    dense(pg, T, heads)


def test_prompts_beside_single_tokens_in_graphs():
    """One captured call serves batches of every mixture, replayed one behind another with nothing between: the same bits as calls alone."""
    from paper_2505_19201_b200 import api
    most, heads = 48, 4
    pg = Pages([200 + 7 * b for b in range(24)], 2, 128, 16, seed=3)
    q = pg.queries(most, heads)
    start, work = i32([0] * 25), torch.empty(api.dream_cache_attn_bytes(pg.cache, most, heads), dtype=torch.uint8, device="cuda")
    lens, out = i32(pg.lengths), torch.zeros_like(q)
    call = lambda o: api.dream_cache_attn(pg.cache, q, start, lens, o, work)  # noqa: E731
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        call(out)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call(out)
    for T in ([1] * 24, [2] * 24, [40] + [0] * 20 + [1, 2, 3], [0] * 24, [0] * 23 + [48], [1] * 20 + [5, 5, 5, 5]):
        starts = [sum(T[:b]) for b in range(25)]
        start.copy_(i32(starts))
        alone = torch.full_like(q, 7.0)
        call(alone)
        torch.cuda.synchronize()
        out.fill_(7.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for _ in range(5):
                graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, alone)
        if starts[-1]:
            want, _, size = dense_reference(pg, q, starts)
            close(out[:starts[-1]], want, size, "bf16")
        assert (out[starts[-1]:] == 7.0).all()


@pytest.mark.parametrize("T", [[1] * 4, [64, 64, 64, 63], [64] * 4, [1, 254, 0, 1], [3, 250, 0, 3]])
@pytest.mark.parametrize("behind", [0, 3, 600])
def test_rows_behind_the_last_do_not_say_how_the_prefix_is_read(T, behind):
    """Around 256 query entries to a sequence, with room for more rows than there are."""
    pg = Pages([64 + max(t, 1) + 5 * b for b, t in enumerate(T)], 2, 128, 32, shared=2, seed=sum(T))
    dense(pg, T, 8, behind=behind)


@pytest.mark.parametrize("T,heads,shared", [([3, 1], 4, 0), ([1, 1], 4, 2), ([90, 70], 8, 2), ([300, 400], 8, 0)])
def test_rows_in_front_of_the_first_sequence_are_nobodys(T, heads, shared):
    """Starts that do not begin at 0 are out of range: reported, and the rows in front are left as they were."""
    from paper_2505_19201_b200 import api
    pg = Pages([t + 64 for t in T], 2, 64, 32, shared=shared)
    front, n = 2, sum(T)
    q = pg.queries(front + n, heads)
    out, lse, status = torch.full_like(q, 77.0), torch.full((front + n, heads), 77.0, device="cuda"), i32([0, 0])
    work = torch.full((api.dream_cache_attn_bytes(pg.cache, front + n, heads),), 255, dtype=torch.uint8, device="cuda")
    api.dream_cache_attn(pg.cache, q, i32([front, front + T[0], front + n]), i32(pg.lengths), out, work, shared_pages=shared, lse=lse, status=status)
    want, wl, size = dense_reference(pg, q[front:], [0, T[0], n])
    close(out[front:], want, size, "bf16")
    close_lse(lse[front:], wl)
    assert (out[:front] == 77.0).all() and (lse[:front] == 77.0).all() and status[0] == 2


def test_selection_with_sums_past_the_largest_number_on_the_way():
    """A part of a page's sum is past the largest number of 32 bits, the sum itself is not: another page's is larger."""
    from paper_2505_19201_b200 import api
    n, big = 40, 2.0 ** 63
    k = torch.zeros(n, 1, 16, 64, dtype=torch.bfloat16, device="cuda")
    bounds = torch.zeros(n, 1, 2, 64, dtype=torch.bfloat16, device="cuda")
    bounds[7, 0, :, [0, 8]], bounds[7, 0, :, 40] = big, -big                    # 2^127 + 2^127 - 2^127
    bounds[30, 0, :, 0] = 1.5 * big
    cache = api.Cache(k, k.clone(), i32([list(range(n))]), bounds)
    q = torch.zeros(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    q[0, 0, [0, 8, 40]] = 2.0 ** 64
    for budget, want in ((3, [0, 30, 39]), (4, [0, 7, 30, 39])):
        ids = torch.zeros(1, 1, budget, dtype=torch.int32, device="cuda")
        work = torch.full((api.dream_cache_select_bytes(cache, 1),), 255, dtype=torch.uint8, device="cuda")
        api.dream_cache_select(cache, q, i32([0]), i32([n * 16 - 1]), ids, work, keep_first=1, keep_last=1)
        assert ids[0, 0].tolist() == want


def test_wrappers_refuse_before_anything_is_enqueued():
    """Every refusal is the library's or the wrapper's own, with its code, and leaves the output and the device as they were."""
    from paper_2505_19201_b200 import api
    E_ARG, E_NOMEM = -1, -3
    pg = Pages([40, 20], 2, 64, 16)
    q, n, start = pg.queries(2, 4), i32([40, 20]), i32([0, 1, 2])
    room = torch.empty(api.dream_cache_attn_bytes(pg.cache, 2, 4), dtype=torch.uint8, device="cuda")
    out, ids, seq, pos = torch.full_like(q, 5.0), i32([[[0, 1]] * 2] * 2), i32([0, 1]), i32([39, 19])
    kv = torch.zeros(2, 2, 64, dtype=q.dtype, device="cuda")
    calls = [
        (api.dream_cache_attn, dict(cache=pg.cache, q=q, q_start=start, kv_len=n, out=out, workspace=room),
         [dict(q=q.half()), dict(q=q.cpu()), dict(q=q[:, :, :32]), dict(q=q[:, ::2]), dict(q=None), dict(q=q[0]), dict(out=out[:1]), dict(out=out[:, :2]), dict(out=q),
          dict(q_start=start[:2]), dict(q_start=start.long()), dict(q_start=None), dict(kv_len=n[:1]), dict(kv_len=None), dict(workspace=None),
          dict(tree_mask=torch.zeros(2, 3, dtype=torch.int32, device="cuda")), dict(lse=torch.zeros(2, 3, device="cuda")), dict(scale=0.0), dict(scale=float("nan")),
          dict(shared_pages=99), dict(q=q[:0], out=out[:0]), dict(cache=None), dict(workspace=room[16:])], [dict(workspace=room[:-256])]),
        (api.dream_cache_attn_pages, dict(cache=pg.cache, q=q, row_seq=seq, row_pos=pos, ids=ids, out=out, workspace=room),
         [dict(ids=ids[:, :1]), dict(ids=ids.long()), dict(ids=None), dict(row_seq=seq[:1]), dict(row_pos=None), dict(ids=ids[:, :, :0])], [dict(workspace=room[:256])]),
        (api.dream_cache_append, dict(cache=pg.cache, q=q, k_new=kv, v_new=kv, row_seq=seq, slots=i32([0, 0]), q_out=out),
         [dict(k_new=kv[:1]), dict(v_new=kv.half()), dict(v_new=None), dict(slots=None), dict(slots=pos[:1]), dict(q_out=None), dict(q=None), dict(q_out=out[:, :2]),
          dict(rope=torch.zeros(4, 32, device="cuda")), dict(rope=torch.zeros(4, 64, 2, device="cuda")), dict(positions=pos.long())], [])]
    k, v = pg.k.clone(), pg.v.clone()
    for call, good, bad_args, short in calls:
        for some, code in ((bad_args, E_ARG), (short, E_NOMEM)):
            for bad in some:
                with pytest.raises(api.DreamError) as e:
                    call(**dict(good, **bad))
                assert e.value.code == code, (call.__name__, bad.keys(), str(e.value))
    with pytest.raises(api.DreamError) as e:                                    # a cache without bounds
        api.dream_cache_select(pg.cache, q, seq, pos, ids, room)
    assert e.value.code == E_ARG
    torch.cuda.synchronize()
    assert (out == 5.0).all() and torch.equal(k.nan_to_num(9.0), pg.k.nan_to_num(9.0)) and torch.equal(v.nan_to_num(9.0), pg.v.nan_to_num(9.0))
    calls[0][0](**calls[0][1])
    want, _, size = dense_reference(pg, q, [0, 1, 2])
    close(out, want, size, "bf16")


def test_several_host_threads():
    """Threads that each append, attend, select and attend to the selected on a stream, a cache and a workspace of their own: the same bits as one behind the other."""
    import threading

    from paper_2505_19201_b200 import api
    heads, hkv, rows = 8, 2, 3

    def work(i, out, times):
        d, pt = (64, 128, 256, 128)[i % 4], (16, 32, 64, 16)[i % 4]
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            pg = Pages([700 + i, 90, 1300], hkv, d, pt, seed=i, extra_entries=2)
            bounds = torch.stack((pg.k.contiguous().amin(2), pg.k.contiguous().amax(2)), 2).nan_to_num(0.0)
            cache = api.Cache(pg.k, pg.v, pg.table, bounds)
            room = torch.empty(max(api.dream_cache_attn_bytes(cache, rows, heads), api.dream_cache_select_bytes(cache, rows)), dtype=torch.uint8, device="cuda")
            x = pg.queries(rows, heads + 2 * hkv)
            seq, pos, status = i32([0, 1, 2]), i32([n - 1 for n in pg.lengths]), i32([0, 0])
            for _ in range(times):
                q, dense_out, few = (torch.zeros(rows, heads, d, dtype=x.dtype, device="cuda") for _ in range(3))
                ids = torch.zeros(rows, hkv, 4, dtype=torch.int32, device="cuda")
                api.dream_cache_append(cache, x[:, :heads], x[:, heads:heads + hkv], x[:, heads + hkv:], seq, pos, q, status=status)
                api.dream_cache_attn(cache, q, i32([0, 1, 2, 3]), pos + 1, dense_out, room, status=status)
                api.dream_cache_select(cache, q, seq, pos, ids, room, status=status)
                api.dream_cache_attn_pages(cache, q, seq, pos, ids, few, room, status=status)
                out.append((dense_out, ids, few))
            stream.synchronize()
            assert status.tolist() == [0, 0]

    alone, together = [[] for _ in range(6)], [[] for _ in range(6)]
    for i in range(6):
        work(i, alone[i], 1)
    threads = [threading.Thread(target=work, args=(i, together[i], 8)) for i in range(6)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for a, b in zip(alone, together):
        assert len(b) == 8
        for got in b:
            assert all(torch.equal(x, y) for x, y in zip(a[0], got))


@pytest.mark.parametrize("heads", [1, 4, 16])
@pytest.mark.parametrize("tree", [False, True])
def test_more_rows_than_tokens_behind_shared_pages(heads, tree):
    """Rows in front of a sequence's first token see nothing, whatever the others share."""
    T, lengths = [2, 10, 4, 0], [100, 3, 0, 70]
    out, lse = dense(Pages(lengths, 1, 64, 32, shared=2), T, heads, tree=sum((chain(n, True) for n in T), []) if tree else None)
    if not tree:
        assert (out[2:9] == 0).all() and (out[12:16] == 0).all() and torch.isinf(lse[2:9]).all() and torch.isinf(lse[12:16]).all()


@pytest.mark.parametrize("heads,T", [(1, 1), (8, 3), (4, 130)])
def test_values_as_large_as_may_be(heads, T):
    """Values of 2^119 over the number of keys: sums of weights up to 2^8 times such values are finite."""
    pg = Pages([512], 1, 128, 64)
    pg.k *= torch.linspace(0.1, 2, 64, device="cuda").bfloat16()[:, None]
    pg.v.copy_(torch.sign(pg.v) * 2.0 ** 110)
    dense(pg, [T], heads, gain=2.0, spread=100.0)
