"""Attention over a paged cache of the caller's own against the definition in 64 bits: dream_cache_attn and dream_cache_attn_pages."""
import random

import pytest
import torch

from .util_cache import TYPES, Pages, close, close_lse, dense_reference, pages_reference, tree_words

pytestmark = pytest.mark.gpu


def workspace(pg, rows, heads):
    from paper_2505_19201_b200 import api
    return torch.full((api.dream_cache_attn_bytes(pg.cache, rows, heads),), 255, dtype=torch.uint8, device="cuda")      # NaN wherever it is not written


def dense(pg, T, heads, tree=None, shared=None, scale=None, behind=2, gain=1.0, spread=0.0, stream=None):
    """One call with `behind` rows behind the last sequence; returns out, lse."""
    from paper_2505_19201_b200 import api
    start = [sum(T[:b]) for b in range(len(T) + 1)]
    rows = start[-1] + behind
    q = pg.queries(rows, heads, gain)
    out = torch.full_like(q, 77.0)
    lse = torch.full((rows, heads), 77.0, device="cuda")
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    words = None
    if tree is not None:
        words = torch.tensor(tree + [[0] * 4] * behind, dtype=torch.int32, device="cuda")
    api.dream_cache_attn(pg.cache, q, torch.tensor(start, dtype=torch.int32, device="cuda"), torch.tensor(pg.lengths, dtype=torch.int32, device="cuda"),
                         out, workspace(pg, rows, heads), shared_pages=pg.shared if shared is None else shared, tree_mask=words, scale=scale, lse=lse,
                         status=status)
    want, wl, size = dense_reference(pg, q, start, words, scale)
    n = start[-1]
    close(out[:n], want, size, pg.dtype, spread)
    close_lse(lse[:n], wl, spread)
    assert (out[n:] == 77.0).all() and (lse[n:] == 77.0).all()
    assert status.tolist() == [0, 0]
    return out, lse


MODELS = [(1, 1, 64), (4, 4, 128), (8, 2, 128), (6, 2, 64), (14, 2, 128), (4, 2, 256), (16, 1, 128), (40, 1, 64), (100, 1, 64)]


@pytest.mark.parametrize("heads,hkv,d", MODELS)
@pytest.mark.parametrize("dtype,pt,layout", [("bf16", 64, "hnd"), ("f16", 16, "nhd"), ("bf16", 128, "room"), ("bf16", 32, "heads"), ("f16", 256, "hnd")])
def test_ragged_batch_behind_a_shared_prefix(heads, hkv, d, dtype, pt, layout):
    shared = 3 if pt < 256 else 1
    P = shared * pt
    pg = Pages([P + 1, P + 77, P + 64, P + 300], hkv, d, pt, dtype, shared, layout, seed=heads + d + pt)
    dense(pg, [1, 5, 64, 2], heads)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200, 513])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_lengths_of_one_sequence(n, d):
    pg = Pages([n], 2, d, 64, seed=n)
    dense(pg, [1], 4)
    pg = Pages([n], 2, d, 16, seed=n)
    dense(pg, [n], 2)                                            # a prompt from its first token on


@pytest.mark.parametrize("shared", [0, 1, 2, 5])
def test_what_is_shared_changes_nothing_but_the_order_of_sums(shared):
    pg = Pages([5 * 64 + n for n in (1, 40, 64, 100)], 2, 128, 64, shared=5)
    dense(pg, [1, 2, 3, 1], 8, shared=shared)


def test_nothing_but_the_prefix_and_nothing_at_all():
    pg = Pages([128, 128, 130], 2, 64, 64, shared=2)
    dense(pg, [1, 128, 3], 4)                                    # rows whose own tokens are the prefix's last
    pg = Pages([0, 5, 0, 64], 2, 64, 16)
    out, lse = dense(pg, [1, 2, 0, 70], 4)                       # rows in front of the first token see nothing
    assert (out[0] == 0).all() and (lse[0] == -float("inf")).all() and (out[3:9] == 0).all()
    dense(Pages([0, 0], 1, 64, 16), [0, 0], 2)                   # no rows but those behind
    dense(Pages([0], 1, 128, 16), [3], 2)


@pytest.mark.parametrize("heads,hkv,d,pt", [(4, 4, 128, 64), (8, 2, 64, 16), (4, 2, 256, 32)])
def test_trees(heads, hkv, d, pt):
    rng = random.Random(heads)
    T, tree = [61, 1, 128, 33], []
    for n in T:
        tree += tree_words([-1] + [rng.randrange(i) for i in range(1, n)])
    pg = Pages([2 * pt + n for n in (61, 90, 128, 500)], hkv, d, pt, shared=2)
    dense(pg, T, heads, tree=tree)


def test_masks_that_leave_a_row_empty():
    tree = tree_words([-1, 0, 0, 1])
    tree[2] = [0, 0, 0, 0]
    pg = Pages([4, 20], 2, 64, 16)
    out, lse = dense(pg, [4, 4], 4, tree=tree + tree)
    assert (out[2] == 0).all() and torch.isinf(lse[2]).all()


@pytest.mark.parametrize("n_seqs", [1, 31, 200])
def test_many_sequences_of_odd_lengths(n_seqs):
    rng = random.Random(n_seqs)
    pg = Pages([128 + rng.randrange(1, 200) for _ in range(n_seqs)], 2, 64, 32, shared=4)
    dense(pg, [1] * n_seqs, 4)


def test_long_context_few_rows():
    pg = Pages([20001], 2, 128, 64)
    dense(pg, [1], 8)
    pg = Pages([16384 + 5, 16384 + 64], 1, 64, 128, shared=128)
    dense(pg, [1, 3], 2)


def test_many_rows_over_the_prefix():
    pg = Pages([1024 + n for n in (130, 257, 391)], 2, 128, 64, shared=16)
    dense(pg, [130, 257, 391], 4)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_peaked_rows_and_growing_maxima(dtype):
    """Scores of up to a few hundred, which rise along the keys, so that the softmax's reference moves again and again."""
    pg = Pages([700], 1, 64, 64, dtype, gain=0.3)
    ramp = torch.linspace(0, 6, 704, device="cuda").view(-1, 64)
    for j in range(11):
        n = min(64, 700 - 64 * j)
        pg.k[int(pg.table[0, j]), 0, :n] += ramp[j, :n, None].to(pg.k.dtype)
    dense(pg, [3], 4, gain=4.0, spread=400.0)


def test_scale_and_values_of_the_largest_size():
    pg = Pages([100], 1, 64, 32)
    dense(pg, [2], 2, scale=1e-4)
    dense(pg, [2], 2, scale=2.0, spread=100.0)
    pg.v *= 1e30
    dense(pg, [2], 2)


def test_strided_rows():
    from paper_2505_19201_b200 import api
    pg = Pages([90, 33], 2, 64, 16)
    fused = torch.randn(5, 4 + 2 * 2, 64, device="cuda").bfloat16()
    q, big = fused[:, :4], torch.full((5, 7, 64), 5.0, device="cuda").bfloat16()
    out = big[:, 1:5]
    start = [0, 3, 5]
    api.dream_cache_attn(pg.cache, q, torch.tensor(start, dtype=torch.int32, device="cuda"), torch.tensor([90, 33], dtype=torch.int32, device="cuda"), out,
                         workspace(pg, 5, 4))
    want, _, size = dense_reference(pg, q, start)
    close(out, want, size, "bf16")
    assert (big[:, 0] == 5).all() and (big[:, 5:] == 5).all()


def test_the_same_bits_at_every_run():
    pg = Pages([640 + n for n in (5, 100, 260)], 2, 128, 64, shared=10)
    from paper_2505_19201_b200 import api
    q = pg.queries(9, 8)
    args = torch.tensor([0, 1, 5, 9], dtype=torch.int32, device="cuda"), torch.tensor(pg.lengths, dtype=torch.int32, device="cuda")
    got = []
    for _ in range(3):
        out = torch.empty_like(q)
        api.dream_cache_attn(pg.cache, q, *args, out, workspace(pg, 9, 8), shared_pages=10)
        got.append(out)
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_numbers_out_of_range_are_left_out():
    """A page number that is none, and a length past the table: the kernels' own checks turn them into a status, nothing is read there."""
    from paper_2505_19201_b200 import api
    pg = Pages([200], 2, 64, 64)
    pg.table[0, 1] = 10 ** 6
    q, status = pg.queries(1, 4), torch.zeros(2, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(q)
    start = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    api.dream_cache_attn(pg.cache, q, start, torch.tensor([200], dtype=torch.int32, device="cuda"), out, workspace(pg, 1, 4), status=status)
    k, v = pg.context(0, list(range(64)) + list(range(128, 200)))
    from .util_cache import attend
    want, _, size = attend(q, k, v, torch.ones(1, 136, dtype=torch.bool, device="cuda"), 0.125)
    close(out, want, size, "bf16")
    assert status[0] == 2
    status.zero_()
    api.dream_cache_attn(pg.cache, q, start, torch.tensor([10 ** 9], dtype=torch.int32, device="cuda"), out, workspace(pg, 1, 4), status=status)
    assert status[0] == 2


# ---------------------------------------------------------------------------------- selected pages

def some_ids(pg, row_seq, row_pos, budget, rng):
    ids = []
    for s, p in zip(row_seq, row_pos):
        row = []
        for _ in range(pg.hkv):
            own = p // pg.pt
            some = sorted(rng.sample(range(own), min(own, budget - 1))) + [own] if s >= 0 and p >= 0 else []
            row.append(some + [-1] * (budget - len(some)))
        ids.append(row)
    return ids


def paged(pg, row_seq, row_pos, ids, heads, gain=1.0):
    from paper_2505_19201_b200 import api
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    R = len(row_seq)
    q = pg.queries(R, heads, gain)
    out, lse, status = torch.full_like(q, 77.0), torch.full((R, heads), 77.0, device="cuda"), i32([0, 0])
    ids = i32(ids)
    api.dream_cache_attn_pages(pg.cache, q, i32(row_seq), i32(row_pos), ids, out, workspace(pg, R, heads), lse=lse, status=status)
    want, wl, size = pages_reference(pg, q, row_seq, row_pos, ids)
    real = torch.tensor([s >= 0 for s in row_seq], device="cuda")
    close(out[real], want[real], size[real], pg.dtype)
    close_lse(lse[real], wl[real])
    assert (out[~real] == 77.0).all() and (lse[~real] == 77.0).all()
    assert status.tolist() == [0, 0]
    return out, lse


@pytest.mark.parametrize("heads,hkv,d", MODELS)
@pytest.mark.parametrize("dtype,pt,budget", [("bf16", 64, 5), ("f16", 16, 9), ("bf16", 256, 2), ("bf16", 32, 3), ("f16", 128, 1)])
def test_pages(heads, hkv, d, dtype, pt, budget):
    rng = random.Random(pt + d)
    pg = Pages([1, 700, 16 * pt, 16 * pt - 3], hkv, d, pt, dtype, layout=rng.choice(["hnd", "nhd", "room"]), seed=pt)
    seqs, pos = [0, 1, 1, 2, 3, 3, -1], [0, 699, 650, 16 * pt - 1, 16 * pt - 4, pt, 5]
    paged(pg, seqs, pos, some_ids(pg, seqs, pos, budget, rng), heads)


def test_pages_of_a_programs_own_choice():
    pg = Pages([640, 640], 2, 64, 64)
    lists = [[[0, 3, 9, -1], [1, 2, 3, 4]], [[5, -1, -1, -1], [-1, -1, -1, -1]], [[2, 2, 7, 7], [9, 1, 3, -1]], [[0, 1, 8, 9], [8, 9, 20, 30]]]
    seqs, pos = [0, 1, 0, 1], [639, 400, 600, 520]
    out, lse = paged(pg, seqs, pos, lists, 4)
    assert (out[1, 2:] == 0).all() and torch.isinf(lse[1, 2:]).all()
    paged(pg, [0, 0], [-1, 63], [[[0, 1, -1, -1]] * 2] * 2, 4)           # a row without a place, a row on a page's last token


def test_pages_long_lists():
    rng = random.Random(1)
    pg = Pages([40000], 1, 128, 16)
    paged(pg, [0], [39990], some_ids(pg, [0], [39990], 1000, rng), 4)


def test_pages_all_of_them_is_the_dense_call():
    from paper_2505_19201_b200 import api
    pg = Pages([500, 300], 2, 128, 64)
    q = pg.queries(2, 8)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    a, b, w = torch.empty_like(q), torch.empty_like(q), workspace(pg, 2, 8)
    api.dream_cache_attn(pg.cache, q, i32([0, 1, 2]), i32(pg.lengths), a, w)
    ids = i32([[[j if j * 64 < n else -1 for j in range(9)]] * 2 for n in pg.lengths])
    api.dream_cache_attn_pages(pg.cache, q, i32([0, 1]), i32([499, 299]), ids, b, w)
    want, _, size = dense_reference(pg, q, [0, 1, 2])
    close(a, want, size, "bf16")
    close(b, want, size, "bf16")


def test_page_numbers_out_of_range_in_pages():
    from paper_2505_19201_b200 import api
    pg = Pages([256], 1, 64, 64)
    pg.table[0, 2] = -3
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q, status = pg.queries(1, 2), i32([0, 0])
    out = torch.zeros_like(q)
    api.dream_cache_attn_pages(pg.cache, q, i32([0]), i32([255]), i32([[[0, 2, 3]]]), out, workspace(pg, 1, 2), status=status)
    want, _, size = pages_reference(pg, q, [0], [255], i32([[[0, 3]]]))
    close(out, want, size, "bf16")
    assert status[0] == 2
    for seq, pos in ((5, 10), (0, 10 ** 6)):
        status.zero_()
        api.dream_cache_attn_pages(pg.cache, q, i32([seq]), i32([pos]), i32([[[0, 1, 3]]]), out, workspace(pg, 1, 2), status=status)
        assert status[0] == 2 and (out == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_types_are_the_caches(dtype):
    assert Pages([5], 1, 64, 16, dtype).queries(1, 1).dtype is TYPES[dtype]
