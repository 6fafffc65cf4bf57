"""What the calls on a paged cache refuse, without a GPU: every check comes before anything is enqueued."""
import ctypes as C

import pytest
import torch

E_ARG, E_NOMEM, E_CAPACITY, E_UNSUPPORTED = -1, -3, -4, -7
A, B, W, I = 1 << 20, 1 << 40, 1 << 41, 1 << 42              # addresses nobody looks at


def _api():
    from paper_2505_19201_b200 import api, build
    build.build()
    api.lib()
    return api


def cache(**over):
    f = dict(k=B, v=B + (1 << 30), bounds=B + (1 << 31), page_table=I, page_stride=2 * 64 * 128, head_stride=64 * 128, token_stride=128, table_stride=40,
             dtype=1, n_pages=50, page_tokens=64, n_kv_heads=2, head_dim=128, n_seqs=3, pages_per_seq=40)
    f.update(over)
    return _api().dream_cache(**f)


def ptr(x):
    return C.c_void_p(x) if x else None


def ref(c):
    return C.byref(c) if c is not None else None


def append(c, q=A, q_ld=1024, heads=8, k=A, k_ld=256, v=A, v_ld=256, rows=4, seq=I, slots=I, pos=None, rope=B, n_pos=10, rot=128, q_out=W, out_ld=1024, status=None):
    return _api().lib().dream_cache_append(ref(c), ptr(q), q_ld, heads, ptr(k), k_ld, ptr(v), v_ld, rows, ptr(seq), ptr(slots), ptr(pos), ptr(rope), n_pos, rot, 0,
                                           ptr(q_out), out_ld, ptr(status), None)


def attn(c, q=A, q_ld=1024, heads=8, rows=4, start=I, lens=I, shared=0, tree=None, scale=1.0, out=W, out_ld=1024, lse=None, ws=W << 1, n=1 << 40, status=None):
    return _api().lib().dream_cache_attn(ref(c), ptr(q), q_ld, heads, rows, ptr(start), ptr(lens), shared, ptr(tree), scale, ptr(out), out_ld, ptr(lse), ptr(ws), n,
                                         ptr(status), None)


def select(c, q=A, q_ld=1024, heads=8, rows=4, seq=I, pos=I, budget=8, first=1, last=1, ids=I, ws=W << 1, n=1 << 40, status=None):
    return _api().lib().dream_cache_select(ref(c), ptr(q), q_ld, heads, rows, ptr(seq), ptr(pos), budget, first, last, ptr(ids), ptr(ws), n, ptr(status), None)


def pages(c, q=A, q_ld=1024, heads=8, rows=4, seq=I, pos=I, ids=I, budget=8, scale=1.0, out=W, out_ld=1024, lse=None, ws=W << 1, n=1 << 40, status=None):
    return _api().lib().dream_cache_attn_pages(ref(c), ptr(q), q_ld, heads, rows, ptr(seq), ptr(pos), ptr(ids), budget, scale, ptr(out), out_ld, ptr(lse), ptr(ws), n,
                                               ptr(status), None)


CALLS = [append, attn, select, pages]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("bad,code", [
    (dict(k=None), E_ARG), (dict(v=None), E_ARG), (dict(page_table=None), E_ARG), (dict(page_table=I + 2), E_ARG), (dict(k=B + 8), E_ARG), (dict(bounds=B + 2), E_ARG),
    (dict(dtype=0), E_UNSUPPORTED), (dict(dtype=3), E_UNSUPPORTED), (dict(head_dim=96), E_UNSUPPORTED), (dict(page_tokens=8), E_UNSUPPORTED),
    (dict(page_tokens=48), E_UNSUPPORTED), (dict(page_tokens=512), E_UNSUPPORTED), (dict(n_pages=0), E_ARG), (dict(n_seqs=0), E_ARG), (dict(n_kv_heads=0), E_ARG),
    (dict(pages_per_seq=0), E_ARG), (dict(n_seqs=4097), E_CAPACITY), (dict(pages_per_seq=1 << 25, table_stride=1 << 25), E_CAPACITY), (dict(table_stride=39), E_ARG),
    (dict(token_stride=132), E_ARG), (dict(token_stride=0), E_ARG), (dict(token_stride=64), E_ARG), (dict(head_stride=-8192), E_ARG), (dict(head_stride=8000), E_ARG),
    (dict(page_stride=8192), E_ARG), (dict(page_stride=2 * 64 * 128 - 8), E_ARG)])
def test_cache(call, bad, code):
    assert call(cache(**bad)) == code
    assert _api().lib().dream_last_error(None)


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("bad,code", [(dict(rows=0), E_ARG), (dict(rows=-3), E_ARG), (dict(rows=(1 << 20) + 1), E_CAPACITY), (dict(heads=0), E_ARG), (dict(heads=3), E_ARG),
                                      (dict(heads=258, q_ld=258 * 128), E_UNSUPPORTED), (dict(q=None), E_ARG), (dict(q=A + 8), E_ARG), (dict(q_ld=1016), E_ARG),
                                      (dict(q_ld=1028), E_ARG), (dict(status=I + 1), E_ARG), (dict(seq=None), E_ARG), (dict(seq=I + 1), E_ARG)])
def test_rows(call, bad, code):
    if call is attn and "seq" in bad:
        bad = {"start": bad["seq"]}
    assert call(cache(), **bad) == code


@pytest.mark.parametrize("call,bad,code", [
    (append, dict(k=None), E_ARG), (append, dict(v=None), E_ARG), (append, dict(k_ld=255), E_ARG), (append, dict(v_ld=248), E_ARG), (append, dict(slots=None), E_ARG),
    (append, dict(pos=I + 3), E_ARG), (append, dict(rope=B + 8), E_ARG), (append, dict(n_pos=0), E_ARG), (append, dict(rot=0), E_ARG), (append, dict(rot=24), E_ARG),
    (append, dict(rot=144), E_ARG), (append, dict(q_out=None), E_ARG), (append, dict(q=None, q_out=None), E_ARG), (append, dict(q_out=A + 2048), E_ARG),
    (append, dict(q_out=A, out_ld=2048), E_ARG), (append, dict(out_ld=1000), E_ARG),
    (attn, dict(lens=None), E_ARG), (attn, dict(shared=-1), E_ARG), (attn, dict(shared=41), E_ARG), (attn, dict(tree=I + 1), E_ARG), (attn, dict(scale=0.0), E_ARG),
    (attn, dict(scale=-1.0), E_ARG), (attn, dict(scale=float("nan")), E_ARG), (attn, dict(scale=float("inf")), E_ARG), (attn, dict(out=None), E_ARG),
    (attn, dict(out=A), E_ARG), (attn, dict(out=A + 1024), E_ARG), (attn, dict(out_ld=1016), E_ARG), (attn, dict(lse=I + 1), E_ARG), (attn, dict(ws=None), E_ARG),
    (attn, dict(ws=W + 16), E_ARG), (attn, dict(n=0), E_NOMEM),
    (select, dict(pos=None), E_ARG), (select, dict(ids=None), E_ARG), (select, dict(budget=1), E_ARG), (select, dict(first=-1), E_ARG), (select, dict(last=0), E_ARG),
    (select, dict(first=2000000000, last=2000000000), E_ARG), (select, dict(budget=4097), E_CAPACITY), (select, dict(ws=None), E_ARG), (select, dict(n=100), E_NOMEM),
    (pages, dict(pos=None), E_ARG), (pages, dict(ids=None), E_ARG), (pages, dict(budget=0), E_ARG), (pages, dict(budget=4097), E_CAPACITY), (pages, dict(scale=0.0), E_ARG),
    (pages, dict(out=A), E_ARG), (pages, dict(n=0), E_NOMEM)])
def test_the_other_arguments(call, bad, code):
    assert call(cache(), **bad) == code


def test_selection_needs_bounds_and_has_room_for_so_many_pages():
    assert select(cache(bounds=None)) == E_ARG
    assert select(cache(pages_per_seq=32769, table_stride=32769)) == E_CAPACITY
    assert all(call(None) == E_ARG for call in CALLS)


@pytest.mark.parametrize("over,rows", [(dict(page_tokens=256, pages_per_seq=1 << 22, n_kv_heads=64), 129), (dict(page_tokens=256, pages_per_seq=1 << 22, n_kv_heads=128), 1),
                                       (dict(page_tokens=16, pages_per_seq=1 << 23, n_kv_heads=2), 1 << 20)])
def test_work_that_is_not_counted_in_32_bits(over, rows):
    """A prefix of so many keys in so many tiles; a table may well name one page over and over."""
    h = over["n_kv_heads"]
    c = cache(**over, table_stride=1 << 23, head_stride=256 * 128, page_stride=256 * 128 * h)
    assert attn(c, heads=h, q_ld=h * 128, out_ld=h * 128, rows=rows, out=1 << 50, shared=over["pages_per_seq"], n=1 << 60) == E_CAPACITY


def test_strides_that_nothing_steps_along_do_not_count():
    n = C.c_size_t()
    for ok in (dict(n_pages=1, page_stride=0), dict(n_kv_heads=1, head_stride=-5), dict(n_seqs=1, table_stride=0), dict(page_stride=128, token_stride=50 * 128, head_stride=64 * 50 * 128)):
        assert _api().lib().dream_cache_attn_bytes(ref(cache(**ok)), 8, 4, C.byref(n)) == 0 and n.value > 0
    assert _api().lib().dream_cache_attn_bytes(ref(cache()), 8, 4, None) == E_ARG and _api().lib().dream_cache_select_bytes(ref(cache()), 4, None) == E_ARG


@pytest.mark.parametrize("bad", [dict(n_pos=0), dict(rot=8), dict(rot=24), dict(rot=272), dict(theta=0.0), dict(theta=float("inf")), dict(theta=float("nan")),
                                 dict(table=None), dict(table=A + 4)])
def test_rope_table(bad):
    f = dict(table=A, n_pos=5, rot=64, theta=1e4)
    f.update(bad)
    assert _api().lib().dream_rope_table(ptr(f["table"]), f["n_pos"], f["rot"], f["theta"], None) == E_ARG


def test_wrappers_name_what_is_wrong():
    api = _api()
    k, t = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(1, 4, dtype=torch.int32)
    for args, name in (((None, k, t), "k"), ((k, None, t), "v"), ((k, k, None), "page_table"), ((k.float(), k, t), "k"), ((k[0], k[0], t), "k"), ((k, k, t), "CUDA")):
        with pytest.raises(api.DreamError) as e:
            api.Cache(*args)
        assert e.value.code == E_ARG and name in str(e.value)
    for call in (lambda: api.dream_cache_append(None, None, k, k, t, t, None), lambda: api.dream_cache_attn(k, k, t, t, k, k),
                 lambda: api.dream_cache_select(k, k, t, t, t, k), lambda: api.dream_cache_attn_pages(k, k, t, t, t, k, k),
                 lambda: api.dream_cache_attn_bytes(k, 1, 1), lambda: api.dream_cache_select_bytes(k, 1)):
        with pytest.raises(api.DreamError) as e:
            call()
        assert e.value.code == E_ARG and "Cache" in str(e.value)
    for bad in (None, torch.zeros(3, 8, 2), torch.zeros(3, 8), torch.zeros(3, 8, 2).double()):
        with pytest.raises(api.DreamError) as e:
            api.dream_rope_table(bad)
        assert e.value.code == E_ARG
