"""Calls on a paged cache that are too large to be counted, refused without a GPU."""
import pytest

from .test_cache_refusals import E_CAPACITY, attn, cache


def call(rows, group, hkv, pages, pt, n_seqs=1, shared=0):
    c = cache(n_kv_heads=hkv, page_tokens=pt, pages_per_seq=pages, table_stride=pages, n_seqs=n_seqs, head_stride=256 * 128, page_stride=256 * 128 * hkv)
    h = hkv * group
    return attn(c, heads=h, q_ld=h * 128, out_ld=h * 128, rows=rows, out=1 << 50, shared=shared, n=1 << 60)


@pytest.mark.parametrize("rows,group,hkv,pages,pt,n_seqs", [(1 << 20, 128, 1, 1 << 22, 256, 1), (1 << 20, 64, 8, 1 << 19, 256, 1), (4096, 1, 64, 1 << 21, 256, 4096), (4096, 4, 32, 1 << 22, 256, 4096)])
def test_units_of_a_block_that_are_not_counted_in_32_bits(rows, group, hkv, pages, pt, n_seqs):
    """So many tiles, each against so long a sequence; a table may well name one page over and over."""
    assert call(rows, group, hkv, pages, pt, n_seqs) == E_CAPACITY
