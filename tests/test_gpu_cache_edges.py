"""Calls on a paged cache at the edges of what they allow."""
import pytest

from .test_gpu_cache_attn import dense
from .util_cache import Pages, tree_words

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
