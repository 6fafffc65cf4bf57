"""Rows and settings at which dream_sample and dream_truncate_logits could go wrong by a rounding, against the definition in float64.  Tokens,
kept counts and kept sets are equal, not close; logprob within what tests/test_gpu_sample.py derives."""
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
