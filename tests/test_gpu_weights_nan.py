"""Accumulated weights where a query, a key or a log sum-exp is no number: what a row does not see, and what rows without
a log sum-exp bring, is not touched by it."""
import math

import pytest
import torch

import chunk_ref as ref
from paper_2502_14051_amd import rocketkv as rk

pytestmark = pytest.mark.gpu
NAN, INF = math.nan, math.inf


def check(c, lse, w_in):
    """Against the definition: keys that are NaN there are NaN here, and no others."""
    got = torch.full((len(c.lens), c.hkv, c.cache.pages_cap * c.ps), -5.0, device="cuda")
    rk.accumulate_weights(c.cache, c.chunk, c.q, lse, w_in, got)
    G, spoilt = c.hq // c.hkv, 0
    for b, (n, new) in enumerate(zip(c.lens, c.news)):
        here = c.present(b)
        pos = n - new + torch.arange(new, device="cuda")
        seen = (torch.arange(n, device="cuda")[None, :] <= pos[:, None]) & here[None, :]
        for g in range(c.hkv):
            w, lim = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
            w[:n - new] = w_in[b, g, :n - new].double()
            for h in range(g * G, (g + 1) * G):
                q, k = c.q[c.rows_of(b), h].double(), c.K[b, g, :n].double()
                l = lse[c.rows_of(b), h].double()[:, None]
                adds = seen & (l != -INF)
                p = torch.where(adds, torch.exp(q @ k.T / math.sqrt(ref.D) - l), 0.0)
                rel = ref.EPS[torch.float32] * (136 * (q.abs() @ k.abs().T / math.sqrt(ref.D)) + 4 * l.abs() + 64)
                w += p.sum(0)
                lim += torch.where(p > 0, p * rel, 0.0).sum(0)
            lim += ref.EPS[torch.float32] * (G * new / 16 + 64) * w.abs()
            nan = torch.isnan(w)
            spoilt += int(nan.sum())
            assert torch.equal(torch.isnan(got[b, g, :n]), nan), f"sequence {b}, head {g}: {int((torch.isnan(got[b, g, :n]) & ~nan).sum())} keys too many"
            assert ((got[b, g, :n].double() - w).abs() <= lim + 1e-37)[~nan].all()
        assert (got[b, :, n:] == -5).all()
    return spoilt


def case(seed, lens, news, **kw):
    c = ref.Case(seed, lens, news, 8, 2, shuffled=False, **kw)
    lse = ref.attention(c)[1].float()
    return c, lse, torch.rand((len(lens), 2, c.cache.pages_cap * 16), generator=torch.Generator().manual_seed(seed)).cuda()


# many rows; few rows; rows that end inside a step and keys that begin inside one
SHAPES = [([700], [130]), ([700, 64], [3, 1]), ([90], [90]), ([400, 257], [150, 77]), ([5000], [33])]


@pytest.mark.parametrize("lens,news", SHAPES)
@pytest.mark.parametrize("bad", [NAN, INF])
def test_a_log_sum_exp(lens, news, bad):
    """NaN spoils what the row sees and nothing behind it; a row of infinite sum has no weight to give."""
    c, lse, w = case(70, lens, news)
    for b, new in enumerate(news):
        for i in {0, new // 2}:
            lse[c.starts[b] + i, 2 + b] = bad
    spoilt = check(c, lse, w)
    assert (spoilt > 0) == math.isnan(bad)


@pytest.mark.parametrize("lens,news", SHAPES)
@pytest.mark.parametrize("bad", [NAN, INF])
def test_rows_without_one_add_nothing(lens, news, bad):
    """Whatever their queries are."""
    c, lse, w = case(71, lens, news, pad=(0, 2))
    for b, new in enumerate(news):
        for i in {0, new // 2, new - 1}:
            c.q[c.starts[b] + i, 1 + b, 5:70] = bad
            lse[c.starts[b] + i, 1 + b] = -INF
    assert check(c, lse, w) == 0


@pytest.mark.parametrize("lens,news", SHAPES)
@pytest.mark.parametrize("bad", [NAN, INF])
def test_nor_do_they_to_keys_that_are_not_finite(lens, news, bad):
    c, lse, w = case(72, lens, news)
    for b, (n, new) in enumerate(zip(lens, news)):
        for t in {0, n // 3, n - 1}:
            c.cache.k_pool[b * c.cache.pages_cap + t // 16, :, t % 16, 3:60] = bad
            c.K[b, :, t, 3:60] = bad
    lse[:] = -INF
    assert check(c, lse, w) == 0


@pytest.mark.parametrize("lens,news", SHAPES)
def test_a_key(lens, news):
    """It is spoilt if a row sees it, and it alone."""
    c, lse, w = case(73, lens, news)
    for b, (n, new) in enumerate(zip(lens, news)):
        for t in {0, n // 3, n - 1}:
            c.cache.k_pool[b * c.cache.pages_cap + t // 16, :, t % 16, 9] = NAN
            c.K[b, :, t, 9] = NAN
    assert check(c, lse, w) > 0


@pytest.mark.parametrize("lens,news,ps,token_major", [([18000], [40], 16, False), ([18000, 900], [200, 3], 3, True), ([300, 50], [5, 1], 5, True),
                                                      ([9000, 9500], [70, 130], 64, True)])
def test_all_of_them_over_scattered_pages(lens, news, ps, token_major):
    """Whole tiles of keys and halves of them, with pages absent."""
    c = ref.Case(74, lens, news, 8, 2, ps, token_major, pad=(1, 1))
    lse = ref.attention(c)[1].float()
    w = torch.rand((len(lens), 2, c.cache.pages_cap * ps), generator=torch.Generator().manual_seed(74)).cuda()
    for b, (n, new) in enumerate(zip(lens, news)):
        first = c.starts[b]
        lse[first + new // 2, 3] = NAN
        c.q[first, 6], lse[first, 6] = INF, -INF
        c.q[first + new - 1, 5], lse[first + new - 1, 5] = NAN, -INF
        for t, bad in ((n // 5, NAN), (n // 2, INF), (n - 1, NAN)):
            c.cache.k_pool[c.cache.block_table[b, t // ps].long(), 0, t % ps, 77] = bad
            c.K[b, 0, t, 77] = bad
    c.drop_pages([(0, 1), (0, lens[0] // (3 * ps)), (len(lens) - 1, 2)])
    assert check(c, lse, w) > 0
