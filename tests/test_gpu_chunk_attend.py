"""Attention of a chunk of new tokens over the paged cache, against its definition in 64 bits."""
import pytest
import torch

import chunk_ref as ref
from paper_2502_14051_amd import rocketkv as rk

pytestmark = pytest.mark.gpu


def attend(c, ws=None, lse=True, fill=7.0):
    out = torch.full((c.rows, c.hq, ref.D), fill, dtype=torch.bfloat16, device="cuda")
    out_lse = torch.full((c.rows, c.hq), fill, device="cuda") if lse else None
    if ws is None:
        ws = rk.alloc_workspace(rk.OP_CHUNK_ATTEND, c.cache, c.rows)
    rk.chunk_attend(c.cache, c.chunk, c.q, out, out_lse, ws)
    return out, out_lse


LAYOUTS = [(16, False), (1, True), (3, True), (4, True), (16, True), (64, True)]


@pytest.mark.parametrize("ps,token_major", LAYOUTS)
@pytest.mark.parametrize("lens,news", [
    ([1], [1]),                                   # one token of one
    ([64], [64]), ([65], [65]), ([63], [1]),      # around a step of keys
    ([700, 1, 33, 500], [1, 1, 33, 37]),          # single tokens, a whole prompt and a piece of one
    ([1500, 130], [300, 130]),                    # several tiles of rows
    ([400, 300, 0, 200], [0, 20, 0, 1]),          # sequences without new tokens, and without any
])
def test_lengths(ps, token_major, lens, news):
    c = ref.Case(1, lens, news, 8, 2, ps, token_major)
    ref.check_attention(c, *attend(c))


@pytest.mark.parametrize("token_major", [False, True])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (5, 1), (16, 1), (12, 4), (40, 8), (7, 7)])
@pytest.mark.parametrize("new", [1, 9, 70])
def test_groups(token_major, hq, hkv, new):
    c = ref.Case(2, [300, 171], [new, max(1, new // 2)], hq, hkv, 16, token_major)
    ref.check_attention(c, *attend(c))


@pytest.mark.parametrize("ps,token_major", [(16, False), (5, True)])
@pytest.mark.parametrize("lens,news", [([9000], [3]), ([9000], [70]), ([9001, 40, 5000], [1, 5, 4]), ([20000, 19000], [130, 1])])
def test_long_caches_cut(ps, token_major, lens, news):
    """Few rows over many keys: every tile's keys are cut, the parts merged."""
    c = ref.Case(3, lens, news, 4, 1, ps, token_major)
    ref.check_attention(c, *attend(c))


def test_many_sequences():
    """More than one sequence a lane in the division, most of them short."""
    lens = [1 + (37 * b) % 90 for b in range(150)]
    news = [0 if b % 7 == 3 else 1 + (b * 11) % lens[b] if b % 5 == 0 else 1 for b in range(150)]
    c = ref.Case(4, lens, news, 4, 2)
    ref.check_attention(c, *attend(c))


@pytest.mark.parametrize("news,lens", [([1100], [2000]), ([640, 700], [700, 1500]), ([2200], [2300]), ([300, 3, 400], [900, 1400, 400])])
def test_tiles_beside_the_chip(news, lens):
    """From 100 to 290 tiles of 256 rows beside 256 workgroups at a time: cut for one round, for three, or not at all."""
    c = ref.Case(5, lens, news, 32, 8)
    ref.check_attention(c, *attend(c))


@pytest.mark.parametrize("ps,token_major", [(16, False), (4, True)])
def test_caches_beyond_the_last_level(ps, token_major):
    """More room than 256 MiB and few rows: the form that reads past the caches."""
    c = ref.Case(7, [700, 5000, 1], [3, 20, 1], 8, 2, ps, token_major, spare_pages=100000 // ps)
    ref.check_attention(c, *attend(c))


def test_one_workspace_for_all():
    """A workspace that is used for other calls before and after, of other sizes."""
    ws = rk.alloc_workspace(rk.OP_CHUNK_ATTEND, ref.Case(6, [10], [1], 2, 1).cache, 1)
    for lens, news in (([9000], [70]), ([40], [40]), ([9000, 9000], [1, 300]), ([5000], [3])):
        c = ref.Case(6, lens, news, 4, 1)
        ref.check_attention(c, *attend(c, ws))


def test_large_logits():
    """Maxima that move by hundreds from step to step, and rows that one key dominates."""
    c = ref.Case(5, [1000, 600], [150, 3], 8, 2, scale=6.0)
    ref.check_attention(c, *attend(c))


@pytest.mark.parametrize("token_major", [False, True])
def test_absent_pages_and_rows_of_nobody(token_major):
    c = ref.Case(6, [600, 90, 16], [100, 90, 16], 8, 2, 16, token_major, pad=(3, 5))
    c.drop_pages([(0, 0), (0, 7), (0, 31), (0, 36), (1, 0), (1, 1), (2, 0)])  # sequence 1 begins with rows that see nothing
    # whatever lies where no token is must not matter
    free = sorted(set(range(c.cache.k_pool.shape[0])) - set(c.cache.block_table.flatten().tolist()))
    c.cache.k_pool[free], c.cache.v_pool[free] = float("nan"), float("nan")
    out, lse = attend(c)
    ref.check_attention(c, out, lse)
    assert (out[c.rows_of(2)] == 0).all() and torch.isneginf(lse[c.rows_of(2)]).all()
    for r in list(range(3)) + list(range(c.rows - 5, c.rows)):
        assert (out[r] == 7).all() and (lse[r] == 7).all(), "rows of no sequence are left as they were"


@pytest.mark.parametrize("token_major", [False, True])
def test_garbage_behind_the_end(token_major):
    """Slots of the last page behind the sequence, and pages that are listed but not reached, hold NaN."""
    c = ref.Case(7, [35, 100], [35, 2], 4, 1, 16, token_major, shuffled=False, spare_pages=8)
    for b, n in enumerate(c.lens):
        first, cap = b * c.cache.pages_cap, c.cache.pages_cap
        c.cache.k_pool[first + n // 16, :, n % 16:] = float("nan")
        if token_major:
            c.cache.v_pool[first + n // 16, :, n % 16:] = float("inf")
        else:
            c.cache.v_pool[first + n // 16, :, :, n % 16:] = float("nan")
        c.cache.k_pool[first + n // 16 + 1:first + cap] = float("nan")
        c.cache.v_pool[first + n // 16 + 1:first + cap] = float("nan")
    c.cache.k_pool[-5:], c.cache.v_pool[-5:] = float("nan"), float("nan")
    ref.check_attention(c, *attend(c))


def test_future_keys_that_are_not_finite():
    """A key of a row's future may be anything."""
    c = ref.Case(8, [80], [40], 4, 1, 4, True, shuffled=False)
    c.cache.k_pool[60 // 4:, :] = float("nan")
    c.cache.k_pool[62 // 4, :, 1] = float("inf")
    out, lse = attend(c)
    seen = 20  # rows of tokens 40 .. 59
    want = ref.Case(8, [60], [20], 4, 1, 4, True, shuffled=False)
    want.K, want.V, want.q = c.K[:, :, :60], c.V[:, :, :60], c.q[:20]
    ref.check_attention(want, out[:seen], lse[:seen])


@pytest.mark.parametrize("ps,token_major", [(16, False), (4, True)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("lens,news", [([90], [70]), ([300, 70], [200, 3])])
def test_future_values_that_are_not_finite(ps, token_major, bad, lens, news):
    """Rows in front of such a token do not notice it; rows behind it carry what the formula gives."""
    c = ref.Case(16, lens, news, 4, 2, ps, token_major, shuffled=False)
    where = {0: [lens[0] - 40, lens[0] - 39, lens[0] - 9], 1: []}
    if len(lens) > 1:
        where[1] = [lens[1] - 1]
    clean, clean_lse = attend(c)
    want, _, _, _ = ref.attention(c)
    for b, tokens in where.items():
        for n, t in enumerate(tokens):
            at = b * c.cache.pages_cap + t // ps
            if token_major:
                c.cache.v_pool[at, :, t % ps, n::7] = bad
            else:
                c.cache.v_pool[at, :, n::7, t % ps] = bad
    out, lse = attend(c)
    assert torch.equal(lse, clean_lse)
    for b, n in enumerate(lens):
        for i in range(news[b]):
            row = c.starts[b] + i
            hit = torch.zeros(128, dtype=torch.bool, device="cuda")
            for k, t in enumerate(where[b]):
                if t <= n - news[b] + i:
                    hit[k::7] = True
            assert (~torch.isfinite(out[row][:, hit])).all()
            assert torch.equal(out[row][:, ~hit], clean[row][:, ~hit]), f"sequence {b}, row {i}"


@pytest.mark.parametrize("token_major", [False, True])
def test_pools_beyond_32_bits(token_major):
    """All of the operators over pools of more than 4 GiB, at their far ends too, beside small pools of the same tokens."""
    c = ref.Case(17, [500, 70], [100, 1], 8, 2, 16, token_major, shuffled=False, spare_pages=16)
    small = c.cache
    pages = (5 << 30) // (2 * 16 * 128 * 2)
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(0))[:2 * small.pages_cap]
    table[0], table[1], table[35], table[40] = pages - 1, 0, pages - 3, pages - 2
    assert len(set(table.tolist())) == len(table)
    big = rk.alloc_cache(2, 8, 2, 128, 16, small.pages_cap, "cuda", block_table=table.reshape(2, -1).to(torch.int32).cuda(),
                         n_phys_pages=pages, v_layout=small.v_layout)
    at = table.cuda()
    big.k_pool[at], big.v_pool[at] = small.k_pool[:len(at)], small.v_pool[:len(at)]
    big.seq_lens.copy_(small.seq_lens)
    r = rk.Rope(torch.ones(64, dtype=torch.float64, device="cuda") / 100)
    results = []
    for cache in (small, big):
        kmax, kmin = rk.alloc_summaries(cache)
        rk.build_page_summaries(cache, kmax, kmin)
        k = torch.randn((c.rows, 2, 128), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
        rk.append_chunk(cache, c.chunk, k, k, kmax, kmin, rk.alloc_workspace(rk.OP_APPEND_CHUNK, cache, c.rows), rope=r)
        c.cache = cache
        out, lse = attend(c)
        w = rk.alloc_weights(cache)
        rk.accumulate_weights(cache, c.chunk, c.q, lse, None, w)
        dst = rk.alloc_cache(2, 8, 2, 128, 16, 16, "cuda", zero=True, v_layout=cache.v_layout)
        rk.weight_evict(cache, w, 8, 200, dst, None, None, rk.alloc_workspace(rk.OP_WEIGHT_EVICT, cache, 8, 200))
        results.append([kmax, kmin, cache.seq_lens, out, lse, w, dst.k_pool, dst.v_pool, dst.seq_lens])
    for i, (a, b) in enumerate(zip(*results)):
        assert torch.equal(a, b), f"result {i}"
    K, V = rk.unpack_cache(small)
    c.K, c.V, c.lens = K, V, [n + m for n, m in zip(c.lens, c.news)]
    ref.check_attention(c, *results[1][3:5])


def test_more_new_tokens_than_the_cache_holds():
    """Rows in front of the cache's first token see nothing."""
    c = ref.Case(9, [10], [25], 4, 1)
    out, lse = attend(c)
    ref.check_attention(c, out, lse)
    assert torch.isneginf(lse[:15]).all() and (out[:15] == 0).all()


def test_lengths_beyond_the_cache_are_cut():
    c = ref.Case(10, [128], [5], 4, 1)
    c.cache.seq_lens += 1000
    ref.check_attention(c, *attend(c))
    c.cache.seq_lens.fill_(-3)
    out, lse = attend(c)
    assert (out == 0).all() and torch.isneginf(lse).all()


def test_pools_in_one_allocation_and_no_lse():
    c = ref.Case(11, [300, 200], [60, 1], 8, 2, interleaved=True)
    a, _ = attend(c)
    b, _ = attend(c, lse=False)
    assert torch.equal(a, b)
    ref.check_attention(c, a, None)


def test_single_tokens_agree_with_dense_decode():
    c = ref.Case(12, [900, 45, 2], [1, 1, 1], 32, 8)
    out, lse = attend(c)
    other, other_lse = torch.empty_like(out), torch.empty_like(lse)
    rk.dense_decode(c.cache, c.q, other, other_lse, rk.alloc_workspace(rk.OP_DENSE_DECODE, c.cache))
    _, _, mag, big = ref.attention(c)
    de = ref.logit_error(big, 900)
    assert ((out.double() - other.double()).abs() <= 2 * (2 * ref.EPS[torch.bfloat16] * 1.01 + 2 * de[..., None]) * mag).all()
    assert ((lse - other_lse).abs() <= 2 * (de + ref.EPS[torch.float32] * 16 * (lse.abs() + 1))).all()


@pytest.mark.parametrize("lens,news", [([9000], [3]), ([700, 300], [100, 1])])
def test_graph_replays_follow_the_lengths(lens, news):
    """Captured once, replayed as the caches grow, with eager calls and other work between."""
    c = ref.Case(13, lens, news, 8, 2, spare_pages=4)
    ws = rk.alloc_workspace(rk.OP_CHUNK_ATTEND, c.cache, c.rows)
    out, lse = attend(c, ws)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        rk.chunk_attend(c.cache, c.chunk, c.q, out, lse, ws, stream=torch.cuda.current_stream())
    full = list(lens)
    for cut in (0, 200, 70, 0):
        c.lens = [n - cut for n in full]
        c.cache.seq_lens.copy_(torch.tensor(c.lens, dtype=torch.int32))
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        ref.check_attention(c, out, lse)
        other, other_lse = attend(c)
        assert torch.equal(out, other) and torch.equal(lse, other_lse)


def test_two_streams_at_once():
    a, b = ref.Case(14, [8000], [3], 8, 2), ref.Case(15, [8000, 100], [5, 40], 8, 2)
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    results = []
    for c, s in ((a, sa), (b, sb)):
        with torch.cuda.stream(s):
            results.append(attend(c))
    torch.cuda.synchronize()
    for c, r in zip((a, b), results):
        ref.check_attention(c, *r)


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes(seed):
    import random
    rng = random.Random(seed)
    token_major = rng.random() < 0.5
    ps = rng.choice([1, 2, 3, 5, 7, 8, 16, 33, 64]) if token_major else 16
    hkv = rng.choice([1, 2, 3])
    hq = hkv * rng.randint(1, 16)
    B = rng.randint(1, 6)
    lens = [rng.choice([rng.randint(0, 50), rng.randint(0, 1200)]) for _ in range(B)]
    news = [rng.choice([min(1, n), rng.randint(0, n), rng.randint(0, min(n, 20))]) for n in lens]
    c = ref.Case(100 + seed, lens, news, hq, hkv, ps, token_major, shuffled=rng.random() < 0.7, pad=(rng.randint(0, 2), rng.randint(0, 2)))
    if c.rows == 0:
        return
    ref.check_attention(c, *attend(c))
