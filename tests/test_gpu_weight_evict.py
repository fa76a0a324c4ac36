"""Accumulated attention weights and eviction by them."""
import math

import numpy as np
import pytest
import torch

import chunk_ref as ref
from paper_2502_14051_amd import rocketkv as rk

pytestmark = pytest.mark.gpu


def lse_of(c):
    _, lse, _, _ = ref.attention(c)
    return lse.float()


def accumulate(c, lse, w_in, fill=-5.0):
    out = torch.full((len(c.lens), c.hkv, c.cache.pages_cap * c.ps), fill, device="cuda")
    rk.accumulate_weights(c.cache, c.chunk, c.q, lse, w_in, out)
    return out


def check(c, lse, w_in, got, fill=-5.0):
    want, lim = ref.weights(c, lse, w_in)
    for b, n in enumerate(c.lens):
        err = (got[b, :, :n].double() - want[b, :, :n]).abs()
        assert (err <= lim[b, :, :n] + 1e-37).all(), f"sequence {b}: {float((err / (lim[b, :, :n] + 1e-37)).max()):.3g} of the limit"
        assert (got[b, :, n:] == fill).all(), "entries behind the sequence are left as they were"


@pytest.mark.parametrize("ps,token_major", [(16, False), (1, True), (3, True), (16, True), (64, True)])
@pytest.mark.parametrize("lens,news", [([1], [1]), ([300, 1, 40], [1, 1, 40]), ([700, 257], [130, 0]), ([512, 64], [64, 3])])
def test_weights(ps, token_major, lens, news):
    c = ref.Case(30, lens, news, 8, 2, ps, token_major, pad=(2, 1))
    lse = lse_of(c)
    w = torch.rand((len(lens), 2, c.cache.pages_cap * ps), device="cuda")
    check(c, lse, w, accumulate(c, lse, w))
    check(c, lse, None, accumulate(c, lse, None))
    same = w.clone()
    rk.accumulate_weights(c.cache, c.chunk, c.q, lse, same, same)
    got = accumulate(c, lse, w)
    for b, n in enumerate(lens):
        assert torch.equal(same[b, :, :n], got[b, :, :n]) and torch.equal(same[b, :, n:], w[b, :, n:])


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (5, 1), (16, 1), (12, 4), (7, 7)])
@pytest.mark.parametrize("new", [1, 21, 200])
def test_groups(hq, hkv, new):
    c = ref.Case(31, [333, 210], [new, max(1, new // 3)], hq, hkv)
    lse = lse_of(c)
    check(c, lse, None, accumulate(c, lse, None))


def test_every_row_gives_away_one():
    """The weights a row gives add up to one, so a head group's sum to its number of rows and heads."""
    c = ref.Case(32, [900, 130], [300, 130], 8, 2)
    out, lse = torch.empty_like(c.q), torch.empty((c.rows, 8), device="cuda")
    rk.chunk_attend(c.cache, c.chunk, c.q, out, lse, rk.alloc_workspace(rk.OP_CHUNK_ATTEND, c.cache, c.rows))
    w = accumulate(c, lse, None, fill=0.0)
    for b in range(2):
        assert (w[b].double().sum(-1) - 4 * c.news[b]).abs().max() <= 4 * c.news[b] * 1e-4


def test_rows_that_saw_nothing_and_absent_pages():
    c = ref.Case(33, [90, 16], [90, 16], 8, 2, pad=(1, 1))
    c.drop_pages([(0, 0), (0, 3), (1, 0)])
    lse = lse_of(c)
    assert torch.isneginf(lse[c.rows_of(1)]).all()
    # whatever lies in a page that is not listed must not matter
    free = sorted(set(range(c.cache.k_pool.shape[0])) - set(c.cache.block_table.flatten().tolist()))
    c.cache.k_pool[free] = float("nan")
    w = torch.rand((2, 2, c.cache.pages_cap * 16), device="cuda")
    got = accumulate(c, lse, w)
    check(c, lse, w, got)
    assert (got[1, :, :16] == 0).all() and (got[0, :, :16] == 0).all()


def test_no_rows_at_all_copies():
    c = ref.Case(34, [50, 20], [0, 0], 4, 2)
    w = torch.rand((2, 2, c.cache.pages_cap * 16), device="cuda")
    got = accumulate(c, torch.empty((0, 4), device="cuda"), w)
    assert torch.equal(got[0, :, :50], w[0, :, :50]) and torch.equal(got[1, :, :20], w[1, :, :20]) and (got[0, :, 50:] == -5).all()


def test_future_and_garbage_keys():
    c = ref.Case(35, [80], [40], 4, 1, 16, False, shuffled=False, spare_pages=8)
    lse = lse_of(c)
    clean = accumulate(c, lse, None)
    c.cache.k_pool[80 // 16:] = float("nan")
    assert torch.equal(accumulate(c, lse, None), clean)


@pytest.mark.parametrize("tiles,ragged", [(70, 5), (100, 1), (32, 0), (33, 127), (64, 64)])
def test_tails_of_the_launch(tiles, ragged):
    """Tiles of 128 keys of eight KV heads beside the 512 workgroups that run at a time: the last ones halved, or not."""
    n = 128 * tiles - ragged
    c = ref.Case(37, [n], [40], 8, 8)
    w_in = torch.rand((1, 8, c.cache.pages_cap * 16), generator=torch.Generator().manual_seed(0)).cuda()
    lse = ref.attention(c)[1].float()
    check(c, lse, w_in, accumulate(c, lse, w_in))


def test_weights_of_many_sequences():
    """More sequences than lanes, in the form for many rows and in the one for few."""
    lens = [1 + (37 * b) % 290 for b in range(150)]
    for news in ([min(n, 1 + b % 23) for b, n in enumerate(lens)], [1] * 150):
        c = ref.Case(38, lens, news, 8, 2)
        lse = ref.attention(c)[1].float()
        check(c, lse, None, accumulate(c, lse, None))


# ---- eviction ----

def random_weights(gen, shape, kind):
    if kind == "ties":
        return torch.randint(0, 3, shape, generator=gen).float()
    if kind == "zeros":
        return torch.where(torch.rand(shape, generator=gen) < 0.5, 0.0, -0.0)
    if kind == "odd":
        w = torch.randn(shape, generator=gen) * 10.0 ** torch.randint(-30, 30, shape, generator=gen).float()
        w = torch.where(torch.rand(shape, generator=gen) < 0.02, math.nan, w)
        w = torch.where(torch.rand(shape, generator=gen) < 0.02, math.inf, w)
        return torch.where(torch.rand(shape, generator=gen) < 0.02, -math.inf, w)
    return torch.exp(3 * torch.randn(shape, generator=gen) - 6)


def evict_and_check(c, w, recent, keep, dst_ps, dst_tm, shuffled_dst=True):
    B, H = len(c.lens), c.hkv
    cap = ((keep + dst_ps - 1) // dst_ps + 7) // 8 * 8
    n_phys = B * cap + 3
    table = torch.randperm(n_phys, generator=torch.Generator().manual_seed(1))[:B * cap].reshape(B, cap).to(torch.int32).cuda() if shuffled_dst else None
    dst = rk.alloc_cache(B, c.hq, H, 128, dst_ps, cap, "cuda", block_table=table, n_phys_pages=n_phys, zero=True,
                         v_layout=rk.V_TOKEN_MAJOR if dst_tm else rk.V_CHANNEL_MAJOR)
    dst.seq_lens.fill_(-7)
    w_out = torch.full((B, H, dst.pages_cap * dst_ps), -3.0, device="cuda")
    kept = torch.full((B, H, keep), -9, dtype=torch.int32, device="cuda")
    ws = rk.alloc_workspace(rk.OP_WEIGHT_EVICT, c.cache, recent, keep)
    before = [c.cache.k_pool.clone(), c.cache.v_pool.clone(), c.cache.seq_lens.clone(), w.clone()]
    rk.weight_evict(c.cache, w, recent, keep, dst, w_out, kept, ws)
    for a, b in zip(before, (c.cache.k_pool, c.cache.v_pool, c.cache.seq_lens, w)):
        assert torch.equal(torch.nan_to_num(a.float()), torch.nan_to_num(b.float())), "the source is left as it is"
    K, V = rk.unpack_cache(dst)
    wc = w.cpu().numpy()
    for b, n in enumerate(c.lens):
        m = min(n, keep)
        assert int(dst.seq_lens[b]) == m
        for g in range(H):
            want = ref.evicted(wc[b, g], n, recent, keep)
            got = kept[b, g].cpu().numpy()
            assert np.array_equal(got[:m], want), f"sequence {b}, head {g}"
            assert (got[m:] == -1).all()
            idx = torch.from_numpy(want).cuda()
            assert torch.equal(K[b, g, :m], c.K[b, g, idx]) and torch.equal(V[b, g, :m], c.V[b, g, idx])
            assert torch.equal(w_out[b, g, :m].view(torch.int32), w[b, g, idx].view(torch.int32)) and (w_out[b, g, m:] == -3).all()
    # nothing but the sequences' pages was written
    used = set()
    for b, n in enumerate(c.lens):
        for p in range((min(n, keep) + dst_ps - 1) // dst_ps):
            used.add(int(table[b, p]) if table is not None else b * cap + p)
    free = sorted(set(range(n_phys)) - used)
    assert (dst.k_pool[free] == 0).all() and (dst.v_pool[free] == 0).all()
    return dst, w_out


@pytest.mark.parametrize("src_layout", [(16, False), (1, True), (5, True), (16, True), (64, True)])
@pytest.mark.parametrize("dst_layout", [(16, False), (3, True), (16, True)])
def test_layouts(src_layout, dst_layout):
    c = ref.Case(40, [300, 64, 1, 0, 129], [0] * 5, 4, 2, *src_layout)
    w = random_weights(torch.Generator().manual_seed(2), (5, 2, c.cache.pages_cap * c.ps), "plain").cuda()
    evict_and_check(c, w, 16, 100, *dst_layout)


@pytest.mark.parametrize("kind", ["plain", "ties", "zeros", "odd"])
@pytest.mark.parametrize("recent,keep", [(0, 1), (0, 64), (1, 1), (64, 64), (32, 777), (5, 4095)])
def test_weights_of_all_kinds(kind, recent, keep):
    c = ref.Case(41, [5000, 4096, 777], [0] * 3, 2, 2)
    w = random_weights(torch.Generator().manual_seed(3), (3, 2, c.cache.pages_cap * 16), kind).cuda()
    evict_and_check(c, w, recent, keep, 16, False)


@pytest.mark.parametrize("kind", ["plain", "ties", "zeros", "odd"])
@pytest.mark.parametrize("keep", [100, 20000])
def test_long_rows(kind, keep):
    """Rows counted by a launch of their own, and cut between workgroups."""
    c = ref.Case(42, [40000, 33000], [0, 0], 2, 1, 4, True)
    w = random_weights(torch.Generator().manual_seed(4), (2, 1, c.cache.pages_cap * 4), kind).cuda()
    evict_and_check(c, w, 32, keep, 4, True)


def test_nothing_to_evict_and_whole_recent():
    c = ref.Case(43, [64, 65], [0, 0], 2, 1)
    w = random_weights(torch.Generator().manual_seed(5), (2, 1, c.cache.pages_cap * 16), "plain").cuda()
    evict_and_check(c, w, 0, 64, 16, False, shuffled_dst=False)


def test_optional_outputs():
    c = ref.Case(44, [300], [0], 2, 1)
    w = random_weights(torch.Generator().manual_seed(6), (1, 1, c.cache.pages_cap * 16), "plain").cuda()
    a, _ = evict_and_check(c, w, 8, 100, 16, False)
    b = rk.alloc_cache(1, 2, 1, 128, 16, 8, "cuda", block_table=a.block_table, n_phys_pages=a.k_pool.shape[0], zero=True)
    rk.weight_evict(c.cache, w, 8, 100, b, None, None, rk.alloc_workspace(rk.OP_WEIGHT_EVICT, c.cache, 8, 100))
    assert torch.equal(a.k_pool, b.k_pool) and torch.equal(a.v_pool, b.v_pool) and torch.equal(a.seq_lens, b.seq_lens)


def test_length_beyond_the_cache_counts_as_none():
    c = ref.Case(45, [100, 50], [0, 0], 2, 1)
    c.cache.seq_lens[0] = 100000
    w = torch.rand((2, 1, c.cache.pages_cap * 16), device="cuda")
    dst = rk.alloc_cache(2, 2, 1, 128, 16, 8, "cuda", zero=True)
    kept = torch.empty((2, 1, 20), dtype=torch.int32, device="cuda")
    rk.weight_evict(c.cache, w, 4, 20, dst, None, kept, rk.alloc_workspace(rk.OP_WEIGHT_EVICT, c.cache, 4, 20))
    assert dst.seq_lens.tolist() == [0, 20] and (kept[0] == -1).all() and (dst.k_pool[:8] == 0).all()


def test_many_sequences():
    lens = [1 + (37 * b) % 290 for b in range(150)]
    c = ref.Case(46, lens, [0] * 150, 2, 1)
    w = random_weights(torch.Generator().manual_seed(7), (150, 1, c.cache.pages_cap * 16), "plain").cuda()
    evict_and_check(c, w, 3, 70, 16, False)


@pytest.mark.parametrize("lens,keep", [([3000, 500], 300), ([30000, 500], 300)])
def test_graph_of_accumulation_and_eviction(lens, keep):
    """Captured once, replayed over other lengths, with eager calls on the same workspace between."""
    c = ref.Case(47, lens, [40, 3], 4, 2)
    lse = ref.attention(c)[1].float()
    w0 = random_weights(torch.Generator().manual_seed(8), (2, 2, c.cache.pages_cap * 16), "plain").cuda()
    ws = rk.alloc_workspace(rk.OP_WEIGHT_EVICT, c.cache, 16, keep)
    make = lambda: [torch.empty_like(w0), rk.alloc_cache(2, 4, 2, 128, 16, 24, "cuda", zero=True), torch.zeros((2, 2, 24 * 16), device="cuda"),
                    torch.zeros((2, 2, keep), dtype=torch.int32, device="cuda")]

    def run(w, dst, w_out, kept):
        rk.accumulate_weights(c.cache, c.chunk, c.q, lse, w0, w)
        rk.weight_evict(c.cache, w, 16, keep, dst, w_out, kept, ws)

    a, b = make(), make()
    a[0].zero_(), b[0].zero_()
    run(*a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        run(*a)
    for cut in (0, 2500, 100, 0):
        c.cache.seq_lens.copy_(torch.tensor([lens[0] - cut, lens[1] - cut // 10], dtype=torch.int32))
        for x in (a, b):
            for t in (x[0], x[1].k_pool, x[1].v_pool, x[2], x[3]):
                t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        run(*b)
        for x, y in zip([a[0], a[1].k_pool, a[1].v_pool, a[1].seq_lens, *a[2:]], [b[0], b[1].k_pool, b[1].v_pool, b[1].seq_lens, *b[2:]]):
            assert torch.equal(x, y)
    check(c, lse, w0, b[0], fill=0.0)


def test_two_streams_at_once():
    cases = [ref.Case(48 + i, [n], [0], 2, 2) for i, n in enumerate((20000, 3000))]
    ws = [rk.alloc_workspace(rk.OP_WEIGHT_EVICT, c.cache, 8, 256) for c in cases]
    w = [random_weights(torch.Generator().manual_seed(9), (1, 2, c.cache.pages_cap * 16), "plain").cuda() for c in cases]
    kept = [torch.empty((1, 2, 256), dtype=torch.int32, device="cuda") for _ in cases]
    dst = [rk.alloc_cache(1, 2, 2, 128, 16, 16, "cuda", zero=True) for _ in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        for i, c in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                rk.weight_evict(c.cache, w[i], 8, 256, dst[i], None, kept[i], ws[i])
    torch.cuda.synchronize()
    for i, c in enumerate(cases):
        for g in range(2):
            assert np.array_equal(kept[i][0, g].cpu().numpy(), ref.evicted(w[i][0, g].cpu().numpy(), c.lens[0], 8, 256))


# ---- together, as a program uses them ----

def test_prompt_draft_accumulate_evict_decode():
    """A prompt in two pieces and drafted tokens through the cache, weights accumulated on the way, eviction, and a decode
    step over what is left: each state against the definition, given the one before."""
    hq, hkv, B = 8, 2, 2
    gen = torch.Generator().manual_seed(50)
    total = [260, 150]
    theta = (1.0 / 10000.0 ** (torch.arange(0, 128, 2, dtype=torch.float64) / 128)).cuda()
    r = rk.Rope(theta)
    cache = rk.alloc_cache(B, hq, hkv, 128, 16, 24, "cuda", zero=True)
    kmax, kmin = rk.alloc_summaries(cache)
    w = rk.alloc_weights(cache)
    K = [torch.zeros((hkv, 0, 128), dtype=torch.bfloat16, device="cuda") for _ in range(B)]
    V = [k.clone() for k in K]
    for news in ([200, 150], [57, 0], [3, 0]):
        n = sum(news)
        joint = torch.randn((n, hq + 2 * hkv, 128), generator=gen).to(torch.bfloat16).cuda()
        starts = torch.tensor([0, news[0], n], dtype=torch.int32).cuda()
        chunk = rk.Chunk(starts, n)
        ws = rk.alloc_workspace(rk.OP_APPEND_CHUNK, cache, n)
        q = torch.empty((n, hq, 128), dtype=torch.bfloat16, device="cuda")
        pos = torch.cat([K[b].shape[1] + torch.arange(news[b]) for b in range(B)]).to(torch.int32).cuda()
        rk.append_chunk(cache, chunk, joint[:, hq:hq + hkv], joint[:, hq + hkv:], kmax, kmin, ws, rope=r, q=joint[:, :hq], q_out=q)
        ref.check_turned(q, *ref.turned(joint[:, :hq], pos, theta, False))
        held_k, held_v = rk.unpack_cache(cache)
        tk, mag = ref.turned(joint[:, hq:hq + hkv], pos, theta, False)
        at = 0
        for b in range(B):
            o = K[b].shape[1]
            new = held_k[b, :, o:o + news[b]]
            ref.check_turned(new, tk[at:at + news[b]].transpose(0, 1), mag[at:at + news[b]].transpose(0, 1))
            assert torch.equal(held_v[b, :, o:o + news[b]], joint[at:at + news[b], hq + hkv:].transpose(0, 1))
            K[b], V[b] = torch.cat([K[b], new], 1), torch.cat([V[b], held_v[b, :, o:o + news[b]]], 1)
            at += news[b]
        c = ref.Case.__new__(ref.Case)
        c.lens, c.news, c.hq, c.hkv, c.ps, c.cache, c.rows, c.q = [k.shape[1] for k in K], news, hq, hkv, 16, cache, n, q
        c.starts, longest = [0, news[0], n], max(k.shape[1] for k in K)
        pad = lambda t: torch.nn.functional.pad(t, (0, 0, 0, longest - t.shape[1]))
        c.K, c.V = torch.stack([pad(k) for k in K]), torch.stack([pad(v) for v in V])
        out, lse = torch.empty_like(q), torch.empty((n, hq), device="cuda")
        rk.chunk_attend(cache, chunk, q, out, lse, rk.alloc_workspace(rk.OP_CHUNK_ATTEND, cache, n))
        ref.check_attention(c, out, lse)
        before = w.clone()
        rk.accumulate_weights(cache, chunk, q, lse, w, w)
        check(c, lse, before, w, fill=0.0)
    assert cache.seq_lens.tolist() == total
    smax, smin = rk.alloc_summaries(cache)
    rk.build_page_summaries(cache, smax, smin)
    assert torch.equal(smax, kmax) and torch.equal(smin, kmin)
    c.news = [0, 0]
    dst, w_dst = evict_and_check(c, w, 16, 160, 16, False)
    assert dst.seq_lens.tolist() == [160, 150]
    # decode over the evicted cache: new tokens keep counting from the whole sequence's positions
    big = rk.alloc_cache(B, hq, hkv, 128, 16, 16, "cuda", zero=True)
    w_big = rk.alloc_weights(big)
    rk.weight_evict(cache, w, 16, 160, big, w_big, None, rk.alloc_workspace(rk.OP_WEIGHT_EVICT, cache, 16, 160))
    bmax, bmin = rk.alloc_summaries(big)
    rk.build_page_summaries(big, bmax, bmin)
    joint = torch.randn((B, hq + 2 * hkv, 128), generator=gen).to(torch.bfloat16).cuda()
    q = torch.empty((B, hq, 128), dtype=torch.bfloat16, device="cuda")
    chunk = rk.Chunk(torch.tensor([0, 1, 2], dtype=torch.int32).cuda(), B)
    rk.append_chunk(big, chunk, joint[:, hq:hq + hkv], joint[:, hq + hkv:], bmax, bmin,
                    rk.alloc_workspace(rk.OP_APPEND_CHUNK, big, B), rope=r, positions=torch.tensor(total, dtype=torch.int32).cuda(),
                    q=joint[:, :hq], q_out=q)
    dense, sparse, out = (torch.empty_like(q) for _ in range(3))
    lse = torch.empty((B, hq), device="cuda")
    rk.dense_decode(big, q, dense, lse, rk.alloc_workspace(rk.OP_DENSE_DECODE, big))
    rk.hsa_decode(big, q, bmax, bmin, 128, 4096, 0, sparse, None, None, None, rk.alloc_workspace(rk.OP_HSA_DECODE, big, 4096))
    rk.chunk_attend(big, chunk, q, out, None, rk.alloc_workspace(rk.OP_CHUNK_ATTEND, big, B))
    scale = rk.unpack_cache(big)[1].float().abs().amax()
    assert (dense.float() - sparse.float()).abs().max() <= 2.0 ** -6 * scale
    assert (dense.float() - out.float()).abs().max() <= 2.0 ** -6 * scale
    rk.accumulate_weights(big, chunk, q, lse, w_big, w_big)
    assert (w_big[0, :, 160] > 0).all() and (w_big[1, :, 150] > 0).all()
