"""Rotary positions, and new tokens into the cache."""
import dataclasses

import pytest
import torch

import chunk_ref as ref
from paper_2502_14051_amd import rocketkv as rk

pytestmark = pytest.mark.gpu


def freq(rot, theta=500000.0):
    return (1.0 / theta ** (torch.arange(0, rot, 2, dtype=torch.float64) / rot)).cuda()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [2, 6, 16, 50, 64, 96, 112, 126, 128])
@pytest.mark.parametrize("n,heads", [(1, 1), (3, 40), (70, 5)])
def test_rope(interleaved, rot, n, heads):
    gen = torch.Generator().manual_seed(rot)
    x = torch.randn((n, heads, 128), generator=gen).to(torch.bfloat16).cuda()
    pos = torch.randint(0, 131072, (n,), generator=gen, dtype=torch.int32).cuda()
    r = rk.Rope(freq(rot), interleaved, 1.25)
    y = torch.empty_like(x)
    rk.rope(r, pos, x, y)
    want, mag = ref.turned(x, pos, r.inv_freq, interleaved, 1.25)
    ref.check_turned(y, want, mag)
    assert torch.equal(y[..., rot:], x[..., rot:])
    z = x.clone()
    rk.rope(r, pos, z, z)  # in place
    assert torch.equal(y, z)


def test_rope_at_the_ends_of_the_positions():
    pos = torch.tensor([0, 1, -1, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32).cuda()
    x = torch.randn((6, 2, 128), generator=torch.Generator().manual_seed(0)).to(torch.bfloat16).cuda()
    r, y = rk.Rope(freq(128)), torch.empty((6, 2, 128), dtype=torch.bfloat16, device="cuda")
    rk.rope(r, pos, x, y)
    assert torch.equal(y[0], x[0])
    ref.check_turned(y, *ref.turned(x, pos, r.inv_freq, False))


def test_rope_of_strided_rows():
    """Heads in the rows of a joint projection; what lies beside them stays as it was."""
    joint = torch.randn((9, 7, 128), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    before, pos = joint.clone(), torch.arange(5, 14, dtype=torch.int32).cuda()
    r, y = rk.Rope(freq(128)), torch.zeros((9, 12, 128), dtype=torch.bfloat16, device="cuda")
    rk.rope(r, pos, joint[:, 2:5], y[:, 4:7])
    ref.check_turned(y[:, 4:7], *ref.turned(before[:, 2:5], pos, r.inv_freq, False))
    assert torch.equal(joint, before) and (y[:, :4] == 0).all() and (y[:, 7:] == 0).all()
    rk.rope(r, pos, joint[:, 2:5], joint[:, 2:5])
    assert torch.equal(joint[:, 2:5], y[:, 4:7]) and torch.equal(joint[:, :2], before[:, :2])


def test_rope_many_tokens():
    x = torch.randn((5000, 3, 128), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    pos = torch.arange(5000, dtype=torch.int32).cuda()
    r, y = rk.Rope(freq(128), True), torch.empty_like(x)
    rk.rope(r, pos, x, y)
    ref.check_turned(y, *ref.turned(x, pos, r.inv_freq, True))


def clone(cache):
    import dataclasses
    return dataclasses.replace(cache, k_pool=cache.k_pool.clone(), v_pool=cache.v_pool.clone(), seq_lens=cache.seq_lens.clone())


def new_rows(c, seed):
    gen = torch.Generator().manual_seed(1000 + seed)
    mk = lambda h: torch.randn((c.rows, h, 128), generator=gen).to(torch.bfloat16).cuda()
    return mk(c.hq), mk(c.hkv), mk(c.hkv)


def one_by_one(c, cache, k, v, kmax, kmin, fits=lambda b: True):
    """The tokens through append_kv, a token of every sequence a call; the sequences that bring none are put back."""
    for i in range(max(c.news)):
        lens = cache.seq_lens.clone()
        save = [t.clone() for t in (cache.k_pool, cache.v_pool, kmax, kmin)]
        take = [b for b in range(len(c.news)) if i < c.news[b] and fits(b)]
        rows = [c.starts[b] + min(i, max(c.news[b] - 1, 0)) if c.rows else 0 for b in range(len(c.news))]
        rows = [min(r, c.rows - 1) for r in rows]
        full = torch.full_like(lens, cache.pages_cap * cache.page_size)
        mask = torch.zeros_like(lens, dtype=torch.bool)
        mask[take] = True
        cache.seq_lens.copy_(torch.where(mask, lens, full))  # a full sequence is left unchanged
        rk.append_kv(cache, k[rows].contiguous(), v[rows].contiguous(), kmax, kmin)
        cache.seq_lens.copy_(torch.where(mask, cache.seq_lens, lens))
        del save


@pytest.mark.parametrize("ps,token_major", [(16, False), (1, True), (2, True), (3, True), (4, True), (7, True), (16, True), (33, True), (64, True)])
@pytest.mark.parametrize("olds,news", [([0], [1]), ([0, 5, 130], [3, 40, 1]), ([31, 16, 0, 77], [1, 0, 150, 2])])
def test_like_single_appends(ps, token_major, olds, news):
    c = ref.Case(20, olds, news, 6, 3, ps, token_major, spare_pages=(200 + ps - 1) // ps, pad=(1, 2))
    q, k, v = new_rows(c, 1)
    kmax, kmin = rk.alloc_summaries(c.cache)
    rk.build_page_summaries(c.cache, kmax, kmin)
    other, omax, omin = clone(c.cache), kmax.clone(), kmin.clone()
    ws = rk.alloc_workspace(rk.OP_APPEND_CHUNK, c.cache, c.rows)
    for again in range(2):  # the workspace serves the next call
        rk.append_chunk(c.cache, c.chunk, k, v, kmax, kmin, ws)
        room = other.pages_cap * other.page_size - other.seq_lens.cpu()
        one_by_one(c, other, k, v, omax, omin, fits=lambda b: c.news[b] <= room[b])
        assert torch.equal(c.cache.seq_lens, other.seq_lens)
        assert torch.equal(c.cache.k_pool, other.k_pool) and torch.equal(c.cache.v_pool, other.v_pool)
        assert torch.equal(kmax, omax) and torch.equal(kmin, omin)


@pytest.mark.parametrize("ps,token_major", [(16, False), (4, True), (40, True)])
@pytest.mark.parametrize("interleaved,rot,given", [(False, 128, False), (True, 64, True), (False, 36, True)])
def test_turned_on_the_way(ps, token_major, interleaved, rot, given):
    """Keys and queries as rope() turns them, the cache as it is with those keys; rows of no sequence untouched."""
    c = ref.Case(21, [40, 0, 1000], [70, 300, 1], 8, 2, ps, token_major, spare_pages=(320 + ps - 1) // ps, pad=(2, 3))
    gen = torch.Generator().manual_seed(5)
    joint = torch.randn((c.rows, 12, 128), generator=gen).to(torch.bfloat16).cuda()
    q, k, v = joint[:, :8], joint[:, 8:10], joint[:, 10:]
    r = rk.Rope(freq(rot), interleaved, 0.9)
    pos = torch.full((c.rows,), 99, dtype=torch.int32)
    for b, old in enumerate(c.lens):
        pos[c.rows_of(b)] = torch.arange(old, old + c.news[b], dtype=torch.int32) + (5000 if given else 0)
    pos = pos.cuda()
    tq, tk = torch.empty((c.rows, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((c.rows, 2, 128), dtype=torch.bfloat16, device="cuda")
    rk.rope(r, pos, q, tq)
    rk.rope(r, pos, k, tk)
    kmax, kmin = rk.alloc_summaries(c.cache)
    rk.build_page_summaries(c.cache, kmax, kmin)
    other, omax, omin = clone(c.cache), kmax.clone(), kmin.clone()
    ws = rk.alloc_workspace(rk.OP_APPEND_CHUNK, c.cache, c.rows)
    rk.append_chunk(other, c.chunk, tk, v, omax, omin, ws)
    q_out = torch.full((c.rows, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    rk.append_chunk(c.cache, c.chunk, k, v, kmax, kmin, ws, rope=r, positions=pos if given else None, q=q, q_out=q_out)
    assert torch.equal(c.cache.k_pool, other.k_pool) and torch.equal(c.cache.v_pool, other.v_pool)
    assert torch.equal(kmax, omax) and torch.equal(kmin, omin) and torch.equal(c.cache.seq_lens, other.seq_lens)
    assert torch.equal(q_out[2:-3], tq[2:-3])
    assert (q_out[:2] == 7).all() and (q_out[-3:] == 7).all()


def test_without_summaries_and_in_place():
    c = ref.Case(22, [10, 3], [20, 100], 4, 2, 4, True, spare_pages=40)
    q, k, v = new_rows(c, 2)
    r, kmax = rk.Rope(freq(128)), rk.alloc_summaries(c.cache)
    other = clone(c.cache)
    ws = rk.alloc_workspace(rk.OP_APPEND_CHUNK, c.cache, c.rows)
    q_out = torch.empty_like(q)
    rk.append_chunk(other, c.chunk, k, v, *kmax, ws, rope=r, q=q, q_out=q_out)
    rk.append_chunk(c.cache, c.chunk, k, v, None, None, ws, rope=r, q=q, q_out=q)
    assert torch.equal(c.cache.k_pool, other.k_pool) and torch.equal(c.cache.v_pool, other.v_pool)
    assert torch.equal(c.cache.seq_lens, other.seq_lens) and torch.equal(q, q_out)


def test_no_room_and_absent_pages():
    """A sequence without room for all of its tokens is left alone, beside one that fits exactly; tokens of an absent page
    count, as in single appends."""
    c = ref.Case(23, [120, 100, 60], [9, 28, 30], 4, 1)
    assert c.cache.pages_cap == 8
    c.drop_pages([(2, 4)])
    q, k, v = new_rows(c, 3)
    kmax, kmin = rk.alloc_summaries(c.cache)
    rk.build_page_summaries(c.cache, kmax, kmin)
    other, omax, omin = clone(c.cache), kmax.clone(), kmin.clone()
    ws = rk.alloc_workspace(rk.OP_APPEND_CHUNK, c.cache, c.rows)
    q_out = torch.empty_like(q)
    rk.append_chunk(c.cache, c.chunk, k, v, kmax, kmin, ws, q=q, q_out=q_out)
    one_by_one(c, other, k, v, omax, omin, fits=lambda b: b > 0)
    assert c.cache.seq_lens.tolist() == [120, 128, 90] == other.seq_lens.tolist()
    assert torch.equal(c.cache.k_pool, other.k_pool) and torch.equal(c.cache.v_pool, other.v_pool)
    assert torch.equal(kmax, omax) and torch.equal(kmin, omin)
    assert torch.equal(q_out, q)


def test_many_sequences_and_graph():
    """More sequences than lanes; captured, and replayed from lengths that move."""
    B = 130
    c = ref.Case(24, [(7 * b) % 50 for b in range(B)], [b % 4 for b in range(B)], 4, 2, spare_pages=4)
    q, k, v = new_rows(c, 4)
    kmax, kmin = rk.alloc_summaries(c.cache)
    rk.build_page_summaries(c.cache, kmax, kmin)
    r, q_out = rk.Rope(freq(128)), torch.empty_like(q)
    ws = rk.alloc_workspace(rk.OP_APPEND_CHUNK, c.cache, c.rows)
    other, omax, omin, oq = clone(c.cache), kmax.clone(), kmin.clone(), torch.empty_like(q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        rk.append_chunk(c.cache, c.chunk, k, v, kmax, kmin, ws, rope=r, q=q, q_out=q_out, stream=torch.cuda.current_stream())
    ows = rk.alloc_workspace(rk.OP_APPEND_CHUNK, c.cache, c.rows)
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        rk.append_chunk(other, c.chunk, k, v, omax, omin, ows, rope=r, q=q, q_out=oq)
        assert torch.equal(c.cache.k_pool, other.k_pool) and torch.equal(c.cache.v_pool, other.v_pool)
        assert torch.equal(kmax, omax) and torch.equal(kmin, omin) and torch.equal(c.cache.seq_lens, other.seq_lens)
        assert torch.equal(q_out, oq)
    assert c.cache.seq_lens.tolist() == [(7 * b) % 50 + 4 * (b % 4) for b in range(B)]


def test_tensors_of_another_kind_are_refused():
    x = torch.zeros((3, 4, 128), dtype=torch.bfloat16, device="cuda")
    pos, r = torch.zeros(3, dtype=torch.int32, device="cuda"), rk.Rope(freq(128))
    wide = torch.zeros((3, 4, 256), dtype=torch.bfloat16, device="cuda")
    for a, b, p, needle in ((x, x[:2], pos, "y"), (x, x, pos.long(), "int32"), (x, x.cpu(), pos, "y: on"), (x, x, pos[:2], "positions"),
                            (wide[..., :128], x, pos, "contiguous"), (x.transpose(0, 1), x, pos, "contiguous")):
        with pytest.raises(rk.RocketKVError) as e:
            rk.rope(r, p, a, b)
        assert e.value.status == rk.INVALID_ARG and needle in str(e.value)
    c = ref.Case(25, [3, 4], [1, 2], 4, 2)
    q, k, v = new_rows(c, 5)
    kmax, kmin = rk.alloc_summaries(c.cache)
    ws = rk.alloc_workspace(rk.OP_APPEND_CHUNK, c.cache, c.rows)
    for args, kw in (((k[:2], v, kmax, kmin), {}), ((k, v[:, :1], kmax, kmin), {}), ((k, v, kmax[..., :1], kmin), {}),
                     ((k, v, kmax, None), {}), ((k, v, kmax, kmin), dict(q=q)), ((k, v, kmax, kmin), dict(q=q, q_out=q[:, :2])),
                     ((k, v, kmax, kmin), dict(positions=torch.zeros(3, dtype=torch.int32, device="cuda")))):
        with pytest.raises(rk.RocketKVError):
            rk.append_chunk(c.cache, c.chunk, *args, ws, **kw)
    with pytest.raises(rk.RocketKVError):
        rk.append_chunk(c.cache, rk.Chunk(c.chunk.starts[:2], c.rows), k, v, kmax, kmin, ws)
    with pytest.raises(rk.RocketKVError):
        rk.append_chunk(c.cache, c.chunk, k, v, kmax, kmin, ws[:1024])
    for name in ("k_pool", "v_pool", "seq_lens", "block_table"):  # a cache that lies elsewhere, in part or as a whole
        other = dataclasses.replace(c.cache, **{name: getattr(c.cache, name).cpu()})
        for call in (lambda: rk.append_chunk(other, c.chunk, k, v, kmax, kmin, ws),
                     lambda: rk.weight_evict(c.cache, rk.alloc_weights(c.cache), 1, 2, other, None, None, ws)):
            with pytest.raises(rk.RocketKVError, match=name + ": on cpu"):
                call()


def test_no_tokens_at_all():
    c = ref.Case(26, [5, 9], [0, 0], 4, 2)
    kmax, kmin = rk.alloc_summaries(c.cache)
    none = lambda h: torch.empty((0, h, 128), dtype=torch.bfloat16, device="cuda")
    rk.append_chunk(c.cache, c.chunk, none(2), none(2), kmax, kmin, rk.alloc_workspace(rk.OP_APPEND_CHUNK, c.cache, 0))
    rk.rope(rk.Rope(freq(128)), torch.empty(0, dtype=torch.int32, device="cuda"), none(4), none(4))
    rk.chunk_attend(c.cache, c.chunk, none(4), none(4), None, rk.alloc_workspace(rk.OP_CHUNK_ATTEND, c.cache, 0))
    assert c.cache.seq_lens.tolist() == [5, 9]
