"""Attention of a chunk in tiles of 256 rows: many rows a sequence over caches with room for more than 128 MiB of keys and
values, and pools that need 64 bits of offset.  Which form and division a case takes is asserted without a GPU
(test_chunk_forms.py)."""
import dataclasses

import pytest
import torch

import chunk_ref as ref
from paper_2502_14051_amd import rocketkv as rk

pytestmark = pytest.mark.gpu

# name: lens, news, query heads, KV heads, tokens of room
CASES = {
    "one round": ([3000], [100], 64, 8, 40000),            # 56 tiles of 16 tokens and more, keys cut
    "three rounds": ([6000], [300], 128, 8, 40000),        # 152 tiles, keys cut into up to 768 parts
    "between": ([1100], [800], 128, 8, 40000),             # 400 tiles, too many for two rounds
    "not cut": ([1700], [1540], 128, 8, 40000),            # more tiles than parts
    "ragged": ([5100, 70, 900, 1], [900, 70, 33, 1], 40, 8, 20000),  # 51 tokens to a tile, one row left empty
    "prompts": ([513, 640], [513, 640], 64, 8, 20000),     # all of their keys are new
    "one head": ([700, 1500], [700, 900], 16, 1, 140000),  # many query heads over one KV head
}


def make(name, ps, token_major, seed=90):
    lens, news, hq, hkv, room = CASES[name]
    return ref.Case(seed, lens, news, hq, hkv, ps, token_major, shuffled=False, spare_pages=(room - max(lens)) // ps, pad=(1, 2))


def attend(c):
    out = torch.full((c.rows, c.hq, ref.D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((c.rows, c.hq), 7.0, device="cuda")
    rk.chunk_attend(c.cache, c.chunk, c.q, out, lse, rk.alloc_workspace(rk.OP_CHUNK_ATTEND, c.cache, c.rows))
    return out, lse


def check(c, out, lse):
    used = slice(c.starts[0], c.starts[0] + sum(c.news))
    assert torch.isfinite(out[used]).all() and not torch.isnan(lse[used]).any()
    ref.check_attention(c, out, lse)
    for rows in (slice(0, used.start), slice(used.stop, None)):
        assert (out[rows] == 7).all() and (lse[rows] == 7).all(), "rows of no sequence are left as they were"


@pytest.mark.parametrize("ps,token_major", [(16, False), (16, True), (3, True), (64, True)])
@pytest.mark.parametrize("name", list(CASES))
def test_against_the_definition(name, ps, token_major):
    c = make(name, ps, token_major)
    check(c, *attend(c))


@pytest.mark.parametrize("token_major", [False, True])
@pytest.mark.parametrize("name", ["one round", "three rounds", "not cut", "ragged"])
def test_what_lies_where_no_token_is(name, token_major):
    """NaN behind the ends, in pages that are absent and (keys and values) in the future of rows in front of them."""
    c = make(name, 16, token_major, seed=91)
    cap = c.cache.pages_cap
    c.cache.block_table = torch.arange(len(c.lens) * cap, dtype=torch.int32, device="cuda").reshape(-1, cap)
    c.cache.k_pool[-1], c.cache.v_pool[-1] = float("nan"), float("nan")
    c.drop_pages([(0, 0), (0, 9), (0, c.lens[0] // 32)])
    for b, n in enumerate(c.lens):
        for p in [p for p in range(c.cache.pages_cap) if p * 16 >= n][:40] + ([0, 9, c.lens[0] // 32] if b == 0 else []):
            c.cache.k_pool[b * cap + p], c.cache.v_pool[b * cap + p] = float("nan"), float("nan")
        if n % 16:
            c.cache.k_pool[b * cap + n // 16, :, n % 16:] = float("nan")
            if token_major:
                c.cache.v_pool[b * cap + n // 16, :, n % 16:] = float("nan")
            else:
                c.cache.v_pool[b * cap + n // 16, :, :, n % 16:] = float("nan")
    out, lse = attend(c)
    check(c, out, lse)
    # the last tokens of sequence 0 seen by its last rows alone
    n, last = c.lens[0], 5
    first = c.starts[0] + c.news[0] - last
    for t in range(n - last, n):
        c.cache.k_pool[t // 16, :, t % 16] = float("nan")
        if token_major:
            c.cache.v_pool[t // 16, :, t % 16] = float("inf")
        else:
            c.cache.v_pool[t // 16, :, :, t % 16] = float("inf")
    spoilt, spoilt_lse = attend(c)
    assert torch.isnan(spoilt_lse[first:first + last]).all()
    spoilt[first:first + last], spoilt_lse[first:first + last] = out[first:first + last], lse[first:first + last]
    check(c, spoilt, spoilt_lse)


@pytest.mark.parametrize("token_major", [False, True])
def test_large_logits(token_major):
    c = make("ragged", 16, token_major)
    c.q *= 6
    c.cache.k_pool *= 6
    c.K *= 6
    check(c, *attend(c))


@pytest.mark.parametrize("name", ["one round", "three rounds", "not cut"])
def test_graph_replays_follow_the_lengths(name):
    c = make(name, 16, False, seed=92)
    ws = rk.alloc_workspace(rk.OP_CHUNK_ATTEND, c.cache, c.rows)
    out, lse = attend(c)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        rk.chunk_attend(c.cache, c.chunk, c.q, out, lse, ws, stream=torch.cuda.current_stream())
    full = list(c.lens)
    for cut in (0, 130, 0):
        c.lens = [n - cut for n in full]
        c.cache.seq_lens.copy_(torch.tensor(c.lens, dtype=torch.int32))
        out.fill_(7.0), lse.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        other, other_lse = attend(c)
        assert torch.equal(out, other) and torch.equal(lse, other_lse)
    check(c, out, lse)


# lens, news: with keys cut and merged, and with tiles enough
FAR_CASES = [([5000], [3]), ([3000, 900], [150, 1]), ([2500], [2300])]
FAR_PAGES = (5 << 30) // (8 * 16 * 128 * 2)


@pytest.mark.parametrize("lens,news", FAR_CASES)
def test_offsets_of_64_bits(lens, news):
    """Token-major pools of 5 GiB, pages from their beginning to their end."""
    c = ref.Case(93, lens, news, 32, 8, 16, True, shuffled=False)
    cap, B = c.cache.pages_cap, len(lens)
    table = torch.randperm(FAR_PAGES, generator=torch.Generator().manual_seed(3))[:B * cap]
    table[0], table[7] = FAR_PAGES - 1, 0
    assert len(set(table.tolist())) == len(table)
    big = rk.alloc_cache(B, 32, 8, 128, 16, cap, "cuda", block_table=table.reshape(B, cap).to(torch.int32).cuda(),
                         n_phys_pages=FAR_PAGES, v_layout=rk.V_TOKEN_MAJOR)
    big.k_pool[table.cuda()], big.v_pool[table.cuda()] = c.cache.k_pool[:B * cap], c.cache.v_pool[:B * cap]
    big.seq_lens.copy_(c.cache.seq_lens)
    c.cache = dataclasses.replace(big)
    out, lse = attend(c)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    ref.check_attention(c, out, lse)
