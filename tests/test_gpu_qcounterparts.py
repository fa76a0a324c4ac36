"""Operators over quantised caches beside their counterparts over the bf16 caches that hold the same values (as restore makes them):
selections are equal, results differ by the errors of both."""
import random

import pytest
import torch

import chunk_ref as ref
import quant_ref as qr
import test_gpu_qattend as over_codes
from paper_2502_14051_amd import rocketkv as rk

pytestmark = pytest.mark.gpu


def restored(q):
    """With the same pages, so lists of pages mean the same."""
    back = rk.alloc_cache(q.batch, q.n_q_heads, q.n_kv_heads, 128, q.page_size, q.pages_cap, "cuda", block_table=q.block_table,
                          n_phys_pages=q.k_codes.shape[0], v_layout=rk.V_TOKEN_MAJOR)
    rk.restore(q, back)
    return back


def close(c, a, la, b, lb, definition, keys):
    """Twice the limit of ref.check_attention: both are within it of the same definition."""
    want, wlse, mag, big = definition
    de = ref.logit_error(big, keys)
    lim = 2 * (ref.EPS[torch.bfloat16] * (mag + want.abs()) * (1 + 2.0 ** -7) + 2 * de[..., None] * mag)
    assert ((a.double() - b.double()).abs() <= lim).all()
    assert torch.equal(torch.isinf(la), torch.isinf(lb))
    some = ~torch.isinf(la)
    lim = 2 * (de + ref.EPS[torch.float32] * 16 * (torch.where(some, wlse, 0.0).abs() + 1))
    assert ((la.double() - lb.double()).abs()[some] <= lim[some]).all()


@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("ps", [4, 16, 64])
@pytest.mark.parametrize("lens,news", [([1], [1]), ([4000, 900, 20], [1, 1, 1]), ([700, 64], [12, 5]), ([900, 300], [40, 260]), ([5000], [513])])
@pytest.mark.parametrize("kind", [None, "tree", "random"])
def test_chunks(fmt, ps, lens, news, kind):
    c = ref.Case(81, lens, news, 8, 2, 16, True)
    q = qr.take_over(c, fmt, ps)
    back = restored(q)
    m = None if kind is None else qr.MaskedCase(c, over_codes.masked(82, lens, news, kind))
    a, la = over_codes.attend(c, q, m and m.mask)
    b, lb = torch.empty_like(a), torch.empty_like(la)
    ws = rk.alloc_workspace(rk.OP_CHUNK_ATTEND, back, c.rows)
    if m is None:
        rk.chunk_attend(back, c.chunk, c.q, b, lb, ws)
    else:
        rk.masked_attend(back, c.chunk, m.mask, c.q, b, lb, ws)
    close(c, a, la, b, lb, ref.attention(c) if m is None else m.definition(), max(lens))


@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("ps", [4, 16])
@pytest.mark.parametrize("budget", [64, 1024, 100000])
def test_single_tokens(fmt, ps, budget):
    """Over every page, over those that are selected, and as whole steps."""
    lens = [3000, 900, 20]
    c = ref.Case(83, lens, [1, 1, 1], 8, 2, 16, True)
    q = qr.take_over(c, fmt, ps)
    back = restored(q)
    kmax, kmin = rk.alloc_summaries(back)
    rk.build_page_summaries(back, kmax, kmin)
    new = lambda: (torch.empty((3, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((3, 8), device="cuda"))
    (a, la), (b, lb) = new(), new()
    rk.q_attend(q, c.q, None, a, la, rk.q_alloc_workspace(rk.OP_ATTEND, q))
    rk.dense_decode(back, c.q, b, lb, rk.alloc_workspace(rk.OP_DENSE_DECODE, back))
    close(c, a, la, b, lb, ref.attention(c), 3000)
    row = rk.pages_row_len(back, budget)
    pages, want = (torch.full((3, 2, row), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    chan, want_chan = (torch.full((3, 2, 16), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    rk.q_hsa_decode(q, c.q, kmax, kmin, 16, budget, 0, a, la, pages, chan, rk.q_alloc_workspace(rk.OP_HSA_DECODE, q, budget))
    rk.hsa_decode(back, c.q, kmax, kmin, 16, budget, 0, b, lb, want, want_chan, rk.alloc_workspace(rk.OP_HSA_DECODE, back, budget))
    assert torch.equal(pages, want) and torch.equal(chan, want_chan)
    definition = selected(c, q, pages)
    close(c, a, la, b, lb, definition, budget)
    rk.q_attend(q, c.q, pages, a, la, rk.q_alloc_workspace(rk.OP_ATTEND, q, row))
    rk.attend(back, c.q, pages, b, lb, rk.alloc_workspace(rk.OP_ATTEND, back, row))
    close(c, a, la, b, lb, definition, budget)


def selected(c, q, pages):
    """Attention over the listed pages' tokens in 64 bits."""
    parts = [torch.zeros((len(c.lens), c.hq) + tail, dtype=torch.float64, device="cuda") for tail in ((128,), (), (128,), ())]
    G = c.hq // c.hkv
    for b, n in enumerate(c.lens):
        for g in range(c.hkv):
            t = [x for p in pages[b, g].tolist() if p >= 0 for x in range(p * q.page_size, min(n, (p + 1) * q.page_size))]
            one = ref.Case(0, [len(t)], [1], G, 1, 16, True)
            one.K, one.V, one.q = c.K[b:b + 1, g:g + 1, t], c.V[b:b + 1, g:g + 1, t], c.q[b:b + 1, g * G:(g + 1) * G]
            for all_, x in zip(parts, ref.attention(one)):
                all_[b, g * G:(g + 1) * G] = x[0]
    return parts


@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("ps", [4, 16])
def test_a_step_of_a_serving_loop(fmt, ps):
    """Append and step over codes; the same over the restored cache, which takes in the values that the codes stand for."""
    rng = random.Random(ps)
    lens = [700, 33]
    c = ref.Case(84, lens, [1, 1], 8, 2, 16, True, spare_pages=8)
    q = qr.like(c.cache, fmt, ps)
    rk.quantise(c.cache, q)
    kmax, kmin = rk.alloc_summaries(restored(q))
    rk.build_page_summaries(restored(q), kmax, kmin)
    ws, wsa = rk.q_alloc_workspace(rk.OP_HSA_DECODE, q, 128), rk.q_alloc_workspace(rk.OP_APPEND_CHUNK, q, 2)
    rope = rk.rope_frequencies(128, 10000.0, device="cuda")
    gen = torch.Generator().manual_seed(ps)
    row = rk.pages_row_len(q, 128)
    for step in range(20):
        mk = lambda h: torch.randn((2, h, 128), generator=gen).to(torch.bfloat16).cuda()
        query, turned, k, v = mk(8), mk(8), mk(2), mk(2)
        rk.q_append_chunk(q, c.chunk, k, v, kmax, kmin, wsa, rope=rope, q=query, q_out=turned)
        back = restored(q)
        assert back.seq_lens.tolist() == [n + step + 1 for n in lens]
        omax, omin = rk.alloc_summaries(back)
        rk.build_page_summaries(back, omax, omin)
        P = [-(-(n + step + 1) // ps) for n in lens]
        assert all(torch.equal(x[b, :, :, :P[b]], y[b, :, :, :P[b]]) for x, y in ((kmax, omax), (kmin, omin)) for b in range(2))
        outs = [(torch.empty((2, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((2, 8), device="cuda"),
                 torch.full((2, 2, row), -9, dtype=torch.int32, device="cuda")) for _ in range(2)]
        recent = rng.randrange(3)
        rk.q_hsa_decode(q, turned, kmax, kmin, 32, 128, recent, *outs[0], None, ws)
        rk.hsa_decode(back, turned, omax, omin, 32, 128, recent, *outs[1], None, rk.alloc_workspace(rk.OP_HSA_DECODE, back, 128))
        assert torch.equal(outs[0][2], outs[1][2])
        k_all, v_all = rk.unpack_cache(back)
        now = ref.Case(0, [n + step + 1 for n in lens], [1, 1], 8, 2, 16, True)
        now.K, now.V, now.q = k_all, v_all, turned
        close(now, *outs[0][:2], *outs[1][:2], selected(now, q, outs[0][2]), 128)
