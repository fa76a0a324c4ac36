"""Quantised caches: what is put into them, read back, and moved in them."""
import numpy as np
import pytest
import torch

import chunk_ref as ref
import quant_ref as qr
from paper_2502_14051_amd import rocketkv as rk

pytestmark = pytest.mark.gpu
LAYOUTS = [(16, False), (1, True), (3, True), (16, True), (64, True)]


def rows_with_everything(fmt):
    """Blocks whose values meet every code, the middles between codes and their neighbours, at several powers of two; blocks
    of zeros, of the smallest and largest numbers, and ones with values that are none."""
    g = qr.grid(fmt)
    g = g[:127] if fmt == rk.Q_E4M3 else g
    mids = (g[1:] + g[:-1]) / 2
    some = np.concatenate((g, mids, mids * (1 + 2.0 ** -7), mids * (1 - 2.0 ** -7)))
    some = torch.from_numpy(np.concatenate((some, -some))).to(torch.bfloat16)
    rng = np.random.default_rng(0)
    rows = []
    for scale in (0, 1, -3, 17, -40, -90, 110):
        v = some.double().numpy()[rng.permutation(len(some))]
        v = np.resize(v, (len(v) + 30) // 31 * 31).reshape(-1, 31)
        rows.append(np.ldexp(np.concatenate((v, np.full((len(v), 1), g[-1])), 1), scale))  # (the largest code in every block)
    rows.append(rng.standard_normal((64, 32)))
    rows.append(np.exp(4 * rng.standard_normal((64, 32))))
    top = float(torch.finfo(torch.bfloat16).max)
    odd = np.zeros((12, 32))
    odd[1, 3], odd[2, 5], odd[3, 0], odd[4, 31] = np.nan, np.inf, -np.inf, 2.0 ** -133
    odd[5], odd[6], odd[7, 1], odd[8] = top, -top, -0.0, 2.0 ** -126
    odd[9] = np.linspace(-top, top, 32)
    odd[10], odd[11] = 2.0 ** -105 * np.arange(32), 448.0 * 2.0 ** -100 / 32 * np.arange(32)
    rows.append(odd)
    x = np.concatenate(rows)
    x = np.concatenate((x, np.zeros((-len(x) % 4, 32)))).reshape(-1, 128)
    return torch.from_numpy(x).to(torch.bfloat16)


def same_numbers(a, b):
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a, 7.0), torch.nan_to_num(b, 7.0))


@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("ps,token_major", LAYOUTS)
def test_quantise_and_restore(fmt, ps, token_major):
    x = rows_with_everything(fmt)
    n = len(x)
    K = torch.stack((torch.stack((x, x.flip(0))), torch.stack((x.flip(1), x)))).cuda()  # [2 sequences][2 heads]
    lens = [n, n - 5]
    cache = rk.pack_cache(K, K.flip(1), lens, 4, ps, v_layout=rk.V_TOKEN_MAJOR if token_major else rk.V_CHANNEL_MAJOR)
    q = qr.like(cache, fmt, 5)
    before = [t.clone() for t in (q.k_codes, q.v_codes, q.k_scales, q.v_scales)]
    rk.quantise(cache, q)
    assert q.seq_lens.tolist() == lens
    used = torch.zeros(q.k_codes.shape[:3], dtype=torch.bool)
    for b, m in enumerate(lens):
        kc, ks, vc, vs = qr.tokens(q, b, m)
        for codes, scales, src in ((kc, ks, K[b]), (vc, vs, K[b].flip(0))):
            want, want_s = qr.quantise(src[:, :m].double().cpu().numpy(), fmt)
            assert np.array_equal(scales, want_s)
            assert np.array_equal(codes, want)
        t = torch.arange(m)
        used[q.block_table[b].cpu().long()[t // 5], :, t % 5] = True
    for t, old in zip((q.k_codes, q.v_codes, q.k_scales, q.v_scales), before):
        assert torch.equal(t.cpu()[~used], old.cpu()[~used]), "nothing but the tokens is written"
    for layout, other in ((rk.V_TOKEN_MAJOR, 7), (rk.V_TOKEN_MAJOR, 16), (rk.V_CHANNEL_MAJOR, 16)):
        back = rk.alloc_cache(2, 4, 2, 128, other, (n + other - 1) // other, "cuda", v_layout=layout)
        back.k_pool.fill_(3.0), back.v_pool.fill_(3.0)
        rk.restore(q, back)
        assert back.seq_lens.tolist() == lens
        k, v = rk.unpack_cache(back)
        for b, m in enumerate(lens):
            kc, ks, vc, vs = qr.tokens(q, b, m)
            assert same_numbers(k[b, :, :m].cpu().double(), torch.from_numpy(qr.values(kc, ks, fmt)))
            assert same_numbers(v[b, :, :m].cpu().double(), torch.from_numpy(qr.values(vc, vs, fmt)))
            assert (k[b, :, m:] == 3).all(), "keys behind the last token are left as they were"
            behind = v[b, :, m:] if layout == rk.V_TOKEN_MAJOR else v[b, :, (m + 15) // 16 * 16:]
            assert (behind == 3).all()
            if layout == rk.V_CHANNEL_MAJOR:
                assert (v[b, :, m:(m + 15) // 16 * 16] == 0).all(), "zeros to the end of the tile"
        # what was restored quantises to the same values
        again = qr.like(back, fmt, 16)
        rk.quantise(back, again)
        for b, m in enumerate(lens):
            one, two = qr.tokens(q, b, m), qr.tokens(again, b, m)
            for i in (0, 2):
                assert np.array_equal(qr.values(one[i], one[i + 1], fmt), qr.values(two[i], two[i + 1], fmt), equal_nan=True)


@pytest.mark.parametrize("token_major", [False, True])
def test_convert_absent_pages_and_lengths(token_major):
    c = ref.Case(3, [100, 0, 1, 16, 333], [0] * 5, 4, 2, 16, token_major)
    c.drop_pages([(0, 2), (4, 0), (4, 20)])
    q = qr.like(c.cache, rk.Q_E4M3, 4)
    q.block_table[0, 3] = -1
    q.block_table[4, 82] = 1 << 30
    rk.quantise(c.cache, q)
    assert q.seq_lens.tolist() == c.lens
    back = rk.alloc_cache(5, 4, 2, 128, 16, c.cache.pages_cap, "cuda", v_layout=c.cache.v_layout)
    back.k_pool.fill_(3.0), back.v_pool.fill_(3.0)
    rk.restore(q, back)
    k, v = rk.unpack_cache(back)
    for b, n in enumerate(c.lens):
        for got, src in ((k, c.K), (v, c.V)):
            codes, scales = qr.quantise(src[b, :, :n].double().cpu().numpy(), rk.Q_E4M3)
            want = torch.from_numpy(qr.values(codes, scales, rk.Q_E4M3)) if n else torch.zeros(2, 0, 128)
            t = torch.arange(n)
            gone = ~c.present(b).cpu() if n else torch.zeros(0, dtype=torch.bool)
            if b == 0:
                gone |= t // 4 == 3
            if b == 4:
                gone |= t // 4 == 82
            assert torch.equal(got[b, :, :n].cpu().double(), torch.where(gone[:, None], 0.0, want))
    # a length that either side has no room for counts as none
    small = rk.alloc_qcache(5, 4, 2, 4, 64, "cuda")
    rk.quantise(c.cache, small)
    assert small.seq_lens.tolist() == [100, 0, 1, 16, 0]
    c.cache.seq_lens[0] = -3
    rk.quantise(c.cache, small)
    assert small.seq_lens.tolist() == [0, 0, 1, 16, 0]


def appended(c, old, fmt, ps, k, v, chunk, q=None, **kw):
    """A quantised cache that held the Case's tokens `old` and took in the chunk; its summaries."""
    qc = qr.like(c.cache, fmt, ps)
    rk.quantise(c.cache, qc)
    kmax, kmin = (torch.full((c.cache.batch, c.hkv, 128, qc.pages_cap), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    fill_summaries(qc, old, kmax, kmin)
    ws = rk.q_alloc_workspace(rk.OP_APPEND_CHUNK, qc, c.rows)
    rk.q_append_chunk(qc, chunk, k, v, kmax, kmin, ws, q=q, **kw)
    return qc, kmax, kmin


def fill_summaries(qc, lens, kmax, kmin):
    """By way of the restored cache."""
    back = rk.alloc_cache(qc.batch, qc.n_q_heads, qc.n_kv_heads, 128, qc.page_size, qc.pages_cap, "cuda",
                          block_table=qc.block_table, n_phys_pages=qc.k_codes.shape[0], v_layout=rk.V_TOKEN_MAJOR)
    rk.restore(qc, back)
    rk.build_page_summaries(back, kmax, kmin)


@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("ps", [1, 3, 16, 64])
@pytest.mark.parametrize("olds,news", [([5], [1]), ([0, 30, 17], [200, 1, 0]), ([100, 3, 64, 0], [29, 300, 64, 1])])
def test_append(fmt, ps, olds, news):
    """As the bf16 append followed by a conversion, where nothing is turned; summaries are of what the cache holds."""
    c = ref.Case(11, olds, [0] * len(olds), 8, 2, 16, True, spare_pages=40)
    rows = 2 + sum(news) + 3
    c.rows = rows
    gen = torch.Generator().manual_seed(5)
    joint = torch.randn((rows, 5, 128), generator=gen).to(torch.bfloat16).cuda()
    k, v = joint[:, :2], joint[:, 3:]
    starts = torch.tensor([2 + sum(news[:b]) for b in range(len(news) + 1)], dtype=torch.int32).cuda()
    chunk = rk.Chunk(starts, rows)
    q, kmax, kmin = appended(c, olds, fmt, ps, k, v, chunk)
    lens = [o + n for o, n in zip(olds, news)]
    assert q.seq_lens.tolist() == lens
    for b, (o, n) in enumerate(zip(olds, lens)):
        kc, ks, vc, vs = qr.tokens(q, b, n)
        at = slice(int(starts[b]), int(starts[b + 1]))
        for codes, scales, old, new in ((kc, ks, c.K, k), (vc, vs, c.V, v)):
            x = torch.cat((old[b, :, :o], new[at].transpose(0, 1)), 1).double().cpu().numpy()
            want, want_s = qr.quantise(x, fmt)
            assert np.array_equal(scales, want_s) and np.array_equal(codes, want)
    wmax, wmin = torch.full_like(kmax, 5.0), torch.full_like(kmin, 5.0)
    fill_summaries(q, lens, wmax, wmin)
    assert torch.equal(kmax, wmax) and torch.equal(kmin, wmin)


@pytest.mark.parametrize("rot,interleaved", [(128, False), (128, True), (64, False), (36, False)])
@pytest.mark.parametrize("fmt", qr.FORMATS)
def test_append_turned(fmt, rot, interleaved):
    """Codes of turned keys: the code of the key in 64 bits, but where fp32 falls on the other side of a middle."""
    olds, news = [40, 0], [7, 60]
    c = ref.Case(12, olds, [0, 0], 4, 2, 16, True, spare_pages=8)
    c.rows = 67
    gen = torch.Generator().manual_seed(6)
    k, v = (torch.randn((67, 2, 128), generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    q = torch.randn((67, 4, 128), generator=gen).to(torch.bfloat16).cuda()
    q_out, q_want = torch.empty_like(q), torch.empty_like(q)
    rope = rk.rope_frequencies(rot, 500000.0, device="cuda", interleaved=interleaved)
    pos = torch.randint(0, 131072, (67,), generator=gen, dtype=torch.int32).cuda()
    chunk = rk.Chunk(torch.tensor([0, 7, 67], dtype=torch.int32).cuda(), 67)
    qc, kmax, kmin = appended(c, olds, fmt, 16, k, v, chunk, q=q, rope=rope, positions=pos, q_out=q_out)
    rk.rope(rope, pos, q, q_want)
    assert torch.equal(q_out, q_want)
    f = rope.inv_freq.cpu().double().numpy()
    ang = pos.cpu().double().numpy()[:, None] * f
    cos, sin = np.cos(ang)[:, None], np.sin(ang)[:, None]
    x = k.double().cpu().numpy()
    y = x.copy()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
    for b, at in enumerate((slice(0, 7), slice(7, 67))):
        kc, ks, vc, vs = qr.tokens(qc, b, olds[b] + news[b])
        got = qr.values(kc, ks, fmt)[:, olds[b]:]
        want = y[at].transpose(1, 0, 2)
        # half a step of the code's binade (of the smallest one below), and of the next power of two where fp32 sees a
        # block's maximum beyond the largest code; the turn in fp32: sine and cosine to 2^-22, two products and a sum
        scale = np.repeat(np.ldexp(1.0, ks[:, olds[b]:].astype(np.int64) - 127), 32, -1)
        bits, low = (3, -6) if fmt == rk.Q_E4M3 else (1, 0)
        half = np.maximum(np.abs(want) * 2.0 ** (-bits - 1), scale * 2.0 ** (low - bits - 1))
        assert (np.abs(got - want) <= half + 2.0 ** -20 * np.abs(x).max()).all()
        top = np.abs(want).reshape(want.shape[:-1] + (4, 32)).max(-1)
        limit = (448.0 if fmt == rk.Q_E4M3 else 6.0) * np.ldexp(1.0, ks[:, olds[b]:].astype(np.int64) - 127)
        assert (top <= limit * (1 + 2.0 ** -20)).all() and (top > limit / 2 * (1 - 2.0 ** -20)).all()
    wmax, wmin = torch.full_like(kmax, 5.0), torch.full_like(kmin, 5.0)
    fill_summaries(qc, None, wmax, wmin)
    assert torch.equal(kmax, wmax) and torch.equal(kmin, wmin)


@pytest.mark.parametrize("fmt", qr.FORMATS)
def test_append_without_room_or_pages(fmt):
    """A sequence without room is left as it was; a token of an absent page goes nowhere; no summaries."""
    qc = rk.alloc_qcache(3, 4, 1, 4, 8, "cuda", fmt, torch.arange(24, dtype=torch.int32).reshape(3, 8).cuda(), 24)
    for x in (qc.k_codes, qc.v_codes, qc.k_scales, qc.v_scales):
        x.fill_(9)
    qc.seq_lens.copy_(torch.tensor([30, 2, 0]))
    qc.block_table[1, 1] = -1
    new = [3, 8, 32]
    k = torch.randn((43, 1, 128)).to(torch.bfloat16).cuda()
    chunk = rk.Chunk(torch.tensor([0, 3, 11, 43], dtype=torch.int32).cuda(), 43)
    ws = rk.q_alloc_workspace(rk.OP_APPEND_CHUNK, qc, 43)
    rk.q_append_chunk(qc, chunk, k, k, None, None, ws)
    assert qc.seq_lens.tolist() == [30, 10, 32]
    assert (qc.k_codes[:8] == 9).all() and (qc.v_scales[:8] == 9).all(), "without room"
    assert (qc.k_codes[9] == 9).all() and (qc.k_codes[8, :, :2] == 9).all()
    want, scales = qr.quantise(k[:, 0].double().cpu().numpy(), fmt)
    want = torch.from_numpy(qr.packed(want, fmt))
    assert torch.equal(qc.k_codes[8, 0, 2:].cpu(), want[3:5]) and torch.equal(qc.k_codes[10, 0, :2].cpu(), want[9:11])
    assert torch.equal(qc.v_codes[16:, 0].reshape(32, -1).cpu(), want[11:])
    assert torch.equal(qc.v_scales[16:, 0].reshape(32, 4).cpu(), torch.from_numpy(scales[11:]))


def move(lens, news, keep, starts, K):
    """Tokens [b] -> list of source tokens after keeping."""
    order = []
    for b, (n, new) in enumerate(zip(lens, news)):
        old = n - new
        flags = keep[starts[b]:starts[b] + new].tolist()
        order.append(list(range(old)) + [old + i for i, f in enumerate(flags) if f])
    return order


KEPT = [([50], [10], 0.4), ([300, 40, 7, 31], [300, 0, 1, 20], 0.5), ([17, 700], [17, 600], 0.9), ([64, 64], [32, 5], 0.0), ([33, 90], [2, 40], 1.0)]


@pytest.mark.parametrize("ps,token_major", LAYOUTS)
@pytest.mark.parametrize("lens,news,share", KEPT)
def test_keep_tokens(ps, token_major, lens, news, share):
    c = ref.Case(21, lens, news, 4, 2, ps, token_major, pad=(3, 2))
    keep = (torch.rand((c.rows,), generator=torch.Generator().manual_seed(1)) < share).cuda()
    order = move(lens, news, keep, c.starts, c.K)
    kmax, kmin = rk.alloc_summaries(c.cache)
    rk.build_page_summaries(c.cache, kmax, kmin)
    ws = rk.alloc_workspace(rk.OP_APPEND_CHUNK, c.cache, c.rows)
    rk.keep_tokens(c.cache, c.chunk, keep, kmax, kmin, ws)
    assert c.cache.seq_lens.tolist() == [len(o) for o in order]
    k, v = rk.unpack_cache(c.cache)
    wmax, wmin = rk.alloc_summaries(c.cache)
    rk.build_page_summaries(c.cache, wmax, wmin)
    for b, o in enumerate(order):
        assert torch.equal(k[b, :, :len(o)], c.K[b][:, o]) and torch.equal(v[b, :, :len(o)], c.V[b][:, o])
        # what stands behind the last of the chunk's tokens is left as it was
        P = (len(o) + ps - 1) // ps
        assert torch.equal(kmax[b, :, :, :P], wmax[b, :, :, :P]) and torch.equal(kmin[b, :, :, :P], wmin[b, :, :, :P])


@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("ps", [1, 5, 16, 64])
@pytest.mark.parametrize("lens,news,share", KEPT)
def test_q_keep_tokens(fmt, ps, lens, news, share):
    c = ref.Case(22, lens, news, 4, 2, 16, True, pad=(3, 2))
    keep = (torch.rand((c.rows,), generator=torch.Generator().manual_seed(2)) < share).to(torch.uint8).cuda() * 200
    order = move(lens, news, keep, c.starts, c.K)
    q = qr.like(c.cache, fmt, ps)
    rk.quantise(c.cache, q)
    before = [qr.tokens(q, b, n) for b, n in enumerate(lens)]
    kmax, kmin = (torch.zeros((len(lens), 2, 128, q.pages_cap), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    fill_summaries(q, lens, kmax, kmin)
    ws = rk.q_alloc_workspace(rk.OP_APPEND_CHUNK, q, c.rows)
    rk.q_keep_tokens(q, c.chunk, keep, kmax, kmin, ws)
    assert q.seq_lens.tolist() == [len(o) for o in order]
    wmax, wmin = torch.zeros_like(kmax), torch.zeros_like(kmin)
    fill_summaries(q, lens, wmax, wmin)
    for b, o in enumerate(order):
        for got, had in zip(qr.tokens(q, b, len(o)), before[b]):
            assert np.array_equal(got, had[:, o])
        P = (len(o) + ps - 1) // ps
        assert torch.equal(kmax[b, :, :, :P], wmax[b, :, :, :P]) and torch.equal(kmin[b, :, :, :P], wmin[b, :, :, :P])


@pytest.mark.parametrize("token_major", [False, True])
def test_keep_absent_pages_and_bad_lengths(token_major):
    c = ref.Case(23, [60, 40, 5], [40, 10, 5], 4, 2, 16, token_major)
    c.drop_pages([(0, 1), (1, 2)])
    c.cache.seq_lens[2] = 4  # fewer tokens than rows
    keep = torch.zeros((c.rows,), dtype=torch.uint8, device="cuda")
    keep[[5, 20, 39]] = 1   # of sequence 0: token 25 in the absent page 1, tokens 40 and 59; places 20, 21, 22, all in it
    keep[[40, 44]] = 1      # of sequence 1: tokens 30 and 34 (absent) to 30 and 31
    kmax, kmin = rk.alloc_summaries(c.cache)
    rk.build_page_summaries(c.cache, kmax, kmin)
    k0, v0 = c.cache.k_pool.clone(), c.cache.v_pool.clone()
    max0 = kmax.clone()
    ws = rk.alloc_workspace(rk.OP_APPEND_CHUNK, c.cache, c.rows)
    rk.keep_tokens(c.cache, c.chunk, keep, kmax, kmin, ws)
    assert c.cache.seq_lens.tolist() == [23, 32, 4]
    page = int(c.cache.block_table[1, 1])
    want_k, want_v = k0.clone(), v0.clone()
    want_k[page, :, 15] = 0
    if token_major:
        want_v[page, :, 15] = 0
    else:
        want_v[page, :, :, 15] = 0
    assert torch.equal(c.cache.k_pool, want_k) and torch.equal(c.cache.v_pool, want_v)
    assert torch.equal(kmax[0, :, :, 1], max0[0, :, :, 1]), "no summary of an absent page"
    assert torch.equal(kmax[1, :, :, 1], want_k[page].amax(1))
    assert torch.equal(kmax[2], max0[2])
