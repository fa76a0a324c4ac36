"""Appends of chunks in every shape of block that a launch may divide them into: blocks of one page to 32, of several lots of 32
tokens, one head of keys or several to a workgroup, blocks of one query token to 17; into bf16 caches and into codes.

What a token's key, value and query become depends on nothing but the token and its position.  So bf16 caches are compared with
the rows that rope() turns; quantised ones with appends of 64 tokens at a time into pages of 16, whose codes test_gpu_qcache
compares with their definition.  Summaries are formed anew from what the caches hold."""
import pytest
import torch

import chunk_ref as ref
import quant_ref as qr
from paper_2502_14051_amd import rocketkv as rk

KINDS = [("channel", 16), ("token", 1), ("token", 3), ("token", 16), ("token", 33), ("token", 64)]
CODE_PAGES = [1, 3, 16, 33, 64]


def forms(n_tokens, batch, hq, hkv, ps):
    """How launch_append_any divides a chunk: pages of a block, heads of a workgroup, tokens of a block of queries."""
    pages = min(((128 + ps - 1) // ps + 7) // 8 * 8, 32)
    blocks = lambda p: min(n_tokens // (p * ps) + 2 * batch, n_tokens)
    while pages > 8 and blocks(pages) * hkv < 1024:
        pages -= 8
    while pages > 1 and pages * ps > 32 and min(n_tokens // (pages * ps) + batch, n_tokens) * hkv < 432:
        pages //= 2
    heads = min(hkv, 4)
    while heads > 1 and blocks(pages) * -(-hkv // heads) < 1024:
        heads //= 2
    while heads > 1 and heads * 2 * 128 * pages * 2 > 32 * 1024:
        heads //= 2
    q_block = min(max(min(-(-n_tokens // 512), max(128 // hq, 1)), -(-n_tokens // 2048)), 32)
    return pages, heads, q_block


# sequences' tokens, new ones, heads of queries and of keys
CASES = {
    "over 512": ([7, 0], [300, 250], 32, 8),
    "over 2048": ([70, 5, 33], [2000, 1, 157], 32, 8),
    "8192 of one": ([130], [8193], 8, 8),
    "blocks of 4 pages": ([3], [6000], 8, 8),
    "10000 of one": ([3], [10000], 8, 8),
    "many sequences": ([(7 * b) % 50 for b in range(130)], [0 if b % 9 == 4 else 290 + b if b % 26 == 3 else 15 + b % 40 for b in range(130)], 32, 16),
    "fewer heads": ([(5 * b) % 40 for b in range(130)], [1 + (b * 11) % 70 for b in range(130)], 8, 8),
    "a long prompt": ([11], [33000], 8, 8),
}
# rotated channels, pairs of neighbours, positions given
ROPES = {"half": (128, False, False), "pairs": (128, True, True), "odd": (36, False, False), "part": (64, False, True)}
# every case in every page size, the rotations in turn
BF16 = [(layout, ps, name, list(ROPES)[(i + j) % 4]) for i, (layout, ps) in enumerate(KINDS) for j, name in enumerate(CASES)]
CODES = [(ps, name, list(ROPES)[(i + j) % 4]) for i, ps in enumerate(CODE_PAGES) for j, name in enumerate(CASES)]


def test_the_cases_take_every_form():
    """What the launch divides by, as it stands; a rule that moves has to move this."""
    have = {ps: {n: forms(sum(news) + 5, len(news), hq, hkv, ps) for n, (_, news, hq, hkv) in CASES.items()} for ps in CODE_PAGES}
    every = [f for by in have.values() for f in by.values()]
    assert {f[0] for f in every} == {1, 2, 4, 8, 16, 24, 32} and {f[1] for f in every} == {1, 2, 4} and {f[2] for f in every} == {2, 4, 9, 12, 16, 17}
    assert have[16]["many sequences"][1] == 4 and have[16]["fewer heads"][1] == 2 and have[16]["a long prompt"][:2] == (8, 2)
    assert have[16]["blocks of 4 pages"][0] == 4 and have[64]["over 2048"][0] == 1 and have[16]["over 512"][0] == 2


class Chunk:
    """What a program has in hand: the rows of one joint projection, a few in front of and behind the sequences' among them."""

    def __init__(self, olds, news, hq, hkv, rot, interleaved, given):
        gen = torch.Generator().manual_seed(sum(news) + hq)
        self.olds, self.news, self.hq, self.hkv = olds, news, hq, hkv
        self.rows = 2 + sum(news) + 3
        starts = torch.cat((torch.zeros(1, dtype=torch.int64), torch.cumsum(torch.tensor(news), 0))) + 2
        self.starts = starts.tolist()
        self.chunk = rk.Chunk(starts.to(torch.int32).cuda(), self.rows)
        joint = torch.randn((self.rows, hq + 2 * hkv, 128), generator=gen).to(torch.bfloat16).cuda()
        self.q, self.k, self.v = joint[:, :hq], joint[:, hq:hq + hkv], joint[:, hq + hkv:]
        self.rope = rk.rope_frequencies(rot, 500000.0, device="cuda", interleaved=interleaved)
        pos = torch.zeros(self.rows, dtype=torch.int32)
        for b, (o, n) in enumerate(zip(olds, news)):
            pos[self.rows_of(b)] = torch.arange(o, o + n, dtype=torch.int32)
        self.pos = pos.cuda()
        if given:
            self.pos += torch.randint(0, 90000, (self.rows,), generator=gen, dtype=torch.int32).cuda()
        self.given = self.pos if given else None

    def rows_of(self, b):
        return slice(self.starts[b], self.starts[b + 1])

    def turned(self, x):
        y = torch.empty(x.shape, dtype=x.dtype, device="cuda")
        rk.rope(self.rope, self.pos, x, y)
        return y

    def check_queries(self, q_out):
        at = slice(self.starts[0], self.starts[-1])
        assert torch.equal(q_out[at], self.turned(self.q)[at])
        assert (q_out[:2] == 7).all() and (q_out[-3:] == 7).all(), "rows of no sequence are left as they were"


def check_summaries(K, olds, lens, ps, kmax, kmin, before):
    """K: [batch][heads][room][128], what the cache holds."""
    for b, (o, n) in enumerate(zip(olds, lens)):
        if n == o:
            assert torch.equal(kmax[b], before[0][b]) and torch.equal(kmin[b], before[1][b])
            continue
        first, last = o // ps, (n - 1) // ps + 1
        x = K[b, :, first * ps:last * ps].float()
        there = (torch.arange(first * ps, last * ps, device="cuda") < n)[None, :, None]
        pages = lambda y, f: f(y.reshape(y.shape[0], last - first, ps, 128), 2).transpose(1, 2)
        assert torch.equal(kmax[b, :, :, first:last].float(), pages(torch.where(there, x, -torch.inf), torch.amax))
        assert torch.equal(kmin[b, :, :, first:last].float(), pages(torch.where(there, x, torch.inf), torch.amin))
        for s, w in ((kmax, before[0]), (kmin, before[1])):
            assert torch.equal(s[b, :, :, :first], w[b, :, :, :first]) and torch.equal(s[b, :, :, last:], w[b, :, :, last:]), "other pages' columns"


def summaries(cache, K, olds, ps):
    """Of the tokens there are; 5 elsewhere."""
    kmax, kmin = (torch.full((cache.batch, cache.n_kv_heads, 128, cache.pages_cap), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for b, o in enumerate(olds):
        for p in range((o + ps - 1) // ps):
            x = K[b, :, p * ps:min(o, (p + 1) * ps)]
            kmax[b, :, :, p], kmin[b, :, :, p] = x.amax(1), x.amin(1)
    return kmax, kmin


@pytest.mark.gpu
@pytest.mark.parametrize("layout,ps,name,rope", BF16)
def test_bf16(layout, ps, name, rope):
    olds, news, hq, hkv = CASES[name]
    t = Chunk(olds, news, hq, hkv, *ROPES[rope])
    lens = [o + n for o, n in zip(olds, news)]
    gen = torch.Generator().manual_seed(3)
    cap = ((max(lens) + ps - 1) // ps + 7) // 8 * 8
    start = [torch.randn((len(olds), hkv, max(olds) + 1, 128), generator=gen).to(torch.bfloat16).cuda() for _ in range(2)]
    table = torch.randperm(len(olds) * cap, generator=gen).reshape(len(olds), cap).to(torch.int32).cuda()
    cache = rk.pack_cache(*start, olds, hq, ps, pages_cap=cap, block_table=table, n_phys_pages=len(olds) * cap,
                          v_layout=rk.V_CHANNEL_MAJOR if layout == "channel" else rk.V_TOKEN_MAJOR)
    want = rk.unpack_cache(cache)
    kmax, kmin = summaries(cache, want[0], olds, ps)
    before = kmax.clone(), kmin.clone()
    q_out = torch.full((t.rows, hq, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = rk.alloc_workspace(rk.OP_APPEND_CHUNK, cache, t.rows)
    rk.append_chunk(cache, t.chunk, t.k, t.v, kmax, kmin, ws, rope=t.rope, positions=t.given, q=t.q, q_out=q_out)
    t.check_queries(q_out)
    for b, (o, n) in enumerate(zip(olds, lens)):
        for w, rows in zip(want, (t.turned(t.k), t.v)):
            w[b, :, o:n] = rows[t.rows_of(b)].transpose(0, 1)
    assert cache.seq_lens.tolist() == lens
    have = rk.unpack_cache(cache)
    assert torch.equal(have[0], want[0]), "keys"
    assert torch.equal(have[1], want[1]), "values"
    check_summaries(want[0], olds, lens, ps, kmax, kmin, before)


def by_pieces(t, start, fmt, cap):
    """A cache with pages of 16 that takes the same tokens in by 64 at most of each sequence a call."""
    qc = rk.alloc_qcache(len(t.olds), t.hq, t.hkv, 16, cap, "cuda", fmt)
    rk.quantise(start, qc)
    ws = rk.q_alloc_workspace(rk.OP_APPEND_CHUNK, qc, t.rows)
    q_out = torch.empty((64 * len(t.olds), t.hq, 128), dtype=torch.bfloat16, device="cuda")
    for i in range(0, max(t.news), 64):
        rows, starts = [], [0]
        for b, n in enumerate(t.news):
            rows += range(t.starts[b] + min(i, n), t.starts[b] + min(i + 64, n))
            starts.append(len(rows))
        at = torch.tensor(rows, device="cuda")
        chunk = rk.Chunk(torch.tensor(starts, dtype=torch.int32, device="cuda"), len(rows))
        rk.q_append_chunk(qc, chunk, t.k[at], t.v[at], None, None, ws, rope=t.rope, positions=t.pos[at], q=t.q[at], q_out=q_out[:len(rows)])
    return qc


def by_token(qc):
    """Codes and scales [batch][heads][room][...] of the keys, then of the values."""
    b = torch.arange(qc.batch * qc.pages_cap, device="cuda") if qc.block_table is None else qc.block_table.reshape(-1).long()
    return [x[b].reshape(qc.batch, qc.pages_cap, qc.n_kv_heads, qc.page_size, -1).transpose(1, 2).reshape(qc.batch, qc.n_kv_heads, qc.pages_cap * qc.page_size, -1)
            for x in (qc.k_codes, qc.k_scales, qc.v_codes, qc.v_scales)]


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("ps,name,rope", CODES)
def test_codes(fmt, ps, name, rope):
    olds, news, hq, hkv = CASES[name]
    t = Chunk(olds, news, hq, hkv, *ROPES[rope])
    lens = [o + n for o, n in zip(olds, news)]
    gen = torch.Generator().manual_seed(4)
    start = rk.pack_cache(*(torch.randn((len(olds), hkv, max(olds) + 1, 128), generator=gen).to(torch.bfloat16).cuda() for _ in range(2)), olds, hq, 16)
    other = by_pieces(t, start, fmt, (max(lens) + 15) // 16)
    assert other.seq_lens.tolist() == lens
    cap = ((max(lens) + ps - 1) // ps + 7) // 8 * 8
    table = torch.randperm(len(olds) * cap, generator=gen).reshape(len(olds), cap).to(torch.int32).cuda()
    qc = rk.alloc_qcache(len(olds), hq, hkv, ps, cap, "cuda", fmt, table)
    for x in (qc.k_codes, qc.v_codes, qc.k_scales, qc.v_scales):
        x.fill_(255)
    rk.quantise(start, qc)
    untouched = by_token(qc)
    k0 = values(untouched[0], untouched[1], fmt)
    kmax, kmin = summaries(qc, k0, olds, ps)
    before = kmax.clone(), kmin.clone()
    q_out = torch.full((t.rows, hq, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = rk.q_alloc_workspace(rk.OP_APPEND_CHUNK, qc, t.rows)
    rk.q_append_chunk(qc, t.chunk, t.k, t.v, kmax, kmin, ws, rope=t.rope, positions=t.given, q=t.q, q_out=q_out)
    t.check_queries(q_out)
    assert qc.seq_lens.tolist() == lens
    have, want = by_token(qc), by_token(other)
    for what, h, w, u in zip(("codes of keys", "scales of keys", "codes of values", "scales of values"), have, want, untouched):
        for b, n in enumerate(lens):
            assert torch.equal(h[b, :, :n], w[b, :, :n]), f"{what} of sequence {b}"
            assert torch.equal(h[b, :, n:], u[b, :, n:]), f"{what} behind sequence {b}"
    check_summaries(values(have[0], have[1], fmt), olds, lens, ps, kmax, kmin, before)


def values(codes, scales, fmt):
    """What they stand for, in bf16."""
    g = torch.from_numpy(qr.grid(fmt)).float().cuda()
    if fmt == rk.Q_E2M1:
        codes = torch.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[:-1] + (128,))
    half = 128 if fmt == rk.Q_E4M3 else 8
    v = torch.where(codes >= half, -1.0, 1.0) * g[(codes % half).long()]
    s = torch.where(scales == 255, torch.nan, torch.ldexp(torch.ones((), device="cuda"), scales.int() - 127))
    return (v * s.repeat_interleave(32, -1)).to(torch.bfloat16)
