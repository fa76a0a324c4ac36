"""Attention over quantised caches, and by masks over any, against its definition in 64 bits over the values they hold."""
import random

import pytest
import torch

import chunk_ref as ref
import quant_ref as qr
from paper_2502_14051_amd import rocketkv as rk

pytestmark = pytest.mark.gpu


def attend(c, q, mask=None, ws=None, lse=True, fill=7.0):
    out = torch.full((c.rows, c.hq, ref.D), fill, dtype=torch.bfloat16, device="cuda")
    out_lse = torch.full((c.rows, c.hq), fill, device="cuda") if lse else None
    if isinstance(q, rk.QCache):
        ws = rk.q_alloc_workspace(rk.OP_CHUNK_ATTEND, q, c.rows) if ws is None else ws
        rk.q_chunk_attend(q, c.chunk, c.q, out, out_lse, ws, mask=mask)
    else:
        ws = rk.alloc_workspace(rk.OP_CHUNK_ATTEND, q, c.rows) if ws is None else ws
        rk.masked_attend(q, c.chunk, mask, c.q, out, out_lse, ws)
    return out, out_lse


@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("ps", [1, 3, 16, 64])
@pytest.mark.parametrize("lens,news", [
    ([1], [1]),                                   # one token of one
    ([64], [64]), ([65], [65]), ([63], [1]),      # around a step of keys
    ([700, 1, 33, 500], [1, 1, 33, 37]),          # single tokens, a whole prompt and a piece of one
    ([1500, 130], [300, 130]),                    # several tiles of rows
    ([400, 300, 0, 200], [0, 20, 0, 1]),          # sequences without new tokens, and without any
])
def test_lengths(fmt, ps, lens, news):
    c = ref.Case(1, lens, news, 8, 2, 16, True)
    ref.check_attention(c, *attend(c, qr.take_over(c, fmt, ps)))


@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (5, 1), (16, 1), (12, 4), (40, 8), (7, 7)])
@pytest.mark.parametrize("new", [1, 2, 9, 70])
def test_groups(fmt, hq, hkv, new):
    c = ref.Case(2, [300, 171], [new, max(1, new // 2)], hq, hkv, 16, True)
    ref.check_attention(c, *attend(c, qr.take_over(c, fmt)))


@pytest.mark.parametrize("fmt,ps", [(rk.Q_E4M3, 16), (rk.Q_E2M1, 5)])
@pytest.mark.parametrize("lens,news", [([9000], [1]), ([9000], [3]), ([9000], [70]), ([9001, 40, 5000], [1, 5, 4]), ([20000, 19000], [130, 1])])
def test_long_caches_cut(fmt, ps, lens, news):
    """Few rows over many keys: every tile's keys are cut, the parts merged."""
    c = ref.Case(3, lens, news, 4, 1, 16, True)
    ref.check_attention(c, *attend(c, qr.take_over(c, fmt, ps)))


@pytest.mark.parametrize("fmt", qr.FORMATS)
def test_many_sequences(fmt):
    """More than one sequence a lane in the division, most of them short."""
    lens = [1 + (37 * b) % 90 for b in range(150)]
    news = [0 if b % 7 == 3 else 1 + (b * 11) % lens[b] if b % 5 == 0 else 1 for b in range(150)]
    c = ref.Case(4, lens, news, 4, 2, 16, True)
    ref.check_attention(c, *attend(c, qr.take_over(c, fmt)))


@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("news,lens", [([1100], [2000]), ([640, 700], [700, 1500]), ([300, 3, 400], [900, 1400, 400])])
def test_tiles_beside_the_chip(fmt, news, lens):
    c = ref.Case(5, lens, news, 32, 8, 16, True)
    ref.check_attention(c, *attend(c, qr.take_over(c, fmt)))


@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("news,lens", [([640, 700], [700, 1500]), ([300, 3, 400], [900, 1400, 400]), ([40], [40])])
@pytest.mark.parametrize("kind", ["causal", "tree", "random"])
def test_tiles_where_there_is_room_for_more(fmt, news, lens, kind):
    """The same over caches that could hold more than 2048 tokens of a sequence, which take the larger tiles; and by masks."""
    c = ref.Case(23, lens, news, 16, 2, 16, True)
    q = qr.take_over(c, fmt, 16, spare=130)
    assert q.pages_cap * 16 > 2048
    if kind == "causal":
        ref.check_attention(c, *attend(c, q))
    else:
        m = qr.MaskedCase(c, masked(24, lens, news, kind))
        m.check(*attend(c, q, m.mask))


@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("hq,hkv", [(8, 2), (3, 1), (16, 1), (40, 8)])
@pytest.mark.parametrize("lens,news", [
    ([60] * 5 + [300], [1] * 5 + [60]),          # single tokens, and a sequence of many tiles among them
    ([5000, 3000, 17, 900], [4, 3, 2, 1]),        # pieces that end inside one tile and go on in the next
    ([2000, 0, 33, 7000, 1], [8, 0, 7, 1, 1]),
    ([40000, 64], [1, 1]), ([33] * 70, [1] * 70), ([600] * 40, [2] * 40),
])
def test_few_rows(fmt, hq, hkv, lens, news):
    """Wavefronts with keys of their own: tiles of 16, 32 and 64 rows, cut where the pieces of the work end."""
    c = ref.Case(8, lens, news, hq, hkv, 16, True)
    ref.check_attention(c, *attend(c, qr.take_over(c, fmt, 8)))


@pytest.mark.parametrize("fmt", qr.FORMATS)
def test_one_workspace_for_all(fmt):
    ws = None
    for lens, news in (([9000], [70]), ([40], [40]), ([9000, 9000], [1, 300]), ([5000], [3]), ([5000], [1])):
        c = ref.Case(6, lens, news, 4, 1, 16, True)
        q = qr.take_over(c, fmt)
        ws = rk.q_alloc_workspace(rk.OP_CHUNK_ATTEND, q, 1) if ws is None else ws
        ref.check_attention(c, *attend(c, q, ws=ws))


@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("news", [[150, 3], [1, 4]])
def test_large_logits(fmt, news):
    """Maxima that move by hundreds from step to step, and rows that one key dominates."""
    c = ref.Case(5, [1000, 600], news, 8, 2, 16, True, scale=6.0)
    ref.check_attention(c, *attend(c, qr.take_over(c, fmt)))


@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("news", [[100, 90, 16], [1, 2, 1]])
def test_absent_pages_and_rows_of_nobody(fmt, news):
    c = ref.Case(6, [600, 90, 16], news, 8, 2, 16, True, pad=(3, 5))
    q = qr.take_over(c, fmt, 16)
    for b, p in [(0, 0), (0, 7), (0, 31), (0, 36), (1, 0), (1, 1), (2, 0)]:
        q.block_table[b, p] = -1 if p % 2 else 1 << 30
        c.cache.block_table[b, p] = -1
    out, lse = attend(c, q)
    ref.check_attention(c, out, lse)
    assert (out[c.rows_of(2)] == 0).all() and torch.isneginf(lse[c.rows_of(2)]).all()
    for r in list(range(3)) + list(range(c.rows - 5, c.rows)):
        assert (out[r] == 7).all() and (lse[r] == 7).all(), "rows of no sequence are left as they were"


@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("side", ["key", "value"])
@pytest.mark.parametrize("news", [[70, 1], [3, 1]])
def test_blocks_that_are_no_numbers(fmt, side, news):
    """A row that sees such a block's key is NaN as a whole, one that sees its value in the block's channels; others and
    rows in front of it do not notice."""
    lens = [90, 200]
    c = ref.Case(16, lens, news, 4, 2, 16, True)
    q = qr.take_over(c, fmt, 4)
    clean, clean_lse = attend(c, q)
    where = [(0, 1, 88), (1, 0, 100)]  # (sequence, head, token); token 88 is a new one where there are 70 or 3
    for b, g, t in where:
        (q.k_scales if side == "key" else q.v_scales)[int(q.block_table[b, t // 4]), g, t % 4, 2] = 255
    out, lse = attend(c, q)
    bad = torch.zeros((c.rows, 4), dtype=torch.bool, device="cuda")
    for b, g, t in where:
        for i in range(news[b]):
            if lens[b] - news[b] + i >= t:
                bad[c.starts[b] + i, 2 * g:2 * g + 2] = True
    assert bad.any() and not bad.all()
    if side == "key":
        assert torch.isnan(out[bad]).all() and torch.isnan(lse[bad]).all()
        # (not to the bit: whether weights count as rounded is decided for the rows of a wavefront together)
        out[bad], lse[bad] = clean[bad], clean_lse[bad]
        ref.check_attention(c, out, lse)
    else:
        assert torch.isnan(out[bad][:, 64:96]).all()
        for ch in (slice(0, 64), slice(96, 128)):
            assert torch.equal(out[bad][:, ch], clean[bad][:, ch])
        assert torch.equal(lse, clean_lse) and torch.equal(out[~bad], clean[~bad])


def masked(seed, lens, news, kind):
    rng, gen = random.Random(seed), torch.Generator().manual_seed(seed)
    seen = []
    for b, n in enumerate(news):
        if kind == "tree":
            seen.append(qr.tree(rng, n)[1])
        elif kind == "random":  # with the future, without themselves, now and then nothing at all
            seen.append((torch.rand((n, n), generator=gen) < 0.3) & (torch.rand((n, 1), generator=gen) < 0.8))
        else:
            seen.append(torch.zeros((n, n), dtype=torch.bool) if kind == "none" else torch.ones((n, n), dtype=torch.bool))
    return seen


CACHES = [(None, 16, False), (None, 16, True), (None, 3, True), (rk.Q_E4M3, 16, True), (rk.Q_E4M3, 5, True), (rk.Q_E2M1, 16, True)]


@pytest.mark.parametrize("fmt,ps,token_major", CACHES)
@pytest.mark.parametrize("kind", ["tree", "random", "none", "all"])
@pytest.mark.parametrize("lens,news", [([1], [1]), ([40], [40]), ([300, 64, 33, 129], [33, 64, 1, 32]), ([130, 700], [70, 300]), ([5000, 9000], [12, 6]),
                                       ([300, 8, 77], [5, 3, 4]), ([90, 3000], [8, 7]), ([200, 1, 40, 33], [1, 1, 40, 1])])
def test_masks(fmt, ps, token_major, kind, lens, news):
    c = ref.Case(31, lens, news, 8, 2, ps if fmt is None else 16, token_major, pad=(2, 1))
    q = c.cache if fmt is None else qr.take_over(c, fmt, ps)
    m = qr.MaskedCase(c, masked(sum(lens), lens, news, kind))
    out, lse = attend(c, q, m.mask)
    m.check(out, lse)
    for r in [0, 1, c.rows - 1]:
        assert (out[r] == 7).all() and (lse[r] == 7).all(), "rows of no sequence are left as they were"


@pytest.mark.parametrize("fmt,ps,token_major", CACHES)
@pytest.mark.parametrize("words,n", [(1, 40), (2, 65), (3, 64)])
def test_masks_with_fewer_or_more_words(fmt, ps, token_major, words, n):
    """Rows behind the words are seen by none; words behind the rows do not count."""
    c = ref.Case(32, [200], [n], 4, 1, ps if fmt is None else 16, token_major)
    q = c.cache if fmt is None else qr.take_over(c, fmt, ps)
    seen = torch.ones((n, n), dtype=torch.bool)
    seen[:, 32 * words:] = False
    m = qr.MaskedCase(c, [seen])
    m.mask = rk.Mask(torch.full((n, words), -1, dtype=torch.int32, device="cuda"))
    m.check(*attend(c, q, m.mask))


@pytest.mark.parametrize("fmt,ps,token_major", [(None, 16, False), (None, 4, True)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_unseen_tokens_may_be_anything(fmt, ps, token_major, bad):
    """A token that a mask hides does not reach the row, whatever its key and value hold; those that see it carry it."""
    c = ref.Case(33, [300, 90], [40, 20], 4, 2, ps, token_major, shuffled=False)
    seen = masked(7, [300, 90], [40, 20], "tree")
    node = 9
    m = qr.MaskedCase(c, seen)
    clean, clean_lse = attend(c, c.cache, m.mask)
    t = 260 + node
    page, slot = t // ps, t % ps
    for what in ("value", "key"):
        if what == "value":
            (c.cache.v_pool[page, 1, slot] if token_major else c.cache.v_pool[page, 1, :, slot])[5] = bad
        else:
            c.cache.k_pool[page, 1, slot, 3] = float("nan")
        out, lse = attend(c, c.cache, m.mask)
        hit = torch.zeros((c.rows, 4), dtype=torch.bool, device="cuda")
        hit[c.rows_of(0), 2:] = seen[0][:, node, None].cuda()
        assert hit.any() and not hit[c.rows_of(0), 2:].all()
        if what == "value":
            assert not torch.isfinite(out[hit][:, 5]).any() and torch.equal(lse, clean_lse)
            assert torch.equal(out[~hit], clean[~hit])
        else:
            assert torch.isnan(out[hit]).all() and torch.isnan(lse[hit]).all()
            out[hit], lse[hit] = clean[hit], clean_lse[hit]
            m.check(out, lse)


@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("hq,hkv", [(4, 2), (16, 1)])
@pytest.mark.parametrize("kind", ["causal", "tree", "random", "none"])
@pytest.mark.parametrize("lens,news,room", [([300, 90], [1, 1], 0), ([300, 90], [3, 2], 0), ([300, 90], [9, 6], 0), ([300, 90], [40, 20], 0),
                                            ([300, 200], [150, 90], 0), ([300, 200], [150, 90], 500)])
def test_unseen_codes_may_be_anything(fmt, hq, hkv, kind, lens, news, room):
    """The same of quantised blocks that stand for NaN, of tiles of a single token as well."""
    c = ref.Case(34, lens, news, hq, hkv, 16, True)
    q = qr.take_over(c, fmt, 4, spare=room)
    seen = [torch.tril(torch.ones((n, n), dtype=torch.bool)) for n in news] if kind == "causal" else masked(8, lens, news, kind)
    m = qr.MaskedCase(c, seen)
    mask = None if kind == "causal" else m.mask
    clean, clean_lse = attend(c, q, mask)
    node, g = news[0] // 2, hkv - 1
    t = lens[0] - news[0] + node
    hit = torch.zeros((c.rows, hq), dtype=torch.bool, device="cuda")
    hit[c.rows_of(0), hq // hkv * g:] = seen[0][:, node, None].cuda()
    for scales in (q.v_scales, q.k_scales):
        scales[int(q.block_table[0, t // 4]), g, t % 4, 2] = 255
        out, lse = attend(c, q, mask)
        if scales is q.v_scales:
            assert torch.isnan(out[hit][:, 64:96]).all() and torch.equal(lse, clean_lse)
            assert torch.equal(out[~hit], clean[~hit])
        else:
            assert torch.isnan(out[hit]).all() and torch.isnan(lse[hit]).all()
            out[hit], lse[hit] = clean[hit], clean_lse[hit]
            m.check(out, lse)


@pytest.mark.parametrize("news", [[1], [5, 0, 33], [64, 65, 31, 200], [700], [5000, 3]])
@pytest.mark.parametrize("late", [0.1, 0.7, 3.0])
def test_tree_mask(news, late):
    rng = random.Random(len(news))
    rows = 2 + sum(news) + 4
    starts = [2 + sum(news[:b]) for b in range(len(news) + 1)]
    parents = torch.full((rows,), 5, dtype=torch.int32)
    words = max(1, (max(news) + 31) // 32) + 1
    bits = torch.full((rows, words), 77, dtype=torch.int32)
    positions, base = torch.full((rows,), 77, dtype=torch.int32), torch.arange(len(news), dtype=torch.int32) * 1000 + 10
    want_bits, want_pos = bits.clone(), positions.clone()
    for b, n in enumerate(news):
        p, seen = qr.tree(rng, n, late) if n <= 700 else ([i - 1 if i % 50 else -1 for i in range(n)], None)
        if seen is None:  # chains of 50
            i = torch.arange(n)
            seen = (i[:, None] // 50 == i[None, :] // 50) & (i[None, :] <= i[:, None])
        at = slice(starts[b], starts[b] + n)
        bad = [i + 3 if i % 4 == 1 and x < 0 else x for i, x in enumerate(p)]  # a parent that cannot be one counts as none
        parents[at] = torch.tensor(bad, dtype=torch.int32)
        wide = torch.zeros((n, words * 32), dtype=torch.int64)
        wide[:, :n] = seen
        w = (wide.reshape(n, words, 32) << torch.arange(32)).sum(-1)
        want_bits[at] = torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)
        want_pos[at] = base[b] + seen.sum(1).to(torch.int32) - 1
    chunk = rk.Chunk(torch.tensor(starts, dtype=torch.int32).cuda(), rows)
    mask, pos = rk.Mask(bits.cuda()), positions.cuda()
    rk.tree_mask(chunk, parents.cuda(), mask, base.cuda(), pos)
    assert torch.equal(mask.bits.cpu(), want_bits) and torch.equal(pos.cpu(), want_pos)
    few = rk.Mask(torch.zeros((rows, 1), dtype=torch.int32, device="cuda"))
    rk.tree_mask(chunk, parents.cuda(), few)
    for b, n in enumerate(news):
        at = slice(starts[b], starts[b] + n)
        assert torch.equal(few.bits[at, 0].cpu(), want_bits[at, 0])


def listed(c, q, pages, out_lse=True):
    out = torch.full((len(c.lens), c.hq, ref.D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((len(c.lens), c.hq), 7.0, device="cuda") if out_lse else None
    ws = rk.q_alloc_workspace(rk.OP_ATTEND, q, 0 if pages is None else pages.shape[-1])
    rk.q_attend(q, c.q, pages, out, lse, ws)
    return out, lse


def check_listed(c, q, pages, out, lse):
    """Against the definition: a Case whose sequences are the listed tokens of one (sequence, KV head)."""
    G = c.hq // c.hkv
    for b, n in enumerate(c.lens):
        for g in range(c.hkv):
            t = []
            for p in (pages[b, g].tolist() if pages is not None else range(q.pages_cap)):
                if 0 <= p < q.pages_cap and 0 <= int(q.block_table[b, p]) < q.k_codes.shape[0]:
                    t += [x for x in range(p * q.page_size, (p + 1) * q.page_size) if x < n]
            one = ref.Case(0, [max(len(t), 1)], [1], G, 1, 16, True)
            one.lens = [len(t)]
            one.K, one.V = c.K[b:b + 1, g:g + 1, t], c.V[b:b + 1, g:g + 1, t]
            one.q = c.q[b:b + 1, g * G:(g + 1) * G]
            ref.check_attention(one, out[b:b + 1, g * G:(g + 1) * G], lse[b:b + 1, g * G:(g + 1) * G], f"{b} {g}")


@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("ps", [1, 4, 7, 16, 64])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (16, 1), (3, 3)])
def test_listed_pages(fmt, ps, hq, hkv):
    lens = [900, 1, 64, 0, 333]
    c = ref.Case(41, lens, [1 if n else 0 for n in lens], hq, hkv, 16, True)
    c.q = torch.randn((5, hq, 128), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    q = qr.take_over(c, fmt, ps)
    q.block_table[0, 1] = -1
    rng = random.Random(ps)
    row = 40
    pages = torch.full((5, hkv, row), -1, dtype=torch.int32)
    for b, n in enumerate(lens):
        P = (n + ps - 1) // ps
        for g in range(hkv):
            some = [rng.randrange(P) for _ in range(min(P, 17))] if P else []   # in any order, some of them twice
            some += [P, q.pages_cap, 1 << 30, -5]                               # behind the sequence, behind the table
            rng.shuffle(some)
            pages[b, g, 3:3 + len(some)] = torch.tensor(some, dtype=torch.int32)
    pages = pages.cuda()
    out, lse = listed(c, q, pages)
    check_listed(c, q, pages, out, lse)
    assert (out[3] == 0).all() and torch.isneginf(lse[3]).all()
    again, _ = listed(c, q, pages, False)
    assert torch.equal(out, again)
    out, lse = listed(c, q, None)
    check_listed(c, q, None, out, lse)


@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("row", [1, 64, 700])
def test_long_lists(fmt, row):
    """Lists that are cut into parts."""
    c = ref.Case(42, [20000, 12000], [1, 1], 4, 1, 16, True)
    c.q = torch.randn((2, 4, 128), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    q = qr.take_over(c, fmt, 16)
    gen = torch.Generator().manual_seed(3)
    pages = torch.stack([torch.randperm(750, generator=gen)[:row].sort().values for _ in range(2)])[:, None].to(torch.int32).cuda()
    check_listed(c, q, pages, *listed(c, q, pages))


@pytest.mark.parametrize("fmt", qr.FORMATS)
@pytest.mark.parametrize("ps,channels,budget", [(16, 16, 256), (4, 60, 200), (16, 128, 100000)])
def test_hsa_decode(fmt, ps, channels, budget):
    """The selection by the summaries of what the cache holds, and attention over what it selects."""
    lens = [3000, 900, 20]
    c = ref.Case(43, lens, [1, 1, 1], 8, 2, 16, True)
    q = qr.take_over(c, fmt, ps)
    back = rk.alloc_cache(3, 8, 2, 128, ps, q.pages_cap, "cuda", block_table=q.block_table, n_phys_pages=q.k_codes.shape[0],
                          v_layout=rk.V_TOKEN_MAJOR)
    rk.restore(q, back)
    kmax, kmin = rk.alloc_summaries(back)
    rk.build_page_summaries(back, kmax, kmin)
    row = rk.pages_row_len(back, budget)
    pages, want = (torch.full((3, 2, row), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    chan, want_chan = (torch.full((3, 2, channels), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    out, lse = torch.empty((3, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((3, 8), device="cuda")
    ws = rk.q_alloc_workspace(rk.OP_HSA_DECODE, q, budget)
    rk.q_hsa_decode(q, c.q, kmax, kmin, channels, budget, 1, out, lse, pages, chan, ws)
    rk.hsa_select(back, c.q, kmax, kmin, channels, budget, 1, want, want_chan)
    assert torch.equal(pages, want) and torch.equal(chan, want_chan)
    check_listed(c, q, want, out, lse)


@pytest.mark.parametrize("fmt", [None] + qr.FORMATS)
def test_a_tree_verified_step_by_step(fmt):
    """Drafts as they are used, captured in a graph: positions and mask from the parents, append, attention, the accepted path
    kept; then the next token over the cache.  Three rounds, replayed with new drafts, beside the same calls without a graph."""
    B, hq, hkv, n, ps = 2, 8, 2, 24, 16
    rng, gen = random.Random(5), torch.Generator().manual_seed(5)
    lens = [77, 300]
    rope = rk.rope_frequencies(128, 10000.0, device="cuda")
    static = dict(q=torch.zeros((B * n, hq, 128)), k=torch.zeros((B * n, hkv, 128)), v=torch.zeros((B * n, hkv, 128)))
    static = {k: v.to(torch.bfloat16).cuda() for k, v in static.items()}
    parents = torch.zeros((B * n,), dtype=torch.int32, device="cuda")
    keep = torch.zeros((B * n,), dtype=torch.bool, device="cuda")
    chunk = rk.Chunk(torch.tensor([0, n, 2 * n], dtype=torch.int32).cuda(), B * n)

    def state():
        c = ref.Case(51, lens, [0, 0], hq, hkv, ps, True, spare_pages=8)
        cache = c.cache if fmt is None else qr.like(c.cache, fmt, ps)
        if fmt is not None:
            rk.quantise(c.cache, cache)
        alloc = rk.alloc_workspace if fmt is None else rk.q_alloc_workspace
        s = dict(cache=cache, mask=rk.alloc_mask(B * n, n, "cuda"), pos=torch.zeros((B * n,), dtype=torch.int32, device="cuda"),
                 out=torch.zeros((B * n, hq, 128), dtype=torch.bfloat16, device="cuda"), lse=torch.zeros((B * n, hq), device="cuda"),
                 q=torch.zeros((B * n, hq, 128), dtype=torch.bfloat16, device="cuda"),
                 ws=alloc(rk.OP_CHUNK_ATTEND, cache, B * n))
        s["kmax"], s["kmin"] = (torch.zeros((B, hkv, 128, cache.pages_cap), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        s["wsa"] = alloc(rk.OP_APPEND_CHUNK, cache, B * n)
        return s

    def step(s):
        rk.tree_mask(chunk, parents, s["mask"], s["cache"].seq_lens, s["pos"])
        a = (rk.append_chunk if fmt is None else rk.q_append_chunk)
        a(s["cache"], chunk, static["k"], static["v"], s["kmax"], s["kmin"], s["wsa"], rope=rope, positions=s["pos"], q=static["q"], q_out=s["q"])
        if fmt is None:
            rk.masked_attend(s["cache"], chunk, s["mask"], s["q"], s["out"], s["lse"], s["ws"])
            rk.keep_tokens(s["cache"], chunk, keep, s["kmax"], s["kmin"], s["wsa"])
        else:
            rk.q_chunk_attend(s["cache"], chunk, s["q"], s["out"], s["lse"], s["ws"], mask=s["mask"])
            rk.q_keep_tokens(s["cache"], chunk, keep, s["kmax"], s["kmin"], s["wsa"])

    def everything(s):
        pools = (s["cache"].k_pool, s["cache"].v_pool) if fmt is None else (s["cache"].k_codes, s["cache"].v_codes, s["cache"].k_scales, s["cache"].v_scales)
        return (s["out"], s["lse"], s["pos"], s["mask"].bits, s["cache"].seq_lens) + pools

    warm = state()
    step(warm)
    eager, captured, alone = state(), state(), state()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured)
    total = list(lens)
    for _ in range(3):
        for x in static.values():
            x.copy_(torch.randn(x.shape, generator=gen))
        flags = torch.zeros((B, n), dtype=torch.bool)
        for b in range(B):
            p, seen = qr.tree(rng, n)
            parents[b * n:(b + 1) * n] = torch.tensor(p, dtype=torch.int32)
            leaf = rng.randrange(n)
            flags[b] = seen[leaf]  # the path to some node
            total[b] += int(seen[leaf].sum())
        keep.copy_(flags.flatten())
        graph.replay()
        step(eager)
        torch.cuda.synchronize()
        assert captured["cache"].seq_lens.tolist() == total
        for x, y in zip(everything(captured), everything(eager)):
            assert torch.equal(x, y)
        # the paths' tokens stand behind each other, at the positions they were turned for: as if they alone had been appended
        rows = [r for r in range(B * n) if flags.flatten()[r]]
        few = rk.Chunk(torch.tensor([0, int(flags[0].sum()), len(rows)], dtype=torch.int32).cuda(), len(rows))
        (rk.append_chunk if fmt is None else rk.q_append_chunk)(alone["cache"], few, static["k"][rows], static["v"][rows], alone["kmax"],
                                                                 alone["kmin"], alone["wsa"], rope=rope)
        for b in range(B):
            if fmt is None:
                got, want = ([x[b, :, :total[b]] for x in rk.unpack_cache(s["cache"])] for s in (eager, alone))
                assert all(torch.equal(x, y) for x, y in zip(got, want))
            else:
                assert all((x == y).all() for x, y in zip(qr.tokens(eager["cache"], b, total[b]), qr.tokens(alone["cache"], b, total[b])))
            at = slice(lens[b] // ps + 1, (total[b] + ps - 1) // ps)  # (the pages before hold older keys, whose summaries nobody made)
            assert torch.equal(eager["kmax"][b, :, :, at], alone["kmax"][b, :, :, at])
    assert torch.isfinite(eager["lse"]).all()


@pytest.mark.parametrize("fmt", qr.FORMATS)
def test_two_graphs_one_workspace_and_another_stream(fmt):
    """Two captured calls that take turns with one workspace, and a stream of the caller's."""
    cases = [ref.Case(61, [9000, 100], [3, 1], 4, 1, 16, True), ref.Case(62, [700], [300], 4, 1, 16, True)]
    qs = [qr.take_over(c, fmt) for c in cases]
    ws = rk.q_alloc_workspace(rk.OP_CHUNK_ATTEND, qs[0], 300)
    outs = [(torch.zeros((c.rows, c.hq, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((c.rows, c.hq), device="cuda")) for c in cases]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    for c, q, (out, lse) in zip(cases, qs, outs):
        rk.q_chunk_attend(q, c.chunk, c.q, out, lse, ws, stream=side)
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            rk.q_chunk_attend(q, c.chunk, c.q, out, lse, ws)
        graphs.append(g)
    want = [(o.clone(), l.clone()) for o, l in outs]
    for i in (0, 1, 0, 0, 1, 1, 0):
        outs[i][0].zero_(), outs[i][1].zero_()
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i][0], want[i][0]) and torch.equal(outs[i][1], want[i][1])
    for c, (out, lse) in zip(cases, outs):
        ref.check_attention(c, out, lse)


@pytest.mark.parametrize("fmt", qr.FORMATS)
def test_more_heads_than_workgroups_fill(fmt):
    """300 KV heads: no tile is cut."""
    for news in ([1, 1, 1], [2, 1, 9]):
        c = ref.Case(63, [1500, 40, 700], news, 300, 300, 16, True)
        ref.check_attention(c, *attend(c, qr.take_over(c, fmt)))


@pytest.mark.parametrize("fmt", qr.FORMATS)
def test_calls_at_once(fmt):
    """Calls on two streams, each with a workspace of its own, whose parts are joined by workgroups of the same call."""
    cases = [ref.Case(64, [9000, 6000], [3, 1], 4, 2, 16, True), ref.Case(65, [20000], [1], 4, 2, 16, True)]
    qs = [qr.take_over(c, fmt) for c in cases]
    want = [attend(c, q) for c, q in zip(cases, qs)]
    spaces = [rk.q_alloc_workspace(rk.OP_CHUNK_ATTEND, q, c.rows) for c, q in zip(cases, qs)]
    outs = [[(torch.zeros_like(o), torch.zeros_like(l)) for _ in range(20)] for o, l in want]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for i in range(20):
        for c, q, ws, out, st in zip(cases, qs, spaces, outs, streams):
            rk.q_chunk_attend(q, c.chunk, c.q, out[i][0], out[i][1], ws, stream=st)
    torch.cuda.synchronize()
    for (o, l), out in zip(want, outs):
        for got, got_lse in out:
            assert torch.equal(got, o) and torch.equal(got_lse, l)


def far_cache(c, fmt, ps=64):
    """The Case's tokens in a quantised cache whose rows lie beyond 4 GiB of codes, pages and heads at strides of their own."""
    per = (max(c.lens) + 40) // ps + 2
    per = (per + 7) // 8 * 8
    width = rk.q_row_bytes(fmt)
    n_phys = (5 << 30) // (c.hkv + 1) // ps // width
    mk = lambda w: torch.empty((n_phys, c.hkv + 1, ps, w), dtype=torch.uint8, device="cuda")[:, 1:]
    table = (n_phys - 1 - torch.arange(len(c.lens) * per)).reshape(len(c.lens), per).to(torch.int32).cuda()
    return rk.QCache(len(c.lens), c.hq, c.hkv, 128, ps, per, mk(width), mk(width), mk(4), mk(4),
                     torch.zeros((len(c.lens),), dtype=torch.int32, device="cuda"), table, fmt)


@pytest.mark.parametrize("fmt", qr.FORMATS)
def test_codes_beyond_4_gib(fmt):
    """Offsets that take more than 32 bits: conversion there and back, append, attention of few and many rows, keeping."""
    lens = [500, 300]
    c = ref.Case(71, lens, [1, 2], 8, 2, 16, True)
    q = far_cache(c, fmt)
    rk.quantise(c.cache, q)
    near = qr.take_over(c, fmt)
    back = rk.alloc_cache(2, 8, 2, 128, 16, 40, "cuda", v_layout=rk.V_TOKEN_MAJOR)
    rk.restore(q, back)
    k, v = rk.unpack_cache(back)
    for b, n in enumerate(lens):
        assert torch.equal(k[b, :, :n], c.K[b, :, :n]) and torch.equal(v[b, :, :n], c.V[b, :, :n])
        for got, want in zip(qr.tokens(q, b, n), qr.tokens(near, b, n)):
            assert (got == want).all()
    ref.check_attention(c, *attend(c, q))
    new = torch.randn((40, 2, 128), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    chunk = rk.Chunk(torch.tensor([0, 30, 40], dtype=torch.int32).cuda(), 40)
    ws = rk.q_alloc_workspace(rk.OP_APPEND_CHUNK, q, 40)
    for cache in (q, near):
        if cache is near:
            near = cache = qr.like(c.cache, fmt, 16, spare=8)
            rk.quantise(c.cache, cache)
        rk.q_append_chunk(cache, chunk, new, new, None, None, ws)
    qs = torch.randn((40, 8, 128), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    outs = []
    for cache in (q, near):
        out, lse = torch.empty_like(qs), torch.empty((40, 8), device="cuda")
        rk.q_chunk_attend(cache, chunk, qs, out, lse, rk.q_alloc_workspace(rk.OP_CHUNK_ATTEND, cache, 40))
        keep = (torch.arange(40) % 3 == 0).cuda()
        rk.q_keep_tokens(cache, chunk, keep, None, None, ws)
        outs.append((out, lse, cache.seq_lens.clone()) + tuple(torch.from_numpy(x) for b, n in enumerate((510, 304)) for x in qr.tokens(cache, b, n)))
    for x, y in zip(*outs):
        assert torch.equal(x, y)


def test_masked_beyond_4_gib():
    """The form for pools whose rows take more than 32 bits of offset, with a mask."""
    lens, news = [700, 90], [40, 12]
    c = ref.Case(72, lens, news, 8, 2, 16, True, shuffled=False)
    per, n_phys = c.cache.pages_cap, (5 << 30) // (2 * 16 * 256)
    pools = [torch.empty((n_phys, 2, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for pool, old in zip(pools, (c.cache.k_pool, c.cache.v_pool)):
        pool[-2 * per:] = old[:2 * per]
    table = (n_phys - 2 * per + torch.arange(2 * per)).reshape(2, per).to(torch.int32).cuda()
    far = rk.Cache(2, 8, 2, 128, 16, per, pools[0], pools[1], c.cache.seq_lens, table, rk.V_TOKEN_MAJOR)
    m = qr.MaskedCase(c, masked(5, lens, news, "tree"))
    m.check(*attend(c, far, m.mask))
