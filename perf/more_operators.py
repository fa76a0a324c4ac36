"""Operators of caches held in 8 or 4 bits, and of trees of drafted tokens, as measurable cases.

    append   new tokens of several sequences rotated, quantised and put into their pages, with the pages' summaries
             (``q_append_chunk``); with ``read``, the whole cache read back into bf16 behind it (``restore``)
    convert  a whole bf16 cache quantised (``quantise``), or a quantised one read back (``restore``)
    attend   causal attention of the new tokens over the quantised cache (``q_chunk_attend``)
    pages    attention of one token per sequence over a list of pages of the quantised cache (``q_attend``)
    tree     which drafted tokens see each other, from their parents (``tree_mask``), and attention by that over a
             bf16 cache (``masked_attend``) or a quantised one (``q_chunk_attend``)
    keep     the accepted ones among the drafted tokens moved together, the others dropped (``keep_tokens``, ``q_keep_tokens``)

A quantised cache holds a token's key and value in blocks of 32 channels: codes of 8 bits (``e4m3``) or 4 (``e2m1``), and a
power of two for each block, the smallest with which no value of the block exceeds the largest code.

``run`` computes the plain form of each in torch, or, where ``own`` is true, calls the library.  Sequences hold
unequal numbers of tokens where a case says ``ragged``; their pages are scattered over the pool where it says ``paged``.
"""
import math

import torch

own = False

D = 128
BLOCK = 32
SCALE = 1.0 / math.sqrt(D)
THETA = 500000.0

#: mantissa bits, lowest exponent, largest value, and the range of block exponents whose values are normal in bf16
FORMATS = {"e4m3": (3, -6, 448.0, -100, 119), "e2m1": (1, 0, 6.0, -100, 125)}


def _append(name, batch, hq, hkv, old, new, fmt, *, ps=16, ragged=False, paged=False, rot=D, interleaved=False, read=False):
    """``old``: tokens a sequence holds, ``new``: tokens it receives (the longest one's if ``ragged``); ``rot``: channels
    rotated, 0 where queries and keys come rotated and only keys and values are put away."""
    return dict(name=name, kind="append", batch=batch, hq=hq, hkv=hkv, old=old, new=new, fmt=fmt, ps=ps, ragged=ragged,
                paged=paged, rot=rot, interleaved=interleaved, read=read)


def _convert(name, batch, hkv, old, fmt, back, *, ps=16, other_ps=16, token_major=False, ragged=False, paged=False):
    """``back``: from the quantised cache of pages of ``ps`` tokens to the bf16 one of ``other_ps``; else the other way."""
    return dict(name=name, kind="convert", batch=batch, hq=hkv, hkv=hkv, old=old, new=0, fmt=fmt, back=back, ps=ps,
                other_ps=other_ps, token_major=token_major, ragged=ragged, paged=paged)


def _attend(name, batch, hq, hkv, old, new, fmt, *, ps=16, ragged=False, paged=False):
    return dict(name=name, kind="attend", batch=batch, hq=hq, hkv=hkv, old=old, new=new, fmt=fmt, ps=ps, ragged=ragged,
                paged=paged)


def _pages(name, batch, hq, hkv, old, listed_pages, fmt, *, ps=16, ragged=False, paged=False):
    return dict(name=name, kind="pages", batch=batch, hq=hq, hkv=hkv, old=old, new=0, listed_pages=listed_pages, fmt=fmt,
                ps=ps, ragged=ragged, paged=paged)


def _tree(name, batch, hq, hkv, old, new, fmt, *, ps=16, token_major=False, ragged=False, paged=False):
    """``fmt`` None: a bf16 cache."""
    return dict(name=name, kind="tree", batch=batch, hq=hq, hkv=hkv, old=old, new=new, fmt=fmt, ps=ps,
                token_major=token_major, ragged=ragged, paged=paged)


def _keep(name, batch, hq, hkv, old, new, kept, fmt, *, ps=16, token_major=False, ragged=False, paged=False):
    return dict(name=name, kind="keep", batch=batch, hq=hq, hkv=hkv, old=old, new=new, kept=kept, fmt=fmt, ps=ps,
                token_major=token_major, ragged=ragged, paged=paged)


def listed():
    return [
        # one decode step of the serving batch: a token of every sequence put away
        _append("append_step", 16, 32, 8, 4121, 1, "e4m3"),
        # a prompt of the 32768-token context in 4 bits, and the cache read back for an operator that takes bf16
        _append("append_prompt", 1, 32, 8, 0, 32768, "e2m1", rot=0, read=True),
        # the serving batch's compressed caches brought to 8 bits, once per prompt
        _convert("quantise_batch", 16, 8, 4096, "e4m3", False),
        # a long conversation read back for the next turn's filter
        _convert("restore_turns", 1, 8, 131072, "e4m3", True, ps=4, other_ps=4, token_major=True),
        # one decode step of the serving batch over every token of the compressed caches
        _attend("attend_step", 16, 32, 8, 4121, 1, "e4m3"),
        # one chunk of a prompt fed in chunks
        _attend("attend_chunk", 1, 32, 8, 32768, 2048, "e2m1"),
        # one decode step over the 1024 tokens selected of uncompressed caches
        _pages("pages_batch", 16, 32, 8, 32768, 64, "e4m3", paged=True),
        # the same of one long conversation, at the small pages of the decomposed operating point
        _pages("pages_turns", 1, 32, 8, 131072, 512, "e2m1", ps=4),
        # drafted trees of a serving batch of unequal contexts
        _tree("tree_batch", 16, 32, 8, 32768, 32, None, ragged=True, paged=True),
        # a wide tree behind a long conversation
        _tree("tree_turns", 1, 32, 8, 131072, 200, "e4m3", ps=4),
        # what the batch's drafts came to: five of 32 accepted
        _keep("keep_batch", 16, 32, 8, 4096, 32, 5, None),
        # the wide tree's, over small pages
        _keep("keep_turns", 1, 32, 8, 131072, 200, 9, "e4m3", ps=4),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "convert", "attend", "attend", "pages", "tree", "tree", "keep"])
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.choice([1, 3, 4, 5, 8])
    fmt = rng.choice(["e4m3", "e2m1"])
    ps = rng.choice([1, 2, 3, 4, 5, 8, 16, 16, 16, 32, 64])
    ragged, paged = rng.random() < 0.6, rng.random() < 0.5
    batch = _log(rng, 1, 16)
    if kind == "append":
        new, old = _log(rng, 1, 32768 // batch), rng.choice([0, _log(rng, 1, 65536 // batch)])
        rot = rng.choice([D, 64, 2 * rng.randint(8, 64)]) if fmt == "e4m3" else 0
        return _append(None, batch, hq, hkv, old, new, fmt, ps=ps, ragged=ragged, paged=paged, rot=rot,
                       interleaved=rng.random() < 0.5, read=fmt == "e2m1")
    if kind == "convert":
        token_major = rng.random() < 0.5
        other = rng.choice([1, 4, 7, 16, 64]) if token_major else 16
        back = fmt == "e2m1" or rng.random() < 0.5
        return _convert(None, batch, hkv, _log(rng, 16, 131072 // batch), fmt, back, ps=ps, other_ps=other,
                        token_major=token_major, ragged=ragged, paged=paged)
    if kind == "pages":
        old = _log(rng, 64, 131072 // batch)
        return _pages(None, batch, hq, hkv, old, _log(rng, 1, max(1, min(4096, old) // ps)), fmt, ps=ps, ragged=ragged, paged=paged)
    old = rng.choice([0, _log(rng, 1, 65536 // batch)])
    if kind == "attend":
        new = rng.choice([1, _log(rng, 1, 16), _log(rng, 1, 2048)])
        # pairs of a query and a key: at most those of a 2048-token chunk over 32768 tokens
        while batch * hq * new * (old + new) > 32 * 2048 * 34816:
            new = max(1, new // 2)
        return _attend(None, batch, hq, hkv, old, new, fmt, ps=ps, ragged=ragged, paged=paged)
    held = rng.choice([None, fmt])
    token_major = rng.random() < 0.5 if held is None else True
    if not token_major:
        ps = 16
    new = _log(rng, 2, 300)
    if kind == "tree":
        return _tree(None, batch, hq, hkv, old, new, held, ps=ps, token_major=token_major, ragged=ragged, paged=paged)
    return _keep(None, batch, hq, hkv, old, new, rng.randint(1, max(1, min(12, new // 2))), "e4m3" if held else None, ps=ps,
                 token_major=token_major, ragged=ragged, paged=paged)


# ---- inputs -----------------------------------------------------------------------------------------------------------

def _lengths(case):
    """Old and new tokens of every sequence, the same for every seed: with them the work of a case is fixed."""
    B, old, new = case["batch"], case["old"], case["new"]
    if not case["ragged"]:
        return [old] * B, [new] * B
    share = [1.0 if B == 1 else (b * 5 % B + 1) / B for b in range(B)]  # the longest among shorter ones
    olds = [int(round(old * s)) for s in share]
    news = [max(1 if new else 0, int(round(new * share[(b + 1) % B]))) for b in range(B)]
    if case["kind"] in ("append", "attend") and B > 2:
        for b in range(0, B, 3):
            news[b] = 1  # sequences that decode beside those that prefill
    return olds, news


def _frequencies(rot):
    """Angles per position in 64 bits: the low frequencies stretched for contexts eight times the original 8192."""
    f = 1.0 / THETA ** (torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    turns = 8192.0 * f / (2.0 * math.pi)  # over the original context
    mix = ((turns - 1.0) / 3.0).clamp(0.0, 1.0)
    return f / 8.0 * (1.0 - mix) + f * mix


def _bf16(gen, scales, n):
    """Rows of heads whose channels have unequal scales, as keys have after training."""
    x = torch.randn((n,) + tuple(scales.shape), generator=gen, device="cuda")
    return (x * scales).to(torch.bfloat16)


class _Pool:
    """A paged cache in torch tensors.  bf16: keys and values of pages of ``ps`` tokens, values by channel or by token;
    quantised (``fmt``): codes and block exponents of both by token."""

    def __init__(self, gen, case, lens, capacity, fmt, ps, token_major):
        B, H = case["batch"], case["hkv"]
        self.batch, self.hq, self.hkv, self.ps, self.fmt, self.tm = B, case["hq"], H, ps, fmt, token_major
        self.cap = ((max(capacity, 1) + ps - 1) // ps + 7) // 8 * 8
        self.n_phys = B * self.cap + (17 if case["paged"] else 0)
        self.table = None
        if case["paged"]:
            self.table = torch.randperm(self.n_phys, generator=gen, device="cuda")[:B * self.cap].reshape(B, self.cap).to(torch.int32)
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        zeros = lambda *shape, dtype: torch.zeros((self.n_phys, H) + shape, dtype=dtype, device="cuda")
        if fmt is None:
            self.k = zeros(ps, D, dtype=torch.bfloat16)
            self.v = zeros(*((ps, D) if token_major else (D, ps)), dtype=torch.bfloat16)
        else:
            width = D if fmt == "e4m3" else D // 2
            self.k, self.v = (zeros(ps, width, dtype=torch.uint8) for _ in range(2))
            self.ks, self.vs = (zeros(ps, D // BLOCK, dtype=torch.uint8) for _ in range(2))

    def fill(self, gen, scales):
        """Keys whose channels have unequal scales, standard normal values."""
        for first in range(0, self.n_phys, 4096):
            n = min(4096, self.n_phys - first)
            at = slice(first, first + n)
            k = torch.randn((n, self.hkv, self.ps, D), generator=gen, device="cuda").mul_(scales[None, :, None, :])
            v = torch.randn((n, self.hkv, self.ps, D), generator=gen, device="cuda")
            if self.fmt is None:
                self.k[at], self.v[at] = k, v if self.tm else v.transpose(2, 3)
            else:
                (self.k[at], self.ks[at]), (self.v[at], self.vs[at]) = _quantised(k, self.fmt), _quantised(v, self.fmt)

    def page(self, b, t):
        """Physical pages of tokens t of sequences b."""
        return b * self.cap + t // self.ps if self.table is None else self.table[b, t // self.ps].long()

    def rows(self, b, t, dtype=torch.float32):
        """Keys and values of tokens t of sequences b: [...][heads][D]."""
        pp, slot = self.page(b, t), t % self.ps
        if self.fmt is None:
            return self.k[pp, :, slot].to(dtype), (self.v[pp, :, slot] if self.tm else self.v[pp, :, :, slot]).to(dtype)
        return (_values(self.k[pp, :, slot], self.ks[pp, :, slot], self.fmt).to(dtype),
                _values(self.v[pp, :, slot], self.vs[pp, :, slot], self.fmt).to(dtype))

    def outputs(self):
        if self.fmt is None:
            return {"k": self.k, "v": self.v}
        # (codes of 8 bits are numbers of torch's, and so are the blocks' powers of two)
        out = {"k_scales": self.ks.view(torch.float8_e8m0fnu), "v_scales": self.vs.view(torch.float8_e8m0fnu)}
        return dict(out, k=self.k.view(torch.float8_e4m3fn), v=self.v.view(torch.float8_e4m3fn))

    def handle(self):
        from paper_2502_14051_amd import rocketkv as rk

        if self.fmt is None:
            return rk.Cache(self.batch, self.hq, self.hkv, D, self.ps, self.cap, self.k, self.v, self.lens, self.table,
                            rk.V_TOKEN_MAJOR if self.tm else rk.V_CHANNEL_MAJOR)
        return rk.QCache(self.batch, self.hq, self.hkv, D, self.ps, self.cap, self.k, self.v, self.ks, self.vs, self.lens,
                         self.table, rk.Q_E4M3 if self.fmt == "e4m3" else rk.Q_E2M1)


def _queries(gen, tokens, case, scales):
    """The heads of a group share a part of their query and look along the channels that carry their keys."""
    H, G = case["hkv"], case["hq"] // case["hkv"]
    x = 0.6 * torch.randn((tokens, H, 1, D), generator=gen, device="cuda")
    x = x + 0.8 * torch.randn((tokens, H, G, D), generator=gen, device="cuda")
    return (x * scales[None, :, None, :]).reshape(tokens, H * G, D).to(torch.bfloat16)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    olds, news = _lengths(case)
    B, hq, hkv, kind, fmt = case["batch"], case["hq"], case["hkv"], case["kind"], case["fmt"]
    total, most = sum(news), max(news)
    s = {"case": case, "olds": olds, "news": news}
    scales = torch.exp(0.5 * torch.randn((hkv, D), generator=gen, device="cuda"))
    longest = max(o + n for o, n in zip(olds, news))
    # which rows of the packed tensors are whose: [sequence][its tokens], and whether there is one
    tensor = lambda x: torch.tensor(x, dtype=torch.int64, device="cuda")
    starts = torch.tensor([0] + news, dtype=torch.int64).cumsum(0)
    s["old"], s["starts"] = tensor(olds), starts.to(torch.int32).cuda()
    s["there"] = torch.arange(most, device="cuda") < tensor(news)[:, None]
    s["row"] = (starts[:-1].cuda()[:, None] + torch.arange(most, device="cuda")).clamp(max=max(total - 1, 0))
    s["seq"], s["index"] = s["there"].nonzero(as_tuple=True)
    held = olds if kind in ("append", "convert", "pages") else [o + n for o, n in zip(olds, news)]
    pool = s["pool"] = _Pool(gen, case, held, longest, fmt, case["ps"], fmt is not None or case["token_major"])
    if not (kind == "convert" and not case["back"]):
        pool.fill(gen, scales)
    handles = {}
    if kind == "append":
        s["lens0"] = pool.lens.clone()
        s["k"], s["v"] = _bf16(gen, scales, total), _bf16(gen, torch.ones_like(scales), total)
        if case["rot"]:
            s["q"] = _queries(gen, total, case, scales)
            s["q_out"] = torch.empty_like(s["q"])
            s["freq"] = _frequencies(case["rot"]).cuda()
        # pages that take in a token, and the summaries of all that hold one
        s["pages"] = torch.unique(torch.stack((s["seq"], (s["old"][s["seq"]] + s["index"]) // pool.ps)), dim=1)
        s["kmax"], s["kmin"] = (torch.zeros((B, hkv, D, pool.cap), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        at = [(b, p) for b, n in enumerate(olds) for p in range((n + pool.ps - 1) // pool.ps)]
        if at:
            _summaries(pool, tensor([x[0] for x in at]), tensor([x[1] for x in at]), s["old"], s["kmax"], s["kmin"])
        if case["read"]:
            s["other"] = _Pool(gen, case, [0] * B, longest, None, case["ps"], True)
    if kind == "convert":
        s["other"] = _Pool(gen, case, [0] * B if case["back"] else olds, longest, None, case["other_ps"], case["token_major"])
        if not case["back"]:
            s["other"].fill(gen, scales)
            pool.lens.zero_()
    if kind in ("attend", "tree", "pages"):
        rows = B if kind == "pages" else total
        s["q"] = _queries(gen, rows, case, scales)
        s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty((rows, hq), device="cuda")
    if kind == "pages":
        # distinct pages in ascending order, another choice for every head, the last one among them as a selection has it
        n_pages = [(n + pool.ps - 1) // pool.ps for n in olds]
        s["pages"] = torch.full((B, hkv, case["listed_pages"]), -1, dtype=torch.int32, device="cuda")
        for b, n in enumerate(n_pages):
            m = min(n, case["listed_pages"])
            r = torch.rand((hkv, n), generator=gen, device="cuda")
            r[:, -1] = 2.0
            s["pages"][b, :, :m] = r.topk(m, 1).indices.sort(1).values.to(torch.int32)
    if kind == "tree":
        # the root, and every other node a child of some earlier one, more often of a late one
        u = torch.rand((total,), generator=gen, device="cuda").sqrt()
        i = torch.empty((total,), dtype=torch.int64, device="cuda")
        i[s["row"][s["there"]]] = s["index"]
        s["parents"] = torch.where(i > 0, (u * i).long().clamp(max=i - 1), -1).to(torch.int32)
        s["bits"] = torch.zeros((total, (most + 31) // 32), dtype=torch.int32, device="cuda")
        s["positions"] = torch.zeros((total,), dtype=torch.int32, device="cuda")
        s["base"] = s["old"].to(torch.int32)
    if kind == "keep":
        # the root and nodes behind it, such that no accepted one stands where another goes: a pass taken again on the
        # same caches finds the same tokens
        s["lens0"] = pool.lens.clone()
        s["keep"] = torch.zeros((total,), dtype=torch.uint8, device="cuda")
        for b, n in enumerate(news):
            m = max(1, min(case["kept"], n // 2))
            late = m + torch.randperm(max(n - m, 0), generator=gen, device="cuda")[:m - 1]
            s["keep"][int(starts[b])] = 1
            s["keep"][int(starts[b]) + late] = 1
        s["kmax"], s["kmin"] = (torch.zeros((B, hkv, D, pool.cap), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        at = torch.arange(most // pool.ps + 2, device="cuda") + (s["old"] // pool.ps)[:, None]
        s["pages"] = (torch.arange(B, device="cuda")[:, None].expand_as(at)[at < pool.cap], at[at < pool.cap])
    if own:
        from paper_2502_14051_amd import rocketkv as rk

        handles["cache"] = pool.handle()
        handles["chunk"] = rk.Chunk(s["starts"], total)
        if "other" in s:
            handles["other_cache"] = s["other"].handle()
        if kind == "append":
            handles["rope"] = rk.Rope(s["freq"], case["interleaved"]) if case["rot"] else None
            handles["ws"] = rk.q_alloc_workspace(rk.OP_APPEND_CHUNK, handles["cache"], total)
        if kind == "keep":
            alloc = rk.alloc_workspace if fmt is None else rk.q_alloc_workspace
            handles["ws"] = alloc(rk.OP_APPEND_CHUNK, handles["cache"], total)
        if kind in ("attend", "tree"):
            alloc = rk.alloc_workspace if fmt is None else rk.q_alloc_workspace
            handles["ws"] = alloc(rk.OP_CHUNK_ATTEND, handles["cache"], total)
        if kind == "pages":
            handles["ws"] = rk.q_alloc_workspace(rk.OP_ATTEND, handles["cache"], case["listed_pages"])
        if kind == "tree":
            handles["mask"] = rk.Mask(s["bits"])
    return dict(s, **handles)


# ---- one pass -----------------------------------------------------------------------------------------------------------

def run(s):
    return {"append": _run_append, "convert": _run_convert, "attend": _run_attend, "pages": _run_pages, "tree": _run_tree,
            "keep": _run_keep}[s["case"]["kind"]](s)


def _pow2(e):
    """Powers of two by their bits, which no library function can round."""
    return (e + 127 << 23).to(torch.int32).view(torch.float32)


def _exponent(x):
    """Of the leading bit of numbers in 32 bits, -127 where there is none."""
    return (x.view(torch.int32) >> 23 & 255) - 127


def _quantised(x, fmt):
    """Codes and block exponents of rows of D channels."""
    bits, low, top, least, most = FORMATS[fmt]
    x = x.float().unflatten(-1, (-1, BLOCK))
    big = x.abs().amax(-1, keepdim=True)
    e = (_exponent(big) - math.frexp(top)[1] + 1).clamp(least, most)
    e = torch.where(big > top * _pow2(e), e + 1, e).clamp(max=most)
    y = (x * _pow2(-e)).clamp(-top, top)
    step = _exponent(y).clamp(min=low) - bits  # of the code's grid; a half goes to the even neighbour
    y = (torch.round(y * _pow2(-step)) * _pow2(step)).flatten(-2)
    scales = (e.squeeze(-1) + 127).to(torch.uint8)
    if fmt == "e4m3":
        return y.to(torch.float8_e4m3fn).view(torch.uint8), scales
    a = y.abs()  # 0, 0.5, 1, 1.5, 2, 3, 4, 6
    code = torch.where(a <= 2, 2 * a, torch.where(a <= 4, a + 2, 7.0)).to(torch.uint8) | torch.signbit(y).to(torch.uint8) << 3
    return code[..., 0::2] | code[..., 1::2] << 4, scales


def _values(codes, scales, fmt):
    """What codes and block exponents stand for."""
    if fmt == "e4m3":
        x = codes.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
        table = torch.cat((table, -table))
        x = table[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    return (x.unflatten(-1, (-1, BLOCK)) * _pow2(scales.int() - 127)[..., None]).flatten(-2)


def _rotate(x, pos, freq, interleaved):
    """Channels in pairs turned by the position's angle: angles in 64 bits, the rest in x's type."""
    half = freq.numel()
    ang = pos.double()[:, None] * freq[None, :]
    cos, sin = torch.cos(ang).to(x.dtype)[:, None, :], torch.sin(ang).to(x.dtype)[:, None, :]
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        y[..., :half], y[..., half:2 * half] = a * cos - b * sin, b * cos + a * sin
    return y


def _summaries(pool, b, p, lens, kmax, kmin):
    """Maximum and minimum of the keys that pages p of sequences b hold."""
    t = p[:, None] * pool.ps + torch.arange(pool.ps, device="cuda")
    k, _ = pool.rows(b[:, None], t)
    seen = (t < lens[b][:, None])[..., None, None]
    some = seen.any(1)
    for to, x in ((kmax, torch.where(seen, k, -math.inf).amax(1)), (kmin, torch.where(seen, k, math.inf).amin(1))):
        to[b, :, :, p] = torch.where(some, x.to(torch.bfloat16), to[b, :, :, p])


def _read_all(pool, lens, other):
    """Every token of the quantised cache into the bf16 one."""
    b, t = (torch.arange(int(pool.cap * pool.ps), device="cuda") < lens[:, None]).nonzero(as_tuple=True)
    k, v = pool.rows(b, t, torch.bfloat16)
    _put(other, b, t, k, v)


def _put(pool, b, t, k, v):
    pp, slot = pool.page(b, t), t % pool.ps
    if pool.fmt is None:
        pool.k[pp, :, slot] = k
        if pool.tm:
            pool.v[pp, :, slot] = v
        else:
            pool.v[pp, :, :, slot] = v
    else:
        pool.k[pp, :, slot], pool.ks[pp, :, slot] = _quantised(k, pool.fmt)
        pool.v[pp, :, slot], pool.vs[pp, :, slot] = _quantised(v, pool.fmt)


def _run_append(s):
    case, pool = s["case"], s["pool"]
    pool.lens.copy_(s["lens0"])  # a pass starts from the same lengths each time, as one taken again
    if own:
        from paper_2502_14051_amd import rocketkv as rk

        rk.q_append_chunk(s["cache"], s["chunk"], s["k"], s["v"], s["kmax"], s["kmin"], s["ws"], rope=s["rope"],
                          q=s.get("q"), q_out=s.get("q_out"))
        if case["read"]:
            rk.restore(s["cache"], s["other_cache"])
    else:
        pos = s["old"][s["seq"]] + s["index"]
        k = s["k"].float()
        if case["rot"]:
            s["q_out"].copy_(_rotate(s["q"].float(), pos, s["freq"], case["interleaved"]))
            k = _rotate(k, pos, s["freq"], case["interleaved"])
        _put(pool, s["seq"], pos, k, s["v"])
        pool.lens += s["there"].sum(1).to(torch.int32)
        _summaries(pool, s["pages"][0], s["pages"][1], pool.lens, s["kmax"], s["kmin"])
        if case["read"]:
            _read_all(pool, pool.lens, s["other"])
            s["other"].lens.copy_(pool.lens)
    out = {"kmax": s["kmax"], "kmin": s["kmin"], "lens": pool.lens}
    if case["rot"]:
        out["q"] = s["q_out"]
    if case["read"]:
        return dict(out, k_read=s["other"].k, v_read=s["other"].v)
    return dict(out, **pool.outputs())


def _run_convert(s):
    case, pool = s["case"], s["pool"]
    if own:
        from paper_2502_14051_amd import rocketkv as rk

        if case["back"]:
            rk.restore(s["cache"], s["other_cache"])
            return dict(s["other"].outputs(), lens=s["other"].lens)
        rk.quantise(s["other_cache"], s["cache"])
        return dict(pool.outputs(), lens=pool.lens)
    if case["back"]:
        _read_all(pool, pool.lens, s["other"])
        s["other"].lens.copy_(pool.lens)
        return dict(s["other"].outputs(), lens=s["other"].lens)
    b, t = (torch.arange(int(pool.cap * pool.ps), device="cuda") < s["other"].lens[:, None]).nonzero(as_tuple=True)
    k, v = s["other"].rows(b, t)
    _put(pool, b, t, k, v)
    pool.lens.copy_(s["other"].lens)
    return dict(pool.outputs(), lens=pool.lens)


def _attention(s, q, k, v, seen):
    """out and log sum-exp of q [B][rows][heads][D] over k, v [B][heads][tokens][D]; seen [B][rows][1 or heads][tokens]."""
    B, n, hq, hkv = q.shape[0], q.shape[1], s["case"]["hq"], s["case"]["hkv"]
    x = q.float().reshape(B, n, hkv, hq // hkv, D).transpose(1, 2).flatten(2, 3) @ k.transpose(2, 3)
    x = x.mul_(SCALE).reshape(B, hkv, n, hq // hkv, -1)
    x.masked_fill_(~seen.transpose(1, 2)[:, :, :, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    p = x.sub_(m).exp_()
    z = p.sum(-1, keepdim=True)
    o = (p.flatten(2, 3) @ v).reshape(B, hkv, n, -1, D) / z
    return o.transpose(1, 2).flatten(2, 3), (m + z.log()).squeeze(-1).transpose(1, 2).flatten(2, 3)


def _run_rows(s, seen_new):
    """Attention of the new tokens; seen_new(t) says which tokens at places t of the chunk each of them sees."""
    pool, B = s["pool"], s["case"]["batch"]
    t = torch.arange(max(o + n for o, n in zip(s["olds"], s["news"])), device="cuda").expand(B, -1)
    k, v = (x.transpose(1, 2) for x in pool.rows(torch.arange(B, device="cuda")[:, None], t))
    place = t - s["old"][:, None]
    seen = (place < 0)[:, None, :] | seen_new(place) & (place >= 0)[:, None, :]
    out, lse = _attention(s, s["q"][s["row"]], k, v, seen[:, :, None])
    s["out"][s["row"][s["there"]]] = out[s["there"]].to(torch.bfloat16)
    s["lse"][s["row"][s["there"]]] = lse[s["there"]]
    return {"out": s["out"], "lse": s["lse"]}


def _run_attend(s):
    if own:
        from paper_2502_14051_amd import rocketkv as rk

        rk.q_chunk_attend(s["cache"], s["chunk"], s["q"], s["out"], s["lse"], s["ws"])
        return {"out": s["out"], "lse": s["lse"]}
    rows = torch.arange(max(s["news"]), device="cuda")[:, None]
    return _run_rows(s, lambda place: place[:, None, :] <= rows)


def _run_pages(s):
    if own:
        from paper_2502_14051_amd import rocketkv as rk

        rk.q_attend(s["cache"], s["q"], s["pages"], s["out"], s["lse"], s["ws"])
        return {"out": s["out"], "lse": s["lse"]}
    pool, B, H = s["pool"], s["case"]["batch"], s["case"]["hkv"]
    t = (s["pages"].long()[..., None] * pool.ps + torch.arange(pool.ps, device="cuda")).flatten(2)  # [B][heads][tokens]
    seen = (t >= 0) & (t < s["old"][:, None, None])
    t = t.clamp(min=0)
    pp, slot, g = pool.page(torch.arange(B, device="cuda")[:, None, None], t), t % pool.ps, torch.arange(H, device="cuda")[:, None]
    k = _values(pool.k[pp, g, slot], pool.ks[pp, g, slot], pool.fmt)
    v = _values(pool.v[pp, g, slot], pool.vs[pp, g, slot], pool.fmt)
    out, lse = _attention(s, s["q"][:, None], k, v, seen[:, None])
    s["out"].copy_(out[:, 0])
    s["lse"].copy_(lse[:, 0])
    return {"out": s["out"], "lse": s["lse"]}


def _run_tree(s):
    if own:
        from paper_2502_14051_amd import rocketkv as rk

        rk.tree_mask(s["chunk"], s["parents"], s["mask"], base=s["base"], positions=s["positions"])
        if s["case"]["fmt"] is None:
            rk.masked_attend(s["cache"], s["chunk"], s["mask"], s["q"], s["out"], s["lse"], s["ws"])
        else:
            rk.q_chunk_attend(s["cache"], s["chunk"], s["q"], s["out"], s["lse"], s["ws"], mask=s["mask"])
        return {"out": s["out"], "lse": s["lse"], "bits": s["bits"], "positions": s["positions"]}
    n = max(s["news"])
    at = torch.arange(n, device="cuda")
    parent = s["parents"].long()[s["row"]]  # (of rows that are not there: of some other, and unused)
    reach = ((parent[..., None] == at) | (at[:, None] == at)).float()  # itself and its parent
    for _ in range((n - 1).bit_length()):
        reach = (reach @ reach > 0).float()  # twice as far
    seen = reach > 0
    words = s["bits"].shape[1]
    wide = torch.zeros((seen.shape[0], n, words * 32), dtype=torch.int64, device="cuda")
    wide[..., :n] = seen
    word = (wide.unflatten(-1, (words, 32)) << torch.arange(32, device="cuda")).sum(-1)
    rows = s["row"][s["there"]]
    s["bits"][rows] = torch.where(word >= 1 << 31, word - (1 << 32), word)[s["there"]].to(torch.int32)
    s["positions"][rows] = (s["base"][:, None] + seen.sum(-1) - 1)[s["there"]].to(torch.int32)
    pick = lambda place: seen.gather(2, place.clamp(0, n - 1)[:, None, :].expand(-1, n, -1)) & (place < n)[:, None, :]
    return dict(_run_rows(s, pick), bits=s["bits"], positions=s["positions"])


def _run_keep(s):
    case, pool = s["case"], s["pool"]
    pool.lens.copy_(s["lens0"])  # a pass starts from the same lengths each time
    if own:
        from paper_2502_14051_amd import rocketkv as rk

        keep = rk.keep_tokens if case["fmt"] is None else rk.q_keep_tokens
        keep(s["cache"], s["chunk"], s["keep"], s["kmax"], s["kmin"], s["ws"])
    else:
        kept = (s["keep"][s["row"]] != 0) & s["there"]
        b, i = kept.nonzero(as_tuple=True)
        to = s["old"][b] + (kept.cumsum(1) - 1)[b, i]
        src, dst = (pool.page(b, s["old"][b] + i), (s["old"][b] + i) % pool.ps), (pool.page(b, to), to % pool.ps)
        for x in (pool.k, pool.v) + ((pool.ks, pool.vs) if pool.fmt else ()):
            if x is pool.v and not pool.tm:
                x[dst[0], :, :, dst[1]] = x[src[0], :, :, src[1]]
            else:
                x[dst[0], :, dst[1]] = x[src[0], :, src[1]]
        pool.lens.copy_(s["old"] + kept.sum(1))
        _summaries(pool, s["pages"][0], s["pages"][1], pool.lens, s["kmax"], s["kmin"])
    return dict(pool.outputs(), kmax=s["kmax"], kmin=s["kmin"], lens=pool.lens)


# ---- what a pass cannot do without --------------------------------------------------------------------------------------

def work(case):
    olds, news = _lengths(case)
    hq, hkv, total = case["hq"], case["hkv"], sum(news)
    lens = [o + n for o, n in zip(olds, news)]
    held = {None: 4 * D, "e4m3": 2 * D + 8, "e2m1": D + 8}[case["fmt"]]  # bytes of a token's key and value
    pages = sum((l + case["ps"] - 1) // case["ps"] - o // case["ps"] for o, l in zip(olds, lens))
    kind = case["kind"]
    if kind == "append":
        rot = case["rot"]
        heads = 2 * hq if rot else 0
        moved = total * (heads * D * 2 + hkv * (4 * D + held)) + 2 * pages * hkv * D * 2
        read = sum(lens) * hkv * (held + 4 * D) if case["read"] else 0
        return {"bytes": moved + read, "flops": total * (3 * (hq + hkv) * rot + 8 * hkv * D)}
    if kind == "convert":
        return {"bytes": sum(olds) * hkv * (held + 4 * D), "flops": sum(olds) * hkv * 2 * D * (2 if case["back"] else 4)}
    if kind == "pages":
        t = hkv * sum(min(o, case["listed_pages"] * case["ps"]) for o in olds)
        return {"bytes": t * held + 4 * hkv * case["batch"] * case["listed_pages"] + case["batch"] * hq * (4 * D + 4),
                "flops": 4 * D * t * hq // hkv}
    if kind == "keep":
        kept = sum(max(1, min(case["kept"], n // 2)) for n in news)
        summed = sum(o % case["ps"] + case["kept"] for o in olds)  # keys of the pages that changed
        return {"bytes": 2 * kept * hkv * held + summed * hkv * held // 2 + total, "flops": 2 * summed * hkv * D}
    if kind == "attend":
        pairs = hq * sum(n * o + n * (n + 1) // 2 for o, n in zip(olds, news))
        bits = 0
    else:  # every drafted token beside the cache: itself and its ancestors, of whom there are few
        pairs = hq * sum(n * o + n for o, n in zip(olds, news))
        bits = total * ((max(news) + 31) // 32 * 4 * 2 + 8)
    return {"bytes": sum(lens) * hkv * held + total * hq * (4 * D + 4) + bits, "flops": 4 * D * pairs}


# ---- the operators' definitions in 64 bits ----------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "convert": _exact_convert, "attend": _exact_rows, "pages": _exact_pages,
            "tree": _exact_rows, "keep": _exact_keep}[case["kind"]](s)


def _grid(fmt):
    """The values of the codes, ascending: every one there is."""
    bits, low, top, _, _ = FORMATS[fmt]
    up = [m * 2.0 ** (low - bits) for m in range(1 << bits)]
    e = low
    while (1 << bits) * 2.0 ** (e - bits) <= top:
        up += [m * 2.0 ** (e - bits) for m in range(1 << bits, 2 << bits) if m * 2.0 ** (e - bits) <= top]
        e += 1
    return torch.tensor(up, dtype=torch.float64, device="cuda")


def _two_to(e):
    return (e.long() + 1023 << 52).view(torch.float64)


def _held(x, fmt):
    """Code values and powers of two of rows of D channels, by the nearest value of the grid (halfway: the even one)."""
    _, _, top, least, most = FORMATS[fmt]
    grid = _grid(fmt)
    x = x.double().reshape(x.shape[:-1] + (D // BLOCK, BLOCK))
    big = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(big / top)).clamp(least, most)
    e = torch.where(big > top * _two_to(e), e + 1, torch.where(big <= top * _two_to(e - 1), e - 1, e)).clamp(least, most)
    y = (x / _two_to(e)).clamp(-top, top)
    a = y.abs()
    hi = torch.searchsorted(grid, a.contiguous()).clamp(max=len(grid) - 1)  # the first that is not below
    lo = (hi - 1).clamp(min=0)
    below, above = a - grid[lo], grid[hi] - a
    near = torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    code = torch.where(torch.signbit(y), -grid[near], grid[near])
    return code.reshape(code.shape[:-2] + (D,)), _two_to(e).squeeze(-1)


def _whole(code, scale):
    return (code.reshape(code.shape[:-1] + (D // BLOCK, BLOCK)) * scale[..., None]).reshape(code.shape)


def _turn(x, pos, freq, interleaved):
    """Every pair of channels as a complex number, times exp(i angle)."""
    half = freq.numel()
    y = x.double()
    pair = y[..., :2 * half].reshape(*y.shape[:-1], half, 2) if interleaved else \
        torch.stack((y[..., :half], y[..., half:2 * half]), -1)
    turn = torch.polar(torch.ones_like(pos, dtype=torch.float64)[:, None], pos.double()[:, None] * freq)
    z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn[:, None, :])
    y = y.clone()
    y[..., :2 * half] = z.flatten(-2) if interleaved else torch.cat((z[..., 0], z[..., 1]), -1)
    return y


def _decoded(pool):
    """Keys and values of every slot of the pools, [pages][heads][slot][D]."""
    if pool.fmt is None:
        return pool.k.double(), (pool.v if pool.tm else pool.v.transpose(2, 3)).double()
    sides = []
    for codes, scales in ((pool.k, pool.ks), (pool.v, pool.vs)):
        if pool.fmt == "e4m3":
            value = codes.view(torch.float8_e4m3fn).double()
        else:
            grid = _grid("e2m1")
            nib = torch.stack((codes % 16, codes // 16), -1).reshape(codes.shape[:-1] + (D,)).long()
            value = torch.where(nib >= 8, -1.0, 1.0) * grid[nib % 8]
        sides.append(_whole(value, _two_to(scales.long() - 127)))
    return sides


def _at(pool, b, n, x):
    """The first n tokens of sequence b out of _decoded's pools: [heads][n][D]."""
    t = torch.arange(n, device="cuda")
    pages = torch.arange(b * pool.cap, (b + 1) * pool.cap, device="cuda") if pool.table is None else pool.table[b].long()
    return x[pages[t // pool.ps], :, t % pool.ps].transpose(0, 1)


def _exact_append(s):
    case, pool = s["case"], s["pool"]
    out = {}
    pos = torch.cat([o + torch.arange(n, device="cuda") for o, n in zip(s["olds"], s["news"])])
    seq = torch.cat([torch.full((n,), b, device="cuda") for b, n in enumerate(s["news"])])
    k = s["k"].double()
    if case["rot"]:
        k = _turn(s["k"], pos, s["freq"], case["interleaved"])
        out["q"] = _turn(s["q"], pos, s["freq"], case["interleaved"])
    lens = pool.lens + torch.tensor(s["news"], dtype=torch.int32, device="cuda")
    page, slot = pos // pool.ps, pos % pool.ps
    phys = seq * pool.cap + page if pool.table is None else pool.table[seq, page].long()
    (kc, ks), (vc, vs) = _held(k, pool.fmt), _held(s["v"], pool.fmt)
    kmax, kmin = s["kmax"].double(), s["kmin"].double()
    value = _whole(kc, ks)
    for b, (old, new) in enumerate(zip(s["olds"], s["news"])):
        mine = seq == b
        fresh = slice((old + pool.ps - 1) // pool.ps, (old + new + pool.ps - 1) // pool.ps)
        for g in range(case["hkv"]):
            # the page that was begun keeps what its older keys gave; the others start here
            kmax[b, g, :, fresh], kmin[b, g, :, fresh] = -math.inf, math.inf
            where = page[mine].expand(D, new)
            kmax[b, g].scatter_reduce_(1, where, value[mine, g].T, "amax")
            kmin[b, g].scatter_reduce_(1, where, value[mine, g].T, "amin")
    out.update(kmax=kmax, kmin=kmin, lens=lens)
    if case["read"]:
        k_all, v_all = _decoded(pool)
        k_all[phys, :, slot], v_all[phys, :, slot] = value, _whole(vc, vs)
        other = s["other"]
        k_read, v_read = other.k.double(), other.v.double()
        for b, n in enumerate(lens.tolist()):
            t = torch.arange(n, device="cuda")
            to = torch.arange(other.cap, device="cuda") + b * other.cap if other.table is None else other.table[b].long()
            k_read[to[t // other.ps], :, t % other.ps] = _at(pool, b, n, k_all).transpose(0, 1)
            v_read[to[t // other.ps], :, t % other.ps] = _at(pool, b, n, v_all).transpose(0, 1)
        return dict(out, k_read=k_read, v_read=v_read)
    for name, codes, scales, c, e in (("k", pool.k, pool.ks, kc, ks), ("v", pool.v, pool.vs, vc, vs)):
        codes, scales = codes.view(torch.float8_e4m3fn).double(), _two_to(scales.long() - 127)
        codes[phys, :, slot], scales[phys, :, slot] = c, e
        out[name], out[name + "_scales"] = codes, scales
    return out


def _exact_convert(s):
    case, pool, other = s["case"], s["pool"], s["other"]
    src, dst = (pool, other) if case["back"] else (other, pool)
    k_src, v_src = _decoded(src)
    if case["back"]:
        k, v = dst.k.double(), dst.v.double()
        for b, n in enumerate(s["olds"]):
            t = torch.arange(n, device="cuda")
            pages = torch.arange(dst.cap, device="cuda") + b * dst.cap if dst.table is None else dst.table[b].long()
            k[pages[t // dst.ps], :, t % dst.ps] = _at(src, b, n, k_src).transpose(0, 1)
            rows = _at(src, b, n, v_src).transpose(0, 1)
            if dst.tm:
                v[pages[t // dst.ps], :, t % dst.ps] = rows
            else:
                v[pages[t // dst.ps], :, :, t % dst.ps] = rows
        return {"k": k, "v": v, "lens": src.lens.clone()}
    out = {"lens": src.lens.clone()}
    for name, x, codes, scales in (("k", k_src, dst.k, dst.ks), ("v", v_src, dst.v, dst.vs)):
        codes, scales = codes.view(torch.float8_e4m3fn).double(), _two_to(scales.long() - 127)
        for b, n in enumerate(s["olds"]):
            t = torch.arange(n, device="cuda")
            pages = torch.arange(dst.cap, device="cuda") + b * dst.cap if dst.table is None else dst.table[b].long()
            c, e = _held(_at(src, b, n, x), dst.fmt)
            codes[pages[t // dst.ps], :, t % dst.ps] = c.transpose(0, 1)
            scales[pages[t // dst.ps], :, t % dst.ps] = e.transpose(0, 1)
        out[name], out[name + "_scales"] = codes, scales
    return out


def _ancestors(s, b):
    """Which of a sequence's drafted tokens each of them sees, a token after the other; and how deep each stands."""
    first, n = sum(s["news"][:b]), s["news"][b]
    parents = s["parents"][first:first + n].tolist()
    seen = torch.eye(n, dtype=torch.bool)
    for i, p in enumerate(parents):
        if p >= 0:
            seen[i] |= seen[p]
    return seen


def _exact_rows(s):
    case, pool = s["case"], s["pool"]
    hq, G, total = case["hq"], case["hq"] // case["hkv"], sum(s["news"])
    out = torch.empty((total, hq, D), dtype=torch.float64, device="cuda")
    lse = torch.empty((total, hq), dtype=torch.float64, device="cuda")
    bits, positions = [], []
    k_all, v_all = _decoded(pool)
    row = 0
    for b, (old, new) in enumerate(zip(s["olds"], s["news"])):
        k, v = _at(pool, b, old + new, k_all), _at(pool, b, old + new, v_all)
        if case["kind"] == "tree":
            among = _ancestors(s, b)
            word = torch.zeros((new, s["bits"].shape[1]), dtype=torch.int64)
            for j in range(new):
                word[:, j // 32] |= among[:, j].long() << j % 32
            bits.append(torch.where(word >= 2 ** 31, word - 2 ** 32, word).to(torch.int32))
            positions.append((old + among.sum(1) - 1).to(torch.int32))
            hidden = ~among.cuda()
        else:
            hidden = torch.ones((new, new), dtype=torch.bool, device="cuda").triu(1)
        for h in range(hq):
            x = s["q"][row:row + new, h].double() @ k[h // G].T / math.sqrt(D)
            x[:, old:][hidden] = -math.inf
            at = slice(row, row + new)
            lse[at, h] = torch.logsumexp(x, 1)
            out[at, h] = torch.exp(x - lse[at, h, None]) @ v[h // G]
        row += new
    if case["kind"] == "tree":
        return {"out": out, "lse": lse, "bits": torch.cat(bits).cuda(), "positions": torch.cat(positions).cuda()}
    return {"out": out, "lse": lse}


def _exact_pages(s):
    case, pool = s["case"], s["pool"]
    hq, hkv = case["hq"], case["hkv"]
    out = torch.empty((case["batch"], hq, D), dtype=torch.float64, device="cuda")
    lse = torch.empty((case["batch"], hq), dtype=torch.float64, device="cuda")
    k_all, v_all = _decoded(pool)
    for b, n in enumerate(s["olds"]):
        k, v = _at(pool, b, n, k_all), _at(pool, b, n, v_all)
        for g in range(hkv):
            chosen = torch.isin(torch.arange(n, device="cuda") // pool.ps, s["pages"][b, g])
            heads = slice(g * hq // hkv, (g + 1) * hq // hkv)
            x = s["q"][b, heads].double() @ k[g, chosen].T / math.sqrt(D)
            lse[b, heads] = torch.logsumexp(x, 1)
            out[b, heads] = torch.softmax(x, 1) @ v[g, chosen]
    return {"out": out, "lse": lse}


def _exact_keep(s):
    case, pool = s["case"], s["pool"]
    k_old, v_old = _decoded(pool)
    copies = [x.clone() for x in ((pool.k, pool.v) if pool.fmt is None else (pool.k, pool.v, pool.ks, pool.vs))]
    kmax, kmin, lens = s["kmax"].double(), s["kmin"].double(), pool.lens.clone()
    row = 0
    for b, (old, new) in enumerate(zip(s["olds"], s["news"])):
        pages = list(range(b * pool.cap, (b + 1) * pool.cap)) if pool.table is None else pool.table[b].tolist()
        flags = s["keep"][row:row + new].tolist()
        accepted = [old + i for i in range(new) if flags[i]]
        for m, i in enumerate(accepted):
            src, dst = (pages[i // pool.ps], i % pool.ps), (pages[(old + m) // pool.ps], (old + m) % pool.ps)
            for j, x in enumerate((pool.k, pool.v) if pool.fmt is None else (pool.k, pool.v, pool.ks, pool.vs)):
                if j == 1 and not pool.tm:
                    copies[j][dst[0], :, :, dst[1]] = x[src[0], :, :, src[1]]
                else:
                    copies[j][dst[0], :, dst[1]] = x[src[0], :, src[1]]
        lens[b] = old + len(accepted)
        order = list(range(old)) + accepted
        for p in range(old // pool.ps, (len(order) + pool.ps - 1) // pool.ps):
            t = order[p * pool.ps:(p + 1) * pool.ps]
            keys = torch.stack([k_old[pages[i // pool.ps], :, i % pool.ps] for i in t])
            kmax[b, :, :, p], kmin[b, :, :, p] = keys.amax(0), keys.amin(0)
        row += new
    out = {"kmax": kmax, "kmin": kmin, "lens": lens}
    if pool.fmt is None:
        return dict(out, k=copies[0].double(), v=copies[1].double())
    out["k"], out["v"] = (x.view(torch.float8_e4m3fn).double() for x in copies[:2])
    out["k_scales"], out["v_scales"] = (_two_to(x.long() - 127) for x in copies[2:])
    return out
