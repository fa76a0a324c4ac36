"""Host-side checks of the calls on quantised caches and on trees of drafted tokens that need no GPU: refusals before
anything is launched, workspace sizes, and what the binding looks at."""
import ctypes as C
import os

import pytest
import torch

from paper_2502_14051_amd import rocketkv as rk


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(rk.LIB_PATH):
        from paper_2502_14051_amd import build
        build.build()
    return rk.lib()


# (addresses that are looked at and never followed)
Q, K, V, OUT, LSE, WS, KX, KN, BITS, STARTS, POS, FREQ, PARENTS, KEEP, LIST = (0x10000 * i for i in range(1, 16))
BIG = 1 << 40


def qcache(**kw):
    d = dict(batch=2, n_q_heads=32, n_kv_heads=8, head_dim=128, page_size=16, pages_cap=256, n_phys_pages=512, stride_page=8 * 16,
             stride_head=16, seq_lens=0x1000, block_table=None, k_codes=0x100000, v_codes=0x200000, k_scales=0x300000,
             v_scales=0x400000, format=rk.Q_E4M3)
    d.update(kw)
    return rk.QCacheStruct(**d)


def cache(**kw):
    d = dict(batch=2, n_q_heads=32, n_kv_heads=8, head_dim=128, page_size=16, pages_cap=256, n_phys_pages=512,
             stride_page=8 * 16 * 128, stride_head=16 * 128, seq_lens=0x2000, block_table=None, k_pool=0x500000,
             v_pool=0x600000)
    d.update(kw)
    return rk.CacheStruct(**d)


def chunk(**kw):
    return rk.ChunkStruct(**dict(dict(n_tokens=10, starts=STARTS), **kw))


def mask(**kw):
    return rk.MaskStruct(**dict(dict(bits=BITS, words=2), **kw))


def rope(**kw):
    return rk.RopeStruct(**dict(dict(rot_dim=128, interleaved=0, inv_freq=FREQ, scale=1.0), **kw))


def by(x):
    return None if x is None else C.byref(x)


def refused(status, want, needle):
    assert status == want and needle in rk.last_error(), (status, rk.last_error())


BAD_CACHES = [
    (None, rk.INVALID_ARG, "cache is NULL"), (dict(batch=0), rk.INVALID_ARG, "positive"), (dict(head_dim=64), rk.UNSUPPORTED, "head_dim"),
    (dict(n_q_heads=33), rk.INVALID_ARG, "multiple"), (dict(n_q_heads=136), rk.UNSUPPORTED, "group size"),
    (dict(page_size=0), rk.INVALID_ARG, "page_size"), (dict(page_size=65, stride_head=65, stride_page=520), rk.UNSUPPORTED, "page_size"),
    (dict(pages_cap=12), rk.INVALID_ARG, "pages_cap"), (dict(format=2), rk.INVALID_ARG, "format"), (dict(format=-1), rk.INVALID_ARG, "format"),
    (dict(seq_lens=None), rk.INVALID_ARG, "NULL"), (dict(k_codes=None), rk.INVALID_ARG, "NULL"), (dict(v_scales=None), rk.INVALID_ARG, "NULL"),
    (dict(stride_head=15), rk.INVALID_ARG, "strides"), (dict(stride_page=127), rk.INVALID_ARG, "strides"),
    (dict(stride_page=-128), rk.INVALID_ARG, "strides"),
    (dict(n_phys_pages=0), rk.INVALID_ARG, "n_phys_pages"), (dict(n_phys_pages=511), rk.INVALID_ARG, "identity"),
    (dict(stride_page=1 << 23), rk.UNSUPPORTED, "2^32"), (dict(stride_head=1 << 31), rk.UNSUPPORTED, "2^32"),
    (dict(n_phys_pages=1 << 31, block_table=0x3000), rk.UNSUPPORTED, "2^32"), (dict(stride_head=1 << 62), rk.UNSUPPORTED, "2^32"),
    (dict(k_codes=0x100008), rk.INVALID_ARG, "16-byte"), (dict(k_scales=0x300002), rk.INVALID_ARG, "4-byte"),
    (dict(batch=2000), rk.UNSUPPORTED, "batch"),
]
CALLS = {
    "append": lambda L, q: L.rocketkv_q_append_chunk(by(q), by(chunk()), None, None, None, 0, None, K, 1024, V, 1024, None, None, WS, BIG, None),
    "chunk_attend": lambda L, q: L.rocketkv_q_chunk_attend(by(q), by(chunk()), None, Q, OUT, None, WS, BIG, None),
    "attend": lambda L, q: L.rocketkv_q_attend(by(q), Q, LIST, 4, OUT, None, WS, BIG, None),
    "hsa_decode": lambda L, q: L.rocketkv_q_hsa_decode(by(q), Q, KX, KN, 16, 1024, 0, OUT, None, None, None, WS, BIG, None),
    "quantise": lambda L, q: L.rocketkv_quantise(by(cache()), by(q), None),
    "restore": lambda L, q: L.rocketkv_restore(by(q), by(cache()), None),
    "keep": lambda L, q: L.rocketkv_q_keep_tokens(by(q), by(chunk()), KEEP, None, None, WS, BIG, None),
}


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("kw,status,needle", BAD_CACHES)
def test_every_call_looks_at_its_cache(L, call, kw, status, needle):
    refused(CALLS[call](L, None if kw is None else qcache(**kw)), status, needle)


APPEND = dict(chunk=chunk(), rope=rope(), pos=None, q=Q, qs=32 * 128, qo=OUT, k=K, ks=8 * 128, v=V, vs=8 * 128, kx=KX, kn=KN, ws=WS, wsb=BIG)


@pytest.mark.parametrize("kw,status,needle", [
    (dict(chunk=None), rk.INVALID_ARG, "chunk is NULL"), (dict(chunk=chunk(starts=None)), rk.INVALID_ARG, "starts"),
    (dict(chunk=chunk(n_tokens=-1)), rk.INVALID_ARG, "n_tokens"), (dict(chunk=chunk(n_tokens=rk.MAX_CHUNK + 1)), rk.UNSUPPORTED, "n_tokens"),
    (dict(rope=rope(rot_dim=9)), rk.INVALID_ARG, "rot_dim"), (dict(rope=None, pos=POS), rk.INVALID_ARG, "positions without rope"),
    (dict(q=None), rk.INVALID_ARG, "go together"), (dict(qs=100), rk.INVALID_ARG, "stride of q"),
    (dict(k=None), rk.INVALID_ARG, "k_new"), (dict(v=V + 2), rk.INVALID_ARG, "v_new"), (dict(ks=7 * 128), rk.INVALID_ARG, "k_new"),
    (dict(kx=None), rk.INVALID_ARG, "kmax and kmin"), (dict(kn=KN + 2), rk.INVALID_ARG, "aligned"),
    (dict(ws=None), rk.WORKSPACE_TOO_SMALL, "workspace"), (dict(wsb=100), rk.WORKSPACE_TOO_SMALL, "workspace"), (dict(ws=WS + 16), rk.INVALID_ARG, "aligned"),
])
def test_append_refusals(L, kw, status, needle):
    a = dict(APPEND, **kw)
    refused(L.rocketkv_q_append_chunk(by(qcache()), by(a["chunk"]), by(a["rope"]), a["pos"], a["q"], a["qs"], a["qo"], a["k"], a["ks"],
                                      a["v"], a["vs"], a["kx"], a["kn"], a["ws"], a["wsb"], None), status, needle)


ATTEND = dict(chunk=chunk(), mask=mask(), q=Q, out=OUT, ws=WS, wsb=BIG)


@pytest.mark.parametrize("kw,status,needle", [
    (dict(chunk=None), rk.INVALID_ARG, "chunk is NULL"), (dict(chunk=chunk(n_tokens=-5)), rk.INVALID_ARG, "n_tokens"),
    (dict(mask=mask(bits=None)), rk.INVALID_ARG, "bits"), (dict(mask=mask(bits=BITS + 2)), rk.INVALID_ARG, "aligned"),
    (dict(mask=mask(words=0)), rk.INVALID_ARG, "words"), (dict(mask=mask(words=1 << 20)), rk.UNSUPPORTED, "words"),
    (dict(q=None), rk.INVALID_ARG, "q must not"), (dict(out=OUT + 2), rk.INVALID_ARG, "out must be"), (dict(out=Q), rk.INVALID_ARG, "distinct"),
    (dict(ws=None), rk.WORKSPACE_TOO_SMALL, "workspace"), (dict(wsb=1000), rk.WORKSPACE_TOO_SMALL, "workspace"), (dict(ws=WS + 8), rk.INVALID_ARG, "aligned"),
])
def test_attend_refusals(L, kw, status, needle):
    a = dict(ATTEND, **kw)
    refused(L.rocketkv_q_chunk_attend(by(qcache()), by(a["chunk"]), by(a["mask"]), a["q"], a["out"], LSE, a["ws"], a["wsb"], None), status, needle)
    refused(L.rocketkv_masked_attend(by(cache()), by(a["chunk"]), by(a["mask"]), a["q"], a["out"], LSE, a["ws"], a["wsb"], None), status, needle)


def test_masked_attend_needs_a_mask_and_a_cache(L):
    refused(L.rocketkv_masked_attend(by(cache()), by(chunk()), None, Q, OUT, None, WS, BIG, None), rk.INVALID_ARG, "mask is NULL")
    refused(L.rocketkv_masked_attend(None, by(chunk()), by(mask()), Q, OUT, None, WS, BIG, None), rk.INVALID_ARG, "cache is NULL")
    refused(L.rocketkv_masked_attend(by(cache(page_size=4, stride_head=512, stride_page=4096)), by(chunk()), by(mask()), Q, OUT, None, WS, BIG, None),
            rk.UNSUPPORTED, "page_size")


@pytest.mark.parametrize("kw,status,needle", [
    (dict(q=Q + 8), rk.INVALID_ARG, "q must be"), (dict(out=None), rk.INVALID_ARG, "out must not"), (dict(out=Q), rk.INVALID_ARG, "distinct"),
    (dict(row=0), rk.INVALID_ARG, "pages_row_len"), (dict(row=1 << 27), rk.UNSUPPORTED, "2^30"),
    (dict(row=1 << 26, batch=512, n_phys_pages=512 * 256), rk.UNSUPPORTED, "2^36"),
    (dict(ws=None), rk.WORKSPACE_TOO_SMALL, "workspace"), (dict(wsb=1000), rk.WORKSPACE_TOO_SMALL, "workspace"), (dict(ws=WS + 8), rk.INVALID_ARG, "aligned"),
])
def test_listed_refusals(L, kw, status, needle):
    a = dict(dict(q=Q, pages=LIST, row=64, out=OUT, ws=WS, wsb=BIG, batch=2, n_phys_pages=512), **kw)
    refused(L.rocketkv_q_attend(by(qcache(batch=a["batch"], n_phys_pages=a["n_phys_pages"])), a["q"], a["pages"], a["row"], a["out"], LSE, a["ws"], a["wsb"], None), status, needle)


@pytest.mark.parametrize("kw,status,needle", [
    (dict(q=None), rk.INVALID_ARG, "q / kmax / kmin"), (dict(kx=KX + 2), rk.INVALID_ARG, "aligned"), (dict(k1=0), rk.INVALID_ARG, "channel_budget"),
    (dict(k1=129), rk.INVALID_ARG, "channel_budget"), (dict(T=0), rk.INVALID_ARG, "token_budget"), (dict(recent=-1), rk.INVALID_ARG, "n_recent"),
    (dict(out=None), rk.INVALID_ARG, "out must not"), (dict(out=Q), rk.INVALID_ARG, "distinct"), (dict(wsb=70000), rk.WORKSPACE_TOO_SMALL, "workspace"),
])
def test_decode_refusals(L, kw, status, needle):
    a = dict(dict(q=Q, kx=KX, k1=16, T=1024, recent=0, out=OUT, wsb=BIG), **kw)
    refused(L.rocketkv_q_hsa_decode(by(qcache()), a["q"], a["kx"], KN, a["k1"], a["T"], a["recent"], a["out"], None, None, None, WS, a["wsb"], None),
            status, needle)


def test_decode_of_more_pages_than_selection_has(L):
    big = qcache(pages_cap=32776, n_phys_pages=2 * 32776)
    refused(L.rocketkv_q_hsa_decode(by(big), Q, KX, KN, 16, 1024, 0, OUT, None, None, None, WS, BIG, None), rk.UNSUPPORTED, "pages_cap")


@pytest.mark.parametrize("kw,qkw,status,needle", [
    (dict(batch=3, n_phys_pages=1000), {}, rk.INVALID_ARG, "agree"), (dict(n_kv_heads=4), {}, rk.INVALID_ARG, "agree"),
    (dict(seq_lens=0x1000), {}, rk.INVALID_ARG, "distinct"), (dict(k_pool=0x100000), {}, rk.INVALID_ARG, "distinct"),
    (dict(page_size=8, stride_head=1024, stride_page=8192), {}, rk.UNSUPPORTED, "page_size"), (dict(v_pool=None), {}, rk.INVALID_ARG, "NULL"),
    (dict(pages_cap=1 << 26, block_table=0x3000), dict(pages_cap=1 << 26, block_table=0x3000), rk.UNSUPPORTED, "too many tokens"),
])
def test_convert_refusals(L, kw, qkw, status, needle):
    refused(L.rocketkv_quantise(by(cache(**kw)), by(qcache(**qkw)), None), status, needle)
    refused(L.rocketkv_restore(by(qcache(**qkw)), by(cache(**kw)), None), status, needle)


@pytest.mark.parametrize("kw,status,needle", [
    (dict(chunk=None), rk.INVALID_ARG, "chunk is NULL"), (dict(keep=None), rk.INVALID_ARG, "keep"), (dict(kn=None), rk.INVALID_ARG, "go together"),
    (dict(kx=KX + 8), rk.INVALID_ARG, "aligned"), (dict(ws=None), rk.WORKSPACE_TOO_SMALL, "workspace"), (dict(ws=WS + 8), rk.INVALID_ARG, "aligned"),
])
def test_keep_refusals(L, kw, status, needle):
    a = dict(dict(chunk=chunk(), keep=KEEP, kx=KX, kn=KN, ws=WS), **kw)
    refused(L.rocketkv_keep_tokens(by(cache()), by(a["chunk"]), a["keep"], a["kx"], a["kn"], a["ws"], BIG, None), status, needle)
    refused(L.rocketkv_q_keep_tokens(by(qcache()), by(a["chunk"]), a["keep"], a["kx"], a["kn"], a["ws"], BIG, None), status, needle)
    refused(L.rocketkv_keep_tokens(by(cache(page_size=8, stride_head=1024, stride_page=8192)), by(chunk()), KEEP, None, None, WS, BIG, None),
            rk.UNSUPPORTED, "page_size")


@pytest.mark.parametrize("kw,status,needle", [
    (dict(batch=0), rk.INVALID_ARG, "batch"), (dict(chunk=None), rk.INVALID_ARG, "chunk is NULL"), (dict(parents=None), rk.INVALID_ARG, "parents"),
    (dict(base=None), rk.INVALID_ARG, "go together"), (dict(pos=None), rk.INVALID_ARG, "go together"), (dict(bits=None), rk.INVALID_ARG, "bits"),
    (dict(words=0), rk.INVALID_ARG, "words"), (dict(chunk=chunk(n_tokens=rk.MAX_CHUNK + 1)), rk.UNSUPPORTED, "n_tokens"),
    (dict(batch=rk.MAX_CHUNK), rk.UNSUPPORTED, "batch"),
])
def test_tree_mask_refusals(L, kw, status, needle):
    a = dict(dict(batch=2, chunk=chunk(), parents=PARENTS, base=LIST, bits=BITS, words=1, pos=POS), **kw)
    refused(L.rocketkv_tree_mask(a["batch"], by(a["chunk"]), a["parents"], a["base"], a["bits"], a["words"], a["pos"], None), status, needle)


def test_workspaces(L):
    def need(op, a, **kw):
        return L.rocketkv_q_workspace_bytes(op, by(qcache(**kw)), a)

    for bad in ((99, 1), (rk.OP_SNAPKV, 32), (rk.OP_ATTEND, -1), (rk.OP_ATTEND, 1 << 27), (rk.OP_HSA_DECODE, 0), (rk.OP_CHUNK_ATTEND, -1),
                (rk.OP_APPEND_CHUNK, rk.MAX_CHUNK + 1)):
        assert need(*bad) == 0 and rk.last_error()
    assert need(rk.OP_CHUNK_ATTEND, 1, format=7) == 0 and "format" in rk.last_error()
    assert need(rk.OP_APPEND_CHUNK, 1) == 65536
    assert need(rk.OP_CHUNK_ATTEND, 0) == 0 and rk.last_error() == ""
    assert need(rk.OP_CHUNK_ATTEND, 1) == need(rk.OP_CHUNK_ATTEND, 100000) > 65536, "one serves calls of any size"
    assert need(rk.OP_CHUNK_ATTEND, 1, seq_lens=None, k_codes=None) > 0, "sizes do not look at pointers"
    assert need(rk.OP_HSA_DECODE, 1024) >= need(rk.OP_ATTEND, 64) + 2 * 8 * (64 + 256) * 4


def test_binding_looks_at_tensors():
    q = rk.alloc_qcache(2, 8, 2, 4, 8, "cpu")
    rk.alloc_qcache(2, 8, 2, 4, 8, "cpu", rk.Q_E2M1).struct()
    assert q.struct().stride_page == 8 and q.struct().stride_head == 4 and q.struct().n_phys_pages == 16
    wide = torch.zeros((16, 4, 4, 128), dtype=torch.uint8)
    wide_s = torch.zeros((16, 4, 4, 4), dtype=torch.uint8)
    q.k_codes = q.v_codes = wide[:, 1:3]
    with pytest.raises(rk.RocketKVError, match="strides"):
        q.struct()
    q.k_scales = q.v_scales = wide_s[:, 1:3]
    assert q.struct().stride_page == 16 and q.struct().stride_head == 4
    q.v_codes = torch.zeros((16, 2, 4, 64), dtype=torch.uint8)
    with pytest.raises(rk.RocketKVError, match="v_codes"):
        q.struct()
    with pytest.raises(rk.RocketKVError, match="format"):
        rk.alloc_qcache(2, 8, 2, 4, 8, "cpu", 5)
    q = rk.alloc_qcache(2, 8, 2, 4, 8, "cpu")
    ch = rk.Chunk(torch.zeros(3, dtype=torch.int32), 5)
    t = torch.zeros((5, 8, 128), dtype=torch.bfloat16)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(rk.RocketKVError, match="q: need"):
        rk.q_chunk_attend(q, ch, t.float(), t, None, ws)
    with pytest.raises(rk.RocketKVError, match="not on the current GPU"):
        rk.q_chunk_attend(q, ch, t, t.clone(), None, ws)
    with pytest.raises(rk.RocketKVError, match="bits"):
        rk.q_chunk_attend(q, ch, t, t.clone(), None, ws, mask=rk.Mask(torch.zeros((4, 1), dtype=torch.int32)))
    with pytest.raises(rk.RocketKVError, match="keep"):
        rk.q_keep_tokens(q, ch, torch.zeros(5, dtype=torch.int32), None, None, ws)
    with pytest.raises(rk.RocketKVError, match="pages"):
        rk.q_attend(q, t[:2], torch.zeros((2, 3, 4), dtype=torch.int32), t[:2].clone(), None, ws)
    with pytest.raises(rk.RocketKVError, match="parents"):
        rk.tree_mask(ch, torch.zeros(4, dtype=torch.int32), rk.alloc_mask(5, 5, "cpu"))


def test_caches_of_another_layout_are_refused():
    """As many bytes in another order of dimensions, or of another type, are no cache."""
    for bad in (torch.zeros((16, 4, 2, 128), dtype=torch.uint8), torch.zeros((16, 2, 4, 64), dtype=torch.bfloat16)):
        q = rk.alloc_qcache(2, 8, 2, 4, 8, "cpu")
        q.k_codes = bad
        with pytest.raises(rk.RocketKVError, match="k_codes"):
            q.struct()
