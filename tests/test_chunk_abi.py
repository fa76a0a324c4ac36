"""Host-side checks of the chunk operators that need no GPU: refusals before anything is launched, workspace sizes, the
frequencies of rotary positions."""
import ctypes as C
import math
import os

import pytest

from paper_2502_14051_amd import rocketkv as rk


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(rk.LIB_PATH):
        from paper_2502_14051_amd import build
        build.build()
    return rk.lib()


# (addresses that are looked at and never followed)
Q, K, V, OUT, LSE, WS, KX, KN, W, STARTS, POS, FREQ = (0x10000 * i for i in range(1, 13))
BIG = 1 << 40


def cache(**kw):
    d = dict(batch=2, n_q_heads=32, n_kv_heads=8, head_dim=128, page_size=16, pages_cap=256, n_phys_pages=512,
             stride_page=8 * 16 * 128, stride_head=16 * 128, seq_lens=0x1000, block_table=None, k_pool=0x100000,
             v_pool=0x200000)
    d.update(kw)
    return rk.CacheStruct(**d)


def chunk(**kw):
    return rk.ChunkStruct(**dict(dict(n_tokens=10, starts=STARTS), **kw))


def rope(**kw):
    return rk.RopeStruct(**dict(dict(rot_dim=128, interleaved=0, inv_freq=FREQ, scale=1.0), **kw))


def refused(status, want, needle):
    assert status == want and needle in rk.last_error(), (status, rk.last_error())


def by(x):
    return None if x is None else C.byref(x)


ROPE = dict(rope=rope(), pos=POS, n=10, heads=32, x=Q, xs=32 * 128, y=OUT, ys=32 * 128)


@pytest.mark.parametrize("kw,status,needle", [
    (dict(rope=None), rk.INVALID_ARG, "rope is NULL"), (dict(rope=rope(rot_dim=0)), rk.INVALID_ARG, "rot_dim"),
    (dict(rope=rope(rot_dim=7)), rk.INVALID_ARG, "rot_dim"), (dict(rope=rope(rot_dim=130)), rk.INVALID_ARG, "rot_dim"),
    (dict(rope=rope(interleaved=2)), rk.INVALID_ARG, "interleaved"), (dict(rope=rope(inv_freq=None)), rk.INVALID_ARG, "inv_freq"),
    (dict(rope=rope(inv_freq=FREQ + 4)), rk.INVALID_ARG, "aligned"), (dict(pos=None), rk.INVALID_ARG, "positions"),
    (dict(n=-1), rk.INVALID_ARG, "n_tokens"), (dict(heads=0), rk.INVALID_ARG, "n_heads"),
    (dict(n=rk.MAX_CHUNK + 1), rk.UNSUPPORTED, "tokens"), (dict(heads=5000, xs=5000 * 128, ys=5000 * 128), rk.UNSUPPORTED, "heads"),
    (dict(x=None), rk.INVALID_ARG, "x must not"), (dict(y=OUT + 8), rk.INVALID_ARG, "y must be 16-byte"),
    (dict(xs=31 * 128), rk.INVALID_ARG, "stride of x"), (dict(ys=32 * 128 + 4), rk.INVALID_ARG, "stride of y"),
    (dict(y=Q, ys=40 * 128), rk.INVALID_ARG, "in place"),
])
def test_rope_refusals(L, kw, status, needle):
    a = dict(ROPE, **kw)
    refused(L.rocketkv_rope(by(a["rope"]), a["pos"], a["n"], a["heads"], a["x"], a["xs"], a["y"], a["ys"], None), status, needle)


APPEND = dict(cache=cache(), chunk=chunk(), rope=rope(), pos=None, q=Q, qs=32 * 128, qo=OUT, k=K, ks=8 * 128, v=V, vs=8 * 128,
              kx=KX, kn=KN, ws=WS, wsb=BIG)


@pytest.mark.parametrize("kw,status,needle", [
    (dict(cache=None), rk.INVALID_ARG, "cache is NULL"), (dict(cache=cache(head_dim=64)), rk.UNSUPPORTED, "head_dim"),
    (dict(cache=cache(page_size=8, stride_head=1024, stride_page=8192)), rk.UNSUPPORTED, "page_size"),
    (dict(chunk=None), rk.INVALID_ARG, "chunk is NULL"), (dict(chunk=chunk(starts=None)), rk.INVALID_ARG, "starts"),
    (dict(chunk=chunk(n_tokens=-1)), rk.INVALID_ARG, "n_tokens"), (dict(chunk=chunk(n_tokens=rk.MAX_CHUNK + 1)), rk.UNSUPPORTED, "n_tokens"),
    (dict(rope=rope(rot_dim=9)), rk.INVALID_ARG, "rot_dim"), (dict(rope=None, pos=POS), rk.INVALID_ARG, "positions without rope"),
    (dict(q=None), rk.INVALID_ARG, "go together"), (dict(qo=None), rk.INVALID_ARG, "go together"),
    (dict(qs=100), rk.INVALID_ARG, "stride of q"), (dict(qo=Q, qs=48 * 128), rk.INVALID_ARG, "in place"),
    (dict(k=None), rk.INVALID_ARG, "k_new"), (dict(v=V + 2), rk.INVALID_ARG, "v_new"), (dict(ks=7 * 128), rk.INVALID_ARG, "k_new"),
    (dict(kx=None), rk.INVALID_ARG, "kmax and kmin"), (dict(kn=KN + 2), rk.INVALID_ARG, "aligned"),
    (dict(ws=None), rk.WORKSPACE_TOO_SMALL, "workspace"), (dict(wsb=100), rk.WORKSPACE_TOO_SMALL, "workspace"),
    (dict(ws=WS + 16), rk.INVALID_ARG, "aligned"),
])
def test_append_refusals(L, kw, status, needle):
    a = dict(APPEND, **kw)
    refused(L.rocketkv_append_chunk(by(a["cache"]), by(a["chunk"]), by(a["rope"]), a["pos"], a["q"], a["qs"], a["qo"], a["k"],
                                    a["ks"], a["v"], a["vs"], a["kx"], a["kn"], a["ws"], a["wsb"], None), status, needle)


ATTEND = dict(cache=cache(), chunk=chunk(), q=Q, out=OUT, lse=LSE, ws=WS, wsb=BIG)


@pytest.mark.parametrize("kw,status,needle", [
    (dict(cache=None), rk.INVALID_ARG, "cache is NULL"), (dict(cache=cache(k_pool=None)), rk.INVALID_ARG, "NULL"),
    (dict(cache=cache(page_size=4, stride_head=512, stride_page=4096)), rk.UNSUPPORTED, "page_size"),
    (dict(chunk=None), rk.INVALID_ARG, "chunk is NULL"), (dict(chunk=chunk(n_tokens=-5)), rk.INVALID_ARG, "n_tokens"),
    (dict(q=None), rk.INVALID_ARG, "q must not"), (dict(out=OUT + 2), rk.INVALID_ARG, "out must be"),
    (dict(out=Q), rk.INVALID_ARG, "distinct"), (dict(ws=None), rk.WORKSPACE_TOO_SMALL, "workspace"),
    (dict(wsb=1000), rk.WORKSPACE_TOO_SMALL, "workspace"), (dict(ws=WS + 8), rk.INVALID_ARG, "aligned"),
    (dict(cache=cache(n_q_heads=256, n_kv_heads=16, stride_page=16 * 2048), chunk=chunk(n_tokens=rk.MAX_CHUNK)), rk.UNSUPPORTED, "too many rows"),
    (dict(cache=cache(n_q_heads=136)), rk.UNSUPPORTED, "group size"),
])
def test_attend_refusals(L, kw, status, needle):
    a = dict(ATTEND, **kw)
    refused(L.rocketkv_chunk_attend(by(a["cache"]), by(a["chunk"]), a["q"], a["out"], a["lse"], a["ws"], a["wsb"], None), status, needle)


@pytest.mark.parametrize("kw,status,needle", [
    (dict(cache=None), rk.INVALID_ARG, "cache is NULL"), (dict(chunk=None), rk.INVALID_ARG, "chunk is NULL"),
    (dict(q=None), rk.INVALID_ARG, "q must not"), (dict(lse=None), rk.INVALID_ARG, "lse"), (dict(out=None), rk.INVALID_ARG, "weights_out"),
    (dict(cache=cache(block_table=0x5000, pages_cap=1 << 26)), rk.UNSUPPORTED, "too many keys"),
])
def test_accumulate_refusals(L, kw, status, needle):
    a = dict(dict(cache=cache(), chunk=chunk(), q=Q, lse=LSE, w=None, out=W), **kw)
    refused(L.rocketkv_accumulate_weights(by(a["cache"]), by(a["chunk"]), a["q"], a["lse"], a["w"], a["out"], None), status, needle)


EVICT = dict(src=cache(), w=W, recent=32, keep=1024, dst=cache(k_pool=0x300000, v_pool=0x400000, seq_lens=0x2000), wo=OUT,
             kept=None, ws=WS, wsb=BIG)


@pytest.mark.parametrize("kw,status,needle", [
    (dict(src=None), rk.INVALID_ARG, "cache is NULL"), (dict(dst=None), rk.INVALID_ARG, "cache is NULL"),
    (dict(src=cache(page_size=8, stride_head=1024, stride_page=8192)), rk.UNSUPPORTED, "page_size"),
    (dict(dst=cache(batch=1)), rk.INVALID_ARG, "agree"), (dict(dst=cache(n_q_heads=16)), rk.INVALID_ARG, "agree"),
    (dict(dst=cache()), rk.INVALID_ARG, "distinct"), (dict(dst=cache(k_pool=0x300000, v_pool=0x400000)), rk.INVALID_ARG, "distinct"),
    (dict(keep=257 * 16, dst=cache(k_pool=0x300000, v_pool=0x400000, seq_lens=0x2000)), rk.INVALID_ARG, "dst holds"),
    (dict(w=None), rk.INVALID_ARG, "weights must not"), (dict(w=W + 4), rk.INVALID_ARG, "aligned"), (dict(wo=W), rk.INVALID_ARG, "distinct"),
    (dict(recent=-1), rk.INVALID_ARG, "n_recent"), (dict(recent=1025), rk.INVALID_ARG, "n_recent"), (dict(keep=0, recent=0), rk.INVALID_ARG, "keep_budget"),
    (dict(ws=None), rk.WORKSPACE_TOO_SMALL, "workspace"), (dict(wsb=65536), rk.WORKSPACE_TOO_SMALL, "workspace"),
])
def test_evict_refusals(L, kw, status, needle):
    a = dict(EVICT, **kw)
    refused(L.rocketkv_weight_evict(by(a["src"]), a["w"], a["recent"], a["keep"], by(a["dst"]), a["wo"], a["kept"], a["ws"],
                                    a["wsb"], None), status, needle)


def test_workspace_sizes(L):
    size = lambda op, a, b=0, **kw: L.rocketkv_workspace_bytes(op, C.byref(cache(**kw)), a, b)
    assert size(rk.OP_APPEND_CHUNK, 0) == size(rk.OP_APPEND_CHUNK, 1 << 20) == 65536
    assert size(rk.OP_CHUNK_ATTEND, 1) > 65536
    assert size(rk.OP_CHUNK_ATTEND, 0) == 0 and rk.last_error() == ""
    assert size(rk.OP_CHUNK_ATTEND, 1 << 20) == size(rk.OP_CHUNK_ATTEND, 1)  # what serves many tokens serves few
    for op in (rk.OP_APPEND_CHUNK, rk.OP_CHUNK_ATTEND):
        assert size(op, -1) == 0 and "n_tokens" in rk.last_error()
        assert size(op, rk.MAX_CHUNK + 1) == 0 and "exceeds" in rk.last_error()
    assert size(rk.OP_WEIGHT_EVICT, 32, 1024) >= 65536 + 16 * 1024 * 4
    for recent, keep in ((-1, 5), (6, 5), (0, 0)):
        assert size(rk.OP_WEIGHT_EVICT, recent, keep) == 0 and "n_recent" in rk.last_error()


# ---- frequencies ----

def frequencies(L, kind, rot=128, theta=500000.0, factor=8.0, low=1.0, high=4.0, original=8192):
    f, s = (C.c_double * (rot // 2))(), C.c_float()
    status = L.rocketkv_rope_frequencies(kind, rot, theta, factor, low, high, original, f, C.byref(s))
    return status, list(f), s.value


def test_frequencies_follow_their_definitions(L):
    for rot, theta in ((128, 500000.0), (64, 10000.0), (2, 10000.0)):
        plain = [theta ** (-2 * i / rot) for i in range(rot // 2)]
        close = lambda got, want: all(math.isclose(g, w, rel_tol=1e-14) for g, w in zip(got, want))
        status, f, s = frequencies(L, rk.ROPE_PLAIN, rot, theta)
        assert status == rk.OK and s == 1 and close(f, plain)
        status, f, s = frequencies(L, rk.ROPE_LINEAR, rot, theta)
        assert status == rk.OK and s == 1 and close(f, [x / 8 for x in plain])
        if rot > 2:
            status, f, s = frequencies(L, rk.ROPE_BASE, rot, theta)
            assert status == rk.OK and s == 1 and f[0] == 1.0 and math.isclose(f[-1], plain[-1] / 8, rel_tol=1e-12)
        status, f, s = frequencies(L, rk.ROPE_BANDS, rot, theta)
        assert status == rk.OK and s == 1
        for g, x in zip(f, plain):
            turns = 8192 * x / (2 * math.pi)
            u = min(max((turns - 1) / 3, 0), 1)
            assert math.isclose(g, x / 8 * (1 - u) + x * u, rel_tol=1e-13)
        status, f, s = frequencies(L, rk.ROPE_RAMP, rot, theta, factor=40.0, low=1.0, high=32.0, original=4096)
        assert status == rk.OK and math.isclose(s, 0.1 * math.log(40) + 1, rel_tol=1e-6)
        at = lambda turns: rot / 2 * math.log(4096 / (turns * 2 * math.pi)) / math.log(theta)
        a, b = max(math.floor(at(32)), 0), min(math.ceil(at(1)), rot - 1)
        for i, (g, x) in enumerate(zip(f, plain)):
            u = 1 - min(max((i - a) / max(b - a, 0.001), 0), 1)
            assert math.isclose(g, x / 40 * (1 - u) + x * u, rel_tol=1e-13)


@pytest.mark.parametrize("kw", [dict(kind=5), dict(kind=-1), dict(rot=3), dict(rot=0), dict(rot=130), dict(theta=1.0), dict(theta=math.nan),
                                dict(theta=math.inf), dict(kind=1, factor=0.5), dict(kind=1, factor=math.nan), dict(kind=2, rot=2),
                                dict(kind=3, low=4.0, high=4.0), dict(kind=3, low=0.0), dict(kind=4, original=0), dict(kind=4, high=math.inf)])
def test_frequency_refusals(L, kw):
    a = dict(dict(kind=rk.ROPE_PLAIN, rot=128, theta=1e4, factor=8.0, low=1.0, high=4.0, original=8192), **kw)
    f, s = (C.c_double * 128)(), C.c_float()
    assert L.rocketkv_rope_frequencies(a["kind"], a["rot"], a["theta"], a["factor"], a["low"], a["high"], a["original"], f,
                                       C.byref(s)) == rk.INVALID_ARG
    assert L.rocketkv_rope_frequencies(0, 128, 1e4, 1.0, 1.0, 4.0, 1, None, C.byref(s)) == rk.INVALID_ARG


# ---- the binding's own checks ----

def test_tensors_of_another_kind_are_refused():
    import torch
    x = torch.zeros((3, 4, 128), dtype=torch.bfloat16)
    pos = torch.zeros(3, dtype=torch.int32)
    r = rk.Rope(torch.zeros(64, dtype=torch.float64))
    for a, b, p, needle in ((x.float(), x, pos, "bfloat16"), (x[..., :64], x, pos, "x: need"), (x[0], x, pos, "x: need"),
                            (x, x, pos, "current GPU")):
        with pytest.raises(rk.RocketKVError) as e:
            rk.rope(r, p, a, b)
        assert e.value.status == rk.INVALID_ARG and needle in str(e.value)
    with pytest.raises(rk.RocketKVError):
        rk.Rope(torch.zeros(64)).struct()
    with pytest.raises(rk.RocketKVError):
        rk.rope_frequencies(-2, 1e4)
    assert rk.rope_frequencies(64, 1e4).inv_freq.shape == (32,)
