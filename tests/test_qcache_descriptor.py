"""What the binding looks at in the tensors of a quantised cache (no GPU): a pointer says neither shape, order nor type."""
import ctypes as C
import os

import pytest
import torch

from paper_2502_14051_amd import rocketkv as rk

BATCH, HEADS, PS, CAP = 3, 2, 4, 8


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(rk.LIB_PATH):
        from paper_2502_14051_amd import build
        build.build()


def cache(fmt=rk.Q_E4M3, table=False):
    t = torch.zeros((BATCH, CAP), dtype=torch.int32) if table else None
    return rk.alloc_qcache(BATCH, 8, HEADS, PS, CAP, "cpu", fmt, t)


N = BATCH * CAP
WRONG = {
    "k_codes": [(torch.uint8, (N, PS, HEADS, 128)), (torch.bfloat16, (N, HEADS, PS, 64)), (torch.uint8, (N, HEADS * PS, 128)), (torch.int32, (N, HEADS, PS, 32))],
    "v_codes": [(torch.uint8, (N, PS, HEADS, 128)), (torch.bfloat16, (N, HEADS, PS, 64)), (torch.bfloat16, (N, HEADS, PS, 128)), (torch.uint8, (N - 1, HEADS, PS, 128)),
                (torch.uint8, (N * HEADS * PS, 128)), (torch.uint8, (N * HEADS * PS * 128,))],
    "k_scales": [(torch.uint8, (N, PS, HEADS, 4)), (torch.int32, (N, HEADS, PS)), (torch.int32, (N, HEADS, PS, 1)), (torch.uint8, (N * HEADS * PS * 4,))],
    "v_scales": [(torch.uint8, (N, PS, HEADS, 4)), (torch.int32, (N, HEADS, PS)), (torch.float32, (N, HEADS, PS, 1)), (torch.uint8, (N, HEADS, PS, 8))],
    "seq_lens": [(torch.int64, (BATCH,)), (torch.int32, (BATCH - 1,)), (torch.int32, (BATCH, 1)), (torch.float32, (BATCH,))],
    "block_table": [(torch.int64, (BATCH, CAP)), (torch.int32, (BATCH - 1, CAP)), (torch.int32, (BATCH, CAP - 1)), (torch.int32, (BATCH * CAP,))],
}


@pytest.mark.parametrize("name,dtype,shape", [(n, d, s) for n, all_ in WRONG.items() for d, s in all_])
def test_what_is_no_cache_is_refused(name, dtype, shape):
    q = cache(table=True)
    q.struct()
    setattr(q, name, torch.zeros(shape, dtype=dtype))
    with pytest.raises(rk.RocketKVError, match=name) as e:
        q.struct()
    assert e.value.status == rk.INVALID_ARG
    with pytest.raises(rk.RocketKVError, match=name):
        rk.q_workspace_bytes(rk.OP_ATTEND, q)


@pytest.mark.parametrize("name", WRONG)
def test_what_lies_apart_is_refused(name):
    """Every other element of larger tensors."""
    q = cache(table=True)
    x = getattr(q, name)
    setattr(q, name, torch.zeros(x.shape[:-1] + (2 * x.shape[-1],), dtype=x.dtype)[..., ::2])
    with pytest.raises(rk.RocketKVError, match=name if name != "k_scales" else "k_codes|k_scales"):
        q.struct()


@pytest.mark.parametrize("fmt,width", [(rk.Q_E4M3, 128), (rk.Q_E2M1, 64)])
@pytest.mark.parametrize("table", [False, True])
def test_what_is_one_passes(fmt, width, table):
    q = cache(fmt, table)
    s = q.struct()
    assert (s.n_phys_pages, s.stride_page, s.stride_head, s.format) == (N, HEADS * PS, PS, fmt)
    for name in ("k_codes", "v_codes", "k_scales", "v_scales", "seq_lens"):
        assert getattr(s, name) == getattr(q, name).data_ptr()
    assert (s.block_table is None) == (not table)
    # any type of one byte, and pages and heads at any stride that all four share
    q.k_codes, q.v_codes = q.k_codes.view(torch.int8), q.v_codes.view(torch.float8_e4m3fn if fmt == rk.Q_E4M3 else torch.uint8)
    s = q.struct()
    assert (s.stride_page, s.stride_head) == (HEADS * PS, PS)
    wide = lambda w: torch.zeros((N, HEADS + 1, PS + 3, w), dtype=torch.uint8)[:, 1:, :PS]
    q.k_codes, q.v_codes, q.k_scales, q.v_scales = wide(width), wide(width), wide(4), wide(4)
    s = q.struct()
    assert (s.stride_page, s.stride_head) == ((HEADS + 1) * (PS + 3), PS + 3)


def test_lengths_that_are_missing_are_the_librarys_to_refuse():
    q = cache()
    q.seq_lens = None
    assert q.struct().seq_lens is None
    assert rk.q_workspace_bytes(rk.OP_ATTEND, q) > 0  # sizes need no lengths
    dst = rk.alloc_cache(BATCH, 8, HEADS, 128, PS, CAP, "cpu", v_layout=rk.V_TOKEN_MAJOR)
    assert rk.lib().rocketkv_restore(C.byref(q.struct()), C.byref(dst.struct()), None) == rk.INVALID_ARG
    assert "seq_lens" in rk.last_error()
