"""Rows that one late key dominates: its weight is all there is, so the result is its value and nothing else."""
import pytest
import torch

import chunk_ref as ref
from paper_2502_14051_amd import rocketkv as rk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ps,token_major", [(16, False), (4, True)])
@pytest.mark.parametrize("lens,news,hq,hkv,spare", [([90], [20], 8, 2, 0), ([700, 300], [90, 3], 8, 2, 0), ([9000], [70], 8, 2, 0),
                                                    ([9000, 3000], [5, 2], 4, 1, 0), ([3000], [300], 64, 8, 37000), ([9000], [3], 4, 2, 140000)])
def test_the_value_of_the_key_that_counts(ps, token_major, lens, news, hq, hkv, spare):
    """One channel makes the logits.  Every 64th key has logit 0 and value 1, one late key a logit of 9 to 15.5 in powers of two
    (as much as sums take without following the maximum) and value 1, the others next to no weight and any value: weights
    may be rounded as they like, their mean is 1, and 1 is what a bf16 result has to be."""
    c = ref.Case(100, lens, news, hq, hkv, ps, token_major, shuffled=False, spare_pages=spare // ps)
    c.K.zero_()
    c.K[..., 5] = -32.0
    n = c.K.shape[2]
    c.K[:, :, ::64, 5] = 0.0
    c.V[:, :, ::64] = 1.0
    for b in range(len(lens)):
        late = (lens[b] - news[b]) * 3 // 4  # every row sees it
        late += 7 if late % 64 == 0 else 0
        c.K[b, :, late, 5], c.V[b, :, late] = 8.0, 1.0
    gen = torch.Generator().manual_seed(0)
    c.q.zero_()
    c.q[..., 5] = (9.0 + 6.5 * torch.rand(c.q.shape[:2], generator=gen)).to(torch.bfloat16).cuda() * 0.98046875
    layout = rk.V_TOKEN_MAJOR if token_major else rk.V_CHANNEL_MAJOR
    c.cache = rk.pack_cache(c.K, c.V, lens, hq, ps, pages_cap=c.cache.pages_cap, n_phys_pages=c.cache.k_pool.shape[0], v_layout=layout)
    out, lse = torch.empty_like(c.q), torch.empty((c.rows, hq), device="cuda")
    rk.chunk_attend(c.cache, c.chunk, c.q, out, lse, rk.alloc_workspace(rk.OP_CHUNK_ATTEND, c.cache, c.rows))
    assert n == max(lens) and (out == 1).all(), f"{int((out != 1).sum())} of {out.numel()}, from {float(out.min())} to {float(out.max())}"
    ref.check_attention(c, out, lse)
