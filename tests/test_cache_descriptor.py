"""What the binding passes on of a cache that lacks a part (no GPU)."""
import dataclasses
import os

import pytest
import torch

from paper_2502_14051_amd import rocketkv as rk


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(rk.LIB_PATH):
        from paper_2502_14051_amd import build
        build.build()


def test_lengths_that_are_missing_are_the_librarys_to_refuse():
    cache = dataclasses.replace(rk.alloc_cache(1, 4, 2, 128, 16, 8, "cpu"), seq_lens=None)
    assert cache.struct().seq_lens is None
    assert rk.workspace_bytes(rk.OP_DENSE_DECODE, cache) > 0  # sizes need no lengths
    kmax, kmin = rk.alloc_summaries(cache)
    with pytest.raises(rk.RocketKVError, match="seq_lens") as e:
        rk.build_page_summaries(cache, kmax, kmin, stream=1)
    assert e.value.status == rk.INVALID_ARG
