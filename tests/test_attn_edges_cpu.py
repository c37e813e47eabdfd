"""Refusals of the 8-bit cache operators that go by more than one argument, without a
GPU: what is refused and what is not is told apart by a later refusal."""
import numpy as np

from paper_2403_01876_amd import attn, dv
from tests.test_attn_cpu import (FAKE, INVALID, KEPT, POS, SCALE, TABLE, UNSUPPORTED, WEIGHT)


def pool(at, table, blocks=128, heads=1 << 16):
    """A paged cache of one-token blocks, wide enough that an eviction which keeps
    `blocks` tokens of each head is more than one call takes."""
    c = dv.Cache(dv.DV_PAGED, 1, heads, 16, 1, [FAKE + at], elem_bytes=1, block_size=1,
                 num_blocks=blocks, max_blocks=blocks, block_tables=[table])
    return attn.QuantCache(c, [SCALE + at], scale_block=1, weights=[WEIGHT + at],
                           positions=[POS + at])


def evict(src, dst, blocks=128):
    n = np.array([blocks], np.int32)
    return attn.dv_evict(src, 0, dst, 0, 0, 1, n, n, 0, KEPT, kept_stride=blocks, stream=0,
                         check=False)


def test_evict_between_pools_of_one_table():
    src = pool(0, TABLE)
    assert evict(src, pool(1 << 45, TABLE)) == UNSUPPORTED
    assert evict(src, pool(1 << 45, TABLE + 256)) == UNSUPPORTED  # tables that overlap in part
    # a table that the call would write is refused still
    for at in (FAKE, SCALE, WEIGHT, POS):
        assert evict(src, pool(1 << 45, at + 64)) == INVALID
        assert evict(pool(0, at + (1 << 45) + 64), pool(1 << 45, TABLE)) == INVALID
    assert evict(src, pool(0, TABLE + 4096)) == INVALID  # one pool, two tables
