"""Refusals of the 8-bit cache operators that go by more than one argument, without a
GPU: what is refused and what is not is told apart by a later refusal."""
import os
import re

import numpy as np
import pytest
import torch

from paper_2403_01876_amd import attn, dv
from tests.test_attn_cpu import (FAKE, INVALID, KEPT, POS, SCALE, SPACE, TABLE, UNSUPPORTED, WEIGHT,
                                 ROOT, attend, cache)


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


@pytest.mark.parametrize("seed", range(40))
def test_attend_rows_of_the_result_that_share_elements(seed):
    """Refused exactly where two rows do, whichever of the strides is the larger."""
    r = np.random.default_rng(seed)
    D, c = 64, cache(S=64)
    seen = set()
    for _ in range(60):
        tokens, heads = int(r.integers(1, 7)), 2 * int(r.integers(1, 5))
        token, head = (8 * int(r.choice([r.integers(0, 9), r.integers(8, 90)])) for _ in range(2))
        starts = np.sort((np.arange(tokens)[:, None] * token + np.arange(heads) * head).ravel())
        shared = bool((np.diff(starts) < D).any())
        got = attend(c, q_len=(tokens, 0, 0), kv_len=(9, 0, 0), q_heads=heads, rows=tokens,
                     q_token=heads * D, out_token=token, out_head=head, weigh=1, workspace_bytes=0)
        assert got == (INVALID if shared else SPACE), (tokens, heads, token, head)
        seen.add((shared, token < head))
    assert len(seen) == 4


def test_inline_assembly_names_the_registers_it_writes():
    """A copy to LDS sets m0, which the compiler may use for itself."""
    text = open(os.path.join(ROOT, "paper_2403_01876_amd", "csrc", "dv_attend.hip")).read()
    blocks = re.findall(r"asm volatile\((.*?)\);", text, re.S)
    writes = [b for b in blocks if re.search(r"\bm0,", b)]
    assert len(writes) == 3
    for b in writes:
        assert re.search(r':[^:]*"m0"[^:]*$', b), b


def test_a_workspace_with_gaps_is_refused():
    """Its bytes are counted as one range."""
    c = dv.Cache(dv.DV_DENSE, 1, 2, 64, 1, [FAKE], elem_bytes=1, max_seq=40)
    qc = attn.QuantCache(c, [SCALE], scale_block=16)
    q = torch.zeros((1, 4, 64), dtype=torch.float16)
    for ws in (torch.zeros(64, dtype=torch.uint8)[::2], torch.zeros(1).expand(64)):
        with pytest.raises(ValueError, match="workspace must be contiguous"):
            attn.dv_attend(qc, 0, 0, [1], [4], q, q.clone(), 1.0, workspace=ws)
