"""The 8-bit cache operators where numbers and places are out of the ordinary.

Tolerances are those of tests/test_gpu_attn.py (its run_attend is used).
"""
import numpy as np
import pytest
import torch

from paper_2403_01876_amd import attn, dv
from tests import attn_ref as ref
from tests.test_gpu_attn import make, run_attend, tie_weights

pytestmark = pytest.mark.gpu


# ---- blocks that nobody maps ----------------------------------------------------------------


def spoil_unowned(c, scale):
    """Frees pool block 0 and fills the blocks that no table names with NaN codes and
    this scale: what memory may hold that nothing was ever written to."""
    owned = np.unique(c.table[(c.table >= 0) & (c.table < c.nblocks)])
    if 0 in owned:
        c.table[c.table == 0] = np.setdiff1d(np.arange(c.nblocks), owned)[-1]
    unowned = np.setdiff1d(np.arange(c.nblocks), c.table)
    assert 0 in unowned
    c.codes[:, :, unowned] = 127
    c.scale[:, :, unowned] = scale


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens", [1, 6, 80])
@pytest.mark.parametrize("scale", [np.nan, np.inf])
def test_attend_unwritten_scales_of_unowned_blocks(dtype, tokens, scale):
    c = make("paged", 1, 2, 64, 4, 160, 8, 21, companions=True,
             holes=[(0, 3, -1), (1, 0, 10 ** 6), (1, 1, -7), (3, 0, -1)])
    spoil_unowned(c, scale)
    lens = [150, 16, 97, 8]
    y = run_attend(c, [min(tokens, n) for n in lens], lens, 2, dtype, decay=0.0)
    assert np.isfinite(y).all()


@pytest.mark.parametrize("scale", [np.nan, np.inf])
@pytest.mark.parametrize("D,bs", [(32, 8), (128, 64)])
@pytest.mark.parametrize("place", ["new", "same"])
def test_evict_unwritten_scales_of_unowned_blocks(scale, D, bs, place):
    """Tokens without a block count as zeros (blocks that a wave holds, and larger)."""
    rng = np.random.default_rng(4)
    c = make("paged", 1, 2, D, 2, 8 * bs, bs, 6, companions=True, holes=[(0, 2, -1), (1, 0, 999)])
    spoil_unowned(c, scale)
    tie_weights(c, rng)
    d = c if place == "same" else make("paged", 1, 2, D, 2, 8 * bs, bs, 7, companions=True)
    (qc, tc) = c.device(dv, attn)
    (qd, td) = (qc, tc) if d is c else d.device(dv, attn)
    length, keep = [8 * bs, 6 * bs + 3], [5 * bs, 3 * bs + 1]
    kept = torch.full((1, 2, 2, 5 * bs), -1, dtype=torch.int32, device="cuda")
    attn.dv_evict(qc, 0, qd, 0, 0, 1, length, keep, 4, kept)
    assert np.array_equal(kept.cpu().numpy(), ref.evict(c, d, 0, 1, length, keep, 4, 5 * bs))
    assert np.array_equal(td["scale"].cpu().numpy(), d.scale, equal_nan=True)
    got = td["codes"].cpu().numpy()
    assert ref.same_codes(got, d.codes), f"{int((got != d.codes).sum())} codes differ"
