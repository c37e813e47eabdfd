"""The 8-bit cache operators where numbers and places are out of the ordinary.

Tolerances are those of tests/test_gpu_attn.py (its run_attend is used).
"""
import numpy as np
import pytest

from tests.test_gpu_attn import make, run_attend

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
