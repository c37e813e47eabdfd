"""Rounding into the 8-bit cache: NaN of every kind takes no part in a block's scale."""
import numpy as np
import pytest
import torch

from paper_2403_01876_amd import attn, dv
from tests.test_gpu_attn import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,quiet,nans", [("f16", 0x7e00, [0x7c01, 0xfc01, 0x7dff, 0xffff]),
                                              ("bf16", 0x7fc0, [0x7f81, 0xff81, 0x7fbf, 0xffff])])
@pytest.mark.parametrize("kind,bs,D", [("dense", 16, 128), ("dense", 100, 64), ("paged", 16, 80),
                                       ("paged", 3, 16)])
def test_nan_of_every_kind_is_one(dtype, quiet, nans, kind, bs, D):
    """Scales are as with quiet NaN, wherever those stand, and so are codes but for NaN's sign."""
    rng = np.random.default_rng(bs)
    L, H, B, S = 1, 2, 3, 100
    lens = [100, 37, 64]
    n = L * 2 * H * D * sum(lens)
    x = torch.from_numpy(rng.normal(size=n) * np.exp2(rng.integers(-9, 9, n)))
    x = x.to(torch.float16 if dtype == "f16" else torch.bfloat16)
    for share in (0.001, 0.05, 0.5):
        at = rng.random(n) < share
        wires = []
        for bits in (np.array([quiet]), np.array(nans)):
            y = x.view(torch.int16).numpy().view(np.uint16).copy()
            y[at] = rng.choice(bits, at.sum())
            wires.append(torch.from_numpy(y.view(np.int16)).view(x.dtype).cuda())
        got = []
        for wire in wires:
            d, t = make(kind, L, H, D, B, S, bs, 5).device(dv, attn)
            attn.dv_quant_in(d, 0, 0, L, None, lens, wire, wire.numel() * 2,
                             attn.DV_F16 if dtype == "f16" else attn.DV_BF16)
            torch.cuda.synchronize()
            got.append((t["codes"], t["scale"]))
        assert torch.equal(got[0][1], got[1][1])
        a, b = (c.int() for c, _ in got)
        assert bool(((a == b) | ((a & 127 == 127) & (b & 127 == 127))).all())
