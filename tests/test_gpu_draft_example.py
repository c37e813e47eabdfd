"""A whole decode loop with drafts: the example runs, more than one token a step is accepted,
and cache, replica and logits are those of the text that it wrote."""
import os
import sys

import numpy as np
import pytest
import torch

from paper_2403_01876_amd import attn, draft

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block,group,temperature", [(16, 2, 0.5), (8, 1, 0.0), (3, 4, 1.0)])
def test_the_example_writes_the_text_its_cache_holds(block, group, temperature):
    import drafted_decode
    prompts = (45, 9, 70)
    r = drafted_decode.main(prompts=prompts, steps=10, block=block, group=group,
                            temperature=temperature)
    added = np.array(r["added"])
    assert added.min() >= 1 and added.max() > 1
    # each step adds the accepted drafts after the root, and one token more
    assert [len(x) for x in r["text"]] == (np.array(prompts) + added.sum(0)).tolist()
    assert r["length"].tolist() == [len(x) - 1 for x in r["text"]]
    # Keys and values are within 2^-4 of themselves; a cache of other tokens' would be off by
    # as much as the logits themselves.
    assert r["worst"] < 2.0 ** -4
    # The replica took each token once, when it was added; codes may have been rounded again
    # since, to a larger scale: by half a step of what 448 of it are, 2^-10 of the largest.
    L, H, D, n = 2, 4, 64, r["length"]
    wire = torch.empty(L * 2 * H * D * int(n.sum()), dtype=torch.float16, device="cuda")
    draft.dv_quant_out(r["cache"], 0, 0, L, None, n, wire, wire.numel() * 2, attn.DV_F16)
    wire = wire.view(L, 2, -1, D)
    first = 0
    for b, m in enumerate(n.tolist()):
        now = wire[:, :, first * H:(first + m) * H].reshape(L, 2, H, m, D)
        first += m
        was = r["mirror"][:, :, b, :, :m]
        assert float((now - was).abs().max()) <= float(was.abs().max()) * 2.0 ** -10 * 4
