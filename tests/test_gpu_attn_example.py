"""The example that runs the 8-bit cache operators together."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load():
    spec = importlib.util.spec_from_file_location(
        "evicting_decode", os.path.join(ROOT, "examples", "evicting_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_evicting_decode():
    r = load().main()
    assert r["evictions"] >= 1
    assert (r["length"] <= 97).all() and (r["seen"] == np.array([114, 85, 152])).all()
    pos = r["positions"].cpu().numpy()
    for b, (n, s) in enumerate(zip(r["length"], r["seen"])):
        p = pos[:, b, :, :n]
        # strictly increasing, up to the newest token; what was evicted is missing
        assert (np.diff(p, axis=-1) > 0).all() and (p[..., -1] == s - 1).all()
        assert n == s or (p[..., 0] >= 0).all()
    assert r["replica_bytes"] < r["full_bytes"] // 2


def test_within_the_budget_nothing_is_lost_but_bits():
    """A budget that is never passed: what is left is the rounding to 8 bits, of keys
    and of values (half a step of 2^-4 each, so a few hundredths in all)."""
    r = load().main(budget=200)
    assert r["evictions"] == 0 and (r["length"] == r["seen"]).all()
    assert r["worst"] < 0.15


@pytest.mark.parametrize("heads,layers", [(4, 2), (8, 1)])
def test_the_replica_is_whole(heads, layers):
    """Codes and scales as streamed into other pages give the same attention, bit for bit."""
    r = load().main(heads=heads, layers=layers)
    assert r["replica_answers_the_same"]
    n = r["length"].astype(np.int64)
    codes = int(n.sum()) * layers * 2 * heads * 64
    assert r["replica_bytes"] == codes + int((-(-n // 16)).sum()) * layers * 2 * heads * 4


def test_prompts_of_any_length():
    r = load().main(layers=1, heads=8, group=4, prompts=(2500,) * 6, steps=2, budget=2501, keep=900)
    assert r["evictions"] == 1 and (r["length"] == 900).all() and r["replica_answers_the_same"]
