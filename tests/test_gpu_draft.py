"""The operators over drafted tokens on the GPU against their plain 64-bit forms.

Attention has the error bounds of dv_attend, whose kernels it shares (test_gpu_attn).
Verification returns whole numbers, which have to be equal: inputs whose closest
decision lies within 1e-9 of its border are not used (sums of 1e5 terms in 64 bits are
exact to 1e-11).  Kept tokens are compared code for code and tokens read back bit for
bit.
"""
import numpy as np
import pytest
import torch

from paper_2403_01876_amd import attn, draft, dv
from tests import attn_ref as ref
from tests import draft_ref as dref
from tests.test_gpu_attn import HALF, PROB, check_state, make

pytestmark = pytest.mark.gpu


# ---- dv_attend_tree -------------------------------------------------------------------------


def run_tree(c, q_len, kv_len, group, dtype, *, shape="tree", broken=0.0, slopes=False,
             strided=False, layer=None, seed=0, parent=None):
    rng = np.random.default_rng(seed + 177)
    layer = c.L - 1 if layer is None else layer
    n, hq = int(np.sum(q_len)), c.H * group
    if parent is None:
        parent = dref.trees(q_len, rng, shape, broken)
    x = torch.from_numpy(rng.normal(size=(n, hq, c.D))).to(ref.TDTYPE[dtype])
    q = x.cuda()
    out = torch.full((n, hq, c.D), 7.0, dtype=q.dtype, device="cuda")
    if strided:  # heads outermost, padded rows
        store = torch.empty((hq, n + 3, c.D + 8), dtype=q.dtype, device="cuda")
        store[:, :n, :c.D] = q.transpose(0, 1)
        q = store[:, :n, :c.D].transpose(0, 1)
        out = torch.full((hq, n + 1, c.D + 16), 7.0, dtype=q.dtype,
                         device="cuda")[:, :n, :c.D].transpose(0, 1)
    sl = (2.0 ** -rng.uniform(0, 6, hq)).astype(np.float32) if slopes else None
    d, t = c.device(dv, attn)
    before = {k: v.clone() for k, v in t.items() if v is not None}
    ls = torch.full((n, hq), 3.0, device="cuda")
    nb = attn.dv_attend_bytes(d, q_len, kv_len, q)
    ws = torch.full((nb + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    scale = float(np.float32(1.0 / np.sqrt(c.D)))
    draft.dv_attend_tree(d, 0, layer, q_len, kv_len, torch.from_numpy(parent).cuda(), q, out, scale,
                         slopes=None if sl is None else torch.from_numpy(sl).cuda(), lse=ls,
                         workspace=ws[:nb])
    torch.cuda.synchronize()
    assert bool((ws[nb:] == 0xA5).all()), "wrote past the workspace"
    for k, v in before.items():
        assert torch.equal(v.view(torch.uint8), t[k].view(torch.uint8)), f"{k} changed"
    want, mass, wlse = dref.attend_tree(c, layer, q_len, kv_len, parent, x.double().numpy(), scale,
                                        None if sl is None else sl.astype(np.float64))
    y = out.double().cpu().numpy()
    nan = np.isnan(want)
    assert np.array_equal(nan, np.isnan(y)), "NaN in other places"
    rows = max([int(m) * group for m in q_len], default=0)
    many = rows > (64 if c.D <= 128 else 32)
    tol = HALF[dtype] * np.abs(want) + (PROB + (HALF[dtype] if many else 0)) * mass + 2.0 ** -24
    err = np.abs(y - want)
    assert not (err > tol)[~nan].any(), \
        f"off by {np.nanmax(err / tol):.2f} tolerances at {np.argwhere(err > tol)[:3].tolist()}"
    z = ls.double().cpu().numpy()
    dead = np.isneginf(wlse)
    assert np.array_equal(dead, np.isneginf(z)) and np.array_equal(np.isnan(wlse), np.isnan(z))
    live = np.isfinite(wlse)
    assert np.all(np.abs(z[live] - wlse[live]) <= 1e-5 * np.maximum(1, np.abs(wlse[live])))
    return y


LENS = [1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 300]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("kind,bs", [("dense", 16), ("dense", 7), ("paged", 16), ("paged", 3)])
@pytest.mark.parametrize("D,group,most", [(64, 1, 1), (64, 1, 20), (128, 1, 64), (128, 8, 8),
                                          (128, 8, 64), (64, 4, 128), (256, 2, 16), (256, 1, 70)])
def test_tree_of_every_path(dtype, kind, bs, D, group, most):
    """Few rows (1, 2 and 4 tiles of 16) and many; trees that begin at every place of a step,
    some of which are all there is."""
    c = make(kind, 2, 2, D, len(LENS), 300, bs, D + bs + most)
    run_tree(c, [min(most, n) for n in LENS], LENS, group, dtype, seed=most)


@pytest.mark.parametrize("shape", ["chain", "star", "roots", "tree"])
@pytest.mark.parametrize("group,most", [(1, 9), (1, 33), (2, 31), (3, 60), (1, 128), (8, 100)])
def test_tree_shapes_with_bias_and_positions(shape, group, most):
    c = make("dense", 2, 2, 128, 5, 420, 16, group * 100 + most, companions=True)
    lens = [420, 5, 131, 64, 300]
    q_len = [min(most, n) for n in lens]
    q_len[3] = 0
    run_tree(c, q_len, lens, group, "f16" if group % 2 else "bf16", shape=shape, slopes=True,
             strided=True, layer=0)
    c = make("paged", 1, 1, 64, 2, 700, 16, most)  # slots for positions
    run_tree(c, [most, min(most, 77)], [700, 77], group, "bf16", shape=shape, slopes=True)


@pytest.mark.parametrize("group,most", [(1, 12), (2, 32), (4, 100), (16, 128)])
@pytest.mark.parametrize("slopes", [False, True])
def test_drafts_that_are_not_there(group, most, slopes):
    """Parents out of range, and drafts that descend from them: rows that see nothing."""
    c = make("paged", 1, 2, 64, 4, 200, 16, most, companions=slopes)
    lens = [200, 150, most, 129]
    q_len = [min(most, n) for n in lens]
    y = run_tree(c, q_len, lens, group, "f16", broken=0.3, slopes=slopes)
    assert (np.abs(y).max((1, 2)) == 0).any()
    parent = np.concatenate([np.full(m, -2 - i) for i, m in enumerate(q_len)]).astype(np.int32)
    assert not run_tree(c, q_len, lens, group, "f16", parent=parent).any()


@pytest.mark.parametrize("D", [16, 48, 80, 112, 144, 208])
@pytest.mark.parametrize("most", [5, 70])
def test_tree_odd_head_dims(D, most):
    c = make("paged", 1, 2, D, 3, 200, 16, D, companions=True)
    lens = [200, 77, 5]
    run_tree(c, [min(most, n) for n in lens], lens, 1 + D % 3, "f16" if D % 32 else "bf16",
             slopes=D % 48 == 0)


@pytest.mark.parametrize("group,most", [(1, 14), (8, 25)])
def test_tree_long_axis_split(group, most):
    c = make("paged", 1, 1, 128, 2, 9000, 16, 8)
    run_tree(c, [most, most], [9000, 4133], group, "bf16")


@pytest.mark.parametrize("group,most", [(1, 20), (4, 40)])
def test_tree_unmapped_blocks(group, most):
    holes = [(0, 0, -1), (0, 3, 1 << 20), (1, 6, -9), (2, 0, -1), (2, 1, -1), (2, 2, -1), (2, 3, -1)]
    c = make("paged", 1, 2, 64, 3, 112, 16, 31, holes=holes)
    run_tree(c, [most, most, min(most, 40)], [112, 110, 40], group, "f16")


@pytest.mark.parametrize("group,most", [(1, 20), (4, 40)])
def test_tree_nan_codes_stay_with_who_sees_them(group, most):
    """NaN among the drafts' own values reaches their descendants only, and one before the
    drafts reaches all that are there."""
    for slot in (90, 117, 139):
        c = make("dense", 1, 1, 64, 2, 140, 16, 3)
        c.codes[0, 1, 0, 0, slot, 5] = 0x7f
        c.codes[0, 1, 1, 0, slot, 7] = 0xff
        run_tree(c, [most, most], [140, 140], group, "f16", broken=0.15, seed=slot)
    c = make("dense", 1, 1, 64, 1, 140, 16, 3)
    c.codes[0, 0, 0, 0, 125] = 0x7f  # a key
    run_tree(c, [most], [140], group, "bf16")


def test_tree_of_many_sequences():
    rng = np.random.default_rng(4)
    kv = rng.integers(0, 60, 400)
    q_len = np.minimum(kv, rng.integers(0, 9, 400))
    c = make("dense", 1, 2, 32, 400, 60, 8, 12)
    run_tree(c, q_len.tolist(), kv.tolist(), 2, "f16")


def test_a_chain_is_what_dv_attend_computes():
    """Drafts in a chain are consecutive queries: the same bits."""
    c = make("paged", 1, 2, 128, 3, 500, 16, 2)
    d, _ = c.device(dv, attn)
    for group, most in ((1, 12), (8, 30)):
        q_len, kv = [most] * 3, [500, 33, 260]
        q = torch.randn((3 * most, 2 * group, 128), device="cuda").half()
        a, b = torch.empty_like(q), torch.empty_like(q)
        ws = torch.empty(attn.dv_attend_bytes(d, q_len, kv, q), dtype=torch.uint8, device="cuda")
        parent = torch.from_numpy(dref.trees(q_len, None, "chain")).cuda()
        draft.dv_attend_tree(d, 0, 0, q_len, kv, parent, q, a, 0.1, workspace=ws)
        attn.dv_attend(d, 0, 0, q_len, kv, q, b, 0.1, workspace=ws)
        assert torch.equal(a, b)


# ---- dv_verify ------------------------------------------------------------------------------


def logits_of(rows, V, rng, dtype, sharp=2.0):
    x = rng.normal(size=(rows, V)) * sharp - 0.8 * np.log1p(rng.permutation(V))
    return torch.from_numpy(x).to(dtype)


def run_verify(q_len, V, dtype, rng, *, shape="tree", drawn=False, temperature=None, pad=0,
               logits=None, token=None, uniform=None, parent=None, q=None, broken=0.0, border=1e-9):
    rows, B = int(np.sum(q_len)), len(q_len)
    parent = dref.trees(q_len, rng, shape, broken) if parent is None else np.asarray(parent, np.int32)
    x = logits_of(rows, V, rng, dtype) if logits is None else logits
    first = np.repeat(np.cumsum(q_len) - q_len, q_len)
    up = first + np.clip(parent, 0, None).clip(max=np.maximum(np.repeat(q_len, q_len) - 1, 0))
    near = x.double().numpy()
    if drawn and q is None:
        y = near + rng.normal(size=near.shape)
        q = np.exp(np.nan_to_num(y - y.max(-1, keepdims=True), nan=-99, neginf=-99))
        q = (q / q.sum(-1, keepdims=True)).astype(np.float32)
    if token is None:  # mostly likely ones, so that some are accepted
        best = np.argsort(-near, axis=-1, kind="stable")[:, :6]
        token = best[up, rng.integers(0, best.shape[1], rows)]
        token = np.where(rng.random(rows) < 0.1, rng.integers(0, V, rows), token)
    u = rng.random(rows).astype(np.float32) if uniform is None else np.asarray(uniform, np.float32)
    want = dref.verify(q_len, parent, token, near, u, temperature, q if drawn else None)
    if want[3] < border:
        pytest.skip("a decision at its border")
    store = torch.full((rows + 2, V + pad), 50.0, dtype=dtype)
    store[:rows, :V] = x
    dq = None
    if drawn:
        dq = torch.full((rows + 1, V + 3), 9.0)
        dq[:rows, :V] = torch.from_numpy(q)
        dq = dq.cuda()[:rows, :V]
    dl = store.cuda()[:rows, :V]
    ints = [torch.from_numpy(np.asarray(a, np.int32)).cuda() for a in (parent, token)]
    path = torch.full((rows + 2,), -7, dtype=torch.int32, device="cuda")
    count, follow = (torch.full((B,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    nb = draft.dv_verify_bytes(q_len, dl, drawn)
    ws = torch.full((nb + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    for _ in range(2):  # nothing carries over
        draft.dv_verify(q_len, ints[0], ints[1], dl, torch.from_numpy(u).cuda(), path, count, follow,
                        temperature=temperature, drawn=dq, workspace=ws[:nb])
    torch.cuda.synchronize()
    assert bool((ws[nb:] == 0xA5).all()), "wrote past the workspace"
    path, count, follow = path.cpu().numpy(), count.cpu().numpy(), follow.cpu().numpy()
    assert np.array_equal(count, want[1]), (count, want[1])
    assert np.array_equal(path[:rows], np.where(want[0] < 0, -7, want[0])) and (path[rows:] == -7).all()
    assert np.array_equal(follow, np.where(want[2] == -2, -7, want[2])), (follow, want[2])
    return want


TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("V", [1, 2, 7, 100, 4089, 4096, 4097, 20001, 131072])
def test_verify_sizes(dtype, drawn, V):
    rng = np.random.default_rng(V)
    q_len = [5, 1, 0, 9] if V > 10000 else [12, 1, 0, 30, 3, 2, 128]
    for k, shape in enumerate(("tree", "chain")):
        run_verify(q_len, V, TYPES[dtype], rng, shape=shape, drawn=drawn, pad=k * 5,
                   temperature=np.array([0.7, 1.3, 1.0, 0.0, 1e-3, 40.0, 1.0][:len(q_len)], np.float32))


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("seed", range(6))
def test_verify_wide_trees(drawn, seed):
    """Many guesses of one token: each is tried against what the ones before left."""
    rng = np.random.default_rng(seed)
    q_len = rng.integers(0, 129, 20)
    run_verify(q_len, 300, torch.float32, rng, shape="star" if seed % 2 else "tree",
               drawn=drawn, temperature=np.full(20, 1.5, np.float32), broken=0.1 * (seed > 3))


@pytest.mark.parametrize("shape", ["chain", "tree"])
def test_verify_long_paths(shape):
    """The drafts that the target is nearly sure of: whole chains are accepted."""
    rng = np.random.default_rng(11)
    q_len = [128, 64, 65, 1, 17]
    rows = sum(q_len)
    x = torch.zeros((rows, 5000), dtype=torch.float32)
    token = rng.integers(0, 5000, rows)
    parent = dref.trees(q_len, rng, shape)
    first = np.repeat(np.cumsum(q_len) - q_len, q_len)
    for i in range(rows):
        if parent[i] >= 0:
            x[first[i] + parent[i], token[i]] = 17.0
    got = run_verify(q_len, 5000, torch.float32, rng, shape=shape, logits=x, token=token,
                     parent=parent)
    if shape == "chain":
        assert got[1][0] > 64


def test_verify_greedy_takes_the_lowest_of_equal_logits():
    rng = np.random.default_rng(0)
    x = torch.zeros((4, 9000), dtype=torch.bfloat16)
    x[:, [8000, 4100, 77]] = 3.0
    got = run_verify([4], 9000, torch.bfloat16, rng, shape="chain", logits=x, token=[0, 77, 77, 4100],
                     temperature=np.zeros(1, np.float32))
    assert got[1].tolist() == [3] and got[2].tolist() == [77]


@pytest.mark.parametrize("dtype", list(TYPES))
def test_verify_next_to_the_border(dtype):
    """Random numbers as near to the probability that decides as 32 bits come, on either side:
    about 1e-8 of it, where sums in 32 bits would not tell.  (5000 shares, each to 3e-13, and
    as many roundings of 1e-16 stay below 1e-12.)"""
    rng = np.random.default_rng(7)
    V = 5000
    for k in range(12):
        x = logits_of(6, V, rng, TYPES[dtype])
        p = dref.target(x[0].double().numpy(), 1.0)
        token = np.argsort(-p)[:6]
        r, u = p.copy(), np.full(6, 0.37, np.float32)
        for i in range(1, 6):  # each rejected at its border, the last accepted
            u[i] = np.float32(r[token[i]])
            if i < 5 and float(u[i]) < r[token[i]]:
                u[i] = np.nextafter(u[i], np.float32(1))
            if i == 5 and float(u[i]) >= r[token[i]]:
                u[i] = np.nextafter(u[i], np.float32(0))
            r[token[i]] = 0
            r /= r.sum()
        got = run_verify([6], V, TYPES[dtype], rng, shape="star", logits=x, token=token, uniform=u,
                         temperature=np.ones(1, np.float32), border=1e-12)
        assert got[0].tolist()[:2] == [0, 5]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [1e4, 1e7, 1e10, 1e30, 3e38])
def test_verify_logits_of_any_size(dtype, size):
    """Offsets and spreads that 32 bits round: a few logits next to the largest share it."""
    rng = np.random.default_rng(8)
    for shift in (size, -size, 0.0):
        x = torch.from_numpy(rng.normal(size=(6, 4500)) * size * 1e-3 + shift).clamp(-3.3e38, 3.3e38)
        x = x.to(TYPES[dtype])
        top = x.max(-1, keepdim=True).values
        x[:, 7:4000:400] = top                         # ten equal ones
        x[:, 9] = torch.nextafter(top[:, 0].float(), torch.tensor(-np.inf)).to(x.dtype)
        token = rng.choice([7, 9, 407, 3], 6)
        for T in (0.7, 1e-3, size * 1e-4):
            run_verify([6], 4500, TYPES[dtype], rng, shape="star", logits=x, token=token,
                       temperature=np.full(1, T, np.float32), border=1e-11)


def test_verify_special_logits():
    """Infinities, NaN, rows without any probability; greedy and not."""
    rng = np.random.default_rng(1)
    V, inf, nan = 5000, np.inf, np.nan
    for T in (0.0, 0.8):
        t = np.full(1, T, np.float32)
        for fill, at in (({3: inf, 4500: inf}, 3), ({10: nan, 11: inf}, 11), ({0: nan}, None)):
            x = logits_of(3, V, rng, torch.float32)
            for k, v in fill.items():
                x[:, k] = v
            run_verify([3], V, torch.float32, rng, shape="chain", logits=x, temperature=t,
                       token=[0, at or 5, 4500])
        for fill in (-inf, nan):
            x = torch.full((3, V), fill)
            got = run_verify([3], V, torch.float32, rng, shape="star", logits=x, temperature=t,
                             token=[0, 4, 5])
            assert got[2].tolist() == [-1] and got[1].tolist() == [1]
            x[0, 4321] = 0.5  # one token has it all; what follows it has nothing
            got = run_verify([3], V, torch.float32, rng, shape="chain", logits=x, temperature=t,
                             token=[0, 4321, 5])
            assert got[1].tolist() == [2] and got[2].tolist() == [-1]
            got = run_verify([3], V, torch.float32, rng, shape="chain", logits=x, temperature=t,
                             token=[0, 4320, 5])
            assert got[1].tolist() == [1] and got[2].tolist() == [4321]


@pytest.mark.parametrize("drawn", [False, True])
def test_verify_special_chances_and_tokens(drawn):
    rng = np.random.default_rng(2)
    V = 6000
    for u0 in (0.0, 1.0, 2.0, -1.0, np.nan, 1 - 2.0 ** -24):
        for u in (0.0, np.nan, 1.0, 0.5):
            x = logits_of(5, V, rng, torch.float32)
            run_verify([5], V, torch.float32, rng, shape="star", logits=x, drawn=drawn,
                       uniform=[u0, u, u, u, u], token=[0, 17, -1, V, V - 1])
    # what drafts were drawn from covers the target, or is no distribution at all
    x = logits_of(4, V, rng, torch.float32)
    p = np.stack([dref.target(r, 1.0) for r in x.double().numpy()])
    for q in (np.full((4, V), 2.0), np.zeros((4, V)), np.full((4, V), np.nan), -p):
        run_verify([4], V, torch.float32, rng, shape="star", logits=x, drawn=True,
                   q=q.astype(np.float32), token=[0, 5, 5, 9], uniform=[0.4, 0.9, 0.9, 0.9])


def test_verify_of_many_sequences_and_of_none():
    rng = np.random.default_rng(5)
    q_len = rng.integers(0, 5, 450)
    run_verify(q_len, 60, torch.float16, rng)
    count = torch.full((3,), -7, dtype=torch.int32, device="cuda")
    z, f = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, device="cuda")
    draft.dv_verify([0, 0, 0], z, z, torch.zeros((0, 50), device="cuda"), f, z, count, count.clone(),
                    workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))
    assert count.tolist() == [0, 0, 0]


# ---- dv_keep_path ---------------------------------------------------------------------------


def run_keep(c, l0, l1, q_len, kv_len, path, count):
    d, t = c.device(dv, attn)
    p, n = (torch.from_numpy(np.asarray(x, np.int32)).cuda() for x in (path, count))
    draft.dv_keep_path(d, 0, l0, l1, q_len, kv_len, p, n)
    torch.cuda.synchronize()
    dref.keep_path(c, l0, l1, q_len, kv_len, np.asarray(path), np.asarray(count))
    check_state(c, t, "keep")


def paths(q_len, rng, most=200):
    path, count = [], []
    for n in q_len:
        k = int(rng.integers(0, min(n, most) + 1))
        path += sorted(rng.permutation(n)[:k].tolist()) + [-1] * (n - k)
        count.append(k)
    return path, count


@pytest.mark.parametrize("kind", ["dense", "paged"])
@pytest.mark.parametrize("D,bs", [(16, 1), (48, 5), (64, 16), (80, 8), (128, 16), (128, 64),
                                  (256, 16), (256, 100), (128, 1000)])
def test_keep_path(kind, D, bs):
    rng = np.random.default_rng(D + bs)
    for most in (3, 64, 128):
        c = make(kind, 3, 3, D, 6, 300, min(bs, 300) if kind == "paged" else bs, D + bs,
                 companions=True)
        lens = [300, 129, most, 0, 177, 1]
        q_len = [min(most, n) for n in lens]
        run_keep(c, 0, 3, q_len, lens, *paths(q_len, rng))
        run_keep(c, 1, 2, q_len, lens, *paths(q_len, rng, 5))


def test_keep_path_entries_that_end_it():
    rng = np.random.default_rng(1)
    for path, count in (([0, 3, 3, 4, 5, 6], 6), ([0, 3, 2, 4, 5, 6], 6), ([2, 9, 3, 4, 5, 6], 6),
                        ([-1, 0, 1, 2, 3, 4], 6), ([0, 1, 5, -1, -1, -1], 1 << 30),
                        ([0, 1, 2, 3, 4, 5], 6), ([0, 2, 4, 5, -1, -1], -5), ([5, 0, 0, 0, 0, 0], 1),
                        ([1 << 30] * 6, 6)):
        c = make("dense", 1, 2, 64, 2, 64, 16, int(rng.integers(99)), companions=True)
        run_keep(c, 0, 1, [6, 6], [64, 21], path * 2, [count] * 2)


def test_keep_path_unmapped_and_special():
    holes = [(0, 4, -1), (0, 6, 1000), (1, 2, -5)]
    c = make("paged", 1, 2, 64, 2, 64, 8, 4, holes=holes)
    run_keep(c, 0, 1, [40, 40], [64, 60], [0, 3, 9, 17, 18, 30] + [-1] * 34 + [2, 5, 30] + [-1] * 37,
             [6, 3])
    # NaN, zeros under the largest and the smallest scale, scales far apart
    c = make("dense", 1, 1, 16, 1, 64, 4, 4)
    c.scale[0, :, 0, 0, :] = np.ldexp(1.0, [-64, 100, -64, 0, 40, -30, 7, 8, 100, -64, 0, 0, 1, 2, 3, 4])
    c.codes[0, 0, 0, 0, 37] = 0x7f
    c.codes[0, 0, 0, 0, 33:36] = 0
    c.codes[0, 1, 0, 0, 32:36] = 0x80
    run_keep(c, 0, 1, [40], [64], [9, 10, 13, 16, 20, 33, 39] + [-1] * 33, [7])


def test_keep_path_of_many_sequences():
    rng = np.random.default_rng(6)
    kv = rng.integers(0, 40, 450)
    q_len = np.minimum(kv, rng.integers(0, 12, 450))
    c = make("dense", 2, 1, 16, 450, 40, 4, 5, companions=True)
    run_keep(c, 0, 2, q_len.tolist(), kv.tolist(), *paths(q_len, rng))


# ---- dv_quant_out ---------------------------------------------------------------------------


def run_out(c, l0, l1, t0, t1, dtype):
    d, t = c.device(dv, attn)
    x, there = dref.quant_out(c, l0, l1, t0, t1)
    wire = torch.full((l1 - l0, 2, x.shape[2], c.D), 7.0, dtype=ref.TDTYPE[dtype], device="cuda")
    guard = torch.full((wire.numel() + 64,), 7.0, dtype=wire.dtype, device="cuda")
    n = draft.dv_quant_out(d, 0, l0, l1, t0, t1, guard, wire.numel() * 2,
                           attn.DV_F16 if dtype == "f16" else attn.DV_BF16)
    assert n == wire.numel() * 2
    got = guard[:wire.numel()].view(wire.shape)
    top = dref.LARGEST[dtype]
    want = torch.from_numpy(np.clip(x, -top, top))
    want = want.to(ref.TDTYPE[dtype]) if dtype == "bf16" else \
        torch.from_numpy(want.numpy().astype(np.float16))
    want[:, :, ~torch.from_numpy(there)] = 7.0
    got = got.cpu()
    assert torch.equal(got.isnan(), want.isnan())
    same = (got.view(torch.int16) == want.view(torch.int16)) | want.isnan()
    assert bool(same.all()), int((~same).sum())
    assert bool((guard[wire.numel():] == 7.0).all())


@pytest.mark.parametrize("kind", ["dense", "paged"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D,bs", [(16, 1), (48, 5), (64, 16), (80, 8), (128, 16), (128, 64),
                                  (256, 40)])
def test_quant_out(kind, dtype, D, bs):
    c = make(kind, 3, 3, D, 4, 150, bs, D + bs)
    run_out(c, 0, 3, [0, 0, 0, 0], [149, 0, 1, bs], dtype)
    run_out(c, 1, 2, [140, 0, 1, bs], [150, 7, 2, bs], dtype)
    run_out(c, 0, 2, [7, 3, 149, 0], [8, 4, 150, 150], dtype)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_quant_out_every_code_and_scale(dtype):
    """All codes under scales from the smallest to the largest: roundings, numbers beyond
    the type's, NaN."""
    c = make("dense", 1, 1, 16, 1, 16 * 185, 16, 1)
    c.codes[0, :, 0, 0] = np.tile(np.arange(256, dtype=np.uint8), 185).reshape(-1, 16)
    c.scale[0, :, 0, 0, :] = np.ldexp(1.0, np.arange(-64, 121))
    run_out(c, 0, 1, [0], [16 * 185], dtype)


def test_quant_out_unmapped_blocks_and_many_sequences():
    rng = np.random.default_rng(9)
    c = make("paged", 1, 2, 64, 3, 64, 8, 4, holes=[(0, 1, -1), (1, 0, 1000), (2, 7, -5)])
    run_out(c, 0, 1, [0, 0, 3], [64, 20, 64], "f16")
    c = make("dense", 2, 1, 16, 450, 6, 4, 5)
    t0 = rng.integers(0, 4, 450).astype(np.int32)
    run_out(c, 0, 2, t0, (t0 + rng.integers(0, 3, 450)).astype(np.int32), "bf16")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_what_went_in_comes_back(dtype):
    """Rounding what was read back changes nothing, and attention is over the same numbers."""
    c = make("paged", 2, 2, 64, 3, 90, 16, 7)
    d, t = c.device(dv, attn)
    lens, code = [90, 33, 16], attn.DV_F16 if dtype == "f16" else attn.DV_BF16
    wire = torch.empty(2 * 2 * 2 * 64 * sum(lens), dtype=ref.TDTYPE[dtype], device="cuda")
    draft.dv_quant_out(d, 0, 0, 2, None, lens, wire, wire.numel() * 2, code)
    back = torch.empty_like(wire)
    attn.dv_quant_in(d, 0, 0, 2, None, lens, wire, wire.numel() * 2, code)
    draft.dv_quant_out(d, 0, 0, 2, None, lens, back, back.numel() * 2, code)
    assert torch.equal(wire, back)
