"""The 8-bit cache operators on the GPU against their plain 64-bit forms.

Rounding and eviction are compared code for code.  Attention: the result differs
from the 64-bit one by its own rounding (half a step of its type), by what 32-bit
scores of magnitude up to about 30 put on the probabilities (2e-5 of sum p |v|,
see PROB) and, for many rows, by the probabilities' rounding to the 16-bit type
(half a step of sum p |v|).
"""
import numpy as np
import pytest
import torch

from paper_2403_01876_amd import attn, dv
from tests import attn_ref as ref

pytestmark = pytest.mark.gpu

# exp(s) of a score s held in 32 bits (s < 32 after scaling to powers of two: half
# a step is 2^-20), its product sums of up to 256 terms (a few 2^-24 of their
# magnitude) and the sum over the tokens.
PROB = 2e-5
HALF = {k: torch.finfo(t).eps / 2 for k, t in ref.TDTYPE.items()}  # half a step, relative


def make(kind, L, H, D, B, cap, bs, seed, **kw):
    return ref.Cache8(kind, L, H, D, B, cap, bs, np.random.default_rng(seed), **kw)


def check_state(c, t, what):
    """The device's cache equals the host's."""
    got, scale = t["codes"].cpu().numpy(), t["scale"].cpu().numpy()
    assert np.array_equal(scale, c.scale), f"{what}: {int((scale != c.scale).sum())} scales"
    assert ref.same_codes(got, c.codes), f"{what}: {int((got != c.codes).sum())} codes differ"
    for name in ("weight", "position"):
        x = getattr(c, name)
        if x is not None:
            assert np.array_equal(t[name].cpu().numpy(), x, equal_nan=True), f"{what}: {name}"


# ---- dv_quant_in ----------------------------------------------------------------------------


def wire_of(c, l0, l1, n, dtype, rng, special=()):
    x = rng.normal(size=(l1 - l0, 2, n * c.H, c.D)) * 2.0 ** rng.integers(
        -6, 7, size=(l1 - l0, 2, n * c.H, 1))
    flat = x.reshape(-1)
    for i, v in enumerate(special):
        if flat.size:
            flat[(i * 7919) % flat.size] = v
    w = torch.from_numpy(x).to(ref.TDTYPE[dtype])
    return w, w.double().numpy()


def run_quant(c, l0, l1, t0, t1, dtype, rng, special=()):
    q, t = c.device(dv, attn)
    n = int((np.asarray(t1) - np.asarray(t0)).sum())
    w, x = wire_of(c, l0, l1, n, dtype, rng, special)
    src = w.cuda()
    attn.dv_quant_in(q, 0, l0, l1, t0, t1, src, src.numel() * 2,
                     attn.DV_F16 if dtype == "f16" else attn.DV_BF16)
    torch.cuda.synchronize()
    ref.quant_in(c, l0, l1, t0, t1, x, dtype)
    check_state(c, t, "quant")


@pytest.mark.parametrize("kind", ["dense", "paged"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D,bs", [(16, 1), (48, 5), (64, 16), (80, 8), (128, 16), (128, 64),
                                  (256, 16), (256, 40)])
def test_quant_prompts_and_appends(kind, dtype, D, bs):
    rng = np.random.default_rng(D * 100 + bs)
    c = make(kind, 3, 3, D, 4, 150, bs, D + bs, companions=True)
    ends = [149, 0, 1, bs]
    run_quant(c, 0, 3, [0, 0, 0, 0], ends, dtype, rng)
    # tokens appended to blocks that hold some, one layer only, a sequence idle
    run_quant(c, 1, 2, [140, 0, 1, bs], [150, 7, 2, bs], dtype, rng)
    for step in range(3):
        t0 = np.array([100 + step, 7 + step, 2 + step, bs + step], np.int32)
        run_quant(c, 0, 3, t0, t0 + 1, dtype, rng)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_quant_special_numbers(dtype):
    """Infinities, NaN, the type's largest and smallest numbers, zeros, ties."""
    big = 65504.0 if dtype == "f16" else 3.3895313892515355e38
    tiny = 2.0 ** -24 if dtype == "f16" else 2.0 ** -133
    special = [np.inf, -np.inf, np.nan, big, -big, 0.0, -0.0, tiny, -tiny, 61440.0, 61504.0,
               1.0625, 1.1875, 448.0, 464.0, 2.0 ** -14]
    rng = np.random.default_rng(5)
    c = make("dense", 1, 2, 32, 3, 64, 4, 1)
    run_quant(c, 0, 1, [0, 0, 0], [64, 33, 64], dtype, rng, special * 4)
    # a block of nothing but NaN, one of nothing but zeros, and appends to both
    c = make("dense", 1, 1, 16, 2, 8, 8, 2)
    q, t = c.device(dv, attn)
    x = torch.zeros((1, 2, 8, 16))
    x[0, 0, :4] = float("nan")
    w = x.to(ref.TDTYPE[dtype])
    src = w.cuda()
    code = attn.DV_F16 if dtype == "f16" else attn.DV_BF16
    attn.dv_quant_in(q, 0, 0, 1, [0, 0], [4, 4], src, src.numel() * 2, code)
    ref.quant_in(c, 0, 1, [0, 0], [4, 4], w.double().numpy(), dtype)
    check_state(c, t, "NaN and zeros")
    w, y = wire_of(c, 0, 1, 2, dtype, rng)
    src = w.cuda()
    attn.dv_quant_in(q, 0, 0, 1, [4, 4], [5, 5], src, src.numel() * 2, code)
    ref.quant_in(c, 0, 1, [4, 4], [5, 5], y, dtype)
    check_state(c, t, "appended to them")


def test_quant_unmapped_blocks_and_many_sequences():
    rng = np.random.default_rng(9)
    c = make("paged", 1, 2, 64, 3, 64, 8, 4, holes=[(0, 1, -1), (1, 0, 1000), (2, 7, -5)])
    run_quant(c, 0, 1, [0, 0, 3], [64, 20, 64], "f16", rng)
    c = make("dense", 2, 1, 16, 450, 6, 4, 5, companions=True)
    t0 = rng.integers(0, 4, 450).astype(np.int32)
    run_quant(c, 0, 2, t0, (t0 + rng.integers(0, 3, 450)).astype(np.int32), "bf16", rng)


# ---- dv_attend ------------------------------------------------------------------------------


def run_attend(c, q_len, kv_len, group, dtype, *, layer=None, slopes=False, decay=None,
               strided=False, lse=True, seed=0, spread=1.0):
    rng = np.random.default_rng(seed + 77)
    layer = c.L - 1 if layer is None else layer
    n, hq = int(np.sum(q_len)), c.H * group
    x = torch.from_numpy(rng.normal(size=(n, hq, c.D)) * spread).to(ref.TDTYPE[dtype])
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
    before = None if t["weight"] is None else t["weight"].clone()
    ls = torch.full((n, hq), 3.0, device="cuda") if lse else None
    nb = attn.dv_attend_bytes(d, q_len, kv_len, q, weights=decay is not None)
    ws = torch.full((nb + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    scale = float(np.float32(1.0 / np.sqrt(c.D)))
    attn.dv_attend(d, 0, layer, q_len, kv_len, q, out, scale,
                   slopes=None if sl is None else torch.from_numpy(sl).cuda(), decay=decay,
                   lse=ls, workspace=ws[:nb])
    torch.cuda.synchronize()
    assert bool((ws[nb:] == 0xA5).all()), "wrote past the workspace"
    want, mass, wlse, got = ref.attend(c, layer, q_len, kv_len, x.double().numpy(), scale,
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
    if lse:
        z = ls.double().cpu().numpy()
        dead = np.isneginf(wlse)
        assert np.array_equal(dead, np.isneginf(z)) and np.array_equal(np.isnan(wlse), np.isnan(z))
        live = np.isfinite(wlse)
        assert np.all(np.abs(z - wlse)[live] <= 1e-5 * np.maximum(1, np.abs(wlse[live])))
    if t["weight"] is not None:
        w, b4 = t["weight"].double().cpu().numpy(), before.double().cpu().numpy()
        if decay is None:
            assert np.array_equal(w, b4)
        else:
            fresh = np.zeros(w.shape, bool)
            for b in range(c.B):
                if q_len[b]:
                    fresh[layer, b, :, :kv_len[b]] = True
            assert np.array_equal(w[~fresh], b4[~fresh]), "weights of other slots changed"
            exp = np.zeros(w.shape)
            exp[layer] = got
            exp += decay * b4 if decay else 0
            bad = np.isnan(exp) & fresh
            assert np.array_equal(bad, np.isnan(w) & fresh)
            fresh &= ~bad
            e = np.abs(w - exp)[fresh]
            assert np.all(e <= PROB * np.abs(exp[fresh]) + 1e-7), float(np.max(e))
    return y


LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 300]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("kind,bs", [("dense", 16), ("dense", 7), ("paged", 16), ("paged", 3),
                                     ("paged", 1), ("paged", 64)])
@pytest.mark.parametrize("D,group", [(64, 1), (128, 8), (256, 2)])
def test_attend_single_tokens(dtype, kind, bs, D, group):
    c = make(kind, 2, 2, D, len(LENS), 300, bs, D + bs)
    run_attend(c, [1] * c.B, LENS, group, dtype)


@pytest.mark.parametrize("D", [16, 32, 48, 80, 96, 112, 144, 176, 208, 240])
@pytest.mark.parametrize("tokens", [1, 5, 70])
def test_attend_odd_head_dims(D, tokens):
    c = make("paged", 1, 2, D, 3, 200, 16, D, companions=True)
    lens = [200, 77, 5]
    run_attend(c, [min(tokens, n) for n in lens], lens, 1 + D % 3, "f16" if D % 32 else "bf16",
               slopes=D % 48 == 0, decay=0.0)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("group,tokens", [(1, 1), (1, 3), (7, 2), (8, 4), (16, 4), (3, 21),
                                          (1, 65), (4, 40), (8, 150), (5, 129)])
def test_attend_rows_of_every_path(dtype, group, tokens):
    """Few rows (1, 2 and 4 tiles of 16) and many, with weights, slopes,
    positions and strides."""
    c = make("dense", 2, 2, 128, 5, 420, 16, group * 100 + tokens, companions=True)
    lens = [420, 0, 131, 64, 300]
    q_len = [min(tokens, n) for n in lens]
    q_len[3] = 0
    run_attend(c, q_len, lens, group, dtype, slopes=True, decay=0.5, strided=True, layer=0)


@pytest.mark.parametrize("tokens", [1, 90])
def test_attend_queries_before_the_first_token(tokens):
    """More queries than tokens: those before slot 0 see nothing."""
    c = make("dense", 1, 1, 64, 3, 64, 16, 3, companions=True)
    run_attend(c, [tokens + 3, tokens, 2], [2, 0, 1], 2, "f16", decay=0.0)


@pytest.mark.parametrize("tokens", [1, 40])
@pytest.mark.parametrize("weights", [False, True])
def test_attend_long_axis_split(tokens, weights):
    c = make("paged", 1, 1, 128, 2, 9000, 16, 8, companions=weights)
    run_attend(c, [tokens, 1], [9000, 4097], 4, "bf16", decay=0.0 if weights else None)


@pytest.mark.parametrize("D,tokens", [(64, 700), (128, 333), (256, 130)])
def test_attend_weights_of_rows_in_shares(D, tokens):
    """Rows enough for several workgroups to add up each token's weight, some of
    which see none of its tokens."""
    c = make("paged", 1, 1, D, 3, 1500, 8, D + 1, companions=True)
    run_attend(c, [tokens, 1, 90], [1500, 700, 90], 8, "f16" if D == 128 else "bf16",
               slopes=D != 64, decay=0.25)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens", [1, 6, 80])
def test_attend_unmapped_blocks_and_nan(dtype, tokens):
    """Unmapped blocks are not seen; NaN in slots past a query's own, in slots past
    the sequence's end and in unmapped places stays out of its result, NaN that a
    query sees reaches the dimensions it should."""
    c = make("paged", 1, 2, 64, 4, 160, 8, 21, holes=[(0, 3, -1), (1, 0, 10 ** 6), (1, 1, -7),
                                                      (3, 0, -1)], companions=True)
    lens = [150, 16, 97, 8]
    used = np.zeros(c.nblocks, bool)
    for b, n in enumerate(lens):
        for j in range(-(-n // 8)):
            if c.place(b, j) is not None:
                used[c.table[b, j]] = True
    c.codes[:, :, ~used] = 127                      # blocks nobody maps
    for b, n in enumerate(lens):                    # slots past the end
        j = n // 8
        if n % 8 and c.place(b, j) is not None:
            c.codes[:, :, c.table[b, j], :, n % 8:] = 255
    c.codes[0, 1, c.table[2, 12], 0, 0, 5] = 127    # a value at the last slot, 96
    c.codes[0, 1, c.table[2, 11], 1, 3, 60] = 255   # and at slot 91, head 1
    c.codes[0, 0, c.table[0, 18], 1, 1, 7] = 127    # a key at slot 145
    y = run_attend(c, [min(tokens, n) for n in lens], lens, 2, dtype, decay=0.0)
    assert np.isnan(y).any() and not np.isnan(y).all()


def test_attend_many_sequences():
    rng = np.random.default_rng(2)
    c = make("dense", 1, 1, 32, 420, 40, 8, 11, companions=True)
    lens = rng.integers(0, 41, 420).astype(np.int32)
    run_attend(c, rng.integers(0, 3, 420).astype(np.int32), lens, 2, "f16", decay=0.0)
    c = make("dense", 1, 1, 32, 200, 90, 8, 12, companions=True)
    run_attend(c, rng.integers(0, 80, 200).astype(np.int32), np.full(200, 90, np.int32), 1, "f16",
               decay=0.0)


@pytest.mark.parametrize("tokens", [1, 70])
def test_attend_large_scores(tokens):
    """Scores of hundreds: one token takes all the weight, nothing overflows."""
    c = make("dense", 1, 1, 64, 1, 200, 16, 31, companions=True)
    c.scale *= 64
    rng = np.random.default_rng(1)
    d, t = c.device(dv, attn)
    q = torch.from_numpy(rng.normal(size=(tokens, 1, 64)) * 8).half().cuda()
    out = torch.empty_like(q)
    nb = attn.dv_attend_bytes(d, [tokens], [200], q, weights=True)
    ws = torch.empty(max(nb, 16), dtype=torch.uint8, device="cuda")
    attn.dv_attend(d, 0, 0, [tokens], [200], q, out, 0.125, decay=0.0, workspace=ws)
    want, mass, _, got = ref.attend(c, 0, [tokens], [200], q.double().cpu().numpy(), 0.125)
    # scores up to 2^12 carry 2^-12 in 32 bits, which is what the probabilities get
    y = out.double().cpu().numpy()
    assert np.isfinite(y).all()
    assert np.all(np.abs(y - want) <= 2.0 ** -12 * np.abs(want) + 4e-3 * mass)
    w = t["weight"].double().cpu().numpy()[0, :, :, :200]
    assert np.all(np.abs(w - got[:, :, :200]) <= 4e-3 * (1 + got[:, :, :200]))


# ---- dv_evict -------------------------------------------------------------------------------


def run_evict(c, d, l0, l1, length, keep, recent):
    (qc, tc) = c.device(dv, attn)
    (qd, td) = (qc, tc) if d is c else d.device(dv, attn)
    stride = max(1, max(min(int(a), int(b)) for a, b in zip(length, keep))) + 2
    kept = torch.full((l1 - l0, c.B, c.H, stride), -1, dtype=torch.int32, device="cuda")
    attn.dv_evict(qc, 0, qd, 0, l0, l1, length, keep, recent, kept)
    torch.cuda.synchronize()
    want = ref.evict(c, d, l0, l1, length, keep, recent, stride)
    assert np.array_equal(kept.cpu().numpy(), want)
    check_state(d, td, "evict")
    if d is not c:
        check_state(c, tc, "source")


def tie_weights(c, rng):
    w = rng.exponential(size=c.weight.shape).astype(np.float32)
    w = np.where(rng.random(w.shape) < 0.4, np.round(w * 2) / 2, w)
    c.weight[...] = np.where(rng.random(w.shape) < 0.2, 0, w)


@pytest.mark.parametrize("place", ["new", "same"])
@pytest.mark.parametrize("kind,bs", [("dense", 16), ("paged", 16), ("paged", 5), ("dense", 64),
                                     ("paged", 1)])
@pytest.mark.parametrize("D", [16, 80, 128, 256])
def test_evict(place, kind, bs, D):
    rng = np.random.default_rng(D + bs)
    c = make(kind, 2, 2, D, 6, 330, bs, D * 3 + bs, companions=True)
    tie_weights(c, rng)
    length = [330, 0, 1, 17, 200, 330]
    keep = [100, 5, 1, 40, 199, 0]
    if place == "same":
        run_evict(c, c, 0, 2, length, keep, 10)
    else:
        d = make("paged" if kind == "dense" else "dense", 2, 2, D, 6, 200, 16, 99,
                 companions=True)
        run_evict(c, d, 1, 2, length, keep, 10)


@pytest.mark.parametrize("recent", [0, 1, 50, 1000])
def test_evict_recent_tokens_and_odd_weights(recent):
    rng = np.random.default_rng(recent)
    c = make("dense", 1, 2, 32, 3, 300, 16, 7, companions=True)
    tie_weights(c, rng)
    c.weight[0, 0, 0, :40] = [np.nan, np.inf, -np.inf, -0.0, 0.0, -1.5, 1e-45, 3e38] * 5
    c.weight[0, 1] = 0.25  # nothing but ties
    c.position = None
    d = make("dense", 1, 2, 32, 3, 128, 16, 8, companions=True)
    run_evict(c, d, 0, 1, [300, 300, 64], [30, 128, 63], recent)


def test_evict_nan_is_evicted_first():
    c = make("dense", 1, 1, 16, 1, 8, 4, 3, companions=True)
    c.weight[0, 0, 0] = [np.nan, -np.inf, -3.0, np.nan, 0, 1, -np.inf, 2]
    run_evict(c, c, 0, 1, [8], [6], 0)


def test_evict_long_sequences():
    rng = np.random.default_rng(3)
    c = make("paged", 1, 1, 16, 2, 21000, 16, 5, companions=True)
    tie_weights(c, rng)
    run_evict(c, c, 0, 1, [21000, 4100], [9000, 4097], 33)


def test_evict_unmapped_blocks_and_many_sequences():
    rng = np.random.default_rng(4)
    c = make("paged", 1, 2, 32, 2, 64, 8, 6, companions=True, holes=[(0, 2, -1), (1, 0, 999)])
    tie_weights(c, rng)
    d = make("paged", 1, 2, 32, 2, 32, 8, 7, companions=True, holes=[(0, 1, 12345)])
    run_evict(c, d, 0, 1, [64, 50], [30, 25], 4)
    c = make("dense", 1, 1, 16, 400, 12, 4, 8, companions=True)
    tie_weights(c, rng)
    run_evict(c, c, 0, 1, rng.integers(0, 13, 400).astype(np.int32),
              rng.integers(0, 9, 400).astype(np.int32), 2)


# ---- together -------------------------------------------------------------------------------


def test_append_attend_evict_append():
    """A short generation: prompt, steps with weights, eviction, more steps with
    distances from the kept positions."""
    rng = np.random.default_rng(12)
    c = make("paged", 1, 2, 64, 2, 96, 16, 40, companions=True)
    run_quant(c, 0, 1, [0, 0], [60, 33], "f16", rng)
    run_attend(c, [60, 33], [60, 33], 2, "f16", slopes=True, decay=0.0)
    tie_weights(c, rng)
    run_evict(c, c, 0, 1, [60, 33], [24, 24], 8)
    run_quant(c, 0, 1, [24, 24], [25, 25], "f16", rng)
    assert (c.position[0, :, :, 24] == np.array([[60], [33]])).all()
    run_attend(c, [1, 1], [25, 25], 2, "f16", slopes=True, decay=1.0)


def test_attend_graph_replay_and_stream():
    """Captured on a stream of its own, replayed, and equal to the eager call."""
    c = make("paged", 1, 2, 128, 2, 700, 16, 50, companions=True)
    d, t = c.device(dv, attn)
    q = torch.randn((2, 8, 128), device="cuda").half()
    out, eager = torch.empty_like(q), torch.empty_like(q)
    nb = attn.dv_attend_bytes(d, [1, 1], [700, 300], q, weights=True)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    attn.dv_attend(d, 0, 0, [1, 1], [700, 300], q, eager, 0.1, decay=0.0, workspace=ws)
    torch.cuda.synchronize()
    weights = t["weight"].clone()
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        attn.dv_attend(d, 0, 0, [1, 1], [700, 300], q, out, 0.1, decay=0.0, workspace=ws)
    for _ in range(3):
        out.zero_()
        t["weight"].zero_()
        ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        assert torch.equal(t["weight"][:, 0], weights[:, 0] * (torch.arange(
            c.cap, device="cuda") < 700))
