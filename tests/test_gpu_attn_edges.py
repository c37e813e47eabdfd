"""The 8-bit cache operators where numbers and places are out of the ordinary.

Tolerances are those of tests/test_gpu_attn.py (its run_attend is used).
"""
import numpy as np
import pytest
import torch

from paper_2403_01876_amd import attn, dv
from tests import attn_ref as ref
from tests.test_gpu_attn import HALF, PROB, make, run_attend, tie_weights

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


# ---- numbers that a 16-bit type does not hold -----------------------------------------------


class Saturated(ref.Cache8):
    """What queries in f16 make of a cache where a call rounds what it reads."""

    def values(self, l, kv, b, h, n):
        x, ok = super().values(l, kv, b, h, n)
        return np.clip(x, -65504.0, 65504.0), ok


@pytest.mark.parametrize("D,group,tokens", [(64, 2, 150), (128, 8, 40), (256, 1, 70)])
def test_attend_values_beyond_f16(D, group, tokens):
    """Hidden from a row they do not touch it; seen, they count as f16's largest."""
    rng = np.random.default_rng(D)
    c = Saturated("dense", 1, 2, D, 2, 300, 16, rng, companions=True)
    c.scale[0, 1, :, :, 18] = 2.0 ** 12  # values of slots 288 to 299
    c.scale[0, 1, 0, 1, 17] = 2.0 ** 60
    y = run_attend(c, [tokens, 9], [300, 300], group, "f16", decay=0.0)
    assert np.isfinite(y).all() and np.abs(y).max() > 1000


@pytest.mark.parametrize("D,group,tokens", [(64, 2, 150), (128, 8, 40), (256, 1, 70)])
def test_attend_keys_beyond_f16(D, group, tokens):
    rng = np.random.default_rng(D)
    c = Saturated("paged", 1, 2, D, 2, 300, 16, rng, companions=True)
    for j in (3, 18):
        c.scale[0, 0, c.table[0, j]] = 2.0 ** 12
    c.scale[0, 0, c.table[1, 18], 0] = 2.0 ** 100
    y = run_attend(c, [tokens, 9], [300, 300], group, "f16", decay=0.0, spread=2.0 ** -14)
    assert np.isfinite(y).all()


@pytest.mark.parametrize("tokens", [1, 70])
def test_attend_far_scales(tokens):
    """bf16 holds every number of a cache rounded from it."""
    c = make("paged", 1, 2, 64, 2, 200, 8, 5, companions=True)
    c.scale[0, 0] *= 2.0 ** -54
    c.scale[0, 1] *= 2.0 ** 100
    run_attend(c, [tokens, 1], [200, 77], 2, "bf16", decay=0.0, spread=2.0 ** 53)


@pytest.mark.parametrize("tokens", [1, 70])
def test_attend_numbers_below_the_normal_ones_of_f16(tokens):
    """Keys and values that are multiples of 2^-24, as rounded from f16's smallest."""
    rng = np.random.default_rng(6)
    c = make("dense", 1, 2, 64, 2, 200, 8, 6, companions=True)
    c.codes = ref.encode(np.round(rng.normal(size=c.codes.shape) * 6).clip(-28, 28) * 16)
    c.scale[...] = 2.0 ** -28
    run_attend(c, [tokens, 1], [200, 77], 2, "f16", decay=0.0, spread=2.0 ** 12)


def test_attend_few_rows_keep_numbers_beyond_f16():
    c = make("dense", 1, 2, 64, 2, 300, 16, 7, companions=True)
    c.scale[0, 0, :, :, 3] = 2.0 ** 12
    c.scale[0, 1, :, :, 4] = 2.0 ** 9
    run_attend(c, [1, 1], [300, 211], 2, "f16", decay=0.0, spread=2.0 ** -16)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens,length", [(1, 200), (70, 200), (1, 3000), (70, 3000)])
def test_attend_one_value_as_large_as_can_be(dtype, tokens, length):
    """What an infinity of a bf16 stream becomes, seen by rows that give it about half
    (or less) of their weight after smaller scores: finite, and in its own dimension."""
    c = make("dense", 1, 1, 64, 1, length, 16, 18)
    c.codes[0, 0] = 0
    c.codes[0, 0, 0, 0, 150] = ref.encode(np.array(0.6875))
    c.scale[0, 0] = 1.0
    big = c.codes[0, 1, 0, 0, 144:160]  # the block around slot 150
    big[...] = 0
    big[6, 5] = ref.encode(np.array(240.0))
    c.scale[0, 1, 0, 0, 9] = 2.0 ** 120
    d, _ = c.device(dv, attn)
    q = torch.ones((tokens, 1, 64), dtype=ref.TDTYPE[dtype], device="cuda")
    out = torch.empty_like(q)
    nb = attn.dv_attend_bytes(d, [tokens], [length], q)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    attn.dv_attend(d, 0, 0, [tokens], [length], q, out, 0.125, workspace=ws)
    if dtype == "f16" and tokens > 64:  # its largest number, there
        c = Saturated.__new__(Saturated)
        c.__dict__.update(make("dense", 1, 1, 64, 1, length, 16, 18).__dict__)
        c.codes[0, 0], c.scale[0, 0] = 0, 1.0
        c.codes[0, 0, 0, 0, 150] = ref.encode(np.array(0.6875))
        c.codes[0, 1, 0, 0, 144:160] = big
        c.scale[0, 1, 0, 0, 9] = 2.0 ** 120
    want, mass, _, _ = ref.attend(c, 0, [tokens], [length], q.double().cpu().numpy(), 0.125)
    y = out.double().cpu().numpy()
    past = np.abs(want) > 65520.0 if dtype == "f16" else np.zeros(want.shape, bool)
    assert np.isinf(y[past]).all()
    tol = HALF[dtype] * np.abs(want) + (PROB + (HALF[dtype] if tokens > 64 else 0)) * mass + 2.0 ** -24
    assert np.all(np.abs(y - want)[~past] <= tol[~past])
    assert np.abs(want).max() > 1000


# ---- positions past 2^24, scores past 1e30 ---------------------------------------------------


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens", [1, 90])
@pytest.mark.parametrize("first", [2 ** 25 - 300, 2 ** 31 - 2000])
def test_attend_distances_of_late_positions(dtype, tokens, first):
    c = make("dense", 1, 2, 64, 2, 300, 16, 8, companions=True)
    c.position += np.int32(first)
    run_attend(c, [tokens, 3], [300, 41], 2, dtype, slopes=True, decay=0.0)


@pytest.mark.parametrize("tokens,length", [(1, 200), (1, 3000), (70, 200), (70, 3000)])
def test_attend_scores_below_minus_1e30(tokens, length):
    """Equal scores of about -1e32: the mean of the values."""
    c = make("dense", 1, 1, 64, 1, length, 16, 9)
    c.codes[0, 0] = 126
    c.scale[0, 0] = 2.0 ** 100
    d, _ = c.device(dv, attn)
    q = torch.full((tokens, 1, 64), -2.0 ** -3, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((tokens, 1), device="cuda")
    nb = attn.dv_attend_bytes(d, [tokens], [length], q)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    attn.dv_attend(d, 0, 0, [tokens], [length], q, out, 0.125, lse=lse, workspace=ws)
    want, mass, wlse, _ = ref.attend(c, 0, [tokens], [length], q.double().cpu().numpy(), 0.125)
    many = tokens > 64
    tol = HALF["bf16"] * np.abs(want) + (PROB + (HALF["bf16"] if many else 0)) * mass + 2.0 ** -24
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)
    assert np.all(wlse < -1e31)
    assert np.all(np.abs(lse.double().cpu().numpy() - wlse) <= 1e-5 * np.abs(wlse))


# ---- tables, sizes --------------------------------------------------------------------------


def test_evict_between_pools_of_one_table():
    """Two pools that one block table serves: both only read it."""
    rng = np.random.default_rng(13)
    c = make("paged", 1, 2, 32, 2, 64, 8, 14, companions=True)
    d = make("paged", 1, 2, 32, 2, 64, 8, 15, companions=True)
    d.table = c.table
    tie_weights(c, rng)
    (qc, tc), (_, td) = c.device(dv, attn), d.device(dv, attn)
    qd = attn.QuantCache(
        dv.Cache(dv.DV_PAGED, 1, 2, 32, 2, [td["codes"]], elem_bytes=1, block_size=8,
                 num_blocks=d.nblocks, max_blocks=d.mb, block_tables=[tc["table"]]),
        [td["scale"]], weights=[td["weight"]], positions=[td["position"]])
    kept = torch.full((1, 2, 2, 30), -1, dtype=torch.int32, device="cuda")
    attn.dv_evict(qc, 0, qd, 0, 0, 1, [64, 50], [30, 25], 4, kept)
    want = ref.evict(c, d, 0, 1, [64, 50], [30, 25], 4, 30)
    assert np.array_equal(kept.cpu().numpy(), want)
    assert np.array_equal(td["scale"].cpu().numpy(), d.scale)
    assert ref.same_codes(td["codes"].cpu().numpy(), d.codes)


@pytest.mark.parametrize("kind", ["dense", "paged"])
def test_scales_stream_as_a_cache(kind):
    """As the header describes them: what arrives is the sender's, block by block."""
    L, H, D, B, bs = 2, 4, 32, 3, 16
    c = make(kind, L, H, D, B, 176, bs, 16)
    d = make(kind, L, H, D, B, 176, bs, 17)
    d.scale[...] = 3.0
    lens, caches = np.array([170, 16, 0]), []
    if kind == "dense":  # 11 blocks, so that 12 are allocated
        for x in (c, d):
            x.scale = np.concatenate([x.scale, x.scale[..., :1]], -1)
    for x in (c, d):
        t = {k: torch.from_numpy(v).cuda() for k, v in (("s", x.scale), ("t", x.table))
             if v is not None}
        caches.append((t, dv.Cache(dv.DV_PAGED, L, 1, H, B, [t["s"]], elem_bytes=4, block_size=1,
                                   num_blocks=x.nblocks, max_blocks=x.mb, block_tables=[t["t"]])
                       if kind == "paged" else
                       dv.Cache(dv.DV_DENSE, L, H, 4, B, [t["s"]], elem_bytes=4, max_seq=3)))
    (_, src), (td, dst) = caches
    blocks = -(-lens // bs)
    n = blocks if kind == "paged" else -(-blocks // 4)
    wire = torch.empty(dv.dv_packed_bytes(src, 0, L, None, n), dtype=torch.uint8, device="cuda")
    sent = dv.dv_stream_out_prompt(src, 0, 0, L, None, n, wire, wire.numel())
    dv.dv_stream_in(dst, 0, 0, L, None, n, wire, sent)
    got = td["s"].cpu().numpy()
    for b in range(B):
        for j in range(int(blocks[b])):
            here, there = c.place(b, j), d.place(b, j)
            if kind == "paged":
                assert np.array_equal(got[:, :, there], c.scale[:, :, here])
            else:
                assert np.array_equal(got[:, :, b, :, there], c.scale[:, :, b, :, here])
    assert (got == 3.0).any()


@pytest.mark.parametrize("H,D,group", [(3, 128, 4), (2, 192, 20), (2, 96, 64)])
def test_attend_codes_read_past_the_caches(H, D, group):
    """Codes of 96 MB or more take loads of their own."""
    n, bs = -(-(96 << 20) // (2 * H * D)), 16
    pages = -(-n // bs)
    gen = torch.Generator(device="cuda").manual_seed(D)
    codes = torch.randint(0, 127, (1, 2, pages, H, bs, D), device="cuda", generator=gen)
    codes += 128 * torch.randint(0, 2, codes.shape, device="cuda", generator=gen)
    codes = codes.to(torch.uint8)
    scale = torch.ldexp(torch.ones((), device="cuda"),
                        torch.randint(-10, -7, (1, 2, pages, H), device="cuda", generator=gen))
    table = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)[None].contiguous()
    c = attn.QuantCache(
        dv.Cache(dv.DV_PAGED, 1, H, D, 1, [codes], elem_bytes=1, block_size=bs, num_blocks=pages,
                 max_blocks=pages, block_tables=[table]), [scale])
    q = torch.randn((1, H * group, D), device="cuda", generator=gen).half()
    out, lse = torch.empty_like(q), torch.empty((1, H * group), device="cuda")
    ws = torch.empty(attn.dv_attend_bytes(c, [1], [n], q), dtype=torch.uint8, device="cuda")
    attn.dv_attend(c, 0, 0, [1], [n], q, out, D ** -0.5, lse=lse, workspace=ws)
    value = torch.from_numpy(ref.VALUE).cuda()
    for h in range(H):
        K, V = (value[codes[0, half, table[0].long(), h].long()].mul(
            scale[0, half, table[0].long(), h].double()[:, None, None]).view(-1, D)[:n]
            for half in (0, 1))
        for g in range(h * group, (h + 1) * group):
            s = K @ q[0, g].double() * D ** -0.5
            p = torch.softmax(s, 0)
            want, mass = p @ V, p @ V.abs()
            tol = HALF["f16"] * want.abs() + PROB * mass + 2.0 ** -24
            assert bool(((out[0, g].double() - want).abs() <= tol).all()), (h, g)
            assert abs(float(lse[0, g]) - float(torch.logsumexp(s, 0))) <= 1e-5 * 20
