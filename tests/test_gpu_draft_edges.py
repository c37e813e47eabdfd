"""Verification where rounding could decide: guesses that cover all that has any
probability, remainders far below the rounding of what they are left from, numbers at and
past the end of [0, 1), logits whose differences 32 bits do not hold, NaN of every
kind; vocabularies that end next to a piece; and where results may lie.

Results are whole numbers and have to be equal to the plain 64-bit form's.  A number of 1 or
more lets no draft pass whatever the rounding, so such draws need no distance from a border;
draws with others are made anew until their closest decision lies 1e-9 from its border, and
a test without a clear draw fails.
"""
import numpy as np
import pytest
import torch

from paper_2403_01876_amd import draft, dv
from tests import draft_ref as dref
from tests.test_gpu_draft import TYPES, logits_of, run_verify

pytestmark = pytest.mark.gpu


def run_clear(draws, border=1e-9):
    """run_verify of the first of `draws` (dictionaries of its arguments) that is clear of
    its borders."""
    for kw in draws:
        try:
            return run_verify(**kw, border=border)
        except pytest.skip.Exception:
            pass
    raise AssertionError("no draw was clear of its borders")


def masked(B, most, V, live, rng, spread=2.0):
    """Logits of B sequences of `most` drafts, all but `live` tokens of each row -infinity, and
    those tokens [B, live]: some next to each other on both sides of 2048."""
    x = torch.full((B * most, V), -np.inf)
    tokens = np.empty((B, live), np.int64)
    for b in range(B):
        near = 2048 - live // 2 + np.arange(live)
        at = near if b % 3 == 0 and V > 2048 + live else rng.choice(V, live, replace=False)
        tokens[b] = rng.permutation(at)
        for row in range(b * most, (b + 1) * most):
            x[row, at] = torch.from_numpy(rng.normal(size=live) * spread).float()
    return x, tokens


def stars(tokens, rng, again):
    """Drafts that guess all of `tokens` after the first row, `again` of them twice: how
    many drafts a sequence has, and all their tokens."""
    guesses = [np.concatenate([[0], rng.permutation(np.concatenate([t, t[:again]]))]) for t in tokens]
    return len(guesses[0]), np.concatenate(guesses)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("live", [2, 3, 4, 5, 40])
@pytest.mark.parametrize("again", [0, 2])
def test_guesses_of_all_that_is_left(dtype, live, again):
    """Every token with any probability is guessed and refused: the last of them stays, and
    is what follows."""
    rng = np.random.default_rng(live + 100 * again)
    B, V = 64, 4500
    for u in (1.0, np.nan, 2.0):
        x, tokens = masked(B, 1 + live + again, V, live, rng)
        most, token = stars(tokens, rng, again)
        uniform = np.full(B * most, u, np.float32)
        uniform[::most] = rng.choice([0.0, 0.25, 0.5, 0.999, 1.0], B)
        got = run_verify([most] * B, V, TYPES[dtype], rng, shape="star", logits=x.to(TYPES[dtype]),
                         token=token, uniform=uniform, border=0.0,
                         temperature=rng.uniform(0.5, 2, B).astype(np.float32))
        assert (got[1] == 1).all()
        last = [list(dict.fromkeys(g))[-1] for g in token.reshape(B, most)[:, 1:].tolist()]
        assert got[2].tolist() == last


@pytest.mark.parametrize("seed", range(4))
def test_guesses_of_all_that_is_left_among_others(seed):
    """The same with ordinary numbers among those past the end."""
    rng = np.random.default_rng(seed)
    B, V, live = 48, 3001, 3 + seed

    def draws():
        for _ in range(20):
            x, tokens = masked(B, 1 + live, V, live, rng)
            most, token = stars(tokens, rng, 0)
            u = np.where(rng.random(B * most) < 0.4, rng.random(B * most), 1.0)
            yield dict(q_len=[most] * B, V=V, dtype=torch.float32, rng=rng, shape="star", logits=x,
                       token=token, uniform=u)
    run_clear(draws())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_remainder_far_below_the_rest(dtype):
    """What is left of a row may be 1e-20 or 1e-200 of it: it is what counts from there on."""
    rng = np.random.default_rng(4)
    B, V = 32, 2500
    for gap in (45.0, 60.0, 200.0):
        x = torch.full((B * 4, V), -np.inf)
        token = np.zeros((B, 4), np.int64)
        for b in range(B):
            at = rng.choice(V, 5, replace=False)
            x[b * 4:b * 4 + 4, at] = torch.tensor([0.0, -gap, -gap - 1, -gap - 0.5, -2 * gap])
            token[b, 1:] = at[[0, 1, 3] if b % 2 else [0, 4, 2]]
        uniform = np.full(B * 4, 1.0, np.float32)
        uniform[::4] = rng.choice([0.0, 0.125, 0.5, 0.875], B)
        got = run_verify([4] * B, V, TYPES[dtype], rng, shape="star", logits=x.to(TYPES[dtype]),
                         token=token.reshape(-1), uniform=uniform, border=0.0)
        assert (got[1] == 1).all()


@pytest.mark.parametrize("side", [-1, 1])
def test_rejections_of_nearly_all_there_is(side):
    """Two rejections leave 2^-44 of a row; the third guess is decided 1e-5 from its border,
    which sums that err by 2^-53 of the whole row would not tell."""
    rng = np.random.default_rng(9)
    V, e = 3000, 2.0 ** -22
    x = torch.full((4 * 16, V), -np.inf)
    token, uniform = [], []
    for b in range(16):
        at = rng.choice(V, 4, replace=False)
        share = rng.uniform(0.3, 0.7)
        # shares e^... of the row: nearly all, nearly all of the rest, and two of what is left
        x[4 * b, at] = torch.tensor([0.0, np.log(e), 2 * np.log(e) + np.log(share),
                                     2 * np.log(e) + np.log(1 - share)]).float()
        p = dref.target(x[4 * b].double().numpy(), 1.0)
        u3 = p[at[2]] / (p[at[2]] + p[at[3]]) * (1 + side * 1e-5)
        token += [0, *at[:3]]
        uniform += [rng.random(), 1 - 2.0 ** -24, 1 - 2.0 ** -24, u3]
    got = run_verify([4] * 16, V, torch.float32, rng, shape="star", logits=x, token=token,
                     uniform=uniform, border=1e-8)
    assert (got[1] == (1 if side > 0 else 2)).all()


def test_many_guesses_of_all_that_is_left():
    """127 guesses that cover a row, on both sides of several pieces."""
    rng = np.random.default_rng(6)
    B, V = 4, 9001
    x, tokens = masked(B, 128, V, 127, rng, 1.0)
    most, token = stars(tokens, rng, 0)
    uniform = np.full(B * most, 1.0, np.float32)
    got = run_verify([most] * B, V, torch.float32, rng, shape="star", logits=x, token=token,
                     uniform=uniform, border=0.0)
    assert got[2].tolist() == token.reshape(B, most)[:, -1].tolist()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("V,B", [(900, 64), (5000, 64), (140001, 12)])
def test_a_number_of_one_takes_the_last_token(V, B, drawn, dtype):
    """However little the last token holds beside the rest: shares down to 1e-150."""
    rng = np.random.default_rng(V)
    n = rng.integers(1, 4, B)
    for u0 in (1.0, 2.0, np.nan):
        def draws():
            for _ in range(20):
                u = rng.random(n.sum())
                u[np.cumsum(n) - n] = u0
                yield dict(q_len=n, V=V, dtype=TYPES[dtype], rng=rng, drawn=drawn, uniform=u,
                           temperature=rng.uniform(0.06, 0.3, B).astype(np.float32),
                           logits=torch.from_numpy(rng.normal(size=(n.sum(), V)) * 2).to(TYPES[dtype]))
        run_clear(draws())


def test_logits_as_far_apart_as_they_come():
    """Differences of logits past 32 bits' range, under temperatures that make them count, in
    rows with NaN and without."""
    rng = np.random.default_rng(3)
    B, V = 32, 300
    x = torch.full((2 * B, V), -np.inf)
    token, uniform = [], []
    for b in range(B):
        at = rng.choice(V, 4, replace=False)
        x[2 * b, at] = torch.tensor([3.3e38, -3.3e38, -3.2e38, -3.1e38])
        if b % 2:
            x[2 * b, rng.choice(np.setdiff1d(np.arange(V), at))] = np.nan
        p = dref.target(x[2 * b].double().numpy(), 3e38)
        token += [0, at[b // 2 % 2]]
        uniform += [rng.random(), p[token[-1]] * (1.02 if b % 4 < 2 else 0.98)]
    got = run_verify([2] * B, V, torch.float32, rng, shape="chain", logits=x, token=token,
                     uniform=uniform, temperature=np.full(B, 3e38, np.float32))
    assert got[1].tolist() == [1 if b % 4 < 2 else 2 for b in range(B)]


def test_results_in_pinned_memory_and_none_in_pageable():
    """What a step reads on the host may lie in pinned memory; pageable memory is refused."""
    q_len, V = [5, 0, 9], 3000
    rows = sum(q_len)
    rng = np.random.default_rng(1)
    ints = torch.from_numpy(dref.trees(q_len, rng)).cuda()
    token = torch.from_numpy(rng.integers(0, V, rows).astype(np.int32)).cuda()
    x, u = logits_of(rows, V, rng, torch.float32).cuda(), torch.rand(rows, device="cuda")
    room = torch.empty(draft.dv_verify_bytes(q_len, x), dtype=torch.uint8, device="cuda")

    def results(**where):
        return [torch.full((n,), -7, dtype=torch.int32, **where) for n in (rows, 3, 3)]
    a, b, host = results(device="cuda"), results(pin_memory=True), results()
    for r in (a, b):
        draft.dv_verify(q_len, ints, token, x, u, *r, workspace=room)
    torch.cuda.synchronize()
    assert all(torch.equal(y.cpu(), z) for y, z in zip(a, b))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        draft.dv_verify(q_len, ints, token, x, u, *b, workspace=room)
    for _ in range(3):
        u.copy_(torch.rand(rows, device="cuda"))
        graph.replay()
        draft.dv_verify(q_len, ints, token, x, u, *a, workspace=room)
        torch.cuda.synchronize()
        assert torch.equal(a[1].cpu(), b[1]) and torch.equal(a[2].cpu(), b[2])
    with pytest.raises(dv.DvError, match=r"\(path, count, next: not in"):
        draft.dv_verify(q_len, ints, token, x, u, *host, workspace=room)
    torch.cuda.synchronize()
    assert all((h == -7).all() for h in host)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("V", [2040, 2041, 2042, 2047, 2048, 2049, 4088, 4089, 4090, 6143, 6145])
def test_sizes_next_to_a_piece(dtype, drawn, V):
    """Vocabularies that end next to a piece of 2048 tokens, in rows of an odd stride, which
    begin at every place of 16 bytes."""
    rng = np.random.default_rng(V)
    q_len = [9, 1, 0, 11, 2]

    def draws(shape):
        for _ in range(20):
            yield dict(q_len=q_len, V=V, dtype=TYPES[dtype], rng=rng, shape=shape, drawn=drawn,
                       pad=1 - V % 2 + 2 * (V % 3),
                       temperature=np.array([0.7, 1.3, 1.0, 0.0, 40.0], np.float32))
    for shape in ("tree", "chain", "star"):
        run_clear(draws(shape))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_the_last_token_next_to_a_piece(dtype):
    """One token has nearly all, the last of the vocabulary or the first of a piece: it is
    accepted and follows, from every place that a row may begin at."""
    for V in (2041, 2042, 2048, 2049, 4097):
        for at in sorted({0, V - 1, min(2047, V - 1), min(2048, V - 1), V - 8}):
            x = torch.zeros((16, V))
            x[:, at] = 30.0
            got = run_verify([16], V, TYPES[dtype], np.random.default_rng(at), shape="chain",
                             logits=x.to(TYPES[dtype]), token=[at] * 16, pad=1 - V % 2,
                             uniform=[0.5] * 16)
            assert got[1].tolist() == [16] and got[2].tolist() == [at]


@pytest.mark.parametrize("dtype,nans", [("f16", [0x7c01, 0x7e00, 0xfc01, 0xffff]),
                                        ("bf16", [0x7f81, 0x7fc0, 0xff81, 0xffff]),
                                        ("f32", [0x7f800001, 0x7fc00000, 0xff800001, 0xffffffff])])
@pytest.mark.parametrize("drawn", [False, True])
def test_nan_of_every_kind(dtype, nans, drawn):
    """NaN, quiet and signalling, of either sign: none is a largest logit or part of a sum; with
    an infinite logit and without."""
    rng = np.random.default_rng(len(nans))
    V, n = 4500, 8
    bits = np.array(nans, np.uint32 if dtype == "f32" else np.uint16)
    for infinite in (False, True):
        def draws():
            for _ in range(20):
                x = logits_of(n, V, rng, TYPES[dtype])
                y = x.numpy().view(bits.dtype) if dtype != "bf16" else \
                    x.view(torch.int16).numpy().view(np.uint16)
                for row in range(n):
                    at = rng.choice(V, 200, replace=False)
                    y[row, at] = rng.choice(bits, 200)
                    if infinite and row % 2:
                        x[row, rng.choice(V, 3, replace=False)] = np.inf
                yield dict(q_len=[n], V=V, dtype=TYPES[dtype], rng=rng, drawn=drawn, logits=x,
                           temperature=np.array([rng.choice([0.0, 0.8])], np.float32))
        for _ in range(4):
            run_clear(draws())


@pytest.mark.parametrize("drawn", [False, True])
def test_probabilities_that_count_as_none(drawn):
    """Below 2^-1020 of the largest (e^-707) a token is not there; above it is."""
    V, T = 3000, np.full(2, 0.125, np.float32)
    x = torch.full((4, V), -np.inf)
    x[:, 100] = 0.0
    x[:, 2500] = -706 * 0.125
    x[:, 2900] = -708 * 0.125
    q = torch.zeros((4, V))
    q[:, 100] = 0.5
    ints = torch.tensor([-1, 0, -1, 0], dtype=torch.int32).cuda()
    path, count, follow = (torch.full((n,), -7, dtype=torch.int32, device="cuda") for n in (4, 2, 2))
    for kind in TYPES.values():
        logits = x.to(kind).cuda()
        room = torch.empty(draft.dv_verify_bytes([2, 2], logits, drawn), dtype=torch.uint8,
                           device="cuda")
        # a guess of either with the number 0, which any probability is above
        draft.dv_verify([2, 2], ints, torch.tensor([0, 2500, 0, 2900], dtype=torch.int32).cuda(),
                        logits, torch.tensor([1.0, 0.0, 1.0, 0.0], device="cuda"), path, count,
                        follow, temperature=T, drawn=q.cuda() if drawn else None, workspace=room)
        assert count.tolist() == [2, 1] and follow.tolist() == [2500, 2500]
