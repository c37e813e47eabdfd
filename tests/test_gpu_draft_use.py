"""The operators over drafted tokens as programs use them: captured and replayed, on streams of
their own, several at once, with one workspace for several calls."""
import numpy as np
import pytest
import torch

from paper_2403_01876_amd import attn, draft, dv
from tests import draft_ref as dref
from tests.test_gpu_attn import make

pytestmark = pytest.mark.gpu


class Step:
    """A step's buffers over a paged cache: drafts' tree, queries, logits, random numbers."""

    def __init__(self, seed, group=2, drawn=False, V=3001, most=20):
        rng = np.random.default_rng(seed)
        self.c = make("paged", 2, 2, 64, 3, 400, 16, seed, companions=True)
        self.cache, self.t = self.c.device(dv, attn)
        self.kv = np.array([400, 133, 57], np.int32)
        self.n = np.array([most, most - 3, 1], np.int32)
        rows = int(self.n.sum())
        self.parent = torch.from_numpy(dref.trees(self.n, rng)).cuda()
        self.q = torch.from_numpy(rng.normal(size=(rows, 2 * group, 64))).half().cuda()
        self.out = torch.zeros_like(self.q)
        self.lse = torch.zeros((rows, 2 * group), device="cuda")
        self.logits = torch.from_numpy(rng.normal(size=(rows, V)) * 3).to(torch.bfloat16).cuda()
        self.drawn = torch.softmax(self.logits.float(), -1) if drawn else None
        self.token = torch.from_numpy(rng.integers(0, V, rows).astype(np.int32)).cuda()
        up = torch.from_numpy(np.repeat(np.cumsum(self.n) - self.n, self.n)).cuda() + \
            self.parent.clamp(min=0)
        best = self.logits.float().argmax(-1)[up]
        self.token = torch.where(torch.from_numpy(rng.random(rows) < 0.7).cuda(), best.int(),
                                 self.token)
        self.uniform = torch.from_numpy(rng.random(rows).astype(np.float32)).cuda()
        self.path = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
        self.count, self.next = (torch.zeros(3, dtype=torch.int32, device="cuda")
                                 for _ in range(2))
        L, H, D = 2, 2, 64
        self.lo = np.maximum(self.kv - 30, 0).astype(np.int32)
        self.wire = torch.zeros(L * 2 * H * D * int((self.kv - self.lo).sum()),
                                dtype=torch.float16, device="cuda")
        need = max(attn.dv_attend_bytes(self.cache, self.n, self.kv, self.q),
                   draft.dv_verify_bytes(self.n, self.logits, drawn))
        self.room = torch.zeros(need, dtype=torch.uint8, device="cuda")

    def run(self, stream=None, room=None):
        room = self.room if room is None else room
        for layer in range(2):
            draft.dv_attend_tree(self.cache, 0, layer, self.n, self.kv, self.parent, self.q,
                                 self.out, 0.125, lse=self.lse, workspace=room, stream=stream)
        draft.dv_verify(self.n, self.parent, self.token, self.logits, self.uniform, self.path,
                        self.count, self.next, temperature=0.9, drawn=self.drawn, workspace=room,
                        stream=stream)
        draft.dv_keep_path(self.cache, 0, 0, 2, self.n, self.kv, self.path, self.count,
                           stream=stream)
        draft.dv_quant_out(self.cache, 0, 0, 2, self.lo, self.kv, self.wire,
                           self.wire.numel() * 2, attn.DV_F16, stream=stream)

    def result(self):
        torch.cuda.synchronize()
        return [x.clone() for x in (self.out, self.lse, self.path, self.count, self.next,
                                    self.wire, self.t["codes"], self.t["scale"],
                                    self.t["weight"], self.t["position"])]


def same(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("group", [1, 8])
def test_a_captured_step_replays_as_it_runs(drawn, group):
    """Every replay equals the eager step on the same buffers, with eager work between."""
    s, e = Step(3, group, drawn), Step(3, group, drawn)
    e.run()
    e.result()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run()
    torch.cuda.current_stream().wait_stream(side)
    assert same(s.result(), e.result())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.run()
    assert same(s.result(), e.result())  # (capturing runs nothing)
    rng = np.random.default_rng(5)
    for _ in range(4):
        # new numbers in the same buffers
        u = torch.from_numpy(rng.random(s.uniform.numel()).astype(np.float32)).cuda()
        q = torch.from_numpy(rng.normal(size=tuple(s.q.shape))).half().cuda()
        for x in (s, e):
            x.uniform.copy_(u)
            x.q.copy_(q)
            x.room.fill_(0xA5)
        g.replay()
        e.run()
        assert same(s.result(), e.result())


def test_two_captured_steps_may_share_a_workspace_in_turn():
    a, b, x, y = Step(5), Step(6, drawn=True), Step(5), Step(6, drawn=True)
    room = torch.zeros(max(a.room.numel(), b.room.numel()), dtype=torch.uint8, device="cuda")
    graphs = []
    for s in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.run(room=room)
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
        x.run()
        y.run()
        assert same(a.result(), x.result()) and same(b.result(), y.result())


def test_steps_on_two_streams_at_once():
    a, b, x, y = Step(7, 8), Step(8, 1, True), Step(7, 8), Step(8, 1, True)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, st in ((a, streams[0]), (b, streams[1])):
            s.run(stream=st)
    for _ in range(5):
        x.run()
        y.run()
    assert same(a.result(), x.result()) and same(b.result(), y.result())


def test_runs_are_equal_bit_for_bit():
    """Sums do not depend on the order in which workgroups run."""
    first = None
    for _ in range(6):
        s = Step(9, 8, True, V=20011)
        s.run()
        r = s.result()
        first = first or r
        assert same(first, r)


def test_rows_behind_the_last_draft_and_other_sequences_stay():
    """Results, paths and slots that no draft owns are left as they were."""
    s = Step(10)
    rows = s.q.shape[0]
    wide = [torch.full((rows + 5, *x.shape[1:]), 9, dtype=x.dtype, device="cuda")
            for x in (s.out, s.lse, s.path)]
    before = s.t["codes"].clone()
    draft.dv_attend_tree(s.cache, 0, 1, s.n, s.kv, s.parent, s.q, wide[0], 0.125, lse=wide[1],
                         workspace=s.room)
    draft.dv_verify(s.n, s.parent, s.token, s.logits, s.uniform, wide[2], s.count, s.next,
                    workspace=s.room)
    torch.cuda.synchronize()
    assert torch.equal(before, s.t["codes"])
    for x in wide:
        assert bool((x[rows:] == 9).all())
    draft.dv_keep_path(s.cache, 0, 1, 2, s.n, s.kv, wide[2], s.count)
    torch.cuda.synchronize()
    changed = (before != s.t["codes"]).any(-1)       # [L, 2, blocks, H, slots]
    assert not bool(changed[0].any())
    table = s.t["table"].cpu().numpy()
    owned = np.zeros(changed.shape[2:3] + changed.shape[4:], bool)
    for b in range(3):
        for t in range(int(s.kv[b] - s.n[b]) // 16 * 16, int(s.kv[b])):
            owned[table[b, t // 16], t % 16] = True
    assert not bool((changed[1].any(0).any(1).cpu() & ~torch.from_numpy(owned)).any())
