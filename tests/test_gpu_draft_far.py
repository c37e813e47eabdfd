"""The operators over drafted tokens where offsets pass 32 bits: a pool of more than 4 GiB a slab,
and logits whose rows lie more than 4 GiB apart.  What they compute is what they compute of the
same numbers close together, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2403_01876_amd import attn, draft, dv
from tests import draft_ref as dref
from tests.test_gpu_attn import make

pytestmark = pytest.mark.gpu

L, H, D, BS, B, CAP = 2, 2, 128, 16, 2, 208
FAR = (1 << 20) + (1 << 16)  # blocks of 4 KiB: 4.25 GiB a slab


def need(gib):
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB of device memory")


def moved(c, t):
    """The cache with its blocks at the far end of a large pool, but for every third one."""
    table = c.table.copy()
    used = table.reshape(-1)
    to = np.where(np.arange(used.size) % 3 == 0, used, FAR - 1 - used)
    codes = torch.empty((L, 2, FAR, H, BS, D), dtype=torch.uint8, device="cuda")
    scale = torch.empty((L, 2, FAR, H), device="cuda")
    for x, y in zip(used.tolist(), to.tolist()):
        for l in range(L):
            for kv in range(2):
                codes[l, kv, y].copy_(t["codes"][l, kv, x])
                scale[l, kv, y].copy_(t["scale"][l, kv, x])
    at = torch.from_numpy(to.reshape(table.shape).astype(np.int32)).cuda()
    pool = dv.Cache(dv.DV_PAGED, L, H, D, B, [codes], elem_bytes=1, block_size=BS, num_blocks=FAR,
                    max_blocks=table.shape[1], block_tables=[at])
    return attn.QuantCache(pool, [scale], scale_block=BS), codes, scale, used.tolist(), to.tolist()


@pytest.mark.parametrize("group,most", [(1, 24), (8, 40)])
def test_a_pool_past_4_gib(group, most):
    need(24)
    rng = np.random.default_rng(most)
    c = make("paged", L, H, D, B, CAP, BS, most)
    near, t = c.device(dv, attn)
    far, codes, scale, used, to = moved(c, t)
    kv, n = np.array([CAP, 101], np.int32), np.array([most, most - 7], np.int32)
    rows = int(n.sum())
    parent = torch.from_numpy(dref.trees(n, rng)).cuda()
    q = torch.from_numpy(rng.normal(size=(rows, H * group, D))).half().cuda()
    path = torch.tensor(([0, 2, 3, 9, 16] + [-1] * (most - 5) + [0, 1, 11] + [-1] * (most - 10)),
                        dtype=torch.int32, device="cuda")
    count = torch.tensor([5, 3], dtype=torch.int32, device="cuda")
    results = []
    for cache in (near, far):
        out = torch.zeros((L, *q.shape), dtype=q.dtype, device="cuda")
        ws = torch.empty(attn.dv_attend_bytes(cache, n, kv, q), dtype=torch.uint8, device="cuda")
        for layer in range(L):
            draft.dv_attend_tree(cache, 0, layer, n, kv, parent, q, out[layer], 0.1, workspace=ws)
        draft.dv_keep_path(cache, 0, 0, L, n, kv, path, count)
        wire = torch.zeros(L * 2 * H * D * int(kv.sum()), dtype=torch.float16, device="cuda")
        draft.dv_quant_out(cache, 0, 0, L, None, kv, wire, wire.numel() * 2, attn.DV_F16)
        results.append((out, wire))
    torch.cuda.synchronize()
    for a, b in zip(*results):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    for x, y in zip(used, to):
        assert torch.equal(codes[:, :, y], t["codes"][:, :, x])
        assert torch.equal(scale[:, :, y], t["scale"][:, :, x])


@pytest.mark.parametrize("drawn", [False, True])
def test_logits_rows_far_apart(drawn):
    need(40)
    rng = np.random.default_rng(3)
    V, far = 5003, (1 << 31) + 13
    x = torch.from_numpy(rng.normal(size=(4, V)) * 3).half().cuda()
    p = torch.softmax(x.float() + torch.from_numpy(rng.normal(size=(4, V))).float().cuda(), -1)
    row = torch.empty(3 * far + V, dtype=torch.float16, device="cuda").as_strided((4, V), (far, 1))
    q = None
    if drawn:
        q = torch.empty(3 * far + V, device="cuda").as_strided((4, V), (far, 1))
    for i in range(4):
        row[i].copy_(x[i])
        if drawn:
            q[i].copy_(p[i])
    parent = torch.tensor([-1, 0, 1, 1], dtype=torch.int32, device="cuda")
    token = torch.cat([x[0].argmax()[None], x[0].argmax()[None], x[1].argmin()[None],
                       x[1].argmax()[None]]).int()
    for u in ([0.3, 0.0, 0.9, 0.0], [0.7, 0.0, 0.99, 0.999], [0.01, 0.999, 0.5, 0.5]):
        got = []
        for logits, given in ((x, p if drawn else None), (row, q)):
            path, count, follow = (torch.full((k,), -7, dtype=torch.int32, device="cuda")
                                   for k in (4, 1, 1))
            ws = torch.empty(draft.dv_verify_bytes([4], logits, drawn), dtype=torch.uint8,
                             device="cuda")
            draft.dv_verify([4], parent, token, logits, torch.tensor(u, device="cuda"), path, count,
                            follow, drawn=given, workspace=ws)
            got.append(path.tolist() + count.tolist() + follow.tolist())
        assert got[0] == got[1]
