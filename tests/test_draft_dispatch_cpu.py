"""What calls of the operators over drafted tokens launch, without a GPU: their host code is
linked with launchers that write down what they are asked (tests/c/
draft_dispatch_record.cpp) and called with made-up addresses, which nothing reads."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2403_01876_amd import attn, draft, dv
from tests.test_attn_cpu import FAKE, OUT, ROOT, SCALE, SRC, WORK
from tests.test_draft_cpu import COUNT, NEXT, PARENT, PATH, TOKEN, UNIFORM

ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("dispatch") / "libdraftdispatch.so")
    csrc = os.path.join(ROOT, "paper_2403_01876_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-Wall", "-Werror",
                    "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"),
                    os.path.join(csrc, "dv_attn.cpp"), os.path.join(csrc, "dv_draft.cpp"),
                    os.path.join(ROOT, "tests", "c", "draft_dispatch_record.cpp"),
                    "-L", os.path.join(ROCM, "lib"), "-lamdhip64",
                    "-Wl,-rpath," + os.path.join(ROCM, "lib"), "-o", out], check=True, timeout=300)
    lib = ctypes.CDLL(out)
    for name in draft.EXPORTS + ("dv_attend_bytes",):
        getattr(lib, name).argtypes = getattr(attn.lib, name).argtypes
    lib.dispatch_record_take.restype = ctypes.c_char_p
    return lib


def taken(lib):
    return [(ln.split()[0], {k: int(v) for k, v in (f.split("=") for f in ln.split()[1:])})
            for ln in lib.dispatch_record_take().decode().splitlines()]


def dense(L, H, D, B, S):
    c = dv.Cache(dv.DV_DENSE, L, H, D, B, [FAKE], elem_bytes=1, max_seq=S)
    return attn.QuantCache(c, [SCALE + (1 << 45)], scale_block=16)


@pytest.mark.parametrize("seed", range(12))
def test_tree_tables_name_every_draft_once(lib, seed):
    """The longest sequences first under many rows, in the batch's order under few; each with
    its own rows, and work items in the order of the table."""
    r = np.random.default_rng(seed)
    B, group, H = int(r.integers(1, 500)), int(r.choice([1, 8])), 2
    kv = r.integers(0, 700, B).astype(np.int32)
    n = np.minimum(kv, r.integers(0, 129 if seed % 2 else 9, B)).astype(np.int32)
    if n.sum() == 0:
        n[0] = kv[0] = 1
    c = dense(1, H, 64, B, 700)
    far = 1 << 52
    a = attn.dv_attend_args(type=attn.DV_F16, q_heads=H * group, scale=0.1, rows=int(n.sum()),
                            q=far, out=2 * far, q_token=64 * H * group, q_head=64,
                            out_token=64 * H * group, out_head=64, workspace=3 * far,
                            workspace_bytes=1 << 50)
    assert lib.dv_attend_tree(c.ref, 0, 0, n.ctypes.data, kv.ctypes.data, 5 * far,
                              ctypes.byref(a), None) == 0
    ran = taken(lib)
    many = int(n.max()) * group > 64
    at, b0, row0 = 0, 0, 0
    while at < len(ran):
        what, f = ran[at]
        assert what == ("tile" if many else "split") and f["b0"] >= b0 and f["row0"] >= row0
        # (a launch without drafts is left out)
        assert n[b0:f["b0"]].sum() == 0
        b0 = f["b0"]
        assert f["parent"] == 5 * far + 4 * f["row0"] and f["row0"] == n[:b0].sum()
        seqs = [x for _, x in ran[at + 1:at + 1 + f["nseq"]]]
        assert sorted(x["b"] for x in seqs) == list(range(f["nseq"]))
        lens = [x["len"] for x in seqs]
        if many:
            assert lens == sorted(lens, reverse=True)
        else:
            assert [x["b"] for x in seqs] == list(range(f["nseq"]))
        item = 0
        for x in seqs:
            b = b0 + x["b"]
            assert x["len"] == kv[b] and x["nq"] == n[b]
            assert x["tok"] == n[b0:b].sum() and x["item"] == item
            if n[b]:
                R = 128 if many else 64 if n.max() * group > 32 else 32 if n.max() * group > 16 else 16
                item += -(-int(n[b]) * group // R) * H * max(1, -(-int(kv[b]) // f["chunk"]))
        assert item == f["items"]
        b0, row0 = b0 + f["nseq"], f["row0"] + int(sum(x["nq"] for x in seqs))
        at += 1 + f["nseq"]
        if at < len(ran) and ran[at][0] == "join":
            assert ran[at][1]["items"] == f["items"] and not f["direct"]
            at += 1
        else:
            assert f["direct"]
    assert row0 == n.sum()


@pytest.mark.parametrize("B,most,V", [(1, 1, 1), (3, 128, 1 << 24), (20, 128, 1 << 22), (700, 9, 32000),
                                      (5000, 3, 2041), (5000, 2, 2042), (192, 128, 16385)])
def test_verify_launches_stay_within_a_grid(lib, B, most, V):
    r = np.random.default_rng(B)
    n = r.integers(0, most + 1, B).astype(np.int32)
    n[0] = most
    t = r.choice([0.0, 0.5, 1.0], B).astype(np.float32)
    far = 1 << 55
    a = draft.dv_verify_args(type=attn.DV_BF16, batch=B, vocab=V, rows=int(n.sum()), logits=far,
                             logits_row=V, parent=PARENT, token=TOKEN, uniform=UNIFORM, path=PATH,
                             count=COUNT, next=NEXT, workspace=2 * far, workspace_bytes=1 << 40)
    size = ctypes.c_uint64(0)
    assert lib.dv_verify_bytes(n.ctypes.data, ctypes.byref(a), ctypes.byref(size)) == 0
    assert lib.dv_verify(n.ctypes.data, t.ctypes.data, ctypes.byref(a), None) == 0
    ran = taken(lib)
    pieces = (V + 7 + 2047) // 2048
    walks = [f for k, f in ran if k == "walk"]
    assert [f["b0"] for f in walks] == list(np.cumsum([0] + [f["nseq"] for f in walks[:-1]]))
    assert sum(f["nseq"] for f in walks) == B and sum(f["rows"] for f in walks) == n.sum()
    for k, f in ran:
        if k == "sums":
            assert -(-f["rows"] * f["pieces"] // 4) * 256 < 1 << 32
        if k in ("sums", "walk"):
            assert f["pieces"] == pieces and f["row0"] == n[:f["b0"]].sum()
            assert f["nseq"] * f["parts"] * 512 < 1 << 32
            # every piece is some part's, and no part is without one
            per = -(-pieces // f["parts"])
            assert (f["parts"] - 1) * per < pieces <= f["parts"] * per
    rows = [f for k, f in ran if k == "rows"]
    assert [f["n"] for f in rows] == n.tolist()
    assert [f["zero"] for f in rows] == (t == 0).astype(int).tolist()
    # the workspace holds its parts
    assert size.value >= int(n.sum()) * pieces * 16 + B * pieces * 16 + B * 4


@pytest.mark.parametrize("L,H,B", [(40000, 2, 3), (2, 40, 450), (1, 1 << 20, 3), (3, 7, 1)])
def test_keep_and_out_launches_cover_all(lib, L, H, B):
    r = np.random.default_rng(L)
    kv = r.integers(1, 40, B).astype(np.int32)
    n = np.minimum(kv, r.integers(0, 12, B)).astype(np.int32)
    n[0] = 1
    c = dense(L, H, 16, B, 40)
    far = 1 << 55
    assert lib.dv_keep_path(c.ref, 0, 0, L, n.ctypes.data, kv.ctypes.data, far, 2 * far, None) == 0
    ran = taken(lib)
    keeps = [f for k, f in ran if k == "keep"]
    for f in keeps:
        assert -(-f["nseq"] * f["heads"] // 4) * 256 < 1 << 32 and f["layers"] <= 65535
        assert f["path"] == far + 4 * n[:f["b0"]].sum() and f["count"] == 2 * far + 4 * f["b0"]
    layers = sorted({(f["l0"], f["layers"]) for f in keeps})
    assert sum(x for _, x in layers) == L and [x for x, _ in layers] == \
        list(np.cumsum([0] + [x for _, x in layers[:-1]]))
    assert len(keeps) == len(layers) * len({f["b0"] for f in keeps})
    one = [f for k, f in ran if k == "kept"][:B]
    if len({f["b0"] for f in keeps}) == 1:
        assert [f["base"] for f in one] == (kv - n).tolist()
        assert [f["tok"] for f in one] == (np.cumsum(n) - n).tolist()
    size = ctypes.c_uint64(0)
    t0 = (kv - n).astype(np.int32)
    assert lib.dv_quant_out(c.ref, 0, 0, L, t0.ctypes.data, kv.ctypes.data, far, 1 << 50,
                            attn.DV_F16, ctypes.byref(size), None) == 0
    assert size.value == L * 2 * H * 16 * 2 * int(n.sum())
    ran = [f for k, f in taken(lib) if k == "out"]
    for f in ran:
        assert -(-f["items"] * f["lanes"] // 256) * 256 < 1 << 32 and f["rows"] <= 65535
    assert sum(f["rows"] for f in ran) == 2 * L * len({f["b0"] for f in ran})


def test_nothing_is_launched_for_nothing(lib):
    c, zero, kv = dense(2, 2, 64, 3, 40), np.zeros(3, np.int32), np.full(3, 20, np.int32)
    a = attn.dv_attend_args(type=attn.DV_F16, q_heads=2, scale=1.0, rows=0, q=SRC, out=OUT,
                            workspace=WORK)
    z, k = zero.ctypes.data, kv.ctypes.data
    assert lib.dv_attend_tree(c.ref, 0, 0, z, k, PARENT, ctypes.byref(a), None) == 0
    assert lib.dv_keep_path(c.ref, 0, 0, 2, z, k, PATH, COUNT, None) == 0
    assert lib.dv_quant_out(c.ref, 0, 0, 2, k, k, SRC, 0, attn.DV_F16, None, None) == 0
    assert taken(lib) == []
