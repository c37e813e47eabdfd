"""The operators over drafted tokens without a GPU: the library exports what
include/dv_draft.h declares, sizes and refusals come from the host alone (no call here
reaches the HIP runtime), and the plain forms agree with themselves."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest
import torch

from paper_2403_01876_amd import attn, draft, dv
from tests import draft_ref as dref
from tests.test_attn_cpu import (BAD_CACHES, FAKE, INVALID, LSE, OUT, POS, RANGE, ROOT, SCALE,
                                 SPACE, SRC, TABLE, UNSUPPORTED, WEIGHT, WORK, cache)

B = 3
PARENT, TOKEN, UNIFORM, PATH, COUNT, NEXT, LOGITS, DRAWN = (FAKE + (i << 36) for i in range(20, 28))


def test_library_exports_every_declared_function():
    text = open(os.path.join(ROOT, "include", "dv_draft.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"DV_API int (dv_\w+)\s*\(", text))
    assert names == set(draft.EXPORTS)
    lib = ctypes.CDLL(dv.LIB_PATH)
    for n in names:
        assert hasattr(lib, n), n


def test_header_compiles_as_c99_with_the_bindings_layout(tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "dv_draft.h"\n'
                   "int main(void) { printf(\"%zu %zu %zu %d %d\", sizeof(dv_verify_args), "
                   "offsetof(dv_verify_args, drawn_row), offsetof(dv_verify_args, workspace_bytes), "
                   "DV_MAX_DRAFTS, DV_F32); return 0; }\n")
    exe = tmp_path / "t"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I",
                    os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()
    a = draft.dv_verify_args
    assert [int(x) for x in got] == [ctypes.sizeof(a), a.drawn_row.offset,
                                     a.workspace_bytes.offset, draft.DV_MAX_DRAFTS, draft.DV_F32]


def ints(x):
    return np.array(x, np.int32)


def tree(c, q_len=(1, 2, 0), kv_len=(50, 3, 0), mb=0, layer=0, parent=PARENT, **kw):
    a = attn.dv_attend_args(type=attn.DV_F16, q_heads=4, scale=0.1, decay=0.0, weigh=0, rows=3,
                            q=SRC, out=OUT, q_token=256, q_head=64, out_token=256, out_head=64,
                            workspace=WORK, workspace_bytes=1 << 30)
    for k, v in kw.items():
        setattr(a, k, v)
    x, y = ints(q_len), ints(kv_len)
    return attn.lib.dv_attend_tree(c.ref, mb, layer, x.ctypes.data, y.ctypes.data, parent,
                                   ctypes.byref(a), 0)


def verify(q_len=(1, 2, 0), temperature=None, **kw):
    a = draft.dv_verify_args(type=attn.DV_F16, batch=B, vocab=100, rows=3, logits=LOGITS,
                             logits_row=100, drawn=None, drawn_row=0, parent=PARENT, token=TOKEN,
                             uniform=UNIFORM, path=PATH, count=COUNT, next=NEXT, workspace=WORK,
                             workspace_bytes=1 << 30)
    for k, v in kw.items():
        setattr(a, k, v)
    x = None if q_len is None else ints(q_len)
    t = None if temperature is None else np.array(temperature, np.float32)
    return attn.lib.dv_verify(None if x is None else x.ctypes.data,
                              None if t is None else t.ctypes.data, ctypes.byref(a), 0)


def keep(c, q_len=(1, 2, 0), kv_len=(50, 3, 0), mb=0, l0=0, l1=2, path=PATH, count=COUNT):
    x, y = ints(q_len), ints(kv_len)
    return attn.lib.dv_keep_path(c.ref, mb, l0, l1, x.ctypes.data, y.ctypes.data, path, count, 0)


def out(c, t0=(0, 0, 0), t1=(50, 3, 0), mb=0, l0=0, l1=2, dst=SRC, cap=1 << 30,
        dtype=attn.DV_F16):
    return draft.dv_quant_out(c, mb, l0, l1, t0, t1, dst, cap, dtype, stream=0, check=False)


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_every_call_refuses_a_bad_cache(bad, status):
    c = cache(**bad)
    assert tree(c, kv_len=(5, 3, 0)) == status
    assert keep(c, kv_len=(5, 3, 0)) == status
    assert out(c, t1=(5, 3, 0))[0] == status


def test_attend_tree_refusals():
    c = cache()
    assert tree(c, mb=1) == RANGE and tree(c, layer=2) == RANGE and tree(c, layer=-1) == RANGE
    assert tree(c, kv_len=(51, 3, 0)) == RANGE and tree(c, q_len=(-1, 1, 1)) == RANGE
    assert tree(c, kv_len=(50, 1, 0)) == RANGE  # drafts before the first slot
    assert tree(cache(S=500), q_len=(129, 0, 0), kv_len=(200, 0, 0), rows=200) == UNSUPPORTED
    assert tree(c, weigh=1) == UNSUPPORTED
    assert tree(c, parent=None) == INVALID and tree(c, parent=PARENT + 2) == INVALID
    assert tree(c, type=2) == INVALID and tree(c, q_heads=3) == INVALID and tree(c, rows=2) == SPACE
    assert tree(c, q=None) == INVALID and tree(c, out=SRC) == INVALID and tree(c, out=FAKE) == INVALID
    assert tree(c, lse=OUT) == INVALID
    assert tree(c, out_head=32) == INVALID and tree(c, q_token=4) == INVALID
    # the parents are read while these are written
    assert tree(c, parent=OUT + 64) == INVALID and tree(c, lse=LSE, parent=LSE) == INVALID
    long = cache(S=9000)
    assert tree(long, kv_len=(9000, 3, 0), workspace_bytes=0) == SPACE
    assert tree(long, kv_len=(9000, 3, 0), parent=WORK) == INVALID
    assert tree(cache(D=272)) == UNSUPPORTED
    assert tree(c, q_len=(0, 0, 0), q=None, out=None, parent=None) == 0  # nothing to do


def test_verify_refusals():
    assert verify(q_len=None) == INVALID and verify(type=3) == INVALID and verify(type=-1) == INVALID
    assert verify(vocab=0) == INVALID and verify(vocab=(1 << 24) + 1, logits_row=1 << 25) == UNSUPPORTED
    assert verify(batch=-1) == RANGE and verify(q_len=(1, -1, 0)) == RANGE
    assert verify(rows=-1) == RANGE
    assert verify(q_len=(129, 0, 0), rows=200) == UNSUPPORTED
    assert verify(rows=2) == SPACE and verify(workspace_bytes=8) == SPACE
    for k in ("logits", "parent", "token", "uniform", "path", "count", "next", "workspace"):
        assert verify(**{k: None}) == INVALID, k
        assert verify(**{k: FAKE + 1}) == INVALID, k
    assert verify(workspace=WORK + 8) == INVALID and verify(logits=LOGITS + 2, type=2) == INVALID
    assert verify(drawn=DRAWN + 2, drawn_row=100) == INVALID
    assert verify(logits_row=99) == INVALID and verify(drawn=DRAWN, drawn_row=99) == INVALID
    assert verify(logits_row=(1 << 33) + 1) == INVALID
    for t in ([1, 1, -0.5], [1, np.nan, 1], [np.inf, 1, 1]):
        assert verify(temperature=t) == INVALID, t
    # what is written overlaps what is read, or each other
    for k in ("path", "count", "next", "workspace"):
        for at in (LOGITS + 32, PARENT, TOKEN, UNIFORM):
            assert verify(**{k: at}) == INVALID, (k, at)
        assert verify(**{k: DRAWN, "drawn": DRAWN, "drawn_row": 100}) == INVALID, k
    assert verify(path=COUNT) == INVALID and verify(next=COUNT + 8) == INVALID
    assert verify(next=PATH + 8) == INVALID and verify(count=WORK + 64) == INVALID
    # the last row's end counts, not a whole stride
    assert verify(path=LOGITS + 2 * (2 * 1000 + 100) - 4, logits_row=1000) == INVALID
    assert verify(batch=0, q_len=()) == 0


def test_verify_workspace():
    a = draft.dv_verify_args(type=attn.DV_BF16, batch=B, vocab=32000)
    size = ctypes.c_uint64(0)

    def of(q_len):
        x = ints(q_len)
        assert attn.lib.dv_verify_bytes(x.ctypes.data, ctypes.byref(a), ctypes.byref(size)) == 0
        return size.value
    assert of((0, 0, 0)) == 0
    # 8 pieces of 4096 tokens, 16 bytes for each piece of a row and of a sequence
    assert of((5, 0, 128)) >= 133 * 8 * 16 + 3 * 8 * 16
    a.vocab, a.batch = 1 << 24, 65
    x = np.full(65, 128, np.int32)
    assert attn.lib.dv_verify_bytes(x.ctypes.data, ctypes.byref(a), ctypes.byref(size)) == 0
    a.batch = 260
    x = np.full(260, 128, np.int32)
    assert attn.lib.dv_verify_bytes(x.ctypes.data, ctypes.byref(a),
                                    ctypes.byref(size)) == UNSUPPORTED
    a.batch = 1
    assert attn.lib.dv_verify_bytes(x.ctypes.data, ctypes.byref(a), None) == INVALID


def test_keep_path_refusals():
    c = cache()
    assert keep(c, mb=1) == RANGE and keep(c, l1=3) == RANGE and keep(c, l0=2, l1=1) == RANGE
    assert keep(c, q_len=(-1, 0, 0)) == RANGE and keep(c, kv_len=(51, 3, 0)) == RANGE
    assert keep(c, kv_len=(50, 1, 0)) == RANGE
    assert keep(cache(S=500), q_len=(129, 0, 0), kv_len=(200, 0, 0)) == UNSUPPORTED
    for k in ("path", "count"):
        for at in (None, FAKE, SCALE, WEIGHT, POS, PATH + 2):
            assert keep(c, **{k: at}) == INVALID, (k, at)
        assert keep(cache(kind=dv.DV_PAGED), **{k: TABLE}) == INVALID
    assert keep(c, q_len=(0, 0, 0), path=None, count=None) == 0
    assert keep(c, l0=1, l1=1, path=None, count=None) == 0


def test_quant_out_refusals():
    c = cache()
    assert out(c, mb=1)[0] == RANGE and out(c, l1=3)[0] == RANGE and out(c, l0=2, l1=1)[0] == RANGE
    assert out(c, t1=(51, 0, 0))[0] == RANGE and out(c, t0=(5, 0, 0), t1=(4, 0, 0))[0] == RANGE
    assert out(c, t1=None)[0] == INVALID
    for bad in (2, -1):
        assert out(c, dtype=bad)[0] == INVALID
    need = 2 * 2 * 2 * 64 * 2 * 53
    assert out(c, cap=need - 1) == (SPACE, need)
    for at in (None, SRC + 8, FAKE + 16, SCALE + 16, WEIGHT, POS):
        assert out(c, dst=at)[0] == INVALID, at
    assert out(cache(kind=dv.DV_PAGED), dst=TABLE)[0] == INVALID
    assert out(c, t1=(0, 0, 0), dst=None, cap=0) == (0, 0)


def test_binding_refusals():
    c = dv.Cache(dv.DV_DENSE, 1, 2, 64, 1, [FAKE], elem_bytes=1, max_seq=40)
    qc = attn.QuantCache(c, [SCALE], scale_block=16)
    q = torch.zeros((2, 4, 64), dtype=torch.float16)
    parent = torch.zeros(2, dtype=torch.int32)
    for bad in (parent.long(), torch.zeros(4, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError, match="parent must be"):
            draft.dv_attend_tree(qc, 0, 0, [2], [4], bad, q, q.clone(), 1.0)
    with pytest.raises(dv.DvError):  # too few
        draft.dv_attend_tree(qc, 0, 0, [2], [4], parent[:1], q, q.clone(), 1.0)
    with pytest.raises(ValueError, match="q must be"):
        draft.dv_attend_tree(qc, 0, 0, [2], [4], parent, q[0], q.clone(), 1.0)
    with pytest.raises(dv.DvError):
        draft.dv_attend_tree(qc, 0, 1, [2], [4], parent, q, q.clone(), 1.0)
    logits, u = torch.zeros((2, 50)), torch.zeros(2)
    one = torch.zeros(1, dtype=torch.int32)
    good = dict(q_len=[2], parent=parent, token=parent.clone(), logits=logits, uniform=u,
                path=parent.clone(), count=one, next=one.clone())
    for k, bad in (("logits", logits.double()), ("logits", logits.t()), ("uniform", u.double()),
                   ("token", parent.long()), ("path", parent.short()), ("count", u),
                   ("next", torch.zeros(0, dtype=torch.int32)), ("q_len", [[2, 0]]),
                   ("drawn", logits.half()), ("drawn", logits[:, :40]),
                   ("workspace", torch.zeros((8, 8))[:, :4]), ("temperature", [1.0, 1.0])):
        with pytest.raises(ValueError):
            draft.dv_verify(**{**good, k: bad})
    with pytest.raises(dv.DvError):  # no workspace
        draft.dv_verify(**good)
    room = torch.zeros(1 << 16, dtype=torch.uint8)
    for k in ("logits", "path", "parent", "token", "uniform"):  # more drafts than rows
        with pytest.raises(dv.DvError, match="SPACE|space|capacity|-3|small"):
            draft.dv_verify(**{**good, k: good[k][:1], "workspace": room})
    with pytest.raises(ValueError, match="path must be"):
        draft.dv_keep_path(qc, 0, 0, 1, [2], [4], parent[:1], one)


def test_the_walk_samples_as_the_target_does():
    """Over many random numbers, what the plain walk accepts and samples is distributed as
    the target's own tokens: drafts drawn from another distribution, or not drawn."""
    rng = np.random.default_rng(3)
    V, n = 4, 40000
    logits = rng.normal(size=(3, V)) * 1.5
    p = dref.target(logits[0], 1.0)
    q = dref.target(rng.normal(size=V), 1.0).astype(np.float32)
    parent = np.array([-1, 0, 0])
    for drawn in (True, False):
        got = np.zeros(V)
        for _ in range(n):
            token = np.array([0, *(rng.choice(V, 2, p=q / q.sum()) if drawn else (1, 3))])
            path, count, follow, _ = dref.verify([3], parent, token, logits, rng.random(3),
                                                 drawn=np.tile(q, (3, 1)) if drawn else None)
            got[token[path[1]] if count[0] == 2 else follow[0]] += 1
        # four standard deviations of a count of n
        assert np.all(np.abs(got / n - p) < 4 * np.sqrt(p * (1 - p) / n)), (drawn, got / n, p)


def test_lines_of_broken_trees():
    assert dref.lines([-1, 0, 0, 2, 9, 4, 6, -2, 7]) == \
        [[0], [0, 1], [0, 2], [0, 2, 3], None, None, None, None, None]
    assert dref.kept([0, 2, 2, 3], 4, 4) == [0, 2] and dref.kept([0, 5], 2, 4) == [0]
    assert dref.kept([-1, 0], 2, 4) == [] and dref.kept([1, 2, 3], 2, 4) == [1, 2]
