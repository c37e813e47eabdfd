"""The 8-bit cache operators without a GPU: the library exports what
include/dv_attn.h declares, sizes and refusals come from the host alone (no call
here reaches the HIP runtime)."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest
import torch

from paper_2403_01876_amd import attn, dv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 40  # an aligned address never dereferenced by the host checks
SCALE, WEIGHT, POS, TABLE = (FAKE + (i << 36) for i in (1, 2, 3, 4))
SRC, OUT, WORK, KEPT, LSE = (FAKE + (i << 36) for i in (5, 6, 7, 8, 9))
INVALID, RANGE, SPACE, UNSUPPORTED = -1, -2, -3, -4
B = 3


def cache(kind=dv.DV_DENSE, E=1, D=64, H=2, S=50, base=FAKE, mem=dv.DV_MEM_DEVICE, sb=16,
          scale=SCALE, weight=WEIGHT, position=POS, bs=16, NB=20, MB=4, table=TABLE, L=2):
    paged = kind == dv.DV_PAGED
    c = dv.Cache(kind, L, H, D, B, [base], elem_bytes=E, mem=mem, max_seq=0 if paged else S,
                 block_size=bs if paged else 0, num_blocks=NB if paged else 0,
                 max_blocks=MB if paged else 0, block_tables=[table] if paged else None)
    return attn.QuantCache(c, [scale], scale_block=sb,
                           weights=None if weight is None else [weight],
                           positions=None if position is None else [position])


def test_library_exports_every_declared_function():
    text = open(os.path.join(ROOT, "include", "dv_attn.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"DV_API int (dv_\w+)\s*\(", text))
    assert names == set(attn.EXPORTS)
    lib = ctypes.CDLL(dv.LIB_PATH)
    for n in names:
        assert hasattr(lib, n), n


def test_header_compiles_as_c99_with_the_bindings_layout(tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "dv_attn.h"\n'
                   "int main(void) { printf(\"%zu %zu %zu %zu\", sizeof(dv_quant), "
                   "sizeof(dv_attend_args), offsetof(dv_attend_args, q_token), "
                   "offsetof(dv_attend_args, workspace_bytes)); return 0; }\n")
    exe = tmp_path / "t"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I",
                    os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()
    a = attn.dv_attend_args
    assert [int(x) for x in got] == [ctypes.sizeof(attn.dv_quant), ctypes.sizeof(a),
                                     a.q_token.offset, a.workspace_bytes.offset]


def test_scale_bytes():
    assert attn.dv_quant_scale_bytes(cache()) == 2 * 2 * B * 2 * 4 * 4  # ceil(50 / 16) blocks
    assert attn.dv_quant_scale_bytes(cache(sb=7)) == 2 * 2 * B * 2 * 8 * 4
    assert attn.dv_quant_scale_bytes(cache(kind=dv.DV_PAGED)) == 2 * 2 * 20 * 2 * 4


BAD_CACHES = [
    (dict(E=2), INVALID), (dict(mem=dv.DV_MEM_HOST_PINNED), INVALID), (dict(sb=-1), INVALID),
    (dict(sb=0), INVALID), (dict(kind=dv.DV_DENSE_KSPLIT), UNSUPPORTED),
    (dict(kind=dv.DV_PAGED, sb=8), INVALID), (dict(scale=0), INVALID),
    (dict(scale=SCALE + 2), INVALID), (dict(weight=WEIGHT + 1), INVALID),
    (dict(position=POS + 3), INVALID), (dict(base=FAKE + 8), INVALID), (dict(D=24), INVALID),
    (dict(kind=dv.DV_PAGED, NB=1 << 26, D=64), UNSUPPORTED),
    # parts of one cache on each other
    (dict(scale=FAKE + 64), INVALID), (dict(weight=SCALE), INVALID),
    (dict(position=FAKE + 128), INVALID), (dict(kind=dv.DV_PAGED, table=SCALE + 16), INVALID),
]


def quant(c, t0=(0, 0, 0), t1=(50, 3, 0), mb=0, l0=0, l1=2, src=SRC, nbytes=1 << 30,
          dtype=attn.DV_F16):
    return attn.dv_quant_in(c, mb, l0, l1, t0, t1, src, nbytes, dtype, stream=0, check=False)


def attend(c, q_len=(1, 2, 0), kv_len=(50, 3, 0), mb=0, layer=0, **kw):
    a = attn.dv_attend_args(type=attn.DV_F16, q_heads=4, scale=0.1, decay=0.0, weigh=0, rows=3,
                            q=SRC, out=OUT, q_token=256, q_head=64, out_token=256, out_head=64,
                            workspace=WORK, workspace_bytes=1 << 30)
    for k, v in kw.items():
        setattr(a, k, v)
    x, y = np.array(q_len, np.int32), np.array(kv_len, np.int32)
    return attn.lib.dv_attend(c.ref, mb, layer, x.ctypes.data, y.ctypes.data, ctypes.byref(a), 0)


def evict(c, d=None, length=(50, 3, 0), keep=(10, 10, 10), recent=4, kept=KEPT, stride=10, l0=0,
          l1=2, mb=0):
    return attn.dv_evict(c, mb, c if d is None else d, 0, l0, l1, length, keep, recent, kept,
                         kept_stride=stride, stream=0, check=False)


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_every_call_refuses_a_bad_cache(bad, status):
    if "D" in bad and bad["D"] == 24:
        assert attn.dv_quant_scale_bytes(cache(**bad), check=False)[0] == INVALID
        return
    c = cache(**bad)
    assert quant(c, t1=(5, 3, 0)) == status
    assert attend(c, kv_len=(5, 3, 0)) == status
    assert evict(c, length=(5, 3, 0)) == status


def test_quant_in_refusals():
    c = cache()
    assert quant(c, mb=1) == RANGE and quant(c, mb=-1) == RANGE
    assert quant(c, l1=3) == RANGE and quant(c, l0=-1) == RANGE and quant(c, l0=2, l1=1) == RANGE
    assert quant(c, t1=(51, 0, 0)) == RANGE and quant(c, t0=(5, 0, 0), t1=(4, 0, 0)) == RANGE
    assert quant(c, t0=(-1, 0, 0)) == RANGE
    assert quant(c, dtype=2) == INVALID and quant(c, dtype=-1) == INVALID
    assert quant(c, t1=None) == INVALID
    need = 2 * 2 * 2 * 64 * 2 * 53
    assert quant(c, nbytes=need - 1) == SPACE
    assert quant(c, src=None) == INVALID and quant(c, src=SRC + 8) == INVALID
    for at in (FAKE, SCALE, WEIGHT, POS):
        assert quant(c, src=at + 16) == INVALID
    assert quant(cache(kind=dv.DV_PAGED), src=TABLE) == INVALID
    # nothing to do: no address is looked at
    assert quant(c, t1=(0, 0, 0), src=None, nbytes=0) == 0
    assert quant(c, l0=1, l1=1, src=None, nbytes=0) == 0


def test_attend_refusals():
    c = cache()
    assert attend(c, mb=1) == RANGE and attend(c, layer=2) == RANGE and attend(c, layer=-1) == RANGE
    assert attend(c, kv_len=(51, 3, 0)) == RANGE and attend(c, kv_len=(-1, 3, 0)) == RANGE
    assert attend(c, q_len=(-1, 1, 1)) == RANGE and attend(c, q_len=((1 << 24) + 1, 0, 0)) == RANGE
    assert attend(c, type=2) == INVALID
    for heads in (0, -2, 3):
        assert attend(c, q_heads=heads) == INVALID
    assert attend(c, rows=2) == SPACE and attend(c, workspace_bytes=0, weigh=1) == SPACE
    for k in ("q", "out", "workspace"):
        assert attend(c, **{k: SRC + (1 << 33) + 8}) == INVALID, k
    for k in ("q", "out"):
        assert attend(c, **{k: None}) == INVALID, k
    for k in ("slopes", "lse"):
        assert attend(c, **{k: LSE + 2}) == INVALID, k
    for k in ("q_token", "q_head", "out_token", "out_head"):
        for v in (-8, 4, 1 << 31):
            assert attend(c, **{k: v}) == INVALID, (k, v)
    assert attend(c, out_head=32) == INVALID and attend(c, out_token=0) == INVALID
    assert attend(c, out=SRC) == INVALID and attend(c, out=FAKE) == INVALID
    assert attend(c, out=SCALE) == INVALID and attend(c, lse=OUT) == INVALID
    assert attend(c, lse=POS) == INVALID and attend(c, workspace=OUT, weigh=1) == INVALID
    assert attend(c, slopes=OUT + 16) == INVALID
    assert attend(c, weigh=1, q=WEIGHT) == INVALID
    assert attend(cache(weight=None), weigh=1) == INVALID
    assert attend(cache(D=272)) == UNSUPPORTED
    assert attend(cache(kind=dv.DV_PAGED), out=TABLE) == INVALID
    assert attend(c, q_len=(0, 0, 0), q=None, out=None) == 0  # nothing to do


def test_evict_refusals():
    c = cache()
    far = dict(base=FAKE + (1 << 40), scale=SCALE + (1 << 40), weight=WEIGHT + (1 << 40),
               position=POS + (1 << 40))
    assert evict(c, mb=1) == RANGE and evict(c, l1=3) == RANGE and evict(c, recent=-1) == RANGE
    assert evict(c, length=(51, 0, 0)) == RANGE and evict(c, keep=(-1, 0, 0)) == RANGE
    assert evict(c, stride=9) == RANGE and evict(c, stride=-1) == RANGE
    assert evict(c, cache(S=9, **far)) == RANGE
    assert evict(cache(weight=None)) == INVALID
    assert evict(c, kept=None) == INVALID and evict(c, kept=KEPT + 2) == INVALID
    for at in (FAKE, SCALE, WEIGHT, POS):
        assert evict(c, kept=at) == INVALID
    for other in (dict(H=1), dict(D=32), dict(L=1)):
        assert evict(c, cache(**far, **other)) == INVALID
    # the same codes but not the same cache, and caches that overlap
    assert evict(c, cache(S=64)) == INVALID and evict(c, cache(sb=8)) == INVALID
    assert evict(c, cache(scale=SCALE + (1 << 40))) == INVALID
    assert evict(c, cache(**{**far, "base": FAKE + 16})) == INVALID
    assert evict(c, cache(**{**far, "scale": SCALE})) == INVALID
    assert evict(c, cache(**{**far, "weight": FAKE + 64})) == INVALID
    assert evict(c, keep=(0, 0, 0), kept=None, stride=0) == 0  # nothing to do
    assert evict(c, l0=1, l1=1, kept=None) == 0


@pytest.mark.parametrize("seed", range(30))
def test_workspace_holds_its_parts(seed):
    """dv_attend_bytes: none where one launch does all, enough for the kept scores and
    the splits otherwise, and the same whatever the cache holds."""
    r = np.random.default_rng(seed)
    batch, H = int(r.integers(1, 400)), int(r.integers(1, 9))
    D = int(r.choice([16, 64, 96, 128, 256]))
    cap = int(r.choice([40, 700, 20000]))
    group = int(r.choice([1, 2, 8]))
    c = dv.Cache(dv.DV_DENSE, 1, H, D, batch, [FAKE], elem_bytes=1, max_seq=cap)
    qc = attn.QuantCache(c, [SCALE], scale_block=16, weights=[WEIGHT])
    kv = r.integers(0, cap + 1, batch).astype(np.int32)
    n = r.integers(0, int(r.choice([2, 9, 60])), batch).astype(np.int32)
    a = attn.dv_attend_args(type=attn.DV_BF16, q_heads=H * group)
    out = ctypes.c_uint64(0)

    def size(weigh):
        a.weigh = weigh
        assert attn.lib.dv_attend_bytes(qc.ref, n.ctypes.data, kv.ctypes.data, ctypes.byref(a),
                                        ctypes.byref(out)) == 0
        return out.value

    plain, weighed = size(0), size(1)
    rows = int(n.max()) * group
    if rows <= (64 if D <= 128 else 32):
        most = 0
        for b0 in range(0, batch, 192):  # sequences of a launch
            part = slice(b0, b0 + 192)
            most = max(most, int((n[part].astype(np.int64) * group * H *
                                  ((kv[part].astype(np.int64) + 31) // 32) * 128).sum()))
        assert weighed - plain >= most
    if rows and kv[n > 0].max(initial=0) <= 128:
        assert plain == 0
    assert weighed >= plain


def test_binding_refusals():
    c = dv.Cache(dv.DV_DENSE, 1, 2, 64, 1, [FAKE], elem_bytes=1, max_seq=40)
    qc = attn.QuantCache(c, [SCALE], scale_block=16)
    q = torch.zeros((1, 4, 64), dtype=torch.float16)
    with pytest.raises(ValueError, match="scales has 2 entries"):
        attn.QuantCache(c, [SCALE, SCALE], scale_block=16)
    for bad in (q[0], q.float(), torch.zeros((1, 4, 32), dtype=torch.float16),
                q.transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(ValueError, match="q must be"):
            attn.dv_attend(qc, 0, 0, [1], [4], bad, q, 1.0)
        with pytest.raises(ValueError, match="q must be"):
            attn.dv_attend_bytes(qc, [1], [4], bad)
    with pytest.raises(ValueError, match="out"):
        attn.dv_attend(qc, 0, 0, [1], [4], q, q.bfloat16(), 1.0)
    with pytest.raises(ValueError, match="slopes"):
        attn.dv_attend(qc, 0, 0, [1], [4], q, q.clone(), 1.0, slopes=torch.zeros(3))
    with pytest.raises(ValueError, match="lse"):
        attn.dv_attend(qc, 0, 0, [1], [4], q, q.clone(), 1.0, lse=torch.zeros((1, 4)).double())
    with pytest.raises(ValueError, match="range array"):
        attn.dv_attend(qc, 0, 0, [], [4], q, q.clone(), 1.0)
    with pytest.raises(ValueError, match="kept must be"):
        attn.dv_evict(qc, 0, qc, 0, 0, 1, [4], [2], 0, torch.zeros((1, 1, 2, 4)))
    with pytest.raises(dv.DvError):
        attn.dv_attend(qc, 0, 1, [1], [4], q, q.clone(), 1.0)
