"""Refusals and sizes of the operators over drafted tokens, without a GPU: tensors that no GPU
reaches, and workspaces as large as a verification's pieces."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2403_01876_amd import attn, draft, dv
from tests.test_attn_cpu import FAKE, INVALID, OUT, SCALE, SRC, WORK


class OnDevice(torch.Tensor):
    """A host tensor that says it is on GPU `device`, at a made-up address (that nothing reads)."""

    device_index, at = 0, 0

    def get_device(self):
        return self.device_index

    def is_pinned(self, *a):
        return self.device_index < 0

    def data_ptr(self):
        return self.at


def there(x, at, device=0):
    y = x.as_subclass(OnDevice)
    y.device_index, y.at = device, at
    return y


I32 = dict(dtype=torch.int32)
ADDRESS = {n: FAKE + (i << 36) for i, n in enumerate(
    ("logits", "drawn", "parent", "token", "uniform", "path", "count", "next", "workspace"), 40)}


def verify_tensors():
    x = {"logits": torch.zeros((3, 50)), "drawn": torch.zeros((3, 50)),
         "parent": torch.zeros(3, **I32), "token": torch.zeros(3, **I32),
         "uniform": torch.zeros(3), "path": torch.zeros(3, **I32), "count": torch.zeros(1, **I32),
         "next": torch.zeros(1, **I32), "workspace": torch.zeros(1 << 16, dtype=torch.uint8)}
    return x, {k: there(v, ADDRESS[k]) for k, v in x.items()}


@pytest.fixture
def launched(monkeypatch):
    """Calls that reach the library, with their status there replaced by 0 where the arguments
    hold the address of every tensor: nothing is launched."""
    calls = []

    class Lib:
        def __getattr__(self, name):
            f = getattr(dv.lib, name)

            def call(*args):
                a = next((x._obj for x in args if isinstance(getattr(x, "_obj", None),
                                                            (draft.dv_verify_args,
                                                             attn.dv_attend_args))), None)
                whole = None not in args[2 if name == "dv_verify" else 0:] and \
                    (name != "dv_verify" or a.count is not None)
                calls.append((name, whole))
                return 0 if whole else f(*args)
            return call
    monkeypatch.setattr(draft, "lib", Lib())
    return calls


def test_verify_refuses_tensors_that_no_gpu_reaches(launched):
    host, device = verify_tensors()
    for name in device:
        with pytest.raises(dv.DvError, match=rf"dv_verify \({name}: not in the GPU's memory\)"):
            draft.dv_verify([3], **{**device, name: host[name]})
        assert draft.dv_verify([3], **{**device, name: host[name]}, check=False) == INVALID
        other = there(host[name], ADDRESS[name], 1)  # of another GPU
        with pytest.raises(dv.DvError, match="not in the GPU's memory"):
            draft.dv_verify([3], **{**device, name: other})
        assert not any(whole for _, whole in launched)
    with pytest.raises(dv.DvError, match=r"logits, drawn, parent, token, .* workspace: not in"):
        draft.dv_verify([3], **host)
    assert not any(whole for _, whole in launched)
    assert draft.dv_verify([3], **device) == 0 and launched[-1] == ("dv_verify", True)
    pinned = {k: there(host[k], ADDRESS[k], -1) for k in ("path", "count", "next")}
    assert draft.dv_verify([3], **{**device, **pinned}) == 0 and launched[-1] == ("dv_verify", True)


def dense():
    c = dv.Cache(dv.DV_DENSE, 1, 2, 64, 1, [FAKE], elem_bytes=1, max_seq=40)
    return attn.QuantCache(c, [SCALE], scale_block=16)


def test_attend_tree_refuses_tensors_that_no_gpu_reaches(launched):
    qc = dense()
    q = torch.zeros((2, 4, 64), dtype=torch.float16)
    host = {"parent": torch.zeros(2, **I32), "q": q, "out": q.clone(), "slopes": torch.zeros(4),
            "lse": torch.zeros((2, 4)), "workspace": torch.zeros(1 << 16, dtype=torch.uint8)}
    at = dict(parent=FAKE + (50 << 36), q=SRC, out=OUT, slopes=FAKE + (51 << 36),
              lse=FAKE + (52 << 36), workspace=WORK)
    device = {k: there(v, at[k]) for k, v in host.items()}
    for name in device:
        with pytest.raises(dv.DvError, match=rf"dv_attend_tree \({name}: not in the GPU's memory\)"):
            draft.dv_attend_tree(qc, 0, 0, [2], [4], scale=1.0, **{**device, name: host[name]})
        assert not launched[-1][1]
    assert draft.dv_attend_tree(qc, 0, 0, [2], [4], scale=1.0, **device) == 0


def test_keep_and_out_refuse_tensors_that_no_gpu_reaches(launched):
    qc = dense()
    path, count = torch.zeros(2, **I32), torch.zeros(1, **I32)
    p, n = there(path, FAKE + (60 << 36)), there(count, FAKE + (61 << 36))
    for args, name in (((path, n), "path"), ((p, count), "count"), ((path, count), "path, count")):
        with pytest.raises(dv.DvError, match=rf"dv_keep_path \({name}: not in the GPU's memory\)"):
            draft.dv_keep_path(qc, 0, 0, 1, [2], [4], *args)
        assert not launched[-1][1]
    assert draft.dv_keep_path(qc, 0, 0, 1, [2], [4], p, n) == 0
    wire = torch.zeros(2 * 2 * 4 * 64, dtype=torch.float16)
    with pytest.raises(dv.DvError, match=r"dv_quant_out \(dst: not in the GPU's memory\)"):
        draft.dv_quant_out(qc, 0, 0, 1, [0], [4], wire, wire.numel() * 2, attn.DV_F16)
    with pytest.raises(dv.DvError, match="dst: not in"):
        draft.dv_quant_out(qc, 0, 0, 1, [0], [4], wire.numpy(), wire.numel() * 2, attn.DV_F16)
    assert not any(whole for name, whole in launched if name == "dv_quant_out")
    draft.dv_quant_out(qc, 0, 0, 1, [0], [4], there(wire, SRC), wire.numel() * 2, attn.DV_F16)
    assert launched[-1] == ("dv_quant_out", True)


@pytest.mark.parametrize("V,pieces", [(1, 1), (2041, 1), (2042, 2), (2048, 2), (2049, 2), (4089, 2),
                                      (4090, 3), (32000, 16), (131071, 65), (1 << 24, 8193)])
def test_verify_workspace_of_every_piece(V, pieces):
    """Pieces of 2048 tokens, counted from up to seven tokens before a row's first: 16 bytes
    for each piece of a row and of a sequence, and 4 for a sequence."""
    for batch, q_len in ((1, [1]), (3, [5, 0, 128]), (65, [7] * 65)):
        x = np.array(q_len, np.int32)
        a = draft.dv_verify_args(type=attn.DV_BF16, batch=batch, vocab=V)
        size = ctypes.c_uint64(0)
        assert dv.lib.dv_verify_bytes(x.ctypes.data, ctypes.byref(a), ctypes.byref(size)) == 0
        assert size.value == (sum(q_len) + batch) * pieces * 16 + batch * 4
