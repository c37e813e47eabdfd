"""Wait states after matrix products, in the assembly of the attention kernels.

The compiler puts a wait between a product and the first read of its result.  ROCm
7.2 counts it along one path only where an `if` without `else` lies between, so
the kernels end the wait themselves before they branch; this walks every path of
the assembly after every product and looks for a touch that comes too early.
"""
import os
import re
import subprocess

import pytest

pytestmark = pytest.mark.slow

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = os.path.join(ROOT, "paper_2403_01876_amd", "csrc", "dv_attend.hip")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# passes + 4: four passes for 16x16x32, eight for 32x32x16
NEED = {"16x16x32": 8, "32x32x16": 12}
REG = re.compile(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+))")


def registers(text):
    out = set()
    for m in REG.finditer(text):
        a, b = (int(m[2]), int(m[3])) if m[2] else (int(m[4]), int(m[4]))
        out |= {(m[1], i) for i in range(a, b + 1)}
    return out


def kernels(text):
    name, body = None, []
    for line in text.splitlines():
        m = re.match(r"(_Z\w+):", line)
        if m:
            name, body = m[1], []
        elif line.startswith(".Lfunc_end"):
            yield name, body
            name = None
        elif name:
            body.append(line)


def too_early(body):
    """(number of products, those whose result is touched too early)."""
    ins, labels = [], {}
    for line in body:
        line = line.split(";")[0].strip()
        m = re.match(r"(\.L\w+):", line)
        if m:
            labels[m[1]] = len(ins)
        elif line and not line.startswith("."):
            ins.append(line)

    def successors(i):
        op = ins[i].split()
        if op[0] == "s_endpgm":
            return []
        if op[0] == "s_branch":
            return [labels[op[1]]]
        if op[0].startswith("s_cbranch"):
            return [i + 1, labels[op[1]]]
        return [i + 1] if i + 1 < len(ins) else []

    products, found = 0, []
    for i, text in enumerate(ins):
        m = re.match(r"v_mfma_f32_(\w+?)_", text)
        if not m:
            continue
        products += 1
        result = registers(text.split(None, 1)[1].split(",")[0])
        best, todo = {}, [(j, 0) for j in successors(i)]
        while todo:
            j, states = todo.pop()
            if states >= NEED[m[1]] or best.get(j, 99) <= states:
                continue
            best[j] = states
            op, _, rest = ins[j].partition(" ")
            if not op.startswith("s_") and registers(rest) & result:
                if op.startswith("v_mfma"):  # accumulating on it, or replacing it, is in order
                    factors = re.findall(r"[va]\[\d+:\d+\]|\b0\b", rest)[1:3]
                    if registers(" ".join(factors)) & result:
                        found.append((text, ins[j], states))
                else:
                    found.append((text, ins[j], states))
                continue
            waits = int(rest, 0) + 1 if op == "s_nop" else 1
            todo += [(k, states + waits) for k in successors(j)]
    return products, found


def test_the_check_sees_an_early_read():
    body = """
        v_mfma_f32_32x32x16_f16 a[0:15], v[0:3], v[4:7], 0
        s_cbranch_vccnz .LBB0_2
        s_nop 15
    .LBB0_2:
        v_accvgpr_read_b32 v9, a15
        s_endpgm""".replace("    .LBB", ".LBB").splitlines()
    assert too_early(body)[0] == 1 and len(too_early(body)[1]) == 1
    body.insert(2, "    s_nop 10")
    assert too_early(body) == (1, [])


def test_no_result_is_touched_too_early(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("ROCm compiler not installed")
    out = tmp_path / "attend.s"
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
                    "-fvisibility=hidden", "-Xclang", "-target-feature", "-Xclang",
                    "-packed-fp32-ops", "-c", "-x", "hip", "--cuda-device-only", "-S", SOURCE,
                    "-o", str(out)], check=True, capture_output=True, timeout=900)
    total = 0
    for name, body in kernels(out.read_text()):
        n, found = too_early(body)
        total += n
        assert not found, (name, found[:3])
    assert total > 500
