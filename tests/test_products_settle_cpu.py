"""The products that the library's own assembly issues: the compiler, which does not know how long they take, reads no result early."""
import os
import re
import subprocess

import pytest

from paper_2603_08982_amd import build

# Cycles of 4 between a 32 x 32 x 16 product of 16-bit numbers, which takes 8, and another kind of instruction that reads its result or
# writes over it; a product that reads it as an operand waits as long.
SETTLED = 11


def registers(text):
    found = {f"{kind}{i}" for kind, a, b in re.findall(r"\b([va])\[(\d+):(\d+)\]", text) for i in range(int(a), int(b) + 1)}
    return found | {kind + n for kind, n in re.findall(r"\b([va])(\d+)\b", text)}


def early(lines):
    """Instructions that name a register of a product before it has settled, in the order of the listing."""
    since, found = {}, []
    for line in lines:
        line = line.split(";")[0].strip()
        if not re.match(r"[a-z]\w+(\s|$)", line):
            continue
        op, _, rest = line.partition(" ") if " " in line else line.partition("\t")
        step = 1
        if op == "s_nop":
            step = int(rest) + 1
        elif op.startswith("v_mfma"):
            operands = re.split(r",\s*(?![^\[]*\])", rest)
            if registers(operands[1] + " " + operands[2]) & set(since):
                found.append(line)
        elif registers(rest) & set(since):
            found.append(line)
        since = {r: n + step for r, n in since.items() if n + step < SETTLED}
        if op.startswith("v_mfma"):
            since.update({r: 0 for r in registers(operands[0])})
    return found


def test_the_check_itself():
    product = "v_mfma_f32_32x32x16_bf16 v[0:15], v[16:19], a[0:3], v[0:15]"
    assert early([product, "v_mul_f32_e32 v20, v3, v3"]) and early([product, "s_nop 7", "v_mov_b32_e32 v3, v20"])
    assert early([product, product.replace("v[16:19]", "v[12:15]")])
    assert not early([product, product, "s_nop 15", "v_mul_f32_e32 v20, v3, v3"]) and not early([product, "v_mul_f32_e32 v20, v16, v30"])


def test_no_result_is_read_early(tmp_path):
    if not os.path.exists(build.HIPCC):
        pytest.skip("needs the compiler")
    out = tmp_path / "listing.s"
    flags = [f for f in build.FLAGS if f != "-fPIC"]
    subprocess.run([build.HIPCC, *flags, "-S", "--cuda-device-only", os.path.join(build.CSRC, "dense_backward_bf16.hip"), "-o", str(out)],
                   check=True, capture_output=True)
    kernels = re.findall(r"^(_ZN\S*dense_d(?:q|kv)_kernel\S*):.*?\n(.*?)^\s*\.section", out.read_text(), re.M | re.S)
    assert len(kernels) == 16
    for name, body in kernels:
        lines = body.split("\n")
        assert sum("v_mfma" in line for line in lines) >= 48, name
        assert not early(lines), (name, early(lines)[:3])


def test_no_result_is_read_early_with_far_caps(tmp_path):
    if not os.path.exists(build.HIPCC):
        pytest.skip("needs the compiler")
    out = tmp_path / "listing.s"
    flags = [f for f in build.FLAGS if f != "-fPIC"]
    subprocess.run([build.HIPCC, *flags, "-S", "--cuda-device-only", os.path.join(build.CSRC, "dense_backward_far_cap.hip"), "-o", str(out)],
                   check=True, capture_output=True)
    kernels = re.findall(r"^(_ZN\S*dense_d(?:q|kv)_kernel\S*):.*?\n(.*?)^\s*\.section", out.read_text(), re.M | re.S)
    assert len(kernels) == 8
    for name, body in kernels:
        lines = body.split("\n")
        assert sum("v_mfma" in line for line in lines) >= 48, name
        assert not early(lines), (name, early(lines)[:3])
