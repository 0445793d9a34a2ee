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


def parse(lines):
    """Blocks of a listing: label (or None for what falls through from the one before), instructions, labels that it goes on to."""
    blocks, label, body = [], None, []

    def close(targets, falls):
        nonlocal label, body
        blocks.append((label, body, targets, falls))
        label, body = None, []

    for line in lines:
        line = line.split(";")[0].strip()
        if re.match(r"[.\w$]+:$", line):
            if body or label is not None:
                close([], True)
            label = line[:-1]
            continue
        if not re.match(r"[a-z]\w+(\s|$)", line):
            continue
        body.append(line)
        op = line.split()[0]
        if op.startswith("s_cbranch"):
            close([line.split()[-1]], True)
        elif op == "s_branch":
            close([line.split()[-1]], False)
        elif op in ("s_endpgm", "s_setpc_b64"):
            close([], False)
    if body or label is not None:
        close([], False)
    return blocks


def early_on_any_path(lines):
    """As early(), with what is on its way at the end of a block carried on to every block behind it."""
    blocks = parse(lines)
    at = {b[0]: i for i, b in enumerate(blocks) if b[0] is not None}
    ahead = [[at[t] for t in targets] + ([i + 1] if falls and i + 1 < len(blocks) else []) for i, (_, _, targets, falls) in enumerate(blocks)]
    coming = [{} for _ in blocks]  # the least that has passed, on any path, for each register that has not settled
    found, waiting = set(), set(range(len(blocks)))
    while waiting:
        i = waiting.pop()
        since = dict(coming[i])
        for line in blocks[i][1]:
            op, _, rest = line.replace("\t", " ").partition(" ")
            step = int(rest) + 1 if op == "s_nop" else 1
            if op.startswith("v_mfma"):
                operands = re.split(r",\s*(?![^\[]*\])", rest)
                if registers(operands[1] + " " + operands[2]) & set(since):
                    found.add(line)
            elif op != "s_nop" and registers(rest) & set(since):
                found.add(line)
            since = {r: n + step for r, n in since.items() if n + step < SETTLED}
            if op.startswith("v_mfma"):
                since.update({r: 0 for r in registers(operands[0])})
        for j in ahead[i]:
            less = {r: n for r, n in since.items() if n < coming[j].get(r, SETTLED)}
            if less:
                coming[j].update(less)
                waiting.add(j)
    return sorted(found)


def test_the_check_of_paths_itself():
    product, read = "v_mfma_f32_32x32x16_bf16 a[0:15], v[16:19], v[20:23], a[0:15]", "v_accvgpr_read_b32 v40, a3"
    loop = [".L0:", read, "s_nop 7", product, "s_cbranch_scc1 .L0", "s_nop 15", read, "s_endpgm"]
    assert early_on_any_path(loop) == [read] and not early(loop[:4])
    assert not early_on_any_path(loop[:4] + ["s_nop 15"] + loop[4:])
    skip = [product, "s_cbranch_scc1 .L1", "s_nop 15", ".L1:", read, "s_endpgm"]
    assert early_on_any_path(skip) == [read] and not early(skip)
    assert not early_on_any_path([product, "s_nop 15", "s_branch .L1", read, ".L1:", read, "s_endpgm"])


@pytest.mark.parametrize("source,count", [("dense_backward_bf16.hip", 16), ("dense_backward_far_cap.hip", 8)])
def test_no_result_is_read_early_on_any_path(tmp_path, source, count):
    if not os.path.exists(build.HIPCC):
        pytest.skip("needs the compiler")
    out = tmp_path / "listing.s"
    flags = [f for f in build.FLAGS if f != "-fPIC"]
    subprocess.run([build.HIPCC, *flags, "-S", "--cuda-device-only", os.path.join(build.CSRC, source), "-o", str(out)], check=True, capture_output=True)
    kernels = re.findall(r"^(_ZN\S*dense_d(?:q|kv)_kernel\S*):.*?\n(.*?)^\s*\.section", out.read_text(), re.M | re.S)
    assert len(kernels) == count
    for name, body in kernels:
        lines = body.split("\n")
        assert len(parse(lines)) > 10, name
        found = early_on_any_path(lines)
        assert not found, (name, found[:5])
