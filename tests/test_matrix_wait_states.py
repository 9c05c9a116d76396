"""No result of a matrix instruction is read before it is there, on any way through the attention kernels as this compiler makes
them.  The hardware does not wait by itself: so many instructions (or s_nop cycles) have to lie between."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2604_24073_amd import build

# Wait states from a matrix instruction of the kernels to whatever reads its result but the next one's sum.
NEEDED = {"v_mfma_f32_16x16x4_f32": 10, "v_mfma_f32_16x16x32_bf16": 8}


def operands(text):
    return [x.strip() for x in re.split(r",(?![^\[]*\])", text)] if text else []


def registers(text):
    found = {(m[1], i) for m in re.finditer(r"\b([av])\[(\d+):(\d+)\]", text) for i in range(int(m[2]), int(m[3]) + 1)}
    return found | {(m[1], int(m[2])) for m in re.finditer(r"\b([av])(\d+)\b", text)}


def kernels(assembly):
    """(name, [(instruction, operands, line)], {label: index}) of every function."""
    name, code, labels = None, [], {}
    for number, line in enumerate(assembly.splitlines(), 1):
        line = line.split(";")[0].rstrip()
        if m := re.match(r"(_Z\w+):", line):
            name, code, labels = m[1], [], {}
        elif m := re.match(r"(\.LBB\w+):", line):
            labels[m[1]] = len(code)
        elif line.startswith(".Lfunc_end") and name:
            yield name, code, labels
            name = None
        elif name and (m := re.match(r"\s+([a-z]\w+)\s*(.*)$", line)):
            code.append((m[1], m[2], number))


def early_reads(assembly):
    products, found = 0, []
    for name, code, labels in kernels(assembly):
        for start, (op, args, line) in enumerate(code):
            if not op.startswith("v_mfma"):
                continue
            products += 1
            result, need = registers(operands(args)[0]), NEEDED[op]
            ways, soonest = [(start + 1, 0)], {}
            while ways:
                at, waited = ways.pop()
                while at < len(code) and waited < need and waited < soonest.get(at, need):
                    soonest[at] = waited
                    other, text, where = code[at]
                    parts = operands(text)
                    if other.startswith("v_mfma"):
                        if registers(parts[1] + "," + parts[2]) & result:
                            found.append(f"{name}: line {line}, a factor in line {where} after {waited}")
                        if registers(parts[0] + "," + parts[3]) & result:
                            break                                # goes on with the sum
                    elif registers(text) & result:
                        found.append(f"{name}: line {line}, {other} in line {where} after {waited}")
                        break
                    if other == "s_endpgm":
                        break
                    waited += int(text, 0) + 1 if other == "s_nop" else 1
                    if other.startswith("s_cbranch"):
                        ways.append((labels[text.strip()], waited))
                    at = labels[text.strip()] if other == "s_branch" else at + 1
    return products, found


def sample(between):
    return "_Z1k:\n\tv_mfma_f32_16x16x32_bf16 v[0:3], v[8:11], v[12:15], v[0:3]\n" + between + "\ts_endpgm\n.Lfunc_end0:\n"


@pytest.mark.parametrize("between,early", [
    ("\tv_add_f32_e32 v4, v3, v3\n", True), ("\ts_nop 6\n\tv_add_f32_e32 v4, v3, v3\n", True),
    ("\ts_nop 7\n\tv_add_f32_e32 v4, v3, v3\n", False), ("\tv_add_f32_e32 v4, v5, v5\n", False),
    ("\tv_mfma_f32_16x16x32_bf16 v[0:3], v[8:11], v[12:15], v[0:3]\n\ts_nop 7\n\tglobal_store_dwordx4 v6, v[0:3], s[0:1]\n", False),
    ("\tv_mfma_f32_16x16x32_bf16 v[20:23], v[0:3], v[12:15], v[20:23]\n", True),
    ("\ts_cbranch_scc1 .LBB0_1\n\ts_nop 7\n.LBB0_1:\n\tds_write_b32 v7, v2\n", True),
    ("\ts_nop 7\n\ts_cbranch_scc1 .LBB0_1\n\ts_nop 7\n.LBB0_1:\n\tds_write_b32 v7, v2\n", False),
    ("\ts_branch .LBB0_1\n\ts_nop 7\n.LBB0_1:\n\tv_mov_b32_e32 v9, v0\n", True)])
def test_the_scan_itself(between, early):
    products, found = early_reads(sample(between))
    assert products >= 1 and bool(found) == early


def test_the_attention_kernels(tmp_path):
    def compiled(name):
        out = tmp_path / (name + ".s")
        subprocess.run([build.HIPCC, *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, name + ".hip"), "-o", str(out)],
                       check=True, capture_output=True)
        return out.read_text()

    with ThreadPoolExecutor() as pool:
        for assembly in pool.map(compiled, ("fs_attention", "fs_attention_backward")):
            products, found = early_reads(assembly)
            assert products > 500 and not found, found[:10]
