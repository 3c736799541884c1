"""The compiled attention over pages reads no product's result too early.

The matrix pipe's results are there only some instructions after the product, and it is the compiler that keeps the distance: a
branch between the two has made it miss that once.  The assembly of the kernels as they are built is gone through, over branches too: the
first instruction other than a product that reads a product's result has to come at least eight wait states later, the distance that this
compiler keeps for these products in straight code."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2512_15347_amd import build

NEED = 8


def registers(operand):
    m = re.match(r"^v\[(\d+):(\d+)\]$", operand)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    m = re.match(r"^v(\d+)$", operand)
    return {int(m[1])} if m else set()


def parse(text):
    """[(opcode, operands)] and where labels point; a function ends with an "end"."""
    code, labels = [], {}
    for line in text.splitlines():
        line = line.split(";")[0].rstrip()
        m = re.match(r"^([\w.$]+):", line)
        if m:
            if not m[1].startswith(".L"):
                code.append(("end", []))
            labels[m[1]] = len(code)
            continue
        line = line.strip()
        if line and not line.startswith("."):
            op, _, rest = line.partition(" ")
            op, _, more = op.partition("\t")
            code.append((op, [o.strip().split()[0].strip("-|") for o in (more + rest).split(",") if o.strip()]))
    return code + [("end", [])], labels


def read_by(op, operands):
    stores = op.startswith(("global_store", "ds_write", "buffer_store", "flat_store"))
    return set().union(*[registers(o) for o in (operands if stores else operands[1:])])


def too_early(code, labels):
    """(product, reader, wait states) of every result that is read too early on some path."""
    found = []
    for i, (op, operands) in enumerate(code):
        if "mfma" not in op:
            continue
        paths, seen = [(i + 1, 0, frozenset(registers(operands[0])))], set()
        while paths:
            j, waited, live = paths.pop()
            while waited < NEED and live and (j, waited, live) not in seen:
                seen.add((j, waited, live))
                op, operands = code[j]
                if op in ("end", "s_endpgm"):
                    break
                if op.startswith(("s_cbranch", "s_branch")):
                    target = labels[operands[0]]
                    if op == "s_branch":
                        j, waited = target, waited + 1
                        continue
                    paths.append((target, waited + 1, live))
                elif "mfma" in op:
                    live -= registers(operands[0])
                else:
                    if read_by(op, operands) & live:
                        found.append((i, j, waited))
                        break
                    if operands and not op.startswith(("global_store", "ds_write", "s_")):
                        live -= registers(operands[0])
                waited += int(operands[0]) + 1 if op == "s_nop" else 1
                j += 1
    return found


def test_the_search_finds_an_early_read_behind_a_branch():
    product = "v_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], 0"
    early = f"f:\n\t{product}\n\ts_cbranch_scc1 .LB\n\ts_nop 7\n.LB:\n\tv_mul_f32_e32 v20, v21, v2\n\ts_endpgm\n"
    assert [w for _, _, w in too_early(*parse(early))] == [1]
    assert too_early(*parse(early.replace("\ts_cbranch_scc1 .LB\n", ""))) == []
    assert too_early(*parse(early.replace("v21, v2", "v21, v12"))) == []
    assert [w for _, _, w in too_early(*parse(f"f:\n\t{product}\n\tv_mov_b32_e32 v0, v9\n\tds_write_b32 v30, v1\n"))] == [1]


def test_no_product_is_read_too_early():
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if shutil.which(hipcc) is None:
        pytest.skip("no device compiler")
    flags = [f for f in build.FLAGS if f != "-fPIC"]
    text = subprocess.run([hipcc] + flags + ["-S", "--cuda-device-only", "-o", "-", os.path.join(build.CSRC, "paged_attention.hip")], check=True,
                          capture_output=True, text=True).stdout
    code, labels = parse(text)
    assert sum("mfma" in op for op, _ in code) > 200
    assert too_early(code, labels) == []
