"""Results of matrix instructions are ready some wait states after their products; the compiler keeps the distance, but has been seen to lose it on the
far side of a branch (a sum's last element was read right behind its product and came out wrong).  So the built kernels are looked through: what follows a
product, over all branches, does not read its result within a few instructions."""
import os
import re
import subprocess

import pytest

BUILD = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1606_05688_amd", "_build")
OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
FILES = ("attn_back.hip.o", "attn_window.hip.o", "kv8_attn.hip.o", "linear.hip.o")


def registers(text):
    out = set()
    for m in re.finditer(r"\b([av])\[(\d+):(\d+)\]|\b([av])(\d+)\b", text):
        out |= {(m[1], i) for i in range(int(m[2]), int(m[3]) + 1)} if m[1] else {(m[4], int(m[5]))}
    return out


def least(op):
    """Wait states that a read keeps at the very least (fp32 products of 32 x 32 need 18, 16-bit ones 8 or more)."""
    return 8 if op.startswith("v_mfma_f32_32x32x2_f32") else 4


def early_reads(code):
    """[(product, read)] of a function's [(address, instruction, branch target)] that are too near."""
    index, bad = {a: i for i, (a, _, _) in enumerate(code)}, []
    for i, (_, product, _) in enumerate(code):
        if not product.startswith("v_mfma"):
            continue
        op, operands = product.split(None, 1)
        result, need = registers(operands.split(",")[0]), least(op)
        todo, best = [(i + 1, 0)], {}
        while todo:
            j, waited = todo.pop()
            while j < len(code) and waited < need and best.get(j, need) > waited:
                best[j] = waited
                _, text, target = code[j]
                op = text.split(None, 1)[0]
                if op == "s_endpgm":
                    break
                if op == "s_nop":
                    waited += int(text.split()[1], 0)
                elif target is not None:
                    if target in index:
                        todo.append((index[target], waited + 1))
                    if op == "s_branch":
                        break
                elif op.startswith("v_mfma"):
                    if registers(text.split(None, 1)[1].split(",")[0]) == result:
                        break                                   # the next product of the same sum
                elif not op.startswith("s_") and len(text.split(None, 1)) > 1 and registers(text.split(None, 1)[1]) & result:
                    bad.append((product, text))
                    break
                waited += 1
                j += 1
    return bad


def functions(listing):
    name, start, code = None, 0, []
    for line in listing.splitlines():
        m = re.match(r"^([0-9a-f]+) <(\S+)>:$", line)
        if m:
            if name:
                yield name, code
            name, start, code = m[2], int(m[1], 16), []
            continue
        m = re.match(r"^\s+(\S.*?)\s*// ([0-9A-F]+): [0-9A-F ]+(?:<[^>]*?(?:\+0x([0-9a-f]+))?>)?$", line)
        if m and name:
            branch = m[1].startswith(("s_cbranch", "s_branch"))
            code.append((int(m[2], 16), m[1], start + int(m[3] or "0", 16) if branch else None))
    if name:
        yield name, code


@pytest.mark.parametrize("file", FILES)
def test_results_are_not_read_too_early(file, tmp_path):
    path = os.path.join(BUILD, file)
    if not os.path.exists(path) or not os.path.exists(OBJDUMP):
        pytest.skip("kernels are not built here")
    copy = tmp_path / file
    copy.write_bytes(open(path, "rb").read())
    subprocess.run([OBJDUMP, "--offloading", str(copy)], check=True, capture_output=True)
    (device,) = [p for p in tmp_path.iterdir() if p.name.endswith("gfx950")]
    listing = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(device)], check=True, capture_output=True, text=True).stdout
    products = 0
    for name, code in functions(listing):
        products += sum(text.startswith("v_mfma") for _, text, _ in code)
        assert not early_reads(code), (name, early_reads(code)[:3])
    assert products > 100


def test_what_is_too_early():
    code = [(0, "v_mfma_f32_32x32x2_f32 a[32:47], v68, v71, a[32:47]", None), (8, "s_cbranch_vccnz 3", 24), (12, "v_mov_b32_e32 v1, v2", None),
            (16, "s_nop 15", None), (24, "v_accvgpr_read_b32 v70, a47", None), (32, "s_endpgm", None)]
    assert early_reads(code) == [(code[0][1], code[4][1])]
    assert not early_reads([c for c in code if not c[1].startswith("s_cbranch")])
