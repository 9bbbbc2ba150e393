"""How far behind a product of the matrix units its result may be read, or written over: the wait states that the compiler keeps on straight code in these
kernels, counted over every way that branches leave (it has been seen to keep them on one way to a read and not on another)."""
import os
import subprocess

import pytest

from test_matrix_waits_host import BUILD, OBJDUMP, functions, registers

# 64, 32, 16 and 32 cycles of the matrix unit, and what its last stages take
NEED = {"v_mfma_f32_32x32x2_f32": 18, "v_mfma_f32_32x32x16_bf16": 12, "v_mfma_f32_32x32x16_f16": 12, "v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_16x16x32_f16": 8,
        "v_mfma_f32_16x16x4_f32": 10}
FILES = ("attn_back.hip.o", "attn_window.hip.o", "kv8_attn.hip.o", "linear.hip.o")


def too_near(code):
    """[(product, what touches its result, wait states between them)] of a function's [(address, instruction, branch target)]."""
    index, bad = {a: i for i, (a, _, _) in enumerate(code)}, []
    for i, (_, product, _) in enumerate(code):
        if not product.startswith("v_mfma"):
            continue
        op, operands = product.split(None, 1)
        result, need = registers(operands.split(",")[0]), NEED[op.removesuffix("_e64")]
        todo, best = [(i + 1, 0)], {}
        while todo:
            j, waited = todo.pop()
            while j < len(code) and waited < need and best.get(j, need) > waited:
                best[j] = waited
                _, text, target = code[j]
                op, _, rest = text.partition(" ")
                if op == "s_endpgm":
                    break
                if op == "s_nop":
                    waited += int(rest, 0)
                elif target is not None:
                    if target in index:
                        todo.append((index[target], waited + 1))
                    if op == "s_branch":
                        break
                elif op.startswith("v_mfma"):
                    to, a, b, c = (registers(x) for x in rest.split(", ")[:4])
                    if (a | b) & result or (c & result and c != result):
                        bad.append((product, text, waited))
                        break
                    if to == result:
                        break                                   # the next product of the same sum
                elif not op.startswith("s_") and registers(rest) & result:
                    bad.append((product, text, waited))
                    break
                waited += 1
                j += 1
    return bad


@pytest.mark.parametrize("file", FILES)
def test_results_are_far_enough_behind_their_products(file, tmp_path):
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
        bad = too_near(code)
        assert not bad, (name, len(bad), bad[:3])
    assert products > 100


def test_what_is_too_near():
    product, nop = "v_mfma_f32_32x32x16_f16 v[22:37], v[74:77], v[42:45], v[22:37]", lambda n: f"s_nop {n}"
    read = "v_maximum3_f32 v76, v25, v29, v29"

    def straight(*between):
        return [(8 * i, text, None) for i, text in enumerate((product, *between, read, "s_endpgm"))]

    assert not too_near(straight(nop(11))) and too_near(straight(nop(10))) == [(product, read, 11)]
    assert not too_near(straight(*["v_mov_b32_e32 v1, v2"] * 12)) and too_near(straight(*["v_mov_b32_e32 v1, v2"] * 11))
    # one way is long enough, the other is not
    ways = [(0, product, None), (8, "s_cbranch_scc0 3", 40), (16, nop(11), None), (40, nop(3), None), (48, read, None), (56, "s_endpgm", None)]
    assert too_near(ways) == [(product, read, 5)]
    # operands of the next product, and sums that overlap
    for other in ("v_mfma_f32_32x32x16_f16 v[40:55], v[22:25], v[90:93], 0", "v_mfma_f32_32x32x16_f16 v[40:55], v[90:93], v[34:37], 0",
                  "v_mfma_f32_32x32x16_f16 v[18:33], v[90:93], v[94:97], v[18:33]"):
        assert too_near([(0, product, None), (8, other, None), (16, nop(15), None), (24, nop(15), None), (32, "s_endpgm", None)]) == [(product, other, 0)]
    assert not too_near([(0, product, None), (8, product, None), (16, nop(11), None), (24, read, None), (32, "s_endpgm", None)])
