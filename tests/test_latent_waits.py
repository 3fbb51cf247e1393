"""The products of the decoding over either cache format (latent_decode_kernel) are written in inline assembly
like those of the paged decoding: nothing but a product may touch a product's result within its passes, and
their operands are written two wait states before them or earlier (where the vector ALU writes them).
Checked on the assembly of the library as it was built here."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_27269_amd import _lib as L
from test_matrix_waits import OBJDUMP, registers, violations

OPERAND_STATES = 2


def written_late(lines):
    """The products one of whose operands the vector ALU wrote less than OPERAND_STATES before."""
    age, bad = {}, []                             # register -> wait states since it was written
    for line in lines:
        op, _, rest = line.strip().partition(" ")
        states = int(rest.split()[0], 0) + 1 if op == "s_nop" else 1
        if op.startswith("v_mfma"):
            used = set().union(*(registers(t) for t in rest.split(",")[1:4]))
            if any(age.get(r, OPERAND_STATES) < OPERAND_STATES for r in used):
                bad.append(line)
        age = {r: n + states for r, n in age.items() if n + states < OPERAND_STATES}
        if op.startswith("v_") and not op.startswith("v_mfma"):
            out = rest.split(",")
            for t in out[:2] if "swap" in op else out[:1]:
                age.update((r, 0) for r in registers(t))
    return bad


@pytest.mark.parametrize("code,bad", [
    (["v_mov_b32_e32 v20, v1", "v_mfma_f32_32x32x16_f16 a[0:15], v[20:23], v[24:27], a[0:15]"], 1),
    (["v_mov_b32_e32 v20, v1", "s_nop 0", "v_mfma_f32_32x32x16_f16 a[0:15], v[20:23], v[24:27], a[0:15]"], 1),
    (["v_mov_b32_e32 v20, v1", "s_nop 1", "v_mfma_f32_32x32x16_f16 a[0:15], v[20:23], v[24:27], a[0:15]"], 0),
    (["v_mov_b32_e32 v27, v1", "s_add_u32 s0, s0, s1", "v_mov_b32_e32 v30, v1",
      "v_mfma_f32_32x32x16_f16 a[0:15], v[20:23], v[24:27], a[0:15]"], 0),
    (["v_accvgpr_write_b32 a3, v40", "v_mfma_f32_32x32x16_f16 a[0:15], v[20:23], v[24:27], a[0:15]"], 1),
    (["v_permlane32_swap_b32_e32 v1, v24", "v_mfma_f32_32x32x16_f16 a[0:15], v[20:23], v[24:27], a[0:15]"], 1),
    (["v_mov_b32_e32 v28, v20", "v_mfma_f32_32x32x16_f16 a[0:15], v[20:23], v[24:27], a[0:15]"], 0),
])
def test_the_check_of_operands(code, bad):
    assert len(written_late(code)) == bad


@pytest.mark.skipif(not (os.path.exists(L.LIB_PATH) and os.path.exists(OBJDUMP)),
                    reason="needs the built library and llvm-objdump")
def test_latent_decode_products_are_waited_for(tmp_path):
    lib = shutil.copy(L.LIB_PATH, tmp_path)
    subprocess.run([OBJDUMP, "--offloading", lib], cwd=tmp_path, check=True, stdout=subprocess.DEVNULL)
    kernels = {}
    for f in sorted(tmp_path.glob("*gfx950")):
        names = subprocess.run([OBJDUMP, "-t", f], check=True, capture_output=True, text=True).stdout
        names = sorted(set(re.findall(r"F \.text\s+\S+\s+(?:\.protected )?(\S*latent_decode_kernel\S*)", names)))
        if names:
            text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr",
                                   "--disassemble-symbols=" + ",".join(names), f],
                                  check=True, capture_output=True, text=True).stdout
            for part in re.split(r"^<", text, flags=re.M)[1:]:
                name, _, body = part.partition(">:")
                kernels[name] = [l.split("//")[0] for l in body.splitlines() if l.strip()]
    assert len(kernels) == 12, sorted(kernels)      # each width of rows in each format, with and without images
    for name, lines in kernels.items():
        bad, products = violations(lines)
        dk, dvl, e4m3, images = (int(v) for v in re.search(r"ILi(\d+)ELi(\d+)ELb(\d)ELi\dELb(\d)E", name).groups())
        print(f"[waits] {name}: {products} products, {len(lines)} instructions")
        # S once for own rows, twice for shared ones (the first tile's stands before the loop); P V likewise (the last
        # tile's stands behind it), with two products a piece where the weights are bf16
        own, fp16 = dk // 16 + (dvl // 16 if e4m3 else dvl // 8), dk // 16 + dvl // 16
        assert products == own + 2 * (fp16 if images else own) and not bad, (name, products, bad[:5])
        late = written_late(lines)
        assert not late, (name, late[:5])
