"""The paged decoding's matrix products are written in inline assembly, whose latency the compiler does not know:
nothing but a product may touch a product's result within its passes, whatever the compiler puts between them
(spills and moves of accumulators among it).  Checked on the assembly of the library as it was built here."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_27269_amd import _lib as L

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"

# wait states after which any instruction may touch the result of a product: 19 are the most that the
# hardware asks for (a 16-pass product, its result read by the vector ALU)
STATES = 19


def registers(text):
    """The vector and accumulation registers that an operand list names."""
    out = set()
    for m in re.finditer(r"\b([av])\[(\d+):(\d+)\]|\b([av])(\d+)\b", text):
        if m.group(1):
            out |= {(m.group(1), i) for i in range(int(m.group(2)), int(m.group(3)) + 1)}
        else:
            out.add((m.group(4), int(m.group(5))))
    return out


def violations(lines):
    """The instructions (of a listing in the order of the code) that touch a product's result too early, and
    the number of products.  Every instruction counts as one wait state, s_nop k as k + 1.  A branch within the
    wait counts too: what it leads to is not followed."""
    pending, bad, products = {}, [], 0          # register -> (wait states left, the product's result)
    for line in lines:
        op, _, rest = line.strip().partition(" ")
        states = int(rest.split()[0], 0) + 1 if op == "s_nop" else 1
        if op.startswith("v_mfma"):
            products += 1
            d, a, b, c = (frozenset(registers(t)) for t in rest.split(",")[:4])
            # the accumulator goes on from product to product if both have all of it
            if any(r in pending for r in a | b) or any(r in pending and pending[r][1] != c for r in c | d):
                bad.append(line)
        elif pending and (op.startswith(("s_cbranch", "s_branch", "s_setpc", "s_endpgm")) or registers(rest) & set(pending)):
            bad.append(line)
        pending = {r: (n - states, p) for r, (n, p) in pending.items() if n > states}
        if op.startswith("v_mfma"):
            pending.update((r, (STATES, d)) for r in d)
    return bad, products


P = "v_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[24:27], "


@pytest.mark.parametrize("code,bad", [
    ([P + "0", "s_nop 15", "s_nop 2", "v_add_f32_e32 v30, v0, v1"], 0),
    ([P + "0", "s_nop 15", "s_nop 1", "v_add_f32_e32 v30, v0, v1"], 1),            # one state short
    ([P + "0", P + "v[0:15]", "s_nop 15", "s_nop 7", "v_mov_b32_e32 v0, v1"], 0),  # one accumulator
    ([P + "0", "v_mfma_f32_32x32x16_bf16 v[8:23], v[40:43], v[44:47], v[8:23]"], 1),   # half of another's
    ([P + "0", "v_mfma_f32_32x32x16_bf16 a[0:15], v[12:15], v[44:47], a[0:15]"], 1),   # an operand
    ([P + "0", "scratch_store_dword off, v7, s33"], 1),                            # a spill
    ([P + "0", "v_accvgpr_write_b32 a3, v40", "v_mov_b32_e32 v16, v17"], 0),       # other registers
    ([P.replace("v[0:15]", "a[0:15]") + "a[0:15]", "v_accvgpr_read_b32 v40, a15"], 1),
    ([P + "0", "s_cbranch_scc1 65000"], 1),
    ([P + "0"] + ["s_add_u32 s0, s0, s1"] * 19 + ["v_mov_b32_e32 v0, v1"], 0),
    ([P + "0"] + ["s_add_u32 s0, s0, s1"] * 18 + ["v_mov_b32_e32 v0, v1"], 1),
])
def test_the_check_itself(code, bad):
    assert len(violations(code)[0]) == bad


@pytest.mark.skipif(not (os.path.exists(L.LIB_PATH) and os.path.exists(OBJDUMP)),
                    reason="needs the built library and llvm-objdump")
def test_paged_decode_products_are_waited_for(tmp_path):
    lib = shutil.copy(L.LIB_PATH, tmp_path)
    subprocess.run([OBJDUMP, "--offloading", lib], cwd=tmp_path, check=True, stdout=subprocess.DEVNULL)
    kernels = {}
    for f in sorted(tmp_path.glob("*gfx950")):
        names = subprocess.run([OBJDUMP, "-t", f], check=True, capture_output=True, text=True).stdout
        names = sorted(set(re.findall(r"F \.text\s+\S+\s+(?:\.protected )?(\S*paged_decode_kernel\S*)", names)))
        if names:
            text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr",
                                   "--disassemble-symbols=" + ",".join(names), f],
                                  check=True, capture_output=True, text=True).stdout
            for part in re.split(r"^<", text, flags=re.M)[1:]:
                name, _, body = part.partition(">:")
                kernels[name] = [l.split("//")[0] for l in body.splitlines() if l.strip()]
    assert len(kernels) == 3, sorted(kernels)       # one for each width of rows
    for name, lines in kernels.items():
        bad, products = violations(lines)
        print(f"[waits] {name}: {products} products, {len(lines)} instructions")
        dk, dvl = (int(v) for v in re.search(r"ILi(\d+)ELi(\d+)E", name).groups())
        assert products == dk // 16 + dvl // 8 and not bad, (name, products, bad[:5])
