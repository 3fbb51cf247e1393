"""The products of the decoding over either cache format (latent_decode_kernel) are written in inline assembly
like those of the paged decoding: nothing but a product may touch a product's result within its passes.
Checked on the assembly of the library as it was built here."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_27269_amd import _lib as L
from test_matrix_waits import OBJDUMP, violations


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
    assert len(kernels) == 6, sorted(kernels)       # each width of rows in each format
    for name, lines in kernels.items():
        bad, products = violations(lines)
        dk, dvl, e4m3 = (int(v) for v in re.search(r"ILi(\d+)ELi(\d+)ELb(\d)E", name).groups())
        print(f"[waits] {name}: {products} products, {len(lines)} instructions")
        # S once for own rows, twice for shared ones (the first tile's stands before the loop); P V likewise (the last
        # tile's stands behind it)
        assert products == 3 * (dk // 16 + (dvl // 16 if e4m3 else dvl // 8)) and not bad, (name, products, bad[:5])
