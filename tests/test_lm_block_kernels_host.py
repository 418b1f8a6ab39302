"""The assembly of the matrix loops of the linear and gated layers (CPU only): what test_lm_kernels_host.py checks of
cross entropy's, as their MFMAs are the same inline asm."""
import os
import re
import shutil
import subprocess

import pytest

from test_lm_kernels_host import LIB, OBJDUMP, loops


@pytest.mark.skipif(not (os.path.exists(LIB) and os.path.exists(OBJDUMP)),
                    reason="needs the built library and llvm-objdump")
def test_matrix_loops_neither_copy_nor_spill_accumulators(tmp_path):
    shutil.copy(LIB, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    seen = 0
    for f in (f for f in os.listdir(tmp_path) if "gfx950" in f):
        out = subprocess.run([OBJDUMP, "-d", f], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
        for name, code in re.findall(r"^[0-9a-f]+ <(\w+)>:\n(.*?)(?=^[0-9a-f]+ <|\Z)", out, re.S | re.M):
            if not re.search(r"dense_(forward|dz|grad)_kernel", name):
                continue
            body = [(int(m.group(2), 16), " ".join(m.group(1).split()))
                    for m in re.finditer(r"^\t(.*?)\s*// ([0-9A-F]+):", code, re.M)]
            inner = [(a, b) for a, b in loops(body) if any("v_mfma" in t for _, t in body[a:b])]
            assert len(inner) == 1, (name, len(inner))
            a, b = inner[0]
            loop = [t for _, t in body[a:b + 1]]
            mfmas = [n for n, t in enumerate(loop) if t.startswith("v_mfma")]
            assert all(not t.startswith(("v_accvgpr", "scratch_", "buffer_store")) for t in loop), name
            for n in mfmas:
                regs = re.findall(r"a\[\d+:\d+\]", loop[n])
                assert len(regs) == 2 and regs[0] == regs[1], (name, loop[n])
            assert loop[mfmas[-1] + 1:].count("s_nop 15") == 2, name
            assert sum(t.startswith("v_mfma") for _, t in body) == len(mfmas), f"{name}: an MFMA outside the loop"
            seen += 1
    # Types; linear: four tiles, gated: three, forward and dz; gradients: four tiles, of bfloat16 two ways round.
    assert seen == 2 * 2 * (4 + 3) + 4 + 4 * 2
