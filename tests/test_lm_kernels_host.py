"""The assembly of the matrix loops of cross entropy (CPU only).

Their MFMAs are inline asm, whose results the compiler does not know to wait for: the loops hold if no
accumulator is copied (v_accvgpr_*) or spilled within them, and if the wait states after the last MFMA
stand at the end of the loop. This checks both in the library as it is built.
"""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2310_12298_amd", "libjorge.so")
OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def loops(body):
    """(first, last) line numbers of the innermost loops, from branches backwards."""
    at = {}
    for n, (address, _) in enumerate(body):
        at[address] = n
    found = []
    for n, (address, text) in enumerate(body):
        m = re.match(r"s_cbranch_\w+ (\d+)", text)
        if m:
            off = int(m.group(1))
            target = address + 4 + 4 * (off - 65536 if off > 32767 else off)
            if target in at and at[target] <= n:
                found.append((at[target], n))
    return [a for a in found if not any(b != a and a[0] <= b[0] and b[1] <= a[1] for b in found)]


@pytest.mark.skipif(not (os.path.exists(LIB) and os.path.exists(OBJDUMP)),
                    reason="needs the built library and llvm-objdump")
def test_matrix_loops_neither_copy_nor_spill_accumulators(tmp_path):
    shutil.copy(LIB, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    objects = [f for f in os.listdir(tmp_path) if "gfx950" in f]
    assert objects
    seen = 0
    for f in objects:
        out = subprocess.run([OBJDUMP, "-d", f], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
        for name, code in re.findall(r"^[0-9a-f]+ <(\w+)>:\n(.*?)(?=^[0-9a-f]+ <|\Z)", out, re.S | re.M):
            if not re.search(r"loss_(forward|dz|grad)_kernel", name):
                continue
            body = [(int(m.group(2), 16), " ".join(m.group(1).split()))
                    for m in re.finditer(r"^\t(.*?)\s*// ([0-9A-F]+):", code, re.M)]
            inner = [(a, b) for a, b in loops(body) if any("v_mfma" in t for _, t in body[a:b])]
            assert len(inner) == 1, (name, len(inner))
            a, b = inner[0]
            loop = [t for _, t in body[a:b + 1]]
            mfmas = [n for n, t in enumerate(loop) if t.startswith("v_mfma")]
            assert all(not t.startswith(("v_accvgpr", "scratch_", "buffer_store")) for t in loop), name
            # An MFMA's accumulator is its own result, in place.
            for n in mfmas:
                regs = re.findall(r"a\[\d+:\d+\]", loop[n])
                assert len(regs) == 2 and regs[0] == regs[1], (name, loop[n])
            tail = loop[mfmas[-1] + 1:]
            assert tail.count("s_nop 15") == 2, (name, tail)
            assert sum(t.startswith("v_mfma") for _, t in body) == len(mfmas), f"{name}: an MFMA outside the loop"
            seen += 1
    assert seen == 4 * 2 * 3        # tiles, element types, kernels
