"""The built library holds the waits that its matrix products need.

A vector, memory or LDS instruction that reads or writes a product's result, and a product that takes it as an operand, may issue no earlier than
a number of wait states behind it.  The compiler leaves some of them out where a branch lies between (from a product before a jump back
to moves at the loop's head, for one), for which sources have waits of their own: here every kernel is followed along all its paths."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2507_01652_amd import build

# Wait states: the passes of a product (four cycles each) and 4; of fp32 ones, and 2.
NEED = {"v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_32x32x16_bf16": 12, "v_mfma_f32_16x16x4_f32": 10, "v_mfma_f32_32x32x2_f32": 18}


def registers(operand):
    m = re.match(r"-?\|?([va])\[(\d+):(\d+)\]", operand)
    if m:
        return {(m[1], i) for i in range(int(m[2]), int(m[3]) + 1)}
    m = re.match(r"-?\|?([va])(\d+)\b", operand)
    return {(m[1], int(m[2]))} if m else set()


def functions(text):
    """(name, [(instruction, operands, address, offset of a branch's target)]) of each."""
    out = []
    for line in text.splitlines():
        m = re.match(r"^[0-9a-f]+ <(\S+)>:$", line)
        if m:
            out.append((m[1], []))
            continue
        m = re.match(r"^\s+(\w+)\s*(.*?)\s*// ([0-9A-F]+):[ 0-9A-F]*(?:<\S+?(?:\+0x([0-9a-f]+))?>)?\s*$", line)
        if m and out:
            out[-1][1].append((m[1], [x.split(" ")[0] for x in m[2].split(", ")], int(m[3], 16), int(m[4] or "0", 16)))
    return out


def early(code):
    """Instructions that touch a product's result too early: (product, instruction, wait states between)."""
    found, index = [], {c[2] - code[0][2]: i for i, c in enumerate(code)}
    for i, (op, args, _, _) in enumerate(code):
        if "mfma" not in op:
            continue
        need, result, paths, seen = NEED[op], registers(args[0]), [(i + 1, 0)], {}
        while paths:
            at, waited = paths.pop()
            if at >= len(code) or waited >= need or seen.get(at, need) <= waited:
                continue
            seen[at] = waited
            o, a, _, target = code[at]
            assert o not in ("s_setpc_b64", "s_swappc_b64"), "a path that is not followed"
            if o == "s_endpgm":
                continue
            if o == "s_nop":
                waited += int(a[0])
            elif o.startswith(("s_branch", "s_cbranch")):
                paths.append((index[target], waited + 1))
                if o == "s_branch":
                    continue
            elif "mfma" in o:
                if any(registers(x) & result for x in a[1:3]):
                    found.append((i, at, waited))
                    continue
                if registers(a[0]) & result:               # (and as its own sum's beginning: the matrix cores wait)
                    continue
            elif not o.startswith("s_") and any(registers(x) & result for x in a):
                found.append((i, at, waited))
                continue
            paths.append((at + 1, waited + 1))
    return found


def test_waits_behind_products(tmp_path):
    objdump = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
    if not shutil.which(objdump):
        pytest.skip("no llvm-objdump")
    library = shutil.copy(build.LIB, tmp_path)
    subprocess.run([objdump, "--offloading", library], cwd=tmp_path, check=True, stdout=subprocess.DEVNULL)
    objects = [p for p in tmp_path.iterdir() if p.name.endswith("gfx950")]
    disassemble = lambda p: subprocess.run([objdump, "-d", "--mcpu=gfx950", p], check=True, capture_output=True, text=True).stdout
    kernels, bad = set(), []
    with ThreadPoolExecutor(4) as pool:
        for text in pool.map(disassemble, objects):
            for name, code in functions(text):
                if any("mfma" in c[0] for c in code):
                    kernels.add(name)
                    bad += [(name, code[i][:2], code[at][:2], w) for i, at, w in early(code)]
    assert sum("pages_kernel" in k for k in kernels) == 49 and len(kernels) > 150
    assert not bad, (len(bad), bad[:4])


def test_the_search_finds_what_is_missing():
    text = """0000000000001000 <_Zk>:
	s_mov_b32 s0, 0                   // 000000001000: 00000000
	v_mov_b32_e32 v9, v3              // 000000001004: 00000000
	v_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], 0 // 000000001008: 00000000 00000000
	s_nop {0}                         // 000000001010: 00000000
	s_cbranch_scc1 65532              // 000000001014: 00000000 <_Zk+0x4>
	s_nop {1}                         // 000000001018: 00000000
	{2} // 00000000101C: 00000000
	s_endpgm                          // 000000001020: 00000000
"""
    for loop, behind, last, count in ((6, 0, "v_add_f32_e32 v5, v6, v7", 0), (5, 7, "v_add_f32_e32 v5, v2, v7", 1), (6, 0, "v_add_f32_e32 v5, v2, v7", 0),
                                      (0, 0, "global_store_dword v2, v5, s[0:1]", 2), (0, 0, "v_add_f32_e32 v5, v6, v7", 1),
                                      (6, 0, "v_mfma_f32_16x16x32_bf16 v[12:15], v[0:3], v[8:11], 0", 0),
                                      (4, 0, "v_mfma_f32_16x16x32_bf16 v[12:15], v[0:3], v[8:11], 0", 2),
                                      (4, 0, "v_mfma_f32_16x16x32_bf16 v[0:3], v[16:19], v[8:11], v[0:3]", 1)):
        (_, code), = functions(text.format(loop, behind, last))
        assert len(code) == 8 and len(early(code)) == count, (loop, behind, last)
