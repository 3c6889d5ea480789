"""Every read of a matrix instruction's result in the built kernels waits for it.

The hardware does not: a wave that reads a result register too early gets the old
value. The compiler counts the waits, but was found to leave them out where a
branch lies between (a multiplication moved below one gave outputs without their
last product). So the kernels as built are disassembled and every path after a
matrix instruction is followed to the first read of its result. Runs without a
GPU."""
import glob
import os
import re
import shutil
import subprocess

import pytest

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
# passes (one pass is as long as one wait state), wait states before anything but an accumulation may read the result:
# what the compiler keeps where no branch lies between
MATRIX = {"v_mfma_f32_16x16x32_bf16": (4, 8), "v_mfma_f32_16x16x4_f32": (8, 10)}
NO_RESULT = ("buffer_store", "global_store", "flat_store", "scratch_store", "ds_write", "ds_store", "s_", "v_cmp",
             "buffer_atomic", "global_atomic")


def _registers(text):
    for m in re.finditer(r"\b([va])(\d+)\b|\b([va])\[(\d+):(\d+)\]", text):
        if m[1]:
            yield m[1] + m[2]
        else:
            yield from (m[3] + str(i) for i in range(int(m[4]), int(m[5]) + 1))


def _operands(op, args):
    """(registers written, registers read); the accumulator of a matrix instruction is passed on inside and not counted."""
    a = [set(_registers(x)) for x in re.split(r",(?![^\[]*\])", args)]
    if op in MATRIX:
        return a[0], a[1] | a[2]
    if op.startswith(NO_RESULT) or args.endswith(" lds"):
        return set(), set().union(*a)
    return a[0], set().union(*a[1:])


def early_reads(lines):
    """Pairs of a matrix instruction and a too early read of its result in a function's disassembly."""
    ins, label = [], {}
    for line in lines:
        m = re.match(r"<(\w+)>:", line)
        if m:
            label[m[1]] = len(ins)
        elif line.strip():
            op, _, args = line.split("//")[0].strip().partition(" ")
            ins.append((op, args.strip()))
    ops = [_operands(*i) for i in ins]
    found = []
    for i, (op, _) in enumerate(ins):
        assert not op.startswith("v_mfma") or op in MATRIX, f"{op}: its waits are not known here"
        if op not in MATRIX:
            continue
        passes, need = MATRIX[op]
        # from here: next instruction, wait states so far, result registers not overwritten, wait states with the matrix unit busy
        todo, seen = [(i + 1, 0, frozenset(ops[i][0]), passes - 1)], {}
        while todo:
            j, waited, live, busy = todo.pop()
            while j < len(ins) and live and waited < need:
                if seen.get((j, live), need) <= waited:
                    break
                seen[(j, live)] = waited
                o, args = ins[j]
                written, read = ops[j]
                if o in MATRIX:
                    waited = max(waited, busy)
                    busy = waited + MATRIX[o][0]
                if live & read and waited < need:
                    found.append((" ".join(ins[i]), " ".join(ins[j]), waited))
                    break
                live -= written
                waited += int(args, 0) + 1 if o == "s_nop" else 1
                if o in ("s_endpgm", "s_setpc_b64"):
                    break
                if o.startswith(("s_branch", "s_cbranch")):
                    to = label[args.split()[0]]
                    if o == "s_branch":
                        j = to
                        continue
                    todo.append((to, waited, live, busy))
                j += 1
    return found


def test_early_reads_are_found():
    mfma = "v_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], v[0:3]"
    use = "v_mul_f32_e32 v20, v3, v21"
    assert early_reads([mfma, use]) and early_reads([mfma, "s_nop 6", use])
    assert not early_reads([mfma, "s_nop 7", use])
    assert early_reads([mfma, "s_cbranch_vccnz L0", "s_nop 7", "s_nop 7", "<L0>:", "v_mov_b32_e32 v0, 0", use])
    assert not early_reads([mfma, "s_cbranch_vccnz L0", "s_nop 7", "<L0>:", "s_nop 6", use])
    assert not early_reads([mfma, "v_mov_b32_e32 v3, 0", use])  # overwritten
    assert not early_reads([mfma, mfma, mfma, "s_nop 7", use])
    assert early_reads([mfma, "buffer_store_dwordx4 v[0:3], v12, s[0:3], 0 offen"])
    assert early_reads([mfma, "v_mfma_f32_16x16x32_bf16 v[20:23], v[0:3], v[8:11], 0"])
    assert early_reads(["<L0>:", use, mfma, "s_cbranch_scc1 L0"])


def test_kernels_wait_for_their_matrix_instructions(built_lib, tmp_path):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    shutil.copy(built_lib, tmp_path)
    subprocess.run([OBJDUMP, "--offloading", os.path.basename(built_lib)], cwd=tmp_path, check=True, capture_output=True)
    objects = sorted(glob.glob(str(tmp_path / "*gfx950")))
    assert objects
    early, functions = [], 0
    for o in objects:
        text = subprocess.run([OBJDUMP, "-d", "--symbolize-operands", "--no-show-raw-insn", "--no-leading-addr", o],
                              check=True, capture_output=True, text=True).stdout
        for name, body in re.findall(r"^<(_Z\w+)>:\n(.*?)(?=^<_Z|\Z)", text, re.M | re.S):
            functions += "v_mfma" in body
            early += [(name, *e) for e in early_reads(body.splitlines())]
    print(f"{functions} functions with matrix instructions")
    assert functions > 50
    assert not early, early[:5]
