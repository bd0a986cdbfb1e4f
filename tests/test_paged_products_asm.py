"""The waits between matrix instructions and what reads their results, as
test_matrix_waits_asm and test_matrix_operands_asm follow them, in the paged
attention's compiled code: vector and memory instructions, and other matrix
instructions' A and B operands and accumulators that are other registers.  An
accumulator of exactly the registers of the result is handed over by the matrix
core itself, also where the sum goes to new registers."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2608_01528_amd import build as B
from test_matrix_operands_asm import overlap
from test_matrix_waits_asm import NEED, parse, registers

# 4 passes and 3 states more (bf16; 8 and 3 are test_matrix_waits_asm's 11), 8 and 2
# more (fp32; 16 and 2 its 18)
NEEDED = dict(NEED, v_mfma_f32_16x16x32_bf16=7, v_mfma_f32_16x16x4_f32=10)


def early(body):
    ins, labels = parse(body)

    def after(i):
        op, args = ins[i][0], ins[i][3]
        if op == "s_endpgm":
            return []
        jump = [labels[args.split()[0]]] if op.startswith(("s_branch", "s_cbranch")) else []
        return jump + ([] if op == "s_branch" or i + 1 == len(ins) else [i + 1])

    products, found = 0, []
    for i, (op, wrote, _, _) in enumerate(ins):
        if not op.startswith("v_mfma"):
            continue
        products += 1
        result, need = wrote[0], NEEDED[op]
        least, todo = {}, [(j, 0) for j in after(i)]
        while todo:
            j, waited = todo.pop()
            if waited >= need or least.get(j, need) <= waited:
                continue
            least[j] = waited
            name, _, read, args = ins[j]
            if name.startswith("v_mfma"):
                d, a, b, c = [registers(p) for p in re.split(r",(?![^\[]*\])", args)[:4]]
                read = a + b + (c if c != [result] else [])
                if c == [result] and d == c and not any(overlap(result, x) for x in read):
                    continue            # the chain goes on: followed from there
            if any(overlap(result, x) for x in read):
                found.append((op, ins[i][3], name, args, waited))
                continue
            step = int(args, 0) + 1 if name == "s_nop" else 1
            todo += [(k, waited + step) for k in after(j)]
    return products, found


def test_the_check_sees_early_readers():
    first = "\tv_mfma_f32_16x16x4_f32 v[0:3], v20, v21, v[0:3]\n"
    end = "\tv_mov_b32_e32 v30, v2\n\ts_endpgm"
    assert early(first + "\ts_nop 8\n" + end)[1] and not early(first + "\ts_nop 9\n" + end)[1]
    # a sum into new registers: handed over, but the first result still has to be waited for
    moved = "\tv_mfma_f32_16x16x4_f32 v[8:11], v22, v23, v[0:3]\n"
    assert [x[0] for x in early(first + moved + "\ts_nop 7\n" + end)[1]] == ["v_mfma_f32_16x16x4_f32"]
    assert not early(first + moved + "\ts_nop 8\n" + end)[1]
    for reader in ("v[8:11], v2, v23, v[8:11]", "v[8:11], v22, v0, v[8:11]", "v[8:11], v22, v23, v[2:5]"):
        second = "\tv_mfma_f32_16x16x4_f32 " + reader + "\n\ts_endpgm"
        assert early(first + second)[1] and early(first + "\ts_nop 8\n" + second)[1] and not early(first + "\ts_nop 9\n" + second)[1]


def test_readers_and_operands_wait_for_the_products(tmp_path):
    if not (os.path.exists(B.HIPCC) or shutil.which(B.HIPCC)):
        pytest.skip("hipcc not available")
    out = str(tmp_path / "code.s")
    r = subprocess.run([B.HIPCC] + B.FLAGS + ["--cuda-device-only", "-S", "-o", out,
                                              os.path.join(B.CSRC, "gs_paged_attn.hip")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    total, text = 0, open(out).read()
    assert all(op in text for op in NEEDED)
    for name, body in re.findall(r"^(_Z\S*kernel\S*):[^\n]*\n(.*?)^\s*\.section", text, re.S | re.M):
        products, found = early(body)
        assert not found, (name, found[0])
        total += products
    assert total > 0
