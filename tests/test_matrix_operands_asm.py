"""Matrix instructions as readers of one another's results: what
test_matrix_waits_asm follows for vector and memory instructions, here for a
matrix instruction that takes an earlier one's result as its A or B operand, or
as an accumulator that is not the same registers.  (The next product of a chain,
accumulator and result the same registers, is handed the sum by the matrix core
itself.)  The same wait states apply as for other readers."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2608_01528_amd import build as B
from test_matrix_waits_asm import NEED, parse, registers


def overlap(a, b):
    return a[0] == b[0] and a[1] <= b[2] and b[1] <= a[2]


def early_products(body):
    """(number of products, matrix instructions that read a result too early)."""
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
        result, need = wrote[0], NEED[op]
        least, todo = {}, [(j, 0) for j in after(i)]
        while todo:
            j, waited = todo.pop()
            if waited >= need or least.get(j, need) <= waited:
                continue
            least[j] = waited
            name, _, _, args = ins[j]
            if name.startswith("v_mfma"):
                d, a, b, c = [registers(p) for p in re.split(r",(?![^\[]*\])", args)[:4]]
                chained = d == c == [result]
                if any(overlap(result, x) for x in a + b) or (not chained and any(overlap(result, x) for x in c)):
                    found.append((op, ins[i][3], name, args, waited))
                    continue
                if chained:             # followed from there
                    continue
            step = int(args, 0) + 1 if name == "s_nop" else 1
            todo += [(k, waited + step) for k in after(j)]
    return products, found


def test_the_check_sees_an_early_operand():
    first = "\tv_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[24:27], v[0:15]\n"
    end = "\ts_endpgm"
    for reader in ("v[40:55], v[12:15], v[24:27], v[40:55]", "v[40:55], v[24:27], v[0:3], v[40:55]",
                   "v[8:23], v[24:27], v[28:31], v[8:23]", "v[0:15], v[4:7], v[24:27], v[0:15]"):
        second = "\tv_mfma_f32_32x32x16_bf16 " + reader + "\n"
        assert early_products(first + second + end)[1], reader
        assert early_products(first + "\ts_cbranch_scc1 .LBB0_1\n\ts_nop 15\n.LBB0_1:\n" + second + end)[1], reader
        assert early_products(first + "\ts_nop 9\n" + second + end)[1], reader                  # 10 states
        assert early_products(first + "\ts_nop 10\n" + second + end) == (2, []), reader         # 11
    chain = "\tv_mfma_f32_32x32x16_bf16 v[0:15], v[24:27], v[28:31], v[0:15]\n"
    apart = "\tv_mfma_f32_32x32x16_bf16 v[40:55], v[24:27], v[28:31], v[40:55]\n"
    assert early_products(first + chain + apart + end) == (3, [])


SOURCES = ["gs_xattn.hip", "gs_xattn_grad.hip"]


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    """The sources' gfx950 assembly, compiled side by side."""
    if not (os.path.exists(B.HIPCC) or shutil.which(B.HIPCC)):
        pytest.skip("hipcc not available")
    room = tmp_path_factory.mktemp("asm")
    runs = [subprocess.Popen([B.HIPCC] + B.FLAGS + ["--cuda-device-only", "-S", "-o", str(room / s), os.path.join(B.CSRC, s)],
                             stdout=subprocess.DEVNULL, stderr=subprocess.PIPE, text=True) for s in SOURCES]
    for r in runs:
        _, err = r.communicate()
        assert r.returncode == 0, err[-2000:]
    return {s: (room / s).read_text() for s in SOURCES}


@pytest.mark.parametrize("source", SOURCES)
def test_operands_wait_for_the_products(source, assembly):
    total = 0
    for name, body in re.findall(r"^(_Z\S*kernel\S*):[^\n]*\n(.*?)^\s*\.section", assembly[source], re.S | re.M):
        products, found = early_products(body)
        assert not found, (name, found[0])
        total += products
    assert total > 0
