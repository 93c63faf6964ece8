"""No instruction reads a matrix product's sums before they are written. The
hardware does not wait by itself: the compiler counts wait states, and where the
last product of a loop is read behind its branch it has been seen to leave two in
place of eight. Read off the assembly of every kernel source with products (CPU
only: hipcc cross-compiles), on every path behind each product."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_04181_amd import build as B

hipcc = pytest.mark.skipif(shutil.which(B.HIPCC) is None, reason="no hipcc")

STORES = ("global_store", "global_atomic", "buffer_store", "flat_store", "scratch_store", "ds_write")


def wait_states(product):
    """Between a product and a reader of its sums: its passes (4 for 16x16 with bf16
    or int8 operands, 8 for 32x32 and for fp32 operands) and 4, with fp32 operands 2."""
    if "16x16x4_f32" in product:
        return 10
    return 8 if "16x16" in product else 12


def registers(text):
    out = set()
    for kind, first, last in re.findall(r"\b([va])\[(\d+):(\d+)\]", text):
        out |= {f"{kind}{i}" for i in range(int(first), int(last) + 1)}
    return out | {k + n for k, n in re.findall(r"\b([va])(\d+)\b", re.sub(r"\[[^\]]*\]", "", text))}


def early_reads(text):
    """(products, [(kernel, product, reader, wait states between)])."""
    n, bad = 0, []
    for m in re.finditer(r"^(\w+):[^\n]*@\1\n.*?^\.Lfunc_end", text, re.S | re.M):
        lines, labels = [], {}
        for line in m.group(0).splitlines()[1:]:
            line = line.split(";")[0].strip()
            if line.endswith(":"):
                labels[line[:-1]] = len(lines)
            elif line and not line.startswith("."):
                lines.append(line)

        def behind(i):
            op = lines[i].split()[0]
            if op == "s_endpgm":
                return []
            if op == "s_branch":
                return [labels[lines[i].split()[1]]]
            return ([labels[lines[i].split()[1]]] if op.startswith("s_cbranch") else []) + [i + 1]

        for i, product in enumerate(lines):
            if not product.startswith("v_mfma"):
                continue
            n += 1
            need = wait_states(product)
            todo = [(j, 0, frozenset(registers(product.split(",")[0]))) for j in behind(i)]
            least = {}
            while todo:
                j, waited, sums = todo.pop()
                if j >= len(lines) or waited >= need or not sums or least.get((j, sums), need) <= waited:
                    continue
                least[j, sums] = waited
                op = lines[j].split()[0]
                args = lines[j][len(op):]
                writes = set() if op.startswith(STORES) else registers(args.split(",")[0])
                reads = registers(args if op.startswith(STORES + ("v_cmp",)) else
                                  args.partition(",")[2])
                if not op.startswith("v_mfma") and reads & sums:  # (products wait for products)
                    bad.append((m.group(1), product, lines[j], waited))
                    continue
                waited += int(args) + 1 if op == "s_nop" else 1
                todo += [(k, waited, sums - writes) for k in behind(j)]
    return n, bad


LOOP = """
kernel:                                 ; @kernel
.LBB0_1:
	v_mfma_i32_16x16x64_i8 a[0:3], v[10:13], v[14:17], a[0:3]
	s_cbranch_scc0 .LBB0_1
; %bb.2:
	s_nop {nop}
	v_accvgpr_read_b32 v10, a3
	s_endpgm
.Lfunc_end0:
"""


def test_the_check_counts_wait_states_behind_a_branch():
    for nop in range(9):
        n, bad = early_reads(LOOP.format(nop=nop))
        assert n == 1
        assert [b[3] for b in bad] == ([] if nop >= 6 else [nop + 2])


@hipcc
def test_every_kernel_waits_for_its_products(tmp_path):
    sources = [s for s in B.SOURCES if s.endswith(".hip") and "mfma" in
               open(os.path.join(B.CSRC, s)).read() + (open(os.path.join(B.CSRC, "gemm_prefill.h")).read()
                                                       if s.startswith("gemm_prefill") else "")]
    assert len(sources) >= 10
    jobs = []
    for s in sources:
        out = tmp_path / (s + ".s")
        cmd = [B.HIPCC, *B.FLAGS, "--cuda-device-only", "-S", os.path.join(B.CSRC, s), "-o", str(out)]
        jobs.append((s, out, subprocess.Popen(cmd, stdout=subprocess.DEVNULL,
                                              stderr=subprocess.PIPE, text=True)))
    for s, out, job in jobs:
        err = job.communicate()[1]
        assert job.returncode == 0, err
        n, bad = early_reads(out.read_text())
        assert n > 0, s
        assert not bad, (s, bad[:5])
