"""A matrix product's result is read only after its wait states, on every path of the
assembly that this source compiles to. In straight code the compiler keeps them (8 for
the bf16 product used here, 10 for the float32 one); over the taken side of a branch it
has left three, for v_accvgpr_read behind the products of the join, where a wait of its
own now stands."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2608_18410_amd import build

WAITS = {"v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_16x16x4_f32": 10}


def registers(text):
    out = set()
    for kind, lo, hi, one_kind, one in re.findall(r"\b([va])\[(\d+):(\d+)\]|\b([va])(\d+)\b", text):
        out |= {(kind, i) for i in range(int(lo), int(hi) + 1)} if kind else {(one_kind, int(one))}
    return out


def functions(asm):
    """(name, instructions, where each label stands) of every function."""
    name, ins, labels = None, [], {}
    for line in asm.splitlines():
        line = line.split(";")[0].rstrip()
        if m := re.match(r"(\S+):$", line):
            if m[1].startswith("_Z"):
                name, ins, labels = m[1], [], {}
            labels[m[1]] = len(ins)
        elif name and line.startswith("\t") and not line.startswith("\t."):
            op, _, rest = line.strip().partition(" ")
            op, *more = op.split("\t")
            ins.append((op, [x.strip() for x in re.split(r",(?![^\[]*\])", "".join(more) + rest)]))
        elif line.startswith(".Lfunc_end") or line.startswith("\t.end_amdhsa_kernel"):
            pass
        if line.startswith("\t.size") and name:
            yield name, ins, labels
            name = None


def early_reads(ins, labels):
    """Reads of a product's result before its wait states are over: (product, reader, states)."""
    for i, (op, args) in enumerate(ins):
        if not op.startswith("v_mfma"):
            continue
        need, dst, seen, todo = WAITS[op], registers(args[0]), {}, [(i + 1, 0)]
        while todo:
            j, n = todo.pop()
            if j >= len(ins) or n >= need or seen.get(j, need) <= n:
                continue
            seen[j] = n
            op2, a = ins[j]
            if op2 == "s_nop":
                n += int(a[0], 0)
            elif op2.startswith("v_mfma"):
                if registers(a[0]) >= dst:  # the next product of a chain, which the hardware orders
                    continue
            elif op2.startswith(("v_", "ds_", "global_", "buffer_", "flat_", "scratch_")):
                stores = "store" in op2 or "write" in op2 and op2.startswith("ds_")
                if registers(",".join(a if stores or op2.startswith("v_cmp") else a[1:])) & dst:
                    yield op, op2, n
                    continue
            if op2.startswith(("s_branch", "s_cbranch")):
                todo.append((labels[a[0]], n + 1))
            if op2 not in ("s_branch", "s_endpgm"):
                todo.append((j + 1, n + 1))


def test_the_look_itself():
    asm = "_Zf:\n\tv_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[0:3]\n\ts_cbranch_execnz .L1\n\ts_nop 7\n.L1:\n" \
          "\ts_nop %d\n\tv_accvgpr_read_b32 v4, a3\n\ts_endpgm\n\t.size f\n"
    (_, ins, labels), = functions(asm % 0)
    assert list(early_reads(ins, labels)) == [("v_mfma_f32_16x16x32_bf16", "v_accvgpr_read_b32", 2)]
    (_, ins, labels), = functions(asm % 6)
    assert not list(early_reads(ins, labels))


@pytest.mark.skipif(not shutil.which(build.HIPCC), reason="needs hipcc")
def test_no_result_is_read_early(tmp_path):
    out = str(tmp_path / "k.s")
    r = subprocess.run([build.HIPCC, *build.FLAGS, "-S", "--offload-device-only", os.path.join(build.CSRC, "k_decode.hip"), "-o", out],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    n = 0
    for name, ins, labels in functions(open(out).read()):
        n += sum(op.startswith("v_mfma") for op, _ in ins)
        assert not list(early_reads(ins, labels)), name
    assert n > 1000
