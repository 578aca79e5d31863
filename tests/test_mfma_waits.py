"""The built library, disassembled: what reads or overwrites the result of a matrix instruction comes late enough.

The hardware does not hold an instruction back until a matrix result is there; the compiler counts the instructions in between and puts
s_nop where there are too few.  It miscounts at times behind a branch: the first read of a block then comes 3 to 7 states behind the last
product, and finds what was there before.  Needed are, in states of four clocks between the two: passes + 4 of the bf16 instructions
(8 passes of 32x32x16, 4 of 16x16x32), passes + 2 of the fp32 ones.  An instruction is one state, s_nop n is n + 1, a matrix instruction waits
until the one before is through.  Branches that are taken and waits for memory are longer in truth: what is found here may go well, and
nothing says that it does."""
import glob
import os
import re
import shutil
import subprocess

import pytest

from paper_1910_00932_amd.build import LIB_PATH

TOOL = shutil.which("llvm-objdump") or "/opt/rocm/llvm/bin/llvm-objdump"
NEED = {"v_mfma_f32_32x32x16_bf16": (8, 12), "v_mfma_f32_16x16x32_bf16": (4, 8), "v_mfma_f32_16x16x4_f32": (8, 10), "v_mfma_f32_32x32x2_f32": (16, 18)}
LINE = re.compile(r"^\s+(\S[^/]*?)\s*// ([0-9A-F]{12}): [0-9A-F ]+(?:<[^>]*?(?:\+0x([0-9a-f]+))?>)?")
REG = re.compile(r"\b([va])\[(\d+):(\d+)\]|\b([va])(\d+)\b")


def _regs(text):
    out = set()
    for kind, lo, hi, one, at in REG.findall(text):
        out |= {(kind, i) for i in range(int(lo), int(hi) + 1)} if kind else {(one, int(at))}
    return out


def _functions(listing):
    """(name, [(mnemonic, operands, branch target's index or None)]) of every function."""
    for part in re.split(r"\n(?=[0-9a-f]{16} <)", listing):
        head = re.match(r"\s*([0-9a-f]{16}) <(.*?)>:", part)
        if not head:
            continue
        base, rows = int(head.group(1), 16), []
        for line in part.split("\n")[1:]:
            m = LINE.match(line)
            if m:
                op, _, rest = m.group(1).partition(" ")
                rows.append((op, rest, int(m.group(2), 16), m.group(3)))
        at = {address: i for i, (_, _, address, _) in enumerate(rows)}
        yield head.group(2), [(op, rest, at.get(base + int(to or "0", 16)) if "branch" in op else None) for op, rest, _, to in rows]


def _after(code, i):
    op, _, to = code[i]
    if op == "s_branch":
        return [to] if to is not None else []
    if op.startswith(("s_endpgm", "s_setpc")):
        return []
    return [k for k in (i + 1, to) if k is not None and k < len(code)]


def early_reads(code):
    """(index, index, states): a matrix instruction, and what touches its result too early."""
    found = []
    for i, (op, rest, _) in enumerate(code):
        if not op.startswith("v_mfma"):
            continue
        passes, need = NEED[op]
        result = _regs(rest.split(",")[0])
        best, todo = {}, [(k, 0) for k in _after(code, i)]
        while todo:
            j, d = todo.pop()
            if d >= need or best.get(j, need) <= d:
                continue
            best[j] = d
            other, args, _ = code[j]
            if other.startswith("v_mfma"):
                d = max(d, passes)                                   # (issued when the one before is through)
                to, a, b = args.split(",")[:3]
                if d < need and _regs(a + b) & result:
                    found.append((i, j, d))
                if _regs(to) & result:
                    continue                                         # adds to it: the result is that one's now
            elif other.startswith(("v_", "ds_", "buffer_", "global_", "flat_", "scratch_")) and _regs(args) & result:
                found.append((i, j, d))
                continue
            d += int(args, 0) + 1 if other == "s_nop" else 1
            todo += [(k, d) for k in _after(code, j)]
    return found


def _code(text):
    """A listing by hand: `name:` lines are branch targets."""
    lines, at = [], {}
    for line in filter(None, (raw.strip() for raw in text.split("\n"))):
        if line.endswith(":"):
            at[line[:-1]] = len(lines)
        else:
            lines.append(line.partition(" "))
    return [(op, rest, at[rest] if "branch" in op else None) for op, _, rest in lines]


MFMA = "v_mfma_f32_32x32x16_bf16 v[2:17], v[20:23], v[24:27], v[2:17]\n"


@pytest.mark.parametrize("text,states", [
    (MFMA + "v_add_f32_e32 v30, v30, v2", 0),
    (MFMA + "s_nop 10\nv_add_f32_e32 v30, v30, v2", 11),
    (MFMA + "s_nop 11\nv_add_f32_e32 v30, v30, v2", None),
    (MFMA + "s_nop 2\nv_mov_b32_e32 v9, 0", 3),
    (MFMA + "s_nop 2\nv_mov_b32_e32 v19, 0", None),
    (MFMA + MFMA + "s_nop 11\nv_add_f32_e32 v30, v30, v2", None),
    (MFMA + "v_mfma_f32_32x32x16_bf16 v[40:55], v[20:23], v[24:27], v[40:55]\ns_nop 1\nv_add_f32_e32 v30, v30, v2", 11),
    (MFMA + "v_mfma_f32_32x32x16_bf16 v[40:55], v[2:5], v[24:27], v[40:55]\ns_nop 15", 8),
    (MFMA + "s_cbranch_scc1 far\ns_nop 11\nv_add_f32_e32 v30, v30, v2\ns_endpgm\nfar:\ns_nop 3\nds_write_b32 v0, v5", 5),
])
def test_the_search_itself(text, states):
    found = early_reads(_code(text))
    assert [d for _, _, d in found] == ([] if states is None else [states])


@pytest.mark.skipif(not os.path.exists(TOOL), reason="no disassembler")
def test_no_matrix_result_is_touched_before_it_is_there(tmp_path):
    shutil.copy(LIB_PATH, tmp_path / "lib.so")
    subprocess.run([TOOL, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    objects = sorted(glob.glob(str(tmp_path / "lib.so.*gfx950*")))
    assert len(objects) > 5
    products, bad = 0, []
    for path in objects:
        listing = subprocess.run([TOOL, "-d", path], check=True, capture_output=True, text=True).stdout
        for name, code in _functions(listing):
            products += sum(op.startswith("v_mfma") for op, _, _ in code)
            bad += [(name, d, " ".join(code[i][:2]), " ".join(code[j][:2])) for i, j, d in early_reads(code)]
    assert products > 5000, "the listing was not understood"
    assert not bad, "\n".join(map(str, bad))
