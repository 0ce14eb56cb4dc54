"""Wait states around the copies that the kernels write as inline assembly.

The compiler pads the instructions that it emits itself, but does not look into
an asm text: a copy to LDS needs one wait state behind a scalar write of M0 (its
LDS address), and a load five behind a vector instruction that writes its scalar
address.  Both are checked in the machine code of the built library.  CPU only."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2510_11292_amd", "liblouiskv.so")
OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def scalar_regs(text):
    out = set()
    for lo, hi, one, name in re.findall(r"\bs\[(\d+):(\d+)\]|\bs(\d+)\b|\b(vcc|m0)\b", text):
        out |= {f"s{i}" for i in range(int(lo), int(hi) + 1)} if lo else {f"s{one}" if one else name}
    return out


def hazards(listing):
    """(what is missing, the two instructions) for every copy or load in a listing, and the number of copies to LDS."""
    found, copies, past = [], 0, []      # past: (written by vector code, registers written, wait states, text)
    for line in listing.splitlines():
        text = line.split("//")[0].strip()
        if not line[:1].isspace() or not re.match(r"[a-z]", text):
            past = [] if text.endswith(":") else past
            continue
        op, _, rest = text.partition(" ")
        ops = [x.strip() for x in rest.split(",")]
        memory = op.startswith(("global_", "buffer_", "scratch_", "flat_"))
        to_lds = memory and ("_lds_" in op or text.endswith(" lds"))
        copies += to_lds

        def missing(states, hit):
            for vector, regs, n, before in reversed(past):
                if states <= 0:
                    return
                if hit(vector, regs):
                    found.append((before, text))
                    return
                states -= n
        if to_lds:
            missing(1, lambda vector, regs: not vector and "m0" in regs)
        if memory:
            reads = scalar_regs(rest)
            missing(5, lambda vector, regs: vector and regs & reads)
        writes = set()
        if op.startswith("v_"):      # the result, and the carry of the forms that have one
            carry = "_co_" in op or op.startswith(("v_mad_u64_u32", "v_mad_i64_i32", "v_div_scale"))
            writes = scalar_regs(", ".join(ops[:2] if carry else ops[:1]))
        elif op.startswith("s_") and op not in ("s_nop", "s_waitcnt", "s_barrier"):
            writes = scalar_regs(ops[0])
        past = past[-8:] + [(op.startswith("v_"), writes, int(ops[0], 0) + 1 if op == "s_nop" else 1, text)]
    return found, copies


def test_the_check_finds_what_is_missing():
    near = "0000 <k>:\n\ts_mov_b32 m0, s4   // 0\n\tglobal_load_lds_dwordx4 v1, s[2:3]\n"
    assert hazards(near) == ([("s_mov_b32 m0, s4", "global_load_lds_dwordx4 v1, s[2:3]")], 1)
    assert hazards(near.replace("\tglobal", "\ts_nop 0\n\tglobal")) == ([], 1)
    late = "\tv_readfirstlane_b32 s3, v0\n\ts_nop 3\n\tglobal_load_dword v1, v2, s[2:3]\n"
    assert len(hazards(late)[0]) == 1 and hazards(late.replace("s_nop 3", "s_nop 4")) == ([], 0)
    assert hazards(late.replace("s3, v0", "s4, v0")) == ([], 0)


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="ROCm toolchain not found")
def test_copies_to_lds_have_their_wait_states(tmp_path):
    assert os.path.exists(LIB), "liblouiskv.so is not built"
    shutil.copy(LIB, tmp_path)
    subprocess.run([OBJDUMP, "--offloading", os.path.basename(LIB)], cwd=tmp_path, check=True, capture_output=True)
    parts = [p for p in sorted(os.listdir(tmp_path)) if p.endswith("gfx950")]
    assert parts
    total = 0
    for p in parts:
        r = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", "--no-show-raw-insn", p], cwd=tmp_path, check=True,
                           capture_output=True, text=True)
        found, copies = hazards(r.stdout)
        assert not found, f"{len(found)} of {copies} copies, such as {found[:3]}"
        total += copies
    assert total > 100      # the k-means sweeps and the prompt attention have them
