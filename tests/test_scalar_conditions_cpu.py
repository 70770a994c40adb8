"""The compiled kernels select scalars by a condition that a comparison has set.

Of the lesser of two 64-bit numbers that are the same in a whole wave, under a branch on the same comparison, the compiler compares in the
vector unit, and then selects by the scalar unit's condition bit, which holds the borrow of the subtraction before it: a length that was to
be cut to what is left of an array is not cut.  Looked for in the library that the build made: a scalar select or branch behind scalar
arithmetic, where it is not the extraction of a carry."""
import os
import re
import struct
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2107_01499_amd", "lib", "libbagua_hip.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
LLVM = os.path.join(os.path.dirname(os.path.dirname(HIPCC)), "llvm", "bin")

READS = re.compile(r"s_cselect_|s_cbranch_scc|s_cmov")
SETS = re.compile(r"s_(cmp|cmpk|bitcmp|and|or|xor|andn2|orn2|nand|nor|xnor|not)")       # a comparison, or a mask that is not empty
WRITES = re.compile(r"s_(add|addc|sub|subb|addk|cmp|cmpk|bitcmp|and|or|xor|andn2|orn2|nand|nor|xnor|not|lshl|lshr|ashr|bfe|min|max|abs|absdiff|bcnt|wqm)")
CARRY = re.compile(r"s_cselect_b64 \S+, -1, 0$")


def wrong_conditions(lines):
    """(kernel, instruction, what set the condition), and how many instructions read it, of a disassembly."""
    found, count, kernel, last = [], 0, None, ""
    for line in lines:
        head = re.match(r"[0-9a-f]+ <(.+)>:", line)
        if head:
            kernel, last = head[1], ""
            continue
        text = line.split("//")[0].strip()
        if READS.match(text):
            count += 1
            if last and not SETS.match(last) and not CARRY.match(text):
                found.append((kernel, text, last))
        if WRITES.match(text):
            last = text
        elif text.startswith(("s_branch", "s_endpgm")):     # (behind a conditional branch the condition is still the one it was)
            last = ""
    return found, count


def test_the_rule_sees_a_select_by_a_borrow():
    ours = ["0 <k>:", "s_subb_u32 s17, s7, s11 // 0", "v_cmp_lt_u64_e32 vcc, s[16:17], v[2:3]", "s_cbranch_vccz 38", "s_cselect_b32 s1, s16, 0x100"]
    assert wrong_conditions(ours) == ([("k", "s_cselect_b32 s1, s16, 0x100", "s_subb_u32 s17, s7, s11")], 1)
    assert wrong_conditions(ours[:4] + ["s_and_b64 s[2:3], vcc, exec"] + ours[4:]) == ([], 1)
    assert wrong_conditions(ours[:2] + ["s_cselect_b64 s[8:9], -1, 0"]) == ([], 1)


def test_no_kernel_selects_by_a_carry(tmp_path):
    fat, co = str(tmp_path / "fatbin"), str(tmp_path / "co")
    subprocess.run([os.path.join(LLVM, "llvm-objcopy"), "--dump-section", ".hip_fatbin=" + fat, LIB, os.devnull], check=True)
    with open(fat, "rb") as f:
        data = f.read()
    found, count = [], 0
    for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data):     # one bundle per source file
        at = m.start() + 32
        for _ in range(struct.unpack_from("<Q", data, m.start() + 24)[0]):
            offset, size, name = struct.unpack_from("<QQQ", data, at)
            target = data[at + 24:at + 24 + name]
            at += 24 + name
            if b"gfx950" not in target or not size:
                continue
            with open(co, "wb") as f:
                f.write(data[m.start() + offset:m.start() + offset + size])
            text = subprocess.run([os.path.join(LLVM, "llvm-objdump"), "-d", "--no-show-raw-insn", "--no-leading-addr", co], capture_output=True, text=True, check=True).stdout
            wrong, reads = wrong_conditions(text.splitlines())
            found, count = found + wrong, count + reads
    assert count > 10000
    assert found == []
