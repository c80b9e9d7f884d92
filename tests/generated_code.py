"""Reads the machine code that was built from csrc/: two things that the sources cannot show and no result reliably does.

  short_waits       A load into LDS from inline asm whose scalar base a vector instruction may have written right before.  The hardware wants five wait
                    states between; the compiler does not see into the asm.
  moved_before_exec At the end of a divergent branch or loop the lanes come back by `s_or_b64 exec, exec, ..`.  A copy that register allocation puts
                    in front of it runs for none of them where the block is entered with an empty exec, and the copy holds garbage.
"""
import re
import struct
import subprocess

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def code_objects(library):
    """The device code in a library, one for each translation unit."""
    with open(library, "rb") as f:
        data = f.read()
    found, at = [], data.find(MAGIC)
    while at >= 0:
        count, = struct.unpack_from("<Q", data, at + len(MAGIC))
        p = at + len(MAGIC) + 8
        for _ in range(count):
            offset, size, name = struct.unpack_from("<QQQ", data, p)
            if b"gfx950" in data[p + 24:p + 24 + name]:
                found.append(data[at + offset:at + offset + size])
            p += 24 + name
        at = data.find(MAGIC, at + len(MAGIC))
    return found


def disassembled(path):
    """(function, [(address, instruction, a branch's target or None)]) of a code object."""
    lines = subprocess.run([OBJDUMP, "-d", path], stdout=subprocess.PIPE, check=True, text=True).stdout.splitlines()
    return functions(lines)


def functions(lines):
    name, start, code = None, 0, []
    for line in lines:
        if line.startswith("\t"):
            text, _, note = line.partition("//")
            m = re.match(r"\s*([0-9A-F]+):", note)
            if not m:
                continue
            to = re.search(r"\+0x([0-9a-f]+)>\s*$", note) if text.startswith(("\ts_cbranch", "\ts_branch")) else None
            code.append((int(m[1], 16), text.strip(), start + int(to[1], 16) if to else None))
        else:
            m = re.match(r"([0-9a-f]+) <(.+)>:$", line)
            if m:
                if code:
                    yield name, code
                name, start, code = m[2], int(m[1], 16), []
    if code:
        yield name, code


def short_waits(code):
    """Loads into LDS without their waits: [(address, the instruction)]; and how many loads there are."""
    bad, count = [], 0
    for i, (at, text, _) in enumerate(code):
        if not text.startswith("global_load_lds"):
            continue
        count += 1
        before = re.match(r"s_nop (\d+)", code[i - 1][1]) if i else None
        wanted = 1 if text.endswith(", off") else 5         # (a base in vector registers: M0's alone)
        if not before or int(before[1]) + 1 < wanted:
            bad.append((at, text))
    return bad, count


VECTOR = ("v_", "scratch_", "ds_", "global_", "flat_", "buffer_")
WHOLE = ("v_writelane", "v_readlane", "v_readfirstlane")      # (do not go by exec)
EXEC = re.compile(r"s_\w+ exec\b|s_\w+saveexec")


def moved_before_exec(code):
    """Vector instructions between a place that is entered with an empty exec and the s_or_b64 that fills it: [(address, instruction)]."""
    targets = {to for _, text, to in code if text.startswith("s_cbranch_execz")}
    labels = {to for _, _, to in code if to is not None}
    bad = []
    for i, (at, text, _) in enumerate(code):
        if at not in targets and not (i and code[i - 1][1].startswith("s_cbranch_execnz")):
            continue
        ops = []
        for where, text, _ in code[i:]:
            if where in labels and where != at:         # (another block)
                break
            if EXEC.match(text):
                if text.startswith("s_or_b64 exec, exec"):
                    bad += ops
                break
            if text.startswith(("s_cbranch", "s_branch", "s_endpgm", "s_setpc")):
                break
            if text.startswith(VECTOR) and not text.startswith(WHOLE):
                ops.append((where, text))
    return bad
