"""The machine code of the built library, as instructions that know which ones can run before and after them: for checks of what hand-written assembly has to keep."""
import os
import re
import shutil
import struct
import subprocess

from launches import LIB

OBJDUMP = next((p for p in ("/opt/rocm/llvm/bin/llvm-objdump", shutil.which("llvm-objdump")) if p and os.path.exists(p)), None)
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def code_objects(lib=LIB):
    """The gfx950 ELF images in the library, one of each source."""
    data, at = open(lib, "rb").read(), 0
    while (at := data.find(MAGIC, at)) >= 0:
        count, = struct.unpack_from("<Q", data, at + len(MAGIC))
        p = at + len(MAGIC) + 8
        for _ in range(count if count < 8 else 0):
            offset, size, n = struct.unpack_from("<QQQ", data, p)
            if data[p + 24:p + 24 + n].startswith(b"hip") and size:
                yield data[at + offset:at + offset + size]
            p += 24 + n
        at += len(MAGIC)


def registers(operand):
    """Registers of an operand, as (kind, number)."""
    m = re.match(r"-?\|?([vas])\[(\d+):(\d+)\]|-?\|?([vas])(\d+)\b", operand.strip())
    if not m:
        return set()
    return {(m[1], i) for i in range(int(m[2]), int(m[3]) + 1)} if m[1] else {(m[4], int(m[5]))}


def states(code):
    """Wait states that an instruction takes at least."""
    return int(code.split()[1], 0) + 1 if code.startswith("s_nop") else 1


class Function:
    def __init__(self, name, lines):
        self.name, self.code = name, [c for _, c in lines]
        index = {a: i for i, (a, _) in enumerate(lines)}
        self.before, self.after = [[] for _ in lines], [[] for _ in lines]
        for i, (address, code) in enumerate(lines):
            word = code.split()
            if word[0].startswith(("s_branch", "s_cbranch")):
                jump = int(word[1], 0)
                self._edge(i, index[address + 4 + 4 * (jump - 65536 if jump >= 32768 else jump)])
            if not word[0].startswith(("s_branch", "s_endpgm", "s_setpc")) and i + 1 < len(lines):
                self._edge(i, i + 1)

    def _edge(self, i, j):
        self.after[i].append(j)
        self.before[j].append(i)

    def operands(self, i):
        parts = self.code[i].split(None, 1)
        return [x.strip() for x in parts[1].split(",")] if len(parts) > 1 else []

    def near(self, i, wait, forward, ends=lambda j: False):
        """Instructions that can run with fewer than `wait` states between them and i, on any path up to one that ends() it."""
        left_at, todo = {}, [(j, wait) for j in (self.after if forward else self.before)[i]]
        while todo:
            j, left = todo.pop()
            if left <= left_at.get(j, 0):
                continue
            left_at[j] = left
            yield j
            if ends(j):
                continue
            left -= states(self.code[j])
            todo += [(k, left) for k in (self.after if forward else self.before)[j]]


def functions(image, path):
    """Functions of a code object."""
    open(path, "wb").write(image)
    text = subprocess.run([OBJDUMP, "-d", path], check=True, capture_output=True, text=True).stdout
    name, lines = None, []
    for line in text.splitlines():
        head = re.match(r"[0-9a-f]+ <(.+)>:$", line)
        if head:
            if name and lines:
                yield Function(name, lines)
            name, lines = head[1], []
        elif "//" in line:
            code, at = line.split("//")
            lines.append((int(at.split(":")[0], 16), code.strip()))
    if name and lines:
        yield Function(name, lines)
