"""The library's own gfx950 code, read back: where a memory instruction uses a scalar register too soon after a vector instruction wrote it.

The compiler keeps such pairs five wait states apart, but does not look into blocks of assembly; those have to wait for themselves."""
import glob
import os
import re
import shutil
import subprocess
import tempfile

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
WAIT = 5


def scalars(text):
    out = set()
    for m in re.finditer(r"\bs\[(\d+):(\d+)\]|\bs(\d+)\b", text):
        out |= {int(m.group(3))} if m.group(3) else set(range(int(m.group(1)), int(m.group(2)) + 1))
    return out


def kernels(library):
    """{kernel: [(address, instruction, operands, address it may go to)]} of every bundle."""
    out = {}
    with tempfile.TemporaryDirectory() as d:
        shutil.copy(library, os.path.join(d, "lib"))
        subprocess.run([OBJDUMP, "--offloading", "lib"], cwd=d, check=True, capture_output=True)
        for f in sorted(glob.glob(os.path.join(d, "lib.*gfx950"))):
            text = subprocess.run([OBJDUMP, "-d", f], check=True, capture_output=True, text=True).stdout
            code = None
            for line in text.splitlines():
                m = re.match(r"^([0-9a-f]+) <(.+)>:$", line)
                if m:
                    first, code = int(m.group(1), 16), out.setdefault((os.path.basename(f), m.group(2)), [])
                    continue
                m = re.match(r"^\t(\S+)(.*?)\s*// ([0-9A-F]+):(.*)$", line)
                if m:
                    to = re.search(r"<[^>]*?(?:\+0x([0-9a-f]+))?>\s*$", m.group(4)) if "branch" in m.group(1) else None
                    code.append((int(m.group(3), 16), m.group(1), m.group(2).strip(), first + int(to.group(1) or "0", 16) if to else None))
    return out


def _written_by_vector(op, args):
    part = args.split(",")
    if op.startswith(("v_readlane", "v_readfirstlane", "v_cmp_")):
        return scalars(part[0])
    if op.startswith("v_") and ("_co_" in op or "div_scale" in op):
        return scalars(part[1])
    return set()


def too_soon(code):
    """(number of memory instructions, [(writer, reader, wait states between them)])."""
    index = {c[0]: i for i, c in enumerate(code)}
    before = [[] for _ in code]
    for i, (_, op, _, to) in enumerate(code):
        if op not in ("s_branch", "s_endpgm", "s_setpc_b64") and i + 1 < len(code):
            before[i + 1].append(i)
        if to is not None:
            before[index[to]].append(i)
    n, found = 0, []
    for i, (_, op, args, _) in enumerate(code):
        if not op.startswith(("buffer_", "global_", "flat_", "scratch_")):
            continue
        n += 1
        ways, seen = [(j, 0, frozenset(scalars(args))) for j in before[i]], set()
        while ways:
            j, waited, need = way = ways.pop()
            if waited >= WAIT or not need or way in seen:
                continue
            seen.add(way)
            _, o, a, _ = code[j]
            if _written_by_vector(o, a) & need:
                found.append((o + " " + a, op + " " + args, waited))
                continue
            if o.startswith("s_") and not o.startswith(("s_cmp", "s_bitcmp", "s_cbranch", "s_branch", "s_nop", "s_wait", "s_barrier")):
                need -= scalars(a.split(",")[0])                   # (a scalar instruction waits for the vector one by itself)
            ways += [(k, waited + 1 + (int(a, 0) if o == "s_nop" else 0), need) for k in before[j]]
    return n, found
