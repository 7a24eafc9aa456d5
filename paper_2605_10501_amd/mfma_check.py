"""Wait states around matrix products written as inline assembly (mfma_acc of csrc/gemm_fp8.hip), which the compiler does not look after.

What the products need, in wait states of the wave (every instruction is one, s_nop k is k + 1):
  * 2 between a vector instruction that writes a register and a product that reads it, sums included, and 4 behind one that writes EXEC;
  * 11 between a product and anything but a product that reads its sums (8 passes of the matrix core and the write back); 16 are asked for.
Both are looked for along all paths of a kernel's control flow.  build.py checks the kernels that have such products, so that code which
another compiler orders differently does not become a library."""
import os
import re
import subprocess
import tempfile

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
BEFORE, BEFORE_EXEC, BEHIND = 2, 4, 16
_REG = re.compile(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)")


def _regs(text):
    out = set()
    for m in _REG.finditer(text):
        lo = int(m.group(2) or m.group(4))
        out |= {(m.group(1), i) for i in range(lo, int(m.group(3) or lo) + 1)}
    return out


class Instruction:
    def __init__(self, offset, text, target=None):
        self.offset, self.text, self.target, self.next, self.prev = offset, text, target, [], []
        self.op, _, rest = text.partition(" ")
        first, _, others = rest.partition(",")
        self.product = self.op.startswith("v_mfma")
        self.states = int(rest, 0) + 1 if self.op == "s_nop" else 1
        self.vector = self.op.startswith("v_") and not self.product
        self.writes_exec = self.op.startswith("v_cmpx") or (self.op.startswith("s_") and ("saveexec" in self.op or first.strip().startswith("exec")))
        if "swap" in self.op:                                   # both operands are read and written
            self.reads = self.writes = _regs(rest)
        elif re.match(r"(global|buffer|flat|scratch)_(store|atomic)|ds_write|ds_add", self.op):
            self.reads, self.writes = _regs(rest), set()
        else:
            self.reads, self.writes = _regs(others), _regs(first)


def parse(listing):
    """{kernel: its instructions, with the indices of those behind and in front of each} of a listing by llvm-objdump -d."""
    kernels, code = {}, None
    for line in listing.splitlines():
        head = re.match(r"^[0-9a-f]+ <([^>]+)>:", line)
        if head:
            code = kernels[head.group(1)] = []
            continue
        m = re.match(r"^\s+(\S.*?)\s*// ([0-9A-F]+):", line)
        if m and code is not None:
            to = re.search(r"<[^>]*?(?:\+0x([0-9a-f]+))?>\s*$", line) if "branch" in m.group(1) else None
            code.append(Instruction(int(m.group(2), 16), m.group(1), to and int(to.group(1) or "0", 16)))
    for code in kernels.values():
        at = {i.offset - code[0].offset: k for k, i in enumerate(code)}
        for k, i in enumerate(code):
            if i.target is not None:
                i.next.append(at[i.target])
            if i.op not in ("s_branch", "s_endpgm") and k + 1 < len(code):
                i.next.append(k + 1)
            for n in i.next:
                code[n].prev.append(k)
    return kernels


def _near(code, start, edges, limit):
    """(instruction, wait states between it and `start`) for all with fewer than `limit` along some path."""
    best, todo = {}, [(n, 0) for n in getattr(code[start], edges)]
    while todo:
        k, d = todo.pop()
        if d < limit and best.get(k, limit) > d:
            best[k] = d
            todo += [(n, d + code[k].states) for n in getattr(code[k], edges)]
    return [(code[k], d) for k, d in best.items()]


def hazards(code):
    """What stands too close to the products among a kernel's instructions: (product, other instruction, wait states between)."""
    found = []
    for k, i in enumerate(code):
        if i.product:
            found += [(i, o, d) for o, d in _near(code, k, "prev", BEFORE_EXEC)
                      if o.writes_exec or (d < BEFORE and o.vector and o.writes & (i.reads | i.writes))]
            found += [(i, o, d) for o, d in _near(code, k, "next", BEHIND) if not o.product and o.reads & i.writes]
    return found


def listings(path, kernels):
    """Listings of the gfx950 code in a host object or library, of the parts that have kernels of that name."""
    with tempfile.TemporaryDirectory() as folder:
        copy = os.path.join(folder, "host")
        with open(path, "rb") as src, open(copy, "wb") as dst:
            dst.write(src.read())
        subprocess.run([OBJDUMP, "--offloading", copy], check=True, capture_output=True, cwd=folder)
        out = []
        for part in sorted(os.path.join(folder, f) for f in os.listdir(folder) if f.endswith("gfx950")):
            with open(part, "rb") as f:
                there = kernels.encode() in f.read()
            if there:
                out.append(subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", part], check=True, capture_output=True, text=True).stdout)
        return out


def check(path, kernels):
    """Raises if a product stands too close to something in a kernel of `path` whose name contains `kernels`; returns how many there are of each."""
    count = {}
    for listing in listings(path, kernels):
        for name, code in parse(listing).items():
            if kernels in name and any(i.product for i in code):
                bad = hazards(code)
                if bad:
                    i, o, d = bad[0]
                    raise RuntimeError(f"{name}: {len(bad)} times too few wait states around a product: {d} between\n  {i.text}\nand\n  {o.text}")
                count[name] = sum(i.product for i in code)
    if not count:
        raise RuntimeError(f"{path} has no kernel named {kernels} with products")
    return count
