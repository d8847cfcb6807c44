"""Wait states in the built library's gfx950 code that neither the hardware nor, inside inline assembly, the compiler sees
to.  Reads the listing of the code objects that hipcc made of this repository's sources.

A wait state is an instruction issued in between, or a step of s_nop.  Every way that control can take from the first
instruction is followed, calls excepted (there are none).
"""
import os
import re
import struct
import subprocess

import paper_2603_01639_amd as ltd

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def code_objects(path=ltd.LIB_PATH):
    """The gfx950 code objects that lie in a shared library."""
    data = open(path, "rb").read()
    at, out = data.find(MAGIC), []
    while at >= 0:
        p = at + len(MAGIC) + 8
        for _ in range(struct.unpack_from("<Q", data, p - 8)[0]):
            off, size, length = struct.unpack_from("<QQQ", data, p)
            target = data[p + 24:p + 24 + length].decode()
            p += 24 + length
            if target.endswith("gfx950") and size:
                out.append(data[at + off:at + off + size])
        at = data.find(MAGIC, p)
    return out


def listing(code, tmp):
    path = os.path.join(tmp, "code.o")
    with open(path, "wb") as f:
        f.write(code)
    return subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", path], check=True, capture_output=True, text=True).stdout


REGS = re.compile(r"(?<![\w.])([vas])(?:(\d+)|\[(\d+):(\d+)\])(?![\w])|(?<![\w.])(vcc|m0)(?![\w])")


def regs(operand):
    out = set()
    for kind, one, lo, hi, special in REGS.findall(operand):
        if special:
            out.add(special)
        else:
            a, b = (int(one), int(one)) if one else (int(lo), int(hi))
            out.update((kind, i) for i in range(a, b + 1))
    return out


class Instruction:
    """Mnemonic, registers written and read, and the place a branch goes to."""
    __slots__ = ("text", "name", "writes", "reads", "operands", "goto", "ends")

    def __init__(self, text, target=None):
        self.text = text = text.strip()
        name, _, rest = text.partition(" ")
        self.name, self.goto, self.ends = name, target, name in ("s_endpgm", "s_branch", "s_setpc_b64")
        ops = re.split(r",\s*(?![^\[]*\])", rest) if rest else []
        ops = ops[:-1] + ops[-1].split(" ")[:1] if ops else []
        self.operands = [regs(o) for o in ops]
        writes = 1
        if re.match(r"(global|flat|scratch|buffer)_(store|load_lds)|ds_write|s_cmp|s_bitcmp|s_waitcnt|s_nop|s_barrier|s_cbranch|"
                    r"s_branch|s_endpgm|s_setprio|s_sleep", name):
            writes = 0
        elif re.match(r"v_(add|sub|subrev|addc|subb|subbrev)_co_|v_div_scale|v_mad_[ui]64|v_permlane\d+_swap|v_swap", name):
            writes = 2
        self.writes = set().union(*self.operands[:writes]) if writes else set()
        self.reads = set().union(*self.operands[writes:])
        if re.match(r"v_permlane\d+_swap|v_swap", name) or re.match(r"v_(fmac|dot2c)|v_writelane|v_mac", name):
            self.reads |= self.writes

    @property
    def valu(self):
        return self.name.startswith("v_") and not self.mfma

    @property
    def mfma(self):
        return self.name.startswith(("v_mfma", "v_smfmac"))

    @property
    def memory(self):
        return self.name.startswith(("global_", "flat_", "scratch_", "buffer_"))

    @property
    def states(self):
        return int(self.text.split()[1]) + 1 if self.name == "s_nop" else 1


def functions(text):
    """Lists of instructions, one for each function of a listing."""
    out, base, where = [], 0, {}
    for line in text.splitlines():
        head = re.match(r"^([0-9a-f]+) <(.+)>:$", line)
        if head:
            base, where = int(head.group(1), 16), {}
            out.append((head.group(2), [], where))
            continue
        m = re.match(r"^\s+([sv]_|ds_|global_|flat_|scratch_|buffer_)(.*?)\s*// ([0-9A-F]+):(.*)$", line)
        if not m:
            continue
        goto = re.search(r"<[^>]*?(?:\+0x([0-9a-f]+))?>\s*$", m.group(4)) if "branch" in m.group(2) else None
        where[int(m.group(3), 16)] = len(out[-1][1])
        out[-1][1].append(Instruction(m.group(1) + m.group(2), base + int(goto.group(1) or "0", 16) if goto else None))
    for name, code, where in out:
        for i in code:
            if i.goto is not None:
                i.goto = where[i.goto]
    return [(name, code) for name, code, _ in out]


def after(code, start, reach):
    """(instruction, wait states between it and code[start]) for what can follow within `reach` wait states."""
    best = {}
    todo = [(start + 1, 0)]
    while todo:
        at, states = todo.pop()
        while at < len(code) and states < reach and best.get(at, reach) > states:
            best[at] = states
            i = code[at]
            if i.goto is not None:
                todo.append((i.goto, states + i.states))
            if i.ends:
                break
            at, states = at + 1, states + i.states
    return [(code[at], states) for at, states in best.items()]


def lds_load(code):
    """A direct load to LDS behind the scalar write of m0, its place there: one wait state."""
    for at, i in enumerate(code):
        if i.name.startswith("s_") and "m0" in i.writes:
            for j, states in after(code, at, 1):
                if "load_lds" in j.name:
                    yield i, j, states


def scalar_base(code):
    """A memory instruction that reads a scalar register behind a vector instruction that writes it: five."""
    for at, i in enumerate(code):
        written = {r for r in i.writes if r == "vcc" or r[0] == "s"} if i.valu else ()
        if written:
            for j, states in after(code, at, 5):
                if j.memory and j.reads & written:
                    yield i, j, states


# Passes of the matrix products in use.  What reads or writes a product's sums, but a product that adds to the same ones,
# comes passes + 4 wait states later; so does a product that takes them as factors.  (What hipcc keeps for its own products
# on gfx950: 12 behind one of 8 passes, 8 behind one of 4.)
PASSES = {"v_mfma_f32_32x32x16_bf16": 8, "v_mfma_f32_16x16x32_bf16": 4}


def sums(code):
    """What touches a product's sums before they are there."""
    for at, i in enumerate(code):
        if not i.mfma:
            continue
        need = PASSES[i.name] + 4
        for j, states in after(code, at, need):
            if j.mfma:
                same = i.writes == j.writes and (j.operands[3] == i.writes or not j.operands[3])
                if (j.operands[1] | j.operands[2]) & i.writes or (not same and (j.operands[3] | j.writes) & i.writes):
                    yield i, j, states
            elif (j.reads | j.writes) & i.writes:
                yield i, j, states


def factors(code):
    """A product that reads what a vector instruction (but a dot product) wrote: two wait states."""
    for at, i in enumerate(code):
        written = {r for r in i.writes if r[0] in "va"} if i.valu and not i.name.startswith("v_dot") else ()
        if written:
            for j, states in after(code, at, 2):
                if j.mfma and j.reads & written:
                    yield i, j, states
