"""Wait states that a gfx950 assembly listing owes around inline assembly, whose instructions the compiler does
not know: it puts in those between its own.  The rules, in instructions (s_nop n counts n + 1) on any path:

* a scalar register that a vector instruction wrote (v_readlane, v_readfirstlane, a comparison, a carry) is not read
  as an address by a memory instruction for five;
* M0, written by a scalar instruction, is not read by a copy to LDS for one;
* a vector register that a vector instruction wrote is not read by a matrix product for two.
"""
import re

_LABEL = re.compile(r"^([.\w$]+):")
_REGS = re.compile(r"\b([sva])\[(\d+):(\d+)\]|\b([sva])(\d+)\b|\b(vcc|vcc_lo|vcc_hi|m0)\b")
_CARRY = ("v_add_co_", "v_sub_co_", "v_subrev_co_", "v_addc_co_", "v_subb_co_", "v_subbrev_co_", "v_mad_u64_u32",
          "v_mad_i64_i32", "v_div_scale_")
_MEMORY = ("global_", "buffer_", "flat_", "scratch_")


def _regs(operand):
    out = set()
    for m in _REGS.finditer(operand):
        if m.group(6):
            out |= {"vcc_lo", "vcc_hi"} if m.group(6) == "vcc" else {m.group(6)}
        elif m.group(1):
            out |= {f"{m.group(1)}{i}" for i in range(int(m.group(2)), int(m.group(3)) + 1)}
        else:
            out.add(m.group(4) + m.group(5))
    return out


class Op:
    __slots__ = ("line", "text", "name", "operands", "states")

    def __init__(self, line, text):
        self.line, self.text = line, text
        self.name, _, rest = text.partition(" ")
        self.operands = [x.strip() for x in rest.split(",")]
        self.states = int(self.operands[0], 0) + 1 if self.name == "s_nop" else 1

    def writes(self):
        """(registers of a vector instruction's results, scalar ones among them; M0 by a scalar one)."""
        if self.name.startswith("v_"):
            n = 2 if self.name.startswith(_CARRY) else 1
            regs = set().union(*(_regs(x) for x in self.operands[:n]))
            if self.name.startswith("v_cmpx"):
                regs = set()
            if "_swap_" in self.name:
                regs |= _regs(self.operands[1])
            return regs
        return set()

    def scalar_writes(self):
        if not self.name.startswith("s_") or self.name.startswith(("s_cmp", "s_bitcmp", "s_cbranch", "s_branch", "s_wait",
                                                                   "s_barrier", "s_nop", "s_endpgm", "s_setprio")):
            return set()
        return _regs(self.operands[0])


def _functions(text):
    """(name, [ops], {label: index}) of each function."""
    ops, labels, name = [], {}, None
    for k, raw in enumerate(text.splitlines(), 1):
        line = raw.split(";")[0].split("//")[0].strip()
        if not line:
            continue
        m = _LABEL.match(line)
        if m:
            if not m.group(1).startswith("."):
                if ops:
                    yield name, ops, labels
                ops, labels, name = [], {}, m.group(1)
            labels[m.group(1)] = len(ops)
            line = line[m.end():].strip()
            if not line:
                continue
        if line.startswith(".") or name is None:
            continue
        line = re.sub(r"\s+", " ", line)
        if re.match(r"(s|v|ds|global|buffer|flat|scratch)_", line):
            ops.append(Op(k, line))
    if ops:
        yield name, ops, labels


def _step(op, state, found):
    """state: for each register, how many instructions ago it was written (as far as a rule looks back); what is
    owed goes to found.  Returns the state behind op."""
    name = op.name
    if name.startswith(_MEMORY):
        for x in _regs(" ".join(op.operands)):
            if x[0] == "s" or x.startswith("vcc"):
                if state.get(("V", x), 9) < 5:
                    found.add((op.line, op.text, x, state[("V", x)], 5))
        if "load_lds" in name and state.get(("S", "m0"), 9) < 1:
            found.add((op.line, op.text, "m0", state[("S", "m0")], 1))
    if name.startswith(("v_mfma", "v_smfmac")):
        for x in set().union(*(_regs(o) for o in op.operands[1:4])):
            if state.get(("V", x), 9) < 2:
                found.add((op.line, op.text, x, state[("V", x)], 2))
    new = {}
    vector, scalar = op.writes(), op.scalar_writes()
    if name.startswith(("v_mfma", "v_smfmac")):
        vector = set()  # (a product behind a product is the hardware's)
    for (kind, x), n in state.items():
        if x in scalar or x in vector or (name.startswith("s_load") and x in _regs(op.operands[0])):
            continue
        n += op.states
        if n < (5 if kind == "V" else 1):
            new[(kind, x)] = n
    for x in vector:
        new[("V", x)] = 0
    if "m0" in scalar:
        new[("S", "m0")] = 0
    return new


def scan(text):
    """What is owed in a listing: [(line, instruction, register, instructions between, instructions owed)]."""
    found, copies = set(), 0
    for _, ops, labels in _functions(text):
        copies += sum("load_lds" in o.name for o in ops)
        ends = sorted({i for i in labels.values()} | {i + 1 for i, o in enumerate(ops) if "branch" in o.name or o.name in (
            "s_endpgm", "s_setpc_b64")} | {0, len(ops)})
        starts = [i for i in ends if i < len(ops)]
        stop = {a: b for a, b in zip(ends, ends[1:])}
        entry, todo = {s: None for s in starts}, [s for s in starts if s == 0]
        if starts:
            entry[0] = {}
        while todo:
            s = todo.pop()
            state = entry[s]
            for o in ops[s:stop[s]]:
                state = _step(o, state, found)
            last = ops[stop[s] - 1]
            after = []
            if "branch" in last.name:
                after.append(labels.get(last.operands[0]))
            if last.name not in ("s_branch", "s_endpgm", "s_setpc_b64"):
                after.append(stop[s])
            for t in after:
                if t is None or t >= len(ops):
                    continue
                old = entry[t]
                merged = dict(state) if old is None else {k: min(old.get(k, 9), state.get(k, 9)) for k in {*old, *state}}
                if merged != old:
                    entry[t] = merged
                    todo.append(t)
    return sorted(found), copies
