"""Distances between instructions that the compiler does not keep around hand-written loads.

Loads into LDS are inline assembly, whose operands the compiler sees and whose instructions it does not.  Between a vector instruction's write of a scalar register and a
memory instruction that reads it there have to be five others (two before a vector instruction that does).  Such writes come up where scalar registers are short: words of a
descriptor then wait in lanes of a vector register, and v_readlane brings them back right before the load, which goes out with part of another descriptor.  Waiting in
front of every load cost 2 to 8 % of the products' time, and hardly any build has one that needs it; so the assembly of each source is looked through after it is
compiled, and a source that has such a load is compiled again with waits (POETX_LOAD_WAITS, poetx_common.h).
"""
from __future__ import annotations

import re

MEMORY, VECTOR = 5, 2      # instructions in between
SCALAR = re.compile(r"\bs\[(\d+):(\d+)\]|\bs(\d+)\b|\b(vcc|m0)(?:_lo|_hi)?\b")
LABEL = re.compile(r"([.\w$]+):\s*(;.*)?$")


def scalars(text):
    found = set()
    for first, last, one, name in SCALAR.findall(text):
        found |= {name} if name else set(range(int(first or one), int(last or one) + 1))
    return found


def parse(line):
    """(instructions it stands for, scalar registers a vector instruction writes, those it reads, what they need in between, branch target) or None"""
    line = line.split(";")[0].strip()
    if not line or line[0] in "./#":
        return None
    op, _, rest = line.partition(" ") if "\t" not in line else line.partition("\t")
    operands = [o.strip() for o in rest.split(",")]
    if op == "s_nop":
        return int(operands[0], 0) + 1, set(), set(), 0, None
    if op.startswith(("buffer_", "global_", "flat_", "scratch_")):
        return 1, set(), scalars(rest) | ({"m0"} if re.search(r"\blds\b|_lds_", line) else set()), MEMORY, None
    if op.startswith("v_"):
        out = 2 if "_co_" in op or op.startswith("v_div_scale") else 1
        return 1, scalars(",".join(operands[:out])), scalars(",".join(operands[out:])), VECTOR, None
    return 1, set(), set(), 0, operands[0] if op.startswith(("s_branch", "s_cbranch")) else None


def into_lds(read):
    """Is a memory instruction that reads these registers a load into LDS?  Only those take M0."""
    return "m0" in read


def too_close(assembly):
    """Instructions of hand-written assembly that read a scalar register too soon, as (line number, instruction, the one that writes it).  Every load into LDS is written by hand here: one that is
    not marked as such says that the compiler marks hand-written assembly in another way than this looks for, which is a ValueError."""
    code, labels, by_hand = [], {}, False
    for number, line in enumerate(assembly.splitlines(), 1):
        text = line.strip()
        if text.startswith((";APP", ";;#ASMSTART")):
            by_hand = True
        elif text.startswith((";NO_APP", ";;#ASMEND")):
            by_hand = False
        elif LABEL.match(text):
            labels[LABEL.match(text)[1]] = len(code)
        else:
            at = parse(text)
            if at:
                if at[3] == MEMORY and into_lds(at[2]) and not by_hand:
                    raise ValueError(f"line {number}, {text}: a load into LDS that is not marked as hand-written")
                code.append((number, text, by_hand, at))
    found = set()

    def follow(at, written, writer, passed):
        """From instruction `at` on, registers `written` by `writer`, `passed` instructions before."""
        while at < len(code) and passed < MEMORY:
            number, text, hand, (count, out, read, need, target) = code[at]
            if hand and passed < need and read & written:
                found.add((number, text, writer))
            if target in labels:
                follow(labels[target], written, writer, passed + 1)
            if text.startswith(("s_branch", "s_endpgm", "s_setpc")):
                return
            passed += count
            at += 1

    for i, (_, text, _, (_, out, _, _, _)) in enumerate(code):
        if out:
            follow(i + 1, out, text, 0)
    return sorted(found)
