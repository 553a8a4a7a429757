"""Looks over the assembly of a build for matrix results that are read too early.

A matrix instruction's result may be read by anything but another matrix instruction only after so many wait states, for which the
compiler inserts s_nop.  Behind branches that meet again it has counted those of one path and not of a shorter one, and the
kernel has then read a register's old value (gradients of attention in fp16 at 256 dimensions, off by 18 times their bound).
"""
import re

# wait states from the instruction to a read of its result: passes and three, two where the operands are fp32
WAITS = {"32x32x16": 11, "16x16x32": 7, "32x32x2": 18, "16x16x4": 10, "32x32x8": 19, "16x16x16": 11}
_LOADS = ("ds_read", "buffer_load", "global_load", "flat_load", "scratch_load")


def _registers(text: str) -> frozenset:
    out = set()
    for m in re.finditer(r"\b([va])\[(\d+):(\d+)\]|\b([va])(\d+)\b", text):
        out.update((m[1], i) for i in range(int(m[2]), int(m[3]) + 1)) if m[1] else out.add((m[4], int(m[5])))
    return frozenset(out)


class _Instruction:
    """What it reads and writes, how many wait states it is, and where it may go on (None: the next one)."""

    def __init__(self, op: str, args: str):
        self.op, self.args = op, args
        first, _, rest = args.partition(",")
        vector = op.startswith("v_")
        writes = vector and not op.startswith("v_cmp") or op.startswith(_LOADS)
        self.matrix = re.match(r"v_mfma_\w*?_(\d+x\d+x\d+)", op)
        self.writes = _registers(first) if writes else frozenset()
        # an operation that changes its result in place reads it too
        in_place = op.startswith(("v_fmac", "v_dot2c", "v_pk_fmac", "v_writelane", "v_permlane", "v_swap"))
        self.reads = _registers(args if in_place or not writes else rest) if vector or op.startswith(("ds_", "buffer_", "global_", "flat_", "scratch_")) else frozenset()
        self.states = int(args, 0) + 1 if op == "s_nop" else 1


def early_reads(assembly: str) -> list:
    """A line for every read of a matrix result with too few wait states behind it, along any path."""
    found = []
    for kernel in re.finditer(r"^(\w+):[^\n]*\n(.*?)^\.Lfunc_end", assembly, re.S | re.M):
        if "v_mfma" not in kernel[2]:
            continue
        code, labels = [], {}
        for line in kernel[2].splitlines():
            line = line.split(";")[0].rstrip()
            m = re.match(r"^(\.L\w+):", line)
            if m:
                labels[m[1]] = len(code)
            elif m := re.match(r"^\s+([a-z]\w+)\s*(.*)$", line):
                code.append(_Instruction(m[1], m[2].strip()))
        for at, matrix in enumerate(code):
            if not matrix.matrix:
                continue
            if matrix.matrix[1] not in WAITS:
                found.append(f"{kernel[1]}: wait states of {matrix.op} are not known")
                continue
            need, best, paths = WAITS[matrix.matrix[1]], {}, [(at + 1, 0, matrix.writes)]
            while paths:
                i, states, live = paths.pop()
                if i >= len(code) or states >= need or not live or best.get((i, live), need) <= states:
                    continue
                best[i, live] = states
                x = code[i]
                if x.op == "s_endpgm":
                    continue
                if not x.matrix and x.reads & live:
                    found.append(f"{kernel[1]}: {x.op} {x.args} reads the result of {matrix.op} {matrix.args} after {states} of {need} wait states")
                    continue
                live -= x.writes            # written anew; another matrix instruction's result is looked at from there
                if x.op.startswith(("s_branch", "s_cbranch")):
                    paths.append((labels[x.args], states + 1, live))
                if x.op != "s_branch":
                    paths.append((i + 1, states + x.states, live))
    return found
