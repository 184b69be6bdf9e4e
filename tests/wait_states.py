"""Reads the assembly of the library's own kernels for two ways in which compiled code can read a
register too early or write it for too few lanes, both seen in these kernels:

  short_waits    a way from a matrix instruction to the first vector or memory instruction that touches
                 its result with fewer wait states than the result takes (behind two branches, the
                 compiler counts along one of them)
  masked_copies  a copy of a register at the head of a block where lanes join again, before the
                 execution mask is restored: what it writes is missing in the lanes that were away
"""
import heapq
import re

# passes of the matrix instructions, and wait states until a result may be read: those of 32-bit operands
# take one less than the passes and a half more than the others
PASSES = {"32x32x16": 8, "32x32x2": 16, "16x16x32": 4, "16x16x4": 8}
READ = {4: 7, 8: 11, 16: 19}
READ_F32 = {8: 10, 16: 18}


def _registers(text):
    out = {(k, int(n)) for k, n in re.findall(r"\b([va])(\d+)\b", text)}
    for k, a, b in re.findall(r"\b([va])\[(\d+):(\d+)\]", text):
        out |= {(k, i) for i in range(int(a), int(b) + 1)}
    return out


def _passes(op):
    shape = re.search(r"_(\d+x\d+x\d+)_", op)
    return PASSES[shape.group(1)]


def _states(op, arg):
    if op == "s_nop":
        return int(arg.split()[0], 0) + 1
    return _passes(op) if "mfma" in op else 1


def kernels(asm):
    """(name, instructions as (op, operands), {label: index}) of each function."""
    for m in re.finditer(r"^(_Z\S+):", asm, re.M):
        end = asm.find(".section", m.end())
        ins, labels = [], {}
        for line in asm[m.end():end if end > 0 else None].split("\n"):
            label = re.match(r"^(\.LBB\d+_\d+):", line)
            if label:
                labels[label.group(1)] = len(ins)
                continue
            t = line.split(";")[0].strip()
            if t and not t.startswith("."):
                op, _, arg = t.partition(" ")
                ins.append((op, arg.strip()))
        yield m.group(1), ins, labels


def short_waits(ins, labels):
    """(matrix instruction, reader, wait states, needed) of every way that is too short."""
    bad, touched = [], {}
    for at, (op, arg) in enumerate(ins):
        if "mfma" not in op:
            continue
        f32 = op.endswith(("x2_f32", "x4_f32"))
        need = (READ_F32 if f32 else READ)[_passes(op)]
        result = _registers(arg.split(",")[0])
        best, heap = {}, [(0, at + 1)]
        while heap:
            w, p = heapq.heappop(heap)
            if p >= len(ins) or w >= need or best.get(p, need) <= w:
                continue
            best[p] = w
            o, g = ins[p]
            if o == "s_endpgm":
                continue
            if "mfma" in o:
                parts = re.split(r",(?![^\[]*\])", g)
                if _registers(parts[1] + parts[2]) & result:
                    bad.append((ins[at], ins[p], w, need))
                    continue
                if _registers(parts[0]) & result:
                    continue  # goes on accumulating: that one is looked at itself
            elif o.startswith(("v_", "ds_", "global_", "buffer_", "scratch_", "flat_")):
                if p not in touched:
                    head, _, rest = g.partition(",")
                    write_only = o.startswith("v_")
                    touched[p] = _registers(g), _registers(rest if write_only else g)
                if touched[p][0] & result:
                    # a plain overwrite of a 32-bit product may come one state earlier
                    if not (f32 and w >= need - 1 and not touched[p][1] & result):
                        bad.append((ins[at], ins[p], w, need))
                    continue
            nxt = w + _states(o, g)
            if o in ("s_branch",) or o.startswith("s_cbranch"):
                heapq.heappush(heap, (nxt, labels[g]))
            if o != "s_branch":
                heapq.heappush(heap, (nxt, p + 1))
    return bad


_MASK = re.compile(r"s_(or|and|andn2|xor|mov)_b64 exec|s_\w+_saveexec")


def masked_copies(ins, labels):
    """Copies to another register (or to memory) ahead of the mask's restoration at a join of lanes."""
    bad = []
    for label in {g for o, g in ins if o == "s_cbranch_execz"}:
        ahead = []
        for o, g in ins[labels[label]:labels[label] + 60]:
            if _MASK.match(f"{o} {g}"):
                bad += [(label, x) for x in ahead]
                break
            if o.startswith(("s_cbranch", "s_branch", "s_endpgm")):
                break
            if o.startswith(("v_accvgpr_write", "v_accvgpr_mov", "v_mov_b32", "scratch_store")):
                ahead.append((o, g))
    return bad
