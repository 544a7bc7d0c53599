"""The 4-bit cache, beam selection and page bookkeeping by their definitions, on the CPU: values in 64 bits, pages one row after the other."""
import math

import torch

BLOCK = 32
MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def write(x):
    """x [..., d]: codes [..., d / 2], scales [..., blocks] and the values that they stand for."""
    d = x.shape[-1]
    x = x.double().cpu()
    codes, scales, values = torch.zeros(x.shape, dtype=torch.uint8), torch.zeros((*x.shape[:-1], (d + BLOCK - 1) // BLOCK), dtype=torch.uint8), torch.zeros_like(x)
    grid = torch.tensor(MAGNITUDES, dtype=torch.float64)
    for b in range(scales.shape[-1]):
        part = x[..., BLOCK * b:BLOCK * (b + 1)]
        finite = part.isfinite().all(-1)
        part = torch.where(finite[..., None], part, 0.0)
        largest = part.abs().amax(-1)
        e = sum((largest > 6 * 2.0 ** n).long() for n in range(-125, 125)) - 125
        unit = torch.exp2(e.double())[..., None]
        # the nearest; of two the even code: far / 2 for odd ones would be wrong, so ties are told apart by the code's lowest bit
        far = (part.abs()[..., None] / unit[..., None] - grid).abs()
        least = far.amin(-1, keepdim=True)
        rank = torch.where(far == least, torch.arange(8) % 2, 2)
        code = rank.argmin(-1)
        values[..., BLOCK * b:BLOCK * (b + 1)] = torch.where(finite[..., None], torch.where(part.signbit(), -grid[code], grid[code]) * unit, math.nan)
        codes[..., BLOCK * b:BLOCK * (b + 1)] = torch.where(finite[..., None], code + 8 * part.signbit(), 0).to(torch.uint8)
        scales[..., b] = torch.where(finite, e + 127, 255).to(torch.uint8)
    return codes[..., 0::2] | codes[..., 1::2] << 4, scales, values


def read(codes, scales):
    """The values of codes [..., d / 2] with scales [..., blocks]."""
    codes, scales = codes.cpu(), scales.cpu()
    grid = torch.tensor(MAGNITUDES + [-m for m in MAGNITUDES], dtype=torch.float64)
    values = grid[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()]
    unit = torch.where(scales == 255, math.nan, torch.exp2(scales.double() - 127))
    return values * unit.repeat_interleave(BLOCK, -1)[..., :values.shape[-1]]


def select(logits, scores, keep, end=None, ended=None):
    """tokens, parents, scores, ended, one sequence after the other."""
    logits, scores = logits.double().cpu(), scores.double().cpu()
    seqs, beams = scores.shape
    out = [[], [], [], []]
    for s in range(seqs):
        found = []
        for b in range(beams):
            row, score = s * beams + b, float(scores[s, b])
            if not score > -math.inf:
                continue
            if ended is not None and ended[s, b]:
                found.append((-score, b, 0.0, end, True))
                continue
            x = logits[row]
            value = score + (x - x.logsumexp(0))
            best = torch.sort(x, descending=True, stable=True).indices[:keep]
            found += [(-float(value[t]), b, -float(x[t]), int(t), False) for t in best if value[t] > -math.inf]
        found.sort()
        found = found[:keep] + [(math.inf, -1, 0.0, -1, False)] * (keep - len(found))
        out[0].append([f[3] for f in found])
        out[1].append([s * beams + f[1] if f[1] >= 0 else -1 for f in found])
        out[2].append([-f[0] for f in found])
        out[3].append([f[1] >= 0 and (f[4] or f[3] == end) for f in found])
    return torch.tensor(out[0]).int(), torch.tensor(out[1]).int(), torch.tensor(out[2]).double(), torch.tensor(out[3])


def fork(table, lengths, refs, parents, page, held=None, room=0, caches=()):
    """table, lengths, held, refs, slots; `caches` (on the CPU) are changed."""
    columns, pages = table.shape[1], refs.shape[0]
    table, refs, parents = table.tolist(), refs.tolist(), list(range(len(table))) if parents is None else parents.tolist()
    need = lambda n: -(-n // page)   # noqa: E731
    cut = lambda x: [min(max(n, 0), columns * page) for n in x.tolist()]   # noqa: E731
    lengths, held = cut(lengths), cut(lengths if held is None else held)
    there = lambda p: 0 <= p < pages   # noqa: E731
    rows, counts = [], []
    for row, n in zip(table, held):
        for p in filter(there, row[:need(n)]):
            refs[p] -= 1
    for parent in parents:
        n = lengths[parent] if 0 <= parent < len(table) else 0
        rows.append(table[parent][:need(n)] if 0 <= parent < len(table) else [])
        counts.append(n)
        for p in filter(there, rows[-1]):
            refs[p] += 1
    free, taken, sharers, longest = [p for p, n in enumerate(refs) if n == 0], 0, list(refs), {}   # longest: of the rows that got no copy of a page
    out_held, slots = list(counts), []
    for i, (parent, n) in enumerate(zip(parents, counts)):
        slots.append([-1] * room)
        if not 0 <= parent < len(table) or need(n + room) > columns:
            continue
        last = rows[i][-1] if room and n % page else -1
        copy = there(last) and sharers[last] > 1
        if copy:
            sharers[last] -= 1
        wanted = copy + need(n + room) - need(n)
        taken += wanted
        if wanted and taken > len(free):
            if copy:
                longest[last] = max(longest.get(last, 0), n)
            continue
        if not wanted and longest.get(last, 0) > n:   # (it would write over what they hold)
            continue
        mine = free[taken - wanted:taken]
        for p in mine:
            refs[p] += 1
        if copy:
            refs[last] -= 1
            for c in caches:
                c[mine[0]] = c[last]
            rows[i] = rows[i][:-1] + mine[:1]
        rows[i] = rows[i] + mine[copy:]
        out_held[i] = n + room
        slots[i] = [rows[i][t // page] * page + t % page if there(rows[i][t // page]) else -1 for t in range(n, n + room)]
    i32 = dict(dtype=torch.int32)
    return (torch.tensor([r + [-1] * (columns - len(r)) for r in rows], **i32).view(len(parents), columns), torch.tensor(counts, **i32), torch.tensor(out_held, **i32),
            torch.tensor(refs, **i32), torch.tensor(slots, dtype=torch.int64).view(len(parents), room))


def compact(table, refs, caches=()):
    """table, refs, moved, live; `caches` (on the CPU) are changed."""
    n, pages = refs.tolist(), refs.shape[0]
    live = sum(x > 0 for x in n)
    moved = [p if x > 0 else -1 for p, x in enumerate(n)]
    holes = [p for p in range(live) if n[p] <= 0]
    for p in range(live, pages):
        if n[p] > 0:
            moved[p] = holes.pop(0)
            for c in caches:
                c[moved[p]] = c[p]
    out = [0] * pages
    for p, to in enumerate(moved):
        if to >= 0:
            out[to] = n[p]
    new = [[moved[p] if 0 <= p < pages and moved[p] >= 0 else p for p in row] for row in table.tolist()]
    i32 = dict(dtype=torch.int32)
    return torch.tensor(new, **i32).view(table.shape), torch.tensor(out, **i32), torch.tensor(moved, **i32), torch.tensor([live], **i32)
