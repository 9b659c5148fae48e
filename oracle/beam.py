"""Reference of beam search's selection and of forking and compacting a paged cache, on the CPU, one request, child or page at
a time. Tables, counts and lengths are lists; a cache layer is a tensor [2][blocks][piece]."""
from __future__ import annotations

import math

import numpy as np


def select(logits, scores, keep, done=None, done_token=0):
    """logits float64 [batch][beams][vocab], scores float64 [batch][beams]: (tokens, parents, values), lists of `keep` of each
    request, and the least distance between the value of a chosen candidate and another's that does not equal it. Equal values:
    the lower row first, then the larger logit, then the lower token."""
    res, gap = [], math.inf
    for b in range(logits.shape[0]):
        found = []
        for y in range(logits.shape[1]):
            s, x = float(scores[b, y]), logits[b, y]
            row = b * logits.shape[1] + y
            if not math.isfinite(s):
                continue
            if done is not None and done[b, y]:
                found.append((-s, row, 0.0, done_token))
                continue
            if np.isnan(x).any() or not math.isfinite(x.max()):
                continue
            z = x - x.max()
            lse = x.max() + math.log(math.fsum(np.exp(z)))
            order = np.lexsort((np.arange(len(x)), -x))[: keep + 1]
            found += [(-(s + (float(x[t]) - lse)), row, -float(x[t]), int(t)) for t in order if x[t] > -math.inf]
        found.sort()
        values = [-f[0] for f in found]
        for i in range(min(keep, len(values) - 1)):
            if values[i] != values[i + 1]:
                gap = min(gap, values[i] - values[i + 1])
        found = found[:keep] + [(math.inf, -1, 0.0, -1)] * (keep - len(found))
        res.append(([t for _, _, _, t in found], [r for _, r, _, _ in found], [-v for v, _, _, _ in found]))
    return tuple(np.array([r[i] for r in res]) for i in range(3)) + (gap,)


def fork(table, lens, refs, parents, grow, tokens, max_len, width):
    """(table, lens, refs, free, copies): copies are (from, to) blocks."""
    blocks, refs = len(refs), list(refs)
    for row in table:
        for x in row:
            if 0 <= x < blocks:
                refs[x] -= 1
    out, out_lens, copies = [[-1] * width for _ in parents], [], []
    for i, p in enumerate(parents):
        n = min(max(lens[p], 0), max_len) if 0 <= p < len(table) else 0
        out_lens.append(n)
        for j in range(n // tokens):
            x = table[p][j]
            if 0 <= x < blocks:
                out[i][j] = x
                refs[x] += 1
    wants = []  # (child, place, block that is copied there)
    kept = set()
    loose = [x for x in range(blocks) if refs[x] == 0]
    for i, p in enumerate(parents):
        n = out_lens[i]
        if n % tokens:
            x = table[p][n // tokens]
            if 0 <= x < blocks:
                if x in loose and x not in kept:
                    kept.add(x)
                    out[i][n // tokens] = x
                    refs[x] = 1
                else:
                    wants.append((i, n // tokens, x))
        until = min(-(-(n + max(0, grow[i] if grow else 0)) // tokens), width)
        wants += [(i, j, None) for j in range(-(-n // tokens), until)]
    free = [x for x in range(blocks) if refs[x] == 0]
    for (i, j, x), to in zip(wants, free):
        out[i][j] = to
        refs[to] = 1
        if x is not None:
            copies.append((x, to))
    return out, out_lens, refs, len(free) - len(wants), copies


def compact(table, refs):
    """(table, refs, moved, held, copies)."""
    held = sum(r != 0 for r in refs)
    copies = list(zip((x for x in range(held, len(refs)) if refs[x]), [x for x in range(held) if not refs[x]]))
    moved = [x if r else -1 for x, r in enumerate(refs)]
    out = list(refs)
    for a, b in copies:
        moved[a], out[b], out[a] = b, refs[a], 0
    new = [[moved[x] if 0 <= x < len(refs) and moved[x] >= 0 else x for x in row] for row in table]
    return new, out, moved, held, copies
