"""Reference of the operators on the paged KV cache, in 64 bits on the CPU.

Every function takes and returns plain torch CPU tensors. A cache layer is a flat tensor of its elements (8-bit
ones as uint8 bit patterns); where an entry lies follows from the layout's definition alone: K and V of a layer
are [2][blocks][piece], a piece is [tokens][heads][dim] ("piece"), [heads][tokens][dim] ("hnd"), or x-packed:
keys [heads][dim / x][tokens][x] with x = 16 bytes, values [heads][dim][tokens].
"""
from __future__ import annotations

import math
from dataclasses import dataclass

import numpy as np
import torch

F8 = torch.float8_e4m3fn
F8_MAX = 448.0


@dataclass(frozen=True)
class Cache:
    layout: str
    dtype: torch.dtype
    blocks: int
    tokens: int
    heads: int
    dim: int

    @property
    def elem(self):
        return 1 if self.dtype is F8 else 2

    @property
    def piece(self):
        return self.tokens * self.heads * self.dim

    def index(self, which: int, block: int, token: int, head: int) -> torch.Tensor:
        """Element indices [dim] of one entry's K (which 0) or V (1) of a head in the flat layer."""
        d = torch.arange(self.dim)
        base = (which * self.blocks + block) * self.piece
        if self.layout == "piece":
            return base + (token * self.heads + head) * self.dim + d
        if self.layout == "hnd":
            return base + (head * self.tokens + token) * self.dim + d
        if which == 0:
            x = 16 // self.elem
            return base + ((head * (self.dim // x) + d // x) * self.tokens + token) * x + d % x
        return base + (head * self.dim + d) * self.tokens + token

    def values(self, flat: torch.Tensor, index: torch.Tensor) -> torch.Tensor:
        x = flat[index]
        return (x.view(F8) if self.dtype is F8 else x.view(self.dtype)).double()

    def entry(self, table_row, j: int):
        """(block, token) of entry j, or None where the table has no block for it."""
        b = int(table_row[j // self.tokens])
        return (b, j % self.tokens) if 0 <= b < self.blocks else None


def rope(x, cos, sin, interleaved: bool):
    """x [..., dim], cos and sin [..., r]: the first 2 r values turned in pairs."""
    r = cos.shape[-1]
    y = x.clone()
    for i in range(r):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r)
        y[..., a] = x[..., a] * cos[..., i] - x[..., b] * sin[..., i]
        y[..., b] = x[..., b] * cos[..., i] + x[..., a] * sin[..., i]
    return y


def append(q, k, v, positions=None, table=None, interleaved=False, q_weight=None, k_weight=None, eps=1e-6):
    """Queries and keys (and the values as they are) before any rounding."""
    out = []
    for x, w in ((q.double(), q_weight), (k.double(), k_weight)):
        if w is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
        if table is not None:
            p = positions.long().clamp(0, table.shape[0] - 1)
            r = table.shape[1] // 2
            rows = table.double()[p][:, None]
            x = rope(x, rows[..., :r], rows[..., r:], interleaved)
        out.append(x)
    return out[0], out[1], v.double()


def spans(c: Cache, table, lens, q_start, num_tokens, max_tokens, max_len):
    """(first token row, tokens, entries before, entries in all) of each sequence."""
    res = []
    for s in range(table.shape[0]):
        a, b = (q_start[s], q_start[s + 1]) if q_start is not None else (s * max_tokens, (s + 1) * max_tokens)
        a = min(max(int(a), 0), num_tokens)
        b = min(max(int(b), a), num_tokens)
        before = min(max(int(lens[s]), 0), max_len)
        count = min(b - a, max_tokens)
        res.append((a, count, before, min(before + count, max_len)))
    return res


def attention(c: Cache, flat, table, span, q, group, scale, tree=None, k_scale=None, v_scale=None, scores_in=None,
              decay=1.0, cap=0.0, slopes=None, window=0, prefix=None, max_prefix=None):
    """out, lse, scores [sequences][heads][...] (NaN where nothing is written) and, for error bounds, sum p |V|
    and the largest |logit| of each row. cap, slopes (of each query head), window and prefix (of each sequence) shape the
    logits and what is seen."""
    total, heads_q, dim = q.shape
    out = torch.zeros(total, heads_q, dim, dtype=torch.float64)
    mag = torch.zeros_like(out)
    lse = torch.full((total, heads_q), -math.inf, dtype=torch.float64)
    big = torch.zeros(total, heads_q, dtype=torch.float64)
    longest = max([t for _, _, _, t in span] + [1])
    scores = torch.full((table.shape[0], c.heads, longest), math.nan, dtype=torch.float64)
    for s, (a, t, n, m) in enumerate(span):
        at = [c.entry(table[s], j) for j in range(m)]
        there = torch.tensor([x is not None for x in at], dtype=torch.bool)
        for h in range(c.heads):
            zero = torch.zeros(dim, dtype=torch.float64)
            k = [c.values(flat, c.index(0, *x, h)) if x else zero for x in at]
            v = [c.values(flat, c.index(1, *x, h)) if x else zero for x in at]
            k, v = (torch.stack(x) if m else torch.zeros(0, dim, dtype=torch.float64) for x in (k, v))
            if k_scale is not None:
                k = k * float(k_scale[h])
            if v_scale is not None:
                v = v * float(v_scale[h])
            mass = torch.zeros(m, dtype=torch.float64)
            for i in range(t):
                sees = there.clone()
                if tree is None and (window or prefix is not None):
                    j = torch.arange(m)
                    ahead = 0 if prefix is None else max(0, int(prefix[s]))
                    ahead = ahead if max_prefix is None else min(ahead, max_prefix)
                    sees &= (j < ahead) | ((j <= n + i) & ((n + i - j < window) if window else True))
                for d in range(m - n):
                    if tree is None and (window or prefix is not None):
                        break
                    if tree is None:
                        sees[n + d] &= d <= i
                    else:
                        word = int(tree[a + i, d // 64]) if d // 64 < tree.shape[1] else 0
                        sees[n + d] &= bool((word >> (d % 64)) & 1)
                for e in range(h * group, (h + 1) * group):
                    if not bool(sees.any()):
                        continue
                    x = (k[sees] @ q[a + i, e].double()) * scale
                    if cap:
                        x = cap * torch.tanh(x / cap)
                    if slopes is not None:
                        x = x - float(slopes[e]) * (n + i - torch.arange(m)[sees]).abs()
                    w = torch.logsumexp(x, 0)
                    p = torch.exp(x - w)
                    out[a + i, e] = p @ v[sees]
                    mag[a + i, e] = p @ v[sees].abs()
                    lse[a + i, e] = w
                    big[a + i, e] = (k[sees].abs() @ q[a + i, e].double().abs()).max() * abs(scale)
                    mass[sees] += p
            if scores_in is not None and n:
                mass[:min(n, m)] += decay * scores_in[s, h, :min(n, m)].double()
            scores[s, h, :m] = mass
    return {"out": out, "lse": lse, "scores": scores, "mag": mag, "big": big}


def commit_moves(accepted, counts, span):
    """[(source, destination)] entries of each sequence, and the new lengths."""
    moves, lens = [], []
    for s, (_, t, n, m) in enumerate(span):
        got = []
        for i in range(min(max(int(counts[s]), 0), accepted.shape[1])):
            j = int(accepted[s, i])
            if j < 0 or j >= m - n or (i and j <= int(accepted[s, i - 1])):
                break
            got.append(j)
        moves.append([(n + j, n + i) for i, j in enumerate(got)])
        lens.append(n + len(got))
    return moves, lens


def move_entries(c: Cache, flat, src_row, dst_row, moves, heads=None):
    """Entries [(source, destination)] of a sequence moved in order, in a copy of the layer."""
    out = flat.clone()
    for h in range(c.heads) if heads is None else heads:
        for src, dst in moves:
            a, b = c.entry(src_row, src), c.entry(dst_row, dst)
            if a is None or b is None:
                continue
            for which in (0, 1):
                out[c.index(which, *b, h)] = out[c.index(which, *a, h)]
    return out


def evict_select(scores, n, keep, sinks, recent):
    """Entries kept of one sequence and head, ascending."""
    if n <= keep:
        return list(range(n))
    fixed = list(range(sinks)) + list(range(n - recent, n))
    rest = list(range(sinks, n - recent))
    value = [float(x) for x in scores[:n]]
    rest.sort(key=lambda j: (1, 0.0, j) if math.isnan(value[j]) else (0, -value[j], j))
    return sorted(fixed + rest[: keep - len(fixed)])


def rope_frequencies(rot, base=10000.0, kind="none", factor=1.0, original=0.0, low=1.0, high=32.0):
    """Frequencies of the pairs and the factor of cos and sin."""
    i = np.arange(rot // 2, dtype=np.float64)
    if kind == "base":
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-2 * i / rot)
    if kind == "linear":
        return f / factor, 1.0
    if kind == "ramp":
        def index(turns):
            return rot * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))
        first, last = max(math.floor(index(high)), 0), min(math.ceil(index(low)), rot - 1)
        last = last if last > first else first + 0.001
        scaled = np.clip((i - first) / (last - first), 0, 1)
        return f / factor * scaled + f * (1 - scaled), 0.1 * math.log(factor) + 1
    if kind == "bands":
        keep = np.clip((original * f / (2 * math.pi) - low) / (high - low), 0, 1)
        return keep * f + (1 - keep) * f / factor, 1.0
    return f, 1.0
