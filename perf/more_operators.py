"""Operators of beam search on the paged KV cache, as a serving program calls them, and their plain forms.

attention  a few tokens or a prompt chunk over the cache, with scores that are capped, biased by distance, kept to a window,
           or seen both ways in a prefix
beam       the best continuations over a request's beams and the vocabulary
fork       the beams' sequences go on from their parents: pages shared by count, the last one copied, new ones given
compact    the held pages of a pool moved together, tables and counts with them

listed() names twelve cases, draw() gives more of the same ranges. Where `own` is false, run() computes
the plain form with elementary torch operations in 32 bits (beam: 64, where two candidates lie close), rounded once; where
it is true it makes the calls of this repository's package. exact() computes the definitions in 64 bits, one sequence,
request or page at a time.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "f8": torch.float8_e4m3fn}
F8_MAX = 448.0
DECAY = 0.96
PIECE = {"type": "bf16", "layout": "piece", "cache": "bf16", "tokens": 16, "heads": 8, "dim": 128}


def _case(name, op, **kw):
    c = {"op": op}
    if op != "beam":
        c.update(PIECE)
    if op == "attention":
        c.update(group=4, seqs=1, draft=1, cap=0.0, window=0, prefix=0, slopes=False, scores=False)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One user at the start of a chat, a model whose scores are capped: the smallest call, where latency counts.
        _case("decode_capped_short", "attention", len=101, cap=50.0),
        # Eight users deep into long sessions, a window over the last 4k entries and the first four, half precision.
        _case("decode_window_32k", "attention", layout="hnd", type="f16", cache="f16", seqs=8, len=32768, window=4096,
              prefix=4),
        # 32 users with ragged contexts up to 8k, a model with distances instead of positions.
        _case("decode_slopes_batch", "attention", seqs=32, len=8192, slopes=True),
        # A 2k-token prompt chunk behind 6k tokens that a fetch brought back, capped scores, a window of 4k.
        _case("chunk_window_capped", "attention", layout="hnd", draft=2048, len=6144, window=4096, cap=30.0),
        # Prompts of three users that open with an image (seen both ways), 8-bit cache for paged decode, weights kept.
        _case("chunk_image_f8", "attention", layout="xpacked", cache="f8", seqs=3, draft=1021, len=50, prefix=700,
              scores=True),
        # One request of four beams, a vocabulary of 32000: the smallest selection.
        _case("beam_1x4", "beam", type="bf16", batch=1, beams=4, vocab=32000, keep=8, done=False),
        # 24 requests of 8 beams, a large odd vocabulary, logits in 32 bits.
        _case("beam_24x8_f32", "beam", type="f32", batch=24, beams=8, vocab=128001, keep=16, done=False),
        # 8 requests of 32 beams of which some are finished or have died.
        _case("beam_8x32_done", "beam", type="f16", batch=8, beams=32, vocab=65521, keep=64, done=True),
        # One request's four beams after a step, 32 layers.
        _case("fork_1x4", "fork", groups=1, beams=4, len=1000, grow=1, layers=32),
        # 24 requests of 8 beams, some of them over, an 8-bit paged-decode cache; room for four tokens each.
        _case("fork_24x8_f8", "fork", layout="xpacked", cache="f8", groups=24, beams=8, len=1500, grow=4, layers=12),
        # A small pool between two requests.
        _case("compact_64", "compact", blocks=64, held=0.5, seqs=3, layers=32),
        # A pool of 4096 pages, 60 % of them held, before its end is given back.
        _case("compact_4096", "compact", layout="hnd", blocks=4096, held=0.6, seqs=37, layers=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "beam", "beam", "fork", "compact"])
    if op == "beam":
        beams = _log(rng, 1, 64)
        vocab = _log(rng, 500, 262144)
        batch = _log(rng, 1, max(1, min(64, 24_000_000 // (beams * vocab))))
        return _case(None, op, type=rng.choice(["bf16", "f16", "f32"]), batch=batch, beams=beams, vocab=vocab,
                     keep=rng.randint(1, 2 * beams), done=rng.random() < 0.5)
    cache = rng.choice(["bf16", "bf16", "f16", "f8"])
    layout = rng.choice(["piece", "hnd", "xpacked"])
    kind = "f16" if cache == "f16" or cache == "f8" and rng.random() < 0.3 else "bf16"
    c = {"type": kind, "cache": cache, "layout": layout, "heads": rng.choice([1, 2, 4, 5, 8, 8]),
         "dim": rng.choice([64, 80, 96, 128, 128, 256]),
         "tokens": rng.choice([16, 16, 32] if layout == "xpacked" else [8, 16, 16, 24, 32])}
    row = c["heads"] * c["dim"]
    block = row * c["tokens"] * (1 if cache == "f8" else 2) * 2
    if op == "attention":
        c["group"] = rng.choice([1, 2, 3, 4, 4, 5, 7, 8])
        how = rng.choice(["one", "one", "few", "chunk"])
        draft = 1 if how == "one" else _log(rng, 2, 32) if how == "few" else _log(rng, 33, 2048)
        rows = draft * c["heads"] * c["group"]
        top = min(67_000_000 // row, 520_000_000 // rows, int(2.2e11) // (4 * rows * c["dim"]))
        seqs = _log(rng, 1, max(1, min(64, top // (64 + draft))))
        length = _log(rng, 1, max(1, min(131072, top // seqs - draft)))
        c.update(seqs=seqs, draft=draft, len=length, cap=rng.choice([0.0, 20.0, 30.0, 50.0]), slopes=rng.random() < 0.4,
                 window=rng.choice([0, _log(rng, 1, length + draft)]),
                 prefix=rng.choice([0, 0, rng.randint(1, 16), _log(rng, 1, length + draft)]), scores=rng.random() < 0.4)
    elif op == "fork":
        layers = _log(rng, 1, 32)
        pages = max(8, 1_000_000_000 // (block * layers))
        beams = rng.randint(1, min(32, max(1, pages // 4)))
        groups = _log(rng, 1, max(1, min(256 // beams, pages // (4 * beams))))
        c.update(layers=layers, beams=beams, groups=groups, grow=rng.choice([0, 1, 1, rng.randint(2, 40)]),
                 len=_log(rng, 1, max(2, min(65536, (pages // (groups * beams) - 3) * c["tokens"]))))
    else:
        layers = _log(rng, 1, 32)
        blocks = _log(rng, 8, max(8, min(8192, 900_000_000 // (block * layers))))
        c.update(layers=layers, blocks=blocks, held=rng.choice([0.1, 0.5, 0.5, 0.9]), seqs=_log(rng, 1, 64))
    return _case(None, op, **c)


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0, std, generator=g)


def _i32(values):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(values, dtype=np.int32))).cuda()


def _up(n, to):
    return -(-n // to)


def _sizes(c):
    """Entries, new tokens and prefix of each sequence: of the case, so that shapes are; all but one ragged."""
    rng = random.Random(c["len"] * 131 + c["seqs"])
    more = c["seqs"] - 1
    lens = [c["len"]] + [rng.randint(c["len"] // 8, c["len"]) for _ in range(more)]
    if more >= 7:
        lens[1] = 0
    draft = [c["draft"]] + [rng.randint(max(1, c["draft"] // 2), c["draft"]) for _ in range(more)]
    prefix = [c["prefix"]] + [rng.randint(0, c["prefix"]) for _ in range(more)]
    for x in (lens, draft, prefix):
        rng.shuffle(x)
    return lens, draft, prefix


def _cache(c, blocks, layers, g):
    """A cache [layers][2][blocks][piece] of keys and values."""
    x = _normal(g, layers, 2, blocks, c["tokens"] * c["heads"] * c["dim"])
    return (x * 20).clamp(-F8_MAX, F8_MAX).to(TYPES["f8"]) if c["cache"] == "f8" else x.to(TYPES[c["cache"]])


def _prepare_attention(c, g, rng, s):
    lens, draft, prefix = _sizes(c)
    bt, total = c["tokens"], sum(draft)
    need = [_up(n + t, bt) for n, t in zip(lens, draft)]
    blocks = sum(need) + 3
    order = torch.randperm(blocks, generator=g, device="cuda").to(torch.int32).cpu().numpy()
    table = np.full((c["seqs"], max(need)), -1, np.int32)
    at = 0
    for q, n in enumerate(need):
        table[q, :n] = order[at: at + n]
        at += n
    s["table"], s["lens"], s["start"] = _i32(table), _i32(lens), _i32([0] + list(np.cumsum(draft)))
    s["longest"] = max(n + t for n, t in zip(lens, draft))
    s["cache"] = _cache(c, blocks, 1, g)
    if c["cache"] == "f8":
        s["k_scale"] = torch.rand(c["heads"], generator=g, device="cuda") * 0.02 + 0.02
        s["v_scale"] = torch.rand(c["heads"], generator=g, device="cuda") * 0.02 + 0.02
    s["q"] = _normal(g, total, c["heads"] * c["group"], c["dim"], std=2.0).to(TYPES[c["type"]])
    if c["prefix"]:
        s["prefix"] = _i32(prefix)
    if c["slopes"]:
        # A geometric series over the heads, as models with linear biases have it.
        hq = c["heads"] * c["group"]
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], dtype=torch.float32, device="cuda")
    if c["scores"]:
        s["scores_in"] = torch.exp(_normal(g, c["seqs"], c["heads"], s["longest"]))
        s["scores_out"] = torch.zeros_like(s["scores_in"])


def _prepare_beam(c, g, rng, s):
    # Logits with a few strong continuations, and some words that a rule of the program forbids.
    rows = c["batch"] * c["beams"]
    x = _normal(g, rows, c["vocab"], std=1.5)
    strong = torch.randint(0, c["vocab"], (rows, 12), generator=g, device="cuda")
    x.scatter_add_(1, strong, _normal(g, rows, 12).abs() * 4 + 3)
    banned = torch.randint(0, c["vocab"], (rows, 5), generator=g, device="cuda")
    x.scatter_(1, banned, float("-inf"))
    s["logits"] = x.to(TYPES[c["type"]])
    s["scores"] = -torch.rand(c["batch"], c["beams"], generator=g, device="cuda").sort(-1).values * 6
    if c["done"]:
        u = torch.rand(c["batch"], c["beams"], generator=g, device="cuda")
        s["scores"][u < 0.1] = float("-inf")
        s["done"] = (u > 0.8).to(torch.uint8)


def _prepare_fork(c, g, rng, s):
    bt, groups, beams = c["tokens"], c["groups"], c["beams"]
    sizes = random.Random(c["len"] * 131 + groups)
    lens = [c["len"]] + [sizes.randint(max(1, c["len"] // 2), c["len"]) for _ in range(groups - 1)]
    width = _up(c["len"] + c["grow"], bt) + 1
    table = np.full((groups * beams, width), -1, np.int64)
    used = 0
    for y, n in enumerate(lens):
        full, here = n // bt, _up(n, bt)
        for b in range(beams):
            # A beam left another one somewhere in the second half of the entries; its last open page is its own.
            shared = sizes.randint(full // 2, full) if b else 0
            row = table[y * beams + b]
            if shared:
                row[:shared] = table[y * beams + sizes.randrange(b)][:shared]
            row[shared:here] = np.arange(used, used + here - shared)
            used += here - shared
    others = 5 + used // 8  # pages of other requests
    blocks = used + others + groups * beams * (2 + _up(c["grow"], bt)) + sizes.randint(0, 9)
    order = torch.randperm(blocks, generator=g, device="cuda").cpu().numpy()
    refs = np.zeros(blocks, np.int32)
    np.add.at(refs, order[table[table >= 0]], 1)
    refs[order[used: used + others]] = 1
    refs[order[table[0, : lens[0] // bt // 2]]] += 1  # a prompt that a prefix cache holds too
    s["table"] = _i32(np.where(table >= 0, order[table], -1))
    s["lens"] = _i32([n for n in lens for _ in range(beams)])
    s["refs"] = _i32(refs)
    s["cache"] = _cache(c, blocks, c["layers"], g)
    parents = [y * beams + min(rng.randrange(beams), rng.randrange(beams)) for y in range(groups) for _ in range(beams)]
    grow = [c["grow"]] * len(parents)
    if groups >= 4:  # requests that are over give their pages back
        for y in range(0, groups, 8):
            for b in range(beams):
                parents[y * beams + b], grow[y * beams + b] = -1, 0
    s["parents"], s["grow"] = _i32(parents), _i32(grow)


def _prepare_compact(c, g, rng, s):
    blocks = c["blocks"]
    held = max(1, int(blocks * c["held"]))
    order = torch.randperm(blocks, generator=g, device="cuda").cpu().numpy()
    seqs = min(c["seqs"], held)
    rows = np.array_split(order[:held], seqs)
    table = np.full((seqs, max(len(r) for r in rows) + 2), -1, np.int32)
    refs = np.zeros(blocks, np.int32)
    for q, r in enumerate(rows):
        shared = len(r) // 4 if q else 0  # a prompt shared with the sequence before
        table[q, : len(r)] = r
        if shared:
            n = min(shared, len(rows[q - 1]))
            table[q, :n] = table[q - 1, :n]
            refs[r[:n]] += 1  # its own pages are held by something else
    np.add.at(refs, table[table >= 0], 1)
    s["table"], s["refs"] = _i32(table), _i32(refs)
    s["cache"] = _cache(c, blocks, c["layers"], g)


def prepare(case, seed):
    s = {"case": case}
    {"attention": _prepare_attention, "beam": _prepare_beam, "fork": _prepare_fork, "compact": _prepare_compact}[case["op"]](
        case, _gen(seed), random.Random(seed), s)
    return s


# ------------------------------------------------------------------ plain forms
def _views(layer, c):
    """K and V of one layer [2][blocks][piece] as [blocks][token][head][...] views, the last axes one head's values."""
    n, t, h, d = layer.shape[1], c["tokens"], c["heads"], c["dim"]
    raw = layer.view(torch.uint8) if c["cache"] == "f8" else layer
    if c["layout"] == "piece":
        return raw[0].view(n, t, h, d), raw[1].view(n, t, h, d)
    if c["layout"] == "hnd":
        return raw[0].view(n, h, t, d).transpose(1, 2), raw[1].view(n, h, t, d).transpose(1, 2)
    x = 16 // layer.element_size()
    return raw[0].view(n, h, d // x, t, x).permute(0, 3, 1, 2, 4), raw[1].view(n, h, d, t).permute(0, 3, 1, 2)


def _floats(x, c):
    x = x.contiguous()
    return (x.view(torch.float8_e4m3fn) if c["cache"] == "f8" else x).float()


def _plain_attention(s):
    c = s["case"]
    n, h, g, d, m, t = c["seqs"], c["heads"], c["group"], c["dim"], s["longest"], c["draft"]
    lens, start = s["lens"].long(), s["start"].long()
    at = torch.arange(m, device="cuda")
    held = at < (lens + start[1:] - start[:-1])[:, None]
    block = torch.where(held, s["table"].long()[:, torch.div(at, c["tokens"], rounding_mode="floor")], torch.zeros_like(held).long())
    kv, vv = _views(s["cache"][0], c)
    off = (at % c["tokens"]).expand(n, m)
    k = _floats(kv[block, off].reshape(n, m, h, d), c)
    v = _floats(vv[block, off].reshape(n, m, h, d), c)
    if c["cache"] == "f8":
        k, v = k * s["k_scale"][:, None], v * s["v_scale"][:, None]
    row = torch.arange(s["q"].shape[0], device="cuda")
    seq = torch.searchsorted(start[1:].contiguous(), row, right=True)
    i = row - start[seq]
    q = torch.zeros(n, t, h, g, d, device="cuda")
    q[seq, i] = s["q"].float().view(-1, h, g, d)
    q = q.permute(0, 2, 1, 3, 4).reshape(n * h, t * g, d) * d ** -0.5
    x = torch.bmm(q, k.permute(0, 2, 3, 1).reshape(n * h, d, m)).view(n, h, t, g, m)
    del k, q
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    away = (lens[:, None] + torch.arange(t, device="cuda"))[:, :, None] - at  # of each token from each entry
    if c["slopes"]:
        x = x - s["slopes"].view(1, h, 1, g, 1) * away.abs().float()[:, None, :, None, :]
    sees = away >= 0
    if c["window"]:
        sees = sees & (away < c["window"])
    if c["prefix"]:
        sees = sees | (at < s["prefix"][:, None])[:, None]
    sees = sees & held[:, None]
    del away
    x = x.masked_fill(~sees[:, None, :, None, :], float("-inf"))
    top = x.amax(-1, keepdim=True).clamp_min(-3e38)
    p = torch.exp(x - top)
    del x
    total = p.sum(-1, keepdim=True)
    p = p / total.clamp_min(1e-38)
    o = torch.bmm(p.view(n * h, t * g, m), v.permute(0, 2, 1, 3).reshape(n * h, m, d))
    o = o.view(n, h, t, g, d).permute(0, 2, 1, 3, 4).reshape(n, t, h * g, d)
    lse = (top + torch.log(total)).squeeze(-1).permute(0, 2, 1, 3).reshape(n, t, h * g)
    out = {"out": o[seq, i].to(TYPES[c["type"]]), "lse": lse[seq, i]}
    if c["scores"]:
        real = torch.zeros(n, t, device="cuda")
        real[seq, i] = 1
        mass = (p * real[:, None, :, None, None]).sum((2, 3))
        old = torch.where((at < lens[:, None])[:, None], DECAY * s["scores_in"], torch.zeros_like(s["scores_in"]))
        out["scores"] = torch.where(held[:, None], old + mass, torch.zeros_like(mass))
    return out


def _plain_beam(s):
    c = s["case"]
    x = s["logits"].double()
    top = x.amax(-1, keepdim=True)
    lse = top + torch.log(torch.exp(x - top).sum(-1, keepdim=True))
    score = s["scores"].double().view(-1, 1)
    v = score + (x - lse)
    if c["done"]:
        over = s["done"].view(-1, 1).bool()
        only = torch.full_like(v, float("-inf"))
        only[:, c["vocab"] - 1] = score[:, 0]
        v = torch.where(over, only, v)
    v = torch.where(torch.isnan(v), torch.full_like(v, float("-inf")), v).view(c["batch"], -1)
    best, at = torch.sort(v, dim=-1, descending=True, stable=True)
    best, at = best[:, : c["keep"]], at[:, : c["keep"]]
    some = best > float("-inf")
    beam = torch.div(at, c["vocab"], rounding_mode="floor") + torch.arange(c["batch"], device="cuda")[:, None] * c["beams"]
    none = torch.full_like(at, -1)
    return {"tokens": torch.where(some, at % c["vocab"], none).int(), "parents": torch.where(some, beam, none).int(),
            "scores": best.float()}


def _plain_fork(s):
    c = s["case"]
    bt, table, refs = c["tokens"], s["table"].long(), s["refs"].clone()
    blocks, width = refs.shape[0], table.shape[1]
    there = (table >= 0) & (table < blocks)
    refs.index_add_(0, table[there], torch.full_like(table[there], -1).int())
    p = s["parents"].long()
    child = torch.arange(p.shape[0], device="cuda")
    n = torch.where(p >= 0, s["lens"].long()[p.clamp_min(0)], torch.zeros_like(p))
    full, here = torch.div(n, bt, rounding_mode="floor"), torch.div(n + bt - 1, bt, rounding_mode="floor")
    old = table[p.clamp_min(0)]
    j = torch.arange(width, device="cuda")
    take = j < full[:, None]
    out = torch.where(take, old, torch.full_like(old, -1))
    refs.index_add_(0, out[out >= 0], torch.ones_like(out[out >= 0]).int())
    last = torch.where(here > full, old.gather(1, full[:, None].clamp_max(width - 1))[:, 0], torch.full_like(p, -1))
    has = last >= 0
    first = torch.full((blocks,), p.shape[0], dtype=torch.int64, device="cuda")
    first.scatter_reduce_(0, last[has], child[has], "amin")
    keep = has & (refs[last.clamp_min(0)] == 0) & (first[last.clamp_min(0)] == child)
    out[child[keep], full[keep]] = last[keep]
    refs[last[keep]] = 1
    until = torch.div(n + s["grow"] + bt - 1, bt, rounding_mode="floor").clamp_max(width)
    want = ((j >= here[:, None]) & (j < until[:, None])) | ((j == full[:, None]) & (has & ~keep)[:, None])
    rank = (torch.cumsum(want.flatten(), 0) - 1).view_as(want)
    free = torch.nonzero(refs == 0)[:, 0]
    given = want & (rank < free.shape[0])
    out[given] = free[rank[given]]
    refs[out[given]] = 1
    left = (free.shape[0] - want.sum()).view(1).int()
    copied = has & ~keep
    src, dst = last[copied], out[child[copied], full[copied]]
    raw = s["cache"].view(torch.uint8) if c["cache"] == "f8" else s["cache"]
    raw[:, :, dst[dst >= 0]] = raw[:, :, src[dst >= 0]]
    return {"cache": s["cache"], "table": out.int(), "lens": n.int(), "refs": refs, "free": left}


def _plain_compact(s):
    c = s["case"]
    refs, table = s["refs"], s["table"].long()
    at = torch.arange(refs.shape[0], device="cuda")
    held = refs != 0
    n = held.sum()
    src, dst = torch.nonzero(held & (at >= n))[:, 0], torch.nonzero(~held & (at < n))[:, 0]
    moved = torch.where(held, at, torch.full_like(at, -1))
    moved[src] = dst
    raw = s["cache"].view(torch.uint8) if c["cache"] == "f8" else s["cache"]
    raw[:, :, dst] = raw[:, :, src]
    after = refs.clone()
    after[dst] = refs[src]
    after[src] = 0
    to = moved[table.clamp_min(0)]
    return {"cache": s["cache"], "table": torch.where((table >= 0) & (to >= 0), to, table).int(), "refs": after,
            "moved": moved.int(), "held": n.view(1).int()}


# ------------------------------------------------------------------ the framework's calls
_ready = None


def _mma():
    global _ready
    if _ready is None:
        import paper_2512_16056_amd as mma
        torch.cuda.set_device(0)
        mma.mma_init(0)
        _ready = mma
    return _ready


def _handles(s):
    """The layout, the sequences' description and the layers' table, which a program keeps from call to call."""
    if "handles" not in s:
        mma, c = _mma(), s["case"]
        layout = mma.kv_layout(c.get("layers", 1), c["tokens"], c["heads"], c["dim"], s["cache"].element_size(),
                               s["cache"].shape[2], 1, {"piece": mma.MMA_KV_LAYOUT_PIECE, "hnd": mma.MMA_KV_LAYOUT_HND,
                                                        "xpacked": mma.MMA_KV_LAYOUT_XPACKED}[c["layout"]])
        seqs = None
        if c["op"] == "attention":
            seqs = mma.kv_seqs(s["table"], s["lens"], s["start"], max_tokens=c["draft"], max_len=s["longest"])
        elif c["op"] == "fork":
            seqs = mma.kv_seqs(s["table"], s["lens"], max_tokens=0, max_len=c["len"])
        s["handles"] = layout, seqs, mma.layer_table(list(s["cache"]))
    return s["handles"]


def _own_attention(s):
    mma, c = _mma(), s["case"]
    layout, seqs, _ = _handles(s)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    more = {"scores_in": s["scores_in"], "scores_out": s["scores_out"], "decay": DECAY} if c["scores"] else {}
    out = mma.mma_kv_attention(layout, s["cache"][0], seqs, s["q"], lse=lse, k_scale=s.get("k_scale"),
                               v_scale=s.get("v_scale"), softcap=c["cap"], window=c["window"], slopes=s.get("slopes"),
                               prefix=s.get("prefix"), max_prefix=c["prefix"], **more)
    return {"out": out, "lse": lse, "scores": s["scores_out"]} if c["scores"] else {"out": out, "lse": lse}


def _own_beam(s):
    c = s["case"]
    tokens, parents, scores = _mma().mma_beam_select(s["logits"], s["scores"], c["keep"], done=s.get("done"),
                                                     done_token=c["vocab"] - 1)
    return {"tokens": tokens, "parents": parents, "scores": scores}


def _own_fork(s):
    layout, seqs, layers = _handles(s)
    table, lens, refs, free = _mma().mma_kv_fork(layout, layers, seqs, s["parents"], s["refs"], grow=s["grow"])
    return {"cache": s["cache"], "table": table, "lens": lens, "refs": refs, "free": free}


def _own_compact(s):
    layout, _, layers = _handles(s)
    table, refs, moved, held = _mma().mma_kv_compact(layout, layers, s["table"], s["refs"])
    return {"cache": s["cache"], "table": table, "refs": refs, "moved": moved, "held": held}


def run(state):
    op = state["case"]["op"]
    if own:
        return {"attention": _own_attention, "beam": _own_beam, "fork": _own_fork, "compact": _own_compact}[op](state)
    return {"attention": _plain_attention, "beam": _plain_beam, "fork": _plain_fork, "compact": _plain_compact}[op](state)


# ------------------------------------------------------------------ work and results
def work(case):
    """Bytes and operations; of forks the pages that are copied on average."""
    c = case
    if c["op"] == "beam":
        rows = c["batch"] * c["beams"]
        live = 0.7 if c["done"] else 1.0
        return {"bytes": live * rows * c["vocab"] * (4 if c["type"] == "f32" else 2) + rows * 5 + c["batch"] * c["keep"] * 12,
                "flops": live * rows * c["vocab"] * 20}
    elem = 1 if c["cache"] == "f8" else 2
    entry = 2 * c["heads"] * c["dim"] * elem  # K and V
    page = entry * c["tokens"]
    if c["op"] == "fork":
        seqs, width = c["groups"] * c["beams"], _up(c["len"] + c["grow"], c["tokens"]) + 1
        live = 1 - _up(c["groups"], 8) / c["groups"] if c["groups"] >= 4 else 1
        b = c["beams"]
        # A child takes beam x with probability ((b - x)^2 - (b - x - 1)^2) / b^2; the first child of each keeps its page.
        parents = sum(1 - (1 - ((b - x) ** 2 - (b - x - 1) ** 2) / b ** 2) ** b for x in range(b))
        copied = c["groups"] * live * (b - parents)
        return {"bytes": 2 * copied * page * c["layers"] + 8 * seqs * width + 16 * seqs, "flops": 0}
    if c["op"] == "compact":
        held = max(1, int(c["blocks"] * c["held"]))
        moved = held * (1 - held / c["blocks"])
        return {"bytes": 2 * moved * page * c["layers"] + 8 * held + 12 * c["blocks"], "flops": 0}
    lens, draft, prefix = _sizes(c)
    entries, seen = 0, 0
    for n, t, p in zip(lens, draft, prefix):
        p = min(p, n + t)
        low = max(p, n + 1 - c["window"]) if c["window"] else p
        entries += min(n + t, p + max(0, n + t - low))
        for i in range(n, n + t):
            seen += p + max(0, i + 1 - max(p, i + 1 - c["window"] if c["window"] else 0))
    q = c["heads"] * c["group"] * c["dim"] * 2
    rows = sum(draft) * c["heads"] * c["group"]
    scores = sum(lens) * c["heads"] * 8 + sum(draft) * c["heads"] * 4 if c["scores"] else 0
    return {"bytes": entries * entry + 2 * sum(draft) * q + 4 * rows + scores,
            "flops": 4 * seen * c["heads"] * c["group"] * c["dim"]}


def _entry(s, q, at):
    """K and V [entries][heads][dim] of the entries `at` of sequence q, by plain address arithmetic, in 64 bits."""
    c = s["case"]
    t, h, d = c["tokens"], c["heads"], c["dim"]
    flat = s["cache"][0].reshape(2, -1)
    flat = flat.view(torch.uint8) if c["cache"] == "f8" else flat
    b, o = s["table"][q].long()[at // t][:, None, None] * (t * h * d), (at % t)[:, None, None]
    hh, dd = torch.arange(h, device="cuda").view(1, h, 1), torch.arange(d, device="cuda").view(1, 1, d)
    if c["layout"] == "piece":
        ki = vi = b + (o * h + hh) * d + dd
    elif c["layout"] == "hnd":
        ki = vi = b + (hh * t + o) * d + dd
    else:
        x = 16 // flat.element_size()
        ki, vi = b + ((hh * (d // x) + dd // x) * t + o) * x + dd % x, b + (hh * d + dd) * t + o
    k, v = flat[0][ki], flat[1][vi]
    if c["cache"] == "f8":
        return (k.view(TYPES["f8"]).double() * s["k_scale"].double()[:, None],
                v.view(TYPES["f8"]).double() * s["v_scale"].double()[:, None])
    return k.double(), v.double()


def _exact_attention(s):
    c = s["case"]
    h, g, d = c["heads"], c["group"], c["dim"]
    lens, draft, prefix = _sizes(c)
    out = torch.zeros(sum(draft), h * g, d, dtype=torch.float64, device="cuda")
    lse = torch.full((sum(draft), h * g), -math.inf, dtype=torch.float64, device="cuda")
    scores = torch.zeros(s["scores_out"].shape, dtype=torch.float64, device="cuda") if c["scores"] else None
    a = 0
    for q, (n, t, p) in enumerate(zip(lens, draft, prefix)):
        k, v = _entry(s, q, torch.arange(n + t, device="cuda"))
        i = torch.arange(n, n + t, device="cuda")[:, None]
        j = torch.arange(n + t, device="cuda")[None]
        hidden = ((j > i) | (i - j >= (c["window"] or n + t))) & (j >= p)
        for y in range(h):
            mass = torch.zeros(n + t, dtype=torch.float64, device="cuda")
            for e in range(g):
                x = s["q"][a: a + t, y * g + e].double() @ k[:, y].t().contiguous() / math.sqrt(d)
                if c["cap"]:
                    x = torch.tanh(x / c["cap"]) * c["cap"]
                if c["slopes"]:
                    x -= (i - j).abs() * s["slopes"][y * g + e].double()
                x[hidden] = -math.inf
                w = torch.logsumexp(x, 1)
                x = torch.exp(x - w[:, None])
                out[a: a + t, y * g + e] = x @ v[:, y].contiguous()
                lse[a: a + t, y * g + e] = w
                mass += x.sum(0)
            if c["scores"]:
                mass[:n] += DECAY * s["scores_in"][q, y, :n].double()
                scores[q, y, : n + t] = mass
        a += t
    return {"out": out, "lse": lse, "scores": scores} if c["scores"] else {"out": out, "lse": lse}


def _exact_beam(s):
    c = s["case"]
    x = s["logits"].cpu().double().numpy().reshape(c["batch"], c["beams"], c["vocab"])
    score = s["scores"].cpu().double().numpy()
    done = s["done"].cpu().numpy() if c["done"] else np.zeros(score.shape, np.uint8)
    out = np.full((c["batch"], c["keep"]), -np.inf)
    for b in range(c["batch"]):
        found = []
        for y in range(c["beams"]):
            if score[b, y] == -np.inf:
                continue
            if done[b, y]:
                found.append(score[b, y: y + 1])
                continue
            z = x[b, y] - x[b, y].max()
            z = z - math.log(np.exp(z).sum())
            found.append(score[b, y] + np.sort(z[z > -np.inf])[::-1][: c["keep"]])
        best = np.sort(np.concatenate(found))[::-1][: c["keep"]] if found else np.zeros(0)
        out[b, : len(best)] = best
    return {"tokens": None, "parents": None, "scores": torch.from_numpy(out).cuda()}


def _moves(s, pairs):
    """The cache in 64 bits after pages moved."""
    cache = s["cache"].double()
    for a, b in pairs:
        cache[:, :, b] = s["cache"][:, :, a].double()
    return cache


def _exact_fork(s):
    """Page by page, child by child."""
    bt, table = s["case"]["tokens"], s["table"].tolist()
    refs, lens, parents, grow = s["refs"].tolist(), s["lens"].tolist(), s["parents"].tolist(), s["grow"].tolist()
    width, pairs, need = len(table[0]), [], []
    for row in table:
        for x in row:
            if x >= 0:
                refs[x] -= 1
    for p in parents:
        for x in table[p][: lens[p] // bt] if p >= 0 else []:
            refs[x] += 1
    for i, p in enumerate(parents):
        n = lens[p] if p >= 0 else 0
        if n % bt:
            x = table[p][n // bt]
            if refs[x] == 0:
                refs[x] = 1
            else:
                need.append((i, x))
        need += [(i, None)] * max(0, min(_up(n + grow[i], bt), width) - _up(n, bt))
    free = [x for x, r in enumerate(refs) if r == 0]
    for (_, x), to in zip(need, free):
        if x is not None:
            pairs.append((x, to))
    return {"cache": _moves(s, pairs), "table": None, "lens": None, "refs": None, "free": None}


def _exact_compact(s):
    refs = s["refs"].tolist()
    n = sum(r != 0 for r in refs)
    pairs = zip((x for x in range(n, len(refs)) if refs[x]), [x for x in range(n) if not refs[x]])
    return {"cache": _moves(s, pairs), "table": None, "refs": None, "moved": None, "held": None}


def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "beam": _exact_beam, "fork": _exact_fork, "compact": _exact_compact}[case["op"]](s)
