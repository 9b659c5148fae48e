"""The operators of a decode step on the paged KV cache, as a serving program calls them, and their plain forms.

append     queries and keys normalised per head and rotated, keys and values written into the cache
attention  a few tokens of each sequence (one, a tree of drafted ones, a prompt chunk) over its cache
commit     the accepted tokens of a draft moved together, in every layer
evict      the entries with the highest accumulated attention weight kept, per KV head

listed() names twelve cases, draw() gives more of the same ranges. Where `own` is false, run() computes
the plain form with elementary torch operations in 32 bits, rounded once; where it is true it makes the
calls of this repository's package. exact() computes the definitions in 64 bits, one sequence at a time.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f8": torch.float8_e4m3fn}
F8_MAX = 448.0
EPS = 1e-6


def _case(name, op, layout, cache, **kw):
    c = {"op": op, "layout": layout, "cache": cache, "type": "bf16", "tokens": 16, "heads": 8, "group": 4,
         "dim": 128, "seqs": 1}
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One user, one token: the smallest call, where latency is all there is.
        _case("append_1_token", "append", "piece", "bf16", draft=1, len=1000, rot=128, interleaved=False, norm=True),
        # A 4k-token prompt in chunks of several users, head-major cache, no norms, old half-precision model.
        _case("append_prompts", "append", "hnd", "f16", type="f16", seqs=3, draft=1365, len=700, rot=128,
              interleaved=False, norm=False),
        # Drafts of 17 tokens for 40 users into an 8-bit cache for paged decode; a quarter of the head rotates.
        _case("append_drafts_f8", "append", "xpacked", "f8", seqs=40, draft=17, len=300, rot=32, interleaved=True,
              norm=True),
        # One user at the start of a chat: one token over about a hundred entries.
        _case("decode_short", "attention", "piece", "bf16", draft=1, len=101, tree=False, scores=False),
        # A batch of 32 users with ragged contexts up to 8k, head-major cache.
        _case("decode_batch", "attention", "hnd", "bf16", seqs=32, draft=1, len=8192, tree=False, scores=False),
        # The 64k-token context of the KV-fetch workload, with the weights that eviction goes by.
        _case("decode_64k_scores", "attention", "piece", "bf16", draft=1, len=65535, tree=False, scores=True),
        # Trees of 24 drafted tokens of 4 users over long contexts in an 8-bit cache for paged decode.
        _case("tree_24_f8", "attention", "xpacked", "f8", seqs=4, draft=24, len=15003, tree=True, scores=True),
        # A 2k-token prompt chunk behind 6k tokens that a fetch brought back.
        _case("prompt_chunk", "attention", "hnd", "bf16", draft=2048, len=6144, tree=False, scores=False),
        # One user's draft accepted to depth 5, 32 layers.
        _case("commit_1_seq", "commit", "piece", "bf16", draft=24, len=90, accept=5, layers=32),
        # 24 users' drafts, 8-bit paged-decode cache.
        _case("commit_batch", "commit", "xpacked", "f8", seqs=24, draft=32, len=60, accept=8, layers=24),
        # The 64k-token context cut to a quarter before it is offloaded.
        _case("evict_64k_to_16k", "evict", "piece", "bf16", len=65536, keep=16384, sinks=4, recent=256),
        # A batch of 12 users cut to 1k entries each, 8-bit head-major cache, five KV heads.
        _case("evict_batch_f8", "evict", "hnd", "f8", seqs=12, heads=5, len=4999, keep=1021, sinks=4, recent=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["append", "attention", "attention", "attention", "commit", "evict"])
    cache = rng.choice(["bf16", "bf16", "f16", "f8"])
    layout = rng.choice(["piece", "hnd", "xpacked"])
    kind = "f16" if cache == "f16" or cache == "f8" and rng.random() < 0.3 else "bf16"
    c = {"type": kind, "heads": rng.choice([1, 2, 4, 5, 8, 8]),
         "group": rng.choice([1, 2, 3, 4, 4, 5, 7, 8]), "dim": rng.choice([64, 80, 96, 128, 128, 256]),
         "tokens": rng.choice([16, 16, 32] if layout == "xpacked" else [8, 16, 16, 24, 32])}
    row = c["heads"] * c["dim"]
    if op == "append":
        total = _log(rng, 1, max(1, 4_194_304 // row))
        seqs = min(_log(rng, 1, 64), total)
        half = c["dim"] // 2
        c.update(seqs=seqs, draft=total // seqs, len=_log(rng, 1, 1000),
                 rot=rng.choice([c["dim"], c["dim"], 2 * rng.randint(1, half)]),
                 interleaved=rng.random() < 0.5, norm=rng.random() < 0.6)
    elif op == "attention":
        kind = rng.choice(["one", "one", "tree", "tree", "chunk"])
        draft = 1 if kind == "one" else _log(rng, 2, 128) if kind == "tree" else _log(rng, 16, 2048)
        rows = draft * c["heads"] * c["group"]
        top = min(67_000_000 // row, 520_000_000 // rows, int(2.4e11) // (4 * rows * c["dim"]))
        seqs = _log(rng, 1, max(1, min(64, top // (64 + draft))))
        c.update(seqs=seqs, draft=draft, len=_log(rng, 1, max(1, min(131072, top // seqs - draft))),
                 tree=kind == "tree", scores=rng.random() < 0.5)
    elif op == "commit":
        c.update(seqs=_log(rng, 1, 24), draft=_log(rng, 4, 64), len=rng.randint(1, 90), layers=rng.randint(2, 32))
        c["accept"] = rng.randint(1, min(c["draft"], 12))
    else:
        seqs = _log(rng, 1, 32)
        n = _log(rng, 32, max(32, min(65536, 67_000_000 // row // seqs)))
        keep = rng.randint(8, max(8, n // 2))
        c.update(seqs=seqs, len=n, keep=keep, sinks=rng.randint(0, 4), recent=rng.randint(0, keep // 2))
    return _case(None, op, layout, cache, **c)


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0, std, generator=g)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _lens(c, rng):
    """Entries of each sequence: the case's length is the longest, the others are ragged; in a batch one is new."""
    n = [c["len"]] + [rng.randint(c["len"] // 8, c["len"]) for _ in range(c["seqs"] - 1)]
    if c["seqs"] >= 8 and c["op"] != "evict":
        n[1] = 0
    rng.shuffle(n)
    return n


def _counts(c, rng):
    """New tokens of each sequence: the same for single tokens and drafts of one user, else ragged."""
    t = [c["draft"]] + [rng.randint(max(1, c["draft"] // 2), c["draft"]) for _ in range(c["seqs"] - 1)]
    rng.shuffle(t)
    return t


def _f8(x):
    return x.clamp(-F8_MAX, F8_MAX).to(torch.float8_e4m3fn)


def _blank(c, blocks, layers, g):
    """A cache [layers][2][blocks][piece] with what earlier requests left in it."""
    n = layers * 2 * blocks * c["tokens"] * c["heads"] * c["dim"]
    x = _normal(g, n)
    x = _f8(x * 20) if c["cache"] == "f8" else x.to(TYPES[c["cache"]])
    return x.view(layers, 2, blocks, -1)


def _tables(c, need, spare, g):
    """Block tables [sequences][widest] with blocks in random order, -1 behind each one's last, and the number of blocks."""
    total = sum(need) + spare
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32).cpu().numpy()
    table = np.full((len(need), max(max(need), 1)), -1, np.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at: at + n]
        at += n
    return torch.from_numpy(table).cuda(), total


def _rope_table(rot, rows, base=500000.0):
    """cos and sin of every position and pair, [rows][rot]: what a program keeps for its model."""
    f = base ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    a = np.arange(rows, dtype=np.float64)[:, None] * f
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)).cuda()


def _tree(counts, rng):
    """Bits [tokens][words]: bit d of a token's row says that it sees drafted token d of its sequence (ancestors and itself)."""
    words = (max(counts) + 63) // 64
    rows = []
    for t in counts:
        bits = []
        for i in range(t):
            parent = bits[rng.randrange(max(0, i - 8), i)] if i else 0
            bits.append(parent | (1 << i))
        rows += [[(b >> (64 * w)) & ((1 << 64) - 1) for w in range(words)] for b in bits]
    return torch.from_numpy(np.array(rows, dtype=np.uint64).view(np.int64)).cuda()


def _accepted(c, counts, rng):
    """Ascending drafted tokens of each sequence that were accepted, -1 behind them, and how many."""
    n = [min(c["accept"], t) if s == 0 else rng.randint(0, min(c["accept"], t)) for s, t in enumerate(counts)]
    acc = [sorted(rng.sample(range(t), k)) for t, k in zip(counts, n)]
    return _i32([a + [-1] * (c["accept"] - len(a)) for a in acc]), _i32(n)


def prepare(case, seed):
    c, g, rng = case, _gen(seed), random.Random(seed)
    bt = c["tokens"]
    sizes = random.Random(c["len"] * 131 + c["seqs"])  # which sequence has how many: of the case, so that shapes are
    lens = _lens(c, sizes)
    s = {"case": c, "lens": _i32(lens)}
    if c["op"] == "evict":
        src = [(n + bt - 1) // bt for n in lens]
        dst = [(min(n, c["keep"]) + bt - 1) // bt for n in lens]
        both, blocks = _tables(c, src + dst, 3, g)
        s["table"] = both[: c["seqs"], : max(src)].contiguous()
        s["dst"] = both[c["seqs"]:, : max(dst)].contiguous()
        s["cache"] = _blank(c, blocks, 1, g)
        # A heavy tail, and entries that no query has looked at yet.
        x = torch.exp(2.5 * _normal(g, c["seqs"], c["heads"], c["len"]))
        s["scores"] = torch.where(x < 0.1, torch.zeros_like(x), x)
        return s
    counts = _counts(c, sizes)
    need = [(n + t + bt - 1) // bt for n, t in zip(lens, counts)]
    s["table"], blocks = _tables(c, need, 3, g)
    s["cache"] = _blank(c, blocks, c.get("layers", 1), g)
    s["start"] = _i32([0] + list(np.cumsum(counts)))
    s["longest"] = max(n + t for n, t in zip(lens, counts))
    total, heads, dim = sum(counts), c["heads"], c["dim"]
    if c["op"] == "commit":
        s["accepted"], s["counts"] = _accepted(c, counts, rng)
        s["scores"] = torch.rand(c["layers"], c["seqs"], heads, s["longest"], generator=g, device="cuda")
        return s
    if c["cache"] == "f8":
        s["k_scale"] = torch.rand(heads, generator=g, device="cuda") * 0.02 + 0.02
        s["v_scale"] = torch.rand(heads, generator=g, device="cuda") * 0.02 + 0.02
    if c["op"] == "append":
        # One projection's output: queries, keys and values of a token side by side.
        qkv = _normal(g, total, (c["group"] + 2) * heads, dim, std=1.5).to(TYPES[c["type"]])
        s["qkv"] = qkv
        s["positions"] = _i32([n + i for n, t in zip(lens, counts) for i in range(t)])
        s["rope"] = _rope_table(c["rot"], s["longest"])
        if c["norm"]:
            s["q_weight"] = (1 + _normal(g, dim, std=0.2)).to(TYPES[c["type"]])
            s["k_weight"] = (1 + _normal(g, dim, std=0.2)).to(TYPES[c["type"]])
        return s
    s["q"] = _normal(g, total, heads * c["group"], dim, std=2.0).to(TYPES[c["type"]])
    if c["tree"]:
        s["tree"] = _tree(counts, rng)
    if c["scores"]:
        s["scores_in"] = torch.exp(_normal(g, c["seqs"], heads, s["longest"]))
        s["scores_out"] = torch.zeros_like(s["scores_in"])
    return s


DECAY = 0.96


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


def _where(table, at, c):
    """Block and offset of entry `at` [sequences][...] of each sequence."""
    b = torch.div(at, c["tokens"], rounding_mode="floor")
    rows = torch.arange(table.shape[0], device="cuda").view(-1, *[1] * (at.dim() - 1)).expand_as(at)
    return table.long()[rows, b.clamp(0, table.shape[1] - 1)], at % c["tokens"]


def _floats(x, c):
    x = x.contiguous()
    return (x.view(torch.float8_e4m3fn) if c["cache"] == "f8" else x).float()


def _stored(x, scale, c):
    if c["cache"] == "f8":
        return _f8(x / scale[:, None]).view(torch.uint8)
    return x.to(TYPES[c["cache"]])


def _grid(s):
    """Sequence and index within it of every new token."""
    start = s["start"].long()
    t = torch.arange(int(s["positions"].shape[0] if "positions" in s else s["q"].shape[0]), device="cuda")
    seq = torch.searchsorted(start[1:].contiguous(), t, right=True)
    return seq, t - start[seq]


def _plain_append(s):
    c = s["case"]
    hq, h, d, r = c["heads"] * c["group"], c["heads"], c["dim"], c["rot"]
    x = s["qkv"].float()
    q, k, v = x[:, :hq], x[:, hq: hq + h], x[:, hq + h:]
    if c["norm"]:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + EPS) * s["q_weight"].float()
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + EPS) * s["k_weight"].float()
    x = torch.cat([q, k], 1)
    row = s["rope"][s["positions"].long()][:, None]
    cos, sin = row[..., : r // 2], row[..., r // 2:]
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., : r // 2], x[..., r // 2: r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    x = torch.cat([turned, x[..., r:]], -1)
    seq, i = _grid(s)
    block, off = _where(s["table"][seq], (s["lens"].long()[seq] + i)[:, None], c)
    block, off = block[:, 0], off[:, 0]
    kv, vv = _views(s["cache"][0], c)
    kv[block, off] = _stored(x[:, hq:], s.get("k_scale"), c).view(-1, h, *kv.shape[3:])
    vv[block, off] = _stored(v, s.get("v_scale"), c)
    return {"q": x[:, :hq].to(TYPES[c["type"]]), "cache": s["cache"]}


def _plain_attention(s):
    c = s["case"]
    n, h, g, d, m = c["seqs"], c["heads"], c["group"], c["dim"], s["longest"]
    lens, start = s["lens"].long(), s["start"].long()
    at = torch.arange(m, device="cuda").expand(n, m)
    block, off = _where(s["table"], at, c)
    held = (at < (lens + start[1:] - start[:-1])[:, None])
    block = torch.where(held, block, torch.zeros_like(block))
    kv, vv = _views(s["cache"][0], c)
    k = _floats(kv[block, off].reshape(n, m, h, d), c)
    v = _floats(vv[block, off].reshape(n, m, h, d), c)
    if c["cache"] == "f8":
        k, v = k * s["k_scale"][:, None], v * s["v_scale"][:, None]
    seq, i = _grid(s)
    t = c["draft"]
    q = torch.zeros(n, t, h, g, d, device="cuda")
    q[seq, i] = s["q"].float().view(-1, h, g, d)
    q = q.permute(0, 2, 1, 3, 4).reshape(n * h, t * g, d) * d ** -0.5
    logits = torch.bmm(q, k.permute(0, 2, 3, 1).reshape(n * h, d, m)).view(n, h, t, g, m)
    del k, q
    j = at[:, None, :] - lens[:, None, None]  # of entry j: the drafted token it is, negative for the context
    if c["tree"]:
        bits = torch.zeros(n, t, s["tree"].shape[1], dtype=torch.int64, device="cuda")
        bits[seq, i] = s["tree"]
        word = torch.div(j, 64, rounding_mode="floor").clamp(0, bits.shape[2] - 1)
        sees = ((bits.gather(2, word.expand(n, t, m)) >> (j % 64)) & 1).bool() | (j < 0)
    else:
        sees = j <= torch.arange(t, device="cuda")[None, :, None]
    sees = sees & held[:, None]
    logits = logits.masked_fill(~sees[:, None, :, None, :], float("-inf"))
    top = logits.amax(-1, keepdim=True).clamp_min(-3e38)
    p = torch.exp(logits - top)
    del logits
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


def _plain_commit(s):
    c = s["case"]
    i = torch.arange(c["accept"], device="cuda").expand(c["seqs"], -1)
    live = i < s["counts"][:, None]
    src = s["lens"].long()[:, None] + s["accepted"].long().clamp_min(0)
    dst = s["lens"].long()[:, None] + i
    seq = torch.arange(c["seqs"], device="cuda")[:, None].expand_as(i)[live]
    sb, so = (x[live] for x in _where(s["table"], src, c))
    db, do = (x[live] for x in _where(s["table"], dst, c))
    # every layer at once: [layers][2][blocks][piece] as layers in front of the views' axes
    raw = s["cache"].view(torch.uint8) if c["cache"] == "f8" else s["cache"]
    n, t, h, d, l = raw.shape[2], c["tokens"], c["heads"], c["dim"], c["layers"]
    if c["layout"] == "piece":
        k, v = raw[:, 0].view(l, n, t, h, d), raw[:, 1].view(l, n, t, h, d)
    elif c["layout"] == "hnd":
        k, v = raw[:, 0].view(l, n, h, t, d).transpose(2, 3), raw[:, 1].view(l, n, h, t, d).transpose(2, 3)
    else:
        x = 16 // raw.element_size()
        k = raw[:, 0].view(l, n, h, d // x, t, x).permute(0, 1, 4, 2, 3, 5)
        v = raw[:, 1].view(l, n, h, d, t).permute(0, 1, 4, 2, 3)
    k[:, db, do] = k[:, sb, so]
    v[:, db, do] = v[:, sb, so]
    s["scores"][:, seq, :, dst[live]] = s["scores"][:, seq, :, src[live]]
    return {"cache": s["cache"], "scores": s["scores"], "lens": s["lens"] + s["counts"]}


def _plain_evict(s):
    c = s["case"]
    n, h, m, keep = c["seqs"], c["heads"], c["len"], min(c["keep"], c["len"])
    lens = s["lens"].long()[:, None, None]
    at = torch.arange(m, device="cuda").view(1, 1, m)
    kept = lens.clamp_max(c["keep"])
    x = torch.where((at < c["sinks"]) | (at >= lens - c["recent"]), torch.full_like(s["scores"], float("inf")), s["scores"])
    x = torch.where(at < lens, x, torch.full_like(x, float("-inf")))
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :keep]
    i = torch.arange(keep, device="cuda").view(1, 1, keep)
    order = torch.sort(torch.where(i < kept, order, torch.full_like(order, m)), dim=-1).values
    live = (i < kept).expand_as(order)
    pos = order.clamp_max(m - 1)
    seq, head, slot = (torch.arange(z, device="cuda").view(w).expand_as(order)[live]
                       for z, w in ((n, (-1, 1, 1)), (h, (1, -1, 1)), (keep, (1, 1, -1))))
    sb, so = (x[live] for x in _where(s["table"], pos, c))
    db, do = (x[live] for x in _where(s["dst"], i.expand_as(order), c))
    k, v = _views(s["cache"][0], c)
    k[db, do, head] = k[sb, so, head]
    v[db, do, head] = v[sb, so, head]
    scores = torch.where(live, s["scores"].gather(2, pos), torch.zeros_like(s["scores"][..., :keep]))
    return {"cache": s["cache"], "scores": scores, "entries": torch.where(live, order, torch.full_like(order, -1)).int(),
            "lens": s["lens"].clamp_max(c["keep"])}


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
    """The layout, the sequences' description and the layers' tables, which a program keeps from call to call."""
    if "handles" not in s:
        mma, c = _mma(), s["case"]
        layout = mma.kv_layout(c.get("layers", 1), c["tokens"], c["heads"], c["dim"], s["cache"].element_size(),
                               s["cache"].shape[2], 1, {"piece": mma.MMA_KV_LAYOUT_PIECE, "hnd": mma.MMA_KV_LAYOUT_HND,
                                                        "xpacked": mma.MMA_KV_LAYOUT_XPACKED}[c["layout"]])
        if c["op"] == "evict":
            seqs = mma.kv_seqs(s["table"], s["lens"], max_tokens=0, max_len=c["len"])
        else:
            seqs = mma.kv_seqs(s["table"], s["lens"], s["start"], max_tokens=c["draft"], max_len=s["longest"])
        tables = (mma.layer_table(list(s["cache"])), mma.layer_table(list(s["scores"]))) if c["op"] == "commit" else None
        s["handles"] = layout, seqs, tables
    return s["handles"]


def _own_append(s):
    mma, c = _mma(), s["case"]
    layout, seqs, _ = _handles(s)
    hq, h = c["heads"] * c["group"], c["heads"]
    q, k, v = s["qkv"].split((hq, h, h), 1)
    out = mma.mma_kv_append(layout, s["cache"][0], seqs, q, k, v, s["positions"], s["rope"],
                            interleaved=c["interleaved"], q_weight=s.get("q_weight"), k_weight=s.get("k_weight"),
                            eps=EPS, k_scale=s.get("k_scale"), v_scale=s.get("v_scale"))
    return {"q": out, "cache": s["cache"]}


def _own_attention(s):
    mma, c = _mma(), s["case"]
    layout, seqs, _ = _handles(s)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    more = {"scores_in": s["scores_in"], "scores_out": s["scores_out"], "decay": DECAY} if c["scores"] else {}
    out = mma.mma_kv_attention(layout, s["cache"][0], seqs, s["q"], tree=s.get("tree"), lse=lse,
                               k_scale=s.get("k_scale"), v_scale=s.get("v_scale"), **more)
    return {"out": out, "lse": lse, "scores": s["scores_out"]} if c["scores"] else {"out": out, "lse": lse}


def _own_commit(s):
    mma = _mma()
    layout, seqs, (layers, scores) = _handles(s)
    lens = mma.mma_kv_commit(layout, layers, seqs, s["accepted"], s["counts"], scores=scores,
                             scores_stride=s["longest"])
    return {"cache": s["cache"], "scores": s["scores"], "lens": lens}


def _own_evict(s):
    mma, c = _mma(), s["case"]
    layout, seqs, _ = _handles(s)
    entries, scores, lens = mma.mma_kv_evict(layout, s["cache"][0], seqs, s["dst"], s["scores"], min(c["keep"], c["len"]),
                                             sinks=c["sinks"], recent=c["recent"])
    return {"cache": s["cache"], "scores": scores, "entries": entries, "lens": lens}


def run(state):
    op = state["case"]["op"]
    if own:
        return {"append": _own_append, "attention": _own_attention, "commit": _own_commit, "evict": _own_evict}[op](state)
    return {"append": _plain_append, "attention": _plain_attention, "commit": _plain_commit, "evict": _plain_evict}[op](state)


# ------------------------------------------------------------------ work and results
def work(case):
    """Bytes and operations of the longest sequences' share: ragged ones count by their mean length."""
    c = case
    elem = 1 if c["cache"] == "f8" else 2
    entry = 2 * c["heads"] * c["dim"] * elem  # K and V
    mean = (c["len"] + (c["seqs"] - 1) * c["len"] * 9 / 16) / c["seqs"]
    if c["op"] == "evict":
        kept = c["seqs"] * min(mean, c["keep"])
        return {"bytes": c["seqs"] * mean * c["heads"] * 4 + kept * (2 * entry + 8 * c["heads"]), "flops": 0}
    tokens = c["draft"] * (1 + (c["seqs"] - 1) * 3 / 4)
    if c["op"] == "commit":
        moved = c["accept"] * (1 + (c["seqs"] - 1) / 2) * c["layers"]
        return {"bytes": moved * 2 * (entry + 4 * c["heads"]), "flops": 0}
    q = c["heads"] * c["group"] * c["dim"] * 2
    if c["op"] == "append":
        kv_in = 2 * c["heads"] * c["dim"] * 2
        return {"bytes": tokens * (2 * q + kv_in + entry + 4 * c["rot"]), "flops": tokens * 5 * (q + kv_in)}
    entries = c["seqs"] * mean + tokens
    rows = tokens * c["heads"] * c["group"]
    seen = mean + (c["draft"] / 2 if not c["tree"] else min(8, c["draft"]))
    scores = entries * c["heads"] * 8 if c["scores"] else 0
    return {"bytes": entries * entry + 2 * tokens * q + 4 * rows + scores, "flops": 4 * rows * seen * c["dim"]}


def _entry(layer, table_row, at, c):
    """K and V [entries][heads][dim] of the entries `at` of one sequence, by plain address arithmetic, in 64 bits."""
    t, h, d = c["tokens"], c["heads"], c["dim"]
    flat = layer.reshape(2, -1)
    flat = flat.view(torch.uint8) if c["cache"] == "f8" else flat
    b = table_row.long()[at // t] * (t * h * d)
    o = at % t
    b, o = b[:, None, None], o[:, None, None]
    hh, dd = torch.arange(h, device="cuda").view(1, h, 1), torch.arange(d, device="cuda").view(1, 1, d)
    ki, vi = _index(b, o, hh, dd, c)
    k, v = flat[0][ki], flat[1][vi]
    return tuple((x.view(torch.float8_e4m3fn) if c["cache"] == "f8" else x).double() for x in (k, v))


def _index(b, o, hh, dd, c):
    t, h, d = c["tokens"], c["heads"], c["dim"]
    x = 16 if c["cache"] == "f8" else 8
    if c["layout"] == "piece":
        i = b + (o * h + hh) * d + dd
        return i, i
    if c["layout"] == "hnd":
        i = b + (hh * t + o) * d + dd
        return i, i
    return b + ((hh * (d // x) + dd // x) * t + o) * x + dd % x, b + (hh * d + dd) * t + o


def _exact_append(s):
    c = s["case"]
    hq, h, d, r = c["heads"] * c["group"], c["heads"], c["dim"], c["rot"]
    x = s["qkv"].double()
    out, cache = x[:, :hq].clone(), s["cache"].double()
    flat = cache[0].reshape(2, -1)
    z = [x[:, :hq], x[:, hq: hq + h]]
    for n, w in enumerate(("q_weight", "k_weight")):
        if c["norm"]:
            z[n] = z[n] / ((z[n] ** 2).sum(-1, keepdim=True) / d + EPS) ** 0.5 * s[w].double()
        turned = z[n].clone()
        rows = s["rope"].double()[s["positions"].long()]
        for i in range(r // 2):
            a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + r // 2)
            cos, sin = rows[:, None, i], rows[:, None, r // 2 + i]
            turned[..., a] = z[n][..., a] * cos - z[n][..., b] * sin
            turned[..., b] = z[n][..., b] * cos + z[n][..., a] * sin
        z[n] = turned
    start, lens = s["start"].tolist(), s["lens"].tolist()
    v = x[:, hq + h:]
    if c["cache"] == "f8":
        z[1], v = z[1] / s["k_scale"].double()[:, None], v / s["v_scale"].double()[:, None]
        z[1], v = z[1].clamp(-F8_MAX, F8_MAX), v.clamp(-F8_MAX, F8_MAX)
    hh, dd = torch.arange(h, device="cuda").view(1, h, 1), torch.arange(d, device="cuda").view(1, 1, d)
    for q in range(c["seqs"]):
        at = torch.arange(lens[q], lens[q] + start[q + 1] - start[q], device="cuda")
        b = s["table"][q].long()[at // c["tokens"]] * (c["tokens"] * h * d)
        ki, vi = _index(b[:, None, None], (at % c["tokens"])[:, None, None], hh, dd, c)
        flat[0][ki] = z[1][start[q]: start[q + 1]]
        flat[1][vi] = v[start[q]: start[q + 1]]
    return {"q": z[0], "cache": flat.view(cache.shape)}


def _exact_attention(s):
    c = s["case"]
    h, g, d = c["heads"], c["group"], c["dim"]
    start, lens = s["start"].tolist(), s["lens"].tolist()
    total = start[-1]
    out = torch.zeros(total, h * g, d, dtype=torch.float64, device="cuda")
    lse = torch.full((total, h * g), -math.inf, dtype=torch.float64, device="cuda")
    scores = s["scores_out"].double() * 0 if c["scores"] else None
    for q in range(c["seqs"]):
        a, t, n = start[q], start[q + 1] - start[q], lens[q]
        k, v = _entry(s["cache"][0], s["table"][q], torch.arange(n + t, device="cuda"), c)
        if c["cache"] == "f8":
            k, v = k * s["k_scale"].double()[:, None], v * s["v_scale"].double()[:, None]
        sees = torch.ones(t, n + t, dtype=torch.bool, device="cuda")
        if c["tree"]:
            rows = [[int(w) & ((1 << 64) - 1) for w in r] for r in s["tree"][a: a + t].tolist()]
            sees[:, n:] = torch.tensor([[(r[e // 64] >> (e % 64)) & 1 for e in range(t)] for r in rows], device="cuda").bool()
        else:
            sees[:, n:] = torch.ones(t, t, dtype=torch.bool, device="cuda").tril()
        for y in range(h):
            mass = torch.zeros(n + t, dtype=torch.float64, device="cuda")
            for e in range(g):
                x = s["q"][a: a + t, y * g + e].double() @ k[:, y].t().contiguous() / math.sqrt(d)
                x[~sees] = -math.inf
                w = torch.logsumexp(x, 1)
                p = torch.exp(x - w[:, None])
                out[a: a + t, y * g + e] = p @ v[:, y].contiguous()
                lse[a: a + t, y * g + e] = w
                mass += p.sum(0)
            if c["scores"]:
                mass[:n] += DECAY * s["scores_in"][q, y, :n].double()
                scores[q, y, : n + t] = mass
    return {"out": out, "lse": lse, "scores": scores} if c["scores"] else {"out": out, "lse": lse}


def _exact_commit(s):
    c = s["case"]
    h, d = c["heads"], c["dim"]
    cache, scores = s["cache"].double(), s["scores"].double()
    flat = cache.view(c["layers"], 2, -1)
    hh, dd = torch.arange(h, device="cuda").view(1, h, 1), torch.arange(d, device="cuda").view(1, 1, d)
    lens, counts = s["lens"].tolist(), s["counts"].tolist()
    for q in range(c["seqs"]):
        src = lens[q] + s["accepted"][q, : counts[q]].long()
        dst = torch.arange(lens[q], lens[q] + counts[q], device="cuda")
        ends = []
        for at in (src, dst):
            b = s["table"][q].long()[at // c["tokens"]] * (c["tokens"] * h * d)
            ends.append(_index(b[:, None, None], (at % c["tokens"])[:, None, None], hh, dd, c))
        for y in range(2):
            flat[:, y, ends[1][y]] = flat[:, y, ends[0][y]].clone()
        scores[:, q, :, dst] = scores[:, q, :, src].clone()
    return {"cache": cache, "scores": scores, "lens": None}


def _exact_evict(s):
    c = s["case"]
    h, d, keep = c["heads"], c["dim"], min(c["keep"], c["len"])
    cache = s["cache"].double()
    flat = cache.view(2, -1)
    scores = torch.zeros(c["seqs"], h, keep, dtype=torch.float64, device="cuda")
    dd = torch.arange(d, device="cuda").view(1, d)
    for q, n in enumerate(s["lens"].tolist()):
        w = s["scores"][q, :, :n].double().cpu().numpy()
        for y in range(h):
            if n <= keep:
                kept = np.arange(n)
            else:
                fixed = [j for j in range(min(c["sinks"], n))] + list(range(max(n - c["recent"], c["sinks"]), n))
                rest = np.arange(min(c["sinks"], n), max(n - c["recent"], c["sinks"]))
                best = rest[np.lexsort((rest, -w[y, rest]))][: keep - len(fixed)]
                kept = np.sort(np.concatenate([np.array(fixed, dtype=np.int64), best]))
            src, dst = torch.from_numpy(kept).cuda(), torch.arange(len(kept), device="cuda")
            ends = []
            for table, at in ((s["table"], src), (s["dst"], dst)):
                b = table[q].long()[at // c["tokens"]] * (c["tokens"] * h * d)
                ends.append(_index(b[:, None], (at % c["tokens"])[:, None], y, dd, c))
            for z in range(2):
                flat[z, ends[1][z]] = flat[z, ends[0][z]]
            scores[q, y, : len(kept)] = s["scores"][q, y, src].double()
    return {"cache": cache, "scores": scores, "entries": None, "lens": None}


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attention": _exact_attention, "commit": _exact_commit,
            "evict": _exact_evict}[case["op"]](s)
