"""A speculative decode loop on the paged cache, from a prompt to an evicted, offloaded and resumed context.

    python examples/kv_decode.py [--layers 4] [--prompt 3000] [--keep 512] [--layout hnd] [--cache f8]

One sequence of an untrained model (random projections): its prompt is appended and attended to in
chunks, every layer's cache is cut to the entries that got the most attention, what is left leaves for
pinned host memory over all paths and comes back into other blocks, and then steps of drafted trees run
over it: append, attention, commit. Prints what each part did and, of the attention over the evicted
cache, how much of the full context's weight the kept entries hold.
"""
import argparse
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2512_16056_amd as mma  # noqa: E402

LAYOUTS = {"piece": mma.MMA_KV_LAYOUT_PIECE, "xpacked": mma.MMA_KV_LAYOUT_XPACKED, "hnd": mma.MMA_KV_LAYOUT_HND}
HEADS, GROUP, DIM, TOKENS = 8, 4, 128, 16
DRAFT = [-1, 0, 0, 1, 2, 3, 3, 4]  # the parent of each drafted token of a step
SINKS, RECENT = 4, 64  # entries that an eviction keeps whatever their scores


class Model:
    """Projections of a few attention layers, and the buffers that a serving program keeps for them."""

    def __init__(self, a):
        g = torch.Generator(device="cuda").manual_seed(0)
        self.layers, self.f8 = a.layers, a.cache == "f8"
        self.hidden = HEADS * GROUP * DIM
        rand = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16) * s[0] ** -0.5  # noqa: E731
        self.qkv = [rand(self.hidden, (GROUP + 2) * HEADS * DIM) for _ in range(a.layers)]
        self.out = [rand(self.hidden, self.hidden) for _ in range(a.layers)]
        self.norm = torch.ones(DIM, dtype=torch.bfloat16, device="cuda")
        self.scale = torch.full((HEADS,), 0.05, device="cuda") if self.f8 else None
        rope = mma.mma_rope_table(a.prompt + 4 * a.steps + len(DRAFT), DIM, 500000.0, mma.MMA_ROPE_BANDS, factor=8.0,
                                  original_len=8192, low=1, high=4)
        self.rope = torch.from_numpy(rope).cuda()
        kept = -(-a.keep // TOKENS)
        self.blocks = -(-a.prompt // TOKENS) + kept + -(-(a.keep + 4 * a.steps + len(DRAFT)) // TOKENS)
        self.layout = mma.kv_layout(a.layers, TOKENS, HEADS, DIM, 1 if self.f8 else 2, self.blocks, kept, LAYOUTS[a.layout])
        size = mma.mma_kv_layout_sizes(self.layout)
        self.cache = [torch.zeros(size["layer"], dtype=torch.uint8, device="cuda") for _ in range(a.layers)]
        self.pool = mma.PinnedBuffer(size["pool"])
        self.free = list(range(self.blocks))

    def take(self, entries):
        n = -(-entries // TOKENS)
        got, self.free = self.free[:n], self.free[n:]
        return got

    def step(self, x, seqs, positions, tree=None, scores=None):
        """The layers on [tokens][hidden] new tokens; each layer's scores are updated in place."""
        for l in range(self.layers):
            h = (x @ self.qkv[l]).view(-1, (GROUP + 2) * HEADS, DIM)
            q, k, v = h.split((GROUP * HEADS, HEADS, HEADS), 1)
            q = mma.mma_kv_append(self.layout, self.cache[l], seqs, q, k, v, positions, self.rope, q_weight=self.norm,
                                  k_weight=self.norm, k_scale=self.scale, v_scale=self.scale)
            s = {} if scores is None else {"scores_in": scores[l], "scores_out": scores[l], "decay": 0.98}
            o = mma.mma_kv_attention(self.layout, self.cache[l], seqs, q, tree=tree, k_scale=self.scale,
                                     v_scale=self.scale, **s)
            x = x + o.flatten(1) @ self.out[l]
        return x


def table_of(blocks, width):
    return torch.tensor([blocks + [-1] * (width - len(blocks))], dtype=torch.int32, device="cuda")


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--layers", type=int, default=4)
    p.add_argument("--prompt", type=int, default=3000)
    p.add_argument("--keep", type=int, default=512)
    p.add_argument("--chunk", type=int, default=1024)
    p.add_argument("--steps", type=int, default=8)
    p.add_argument("--layout", choices=list(LAYOUTS), default="hnd")
    p.add_argument("--cache", choices=["bf16", "f8"], default="bf16")
    a = p.parse_args(argv)
    if not SINKS + RECENT <= a.keep <= a.prompt or min(a.layers, a.chunk, a.steps) < 1:
        p.error(f"{SINKS + RECENT} <= keep <= prompt, and at least one layer, token of a chunk and step are wanted")
    torch.cuda.set_device(0)
    mma.mma_init(0)
    try:
        with torch.no_grad():
            result = run(a)
        torch.cuda.synchronize()
    finally:
        mma.mma_finalize()
    return result


def run(a):
    m = Model(a)
    g = torch.Generator(device="cuda").manual_seed(1)
    tokens = lambda n: torch.randn((n, m.hidden), generator=g, device="cuda").bfloat16()  # noqa: E731

    # The prompt, in chunks; the weight of every entry is added up.
    blocks = m.take(a.prompt)
    table = table_of(blocks, len(blocks))
    scores = [torch.zeros((1, HEADS, a.prompt), device="cuda") for _ in range(a.layers)]
    for at in range(0, a.prompt, a.chunk):
        n = min(a.chunk, a.prompt - at)
        seqs = mma.kv_seqs(table, i32(at), i32(0, n), max_tokens=n, max_len=at + n)
        m.step(tokens(n), seqs, torch.arange(at, at + n, dtype=torch.int32, device="cuda"), scores=scores)

    # Cut to the entries that attention went to, into blocks of their own; the old ones are free.
    kept = m.take(a.keep)
    seqs = mma.kv_seqs(table, i32(a.prompt), max_tokens=0, max_len=a.prompt)
    share = []
    for l in range(a.layers):
        _, s, lens = mma.mma_kv_evict(m.layout, m.cache[l], seqs, table_of(kept, len(kept)), scores[l], a.keep,
                                      sinks=SINKS, recent=RECENT)
        share.append((s.sum() / scores[l].sum()).item())
        scores[l] = s
    m.free += blocks
    length = int(lens)
    print(f"evicted {a.prompt} -> {length} entries: {100 * np.mean(share):.1f}% of the weight kept "
          f"({100 * length / a.prompt:.1f}% of the entries)", flush=True)

    # Away over the link, and back into other blocks when the sequence goes on.
    slots = np.arange(len(kept), dtype=np.int32)
    mma.mma_kv_offload(m.layout, m.pool, m.cache, np.array(kept, np.int32), slots)
    m.free += kept
    draft = len(DRAFT)
    width = -(-(length + 4 * a.steps + draft) // TOKENS)
    blocks = m.take(width * TOKENS)
    mma.mma_kv_fetch(m.layout, m.pool, m.cache, slots, np.array(blocks[:len(kept)], np.int32))
    print(f"offloaded and fetched {len(kept)} blocks of {a.layers} layers: "
          f"{2 * len(kept) * mma.mma_kv_layout_sizes(m.layout)['slot'] / 2**20:.0f} MiB over the link", flush=True)

    # Trees of drafted tokens: 8 of them, each a child of an earlier one; a branch is accepted.
    table = table_of(blocks, width)
    room = [torch.zeros((1, HEADS, width * TOKENS), device="cuda") for _ in range(a.layers)]
    for r, s in zip(room, scores):
        r[:, :, :length] = s
    bits = []
    for i, up in enumerate(DRAFT):
        bits.append((bits[up] if up >= 0 else 0) | 1 << i)
    tree = torch.tensor(bits, dtype=torch.int64, device="cuda").view(-1, 1)
    depth = torch.tensor([bin(b).count("1") - 1 for b in bits], dtype=torch.int32, device="cuda")
    accepted, count = i32(0, 1, 3, 6).view(1, -1), i32(4)
    lens, position = i32(length), a.prompt
    for step in range(a.steps):
        seqs = mma.kv_seqs(table, lens, i32(0, draft), max_tokens=draft, max_len=length + 4 * step + draft)
        x = m.step(tokens(draft), seqs, depth + position, tree, room)
        lens = mma.mma_kv_commit(m.layout, m.cache, seqs, accepted, count, scores=room)
        position += 4
    print(f"{a.steps} steps of {draft} drafted tokens, 4 accepted each: {int(lens)} entries, position {position}, "
          f"last hidden states' rms {x.float().square().mean().sqrt().item():.3f}", flush=True)
    torch.cuda.synchronize()
    m.pool.free()
    return {"length": int(lens), "share": share, "x": x}


if __name__ == "__main__":
    main()
