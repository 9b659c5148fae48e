"""Beam search on the paged cache, from prompts to a compacted pool that leaves for the host in one piece.

    python examples/kv_beam.py [--layers 4] [--requests 2] [--beams 4] [--prompt 300] [--steps 32] [--layout hnd] [--cache f8]

An untrained model (random projections) whose scores are capped and whose tokens see the last 256 entries and the first
four, those in both directions: a prompt's first three tokens see ahead up to the fourth. Each request's prompt is
written once and its beams fork from it: they share its pages, and every step a beam that goes on from another shares
that one's pages and gets its own copy of the open one, on the GPU throughout. At the end the held pages are moved to
the front of the pool and offloaded over all paths. Prints what each part did.
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
HEADS, GROUP, DIM, TOKENS, VOCAB = 4, 2, 64, 16, 5000
CAP, WINDOW, FIRST = 30.0, 256, 4  # the model's scores: the cap, the window, the first entries, which every token sees
END = VOCAB - 1  # a beam that takes this token has ended


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Model:
    """Projections of a few attention layers, and the pool of pages."""

    def __init__(self, a):
        g = torch.Generator(device="cuda").manual_seed(0)
        self.layers, self.f8 = a.layers, a.cache == "f8"
        hidden = HEADS * GROUP * DIM
        rand = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16) * s[0] ** -0.5  # noqa: E731
        self.embed = torch.randn((VOCAB, hidden), generator=g, device="cuda", dtype=torch.bfloat16)
        self.qkv = [rand(hidden, (GROUP + 2) * HEADS * DIM) for _ in range(a.layers)]
        self.out = [rand(hidden, hidden) for _ in range(a.layers)]
        self.unembed = rand(hidden, VOCAB) * 3
        self.scale = torch.full((HEADS,), 0.05, device="cuda") if self.f8 else None
        self.width = -(-(a.prompt + a.steps) // TOKENS)
        self.rows = a.requests * a.beams
        # A request's pages, and for each beam the pages of its own steps and a copy of the open one.
        self.blocks = a.requests * self.width + self.rows * (-(-a.steps // TOKENS) + 2)
        self.layout = mma.kv_layout(a.layers, TOKENS, HEADS, DIM, 1 if self.f8 else 2, self.blocks, self.blocks, LAYOUTS[a.layout])
        size = mma.mma_kv_layout_sizes(self.layout)
        self.cache = [torch.zeros(size["layer"], dtype=torch.uint8, device="cuda") for _ in range(a.layers)]
        self.table = mma.layer_table(self.cache)
        rope = mma.mma_rope_table(self.width * TOKENS, DIM, 10000.0)
        self.rope = torch.from_numpy(rope).cuda()

    def step(self, tokens, table, lens, counts):
        """Logits of each sequence's last one of `counts` tokens each, written behind its entries."""
        n = len(counts)
        start = np.cumsum([0] + counts)
        seqs = mma.kv_seqs(table, lens, i32(start), max_tokens=max(counts), max_len=self.width * TOKENS)
        positions = torch.cat([lens[s] + torch.arange(t, dtype=torch.int32, device="cuda") for s, t in enumerate(counts)])
        first = torch.full((n,), FIRST, dtype=torch.int32, device="cuda")
        x = self.embed[tokens]
        for l in range(self.layers):
            h = (x @ self.qkv[l]).view(-1, (GROUP + 2) * HEADS, DIM)
            q, k, v = h.split((GROUP * HEADS, HEADS, HEADS), 1)
            q = mma.mma_kv_append(self.layout, self.cache[l], seqs, q, k, v, positions, self.rope, k_scale=self.scale,
                                  v_scale=self.scale)
            o = mma.mma_kv_attention(self.layout, self.cache[l], seqs, q, k_scale=self.scale, v_scale=self.scale, softcap=CAP,
                                     window=WINDOW, prefix=first, max_prefix=FIRST)
            x = x + o.flatten(1) @ self.out[l]
        return x[torch.from_numpy(start[1:] - 1).cuda()] @ self.unembed


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--layers", type=int, default=4)
    p.add_argument("--requests", type=int, default=2)
    p.add_argument("--beams", type=int, default=4)
    p.add_argument("--prompt", type=int, default=300)
    p.add_argument("--steps", type=int, default=32)
    p.add_argument("--layout", choices=list(LAYOUTS), default="hnd")
    p.add_argument("--cache", choices=["bf16", "f8"], default="bf16")
    a = p.parse_args(argv)
    if min(a.layers, a.requests, a.beams, a.prompt, a.steps) < 1 or a.beams > 64:
        p.error("at least one layer, request, beam, token of a prompt and step are wanted, and at most 64 beams")
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
    refs = torch.zeros(m.blocks, dtype=torch.int32, device="cuda")

    # A sequence for each request, out of nothing, with pages for its prompt.
    none = mma.kv_seqs(torch.full((1, m.width), -1, dtype=torch.int32, device="cuda"), i32([0]), max_tokens=0, max_len=m.width * TOKENS)
    table, lens, refs, _ = mma.mma_kv_fork(m.layout, m.table, none, i32([-1] * a.requests), refs, grow=i32([a.prompt] * a.requests))
    prompts = torch.randint(0, VOCAB - 1, (a.requests * a.prompt,), generator=g, device="cuda")
    logits = m.step(prompts, table, lens, [a.prompt] * a.requests)
    lens = lens + a.prompt

    # Beams: at first one of each request lives, and the best tokens after its prompt make the others.
    scores = torch.full((a.requests, a.beams), -float("inf"), device="cuda")
    scores[:, 0] = 0
    done = torch.zeros((a.requests, a.beams), dtype=torch.bool, device="cuda")
    logits = logits.repeat_interleave(a.beams, 0)
    history = torch.empty((m.rows, 0), dtype=torch.int64, device="cuda")
    for step in range(a.steps):
        tokens, parents, scores = mma.mma_beam_select(logits, scores, a.beams, done=done, done_token=END)
        rows = parents.flatten().clamp_min(0)  # a request with fewer candidates than beams: dead ones go on from anywhere
        done = (done.flatten()[rows.long()].view_as(done) | (tokens == END))
        new = tokens.flatten().clamp_min(0).long()
        history = torch.cat([history[rows.long()] if step else history, new[:, None]], 1)
        seqs = mma.kv_seqs(table, lens, max_tokens=0, max_len=m.width * TOKENS)
        source = rows if step else torch.div(rows, a.beams, rounding_mode="floor").int()
        table, lens, refs, free = mma.mma_kv_fork(m.layout, m.table, seqs, source, refs, grow=i32([1] * m.rows), out=None)
        if step + 1 == a.steps:
            break
        logits = m.step(new, table, lens, [1] * m.rows)
        lens = lens + 1
    held = int((refs != 0).sum())
    print(f"{a.requests} prompts of {a.prompt} tokens, {a.steps} steps of {a.beams} beams: {held} of {m.blocks} pages held "
          f"({m.rows * -(-int(lens[0]) // TOKENS)} without sharing), {int(done.sum())} beams have ended", flush=True)

    # The held pages to the front, and away to the host: one run of blocks.
    table, refs, moved, held = mma.mma_kv_compact(m.layout, m.table, table, refs)
    n = int(held)
    size = mma.mma_kv_layout_sizes(m.layout)
    with mma.PinnedBuffer(size["pool"]) as pool:
        mma.mma_kv_offload(m.layout, pool, m.table, np.arange(n, dtype=np.int32), np.arange(n, dtype=np.int32))
        torch.cuda.synchronize()
    print(f"{int((moved[n:] >= 0).sum())} pages moved to the front, {n} offloaded: {n * size['slot'] / 2**20:.1f} MiB over the link",
          flush=True)
    best = scores.argmax(1) + torch.arange(a.requests, device="cuda") * a.beams
    for y, row in enumerate(best.tolist()):
        print(f"request {y}: {scores.flatten()[row].item():.3f} {history[row, :8].tolist()} ...", flush=True)
    return {"held": n, "history": history, "scores": scores, "refs": refs, "table": table}


if __name__ == "__main__":
    main()
