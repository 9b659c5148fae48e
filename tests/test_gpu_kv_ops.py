"""The operators on the paged KV cache against the 64-bit reference (oracle.kv_ops).

Tolerances, from the types and the arithmetic before any run:
  - a value rounded once to a type with b mantissa bits is within 2^-(b+1) of itself (relative), and within
    half its smallest step where it is subnormal;
  - sums in 32 bits: a logit is a sum of head_dim exact products, whose error stays below
    head_dim * 2^-24 of the sum of their magnitudes (B); p carries twice that (its own logit and the row's sum), plus
    the exponential's and the sum's own few 2^-23;
  - attention rounds p to 16 bits for the product with V: 2^-(b+1) of sum p |V| at most.
Bytes that are moved, entries that are kept and everything that no operator writes are compared exactly.
"""
import math

import numpy as np
import pytest
import torch

from oracle import kv_ops as ok

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2512_16056_amd as mma  # noqa: E402
from gpu_helpers import log, session  # noqa: E402

LAYOUTS = {"piece": mma.MMA_KV_LAYOUT_PIECE, "hnd": mma.MMA_KV_LAYOUT_HND, "xpacked": mma.MMA_KV_LAYOUT_XPACKED}
BF16, F16, F8 = torch.bfloat16, torch.float16, ok.F8
BITS = {BF16: 7, F16: 10, F8: 3}
STEP = {BF16: 2.0 ** -133, F16: 2.0 ** -24, F8: 2.0 ** -9}
EPS = 2.0 ** -23


@pytest.fixture(scope="module", autouse=True)
def library():
    with session():
        yield


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(g, *shape, std=1.0):
    return torch.randn(shape, generator=g) * std


def to_cache(x, dtype):
    """Elements as the flat cache holds them: 8-bit ones as uint8."""
    return x.clamp(-448, 448).to(F8).view(torch.uint8) if dtype is F8 else x.to(dtype)


class Case:
    """A cache layer with random contents, tables in random block order, and the sequences of a call."""

    def __init__(self, layout, cache, lens, counts, dim=128, heads=2, group=4, tokens=16, dtype=BF16, seed=0, layers=1,
                 room=0, q_start=True):
        self.g = gen(seed)
        self.dtype, self.group, self.counts, self.lens, self.layers = dtype, group, counts, lens, layers
        need = [max(1, -(-(n + t + room) // tokens)) for n, t in zip(lens, counts)]
        blocks = sum(need) + 3
        self.c = ok.Cache(layout, cache, blocks, tokens, heads, dim)
        order = torch.randperm(blocks, generator=self.g).int()
        self.table = torch.full((len(lens), max(need)), -1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at: at + n]
            at += n
        self.spare = order[at:]
        self.flat = to_cache(normal(self.g, layers * 2 * blocks * self.c.piece), cache).view(layers, -1)
        self.q_start = torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32) if q_start else None
        self.total = sum(counts)
        self.max_tokens = max(counts + [1])
        self.max_len = max([n + t for n, t in zip(lens, counts)] + [1])
        self.heads_q = heads * group
        self.k_scale = self.v_scale = None
        if cache is F8:
            self.k_scale = torch.rand(heads, generator=self.g) + 0.5
            self.v_scale = torch.rand(heads, generator=self.g) + 0.5

    def layout(self):
        return mma.kv_layout(self.layers, self.c.tokens, self.c.heads, self.c.dim, self.c.elem, self.c.blocks, 1,
                             LAYOUTS[self.c.layout])

    def seqs(self, **kw):
        kw = {"max_tokens": self.max_tokens, "max_len": self.max_len, **kw}
        return mma.kv_seqs(self.table.cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda(),
                           None if self.q_start is None else self.q_start.cuda(), **kw)

    def spans(self, **kw):
        kw = {"num_tokens": self.total, "max_tokens": self.max_tokens, "max_len": self.max_len, **kw}
        return ok.spans(self.c, self.table, self.lens, self.q_start, **kw)

    def scales(self):
        return {"k_scale": None if self.k_scale is None else self.k_scale.cuda(),
                "v_scale": None if self.v_scale is None else self.v_scale.cuda()}


def same_bits(a, b):
    a, b = (x.contiguous().view(torch.uint8) for x in (a, b))
    return torch.equal(a, b)


def rounded_close(got, want, dtype, slack):
    """|got - want| within one rounding of `dtype` and `slack` (absolute, of the arithmetic before it)."""
    got, want = got.double(), want.double()
    if dtype is F8:
        want = want.clamp(-448, 448)
    tol = want.abs() * 2.0 ** -(BITS[dtype] + 1) * (1 + 2.0 ** -6) + STEP[dtype] / 2 + slack
    worst = ((got - want).abs() / tol).max().item() if got.numel() else 0.0
    assert worst <= 1, f"{worst:.3g} of the tolerance"


# ------------------------------------------------------------------ append
def check_append(c, rot, interleaved, norm, q_view=None, positions=None, in_place=False):
    n, D = c.total, c.c.dim
    q = normal(c.g, n, c.heads_q, D, std=1.5).to(c.dtype)
    k = normal(c.g, n, c.c.heads, D, std=1.5).to(c.dtype)
    v = normal(c.g, n, c.c.heads, D, std=1.5).to(c.dtype)
    qw, kw = ((1 + normal(c.g, D, std=0.2)).to(c.dtype) for _ in range(2)) if norm else (None, None)
    table = torch.from_numpy(mma.mma_rope_table(c.max_len + 1, rot, 10000.0)) if rot else None
    if positions is None:
        positions = torch.tensor([m + i for m, t in zip(c.lens, c.counts) for i in range(t)], dtype=torch.int32)
    wq, wk, wv = ok.append(q, k, v, positions, table, interleaved, qw, kw, 1e-6)
    dev = [x if x is None else x.cuda() for x in (q, k, v, positions, table, qw, kw)]
    if q_view is not None:
        dev[:3] = [q_view(x) for x in dev[:3]]
    layer = c.flat[0].cuda()
    out = mma.mma_kv_append(c.layout(), layer, c.seqs(), *dev[:3], dev[3] if rot else None, dev[4],
                            q_out=dev[0] if in_place else None, interleaved=interleaved, q_weight=dev[5], k_weight=dev[6],
                            **c.scales())
    torch.cuda.synchronize()
    # norm: a sum of D squares, a root, a division and two products; rotation: two products and a sum
    slack = lambda x: (D + 16) * EPS * x.abs().amax(-1, keepdim=True)  # noqa: E731
    rounded_close(out.cpu(), wq, c.dtype, slack(wq))
    got, rest = layer.cpu(), c.flat[0].clone()
    for s, (a, t, m, total) in enumerate(c.spans()):
        for i in range(total - m):
            at = c.c.entry(c.table[s], m + i)
            if at is None:
                continue
            for h in range(c.c.heads):
                for which, want, scale in ((0, wk[a + i, h], c.k_scale), (1, wv[a + i, h], c.v_scale)):
                    want = want / float(scale[h]) if scale is not None else want
                    index = c.c.index(which, *at, h)
                    rounded_close(c.c.values(got, index), want, c.c.dtype, slack(want))
                    rest[index] = got[index]
    assert same_bits(got, rest), "something else in the cache changed"
    return out


APPEND = [
    # layout, cache, dim, rot, interleaved, norm, tokens, heads, group
    ("piece", BF16, 128, 128, False, True, 16, 2, 4),
    ("hnd", F16, 128, 128, False, False, 16, 2, 4),
    ("xpacked", F8, 128, 32, True, True, 16, 2, 4),
    ("xpacked", BF16, 64, 64, True, True, 8, 3, 1),
    ("piece", F8, 80, 24, False, True, 5, 1, 7),
    ("hnd", BF16, 96, 50, False, False, 1, 2, 3),
    ("xpacked", F16, 256, 250, False, True, 32, 1, 2),
    ("piece", BF16, 8, 2, True, True, 3, 5, 1),
    ("hnd", F8, 256, 0, False, False, 24, 1, 1),
    ("piece", F16, 72, 10, False, True, 7, 2, 2),
]


@pytest.mark.parametrize("layout,cache,dim,rot,interleaved,norm,tokens,heads,group", APPEND)
def test_append(layout, cache, dim, rot, interleaved, norm, tokens, heads, group):
    log(f"append {layout} {cache} dim {dim} rot {rot}")
    dtype = F16 if cache is F16 else BF16
    check_append(Case(layout, cache, [0, 37, 5, 64], [1, 9, 0, 23], dim, heads, group, tokens, dtype), rot, interleaved, norm)


def test_append_single_token_and_many_sequences():
    check_append(Case("piece", BF16, [999], [1]), 128, False, True)
    n = 70  # more sequences than a wave has lanes
    check_append(Case("hnd", BF16, [i % 11 for i in range(n)], [i % 3 for i in range(n)], dim=64, heads=1, group=1), 64, False, True)


def test_append_strides_alignment_and_in_place():
    def odd(x):  # rows that start at any 2 bytes, heads outermost
        n, h, d = x.shape
        buf = torch.zeros(h, n, d + 3, dtype=x.dtype, device="cuda")
        view = buf[:, :, 1: 1 + d].permute(1, 0, 2)
        view.copy_(x)
        return view
    check_append(Case("piece", BF16, [3, 20], [7, 4], dim=72, tokens=8), 36, False, True, q_view=odd)
    c = Case("hnd", F16, [3, 20], [7, 4], dtype=F16)
    check_append(c, 128, True, True, in_place=True)


def test_append_positions_out_of_range_and_missing_blocks():
    c = Case("xpacked", BF16, [3, 20], [7, 14])
    c.table[1, 1] = -1          # entries 16 .. 31 of sequence 1
    c.table[0, 0] = c.c.blocks  # and all of sequence 0's have no block
    pos = torch.randint(-5, 60, (c.total,), generator=c.g).int()
    check_append(c, 128, False, True, positions=pos)


def test_append_without_q_start_and_zero_norm():
    c = Case("piece", BF16, [5, 0, 17], [2, 2, 2], q_start=False)
    check_append(c, 64, False, True)
    # a row of zeros is zero after the norm, not NaN
    c = Case("piece", BF16, [5], [1])
    q = torch.zeros(1, 8, 128, dtype=BF16, device="cuda")
    w = torch.ones(128, dtype=BF16, device="cuda")
    out = mma.mma_kv_append(c.layout(), c.flat[0].cuda(), c.seqs(), q, q[:, :2], q[:, :2], q_weight=w, k_weight=w)
    assert torch.equal(out, torch.zeros_like(out))


def test_append_f8_saturates_and_keeps_nan():
    c = Case("hnd", F8, [0], [1])
    c.k_scale = c.v_scale = torch.full((2,), 0.5)
    x = torch.zeros(1, 2, 128, dtype=BF16)
    x[0, 0, :4] = torch.tensor([1e6, -1e6, math.inf, math.nan])
    layer = c.flat[0].cuda()
    mma.mma_kv_append(c.layout(), layer, c.seqs(), torch.zeros(1, 8, 128, dtype=BF16, device="cuda"), x.cuda(), x.cuda(), **c.scales())
    for which in (0, 1):
        got = c.c.values(layer.cpu(), c.c.index(which, int(c.table[0, 0]), 0, 0))[:4]
        assert got[:3].tolist() == [448, -448, 448] and math.isnan(got[3])


# ------------------------------------------------------------------ attention
def tree_bits(counts, g, width=None, empty=False):
    words = width or max(1, (max(counts) + 63) // 64)
    rows = []
    for t in counts:
        bits = []
        for i in range(t):
            up = bits[int(torch.randint(max(0, i - 6), i, (1,), generator=g))] if i else 0
            bits.append(up | 1 << i)
        if empty and t:
            bits[0] = 0
        rows += [[(b >> 64 * w) & (2 ** 64 - 1) for w in range(words)] for b in bits]
    return torch.from_numpy(np.array(rows, dtype=np.uint64).reshape(-1, words).view(np.int64))


def check_attention(c, tree=None, scores=False, q=None, q_view=None, in_place=False, std=2.0, stream=None, scale=None,
                    seqs=None, spans=None):
    D = c.c.dim
    if q is None:
        q = normal(c.g, c.total, c.heads_q, D, std=std).to(c.dtype)
    scale = D ** -0.5 if scale is None else scale
    span = spans or c.spans()
    s_in = torch.rand(len(c.lens), c.c.heads, c.max_len + 5, generator=c.g) if scores else None
    want = ok.attention(c.c, c.flat[0], c.table, span, q, c.group, scale, tree, c.k_scale, c.v_scale, s_in, 0.5)
    dev = q.cuda() if q_view is None else q_view(q.cuda())
    lse = torch.full((c.total, c.heads_q), 7.0, device="cuda")
    more = {}
    if scores:
        s_out = torch.full_like(s_in, -3.0).cuda()
        more = {"scores_in": s_in.cuda(), "scores_out": s_out, "decay": 0.5}
    layer = c.flat[0].cuda()
    out = mma.mma_kv_attention(c.layout(), layer, seqs or c.seqs(), dev, out=dev if in_place else None, scale=scale,
                               tree=None if tree is None else tree.cuda(), lse=lse, **c.scales(), **more)
    torch.cuda.synchronize()
    assert same_bits(layer.cpu(), c.flat[0])
    covered = torch.zeros(c.total, dtype=torch.bool)
    for a, t, _, _ in span:
        covered[a: a + t] = True
    out, lse = out.cpu()[covered].double(), lse.cpu()[covered].double()
    w = {x: want[x][covered] for x in ("out", "lse", "mag", "big")}
    finite = torch.isfinite(w["out"]) & torch.isfinite(w["mag"])
    assert torch.equal(torch.isnan(w["out"]), torch.isnan(out))
    assert torch.equal(w["out"][~finite & ~torch.isnan(out)], out[~finite & ~torch.isnan(out)])
    u = 2.0 ** -(BITS[c.dtype] + 1)
    p_err = (2 * D * EPS * w["big"] + 64 * EPS)[..., None]
    tol = u * w["out"].abs() * (1 + 2 * u) + (u + p_err) * w["mag"] * (1 + 2 * u) + STEP[c.dtype]
    worst = ((out - w["out"]).abs() / tol)[finite].max().item() if finite.any() else 0.0
    assert worst <= 1, f"out: {worst:.3g} of the tolerance"
    empty = w["lse"] == -math.inf
    assert torch.equal(lse == -math.inf, empty) and not out[empty].any()
    ok_lse = ~empty & torch.isfinite(w["lse"])
    err = (lse - w["lse"]).abs() / (2 * D * EPS * w["big"] + 64 * EPS * (1 + w["lse"].abs()))
    assert not ok_lse.any() or err[ok_lse].max().item() <= 1
    if scores:
        got = more["scores_out"].cpu().double()
        written = torch.zeros(got.shape, dtype=torch.bool)
        for s, (_, _, _, m) in enumerate(span):
            written[s, :, :m] = True
        assert (got[~written] == -3).all(), "scores past the entries changed"
        exact = torch.zeros_like(got)
        exact[:, :, : want["scores"].shape[2]] = want["scores"]
        rel = 2 * D * EPS * want["big"].max() + 64 * EPS
        err = ((got - exact).abs() / (rel * (1 + exact.abs())))[written]
        assert not err.numel() or err.max().item() <= 1, f"scores: {err.max().item():.3g} of the tolerance"
    return out


ATTENTION = [
    # layout, cache, dim, tokens, heads, group, lens, counts
    ("piece", BF16, 128, 16, 2, 4, [101], [1]),
    ("hnd", F16, 128, 16, 2, 4, [0, 1, 31, 32, 33, 700], [1, 1, 1, 1, 1, 1]),
    ("xpacked", F8, 128, 16, 2, 4, [63, 0, 250], [24, 3, 70]),
    ("xpacked", BF16, 64, 8, 1, 8, [5, 129], [2, 33]),
    ("piece", F8, 80, 24, 1, 7, [77, 20], [9, 1]),
    ("hnd", BF16, 96, 1, 2, 1, [40, 3], [5, 2]),
    ("xpacked", F16, 256, 32, 1, 2, [300, 17], [3, 40]),
    ("piece", F16, 256, 7, 1, 3, [90], [20]),
    ("piece", BF16, 8, 3, 3, 2, [50, 0], [4, 1]),
    ("hnd", F8, 64, 16, 2, 16, [500], [5]),
    ("xpacked", F8, 256, 16, 1, 1, [70], [66]),
    ("hnd", BF16, 72, 24, 1, 5, [200, 64, 65], [1, 13, 0]),
]


@pytest.mark.parametrize("kind", ["chain", "tree", "scores"])
@pytest.mark.parametrize("layout,cache,dim,tokens,heads,group,lens,counts", ATTENTION)
def test_attention(layout, cache, dim, tokens, heads, group, lens, counts, kind):
    log(f"attention {kind} {layout} {cache} dim {dim} {lens} {counts}")
    c = Case(layout, cache, lens, counts, dim, heads, group, tokens, F16 if cache is F16 else BF16)
    check_attention(c, tree_bits(counts, c.g) if kind != "chain" else None, kind == "scores")


@pytest.mark.parametrize("layout", list(LAYOUTS))
def test_attention_over_many_splits(layout):
    """Contexts long enough to be split and joined, next to short and empty ones."""
    c = Case(layout, BF16, [3000, 10, 0, 1025], [2, 1, 1, 3], heads=1, group=2, dim=64)
    check_attention(c, None, True)


@pytest.mark.parametrize("layout", list(LAYOUTS))
def test_attention_rows_that_see_nothing(layout):
    """No context and a tree row without bits: zeros, lse -infinity, and no part in the scores."""
    c = Case(layout, BF16, [0, 0, 40], [3, 1, 2], heads=1, group=4)
    check_attention(c, tree_bits(c.counts, c.g, empty=True), True)


@pytest.mark.parametrize("cache", [BF16, F16, F8])
@pytest.mark.parametrize("layout", list(LAYOUTS))
def test_attention_infinities_where_nobody_looks(layout, cache):
    """Stale blocks, entries past the end and drafted tokens that a row does not see hold NaN and infinities."""
    c = Case(layout, cache, [21, 40], [9, 5], heads=1, group=4, room=30, dtype=F16 if cache is F16 else BF16)
    bad = [math.nan] if cache is F8 else [math.nan, math.inf, -math.inf]
    vals = to_cache(torch.tensor(bad * 400)[:400], cache)
    if cache is F8:
        vals = torch.full((400,), 0x7F, dtype=torch.uint8)
    flat = c.flat[0]
    for s, (_, t, n, m) in enumerate(c.spans()):
        for j in range(m, c.table.shape[1] * c.c.tokens):
            at = c.c.entry(c.table[s], j)
            for which in (0, 1):
                if at is not None:
                    flat[c.c.index(which, *at, 0)] = vals[: c.c.dim]
    for b in c.spare.tolist():
        for tok in range(c.c.tokens):
            flat[c.c.index(0, b, tok, 0)] = flat[c.c.index(1, b, tok, 0)] = vals[: c.c.dim]
    tree = tree_bits(c.counts, c.g)
    out = check_attention(c, tree, True)
    assert torch.isfinite(out).all()
    # drafted token 2 of sequence 0: seen by itself and its children alone
    at = c.c.entry(c.table[0], 21 + 2)
    for which in (0, 1):
        flat[c.c.index(which, *at, 0)] = vals[: c.c.dim]
    tree[:9, 0] &= ~(1 << 2)
    out = check_attention(c, tree, False)
    assert torch.isfinite(out).all()
    keep = flat[c.c.index(0, *at, 0)].clone()
    flat[c.c.index(0, *at, 0)] = to_cache(torch.ones(c.c.dim), cache)
    tree[4, 0] |= 1 << 2  # row 4 sees an infinite V: infinite or NaN itself, the others are not
    out = check_attention(c, tree, False)
    assert not torch.isfinite(out[4]).all() and torch.isfinite(out[:4]).all() and torch.isfinite(out[5:]).all()
    flat[c.c.index(0, *at, 0)] = keep


def test_attention_missing_blocks():
    for layout in LAYOUTS:
        c = Case(layout, BF16, [70, 33], [5, 2], heads=1)
        c.table[0, 1] = -1
        c.table[0, 4] = c.c.blocks + 7
        c.table[1, :] = -1  # nothing there at all
        check_attention(c, tree_bits(c.counts, c.g), True)


def test_attention_large_and_equal_logits():
    c = Case("hnd", BF16, [300], [4], heads=1)
    check_attention(c, std=60.0)
    c = Case("hnd", BF16, [300], [4], heads=1)
    check_attention(c, q=torch.zeros(4, 4, 128, dtype=BF16), scores=True)  # all weights equal
    c = Case("hnd", F16, [300], [4], heads=1, dtype=F16)
    check_attention(c, scale=-0.3)


def test_attention_strides_alignment_and_in_place():
    def odd(x):
        n, h, d = x.shape
        buf = torch.zeros(h, n, d + 3, dtype=x.dtype, device="cuda")
        view = buf[:, :, 1: 1 + d].permute(1, 0, 2)
        view.copy_(x)
        return view
    for in_place in (False, True):
        c = Case("piece", BF16, [30, 100], [7, 40], dim=72, tokens=8)
        check_attention(c, tree_bits(c.counts, c.g), q_view=odd, in_place=in_place)
        c = Case("hnd", BF16, [30, 2000], [7, 3], heads=1)
        check_attention(c, in_place=in_place)


def test_attention_bounds_of_the_call():
    """Lengths, starts and bounds that do not fit: what is past them is left out, and nothing else is touched."""
    c = Case("piece", BF16, [-5, 40, 1000], [3, 4, 2], heads=1)
    c.lens[2] = 20
    c = Case("piece", BF16, [0, 40, 20], [3, 4, 2], heads=1)
    c.lens[0] = -5
    check_attention(c)
    c = Case("piece", BF16, [10, 40, 20], [3, 4, 2], heads=1)
    c.q_start = torch.tensor([2, 5, 4, 9999], dtype=torch.int32)
    check_attention(c)
    c = Case("piece", BF16, [10, 40, 20], [3, 4, 2], heads=1)
    c.max_tokens, c.max_len = 2, 30
    check_attention(c)
    c = Case("piece", BF16, [10, 40, 20], [3, 3, 3], heads=1, q_start=False)
    check_attention(c, scores=True)


def test_attention_trees_wider_than_a_word_and_short_ones():
    c = Case("hnd", BF16, [100, 3], [130, 70], heads=1, group=2, dim=64)
    check_attention(c, tree_bits(c.counts, c.g), True)
    c = Case("hnd", BF16, [100, 3], [130, 70], heads=1, group=2, dim=64)
    check_attention(c, tree_bits(c.counts, c.g)[:, :1].contiguous())  # drafted tokens past the words are not seen


def test_attention_on_another_stream_and_captured():
    c = Case("hnd", BF16, [3000, 70], [2, 3], heads=2)
    q = normal(c.g, c.total, c.heads_q, 128).to(BF16).cuda()
    layer, seqs, lay = c.flat[0].cuda(), c.seqs(), c.layout()
    want = mma.mma_kv_attention(lay, layer, seqs, q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = mma.mma_kv_attention(lay, layer, seqs, q, stream=side)
    side.synchronize()
    assert same_bits(got, want)
    out = torch.empty_like(q)
    ws = torch.empty(mma.kv_attention_workspace(lay, seqs, q.shape[0], q.shape[1], q.dtype), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mma.mma_kv_attention(lay, layer, seqs, q, out=out, workspace=ws)
    for _ in range(3):
        out.zero_()
        ws.random_()
        graph.replay()
        torch.cuda.synchronize()
        assert same_bits(out, want)


# ------------------------------------------------------------------ commit
@pytest.mark.parametrize("layout,cache,dim,tokens", [("piece", BF16, 128, 16), ("hnd", F8, 80, 5), ("xpacked", F16, 64, 8),
                                                     ("xpacked", F8, 128, 16), ("piece", F8, 16, 1)])
def test_commit(layout, cache, dim, tokens):
    log(f"commit {layout} {cache}")
    c = Case(layout, cache, [7, 0, 30, 12, 3], [12, 9, 20, 6, 8], dim, 2, 2, tokens, layers=3)
    acc = torch.full((5, 10), -1, dtype=torch.int32)
    lists = [[0, 2, 3, 7, 8, 9, 11], [0, 1, 2], [], [1, 3, 3, 4], [0, 5, 99, 6]]  # the last two stop short
    for s, a in enumerate(lists):
        acc[s, : len(a)] = torch.tensor(a, dtype=torch.int32)
    counts = torch.tensor([7, 3, -2, 4, 4], dtype=torch.int32)
    moves, lens = ok.commit_moves(acc, counts, c.spans())
    assert [len(m) for m in moves] == [7, 3, 0, 2, 2]
    layers = [x.clone().cuda() for x in c.flat]
    scores = [torch.rand(5, 2, c.max_len + 3, generator=c.g) for _ in layers]
    dev = [x.cuda() for x in scores]
    new = mma.mma_kv_commit(c.layout(), layers, c.seqs(), acc.cuda(), counts.cuda(), scores=dev)
    assert new.tolist() == lens
    for l in range(3):
        want, sc = c.flat[l], scores[l].clone()
        for s in range(5):
            want = ok.move_entries(c.c, want, c.table[s], c.table[s], moves[s])
            for a, b in moves[s]:
                sc[s, :, b] = sc[s, :, a]
        assert same_bits(layers[l].cpu(), want) and torch.equal(dev[l].cpu(), sc)
    again = [x.clone().cuda() for x in c.flat]
    mma.mma_kv_commit(c.layout(), again, c.seqs(), acc.cuda(), counts.cuda())
    assert all(same_bits(a, b) for a, b in zip(again, layers))


def test_commit_more_layers_than_a_launch_and_missing_blocks():
    c = Case("hnd", BF16, [7, 20], [12, 9], 16, 1, 1, 4, layers=200)
    c.table[0, 3] = -1
    acc = torch.tensor([[1, 4, 6, 11], [0, 3, 5, 8]], dtype=torch.int32)
    counts = torch.tensor([4, 9], dtype=torch.int32)  # the second is cut to the width
    moves, lens = ok.commit_moves(acc, counts, c.spans())
    layers = [x.clone().cuda() for x in c.flat]
    assert mma.mma_kv_commit(c.layout(), layers, c.seqs(), acc.cuda(), counts.cuda()).tolist() == lens == [11, 24]
    for l in (0, 1, 191, 192, 199):
        want = c.flat[l]
        for s in range(2):
            want = ok.move_entries(c.c, want, c.table[s], c.table[s], moves[s])
        assert same_bits(layers[l].cpu(), want), l


# ------------------------------------------------------------------ evict
def check_evict(c, keep, sinks, recent, scores):
    S, H = len(c.lens), c.c.heads
    width = -(-keep // c.c.tokens)
    free = [b for b in range(c.c.blocks) if b not in set(c.table.flatten().tolist())]
    dst = torch.full((S, width), -1, dtype=torch.int32)
    for s, n in enumerate(c.lens):
        for b in range(-(-min(max(n, 0), keep) // c.c.tokens)):
            dst[s, b] = free.pop()
    layer = c.flat[0].cuda()
    got, kept, lens = mma.mma_kv_evict(c.layout(), layer, c.seqs(), dst.cuda(), scores.cuda(), keep, sinks=sinks, recent=recent)
    torch.cuda.synchronize()
    want, out = c.flat[0], torch.full((S, H, keep), -1, dtype=torch.int32)
    ws = torch.zeros(S, H, keep)
    for s, n in enumerate(c.lens):
        n = min(max(n, 0), c.max_len)
        for h in range(H):
            stay = ok.evict_select(scores[s, h], n, keep, sinks, recent)
            out[s, h, : len(stay)] = torch.tensor(stay, dtype=torch.int32)
            ws[s, h, : len(stay)] = scores[s, h, stay]
            want = ok.move_entries(c.c, want, c.table[s], dst[s], [(j, i) for i, j in enumerate(stay)], [h])
    assert lens.tolist() == [min(max(n, 0), keep, c.max_len) for n in c.lens]
    assert torch.equal(got.cpu(), out)
    assert same_bits(kept.cpu(), ws)
    assert same_bits(layer.cpu(), want)


def evict_case(layout, cache, lens, keep, dim=64, heads=2, tokens=16, seed=0):
    c = Case(layout, cache, lens, [0] * len(lens), dim, heads, 1, tokens, seed=seed)
    extra = sum(-(-min(max(n, 0), keep) // tokens) for n in lens)  # blocks for what stays
    c.c = ok.Cache(layout, cache, c.c.blocks + extra, tokens, heads, dim)
    c.flat = to_cache(normal(c.g, 2 * c.c.blocks * c.c.piece), cache).view(1, -1)
    c.max_len = max(lens + [1])
    return c


@pytest.mark.parametrize("layout,cache,tokens", [("piece", BF16, 16), ("hnd", F8, 5), ("xpacked", F16, 8), ("xpacked", F8, 16)])
@pytest.mark.parametrize("keep,sinks,recent", [(40, 4, 10), (33, 0, 0), (20, 4, 16), (1, 0, 1), (1, 0, 0)])
def test_evict(layout, cache, tokens, keep, sinks, recent):
    log(f"evict {layout} {cache} keep {keep}")
    c = evict_case(layout, cache, [100, 0, 1, keep, keep + 1, 77], keep, tokens=tokens)
    check_evict(c, keep, sinks, recent, torch.rand(6, 2, c.max_len + 3, generator=c.g))


@pytest.mark.parametrize("n,keep", [(5000, 1200), (1025, 1024), (3000, 1)])
def test_evict_long(n, keep):
    c = evict_case("hnd", F8, [n, n // 2 + 1], keep, dim=16, heads=2)
    check_evict(c, keep, 0, min(3, keep), torch.exp(3 * normal(c.g, 2, 2, n)))


def test_evict_ties_and_special_scores():
    """Equal scores go to the lower entry, zeros of both signs are equal, NaN is below -infinity."""
    c = evict_case("piece", BF16, [300, 200], 90)
    s = torch.randint(0, 4, (2, 2, 300), generator=c.g).float()
    s[0, 1] = 0
    s[1, 0, ::3] = -0.0
    s[1, 1] = torch.tensor([math.nan, -math.inf, math.inf, -1.0, 1e-42, -0.0, 0.0, 3e38]).repeat(38)[:300]
    check_evict(c, 90, 2, 5, s)
    c = evict_case("piece", BF16, [300, 200], 90)
    check_evict(c, 90, 0, 0, -torch.exp(normal(c.g, 2, 2, 300)))


def test_evict_missing_blocks():
    c = evict_case("piece", BF16, [100], 40)
    c.table[0, 2] = -1
    check_evict(c, 40, 4, 4, torch.rand(1, 2, 100, generator=c.g))


# ------------------------------------------------------------------ refusals
def refused(call, name="MMA_ERR_INVALID_ARG"):
    with pytest.raises(mma.MMAError) as e:
        call()
    assert e.value.name == name, e.value


def test_refusals():
    c = Case("piece", BF16, [40], [3], heads=2)
    lay, seqs, layer = c.layout(), c.seqs(), c.flat[0].cuda()
    q = torch.zeros(3, 8, 128, dtype=BF16, device="cuda")
    k = q[:, :2]
    att = lambda lay=lay, layer=layer, seqs=seqs, q=q, **kw: mma.mma_kv_attention(lay, layer, seqs, q, **kw)  # noqa: E731
    app = lambda lay=lay, layer=layer, seqs=seqs, q=q, k=k, **kw: mma.mma_kv_append(lay, layer, seqs, q, k, k, **kw)  # noqa: E731

    def other(**kw):
        f = dict(num_layers=1, block_tokens=16, kv_heads=2, head_dim=128, elem_bytes=2, gpu_num_blocks=c.c.blocks,
                 host_num_slots=1, gpu_layout=0)
        f.update(kw)
        return mma.kv_layout(*f.values())
    for bad in (dict(gpu_layout=3), dict(block_tokens=0), dict(elem_bytes=4), dict(gpu_num_blocks=c.c.blocks + 1000),
                dict(gpu_layout=1, block_tokens=4)):
        refused(lambda: att(other(**bad)))
    wide = torch.zeros(3, 8, 264, dtype=BF16, device="cuda")
    refused(lambda: att(other(head_dim=264), q=wide))
    refused(lambda: att(other(head_dim=12), q=wide[:, :, :12]))
    refused(lambda: att(other(kv_heads=3, gpu_num_blocks=1)))      # 8 query heads over 3
    refused(lambda: att(layer=layer.data_ptr() + 2))               # 16-byte alignment
    refused(lambda: att(layer=torch.zeros(64)))                    # host memory
    refused(lambda: att(layer=0))
    refused(lambda: att(seqs=c.seqs(max_len=0)))
    refused(lambda: att(seqs=c.seqs(max_len=c.table.shape[1] * 16 + 1)))
    refused(lambda: att(scores_out=torch.zeros(1, 2, c.max_len - 1, device="cuda")))
    refused(lambda: att(out=torch.zeros(1, 8, 128, dtype=BF16, device="cuda").expand(3, 8, 128)))  # rows overlap
    refused(lambda: app(q_out=torch.zeros(3, 1, 128, dtype=BF16, device="cuda").expand(3, 8, 128)))
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    for rot in (7, 130):
        refused(lambda: app(positions=pos, rope=torch.zeros(64, rot, device="cuda")))
    refused(lambda: app(q_weight=torch.ones(128, dtype=BF16, device="cuda"), eps=-1.0))
    long = Case("piece", BF16, [4000], [3], heads=2)
    refused(lambda: mma.mma_kv_attention(long.layout(), long.flat[0].cuda(), long.seqs(), q,
                                         workspace=torch.empty(256, dtype=torch.uint8, device="cuda")), "MMA_ERR_BUFFER_TOO_SMALL")
    dst = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    sc = torch.zeros(1, 2, 64, device="cuda")
    ev = lambda keep, dst=dst, sc=sc, **kw: mma.mma_kv_evict(lay, layer, seqs, dst, sc, keep, **kw)  # noqa: E731
    refused(lambda: ev(33))                       # two blocks hold 32
    refused(lambda: ev(20, sinks=10, recent=11))
    refused(lambda: ev(20, sc=torch.zeros(1, 2, 42, device="cuda")))
    acc = torch.zeros(1, 4, dtype=torch.int32, device="cuda")
    refused(lambda: mma.mma_kv_commit(lay, [0], seqs, acc, acc[:, 0].contiguous()))
    refused(lambda: mma.mma_kv_commit(lay, [layer], seqs, acc, acc[0, :1], scores=[torch.zeros(1, 2, 20, device="cuda")]))
    a = mma.mma_kv_commit_t(acc.data_ptr(), acc.data_ptr(), seqs.tensors[1].data_ptr(), 0, 4, 0)
    assert mma.lib.mma_kv_commit(lay, mma.layer_table([layer]), seqs.c, a, 0) == mma.MMA_ERR_INVALID_ARG
    for call in (lambda: att(q=q.float()), lambda: att(q=q[:, :, :64]), lambda: app(k=q[:, :3]),
                 lambda: att(tree=torch.zeros(2, 1, dtype=torch.int64, device="cuda")), lambda: att(q=q.cpu()),
                 lambda: att(lse=torch.zeros(3, 7, device="cuda")), lambda: app(rope=torch.zeros(4, 8, device="cuda")),
                 lambda: att(scores_in=sc), lambda: ev(0)):
        with pytest.raises(ValueError):
            call()


def test_nothing_to_do():
    c = Case("piece", BF16, [40], [0], heads=2)
    q = torch.zeros(0, 8, 128, dtype=BF16, device="cuda")
    layer = c.flat[0].cuda()
    assert mma.mma_kv_attention(c.layout(), layer, c.seqs(), q).shape == (0, 8, 128)
    assert mma.mma_kv_append(c.layout(), layer, c.seqs(), q, q[:, :2], q[:, :2]).shape == (0, 8, 128)
    assert same_bits(layer.cpu(), c.flat[0])


# ------------------------------------------------------------------ many rows, long rows, large caches, together
@pytest.mark.parametrize("layout,cache,dim,tokens,group,lens,counts", [
    ("piece", BF16, 128, 16, 4, [300, 0, 65], [40, 9, 12]),      # 128 rows of a workgroup
    ("hnd", F16, 128, 24, 4, [130], [13]),                       # 64 rows
    ("xpacked", F8, 128, 16, 4, [500, 64, 31], [33, 32, 1]),
    ("hnd", F8, 80, 16, 4, [260, 700], [20, 34]),
    ("piece", F8, 64, 16, 2, [520, 3], [70, 33]),
    ("xpacked", BF16, 256, 16, 2, [150, 33], [30, 50]),
    ("piece", F8, 256, 5, 3, [99], [40]),
    ("xpacked", F16, 64, 32, 8, [400], [12]),
    ("hnd", BF16, 40, 3, 5, [77, 10], [30, 11]),
])
def test_attention_many_rows(layout, cache, dim, tokens, group, lens, counts):
    log(f"attention rows {layout} {cache} dim {dim}")
    dtype = F16 if cache is F16 else BF16
    check_attention(Case(layout, cache, lens, counts, dim, 1, group, tokens, dtype), None, True)
    c = Case(layout, cache, lens, counts, dim, 1, group, tokens, dtype, seed=3)
    check_attention(c, tree_bits(counts, c.g, empty=True), True)


@pytest.mark.parametrize("layout,cache", [("piece", BF16), ("xpacked", F8), ("hnd", F8), ("xpacked", F16)])
def test_attention_many_rows_over_splits_and_missing_blocks(layout, cache):
    """Hundreds of tiles, split and joined, with blocks that are not there at the start, inside and at the end."""
    c = Case(layout, cache, [1500, 0, 700], [20, 17, 3], dim=64, heads=1, group=4, dtype=F16 if cache is F16 else BF16)
    check_attention(c, None, True)
    for b in (0, 3, 50, 93):
        c.table[0, b] = -1
    c.table[1, :] = -1
    c.table[2, 43] = c.c.blocks
    check_attention(c, tree_bits(c.counts, c.g), True)


def test_attention_chunk_without_context():
    """A whole prompt: every row sees its own part of the call's tokens and nothing else."""
    c = Case("hnd", BF16, [0, 0], [300, 37], dim=64, heads=1, group=1)
    check_attention(c, None, True)


@pytest.mark.parametrize("n,keep", [(20000, 7000), (70000, 30000), (70001, 3)])
def test_evict_rows_past_the_registers(n, keep):
    """Rows listed by a launch of their own, and rows that are read anew in each pass, with ties across them."""
    c = evict_case("hnd", F8, [n, n - 4100], keep, dim=16, heads=1)
    s = torch.exp(3 * normal(c.g, 2, 1, n))
    s[1] = torch.randint(0, 3, (1, n), generator=c.g).float()
    check_evict(c, keep, 1, 2, s)


def test_caches_past_32_bits():
    """Blocks whose bytes lie more than 4 GiB into a layer give what the same blocks give in a small one."""
    small = Case("hnd", BF16, [200], [3], heads=8)
    blocks = 80_000  # of 32 KiB, twice: 4.9 GiB
    layer = torch.empty(2 * blocks * small.c.piece, dtype=BF16, device="cuda")
    big = mma.kv_layout(1, 16, 8, 128, 2, blocks, 1, LAYOUTS["hnd"])
    shift = blocks - small.c.blocks
    lay, flat = small.layout(), small.flat[0].cuda()
    view = layer.view(2, blocks, -1)
    view[:, shift:] = flat.view(2, small.c.blocks, -1)
    far = mma.kv_seqs((small.table + shift).cuda(), torch.tensor(small.lens, dtype=torch.int32).cuda(), small.q_start.cuda(),
                      max_tokens=3, max_len=small.max_len)
    near = small.seqs()
    q = normal(small.g, 3, 32, 128).to(BF16).cuda()
    for l, x, s in ((lay, flat, near), (big, layer, far)):
        mma.mma_kv_append(l, x, s, q, q[:, :8], q[:, 8:16])
    a, b = (mma.mma_kv_attention(l, x, s, q) for l, x, s in ((lay, flat, near), (big, layer, far)))
    wide = q.repeat(1, 4, 1)
    c, d = (mma.mma_kv_attention(l, x, s, wide) for l, x, s in ((lay, flat, near), (big, layer, far)))
    acc, one = torch.tensor([[1, 2]], dtype=torch.int32, device="cuda"), torch.tensor([2], dtype=torch.int32, device="cuda")
    for l, x, s in ((lay, flat, near), (big, layer, far)):
        mma.mma_kv_commit(l, [x], s, acc, one)
    assert same_bits(a.cpu(), b.cpu()) and same_bits(c.cpu(), d.cpu())
    assert same_bits(view[:, shift:].contiguous().cpu(), flat.view(2, small.c.blocks, -1).cpu())
    sc = torch.rand(1, 8, small.max_len, device="cuda")
    dst = small.spare[:2].view(1, 2).cuda()
    mma.mma_kv_evict(big, layer, far, dst + shift, sc, 20)
    mma.mma_kv_evict(lay, flat, near, dst, sc, 20)
    assert same_bits(view[:, shift:].contiguous().cpu(), flat.view(2, small.c.blocks, -1).cpu())


def test_all_on_another_stream_and_captured():
    """A decode step (append, attention with scores, commit, evict) on a stream of its own and in a graph, replayed
    with other work between the replays, gives the bits of the eager calls."""
    c = Case("xpacked", F8, [700, 90], [5, 3], heads=2, layers=2)
    extra = ok.Cache("xpacked", F8, c.c.blocks + 6, 16, 2, 128)
    c.c, c.flat = extra, to_cache(normal(c.g, 2, 2 * extra.blocks * extra.piece), F8)
    dst = (torch.arange(6, dtype=torch.int32).view(2, 3) + extra.blocks - 6).cuda()
    lay, seqs, sc = c.layout(), c.seqs(), c.scales()
    q = normal(c.g, 8, 8, 128).to(BF16).cuda()
    k, v = q[:, :2].contiguous(), q[:, 2:4].contiguous()
    scores = torch.rand(2, 2, c.max_len, generator=c.g).cuda()
    other = scores.clone()  # the second layer's
    acc, cnt = torch.tensor([[0, 2, 4], [1, 2, 0]], dtype=torch.int32).cuda(), torch.tensor([3, 2], dtype=torch.int32).cuda()
    ws = torch.empty(max(mma.kv_attention_workspace(lay, seqs, 8, 8, BF16, True), mma.kv_evict_workspace(lay, seqs)),
                     dtype=torch.uint8, device="cuda")

    def step(layers, s_out, stream=None):
        qo = mma.mma_kv_append(lay, layers[0], seqs, q, k, v, **sc, stream=stream)
        out = mma.mma_kv_attention(lay, layers[0], seqs, qo, scores_in=scores, scores_out=s_out, workspace=ws, **sc, stream=stream)
        lens = mma.mma_kv_commit(lay, layers, seqs, acc, cnt, scores=[s_out, other], stream=stream)
        got = mma.mma_kv_evict(lay, layers[1], seqs, dst, s_out, 40, sinks=2, recent=3, workspace=ws, stream=stream)
        return (out, lens, *got)

    def fresh():
        return [x.clone().cuda() for x in c.flat], scores.clone()

    layers, s_out = fresh()
    want = [x.cpu() for x in step(layers, s_out)] + [x.cpu() for x in layers] + [s_out.cpu()]
    side = torch.cuda.Stream()
    layers, s_out = fresh()
    side.wait_stream(torch.cuda.current_stream())
    got = step(layers, s_out, side)
    side.synchronize()
    assert all(same_bits(a.cpu(), b) for a, b in zip([*got, *layers, s_out], want))
    layers, s_out = fresh()
    keep = [x.clone() for x in layers], s_out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(layers, s_out)
    for i in range(3):
        for x, y in zip(layers, keep[0]):
            x.copy_(y)
        s_out.copy_(keep[1])
        ws.random_()
        (torch.randn(512, 512, device="cuda") @ torch.randn(512, 512, device="cuda")).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert all(same_bits(a.cpu(), b) for a, b in zip([*got, *layers, s_out], want)), f"replay {i}"


@pytest.mark.parametrize("layout,cache", [("hnd", "bf16"), ("xpacked", "f8")])
def test_example(layout, cache):
    """The example, in its own process (it initialises the library itself)."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, os.path.join(root, "examples", "kv_decode.py"), "--layers", "2", "--prompt", "700", "--keep",
                        "128", "--steps", "3", "--layout", layout, "--cache", cache], capture_output=True, text=True, timeout=110)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "evicted 700 -> 128 entries" in r.stdout and "140 entries, position 712" in r.stdout, r.stdout


@pytest.mark.parametrize("layout,cache,dim,counts", [("piece", BF16, 128, [1, 2]), ("hnd", F16, 120, [4, 1]), ("xpacked", BF16, 128, [1, 2]),
                                                     ("hnd", F8, 96, [1, 3])])
def test_attention_few_rows_over_thousands_of_entries(layout, cache, dim, counts):
    """With and without the weights of the entries, which take different ways from some length on."""
    for scores in (False, True):
        c = Case(layout, cache, [4300, 0 if layout == "hnd" else 70], counts, dim, 1, 4, dtype=F16 if cache is F16 else BF16)
        c.table[0, 200] = -1
        check_attention(c, tree_bits(c.counts, c.g), scores)


@pytest.mark.parametrize("cache", [BF16, F8])
def test_attention_kept_logits_of_a_whole_tile(cache):
    c = Case("piece", cache, [900, 40], [4, 3], heads=2)
    check_attention(c, tree_bits(c.counts, c.g), True)


def test_append_in_one_part_and_in_several():
    for n in (511, 512):
        check_append(Case("xpacked", BF16, [3], [n], dim=64, heads=1, group=2), 64, False, True)


@pytest.mark.parametrize("layout,cache,dim,lens,counts", [("piece", BF16, 128, [200], [90]), ("hnd", F8, 80, [70, 0], [70, 40]),
                                                          ("xpacked", F16, 256, [130], [70]), ("xpacked", F8, 64, [300, 5], [20, 90])])
def test_attention_scores_of_hundreds_of_rows(layout, cache, dim, lens, counts):
    for tree in (False, True):
        c = Case(layout, cache, lens, counts, dim, 2, 4, dtype=F16 if cache is F16 else BF16)
        c.table[0, 2] = -1
        check_attention(c, tree_bits(c.counts, c.g, empty=True) if tree else None, True)


def odd_rows(x):
    """The rows of x at any 2 bytes, heads outermost."""
    n, h, d = x.shape
    view = torch.zeros(h, n, d + 3, dtype=x.dtype, device="cuda")[:, :, 1: 1 + d].permute(1, 0, 2)
    view.copy_(x)
    return view


@pytest.mark.parametrize("layout,cache,dim,tokens,group,lens,counts", [
    ("piece", F8, 128, 16, 4, [300], [6]),           # 24 rows, entries from memory to registers
    ("piece", BF16, 128, 16, 4, [300, 40], [6, 5]),  # 24 rows through LDS
    ("hnd", F16, 64, 5, 4, [90], [3]),               # blocks of any number of tokens
    ("piece", BF16, 64, 16, 4, [40], [40]),          # 160 rows, one split
    ("xpacked", F8, 64, 16, 2, [1500], [70]),        # 140 rows, several splits
    ("hnd", BF16, 128, 16, 4, [60], [70]),           # 280 rows, past those whose keys stay
    ("hnd", BF16, 256, 16, 2, [600, 9], [20, 40]),
])
def test_attention_in_place_with_scores(layout, cache, dim, tokens, group, lens, counts):
    """The weights of the entries are the queries' though the output takes their place."""
    dtype = F16 if cache is F16 else BF16
    for view in (None, odd_rows):
        c = Case(layout, cache, lens, counts, dim, 2, group, tokens, dtype)
        check_attention(c, tree_bits(counts, c.g), True, q_view=view, in_place=True)
        c = Case(layout, cache, lens, counts, dim, 2, group, tokens, dtype)
        check_attention(c, None, True, q_view=view, in_place=True)


@pytest.mark.parametrize("layers", [1, 200])
def test_commit_of_empty_lists(layers):
    """Lists without places: nothing moves, and the new lengths are the old ones."""
    c = Case("piece", BF16, [7, 0, 30, -4], [3, 2, 5, 0], 16, 2, 1, 8, layers=1)
    layer, scores = c.flat[0].cuda(), torch.rand(4, 2, c.max_len).cuda()
    none, counts = torch.zeros(4, 0, dtype=torch.int32).cuda(), torch.tensor([0, 5, -1, 2], dtype=torch.int32).cuda()
    lay = mma.kv_layout(layers, 8, 2, 16, 2, c.c.blocks, 1, 0)
    torch.full((4,), 77, dtype=torch.int32, device="cuda")  # what the new lengths' memory may hold
    want = scores.clone()
    got = mma.mma_kv_commit(lay, [layer] * layers, c.seqs(), none, counts, scores=[scores] * layers)
    assert got.tolist() == [7, 0, 30, 0]
    assert same_bits(layer.cpu(), c.flat[0]) and torch.equal(scores, want)


@pytest.mark.parametrize("how", ["no tokens", "tokens of no sequence"])
@pytest.mark.parametrize("layout,cache,group,tokens", [("piece", BF16, 4, 16), ("xpacked", F8, 8, 16), ("hnd", F16, 1, 3)])
def test_attention_scores_without_tokens(layout, cache, group, tokens, how):
    """The entries' weights fade all the same, and those past a sequence's entries stay."""
    c = Case(layout, cache, [40, 0, 2100, -3], [0, 0, 0, 0], 64, 2, group, tokens, F16 if cache is F16 else BF16)
    n = 0 if how == "no tokens" else 2
    q = torch.full((n, 2 * group, 64), 3.0, dtype=c.dtype, device="cuda")
    old = torch.rand(4, 2, c.max_len + 3, generator=c.g).cuda()
    new, out = torch.full_like(old, -3.0), torch.full_like(q, 5.0)
    mma.mma_kv_attention(c.layout(), c.flat[0].cuda(), c.seqs(max_tokens=0 if n else 1), q, out=out, scores_in=old,
                         scores_out=new, decay=0.5, **c.scales())
    want = torch.full_like(old, -3.0)
    for s, m in enumerate(c.lens):
        want[s, :, :max(m, 0)] = 0.5 * old[s, :, :max(m, 0)]
    assert torch.equal(new, want) and (out == 5).all()
    mma.mma_kv_attention(c.layout(), c.flat[0].cuda(), c.seqs(max_tokens=0 if n else 1), q, out=out, scores_out=new, **c.scales())
    for s, m in enumerate(c.lens):
        want[s, :, :max(m, 0)] = 0
    assert torch.equal(new, want)


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("seqs,starts", [(0, True), (0, False), (2, True), (2, False)])
def test_append_of_tokens_of_no_sequence(layout, seqs, starts):
    """No sequences, or none that may have tokens: the queries come all the same, and nothing is written to the cache."""
    c = Case(layout, BF16, [7, 5], [17, 3])
    q = normal(c.g, c.total, 8, 128).to(BF16)
    pos = torch.arange(c.total, dtype=torch.int32)
    table = torch.from_numpy(mma.mma_rope_table(30, 128))
    w = (1 + normal(c.g, 128, std=0.2)).to(BF16)
    want, _, _ = ok.append(q, q[:, :2], q[:, :2], pos, table, False, w, w, 1e-6)
    layer, x = c.flat[0].cuda(), q.cuda()
    none = mma.kv_seqs(c.table[:seqs].cuda(), torch.tensor(c.lens[:seqs], dtype=torch.int32).cuda(),
                       c.q_start[:seqs + 1].cuda() if starts else None, max_tokens=0 if seqs else 20, max_len=c.max_len)
    out = torch.full_like(x, 9.0)
    mma.mma_kv_append(c.layout(), layer, none, x, x[:, :2], x[:, :2], pos.cuda(), table.cuda(), q_out=out, q_weight=w.cuda(),
                      k_weight=w.cuda())
    rounded_close(out.cpu(), want, BF16, (128 + 16) * EPS * want.abs().amax(-1, keepdim=True))
    assert same_bits(layer.cpu(), c.flat[0])


@pytest.mark.parametrize("layout,cache,group,tokens,counts", [
    ("piece", BF16, 2, 16, [4, 3]),      # kept logits
    ("hnd", F8, 1, 16, [8, 3]),
    ("hnd", F16, 2, 5, [4, 3]),          # few rows, their keys read again
    ("piece", BF16, 4, 16, [40, 3]),     # many rows, one sequence's past a wave's
    ("xpacked", BF16, 4, 16, [90, 30]),
])
def test_attention_scores_of_rows_that_are_not_numbers(layout, cache, group, tokens, counts):
    """A row that sees a NaN gives NaN to the entries that it sees, and nothing to the others."""
    c = Case(layout, cache, [70, 20], counts, 64, 1, group, tokens, F16 if cache is F16 else BF16)
    tree = tree_bits(counts, c.g)
    tree[:] &= ~4
    tree[1, 0] |= 4  # drafted token 2 is seen by token 1 of its sequence alone
    bad = to_cache(torch.full((64,), math.nan), cache) if cache is not F8 else torch.full((64,), 0x7F, dtype=torch.uint8)
    c.flat[0][c.c.index(0, *c.c.entry(c.table[0], 72), 0)] = bad
    if tokens == 16:
        c.table[0, 1] = -1
    q = normal(c.g, c.total, group, 64).to(c.dtype)
    want = ok.attention(c.c, c.flat[0], c.table, c.spans(), q, group, 0.125, tree, c.k_scale, c.v_scale)
    got = torch.full((2, 1, c.max_len), -3.0, device="cuda")
    mma.mma_kv_attention(c.layout(), c.flat[0].cuda(), c.seqs(), q.cuda(), tree=tree.cuda(), scores_out=got, **c.scales())
    for s, (_, _, _, m) in enumerate(c.spans()):
        a, b = got[s, 0, :m].cpu().double(), want["scores"][s, 0, :m]
        assert s or (torch.isnan(b).any() and not torch.isnan(b).all())
        assert torch.equal(torch.isnan(a), torch.isnan(b)), (torch.isnan(a).sum(), torch.isnan(b).sum())
        rel = 2 * 64 * EPS * want["big"][torch.isfinite(want["big"])].max() + 64 * EPS
        assert ((a - b).abs() / (rel * (1 + b.abs())))[~torch.isnan(b)].max() <= 1


@pytest.mark.parametrize("layout,tokens,count", [("piece", 16, 1), ("xpacked", 16, 3), ("hnd", 5, 1), ("hnd", 16, 12)])
@pytest.mark.parametrize("far", [18.0, 23.5])
def test_attention_of_small_weights_in_half_precision(layout, tokens, count, far):
    """Entries with a weight 2^far times that of each of the others and nothing in their values, as first tokens
    have: the output is the others' alone."""
    n = 3000
    c = Case(layout, F16, [n], [count], 64, 1, 4, tokens, F16)
    for j in range(n + count):
        at = c.c.entry(c.table[0], j)
        k, v = torch.zeros(64), torch.rand(64, generator=c.g) + 0.5
        k[0] = -far / 8 + float(torch.rand(1, generator=c.g)) / 8
        if j % 32 == 5:
            k[0], v = 0, torch.zeros(64)
        c.flat[0][c.c.index(0, *at, 0)], c.flat[0][c.c.index(1, *at, 0)] = k.half(), v.half()
    q = torch.zeros(count, 4, 64)
    q[..., 0] = 8
    check_attention(c, q=q.half(), scale=math.log(2))


@pytest.mark.parametrize("count", [1, 30])
@pytest.mark.parametrize("layout", ["piece", "xpacked"])
def test_attention_scales_that_are_not_numbers(layout, count):
    c = Case(layout, F8, [50], [count], 64)
    q = normal(c.g, count, 8, 64).to(BF16).cuda()
    c.k_scale[1] = math.nan
    out = mma.mma_kv_attention(c.layout(), c.flat[0].cuda(), c.seqs(), q, **c.scales())
    assert torch.isfinite(out[:, :4]).all() and torch.isnan(out[:, 4:]).all()
    out = mma.mma_kv_attention(c.layout(), c.flat[0].cuda(), c.seqs(), q, scale=math.nan)
    assert torch.isnan(out).all()


def test_an_earlier_error_is_not_a_call_s():
    """An error that another call left in the runtime is neither reported as these calls' nor taken away."""
    import ctypes
    hip = ctypes.CDLL("libamdhip64.so.7")
    c = Case("piece", BF16, [40], [3], layers=1)
    lay, seqs, layer = c.layout(), c.seqs(), c.flat[0].cuda()
    q = torch.ones(3, 8, 128, dtype=BF16, device="cuda")
    acc = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    dst, sc = c.spare[:1].view(1, 1).cuda(), torch.rand(1, 2, c.max_len, device="cuda")
    for call in (lambda: mma.mma_kv_append(lay, layer, seqs, q, q[:, :2], q[:, :2]),
                 lambda: mma.mma_kv_attention(lay, layer, seqs, q, scores_out=sc),
                 lambda: mma.mma_kv_commit(lay, [layer], seqs, acc, one),
                 lambda: mma.mma_kv_evict(lay, layer, seqs, dst, sc, 10)):
        call()
        torch.cuda.synchronize()
        try:
            left = hip.hipSetDevice(99)
            assert left != 0
            call()
        finally:
            found = hip.hipGetLastError()
        assert found == left
    torch.cuda.synchronize()


def test_layers_of_another_type_or_order_are_refused():
    c = Case("hnd", BF16, [40], [3])
    lay, seqs, layer = c.layout(), c.seqs(), c.flat[0].cuda()
    q = torch.ones(3, 8, 128, dtype=BF16, device="cuda")
    f8 = Case("hnd", F8, [40], [3])
    small = f8.flat[0].cuda()
    acc, one = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    dst, sc = c.spare[:1].view(1, 1).cuda(), torch.rand(1, 2, c.max_len, device="cuda")
    append = lambda x, l=lay: mma.mma_kv_append(l, x, seqs, q, q[:, :2], q[:, :2])  # noqa: E731
    attend = lambda x, l=lay: mma.mma_kv_attention(l, x, seqs, q)  # noqa: E731
    commit = lambda x: mma.mma_kv_commit(lay, [x], seqs, acc, one)  # noqa: E731
    evict = lambda x: mma.mma_kv_evict(lay, x, seqs, dst, sc, 10)  # noqa: E731
    for call in (append, attend):
        for x in (layer.half(), layer.float(), layer.half().view(2, -1)):
            with pytest.raises(ValueError, match="layer"):
                call(x)
        for t in (torch.float8_e5m2, torch.float8_e4m3fnuz):
            with pytest.raises(ValueError, match="layer"):
                call(small.view(t), f8.layout())
        for x in (small, small.view(F8)):
            call(x, f8.layout())
    strided = torch.zeros(layer.numel(), 2, dtype=BF16, device="cuda")[:, 0]
    for call in (append, attend, commit, evict):
        with pytest.raises(ValueError, match="layer"):
            call(strided)
        for x in (layer, layer.view(torch.uint8), layer.view(2, c.c.blocks, -1), layer.data_ptr()):
            call(x)
    for call in (commit, evict):
        with pytest.raises(ValueError, match="layer"):
            call(layer.float())
    with pytest.raises(ValueError, match="scores"):
        mma.mma_kv_commit(lay, [layer], seqs, acc, one, scores=[])
    assert mma.mma_kv_commit(lay, (x for x in [layer]), seqs, acc, one).tolist() == [41]


def test_attention_padded_heads_take_the_same_time_whatever_ran_before():
    """Heads of 96 are padded to 128 on the chip; what an earlier kernel left in the padding (NaN, here) is not looked
    at. It costs 3.6 times as much if it is; 1.5 leaves room for noise."""
    c = Case("piece", BF16, [0] * 16, [512] * 16, 96, 8, 4)
    layer, seqs, lay = c.flat[0].cuda(), c.seqs(), c.layout()
    q = torch.randn(c.total, 32, 96, device="cuda").to(BF16)
    out = torch.empty_like(q)
    before = Case("piece", BF16, [2000] * 16, [64] * 16, 128, 8, 4)
    other = torch.zeros(before.total, 32, 128, dtype=BF16, device="cuda")
    times = []
    for fill in (0.0, math.nan):
        left = torch.full_like(before.flat[0], fill).cuda()
        took = []
        for _ in range(15):
            mma.mma_kv_attention(before.layout(), left, before.seqs(), other)
            a, b = torch.cuda.Event(True), torch.cuda.Event(True)
            a.record()
            mma.mma_kv_attention(lay, layer, seqs, q, out=out)
            b.record()
            torch.cuda.synchronize()
            took.append(a.elapsed_time(b))
        times.append(sorted(took)[7])
    log(f"padded heads: {times}")
    assert times[1] < 1.5 * times[0], times


def test_an_object_without_a_truth_value_is_refused():
    class Neither:
        def __bool__(self):
            raise RuntimeError("neither")
    c = Case("hnd", BF16, [40], [3])
    q = torch.ones(3, 8, 128, dtype=BF16, device="cuda")
    with pytest.raises(RuntimeError, match="neither"):
        mma.mma_kv_append(c.layout(), c.flat[0].cuda(), c.seqs(), q, q[:, :2], q[:, :2], interleaved=Neither())


def test_commit_with_a_bound_far_above_the_tokens():
    """Without starts each sequence has max_tokens tokens, whatever the product with the sequences before it."""
    c = Case("piece", BF16, [7, 0, 30], [5, 5, 5], 16, 2, 1, 8, layers=1)
    layer = c.flat[0].cuda()
    acc = torch.tensor([[0, 2, 3], [1, 2, 4], [0, 3, 4]], dtype=torch.int32)
    counts = torch.tensor([3, 2, 3], dtype=torch.int32)
    seqs = mma.kv_seqs(c.table.cuda(), torch.tensor(c.lens, dtype=torch.int32).cuda(), max_tokens=1 << 30, max_len=c.max_len)
    moves, lens = ok.commit_moves(acc, counts, [(0, 5, n, n + 5) for n in c.lens])
    assert mma.mma_kv_commit(c.layout(), [layer], seqs, acc.cuda(), counts.cuda()).tolist() == lens == [10, 2, 33]
    want = c.flat[0]
    for s in range(3):
        want = ok.move_entries(c.c, want, c.table[s], c.table[s], moves[s])
    assert same_bits(layer.cpu(), want)


def test_attention_starts_that_descend():
    """Starts that go back, of ranges that do not meet, and a length above the call's bound."""
    c = Case("piece", BF16, [10, 40, 20, 7], [3, 4, 2, 3], heads=1)
    c.q_start = torch.tensor([6, 9, 3, 6, 1], dtype=torch.int32)  # rows 6-8, none, 3-5, none
    check_attention(c)
    c = Case("piece", BF16, [40, 40, 1000], [3, 4, 2], heads=1)
    c.max_len = 300
    check_attention(c, None, True)


@pytest.mark.parametrize("layout,cache,dim", [("hnd", F8, 64), ("piece", BF16, 32), ("xpacked", F8, 128)])
def test_attention_scores_of_12_13_and_16_rows(layout, cache, dim):
    """Rows whose logits are kept up to some number, depending on the keys' bytes, and whose keys are read again above it."""
    for group in (12, 13, 16):
        c = Case(layout, cache, [900, 40], [1, 1], dim, 2, group)
        check_attention(c, tree_bits(c.counts, c.g), True)


FEW_ROWS = [
    # layout, cache, dim, tokens, group, lens, counts
    ("piece", BF16, 128, 16, 4, [700, 33], [1, 3]),     # memory to registers, a tile of rows
    ("xpacked", F8, 128, 16, 4, [700], [4]),
    ("hnd", F16, 64, 16, 8, [300, 90], [2, 2]),
    ("xpacked", F16, 256, 16, 2, [500], [5]),
    ("hnd", BF16, 128, 16, 4, [4400], [1]),             # through LDS, 64 rows of a workgroup
    ("piece", F8, 80, 5, 4, [400], [9]),
    ("xpacked", BF16, 256, 8, 4, [300], [12]),
]


@pytest.mark.parametrize("layout,cache,dim,tokens,group,lens,counts", FEW_ROWS)
def test_attention_of_few_rows_holds_weights_in_two_terms(layout, cache, dim, tokens, group, lens, counts):
    """Where memory bounds a call the products with V lose no more than 2^-15 of a weight (cut to 8 bits, below 2^-7 is
    left, and rounding that to 8 loses 2^-8 of it), and the output's own rounding is what is left of the error."""
    dtype = F16 if cache is F16 else BF16
    c = Case(layout, cache, lens, counts, dim, 1, group, tokens, dtype)
    q = normal(c.g, c.total, group, dim, std=1.0).to(dtype)
    want = ok.attention(c.c, c.flat[0], c.table, c.spans(), q, group, dim ** -0.5, None, c.k_scale, c.v_scale)
    out = mma.mma_kv_attention(c.layout(), c.flat[0].cuda(), c.seqs(), q.cuda(), **c.scales()).cpu().double()
    u = 2.0 ** -(BITS[dtype] + 1)
    p_err = (2 * dim * EPS * want["big"] + 64 * EPS)[..., None]
    tol = u * want["out"].abs() * (1 + 2 * u) + (2.0 ** -15 + p_err) * want["mag"] * (1 + 2 * u) + STEP[dtype]
    worst = ((out - want["out"]).abs() / tol).max().item()
    assert worst <= 1, f"{worst:.3g} of the tolerance"


@pytest.mark.parametrize("layout,cache,dim,tokens,group,lens,counts", FEW_ROWS)
def test_attention_of_few_rows_and_the_ends_of_the_range(layout, cache, dim, tokens, group, lens, counts):
    """An infinite value that all rows see, with weights that one term holds whole, makes infinite outputs; the largest
    finite one that a row does not see does not reach it."""
    dtype = F16 if cache is F16 else BF16
    c = Case(layout, cache, lens, counts, dim, 1, group, tokens, dtype)
    q = torch.zeros(c.total, group, dim, dtype=dtype)
    top = 448.0 if cache is F8 else torch.finfo(cache).max
    at = c.c.index(1, *c.c.entry(c.table[0], lens[0] + counts[0] - 1), 0)
    c.flat[0][at] = to_cache(torch.full((dim,), top), cache)
    out = check_attention(c, q=q)
    if counts[0] > 1:
        assert out[: counts[0] - 1].abs().max() < 16
    if cache is F8:
        return
    c.flat[0][c.c.index(1, *c.c.entry(c.table[0], 9), 0)[0]] = math.inf
    c.flat[0][c.c.index(1, *c.c.entry(c.table[0], 70), 0)[1]] = -math.inf
    out = check_attention(c, q=q)
    assert (out[: counts[0], :, 0] == math.inf).all() and (out[: counts[0], :, 1] == -math.inf).all()


@pytest.mark.parametrize("layout,dim,tokens,lens,counts", [("xpacked", 128, 16, [900], [8]), ("hnd", 128, 16, [300, 70], [24, 9]),
                                                           ("xpacked", 64, 16, [700], [40]), ("piece", 256, 5, [300], [30])])
def test_attention_over_8_bits_loses_no_bits_of_bf16(layout, dim, tokens, lens, counts):
    """8-bit values are exact in f16, so that weights of many rows lose 2^-11 and not bf16's 2^-8."""
    c = Case(layout, F8, lens, counts, dim, 1, 4, tokens)
    q = normal(c.g, c.total, 4, dim, std=0.3).to(BF16)
    want = ok.attention(c.c, c.flat[0], c.table, c.spans(), q, 4, dim ** -0.5, None, c.k_scale, c.v_scale)
    out = mma.mma_kv_attention(c.layout(), c.flat[0].cuda(), c.seqs(), q.cuda(), **c.scales()).cpu().double()
    u = 2.0 ** -8
    p_err = (2 * dim * EPS * want["big"] + 64 * EPS)[..., None]
    tol = u * want["out"].abs() * (1 + 2 * u) + (2.0 ** -11 + p_err) * want["mag"] * (1 + 2 * u) + STEP[BF16]
    worst = ((out - want["out"]).abs() / tol).max().item()
    assert worst <= 1, f"{worst:.3g} of the tolerance"


def test_outputs_that_share_memory_with_inputs_are_refused():
    """Lengths, lists and scores that some workgroups read while others write: refused before a launch."""
    c = Case("piece", BF16, [40, 20], [3, 3], heads=2)
    lay, seqs, layer = c.layout(), c.seqs(), c.flat[0].cuda()
    keep = [layer.clone(), seqs.tensors[1].clone()]
    x = torch.zeros(64, dtype=torch.int32, device="cuda")
    at = lambda i: x.data_ptr() + 4 * i  # noqa: E731
    layers = mma.layer_table([layer])
    call = lambda acc, cnt, out: mma.lib.mma_kv_commit(lay, layers, seqs.c, mma.mma_kv_commit_t(acc, cnt, out, 0, 4, 0), 0)  # noqa: E731
    lens = seqs.tensors[1].data_ptr()
    for out in (at(8), at(9), at(7), at(0), at(6), lens, lens + 4):  # accepted is 0 .. 7, counts 8 and 9
        assert call(at(0), at(8), out) == mma.MMA_ERR_INVALID_ARG
        assert "overlaps" in mma.lib.mma_last_error().decode()
    assert call(at(0), at(8), at(10)) == mma.MMA_OK
    s = torch.rand(2, 2, 64, device="cuda")
    dst = c.spare[:2].view(2, 1).cuda()
    ws = torch.empty(mma.kv_evict_workspace(lay, seqs), dtype=torch.uint8, device="cuda")
    ent = torch.empty(2, 2, 10, dtype=torch.int32, device="cuda")
    ev = lambda entries, out, lens_out: mma.lib.mma_kv_evict(lay, layer.data_ptr(), seqs.c, mma.mma_kv_evict_t(  # noqa: E731
        dst.data_ptr(), s.data_ptr(), entries, out, lens_out, ws.data_ptr(), ws.numel(), 1, 64, 10, 0, 0), 0)
    for bad in ((ent.data_ptr(), s.data_ptr(), 0), (ent.data_ptr(), s.data_ptr() + 4 * 255, 0), (s.data_ptr() + 40, 0, 0),
                (ent.data_ptr(), 0, lens)):
        assert ev(*bad) == mma.MMA_ERR_INVALID_ARG
    q = torch.zeros(6, 8, 128, dtype=BF16, device="cuda")
    more = torch.rand(2 * 2 * 64 + 8, device="cuda")
    a, b = more[:256].view(2, 2, 64), more[8:].view(2, 2, 64)
    refused(lambda: mma.mma_kv_attention(lay, layer, seqs, q, scores_in=a, scores_out=b))
    torch.cuda.synchronize()
    assert same_bits(layer, keep[0]) and torch.equal(seqs.tensors[1], keep[1])
