"""Attention whose scores are capped, biased by distance, kept to a window or seen both ways in a prefix, against the 64-bit
reference (oracle.kv_ops).

Tolerances are those of the plain scores (test_gpu_kv_ops), and of the shape, before any run: c tanh(x / c) is formed as
c (1 - 2 / (1 + 2^y)), whose reciprocal has an error of one unit in its last place, 2^-23 of at most 1, and whose
power's error of 2^-23 counts for half at most: below 2^-21 c. slope * |i - j| is a product and a sum, each rounded
to 2^-24 of at most the logit and the bias. p carries an error in its logit and in the row's sum.
"""
import math

import pytest
import torch

from oracle import kv_ops as ok

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2512_16056_amd as mma  # noqa: E402
from gpu_helpers import session  # noqa: E402
from test_gpu_kv_ops import BF16, BITS, EPS, F8, F16, LAYOUTS, STEP, Case, normal, refused, same_bits, to_cache, tree_bits  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def library():
    with session():
        yield


def i32(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32)


def check(c, cap=0.0, slopes=None, window=0, prefix=None, max_prefix=None, tree=None, scores=False, std=2.0, scale=None, q=None,
          in_place=False):
    D = c.c.dim
    q = normal(c.g, c.total, c.heads_q, D, std=std).to(c.dtype) if q is None else q
    scale = D ** -0.5 if scale is None else scale
    span = c.spans()
    s_in = torch.rand(len(c.lens), c.c.heads, c.max_len + 5, generator=c.g) if scores else None
    shape = dict(slopes=slopes, window=window, prefix=i32(prefix), max_prefix=max_prefix)
    want = ok.attention(c.c, c.flat[0], c.table, span, q, c.group, scale, tree, c.k_scale, c.v_scale, s_in, 0.5, cap, **shape)
    more = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in shape.items()}
    if scores:
        s_out = torch.full_like(s_in, -3.0).cuda()
        more.update(scores_in=s_in.cuda(), scores_out=s_out, decay=0.5)
    lse = torch.full((c.total, c.heads_q), 7.0, device="cuda")
    layer, dev = c.flat[0].cuda(), q.cuda()
    out = mma.mma_kv_attention(c.layout(), layer, c.seqs(), dev, out=dev if in_place else None, scale=scale, softcap=cap,
                               tree=None if tree is None else tree.cuda(), lse=lse, **c.scales(), **more)
    torch.cuda.synchronize()
    assert same_bits(layer.cpu(), c.flat[0])
    covered = torch.zeros(c.total, dtype=torch.bool)
    for a, t, _, _ in span:
        covered[a: a + t] = True
    out, lse = out.cpu()[covered].double(), lse.cpu()[covered].double()
    w = {x: want[x][covered] for x in ("out", "lse", "mag", "big")}
    assert torch.equal(torch.isnan(w["out"]), torch.isnan(out))
    finite = torch.isfinite(w["out"]) & torch.isfinite(w["mag"])
    u = 2.0 ** -(BITS[c.dtype] + 1)
    bias = 0.0 if slopes is None else slopes.abs().max().item() * c.max_len
    x_err = 2 * D * EPS * w["big"] + 64 * EPS + 2 * (4 * EPS * cap + 4 * EPS * bias)
    tol = u * w["out"].abs() * (1 + 2 * u) + (u + x_err[..., None]) * w["mag"] * (1 + 2 * u) + STEP[c.dtype]
    if c.c.dtype is F8:
        # p is in f16 there, 2^11 times what it is to the row's largest: half of f16's last step, 2^-25, is 2^-36 of an entry's V
        tol += 2.0 ** -36 * c.max_len * c.flat.view(F8).float().nan_to_num(0).abs().max().item() * c.v_scale.max().item()
    worst = ((out - w["out"]).abs() / tol)[finite].max().item() if finite.any() else 0.0
    assert worst <= 1, f"out: {worst:.3g} of the tolerance"
    empty = w["lse"] == -math.inf
    assert torch.equal(lse == -math.inf, empty) and not out[empty].any()
    seen = ~empty & torch.isfinite(w["lse"])
    err = (lse - w["lse"]).abs() / (x_err + 64 * EPS * w["lse"].abs())
    assert not seen.any() or err[seen].max().item() <= 1, f"lse: {err[seen].max().item():.3g}"
    if scores:
        got = more["scores_out"].cpu().double()
        written = torch.zeros(got.shape, dtype=torch.bool)
        for s, (_, _, _, m) in enumerate(span):
            written[s, :, :m] = True
        assert (got[~written] == -3).all(), "scores past the entries changed"
        exact = torch.zeros_like(got)
        exact[:, :, : want["scores"].shape[2]] = want["scores"]
        err = ((got - exact).abs() / (x_err.max() * (1 + exact.abs())))[written]
        assert not err.numel() or err.max().item() <= 1, f"scores: {err.max().item():.3g} of the tolerance"
    return out


def alibi(heads):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)])


CASES = [
    # layout, cache, dim, tokens, heads, group, lens, counts: few rows and many, short contexts and split ones
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
    ("hnd", BF16, 72, 24, 1, 5, [200, 64, 65], [1, 13, 0]),
    ("piece", BF16, 128, 16, 2, 4, [300, 0, 65], [40, 9, 12]),
    ("xpacked", F8, 64, 16, 1, 4, [1500, 30], [4, 2]),
    ("hnd", BF16, 64, 16, 1, 2, [10, 0], [200, 130]),
    ("piece", BF16, 64, 16, 1, 2, [3000, 7], [1, 1]),
]
SHAPES = {
    "cap": dict(cap=5.0),
    "slopes": dict(slopes=True),
    "window": dict(window=17),
    "window_1": dict(window=1),
    "window_long": dict(window=200, scores=True),
    "prefix": dict(prefix=45),
    "window_prefix": dict(window=33, prefix=5, scores=True),
    "all": dict(cap=30.0, slopes=True, window=50, prefix=90, scores=True),
}


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("layout,cache,dim,tokens,heads,group,lens,counts", CASES)
def test_shapes(layout, cache, dim, tokens, heads, group, lens, counts, shape):
    c = Case(layout, cache, lens, counts, dim, heads, group, tokens, F16 if cache is F16 else BF16)
    kw = dict(SHAPES[shape])
    if "slopes" in kw:
        kw["slopes"] = alibi(c.heads_q)
    if "prefix" in kw:  # the longest, one, none, and one past the end
        kw["prefix"] = [(kw["prefix"], 1, 0, 10 ** 6)[s % 4] for s in range(len(lens))]
        kw["max_prefix"] = max(kw["prefix"][0], 60)
    check(c, **kw)


@pytest.mark.parametrize("layout", list(LAYOUTS))
def test_window_over_many_splits(layout):
    """A window and a prefix that each take several splits, the gap between them passed over."""
    for count in (1, 3, 40):
        c = Case(layout, BF16, [5000, 10, 0, 1025], [count, 1, 1, count], heads=1, group=2, dim=64)
        check(c, window=1100, prefix=[700, 3, 5, 1000], scores=True)


@pytest.mark.parametrize("cache", [BF16, F8])
def test_edges_of_window_and_prefix(cache):
    """Every place of the window's and the prefix's ends in a tile and a block, one token and some."""
    for n, edge in ((127, 0), (128, 1), (129, 31), (191, 32), (200, 33), (193, 63), (260, 64), (261, 65)):
        for count in (1, 20):
            c = Case("hnd", cache, [n], [count], heads=1, group=4, dim=64, seed=n)
            check(c, window=1 + edge, prefix=[edge], scores=True)
            check(c, window=n - edge, prefix=[n + count - edge])


@pytest.mark.parametrize("layout,cache,lens,counts", [("xpacked", F8, [50], [300]), ("hnd", BF16, [0, 700], [290, 130]),
                                                      ("piece", F16, [5], [520])])
def test_weights_of_rows_in_parts(layout, cache, lens, counts):
    """Many rows over few keys: the rows' weights come in parts that are added up."""
    c = Case(layout, cache, lens, counts, 64, 1, 4, 16, F16 if cache is F16 else BF16)
    n = len(lens)
    check(c, prefix=[200, 13][:n], window=100, scores=True)
    check(c, cap=9.0, slopes=alibi(c.heads_q), scores=True)
    check(c, cap=9.0, tree=tree_bits(c.counts, c.g), scores=True)


def test_prefix_is_bounded_and_may_be_of_nothing():
    c = Case("piece", BF16, [100, 40], [30, 5], heads=1)
    check(c, prefix=[-3, 0], window=7)
    check(c, prefix=[90, 90], max_prefix=13, window=7, scores=True)
    check(c, prefix=[90, 90], max_prefix=0)
    check(c, prefix=[2 ** 31 - 1, 2 ** 31 - 1], max_prefix=2 ** 32 - 1)
    check(c, window=2 ** 32 - 1)


def test_cap_with_a_tree_and_negative_scale():
    for layout in LAYOUTS:
        c = Case(layout, BF16, [70, 0], [24, 5], heads=1)
        check(c, cap=8.0, tree=tree_bits(c.counts, c.g, empty=True), scores=True)
    c = Case("hnd", BF16, [300], [40], heads=1)
    check(c, cap=8.0, scale=-0.3)
    check(c, slopes=-alibi(c.heads_q) * 0.1, scale=-0.3)


@pytest.mark.parametrize("cap", [1e-6, 0.5, 300.0, 1024.0])
def test_caps_from_the_least_to_the_largest(cap):
    for layout, cache, counts in (("hnd", BF16, [1, 3]), ("piece", F16, [40, 5]), ("xpacked", F8, [70, 20])):
        c = Case(layout, cache, [100, 333], counts, heads=1, group=4, dtype=F16 if cache is F16 else BF16)
        check(c, cap=cap, scores=True)
        check(c, cap=cap, std=30.0)
        check(c, cap=cap, slopes=alibi(c.heads_q), window=90, scores=True)


def test_cap_at_both_ends():
    """Logits far past the cap are the cap; infinite ones too, where plain ones would be no numbers."""
    for counts in ([1], [40]):
        c = Case("hnd", BF16, [100], counts, heads=1)
        check(c, cap=3.0, std=300.0)
        c.flat[0][c.c.index(0, *c.c.entry(c.table[0], 7), 0)] = torch.tensor([math.inf] + [0.0] * 127, dtype=BF16)
        q = normal(c.g, c.total, 4, 128).to(BF16)
        q[:, :, 0] = 1.0
        out = check(c, cap=3.0, q=q)
        assert torch.isfinite(out).all()


@pytest.mark.parametrize("cache", [BF16, F16, F8])
@pytest.mark.parametrize("layout", list(LAYOUTS))
def test_infinities_behind_the_window(layout, cache):
    """NaN and infinities in entries out of the window, K and V, reach no row."""
    for counts in ([1, 2], [30, 21]):
        c = Case(layout, cache, [300, 77], counts, heads=1, group=4, dtype=F16 if cache is F16 else BF16)
        bad = torch.full((128,), 0x7F, dtype=torch.uint8) if cache is F8 else \
            to_cache(torch.tensor([math.nan, math.inf, -math.inf, math.nan] * 32), cache)
        for s, n in enumerate(c.lens):
            for j in range(4, n - 40 + 1):
                for which in (0, 1):
                    c.flat[0][c.c.index(which, *c.c.entry(c.table[s], j), 0)] = bad
        out = check(c, window=40, prefix=[4, 4], cap=20.0)
        assert torch.isfinite(out).all()


def test_missing_blocks_and_long_rows_of_tokens():
    for layout in LAYOUTS:
        c = Case(layout, BF16, [170, 33], [50, 2], heads=1)
        c.table[0, 1] = -1
        c.table[0, 8] = c.c.blocks + 7
        c.table[1, :] = -1  # nothing there at all
        check(c, window=60, prefix=[20, 20], cap=9.0, slopes=alibi(4), scores=True)


def test_bounds_of_the_call():
    """Tokens past max_len see what is left of their window; a window that ends before every entry leaves nothing."""
    c = Case("piece", BF16, [10, 40, 20], [3, 40, 2], heads=1)
    c.max_tokens, c.max_len = 30, 30
    check(c, window=4)
    check(c, window=4, prefix=[2, 3, 4])
    for n in (64, 128):  # whole tiles: rows whose walk has no place at all
        for counts in ([40, 1], [3, 2]):
            c = Case("hnd", BF16, [n, n + 5], counts, heads=1, group=4)
            c.max_len = n
            check(c, window=1)
            check(c, window=3, cap=9.0, scores=True)
            check(c, window=2, prefix=[0, 70])
    c = Case("hnd", BF16, [-5, 40, 20], [3, 4, 2], heads=1)
    c.lens[0] = -5
    check(c, window=4, cap=3.0)


def test_in_place_other_stream_and_captured():
    c = Case("hnd", BF16, [3000, 70], [9, 3], heads=2)
    check(c, cap=9.0, window=900, in_place=True, scores=True)
    q = normal(c.g, c.total, c.heads_q, 128).to(BF16).cuda()
    layer, seqs, lay = c.flat[0].cuda(), c.seqs(), c.layout()
    kw = dict(softcap=9.0, window=900, slopes=alibi(c.heads_q).cuda(), prefix=i32([5, 80]).cuda(), max_prefix=80)
    want = mma.mma_kv_attention(lay, layer, seqs, q, **kw)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = mma.mma_kv_attention(lay, layer, seqs, q, stream=side, **kw)
    side.synchronize()
    assert same_bits(got, want)
    out = torch.empty_like(q)
    need = mma.kv_attention_workspace(lay, seqs, q.shape[0], q.shape[1], q.dtype, window=900, prefix=True, max_prefix=80)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mma.mma_kv_attention(lay, layer, seqs, q, out=out, workspace=ws, **kw)
    for _ in range(3):
        out.zero_()
        ws.random_()
        graph.replay()
        torch.cuda.synchronize()
        assert same_bits(out, want)


def test_a_shape_of_nothing_is_the_plain_call():
    c = Case("piece", BF16, [500], [3], heads=2)
    q = normal(c.g, c.total, c.heads_q, 128).to(BF16).cuda()
    layer = c.flat[0].cuda()
    want = mma.mma_kv_attention(c.layout(), layer, c.seqs(), q)
    assert same_bits(mma.mma_kv_attention(c.layout(), layer, c.seqs(), q, softcap=0.0, window=0, max_prefix=3), want)


def test_caches_past_32_bits():
    """A window at the end of a cache whose blocks lie beyond 4 GiB."""
    tokens, heads, dim = 16, 8, 128
    blocks = (5 << 30) // (tokens * heads * dim * 2)
    lay = mma.kv_layout(1, tokens, heads, dim, 2, blocks, 1, mma.MMA_KV_LAYOUT_HND)
    layer = torch.zeros(2 * blocks * tokens * heads * dim, dtype=BF16, device="cuda")
    table = torch.arange(blocks - 20, blocks, dtype=torch.int32, device="cuda")[None].contiguous()
    k = torch.randn(320, heads, dim, device="cuda").to(BF16)
    v = torch.randn(320, heads, dim, device="cuda").to(BF16)
    view = layer.view(2, blocks, heads, tokens, dim)
    view[0, blocks - 20:] = k.view(20, tokens, heads, dim).transpose(1, 2)
    view[1, blocks - 20:] = v.view(20, tokens, heads, dim).transpose(1, 2)
    q = torch.randn(1, heads * 2, dim, device="cuda").to(BF16)
    seqs = mma.kv_seqs(table, torch.tensor([319], dtype=torch.int32, device="cuda"), max_len=320)
    out = mma.mma_kv_attention(lay, layer, seqs, q, window=100)
    kk, vv, qq = k[220:].cpu().double(), v[220:].cpu().double(), q[0].cpu().double().view(heads, 2, dim)
    p = torch.softmax(torch.einsum("hgd,jhd->hgj", qq, kk) * dim ** -0.5, -1)
    want = torch.einsum("hgj,jhd->hgd", p, vv).reshape(1, heads * 2, dim)
    # one rounding of the output and of p, and sums of 128 products in 32 bits
    assert (out.cpu().double() - want).abs().max() <= 2.0 ** -8 * want.abs().max() + 2.0 ** -8 * vv.abs().max()


def test_refusals():
    c = Case("piece", BF16, [40], [3], heads=2)
    lay, seqs, layer = c.layout(), c.seqs(), c.flat[0].cuda()
    q = torch.zeros(3, 8, 128, dtype=BF16, device="cuda")
    att = lambda **kw: mma.mma_kv_attention(lay, layer, seqs, q, **kw)  # noqa: E731
    tree = torch.ones(3, 1, dtype=torch.int64, device="cuda")
    one, pre = torch.ones(8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for kw in (dict(softcap=-1.0), dict(softcap=math.nan), dict(softcap=math.inf), dict(softcap=1e-30), dict(softcap=1e-60), dict(softcap=1025.0),
               dict(tree=tree, window=3), dict(tree=tree, slopes=one), dict(tree=tree, prefix=pre)):
        refused(lambda: att(**kw))
    for kw in (dict(window=-1), dict(window=2 ** 32), dict(slopes=one[:7]), dict(slopes=one.double()), dict(slopes=one.cpu()),
               dict(prefix=pre.long()), dict(prefix=torch.zeros(2, dtype=torch.int32, device="cuda")), dict(prefix=pre, max_prefix=-1)):
        with pytest.raises(ValueError):
            att(**kw)
    with pytest.raises(TypeError):
        att(softcap="3")
    need = mma.kv_attention_workspace(c.layout(), c.seqs(), 3, 8, BF16, True, window=5)
    ws = torch.empty(max(need - 1, 1), dtype=torch.uint8, device="cuda")
    refused(lambda: att(window=5, scores_out=torch.zeros(1, 2, 64, device="cuda"), workspace=ws), "MMA_ERR_BUFFER_TOO_SMALL")


@pytest.mark.parametrize("layout,cache,lens,counts,scores,shape", [
    ("piece", BF16, [4200] + [30] * 31, [1] * 32, False, dict(slopes=True)),    # one token each of many, with more splits than plain
    ("hnd", F16, [4200] + [30] * 31, [1] * 32, False, dict(softcap=20.0)),
    ("xpacked", F8, [50], [300], True, dict(softcap=9.0)),                      # weights of rows in parts
    ("hnd", BF16, [0, 700], [290, 130], True, dict(slopes=True, softcap=9.0)),
])
def test_slopes_and_caps_on_a_stream_and_captured(layout, cache, lens, counts, scores, shape):
    """The workspace is the shape's own, where a plain call's would be too small: the stream's, and one from the query."""
    c = Case(layout, cache, lens, counts, 128 if len(lens) > 2 else 64, 2 if len(lens) > 2 else 1, 4, 16, F16 if cache is F16 else BF16)
    q = normal(c.g, c.total, c.heads_q, c.c.dim, std=2.0).to(c.dtype).cuda()
    layer, seqs, lay = c.flat[0].cuda(), c.seqs(), c.layout()
    size = dict(softcap=shape.get("softcap", 0.0), slopes="slopes" in shape)
    need = mma.kv_attention_workspace(lay, seqs, c.total, c.heads_q, c.dtype, scores, **size)
    assert need > mma.kv_attention_workspace(lay, seqs, c.total, c.heads_q, c.dtype, scores)
    kw = dict(c.scales(), **shape)
    if "slopes" in kw:
        kw["slopes"] = alibi(c.heads_q).cuda()
    weights = lambda: torch.zeros(len(lens), c.c.heads, c.max_len, device="cuda") if scores else None  # noqa: E731
    w = weights()
    want = mma.mma_kv_attention(lay, layer, seqs, q, scores_out=w, **kw)
    side, w2 = torch.cuda.Stream(), weights()
    side.wait_stream(torch.cuda.current_stream())
    got = mma.mma_kv_attention(lay, layer, seqs, q, stream=side, scores_out=w2, **kw)
    side.synchronize()
    assert same_bits(got, want) and (not scores or same_bits(w, w2))
    out, ws = torch.empty_like(q), torch.empty(need, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mma.mma_kv_attention(lay, layer, seqs, q, out=out, workspace=ws, scores_out=w2, **kw)
    for _ in range(3):
        out.zero_()
        ws.random_()
        if scores:
            w2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same_bits(out, want) and (not scores or same_bits(w, w2))


@pytest.mark.parametrize("max_len", [97, 128, 129, 130, 161])
@pytest.mark.parametrize("group", [1, 3])
def test_weights_of_a_last_key_that_few_rows_see(group, max_len):
    """Tokens past max_len whose window ends before the last entry but which the prefix keeps alive, in the same 16 rows as
    tokens that see it: one sequence (keys pass by), several and many rows (keys stay), rows in parts."""
    for lens, counts in (([0], [200]), ([3, 0], [150, 200]), ([0], [400]), ([5, 70], [600, 1])):
        c = Case("hnd", BF16, lens, counts, heads=1, group=group, dim=64)
        c.max_len = max_len
        n = len(lens)
        check(c, window=60, prefix=[5] * n, scores=True)
        check(c, window=41, prefix=[5] * n, cap=9.0, slopes=alibi(c.heads_q), scores=True)


@pytest.mark.parametrize("cap", [1.0, 30.0, 1024.0])
@pytest.mark.parametrize("rows", [False, True])
def test_a_capped_score_by_itself(rows, cap):
    """Tokens that see one entry, whose lse so is the score. Products are exact (one value, times 1); the cap's arithmetic is
    off by 3.5 * 2^-23 of it at most. The factor's seven roundings change the argument by 7 * 2^-24 of itself, what is capped by
    0.448 of that (the maximum of u / cosh^2 u) of the cap. From top to lse there are four more, 2^-24 of it each."""
    lens, counts = ([0], [512]) if rows else ([0] * 512, [1] * 512)
    c = Case("hnd", BF16, lens, counts, heads=1, group=4, dim=8)
    c.flat.zero_()
    for s, (_, _, _, m) in enumerate(c.spans()):
        for j in range(m):
            c.flat[0][c.c.index(0, *c.c.entry(c.table[s], j), 0)[0]] = 1.0
    x = torch.cat([sign * cap * 2.0 ** torch.linspace(-12, 3, 1024) for sign in (-1, 1)])[torch.randperm(2048, generator=c.g)]
    q = torch.zeros(512, 4, 8, dtype=BF16)
    q[:, :, 0] = x.view(512, 4).to(BF16)
    lse = torch.empty(512, 4, device="cuda")
    mma.mma_kv_attention(c.layout(), c.flat[0].cuda(), c.seqs(), q.cuda(), scale=1.0, softcap=cap, window=1, lse=lse)
    want = cap * torch.tanh(q[:, :, 0].double() / cap)
    tol = cap * (3.5 * 2.0 ** -23 + 0.448 * 7 * 2.0 ** -24) + 4 * 2.0 ** -24 * want.abs()
    assert ((lse.cpu().double() - want).abs() / tol).max().item() <= 1


@pytest.mark.parametrize("first", [1, 4, 23])
def test_first_entries_that_stay_in_sight_and_see_nothing_ahead(first):
    """A prompt in two calls, its tokens before entry `first` - 1 without a prefix: every token sees its window and the first
    entries, and nothing behind itself. In one call tokens of the prefix see ahead, and are another's."""
    c = Case("hnd", BF16, [0], [150], heads=1, group=2)
    n, D, window, cut = 150, 128, 40, first - 1
    q = normal(c.g, n, 2, D, std=2.0).to(BF16)
    layer, table = c.flat[0].cuda(), c.table.cuda()

    def part(a, b, **kw):
        seqs = mma.kv_seqs(table, i32([a]).cuda(), max_tokens=b - a, max_len=b)
        return mma.mma_kv_attention(c.layout(), layer, seqs, q[a:b].cuda(), window=window, **kw).cpu()
    with_prefix = dict(prefix=i32([first]).cuda(), max_prefix=first)
    out = torch.cat(([part(0, cut)] if cut else []) + [part(cut, n, **with_prefix)]).double()
    k, v = (torch.stack([c.flat[0][c.c.index(w, *c.c.entry(c.table[0], j), 0)] for j in range(n)]).double() for w in (0, 1))
    i, j = torch.arange(n)[:, None], torch.arange(n)[None]
    sees = (j <= i) & ((i - j < window) | (j < first))
    x = torch.einsum("ihd,jd->hij", q.double(), k) * D ** -0.5
    p = torch.softmax(x.masked_fill(~sees, -math.inf), -1)
    want, mag = (torch.einsum("hij,jd->ihd", p, y) for y in (v, v.abs()))
    big = (torch.einsum("ihd,jd->hij", q.double().abs(), k.abs()) * D ** -0.5).amax(-1).T[..., None]
    u = 2.0 ** -8
    tol = u * want.abs() * (1 + 2 * u) + (u + 2 * D * EPS * big + 64 * EPS) * mag * (1 + 2 * u) + STEP[BF16]
    assert ((out - want).abs() / tol).max().item() <= 1
    ahead = ((part(0, n, **with_prefix).double() - want).abs() / tol).amax((1, 2))
    assert (ahead[cut:] <= 1).all() and (ahead[:cut] > 1).all()


@pytest.mark.parametrize("cap", [1e-3, 1.0, 50.0, 1024.0])
@pytest.mark.parametrize("rows", [False, True])
def test_a_capped_score_near_zero_keeps_its_digits(rows, cap):
    """As test_a_capped_score_by_itself, of scores down to 2^-12 of the cap: off by a part of the score, not of the cap. Its tanh is
    within 2^-21.5 of itself (from 0.55 of the cap on; below 2^-22.5: five roundings of 2^-24, the last of them for what the
    polynomial leaves), and the seven roundings of its factor come to 7 * 2^-24; from top to lse there are four more."""
    lens, counts = ([0], [512]) if rows else ([0] * 512, [1] * 512)
    c = Case("hnd", BF16, lens, counts, heads=1, group=4, dim=8)
    c.flat.zero_()
    for s, (_, _, _, m) in enumerate(c.spans()):
        for j in range(m):
            c.flat[0][c.c.index(0, *c.c.entry(c.table[s], j), 0)[0]] = 1.0
    x = torch.cat([sign * cap * 2.0 ** torch.linspace(-12, 3, 1024) for sign in (-1, 1)])[torch.randperm(2048, generator=c.g)]
    q = torch.zeros(512, 4, 8, dtype=BF16)
    q[:, :, 0] = x.view(512, 4).to(BF16)
    lse = torch.empty(512, 4, device="cuda")
    weights = torch.zeros(len(lens), 1, c.max_len, device="cuda")
    mma.mma_kv_attention(c.layout(), c.flat[0].cuda(), c.seqs(), q.cuda(), scale=1.0, softcap=cap, window=1, lse=lse, scores_out=weights)
    want = cap * torch.tanh(q[:, :, 0].double() / cap)
    tol = (2.0 ** -21.5 + (7 + 4) * 2.0 ** -24) * want.abs()
    assert ((lse.cpu().double() - want).abs() / tol).max().item() <= 1
    # an entry has its token's four rows, of weight 1 each: 2^(x - x), off by twice the error of a logit
    assert (weights.cpu().double() - 4).abs().max().item() <= 4 * 2 * tol.max().item() + 8 * 2.0 ** -24
