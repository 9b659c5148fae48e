"""Beam search's selection, and forking and compacting the paged cache, against the reference (oracle.beam).

Whole numbers and moved bytes are compared exactly; a value of a selection is a 64-bit one rounded to 32 bits: 2^-24 of itself,
and 2^-33 for the sums: each power is formed with a relative error of 5.5e-11 (below 2^-34) at most, so the log of their sum is
off by as much, and its own roundings are of 64 bits. Two beams' candidates may so come closer by 1.1e-10: inputs that come
closer than 2.5e-10 do not tell which is larger.
"""
import math

import numpy as np
import pytest
import torch

from oracle import beam as ob
from oracle import kv_ops as ok

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2512_16056_amd as mma  # noqa: E402
from gpu_helpers import session  # noqa: E402
from test_gpu_kv_ops import BF16, F16, F8, LAYOUTS, Case, normal, refused, same_bits  # noqa: E402

F32 = torch.float32


@pytest.fixture(scope="module", autouse=True)
def library():
    with session():
        yield


def gen(seed):
    return torch.Generator().manual_seed(seed)


def i32(x):
    return torch.tensor(x, dtype=torch.int32)


# ------------------------------------------------------------------ selection
def check_select(logits, scores, keep, done=None, done_token=0, view=None, **kw):
    """logits [batch][beams][vocab] of a type, on the CPU."""
    batch, beams, vocab = logits.shape
    dev = logits.cuda() if view is None else view(logits.cuda())
    tokens, parents, best = mma.mma_beam_select(dev, scores.cuda(), keep, done=None if done is None else done.cuda(),
                                                done_token=done_token, **kw)
    torch.cuda.synchronize()
    t, p, v, gap = ob.select(logits.double().numpy(), scores.double().numpy(), keep, None if done is None else done.numpy(),
                             done_token)
    assert gap > 2.5e-10, "the inputs do not tell which is larger"
    assert np.array_equal(parents.cpu().numpy(), p)
    assert np.array_equal(tokens.cpu().numpy(), t)
    got = best.cpu().double().numpy()
    none = t < 0
    assert (got[none] == -math.inf).all()
    assert (np.abs(got[~none] - v[~none]) <= np.abs(v[~none]) * 2.0 ** -24 + 2.0 ** -33).all()
    return tokens, parents, best


def some_logits(g, batch, beams, vocab, dtype, std=2.0):
    return normal(g, batch, beams, vocab, std=std).to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("batch,beams,vocab,keep", [
    (1, 1, 1, 1), (1, 4, 1, 8), (2, 3, 7, 5), (1, 4, 255, 8), (3, 2, 8191, 4), (2, 1, 8192, 2), (1, 2, 8193, 128), (1, 5, 16385, 10),
    (2, 8, 33001, 16), (1, 64, 1000, 128), (17, 3, 300, 6), (1, 1, 200001, 128), (1, 16, 30000, 128), (1, 2, 8185, 3)])
def test_select(batch, beams, vocab, keep, dtype):
    g = gen(vocab + keep)
    scores = -torch.rand(batch, beams, generator=g) * 6
    check_select(some_logits(g, batch, beams, vocab, dtype), scores, keep)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_select_joins_rows_first(dtype):
    """More parts of a request than one merge takes: 64 beams of 8 parts of 128."""
    g = gen(5)
    check_select(some_logits(g, 1, 64, 60000, dtype), -torch.rand(1, 64, generator=g), 128)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_select_parts_of_several_runs(dtype):
    """Rows enough for the workgroups to take several times 8192 logits each: the best late, early, in between, and equal."""
    g = gen(6)
    x = some_logits(g, 8, 40, 50000, dtype)
    x[0] = torch.linspace(-20, 20, 50000).to(dtype)        # ever better: every logit is among the best of its time
    x[1] = torch.linspace(20, -20, 50000).to(dtype)
    x[2] = 1.0
    x[3, :, 49990:] = 30.0
    x[4, :, :40000] = -math.inf
    x[5, 1, 20000] = math.nan
    x[6, :, 30000:] += 800.0                               # past the range of a power taken from the first ones
    x[7] = torch.where(torch.arange(50000) < 20000, -800.0, 0.0).to(dtype) + x[7]
    scores = -torch.rand(8, 40, generator=g)
    for keep in (3, 80, 128):
        check_select(x, scores, keep)


def test_select_large_vocabularies():
    """More parts than a merge takes of one row, were they not longer: 128 of 2 million, 100 of 1.4 million."""
    g = gen(7)
    for vocab, keep in ((2_000_001, 128), (1_400_000, 100)):
        check_select(some_logits(g, 1, 2, vocab, F16), torch.zeros(1, 2), keep)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_select_rows_anywhere(dtype):
    """Rows that start at any element of 16 bytes, apart from each other, and one row for all beams."""
    g = gen(3)
    logits = some_logits(g, 2, 3, 9001, dtype)

    def view(x):
        for shift in (3,):
            buf = torch.full((6, 9001 + 14), math.nan, dtype=dtype, device="cuda")
            buf[:, shift: shift + 9001] = x.view(6, 9001)
            return buf[:, shift: shift + 9001]
    scores = -torch.rand(2, 3, generator=g)
    check_select(logits, scores, 6, view=view)
    one = some_logits(g, 1, 1, 9001, dtype)
    check_select(one.expand(2, 3, 9001), scores, 6, view=lambda x: one.cuda()[0].expand(6, 9001))


def test_select_ties_go_to_the_lowest():
    for dtype, n in ((F32, 20000), (BF16, 8192), (F16, 100)):
        flat = torch.full((2, 4, n), 0.25, dtype=dtype)  # every logit the same: the list overflows
        check_select(flat, torch.zeros(2, 4), 8)
        check_select(flat, torch.tensor([[-1.0, 0, -1, 0], [0, -2, -2, -2]]), 128 if n > 32 else 8)
    g = gen(1)
    few = (torch.randint(0, 3, (2, 4, 30000), generator=g) - 1).to(BF16) * 0.5  # some thousand of each
    few[:, 1:] = few[:, :1]  # the same in every beam
    check_select(few, torch.zeros(2, 4), 100)
    zeros = torch.zeros(1, 2, 5000)
    zeros[0, :, ::2] = -0.0  # equal to 0
    check_select(zeros, torch.zeros(1, 2), 9)


def test_select_ties_in_a_merge():
    """Thousands of equal candidates over 64 beams and their parts: lower beams first, lower tokens first."""
    flat = torch.zeros(1, 64, 17000, dtype=BF16)
    check_select(flat, torch.zeros(1, 64), 128)                 # joined row by row
    check_select(flat[:, :40], torch.zeros(1, 40), 100)         # in one merge
    scores = torch.zeros(1, 64)
    scores[0, ::3] = -1
    check_select(flat[..., :8000].clone(), scores, 128)


def test_select_near_ties_are_told_apart():
    """Two beams with the same logits but one far below: their sums differ by e^-18, 1.5e-8, less than a 32-bit value tells."""
    for at in range(4):
        x = torch.full((1, 4, 40000), -30.0)
        x[..., 7] = 0.0
        x[..., 9] = -0.5
        x[0, :, 100] = torch.tensor([-18.0] * 4)
        x[0, at, 100] = -18.5
        g = ob.select(x.double().numpy(), np.zeros((1, 4)), 2)
        assert g[1][0][0] == at
        tokens, parents, _ = mma.mma_beam_select(x.cuda(), torch.zeros(1, 4, device="cuda"), 1)
        assert tokens.tolist() == [[7]] and parents.tolist() == [[at]]


def test_select_equal_values_of_a_beam_go_by_logit():
    """Values that are equal though their logits are not, as a score far below or tiny logits make them: the larger logit first, then
    the lower token, the same whether a row is in one part, in several, or has them joined first."""
    g = gen(31)
    vocab, keep = 70001, 100
    for dtype, score in ((F32, -1e9), (F32, -1e30), (BF16, -1e30), (F16, -3e38)):
        if score == -1e9:  # some 32 logits to a value: 2^-28 apart, values 2^-23
            row = 2.0 ** -5 + torch.randperm(vocab, generator=g).double() * 2.0 ** -28
        else:
            row = normal(g, vocab)
        row = row.to(dtype)[None, None]
        s = torch.tensor([[score]])
        tokens, _, best = check_select(row, s, keep)                              # 18 parts
        many = mma.mma_beam_select(row.cuda().expand(1100, 1, vocab), s.cuda().expand(1100, 1).contiguous(), keep)  # one
        assert torch.equal(many[0], tokens.expand(1100, keep)) and torch.equal(many[2], best.expand(1100, keep))
        dead = torch.full((1, 64), -math.inf)
        dead[0, 37] = score
        joined = mma.mma_beam_select(row.cuda().expand(1, 64, vocab), dead.cuda(), keep)
        assert torch.equal(joined[0], tokens) and (joined[1] == 37).all()


@pytest.mark.parametrize("beams,vocab,keep", [(40, 12000, 100), (8, 12000, 20), (3, 9000, 7), (1, 40000, 128)])
def test_select_equal_values_of_many_beams(beams, vocab, keep):
    """Every value equal: the lowest beam's best, also where the list of a merge overflows or is thinned; with some of a later beam's
    before them, and tiny logits, whose values are their beam's alone."""
    g = gen(32)
    for dtype in (F32, BF16):
        x = some_logits(g, 2, beams, vocab, dtype)
        scores = torch.full((2, beams), -1e30)
        x[1, beams // 2, 5:] = -math.inf
        scores[1, beams // 2] = 0.0
        check_select(x, scores, keep)
    tiny = normal(g, 1, beams, vocab) * 1e-30
    check_select(tiny, -torch.rand(1, beams, generator=g), keep)
    tiny[0, :, 3] = 0.0
    tiny[0, :, 8000] = -0.0
    check_select(tiny, torch.zeros(1, beams) if beams == 1 else -torch.rand(1, beams, generator=g), keep)


def test_select_beams_without_candidates():
    g = gen(8)
    inf, nan = math.inf, math.nan
    x = some_logits(g, 6, 4, 9000, F32)
    scores = -torch.rand(6, 4, generator=g)
    scores[0] = torch.tensor([-inf, nan, inf, -1.0])   # one beam lives
    scores[1] = -inf                                   # none does
    x[2, 0, 5000] = nan
    x[2, 1, 8999] = inf
    x[2, 2] = -inf
    x[3, :, 3:] = -inf                                 # three candidates a beam
    x[4] = -inf
    x[4, 2, 77] = 3.0                                  # one in all
    x[5, :, 10:20] = -3.4e38                           # the type's lowest: a candidate, the last
    for keep in (1, 8, 40):
        check_select(x, scores, keep)
    x = x.to(F16)
    check_select(x, scores, 8)                         # -3.4e38 is -infinity there


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_select_beams_with_one_way_on(dtype):
    """Rows of which a rule leaves one token: a value is the score itself, to the last bit, so that beams with the same score
    tie whatever their logits are, in one part, several, or joined."""
    g = gen(34)
    for batch, beams, vocab in ((3, 8, 300), (1, 8, 60000), (1, 64, 60000)):
        x = torch.full((batch, beams, vocab), -math.inf)
        for b in range(batch):
            for y in range(beams):
                x[b, y, torch.randint(0, vocab, (1,), generator=g)] = float(normal(g, 1, std=30.0))
        scores = -(torch.arange(beams) // 4 % 3).float().expand(batch, beams).contiguous()
        _, _, best = check_select(x.to(dtype), scores, 128)
        assert torch.equal(best.cpu()[:, :beams], scores.sort(-1, descending=True).values)


def test_select_done_beams():
    g = gen(9)
    x = some_logits(g, 3, 6, 12345, BF16)
    scores = -torch.rand(3, 6, generator=g) * 4
    done = torch.zeros(3, 6, dtype=torch.uint8)
    done[0, 1::2] = 1
    done[1] = 255
    scores[1, 3] = -math.inf
    x[0, 1] = math.nan  # of a beam that has ended: not looked at
    check_select(x, scores, 12, done, 12344)
    check_select(x, scores, 12, done != 0, 0)


@pytest.mark.parametrize("scale,shift", [(1e-30, 0.0), (300.0, 0.0), (1.0, 1e6), (1.0, -1e6), (3.0, 1e4), (1.0, 3e7), (1e20, 0.0), (1e34, 0.0)])
def test_select_scales(scale, shift):
    g = gen(10)
    x = some_logits(g, 2, 2, 20000, F32)
    if scale == 1e-30:
        x = torch.zeros_like(x)
        x[:, :, :50] = torch.linspace(1, 2, 50) * 1e-3
        x[:, 1] += 0.01  # shifted: the same values, equal up to rounding
        x = x[:, :1]
    check_select(x * (1.0 if scale == 1e-30 else scale) + shift if scale != 1e-30 else x, -torch.rand(2, x.shape[1], generator=g), 4)


@pytest.mark.parametrize("beams,vocab", [(2, 20000), (64, 3000), (1, 70000)])
def test_select_logits_of_every_size(beams, vocab):
    """A few logits far above the others, from 2^10 to 2^126, of both signs: what a part or a thread adds to the sum is nothing beside
    a logit further than 600 above its own, wherever 32 bits do not tell 600 less from the logit itself, or round it to more."""
    g = gen(33)
    for e in list(range(10, 45)) + [60, 90, 126]:
        x = normal(g, 2, beams, vocab)
        x[1] -= 1.75 * 2.0 ** e
        for b in range(beams):
            at = torch.randperm(vocab, generator=g)[:4]
            for sign, far in ((0, (1.5, 1.45, 1.25, 1.0)), (1, (-1.0, -1.25, -1.45, -1.5))):
                x[sign, b, at] = torch.tensor(far) * 2.0 ** e
        check_select(x, -torch.rand(2, beams, generator=g) * 6, 5)


def test_select_peaked_rows():
    """A row whose mass is one logit, and masks of -1e9 and -1e4."""
    x = torch.full((1, 2, 30000), -1e9)
    x[0, 0, 29999] = 5.0
    x[0, 1, :3] = torch.tensor([1.0, 2.0, 1.5])
    x[0, 1, 3:9] = -1e4 - torch.arange(6.0)
    check_select(x, torch.tensor([[-0.5, -0.25]]), 8)


def test_select_other_stream_and_captured():
    g = gen(11)
    x = some_logits(g, 2, 4, 33333, BF16)
    scores = -torch.rand(2, 4, generator=g)
    want = check_select(x, scores, 8)
    x, scores = x.cuda(), scores.cuda()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = mma.mma_beam_select(x, scores, 8, stream=side)
    side.synchronize()
    assert all(same_bits(a, b) for a, b in zip(got, want))
    out = tuple(torch.empty_like(w) for w in want)
    ws = torch.empty(mma.beam_select_workspace(2, 4, 33333, 8, BF16), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mma.mma_beam_select(x, scores, 8, out=out, workspace=ws)
    for _ in range(3):
        for o in out:
            o.zero_()
        ws.random_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(same_bits(a, b) for a, b in zip(out, want))


def test_select_many_requests():
    """More requests than workgroups run at once, of few beams and few logits, odd rows; fewer candidates than are kept."""
    g = gen(21)
    for batch, beams, vocab, keep in ((3001, 2, 37, 3), (700, 1, 1, 2)):
        logits = some_logits(g, batch, beams, vocab, F32)
        check_select(logits, -torch.rand(batch, beams, generator=g), keep)


def test_calls_at_once_on_two_streams():
    """Selections, forks and compactions on two streams side by side, each with its own outputs and workspace."""
    g = gen(22)
    x = [some_logits(g, 3, 5, 20001, F32).cuda() for _ in range(2)]
    scores = -torch.rand(3, 5, generator=g).cuda()
    p = Pool([40, 90, 17, 64, 3], share=0.9, spare=60)
    seqs = mma.kv_seqs(i32(p.table.tolist()).cuda(), i32(p.lens).cuda(), max_tokens=0, max_len=p.max_len)
    counts, grow = i32(p.refs.tolist()).cuda(), i32([2] * 5).cuda()
    parents = [i32([0, 0, 1, 3, 3]).cuda(), i32([4, 2, 2, 1, -1]).cuda()]
    lay = p.layout()

    def calls(i, layers, stream):
        best = mma.mma_beam_select(x[i], scores, 7, stream=stream)
        child = mma.mma_kv_fork(lay, layers, seqs, parents[i], counts, grow=grow, stream=stream)
        return best + child + mma.mma_kv_compact(lay, layers, child[0], child[2], stream=stream)

    want = []
    for i in range(2):
        layers = list(p.flat.cuda())
        want.append((calls(i, layers, None), layers))
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    layers = [list(p.flat.cuda()) for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [calls(i, layers[i], streams[i]) for i in range(2)]
    torch.cuda.synchronize()
    for i in range(2):
        assert all(same_bits(a, b) for a, b in zip(got[i], want[i][0]))
        assert all(torch.equal(a, b) for a, b in zip(layers[i], want[i][1]))


def test_select_refusals_and_nothing_to_do():
    x, s = torch.zeros(2, 3, 50, device="cuda"), torch.zeros(2, 3, device="cuda")
    sel = lambda x=x, s=s, keep=4, **kw: mma.mma_beam_select(x, s, keep, **kw)  # noqa: E731
    refused(lambda: sel(keep=129))
    refused(lambda: sel(x=torch.zeros(2, 65, 50, device="cuda"), s=torch.zeros(2, 65, device="cuda")))
    refused(lambda: sel(x=torch.zeros(2, 0, 50, device="cuda"), s=torch.zeros(2, 0, device="cuda")))
    refused(lambda: sel(x=torch.zeros(2, 3, 0, device="cuda")))
    done = torch.zeros(2, 3, dtype=torch.uint8, device="cuda")
    for token in (-1, 50):
        refused(lambda: sel(done=done, done_token=token))
    refused(lambda: sel(workspace=torch.empty(64, dtype=torch.uint8, device="cuda")), "MMA_ERR_BUFFER_TOO_SMALL")
    t = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    refused(lambda: sel(keep=3, out=(t, t, torch.zeros(2, 3, device="cuda"))))      # outputs that share memory
    refused(lambda: sel(keep=3, out=(t, t.clone(), s)))                               # and with an input
    for bad in (lambda: sel(keep=0), lambda: sel(x=x.double()), lambda: sel(x=x.cpu()), lambda: sel(s=s.double()),
                lambda: sel(x=x[:, :2]), lambda: sel(x=x[..., ::2]), lambda: sel(done=done[:1]), lambda: sel(keep=-1),
                lambda: sel(x=torch.zeros(2, 6, 50, device="cuda")[:, :3]), lambda: sel(done=done, done_token=2 ** 40),
                lambda: sel(done=done, done_token=2.5)):
        with pytest.raises(ValueError):
            bad()
    got = sel(x=torch.zeros(0, 50, device="cuda"), s=torch.zeros(0, 3, device="cuda"))
    assert all(o.shape == (0, 4) for o in got)


# ------------------------------------------------------------------ fork
class Pool:
    """A pool of random contents and tables of sequences, some blocks shared, with their counts."""

    def __init__(self, lens, layout="piece", cache=BF16, tokens=16, heads=2, dim=16, layers=2, width=None, spare=20, seed=0,
                 share=0.5, reserve=0):
        g = np.random.default_rng(seed)
        self.lens, self.tokens, self.layers = list(lens), tokens, layers
        self.max_len = max(self.lens + [1])
        self.width = width or max(-(-self.max_len // tokens) + 1 + reserve, 1)
        table = np.full((len(self.lens), self.width), -1)
        used = 0
        for s, n in enumerate(self.lens):
            here = min(-(-max(n, 0) // tokens) + reserve, self.width)
            same = 0
            if s and g.random() < share:
                same = min(int(g.integers(0, max(n, 0) // tokens + 1)), int((table[s - 1] >= 0).sum()))
                table[s, :same] = table[s - 1, :same]
            table[s, same:here] = np.arange(used, used + here - same)
            used += here - same
        others = 3
        self.blocks = used + others + spare
        order = g.permutation(self.blocks)
        self.table = np.where(table >= 0, order[table], -1)
        refs = np.zeros(self.blocks, int)
        np.add.at(refs, self.table[self.table >= 0], 1)
        refs[order[used: used + others]] = g.integers(1, 4, others)
        self.refs = refs
        self.c = ok.Cache(layout, cache, self.blocks, tokens, heads, dim)
        n = layers * 2 * self.blocks * self.c.piece
        raw = torch.from_numpy(g.integers(0, 256, n * self.c.elem, dtype=np.uint8))
        self.flat = raw.view(layers, 2, self.blocks, -1)  # bytes

    def layout(self):
        return mma.kv_layout(self.layers, self.tokens, self.c.heads, self.c.dim, self.c.elem, self.blocks, 1, LAYOUTS[self.c.layout])

    def copied(self, copies):
        want = self.flat.clone()
        for a, b in copies:
            want[:, :, b] = self.flat[:, :, a]
        return want


def check_fork(p, parents, grow=None, width=None, in_place=False, max_len=None, stream=None):
    max_len = max_len or p.max_len
    table, lens, refs, free, copies = ob.fork(p.table.tolist(), p.lens, p.refs.tolist(), parents, grow, p.tokens, max_len,
                                              width or p.width)
    layers = list(p.flat.cuda())
    counts = i32(p.refs.tolist()).cuda()
    seqs = mma.kv_seqs(i32(p.table.tolist()).view(len(p.lens), p.width).cuda(), i32(p.lens).cuda(), max_tokens=0, max_len=max_len)
    n = len(parents)
    kw = {}
    if in_place:
        new = lambda *s: torch.full(s, -77, dtype=torch.int32, device="cuda")  # noqa: E731
        kw["out"] = (new(n, width or p.width), new(n), counts, new(1))
    got = mma.mma_kv_fork(p.layout(), layers, seqs, i32(parents).cuda(), counts, grow=None if grow is None else i32(grow).cuda(),
                          width=width, stream=stream, **kw)
    torch.cuda.synchronize()
    assert got[1].tolist() == lens
    assert got[0].tolist() == table
    assert got[2].tolist() == refs
    assert got[3].tolist() == [free]
    if not in_place:
        assert counts.tolist() == p.refs.tolist()
    assert torch.equal(torch.stack(layers).cpu(), p.copied(copies))
    return got


@pytest.mark.parametrize("layout,cache,tokens,heads,dim", [("piece", BF16, 16, 2, 128), ("xpacked", F8, 16, 8, 64), ("hnd", F16, 5, 3, 24),
                                                           ("piece", F8, 1, 1, 16), ("hnd", BF16, 32, 8, 256)])
def test_fork(layout, cache, tokens, heads, dim):
    g = np.random.default_rng(dim)
    for seed, lens in enumerate(([40, 40, 40, 40], [7], [0, 1, 16, 17, 100, 15], [33, 64, 64, 2, 90, 90, 90, 1])):
        p = Pool(lens, layout, cache, tokens, heads, dim, seed=seed, spare=6 * len(lens) + 40)
        n = len(lens)
        check_fork(p, list(range(n)))                                     # everyone goes on alone
        check_fork(p, [0] * n, [1] * n)                                   # all from one
        check_fork(p, g.integers(-1, n + 1, n).tolist(), g.integers(0, 20, n).tolist())
        check_fork(p, g.integers(0, n, 2 * n + 1).tolist(), [1] * (2 * n + 1), width=p.width + 2, in_place=True)
        check_fork(p, [n - 1], [3])                                       # the others end


def test_fork_ends_and_begins():
    p = Pool([40, 33, 0])
    check_fork(p, [])                              # all blocks come back
    check_fork(p, [-1, -1, 5], [0, 20, 16])        # new sequences
    p = Pool([], width=3, spare=9)
    p.max_len = 40
    check_fork(p, [-1, 0, 7], [16, 17, 100])       # out of nothing, as far as the row goes


def test_fork_without_enough_blocks():
    for spare in (0, 1, 2, 5):
        p = Pool([40, 41, 42, 43], spare=spare, share=0.9, seed=spare)
        check_fork(p, [0, 0, 0, 1, 1, 2, 2, 2], [30] * 8)
        check_fork(p, [2, 2, 2, 2], [1, 0, -5, 40], in_place=True)


def test_fork_open_blocks_that_are_shared():
    """An open block that several sequences have, or a table elsewhere: nobody may write to it, so all but one child copy it."""
    p = Pool([40, 40, 40], share=0.0, spare=30)
    p.table[1] = p.table[2] = p.table[0]
    p.refs[:] = 0
    np.add.at(p.refs, p.table[p.table >= 0], 1)
    check_fork(p, [2, 0, 1, 1])
    p.refs[p.table[0, 2]] += 1
    check_fork(p, [2, 0, 1, 1], [1] * 4)
    # open in one sequence and whole in another
    p.lens = [40, 48, 30]
    check_fork(Pool([40]), [0])
    q = Pool([40, 48, 30], share=0.0, spare=30)
    q.table[1, :3] = q.table[0, :3]
    q.table[2, :2] = q.table[0, :2]
    q.refs[:] = 0
    np.add.at(q.refs, q.table[q.table >= 0], 1)
    for parents in ([0, 1, 2], [0, 0, 2], [2, 2, 0], [2, 1], [0]):
        check_fork(q, parents, [2] * len(parents))


def test_fork_of_missing_blocks_bounds_and_reserves():
    p = Pool([100, -7, 60], reserve=3)
    p.table[0, 2] = -1
    p.table[2, 3] = p.blocks + 5      # the open one is not there: it is left out
    p.table[0, 6] = -9
    p.refs[:] = 0
    there = (p.table >= 0) & (p.table < p.blocks)
    np.add.at(p.refs, p.table[there], 1)
    check_fork(p, [0, 1, 2, 2, 0], [40] * 5)
    check_fork(p, [0, 2, 0], [1] * 3, max_len=50)   # longer ones are cut


def test_fork_of_counts_that_do_not_fit():
    """Tables that hold more than the counts say: results are of no use, but everything stays within the tensors."""
    p = Pool([40, 40, 41], share=0.9)
    p.refs[:] = 0
    layers = list(p.flat.cuda())
    seqs = mma.kv_seqs(i32(p.table.tolist()).cuda(), i32(p.lens).cuda(), max_tokens=0, max_len=p.max_len)
    table, lens, _, _ = mma.mma_kv_fork(p.layout(), layers, seqs, i32([0, 0, 1, 2, 2]).cuda(), i32(p.refs.tolist()).cuda())
    assert lens.tolist() == [40, 40, 40, 41, 41]
    assert ((table >= -1) & (table < p.blocks)).all()


@pytest.mark.parametrize("n,layers", [(300, 1), (1500, 1), (4, 200)])
def test_fork_many(n, layers):
    """More children than threads of a workgroup; more layers than a launch takes."""
    g = np.random.default_rng(n)
    p = Pool(g.integers(1, 60, n).tolist(), heads=1, dim=8, layers=layers, spare=3 * n, tokens=8)
    check_fork(p, g.integers(0, n, n).tolist(), [1] * n)


def test_fork_of_a_large_pool():
    p = Pool([50, 51, 52], heads=1, dim=8, tokens=1, layers=1, spare=70000)
    check_fork(p, [0, 0, 0, 2, 2], [500] * 5, width=600)
    p.refs[:] += 1  # no block is free but those given back
    check_fork(p, [0, 0, 0, 2, 2], [5] * 5, width=600, in_place=True)


def test_fork_other_stream_and_captured():
    p = Pool([40, 40, 41, 39], share=0.9, spare=40)
    side = torch.cuda.Stream()
    check_fork(p, [0, 0, 1, 3], [1] * 4, stream=side)
    table, lens, refs, free, copies = ob.fork(p.table.tolist(), p.lens, p.refs.tolist(), [0, 0, 1, 3], [1] * 4, 16, p.max_len, p.width)
    layers, counts, parents = list(p.flat.cuda()), i32(p.refs.tolist()).cuda(), i32([0, 0, 1, 3]).cuda()
    seqs = mma.kv_seqs(i32(p.table.tolist()).cuda(), i32(p.lens).cuda(), max_tokens=0, max_len=p.max_len)
    grow = i32([1] * 4).cuda()
    out = tuple(torch.empty(s, dtype=torch.int32, device="cuda") for s in ((4, p.width), (4,), (p.blocks,), (1,)))
    ws = torch.empty(48, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mma.mma_kv_fork(p.layout(), layers, seqs, parents, counts, grow=grow, out=out, workspace=ws)
    for _ in range(3):
        for o in out:
            o.fill_(-5)
        ws.random_()
        graph.replay()
        torch.cuda.synchronize()
        assert [o.tolist() for o in out] == [table, lens, refs, [free]]
        assert torch.equal(torch.stack(layers).cpu(), p.copied(copies))


def test_fork_refusals():
    p = Pool([40, 20])
    layers, counts = list(p.flat.cuda()), i32(p.refs.tolist()).cuda()
    table = i32(p.table.tolist()).cuda()
    seqs = mma.kv_seqs(table, i32(p.lens).cuda(), max_tokens=0, max_len=40)
    par = i32([0, 0]).cuda()
    fork = lambda layers=layers, par=par, counts=counts, **kw: mma.mma_kv_fork(p.layout(), layers, seqs, par, counts, **kw)  # noqa: E731
    refused(lambda: fork(width=2))                                  # 32 entries for 40
    refused(lambda: fork(layers=[layers[0], 0]))
    refused(lambda: fork(layers=[layers[0], torch.zeros(64, dtype=torch.uint8)]))
    refused(lambda: fork(workspace=torch.empty(20, dtype=torch.uint8, device="cuda")), "MMA_ERR_BUFFER_TOO_SMALL")
    new = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    w = p.width
    refused(lambda: fork(out=(table, new(2), new(p.blocks), new(1))))
    refused(lambda: fork(out=(new(2, w), seqs.tensors[1], new(p.blocks), new(1))))
    refused(lambda: fork(out=(new(2, w), par, new(p.blocks), new(1))))
    refused(lambda: fork(out=(new(2, w), new(2), new(p.blocks), counts[:1])))
    both = new(p.blocks + 1)
    refused(lambda: mma.mma_kv_fork(p.layout(), layers, seqs, par, both[:-1], out=(new(2, w), new(2), both[1:], new(1))))
    for bad in (lambda: fork(par=par.long()), lambda: fork(counts=counts[:-1]), lambda: fork(grow=new(3)), lambda: fork(width=-1),
                lambda: fork(out=(new(2, w + 1), new(2), new(p.blocks), new(1))), lambda: fork(layers=layers[:1]),
                lambda: fork(layers=[x.transpose(0, 1) for x in layers])):
        with pytest.raises(ValueError):
            bad()


# ------------------------------------------------------------------ compact
def check_compact(p, in_place=False, stream=None):
    table, refs, moved, held, copies = ob.compact(p.table.tolist(), p.refs.tolist())
    layers, counts = list(p.flat.cuda()), i32(p.refs.tolist()).cuda()
    t = i32(p.table.tolist()).view(len(p.lens), p.width).cuda()
    kw = {}
    if in_place:
        kw["out"] = (t, counts, torch.empty_like(counts), torch.zeros(1, dtype=torch.int32, device="cuda"))
    got = mma.mma_kv_compact(p.layout(), layers, t, counts, stream=stream, **kw)
    torch.cuda.synchronize()
    assert got[3].tolist() == [held]
    assert got[0].tolist() == table
    assert got[1].tolist() == refs
    assert got[2].tolist() == moved
    assert torch.equal(torch.stack(layers).cpu(), p.copied(copies))


@pytest.mark.parametrize("layout,cache,tokens,heads,dim", [("piece", BF16, 16, 2, 128), ("xpacked", F8, 16, 8, 64), ("hnd", F16, 5, 3, 24)])
def test_compact(layout, cache, tokens, heads, dim):
    for seed, (lens, spare) in enumerate((([40, 40, 100, 3], 30), ([7], 0), ([16] * 20, 5), ([], 61), ([300, 200], 200))):
        p = Pool(lens, layout, cache, tokens, heads, dim, seed=seed, spare=spare)
        check_compact(p)
        check_compact(p, in_place=True)


@pytest.mark.parametrize("blocks", [1, 2, 63, 64, 65, 1023, 1024, 1025, 4097, 70001])
def test_compact_pools(blocks):
    """Pools of any size: all held, none held, the first ones, the last ones, one, and any."""
    g = np.random.default_rng(blocks)
    p = Pool([], heads=1, dim=8, tokens=1, layers=1, width=4, spare=max(blocks - 3, 0))
    p.blocks = blocks
    p.c = ok.Cache("piece", BF16, blocks, 1, 1, 8)
    p.flat = torch.from_numpy(g.integers(0, 256, 2 * blocks * 16, dtype=np.uint8)).view(1, 2, blocks, 16)
    p.lens, p.table = [0, 0], np.array([[0, blocks - 1, -1, blocks + 3], [blocks // 2, 0, -5, blocks // 3]])
    half = blocks // 2
    for held in (np.ones(blocks), np.zeros(blocks), np.arange(blocks) < half, np.arange(blocks) >= half,
                 np.arange(blocks) == blocks - 1, g.random(blocks) < 0.3, g.random(blocks) < 0.9, -1.0 * (g.random(blocks) < 0.5)):
        p.refs = (held * g.integers(1, 5, blocks)).astype(int)
        check_compact(p)
    check_compact(p, in_place=True)


def test_compact_more_layers_than_a_launch_and_captured():
    check_compact(Pool([40, 30], heads=1, dim=8, layers=200, spare=30, tokens=8), stream=torch.cuda.Stream())
    p = Pool([40, 40, 41, 39], spare=40)
    table, refs, moved, held, copies = ob.compact(p.table.tolist(), p.refs.tolist())
    layers, counts, t = list(p.flat.cuda()), i32(p.refs.tolist()).cuda(), i32(p.table.tolist()).cuda()
    out = (torch.empty_like(t), torch.empty_like(counts), torch.empty_like(counts), torch.zeros(1, dtype=torch.int32, device="cuda"))
    ws = torch.empty(8 + 8 * p.blocks, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mma.mma_kv_compact(p.layout(), layers, t, counts, out=out, workspace=ws)
    for _ in range(3):
        for o in out:
            o.fill_(-5)
        ws.random_()
        graph.replay()
        torch.cuda.synchronize()
        assert [o.tolist() for o in out] == [table, refs, moved, [held]]
        assert torch.equal(torch.stack(layers).cpu(), p.copied(copies))


def test_compact_refusals():
    p = Pool([40, 20])
    layers, counts, t = list(p.flat.cuda()), i32(p.refs.tolist()).cuda(), i32(p.table.tolist()).cuda()
    com = lambda layers=layers, t=t, counts=counts, **kw: mma.mma_kv_compact(p.layout(), layers, t, counts, **kw)  # noqa: E731
    new = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    refused(lambda: com(layers=[layers[0], 0]))
    refused(lambda: com(workspace=torch.empty(20, dtype=torch.uint8, device="cuda")), "MMA_ERR_BUFFER_TOO_SMALL")
    refused(lambda: com(out=(new(*t.shape), new(p.blocks), counts, new(1))))          # moved over the counts
    refused(lambda: com(out=(new(*t.shape), new(p.blocks), new(p.blocks), counts[:1])))
    x = new(p.blocks)
    refused(lambda: com(out=(new(*t.shape), x, x, new(1))))
    both = new(p.blocks + 1)
    refused(lambda: com(counts=both[:-1], out=(new(*t.shape), both[1:], new(p.blocks), new(1))))
    for bad in (lambda: com(t=t.long()), lambda: com(counts=counts[:-1]), lambda: com(layers=layers[:1]), lambda: com(t=t[0])):
        with pytest.raises(ValueError):
            bad()


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("layout,cache", [("hnd", BF16), ("xpacked", F8), ("piece", F16)])
def test_a_beam_search(layout, cache):
    """Two requests of three beams, 40 steps from prompts of 21 and 5: append, attention with a window, a cap and the first
    entries in sight, selection, fork; the pool compacted on the way. Every step's results are checked against the reference on
    the step's own inputs, and every beam's cache against the keys and values of its history."""
    batch, beams, heads, group, dim, tokens, vocab, steps = 2, 3, 2, 2, 64, 16, 500, 40
    dtype = F16 if cache is F16 else BF16
    g = gen(4)
    blocks, width, rows = 90, 6, batch * beams
    c = ok.Cache(layout, cache, blocks, tokens, heads, dim)
    lay = mma.kv_layout(1, tokens, heads, dim, c.elem, blocks, 1, LAYOUTS[layout])
    layer = torch.zeros(2 * blocks * c.piece, dtype=torch.uint8 if cache is F8 else cache, device="cuda")
    embed = normal(g, vocab, (2 * heads + heads * group) * dim).to(dtype).cuda()
    unembed = (normal(g, heads * group * dim, vocab) * 0.2).cuda()
    prompts = [21, 5]
    # One sequence a request first; its beams fork from it.
    refs = torch.zeros(blocks, dtype=torch.int32, device="cuda")
    nothing = mma.kv_seqs(torch.full((1, width), -1, dtype=torch.int32, device="cuda"), i32([0]).cuda(), max_tokens=0, max_len=1)
    table, lens, refs, free = mma.mma_kv_fork(lay, [layer], nothing, i32([-1, -1]).cuda(), refs, grow=i32(prompts).cuda())
    history = [torch.randint(0, vocab, (n,), generator=g).tolist() for n in prompts]

    def append(new):  # new: tokens of each sequence
        flat = [t for x in new for t in x]
        start = i32([0] + np.cumsum([len(x) for x in new]).tolist()).cuda()
        seqs = mma.kv_seqs(table, lens, start, max_tokens=max(len(x) for x in new), max_len=width * tokens)
        x = embed[torch.tensor(flat)].view(len(flat), -1, dim)
        q, k, v = x.split((heads * group, heads, heads), 1)
        return seqs, mma.mma_kv_append(lay, layer, seqs, q, k, v)
    shape = dict(softcap=6.0, window=24, prefix=i32([4] * 2).cuda(), max_prefix=4)
    seqs, q = append(history)
    out = mma.mma_kv_attention(lay, layer, seqs, q, **shape)
    lens = lens + i32(prompts).cuda()
    last = out[torch.tensor(np.cumsum(prompts) - 1)]
    scores = torch.full((batch, beams), -math.inf, device="cuda")
    scores[:, 0] = 0
    logits = (last.float().view(batch, -1) @ unembed).to(BF16)
    logits = logits[:, None].expand(batch, beams, vocab).contiguous()
    for step in range(steps):
        want = ob.select(logits.cpu().double().numpy(), scores.cpu().double().numpy(), beams)
        toks, parents, scores = mma.mma_beam_select(logits, scores, beams)
        assert want[3] > 2.5e-10 and np.array_equal(toks.cpu().numpy(), want[0]) and np.array_equal(parents.cpu().numpy(), want[1])
        rows_of = parents.flatten() if step else torch.div(parents.flatten(), beams, rounding_mode="floor").int()
        seqs = mma.kv_seqs(table, lens, max_tokens=0, max_len=width * tokens)
        want = ob.fork(table.tolist(), lens.tolist(), refs.tolist(), rows_of.tolist(), [1] * rows, tokens, width * tokens, width)
        table, lens, refs, free = mma.mma_kv_fork(lay, [layer], seqs, rows_of, refs, grow=i32([1] * rows).cuda(), out=None)
        assert (table.tolist(), lens.tolist(), refs.tolist(), free.tolist()) == (want[0], want[1], want[2], [want[3]]) and want[3] > 0
        history = [history[r] + [t] for r, t in zip(rows_of.tolist(), toks.flatten().tolist())]
        if step % 7 == 3:
            table, refs, _, held = mma.mma_kv_compact(lay, [layer], table, refs, out=(table, refs, torch.empty_like(refs), free))
            assert int(table.max()) < int(held)
        seqs, q = append([[h[-1]] for h in history])
        shape["prefix"] = i32([4] * rows).cuda()
        out = mma.mma_kv_attention(lay, layer, seqs, q, **shape)
        span = ok.spans(c, table.cpu(), lens.tolist(), i32(list(range(rows + 1))), rows, 1, width * tokens)
        flat = layer.cpu()
        ref = ok.attention(c, flat, table.cpu(), span, q.cpu(), group, dim ** -0.5, cap=6.0, window=24, prefix=i32([4] * rows))
        # one rounding of the output, p in two terms, and some 2^-12 for logits of 32-bit sums (values of order 1)
        assert ((out.cpu().double() - ref["out"]).abs() <= 2.0 ** -8 * ref["mag"] + 2.0 ** -12).all()
        lens = lens + 1
        for s in (step % rows,):  # the cache of one beam: its history's keys and values
            x = embed[torch.tensor(history[s])].view(len(history[s]), -1, dim).cpu()
            for j in range(len(history[s])):
                at = c.entry(table[s].cpu(), j)
                for which, first in ((0, heads * group), (1, heads * group + heads)):
                    for h in range(heads):
                        want = x[j, first + h].double()
                        if cache is F8:
                            want = want.clamp(-448, 448).float().to(F8).double()
                        assert torch.equal(c.values(flat, c.index(which, *at, h)), want)
        logits = (out.float().view(rows, -1) @ unembed).to(BF16).view(batch, beams, vocab)
    assert refs.sum().item() == (table >= 0).sum().item()


@pytest.mark.parametrize("layout,cache", [("hnd", "bf16"), ("xpacked", "f8")])
def test_example(layout, cache):
    """The example, in its own process (it initialises the library itself)."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, os.path.join(root, "examples", "kv_beam.py"), "--layers", "2", "--prompt", "70", "--steps", "20",
                        "--layout", layout, "--cache", cache], capture_output=True, text=True, timeout=110)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "2 prompts of 70 tokens, 20 steps of 4 beams" in r.stdout and "pages moved to the front" in r.stdout, r.stdout
