"""Host side of beam search's selection, of forking and of compacting (no GPU): the structs of the binding against the header,
refusals that need no device, workspaces, and the reference's own pins."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import beam as ob
from oracle import kv_ops as ok

mma = pytest.importorskip("paper_2512_16056_amd")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_structs_match_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    lines, want = ['#include "mma.h"', "#include <stdio.h>", "#include <stddef.h>", "int main(void) {"], []
    for name in ("mma_kv_shape_t", "mma_beam_select_t", "mma_kv_fork_t", "mma_kv_compact_t"):
        cls = getattr(mma, name)
        lines.append(f'  printf("%zu\\n", sizeof({name}));')
        want.append(ctypes.sizeof(cls))
        for f, _ in cls._fields_:
            lines.append(f'  printf("%zu\\n", offsetof({name}, {f}));')
            want.append(getattr(cls, f).offset)
    src = tmp_path / "l.c"
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    subprocess.run([cc, "-std=c99", f"-I{os.path.join(ROOT, 'include')}", str(src), "-o", str(tmp_path / "l")], check=True)
    out = subprocess.run([str(tmp_path / "l")], check=True, capture_output=True, text=True).stdout
    assert [int(x) for x in out.split()] == want


def test_calls_need_init():
    lay = mma.kv_layout(1, 16, 8, 128, 2, 5000, 1, 0)
    c = mma.mma_kv_seqs_t(0, 0, 0, 1, 4352, 1, 65536)
    shape = mma.mma_kv_shape_t(softcap=3.0)
    assert mma.lib.mma_kv_attention_shaped(lay, None, c, mma.mma_kv_attention_t(), shape, None) == mma.MMA_ERR_NOT_INITIALIZED
    assert mma.lib.mma_beam_select(mma.mma_beam_select_t(), None) == mma.MMA_ERR_NOT_INITIALIZED
    assert mma.lib.mma_kv_fork(lay, None, c, mma.mma_kv_fork_t(), None) == mma.MMA_ERR_NOT_INITIALIZED
    assert mma.lib.mma_kv_compact(lay, None, mma.mma_kv_compact_t(), None) == mma.MMA_ERR_NOT_INITIALIZED


@pytest.mark.parametrize("bad", [dict(softcap=-1.0), dict(softcap=math.nan), dict(softcap=math.inf), dict(softcap=1e-7),
                                 dict(softcap=1e7), dict(tree=1, window=3), dict(tree=1, slopes=1), dict(tree=1, prefix=1)])
def test_shapes_that_are_refused(bad):
    lay = mma.kv_layout(1, 16, 8, 128, 2, 5000, 1, 0)
    c = mma.mma_kv_seqs_t(0, 0, 0, 1, 4352, 1, 65536)
    a = mma.mma_kv_attention_t(num_tokens=1, q_heads=32, tree=bad.pop("tree", None), tree_words=1)
    need = ctypes.c_uint64()
    assert mma.lib.mma_kv_attention_shaped_workspace(lay, c, a, mma.mma_kv_shape_t(**bad), need) == mma.MMA_ERR_INVALID_ARG


def test_a_window_needs_less_workspace():
    """Splits go by what a workgroup walks over: the same for every context that is longer."""
    lay = mma.kv_layout(1, 16, 8, 128, 2, 5000, 1, 0)
    a = mma.mma_kv_attention_t(num_tokens=1, q_heads=32)

    def need(length, **shape):
        c = mma.mma_kv_seqs_t(0, 0, 0, 1, length // 16, 1, length)
        n = ctypes.c_uint64()
        assert mma.lib.mma_kv_attention_shaped_workspace(lay, c, a, mma.mma_kv_shape_t(**shape), n) == mma.MMA_OK
        return n.value
    assert need(65536) == need(65536, softcap=3.0) == need(65536, prefix=1, max_prefix=9) > 0
    assert need(65536, window=1024) == need(1 << 20, window=1024) < need(65536)
    assert need(65536, window=1024, max_prefix=60000) == need(65536, window=1024)  # no prefix
    assert need(65536, window=1024, prefix=1, max_prefix=60000) > need(65536, window=1024)
    assert need(65536, window=2 ** 32 - 1, prefix=1, max_prefix=2 ** 32 - 1) == need(65536)


@pytest.mark.parametrize("bad", [dict(beams=0), dict(beams=65), dict(keep=0), dict(keep=129), dict(vocab=0), dict(vocab=2 ** 31),
                                 dict(type=2), dict(type=4), dict(batch=1 << 22)])
def test_selections_that_are_refused(bad):
    need = ctypes.c_uint64()
    good = dict(batch=2, beams=4, vocab=32000, keep=8, type=0)
    assert mma.lib.mma_beam_select_workspace(mma.mma_beam_select_t(**good), need) == mma.MMA_OK and need.value > 0
    assert mma.lib.mma_beam_select_workspace(mma.mma_beam_select_t(**{**good, **bad}), need) == mma.MMA_ERR_INVALID_ARG


def test_workspaces():
    need = ctypes.c_uint64(3)
    assert mma.lib.mma_kv_fork_workspace(mma.mma_kv_fork_t(num_children=7), need) == mma.MMA_OK and need.value == 84
    assert mma.lib.mma_kv_fork_workspace(None, need) == mma.MMA_ERR_INVALID_ARG
    lay = mma.kv_layout(1, 16, 8, 128, 2, 5000, 1, 0)
    assert mma.lib.mma_kv_compact_workspace(lay, need) == mma.MMA_OK and need.value >= 8 * 5000
    assert mma.lib.mma_kv_compact_workspace(None, need) == mma.MMA_ERR_INVALID_ARG
    assert mma.beam_select_workspace(1, 4, 32000, 8, torch.bfloat16) > 0
    with pytest.raises(ValueError):
        mma.beam_select_workspace(1, 4, 32000, 8, torch.float64)


# ------------------------------------------------------------------ the reference's pins
def test_reference_selection_by_hand():
    """Two beams over two words: probabilities 1/4, 3/4 and 1/2, 1/2, the second beam twice as likely."""
    x = np.log(np.array([[[1.0, 3.0], [5.0, 5.0]]]))
    t, p, v, gap = ob.select(x, np.log(np.array([[0.25, 0.5]])), 3)
    assert t.tolist() == [[0, 1, 1]] and p.tolist() == [[1, 1, 0]]
    assert np.allclose(np.exp(v), [[0.25, 0.25, 0.1875]], rtol=1e-12) and math.isclose(gap, math.log(4 / 3), rel_tol=1e-12)
    t, p, v, _ = ob.select(x, np.array([[-math.inf, -1.0]]), 3, np.array([[0, 1]]), 1)
    assert t.tolist() == [[1, -1, -1]] and p.tolist() == [[1, -1, -1]] and v[0, 0] == -1.0


def test_reference_selection_of_equal_values_goes_by_logit():
    """1e-20 and 0 make the same value: the larger logit first, then the lower token; the lower beam before both."""
    x = np.array([[[0.0, 1e-20, 1e-20], [3e-20, 0.0, 0.0]]])
    t, p, v, _ = ob.select(x, np.full((1, 2), -1.0), 5)
    assert t.tolist() == [[1, 2, 0, 0, 1]] and p.tolist() == [[0, 0, 0, 1, 1]] and len(set(v[0])) == 1


def test_reference_fork_by_hand():
    # blocks of 4: sequence 0 has 6 entries in blocks 5 and 2, sequence 1 4 in block 0; 1 and 3 are free, 4 is held elsewhere
    got = ob.fork([[5, 2, -1], [0, -1, -1]], [6, 4], [1, 0, 1, 0, 1, 1], [0, 0], [1, 3], 4, 12, 3)
    assert got == ([[5, 2, -1], [5, 0, 1]], [6, 6], [1, 1, 1, 0, 1, 2], 1, [(2, 0)])


def test_reference_compact_by_hand():
    got = ob.compact([[4, 1, -1], [1, 5, 2]], [0, 2, 0, 0, 1, 1])
    assert got == ([[0, 1, -1], [1, 2, 2]], [1, 2, 1, 0, 0, 0], [-1, 1, -1, -1, 0, 2], 3, [(4, 0), (5, 2)])


def test_reference_shapes_by_hand():
    """Three keys with equal products: a window of one sees the last, a prefix of one the first too, slopes fall with distance."""
    c = ok.Cache("piece", torch.bfloat16, 1, 4, 1, 8)
    flat = torch.zeros(2 * c.piece, dtype=torch.bfloat16)
    for j in range(3):
        flat[c.index(1, 0, j, 0)[0]] = 2.0 ** j
    q, table, span = torch.zeros(1, 1, 8), torch.tensor([[0]]), [(0, 1, 2, 3)]
    see = lambda **kw: float(ok.attention(c, flat, table, span, q, 1, 1.0, **kw)["out"][0, 0, 0])  # noqa: E731
    assert see(window=1) == 4.0 and math.isclose(see(window=1, prefix=torch.tensor([1])), 2.5)
    assert math.isclose(see(slopes=torch.tensor([math.log(2.0)])), (1 * 0.25 + 2 * 0.5 + 4) / 1.75, rel_tol=1e-6)
    flat[c.index(0, 0, 0, 0)[0]] = 1.0
    q[0, 0, 0] = 1e4
    assert math.isclose(see(cap=math.log(3.0)), (3 * 1 + 2 + 4) / 5, rel_tol=1e-9)


# ------------------------------------------------------------------ workspaces of shaped attention
class Seqs:
    """Bounds of a call's sequences, as the query takes them."""

    def __init__(self, num_seqs, max_tokens, max_len, tokens=16):
        self.max_len = max_len
        self.c = mma.mma_kv_seqs_t(0, 0, 0, num_seqs, -(-max_len // tokens), max_tokens, max_len)


SIZES = [  # layout, bytes of an element, heads, dim, sequences, tokens of each, entries: one token of many, rows in parts, a chunk
    (0, 2, 8, 128, 32, 1, 8192), (2, 2, 8, 128, 8, 1, 32768), (1, 1, 8, 128, 3, 1021, 1071), (2, 2, 1, 64, 1, 300, 350),
    (0, 2, 8, 128, 4, 9, 5000), (2, 2, 8, 128, 1, 2048, 8192), (1, 2, 2, 256, 64, 1, 9000), (0, 1, 8, 64, 2, 1, 100)]


@pytest.mark.parametrize("scores", [False, True])
@pytest.mark.parametrize("layout,elem,heads,dim,num,each,length", SIZES)
def test_the_query_knows_every_part_of_a_shape(layout, elem, heads, dim, num, each, length, scores):
    """What kv_attention_workspace says is what the call of that shape asks for, whatever the shape is made of."""
    lay = mma.kv_layout(1, 16, heads, dim, elem, 70000, 1, layout)
    seqs = Seqs(num, each, length)
    a = mma.mma_kv_attention_t(num_tokens=num * each, q_heads=4 * heads, scores_out=1 if scores else None,
                               cache_type=mma.MMA_TYPE_F8 if elem == 1 else mma.MMA_TYPE_BF16)
    for cap in (0.0, 30.0):
        for slopes in (False, True):
            for window in (0, 700):
                for prefix, most in ((False, None), (True, 40), (True, None)):
                    shape = mma.mma_kv_shape_t(slopes=1 if slopes else None, prefix=1 if prefix else None,
                                               max_prefix=length if most is None else most, window=window, softcap=cap)
                    need = ctypes.c_uint64()
                    assert mma.lib.mma_kv_attention_shaped_workspace(lay, seqs.c, a, shape, need) == mma.MMA_OK
                    got = mma.kv_attention_workspace(lay, seqs, num * each, 4 * heads, torch.bfloat16, scores, window=window,
                                                     prefix=prefix, max_prefix=most, softcap=cap, slopes=slopes)
                    assert got == need.value


def test_slopes_and_caps_need_their_own_workspace():
    lay = mma.kv_layout(1, 16, 8, 128, 2, 70000, 1, 0)
    need = lambda **kw: mma.kv_attention_workspace(lay, Seqs(32, 1, 8192), 32, 32, torch.bfloat16, **kw)  # noqa: E731
    assert need(slopes=True) == need(softcap=30.0) == need(slopes=True, softcap=30.0) > need()
    with pytest.raises(mma.MMAError):
        need(softcap=-1.0)
