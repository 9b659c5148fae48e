"""Host side of the operators on the paged KV cache (no GPU): the rotary table against the reference, the
structs of the binding against the header, refusals that need no device, and the reference's own pins."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import kv_ops as ok

mma = pytest.importorskip("paper_2512_16056_amd")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

KINDS = {"none": mma.MMA_ROPE_NONE, "linear": mma.MMA_ROPE_LINEAR, "base": mma.MMA_ROPE_BASE,
         "ramp": mma.MMA_ROPE_RAMP, "bands": mma.MMA_ROPE_BANDS}


@pytest.mark.parametrize("rot,base", [(128, 10000.0), (64, 500000.0), (6, 100.0)])
@pytest.mark.parametrize("kind", list(KINDS))
def test_rope_table(kind, rot, base):
    """Within one rounding to 32 bits: the angle of position p has an error of p * f * 2^-52 in 64 bits."""
    args = dict(factor=8.0, original=4096.0, low=1.0, high=32.0) if kind != "none" else {}
    f, amp = ok.rope_frequencies(rot, base, kind, **args)
    rows = 5000
    t = mma.mma_rope_table(rows, rot, base, KINDS[kind], 8.0, 4096.0, 1.0, 32.0)
    a = np.arange(rows)[:, None] * f
    want = amp * np.concatenate([np.cos(a), np.sin(a)], 1)
    assert t.dtype == np.float32 and t.shape == (rows, rot)
    assert np.abs(t - want).max() <= amp * (2.0 ** -24 + rows * 2.0 ** -50)


def test_rope_scalings_by_hand():
    # linear: position 8 of factor 8 is position 1; base: the lowest frequency is divided by the factor
    one, eight = mma.mma_rope_table(9, 32), mma.mma_rope_table(9, 32, kind=mma.MMA_ROPE_LINEAR, factor=8.0)
    assert np.allclose(one[1], eight[8], atol=1e-6)
    f, _ = ok.rope_frequencies(32, 10000.0, "base", 4.0)
    g, _ = ok.rope_frequencies(32)
    assert math.isclose(f[-1], g[-1] / 4, rel_tol=1e-12) and f[0] == g[0] == 1
    # bands and ramp keep the highest frequencies and divide the lowest
    for kind in ("ramp", "bands"):
        f, _ = ok.rope_frequencies(128, 10000.0, kind, 4.0, 4096.0, 1.0, 32.0)
        g, _ = ok.rope_frequencies(128)
        assert f[0] == g[0] and math.isclose(f[-1], g[-1] / 4, rel_tol=1e-12) and np.all(np.diff(f) < 0)


@pytest.mark.parametrize("bad", [dict(rot_dim=7), dict(rot_dim=0), dict(base=0.0), dict(base=math.nan), dict(kind=9),
                                 dict(kind=1, factor=0.5), dict(kind=2, rot_dim=2), dict(kind=3), dict(kind=4, low=5.0, high=2.0),
                                 dict(kind=3, factor=4.0, original_len=100.0, base=1.0)])
def test_rope_table_refusals(bad):
    args = {"rot_dim": 64, "factor": 2.0, **bad}
    with pytest.raises(mma.MMAError) as e:
        mma.mma_rope_table(4, **args)
    assert e.value.name == "MMA_ERR_INVALID_ARG"


def test_structs_match_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    lines, want = ['#include "mma.h"', "#include <stdio.h>", "#include <stddef.h>", "int main(void) {"], []
    for name in ("mma_kv_seqs_t", "mma_rows_t", "mma_rope_t", "mma_kv_append_t", "mma_kv_attention_t", "mma_kv_commit_t",
                 "mma_kv_evict_t"):
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


def test_calls_need_init_and_workspace_does_not():
    lay = mma.kv_layout(1, 16, 8, 128, 2, 5000, 1, 0)
    c = mma.mma_kv_seqs_t(0, 0, 0, 1, 4352, 1, 65536)
    for call, args in ((mma.lib.mma_kv_append, mma.mma_kv_append_t()), (mma.lib.mma_kv_attention, mma.mma_kv_attention_t()),
                       (mma.lib.mma_kv_commit, mma.mma_kv_commit_t()), (mma.lib.mma_kv_evict, mma.mma_kv_evict_t())):
        assert call(lay, None, c, args, None) == mma.MMA_ERR_NOT_INITIALIZED
    need = ctypes.c_uint64(7)
    a = mma.mma_kv_attention_t(num_tokens=1, q_heads=32)
    assert mma.lib.mma_kv_attention_workspace(lay, c, a, need) == mma.MMA_OK and need.value > 0
    for bad in (mma.mma_kv_attention_t(num_tokens=1, q_heads=12), mma.mma_kv_attention_t(num_tokens=1, q_heads=32, type=2),
                mma.mma_kv_attention_t(num_tokens=1, q_heads=32, cache_type=1),
                mma.mma_kv_attention_t(num_tokens=1 << 22, q_heads=32)):
        assert mma.lib.mma_kv_attention_workspace(lay, c, bad, need) == mma.MMA_ERR_INVALID_ARG
    assert mma.lib.mma_kv_attention_workspace(None, c, a, need) == mma.MMA_ERR_INVALID_ARG
    assert mma.lib.mma_kv_attention_workspace(lay, None, a, need) == mma.MMA_ERR_INVALID_ARG
    assert mma.lib.mma_kv_attention_workspace(lay, c, None, need) == mma.MMA_ERR_INVALID_ARG
    # one token in all needs no more workspace than it has splits: rows x splits x (head_dim + 2) floats at most
    assert need.value <= 32 * 256 * 130 * 4


# ------------------------------------------------------------------ the reference's pins
@pytest.mark.parametrize("layout", ["piece", "hnd", "xpacked"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, ok.F8])
def test_reference_indices_are_a_permutation(layout, dtype):
    c = ok.Cache(layout, dtype, 3, 16, 2, 32)
    at = torch.cat([c.index(w, b, t, h) for w in (0, 1) for b in range(3) for t in range(16) for h in range(2)])
    assert sorted(at.tolist()) == list(range(2 * 3 * c.piece))


def test_reference_attention_by_hand():
    """Two keys with logits 0 and ln 3: weights 1/4 and 3/4."""
    c = ok.Cache("piece", torch.bfloat16, 1, 2, 1, 8)
    flat = torch.zeros(2 * c.piece, dtype=torch.bfloat16)
    flat[c.index(0, 0, 1, 0)[0]] = 1.0
    flat[c.index(1, 0, 0, 0)[0]] = 4.0
    flat[c.index(1, 0, 1, 0)[1]] = 8.0
    q = torch.zeros(1, 1, 8)
    q[0, 0, 0] = math.log(3)
    r = ok.attention(c, flat, torch.tensor([[0]]), [(0, 1, 1, 2)], q, 1, 1.0)
    assert torch.allclose(r["out"][0, 0, :2], torch.tensor([1.0, 6.0], dtype=torch.float64), rtol=1e-6)
    assert math.isclose(float(r["lse"]), math.log(4), rel_tol=1e-6)
    assert torch.allclose(r["scores"][0, 0], torch.tensor([0.25, 0.75], dtype=torch.float64), rtol=1e-6)


def test_reference_selection_by_hand():
    nan = math.nan
    assert ok.evict_select([5, 1, 1, 3, 1, 9], 6, 4, 1, 1) == [0, 1, 3, 5]
    assert ok.evict_select([nan, -math.inf, 0.0, -0.0], 4, 2, 0, 0) == [2, 3]
    assert ok.evict_select([nan, -math.inf, nan], 3, 2, 0, 0) == [0, 1]
    assert ok.evict_select([1, 2], 2, 5, 0, 0) == [0, 1]


@pytest.mark.parametrize("dim,elem,rows", [(64, 1, 16), (64, 2, 16), (128, 2, 4), (128, 1, 16), (256, 2, 16)])
@pytest.mark.parametrize("seqs,length", [(64, 131072), (1024, 131072), (65535, 1 << 24), (65535, (1 << 31) - 8192)])
def test_workspace_of_weights_is_bounded(dim, elem, rows, seqs, length):
    """Weights of the entries need 1 GiB at most beside the rows' own sums, however long the sequences may be: of a row
    its lse and a copy of its queries, and parts of a row for each of its splits, of which there are 2048 workgroups' or one."""
    lay = mma.kv_layout(1, 16, 8, dim, elem, 5000, 1, 0)
    c = mma.mma_kv_seqs_t(0, 0, 0, seqs, length // 16, 1, length)
    need = ctypes.c_uint64()
    a = mma.mma_kv_attention_t(num_tokens=seqs, q_heads=8 * rows, scores_out=1, cache_type=2 if elem == 1 else 0)
    assert mma.lib.mma_kv_attention_workspace(lay, c, a, need) == mma.MMA_OK
    own, parts = seqs * 8 * rows * (4 + 2 * dim), (2048 + 8 * seqs) * rows * (dim + 2) * 4
    assert seqs * 8 * rows * 4 <= need.value <= max(1 << 30, own) + parts + 1024
