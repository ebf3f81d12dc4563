"""Chunk attention over E4M3 pools at the edges of the row scaling of q: rows of zeros, rows far below one, and
with elements far apart, at cache scales from 0.37 down to 2^-40.

A row of q is multiplied by the power of two that brings its largest element to 2^10 .. 2^11 and rounded to fp16, whose
smallest step there is 2^-24: an element is off by at most 2^-35 of the row's largest one, a score by at most
d * 2^-35 * max |q| * max |k| * scale.  That is added to e_s of test_gpu_chunk; the rest of the bound is the one there.  It
holds where e_s is small against one, which each test sees to.
"""
import math

import numpy as np
import pytest

from oracle import attention_oracle as O
from oracle import chunk_oracle as K

from test_gpu_chunk import Case

pytestmark = pytest.mark.gpu

BATCHES = {"whole": ([20, 140, 1], [300, 200, 90]), "cut": ([20, 3, 1], [3000, 2500, 2000]),
           "longer than the sequence": ([9, 40, 1], [4, 0, 1])}


def case(lib, batch, scales, dim, q_values=None, kv="e4m3", seed=0):
    q_lens, seq_lens = BATCHES[batch]
    c = Case(lib, q_lens, seq_lens, 8, 2, dim, kv=kv, seed=seed, q_values=q_values)
    if kv == "e4m3":
        c.scales = scales
        c.h.set_kv_dtype(lib.KV_E4M3, *scales)
    cuts = len(lib.libra_chunk_plan_host(148, 8, 2, c.q_lens, c.seq_lens)["merges"])
    assert (cuts > 0) == (batch == "cut")
    return c


def run_and_check(c):
    c.plan()
    c.attn()
    c.torch.cuda.synchronize()
    assert int(c.err) == 0
    (ref, lse, spread), (q, kt, vt) = c.reference()
    got, got_lse = O.bf16_bits_to_f64(c.out.cpu().numpy().view(np.uint16)), c.lse.double().cpu().numpy()
    h16 = 2.0 ** -11 if c.kv == "e4m3" else 2.0 ** -8
    r, G = 0, c.hq // c.hkv
    for b, (n, L) in enumerate(zip(c.q_lens, c.seq_lens)):
        rows = slice(r, r + n)
        r += n
        scale, e_s, tiny = 1 / math.sqrt(c.dim), np.zeros((n, c.hq, 1)), 0.0
        if L:
            aq = np.abs(q[rows]).reshape(n, c.hkv, G, c.dim)
            e_s = c.dim * 2.0 ** -23 * scale * np.einsum("nhgd,htd->hgnt", aq, np.abs(kt[b])).max(axis=-1)
            e_s = e_s.transpose(2, 0, 1).reshape(n, c.hq, 1)
            if c.kv == "e4m3":
                e_s = e_s + c.dim * 2.0 ** -35 * scale * np.abs(kt[b]).max() * np.abs(q[rows]).max(axis=-1, keepdims=True)
                tiny = L * 2.0 ** -25 * np.abs(vt[b]).max()
        assert e_s.max() < 0.125
        e = spread[rows] * (h16 + 2 * (e_s + 2.0 ** -21) + 2.0 ** -20) + tiny
        tol = e + 2.0 ** -8 * (np.abs(ref[rows]) + e) + 2.0 ** -134
        err = np.abs(got[rows] - ref[rows])
        assert np.all(err <= tol), (b, np.argwhere(~(err <= tol))[:4])
        seen = np.isfinite(lse[rows])
        assert np.array_equal(np.isneginf(got_lse[rows]), ~seen)
        d = np.abs(got_lse[rows][seen] - lse[rows][seen])
        assert np.all(d <= (np.broadcast_to(e_s[..., 0] + 2.0 ** -20, seen.shape) + 2.0 ** -20 * np.abs(np.where(seen, lse[rows], 0)))[seen])
    c.h.close()


ROWS = {"zeros": [0.0], "mixed": [0.0, 1.0, 2.0 ** -110, 2.0 ** -60, 0.0, 1e-30, 2.0 ** -126, 2.0 ** -133],
        "far below one": [2.0 ** -107, 2.0 ** -108, 2.0 ** -100], "one among zeros": [0.0] * 17 + [1.0]}


@pytest.mark.parametrize("kv,k_scale", [("e4m3", 0.37), ("e4m3", 0.01), ("e4m3", 0.001), ("e4m3", 2.0 ** -40), ("bf16", 1.0)])
@pytest.mark.parametrize("rows", list(ROWS))
@pytest.mark.parametrize("batch", list(BATCHES))
@pytest.mark.parametrize("dim", [64, 128])
def test_rows_of_zeros_and_small_rows(lib, dim, batch, rows, kv, k_scale):
    """A row of zeros weighs every token that it sees alike."""
    n = sum(BATCHES[batch][0])
    rng = np.random.default_rng(21)
    factor = np.resize(np.array(ROWS[rows]), n * 8).reshape(n, 8, 1)
    c = case(lib, batch, (k_scale, 1.7), dim, (rng.standard_normal((n, 8, dim)) * factor).astype(np.float32), kv=kv, seed=22)
    run_and_check(c)


@pytest.mark.parametrize("batch", list(BATCHES))
@pytest.mark.parametrize("dim", [64, 128])
def test_elements_far_apart(lib, dim, batch):
    """Elements of a row over 2^-40 .. 1 of its largest one, the largest anywhere."""
    n = sum(BATCHES[batch][0])
    rng = np.random.default_rng(23)
    q = rng.standard_normal((n, 8, dim)) * 2.0 ** rng.integers(-40, 1, (n, 8, dim))
    run_and_check(case(lib, batch, (0.01, 0.5), dim, q.astype(np.float32), seed=24))


@pytest.mark.parametrize("up", [1, -1])
@pytest.mark.parametrize("batch", ["whole", "cut"])
@pytest.mark.parametrize("dim", [64, 128])
def test_maximum_grows_all_along(lib, dim, batch, up):
    """Scores that rise, or fall, by far more than the slack of the running maximum along the sequence."""
    q_lens, seq_lens = BATCHES[batch]
    c = case(lib, batch, (0.25, 1.7), dim, np.full((sum(q_lens), 8, dim), 0.25, np.float32), seed=25)
    rng = np.random.default_rng(26)
    for b, L in enumerate(seq_lens):
        ramp = K.e4m3_encode(np.arange(L)[::up] * (100.0 / L) + 0.5)
        ramp = ramp[:, None] + rng.integers(0, 2, (L, dim)).astype(np.uint8)
        for t in range(L):
            c.kh[c.bt[b, t // c.page], :, t % c.page] = ramp[t]
    c.k.copy_(c.torch.from_numpy(c.kh))
    run_and_check(c)
