"""Chunk attention with values that are not finite in slots that a sequence owns: what they reach, and what they do not."""
import numpy as np
import pytest

from test_gpu_chunk import Case

pytestmark = pytest.mark.gpu

BATCHES = {"whole": ([20, 140], [300, 200]), "cut": ([20, 3], [3000, 2500])}
NAN, INF = {"bf16": 0x7FC0, "e4m3": 0x7F}, {"bf16": 0x7F80}


def run(lib, batch, kv, dim, seed, change=None):
    """out and lse as float64 [rows, Hq, ..], after `change` has been made to the pools (HND)."""
    c = Case(lib, *BATCHES[batch], 8, 2, dim, kv=kv, seed=seed)
    assert (len(lib.libra_chunk_plan_host(148, 8, 2, c.q_lens, c.seq_lens)["merges"]) > 0) == (batch == "cut")
    if change is not None:
        change(c)
        for dev, host in ((c.k, c.kh), (c.v, c.vh)):
            dev.copy_(c.torch.from_numpy(host.view(np.int16) if kv == "bf16" else host))
    c.plan(); c.attn()
    c.torch.cuda.synchronize()
    assert int(c.err) == 0
    out, lse = c.out.view(c.torch.bfloat16).double().cpu().numpy(), c.lse.double().cpu().numpy()
    c.h.close()
    return out, lse


def slot(c, b, t):
    return c.bt[b, t // c.page], t % c.page


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("batch", list(BATCHES))
def test_a_key_that_every_row_sees(lib, batch, kv, dim):
    """NaN in a key of sequence 0 and KV head 0: its rows' out and lse are NaN, whether or not the range is cut; nothing else
    changes by a bit."""
    def change(c):
        p, s = slot(c, 0, 5)
        c.kh[p, 0, s, 3] = NAN[kv]
    want, want_lse = run(lib, batch, kv, dim, 31)
    out, lse = run(lib, batch, kv, dim, 31, change)
    assert np.isnan(out[:20, :4]).all() and np.isnan(lse[:20, :4]).all()
    for got, ref in ((out, want), (lse, want_lse)):
        assert np.array_equal(got[:20, 4:], ref[:20, 4:]) and np.array_equal(got[20:], ref[20:])


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kv,value", [("bf16", "nan"), ("bf16", "inf"), ("e4m3", "nan")])
@pytest.mark.parametrize("batch", list(BATCHES))
def test_a_key_that_only_the_last_row_sees(lib, batch, kv, value, dim):
    """Masked scores are replaced, not added to: the rows before are the same bits."""
    def change(c):
        p, s = slot(c, 0, int(c.seq_lens[0]) - 1)
        c.kh[p, 0, s] = (NAN if value == "nan" else INF)[kv]
    want, want_lse = run(lib, batch, kv, dim, 32)
    out, lse = run(lib, batch, kv, dim, 32, change)
    keep = np.ones(lse.shape, bool)
    keep[19, :4] = False
    assert np.array_equal(out[keep], want[keep]) and np.array_equal(lse[keep], want_lse[keep])
    assert np.isnan(lse[19, :4]).all() or value == "inf"


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("batch", list(BATCHES))
def test_a_value_stays_within_its_sequence_and_head(lib, batch, kv, dim):
    """NaN in a value: the rows that see it are NaN in that channel; lse, the other channels, heads and sequences are the same bits."""
    def change(c):
        p, s = slot(c, 0, 7)
        c.vh[p, 1, s, 11] = NAN[kv]
    want, want_lse = run(lib, batch, kv, dim, 33)
    out, lse = run(lib, batch, kv, dim, 33, change)
    assert np.isnan(out[:20, 4:, 11]).all()
    keep = np.ones(out.shape, bool)
    keep[:20, 4:, 11] = False
    assert np.array_equal(out[keep], want[keep]) and np.array_equal(lse, want_lse)
