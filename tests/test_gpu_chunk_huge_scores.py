"""Chunk attention with scores so large that their product with the scale is rounded by whole units: the key that outweighs all
others takes everything, and a row that does not see it is as it would be without."""
import numpy as np
import pytest

from oracle import attention_oracle as O

from test_gpu_chunk import Case
from test_gpu_chunk_row_scale import case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [1.0, 2.0 ** 100])
@pytest.mark.parametrize("k_scale", [1.0, 0.001])
@pytest.mark.parametrize("dim", [64, 128])
def test_one_dominant_key_and_huge_rows(lib, dim, k_scale, size):
    """q = size * 64 in channel 0, one key with 448 codes there: rows that see it (its score is 3.5 or more above the others',
    whose softmax weights are compared with the oracle; at 2^100 nothing else counts) and rows before it."""
    for at in (0, 127, 128, 281, 299):
        q = np.zeros((161, 8, dim), np.float32)
        q[..., 0] = 64.0 * size
        c = case(lib, "whole", (k_scale, 1.7), dim, q, seed=27)
        live = [(c.bt[0, t // 16], t % 16) for t in range(300)]
        for p, s in live:
            c.kh[p, :, s] = 0
        c.kh[live[at][0], :, live[at][1], 0] = 0x7E
        c.k.copy_(c.torch.from_numpy(c.kh))
        c.plan(); c.attn()
        assert int(c.err) == 0
        (ref, lse, spread), (_, _, vt) = c.reference()
        got = O.bf16_bits_to_f64(c.out.cpu().numpy().view(np.uint16))[:20]
        # scores: 0, exactly, and one of at most 24 bits times 2^-21
        e = spread[:20] * (2.0 ** -11 + 2.0 ** -20 + 2 * 2.0 ** -21 * (1 + min(size * 64 * 448 * k_scale, 64))) + 300 * 2.0 ** -25 * np.abs(vt[0]).max()
        assert np.all(np.abs(got - ref[:20]) <= e + 2.0 ** -8 * (np.abs(ref[:20]) + e))
        gl = c.lse.double().cpu().numpy()[:20]
        assert np.all(np.abs(gl - lse[:20]) <= 2.0 ** -20 * (1 + np.abs(lse[:20])))
        c.h.close()


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("power", [10, 12, 14, 16, 20, 40, 60])
@pytest.mark.parametrize("q_lens,seq_lens", [([20, 140], [300, 200]), ([20, 3], [3000, 2500])])
@pytest.mark.parametrize("dim", [64, 128])
def test_one_dominant_key_over_bf16_pools(lib, dim, q_lens, seq_lens, power, sign):
    """Scores of +-2^(2 power) * 1.7 * 1.3 / sqrt(dim), exactly, and 0.  Negative: the key weighs nothing, but for a row that
    sees no other."""
    for at in (0, 128, seq_lens[0] - 18, seq_lens[0] - 1):
        n = sum(q_lens)
        q = np.zeros((n, 2, dim), np.float32)
        q[..., 5] = 1.7 * 2.0 ** power
        k = [np.zeros((1, L, dim), np.float32) for L in seq_lens]
        k[0][0, at, 5] = 1.3 * 2.0 ** power * sign
        c = Case(lib, q_lens, seq_lens, 2, 1, dim, q_values=q, k_values=k, seed=28)
        c.plan(); c.attn()
        assert int(c.err) == 0
        (ref, lse, spread), _ = c.reference()
        got, gl = O.bf16_bits_to_f64(c.out.cpu().numpy().view(np.uint16)), c.lse.double().cpu().numpy()
        # all weights but those of equal scores are below 2^-1000 or equal: rounded to 16 bits, one rounding of the result
        e = spread * (2.0 ** -8 + 2.0 ** -18)
        assert np.all(np.abs(got - ref) <= e + 2.0 ** -8 * (np.abs(ref) + e))
        assert np.all(np.abs(gl - lse) <= 2.0 ** -20 * (1 + np.abs(lse)))
        c.h.close()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("dim", [64, 128])
def test_huge_scores_of_either_sign(lib, dim, kv):
    """Random q and k of 2^20 (bf16) or q of 2^60 (E4M3): each row returns a value that its sequence holds, or a mean of equals."""
    q_lens, seq_lens = [20, 140], [300, 200]
    rng = np.random.default_rng(29)
    q = (rng.standard_normal((160, 2, dim)) * (2.0 ** 20 if kv == "bf16" else 2.0 ** 60)).astype(np.float32)
    k = [(rng.standard_normal((1, L, dim)) * 2.0 ** 20).astype(np.float32) for L in seq_lens] if kv == "bf16" else None
    c = Case(lib, q_lens, seq_lens, 2, 1, dim, kv=kv, q_values=q, k_values=k, seed=30)
    c.plan(); c.attn()
    assert int(c.err) == 0
    (_, lse, _), (qs, kt, vt) = c.reference()
    got, gl = O.bf16_bits_to_f64(c.out.cpu().numpy().view(np.uint16)), c.lse.double().cpu().numpy()
    r = 0
    for b, n in enumerate(q_lens):
        most = np.abs(vt[b]).max()
        assert np.all(np.abs(got[r:r + n]) <= most * (1 + 2.0 ** -7))
        size = np.einsum("nhd,td->nht", np.abs(qs[r:r + n]), np.abs(kt[b][0])).max(-1) / np.sqrt(dim)
        assert np.all(np.abs(gl[r:r + n] - lse[r:r + n]) <= (dim * 2.0 ** -23 + dim * 2.0 ** -35 * 2.0 ** 10) * size)
        # where the largest score leads by more than both sides' rounding, its value comes back
        s = np.einsum("nhd,td->nht", qs[r:r + n], kt[b][0]) / np.sqrt(dim)
        for i in range(n):
            seen = seq_lens[b] - n + i + 1
            for h in range(2):
                two = np.sort(s[i, h, :seen])[-2:]
                if two[1] - two[0] > (dim * 2.0 ** -22 + dim * 2.0 ** -24) * size[i, h] + 30:
                    v = vt[b][0, int(np.argmax(s[i, h, :seen]))]
                    assert np.all(np.abs(got[r + i, h] - v) <= 2.0 ** -7 * np.abs(v) + 2.0 ** -20 * most)
        r += n
    c.h.close()
