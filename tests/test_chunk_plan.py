"""The chunk attention's planner (host code): every row and every cached token that a row sees is in exactly one item, the limits
that size the workspace hold, and what the entry points refuse without a GPU."""
import random

import numpy as np
import pytest


def check(lib, n_sm, hq, hkv, q_lens, seq_lens):
    plan = lib.libra_chunk_plan_host(n_sm, hq, hkv, q_lens, seq_lens)
    items, merges, G = plan["items"], plan["merges"], hq // hkv
    starts = np.concatenate([[0], np.cumsum(q_lens)])
    whole, cut = {}, {}
    for b, q_start, row0, n, kv0, kv1, ctx, slot in items.tolist():
        assert q_start == starts[b] and ctx == seq_lens[b] - q_lens[b] and 1 <= n <= 256 and row0 % 256 == 0
        assert kv0 % 128 == 0
        (cut if slot >= 0 else whole).setdefault((b, row0), []).append((kv0, kv1, n, slot))
    assert not set(whole) & set(cut)
    end = {}
    for b, (n, L) in enumerate(zip(q_lens, seq_lens)):
        rows = n * G
        for row0 in range(0, rows, 256):
            m = min(256, rows - row0)
            sees = max(0, L - n + (row0 + m - 1) // G + 1)
            assert sees <= L or L < n
            end[(b, row0)] = sees
            if (b, row0) in whole:
                assert whole[(b, row0)] == [(0, sees, m, -1)]
            else:
                parts = sorted(cut[(b, row0)])
                assert 2 <= len(parts) <= 64 and parts[0][0] == 0 and parts[-1][1] == sees
                assert all(a[1] == c[0] for a, c in zip(parts, parts[1:])) and all(p[2] == m for p in parts)
                assert all(p[0] < p[1] for p in parts)
    assert len(whole) + len(cut) == len(end)
    # merges name exactly the cut tiles; partial rows do not overlap
    used = []
    for q_start, row0, n, slot, chunks, *pad in merges.tolist():
        assert pad == [0, 0, 0]
        key = next(k for k in cut if starts[k[0]] == q_start and k[1] == row0 and q_lens[k[0]] > 0)
        assert sorted(p[3] for p in cut[key]) == [slot + j * n for j in range(chunks)] and len(cut[key]) == chunks
        assert [p[3] for p in sorted(cut[key])] == [slot + j * n for j in range(chunks)]     # chunk order
        used += [(slot + j * n, slot + (j + 1) * n) for j in range(chunks)]
    used.sort()
    assert all(a[1] <= c[0] for a, c in zip(used, used[1:])) and len(merges) == len(cut)
    assert plan["partial_rows"] == sum(e - s for s, e in used)
    assert plan["partial_rows"] * hkv <= 2 * n_sm * 256
    group_items = sum(q_lens) * G // 256 + min(len(q_lens), sum(q_lens)) + 4 * n_sm + 1
    assert len(items) <= group_items
    steps = [-(-(r[5] - r[4]) // 128) for r in items.tolist()]
    assert steps == sorted(steps, reverse=True)
    return plan


@pytest.mark.parametrize("hq,hkv", [(4, 1), (8, 8), (40, 8), (64, 8), (16, 1), (7, 1)])
def test_random_batches(lib, hq, hkv):
    rng = random.Random(hq * 100 + hkv)
    for _ in range(120):
        B = rng.choice([1, 1, 2, 3, 8, 40])
        q = [rng.choice([0, 1, 3, rng.randint(0, 600)]) for _ in range(B)]
        L = [max(0, n + rng.choice([0, 0, -2, 1, 127, 128, rng.randint(0, 40000)])) for n in q]
        check(lib, rng.choice([148, 1, 7]), hq, hkv, q, L)


def test_few_long_sequences_are_cut_and_many_are_not(lib):
    plan = check(lib, 148, 64, 8, [3] * 8, [32768] * 8)
    assert 8 * 8 < len(plan["items"]) * 8 <= 4 * 148 and len(plan["merges"]) == 8
    plan = check(lib, 148, 32, 8, [200] * 64, [4096] * 64)
    assert len(plan["merges"]) == 0
    assert len(check(lib, 148, 32, 8, [], [])["items"]) == 0
    assert len(check(lib, 148, 32, 8, [0, 0], [5, 0])["items"]) == 0


def test_refusals(lib):
    for args, status in [((0, 8, 2, [1], [1]), lib.INVALID_ARGUMENT), ((148, 8, 3, [1], [1]), lib.INVALID_ARGUMENT),
                         ((148, 8, 2, [-1], [1]), lib.INVALID_ARGUMENT), ((148, 8, 2, [1], [-1]), lib.INVALID_ARGUMENT),
                         ((148, 16, 1, [2 ** 28], [2 ** 30]), lib.UNSUPPORTED_SHAPE)]:
        with pytest.raises(lib.LibraError) as e:
            lib.libra_chunk_plan_host(*args)
        assert e.value.status == status, args
    L = lib.lib
    assert L.libra_chunk_workspace_size(None, 1, None) == lib.INVALID_ARGUMENT
    assert L.libra_chunk_plan(None, None, None, 0, None, 0, None) == lib.INVALID_ARGUMENT
    assert L.libra_chunk_attn(None, None, 0, None, None, None, None, None, None, None) == lib.INVALID_ARGUMENT
