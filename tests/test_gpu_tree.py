"""Trees of drafted tokens on the GPU: masks and positions against a walk on the host, attention against the float64 oracle within
the tolerance that test_gpu_chunk.py derives (the mask changes which tokens are summed over, nothing else), kept rows bit for bit,
and the whole step."""
import math

import numpy as np
import pytest

from oracle import attention_oracle as O
from oracle import chunk_oracle as K
from paper_2606_03077_b200 import workloads as W

from test_gpu_chunk import BATCHES, Case
from test_gpu_norm_rope import EPS, f64, forward, rounded
from test_rope import rope_of

pytestmark = pytest.mark.gpu

CANARY = -77


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def up(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def draw_parents(rng, n, kind):
    if kind == "chain":
        return [i - 1 for i in range(n)]
    if kind == "roots":
        return [-1] * n
    return [int(rng.integers(-1 if i < 3 else max(-1, i - 9), i)) for i in range(n)]


def ancestors(parents):
    """[n, n]: i sees j."""
    sees = np.zeros((len(parents),) * 2, bool)
    for i, p in enumerate(parents):
        if p >= 0:
            sees[i] = sees[p]
        sees[i, i] = True
    return sees


def words(sees, ld):
    bits = np.zeros((sees.shape[0], ld * 32), np.int64)
    bits[:, :sees.shape[1]] = sees
    return (bits.reshape(sees.shape[0], ld, 32) << np.arange(32)).sum(-1).astype(np.uint32).view(np.int32)


# ---------------------------------------------------------------------------------------------------------- mask
@pytest.mark.parametrize("kind", ["chain", "roots", "tree"])
@pytest.mark.parametrize("ld", [1, 2, 5, 32])
def test_mask(lib, ld, kind):
    import torch
    rng = np.random.default_rng(ld)
    lens = [0, 1, 2, 31, 32, 33, 0, 64, 100, 1024, 7]
    new = [n for n in lens if n <= 32 * ld]
    seq = [n + int(rng.integers(0, 50)) for n in new]
    seq[1] = 0 if new[1] else seq[1]   # a chunk longer than its sequence: positions below zero
    parents = [draw_parents(rng, n, kind) for n in new]
    rows = sum(new)
    h = lib.Handle(8, 2, 64, 4, len(new), 4)
    mask = torch.full((rows + 3, ld), CANARY, dtype=torch.int32, device="cuda")
    pos, err = torch.full((rows + 3,), CANARY, dtype=torch.int32, device="cuda"), up([0])
    off, dl, dp = up(np.concatenate([[0], np.cumsum(new)])), up(seq), up(sum(parents, []) + [0])
    for want_pos in (True, False):
        h.tree_mask(dp.data_ptr(), off.data_ptr(), dl.data_ptr(), len(new), rows, mask.data_ptr(), ld, pos.data_ptr() if want_pos else 0,
                    err.data_ptr(), stream())
        got, at = mask.cpu().numpy(), 0
        for n, L, p in zip(new, seq, parents):
            sees = ancestors(p)
            assert np.array_equal(got[at:at + n], words(sees, ld))
            if want_pos:
                assert np.array_equal(pos.cpu().numpy()[at:at + n], L - n + sees.sum(1) - 1)
            at += n
        assert np.all(got[rows:] == CANARY) and np.all(pos.cpu().numpy()[rows:] == CANARY) and int(err) == 0
        mask.fill_(CANARY); pos.fill_(CANARY)
    assert np.all(pos.cpu().numpy() == CANARY)
    h.close()


def test_mask_flagged(lib):
    """Parents that do not stand before their child count as -1; sequences that do not fit stay unwritten, the others are written."""
    import torch
    h = lib.Handle(8, 2, 64, 4, 4, 4)

    def call(parents, off, max_rows, ld=1):
        mask = torch.full((max(off) + 1, ld), CANARY, dtype=torch.int32, device="cuda")
        err, dp, do, dl = up([0]), up(parents), up(off), up([100] * (len(off) - 1))
        h.tree_mask(dp.data_ptr(), do.data_ptr(), dl.data_ptr(), len(off) - 1, max_rows, mask.data_ptr(), ld, 0, err.data_ptr(), stream())
        return mask.cpu().numpy(), int(err)

    got, err = call([-1, 0, 2, -2, 9, 3, -1], [0, 6, 7], 7)
    assert err == lib.ERR_BAD_TREE
    assert np.array_equal(got[:7], np.concatenate([words(ancestors([-1, 0, -1, -1, -1, 3]), 1), words(ancestors([-1]), 1)]))
    got, err = call([-1] * 50, [0, 3, 45, 50], 50)
    assert err == lib.ERR_PLAN_OVERFLOW and np.all(got[3:45] == CANARY) and np.all(got[:3] != CANARY) and np.all(got[45:50] != CANARY)
    got, err = call([-1] * 9, [0, 5, 9], 8)
    assert err == lib.ERR_PLAN_OVERFLOW and np.all(got[5:] == CANARY) and np.all(got[:5] != CANARY)
    got, err = call([-1] * 9, [0, 5, 3, 9], 9)
    assert err == lib.ERR_BAD_LENGTH and np.all(got[:5] != CANARY)
    h.close()


# ----------------------------------------------------------------------------------------------------- attention
class TreeCase(Case):
    """A chunk case whose new tokens see what `sees[b]` ([n, n]) says."""

    def __init__(self, lib, q_lens, seq_lens, *args, kind="tree", sees=None, extra_words=0, **kw):
        super().__init__(lib, q_lens, seq_lens, *args, **kw)
        rng = np.random.default_rng(kw.get("seed", 0) + 77)
        self.sees = sees or [ancestors(draw_parents(rng, n, kind)) if kind != "any" else rng.random((n, n)) < 0.4 for n in q_lens]
        self.ld = max(1, -(-int(max(q_lens)) // 32)) + extra_words
        m = [words(s, self.ld) for s in self.sees if len(s)]
        self.mask = up(np.concatenate(m) if m else np.zeros((1, self.ld)))

    def attn(self, lse=True):
        self.h.tree_attn(self.q.data_ptr(), self.q.stride(0), self.k.data_ptr(), self.v.data_ptr(), self.dbt.data_ptr(), self.mask.data_ptr(),
                         self.ld, self.out.data_ptr(), self.lse.data_ptr() if lse else 0, self.err.data_ptr(), stream())

    def reference(self):
        q = O.bf16_bits_to_f64(self.qh)
        kt, vt = (K.sequence_tokens(x, self.bt, self.seq_lens, "HND", s) for x, s in zip((self.kh, self.vh), self.scales))
        rows, Hq, d = q.shape
        scale = self.sm_scale or 1 / math.sqrt(d)
        out, spread, lse = np.zeros((rows, Hq, d)), np.zeros((rows, Hq, d)), np.full((rows, Hq), -np.inf)
        r = 0
        for b, (n, L) in enumerate(zip(self.q_lens, self.seq_lens)):
            place = np.arange(L) - (L - n)
            for i in range(n):
                seen = (place < 0) | ((place <= i) & self.sees[b][i][np.clip(place, 0, n - 1)])
                if seen.any():
                    Kb, Vb = kt[b][:, seen], vt[b][:, seen]
                    s = np.einsum("hgd,htd->hgt", q[r].reshape(self.hkv, -1, d), Kb) * scale
                    m = s.max(-1, keepdims=True)
                    p = np.exp(s - m)
                    z = p.sum(-1, keepdims=True)
                    out[r] = np.einsum("hgt,htd->hgd", p / z, Vb).reshape(Hq, d)
                    spread[r] = np.einsum("hgt,htd->hgd", p / z, np.abs(Vb)).reshape(Hq, d)
                    lse[r] = (m + np.log(z))[..., 0].reshape(Hq)
                r += 1
        return (out, lse, spread), (q, kt, vt)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("batch", list(BATCHES))
@pytest.mark.parametrize("hq,hkv,dim,page,order,kind", [(4, 1, 64, 16, "HND", "tree"), (8, 2, 128, 16, "HND", "any"), (10, 2, 128, 32, "NHD", "tree"),
                                                        (16, 1, 64, 64, "NHD", "any"), (7, 1, 128, 16, "NHD", "roots")])
def test_attention(lib, hq, hkv, dim, page, order, kind, batch, kv):
    q, L = BATCHES[batch]
    TreeCase(lib, q, L, hq, hkv, dim, page, order, kv, seed=hq + dim, gap=8 if page == 32 else 0, kind=kind, extra_words=page == 64).run()


@pytest.mark.parametrize("ctx", [0, 1, 31, 32, 96, 127, 128, 129, 250])
def test_attention_where_the_tree_crosses_steps(lib, ctx):
    """Trees that begin at every kind of place within the 128-token steps and within the mask's words."""
    TreeCase(lib, [5, 70, 150], [ctx + 5, ctx + 70, ctx + 150], 4, 2, 64, seed=ctx, kind="any").run()


def test_rows_that_see_nothing(lib):
    """No cached token and no bit: zeros and -inf, whatever the neighbours see; the mask's bits behind a token count for nothing."""
    n = 140
    sees = np.zeros((n, n), bool)
    sees[3, 3] = sees[130, 0] = True
    sees[60, 61:] = True
    for L in (n, n - 9):
        c = TreeCase(lib, [n, 2], [L, 300], 4, 1, 64, sees=[sees, np.zeros((2, 2), bool)], seed=L)
        c.plan(); c.attn()
        lse = c.lse.cpu().numpy()
        assert np.all(np.isneginf(lse[60])) and np.all(c.out[60].cpu().numpy() == 0)
        assert np.isfinite(lse[130]).all() == (L == n)
        c.check(); c.h.close()


def test_cut_ranges_that_hold_nothing_for_a_row(lib):
    """A tree of 700 tokens and nothing cached, its range cut: rows that see nothing in some of the parts, and in none."""
    rng = np.random.default_rng(11)
    n = 700
    sees = rng.random((n, n)) < 0.004
    sees[::7] = False
    assert len(lib.libra_chunk_plan_host(148, 4, 1, [n], [n])["merges"]) > 0
    for dim in (64, 128):
        c = TreeCase(lib, [n], [n], 4, 1, dim, sees=[sees], seed=dim)
        c.run()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_chain_is_a_chunk(lib, dim, kv):
    """The mask of a chain gives the bits of libra_chunk_attn, cut ranges included."""
    import torch
    c = TreeCase(lib, [3, 40, 200, 1], [3000, 60, 200, 2500], 8, 2, dim, kv=kv, kind="chain", seed=8)
    assert len(lib.libra_chunk_plan_host(148, 8, 2, c.q_lens, c.seq_lens)["merges"]) > 0
    c.plan(); c.attn()
    out, lse = c.out.clone(), c.lse.clone()
    c.out.fill_(0x7FC0); c.lse.fill_(float("nan"))
    Case.attn(c)
    assert torch.equal(c.out, out) and torch.equal(c.lse, lse) and int(c.err) == 0
    c.h.close()


def test_keys_of_others_never_count(lib):
    """K of tokens outside a row's path holds NaN and infinities."""
    n, L, dim = 30, 200, 64
    rng = np.random.default_rng(0)
    k = rng.standard_normal((1, L, dim)).astype(np.float32)
    sees = ancestors(draw_parents(rng, n, "tree"))
    unseen = [j for j in range(n) if not sees[n - 1][j]]
    k[0, [L - n + j for j in unseen[::2]]] = np.nan
    k[0, [L - n + j for j in unseen[1::2]]] = np.inf
    c = TreeCase(lib, [n], [L], 4, 1, dim, sees=[sees], k_values=[k])
    clean = np.nan_to_num(k, nan=0.0, posinf=0.0)
    d = TreeCase(lib, [n], [L], 4, 1, dim, sees=[sees], k_values=[clean])
    for x in (c, d):
        x.plan(); x.attn()
    assert np.array_equal(c.out[n - 1].cpu().numpy(), d.out[n - 1].cpu().numpy())
    d.check()
    c.h.close(); d.h.close()


def test_long_cache_same_bits_recorded(lib):
    import torch
    c = TreeCase(lib, [16, 60, 33], [9000, 20001, 5000], 16, 2, 128, seed=5)
    c.plan(); c.attn()
    torch.cuda.synchronize()
    assert int(c.err) == 0
    c.check()
    first, lse = c.out.clone(), c.lse.clone()
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        c.attn()
    for _ in range(5):
        c.out.fill_(0x7FC0); c.lse.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, first) and torch.equal(c.lse, lse)
    c.plan()              # another plan in the workspace: the recording says so and computes nothing
    c.out.fill_(0x7FC0)
    g.replay()
    torch.cuda.synchronize()
    assert int(c.err) == lib.ERR_PLAN_CHANGED and bool((c.out == 0x7FC0).all())
    del g
    c.h.close()


def test_attention_refused(lib):
    c = TreeCase(lib, [40, 3], [50, 60], 4, 1, 64)
    p = lambda x: x.data_ptr()
    good = [p(c.q), c.q.stride(0), p(c.k), p(c.v), p(c.dbt), p(c.mask), 2, p(c.out), 0, p(c.err), 0]
    with pytest.raises(lib.LibraError) as e:
        c.h.tree_attn(*good)
    assert e.value.status == lib.NOT_PLANNED
    c.plan()
    for i, bad in [(5, 0), (5, p(c.mask) + 2), (6, 0), (6, -1), (6, 1), (0, 0), (1, 255), (1, 260), (7, 0), (9, 0)]:
        args = list(good)
        args[i] = bad
        with pytest.raises(lib.LibraError) as e:
            c.h.tree_attn(*args)
        assert e.value.status == lib.INVALID_ARGUMENT, i
    c.h.close()


# ---------------------------------------------------------------------------------------------------------- keep
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("hkv,dim,page,order", [(1, 64, 16, "HND"), (2, 128, 32, "NHD"), (40, 128, 64, "HND"), (8, 128, 16, "NHD")])
def test_keep(lib, hkv, dim, page, order, kv):
    import torch
    rng = np.random.default_rng(hkv + page)
    new = [5, 0, 33, 150, 1, 64, 20, 70]
    ctx = [0, 40, 15, 100, 7, 64, 300, 1]
    seq = np.add(new, ctx)
    kept = [sorted(rng.choice(n, int(rng.integers(0, n + 1)), replace=False)) if n else [] for n in new]
    kept[3], kept[4], kept[5], kept[7] = list(range(1, 150)), [0], list(range(64)), [69]
    pages = [-(-int(L) // page) for L in seq]
    pool, ld = sum(pages) + 2, max(pages)
    ids = rng.permutation(pool)
    bt, at = np.full((len(new), ld), -1, np.int32), 0
    for b, n in enumerate(pages):
        bt[b, :n] = ids[at:at + n]
        at += n
    shape = (pool, hkv, page, dim) if order == "HND" else (pool, page, hkv, dim)
    top, kind = (1 << 15, np.int16) if kv == "bf16" else (256, np.uint8)
    pools = [torch.from_numpy(rng.integers(0, top, shape).astype(kind)).cuda() for _ in range(2)]
    want = [x.cpu().numpy().copy() for x in pools]
    ld_kept = max(len(x) for x in kept) + 3
    table = np.full((len(new), ld_kept), 10 ** 6, np.int32)
    for b, x in enumerate(kept):
        table[b, :len(x)] = x
        for y in want:
            z = y if order == "NHD" else y.transpose(0, 2, 1, 3)
            rows = [z[bt[b, (ctx[b] + j) // page], (ctx[b] + j) % page].copy() for j in x]
            for i, row in enumerate(rows):
                z[bt[b, (ctx[b] + i) // page], (ctx[b] + i) % page] = row
    strides = (0, 0, 0) if order == "HND" else (page * hkv * dim, dim, hkv * dim)
    h = lib.Handle(hkv, hkv, dim, pool, len(new), ld, page_size=page, kv_strides=strides)
    if kv == "e4m3":
        h.set_kv_dtype(lib.KV_E4M3, 0.5, 0.25)
    dev = [up(table), up([len(x) for x in kept]), up(np.concatenate([[0], np.cumsum(new)])), up(seq), up(bt), up([CANARY] * len(new)), up([0])]
    p = lambda i: dev[i].data_ptr()
    h.tree_keep(p(0), ld_kept, p(1), p(2), p(3), p(4), len(new), pools[0].data_ptr(), pools[1].data_ptr(), p(5), p(6), stream())
    assert int(dev[6]) == 0 and dev[5].cpu().tolist() == [c + len(x) for c, x in zip(ctx, kept)]
    assert all(np.array_equal(x.cpu().numpy(), y) for x, y in zip(pools, want))
    before = [x.clone() for x in pools]
    h.tree_keep(p(0), ld_kept, up([0] * len(new)).data_ptr(), p(2), p(3), p(4), len(new), pools[0].data_ptr(), pools[1].data_ptr(), 0, p(6), stream())
    assert all(torch.equal(x, y) for x, y in zip(pools, before)) and int(dev[6]) == 0
    h.close()


def test_keep_flagged(lib):
    """A sequence whose numbers cannot be stays as it is, with its length; the others move."""
    import torch
    h = lib.Handle(2, 2, 64, 40, 8, 4)

    def call(kept, n_kept, off, lens, bt):
        k, v = (torch.arange(40 * 2 * 16 * 64, device="cuda").to(torch.int16).reshape(40, 2, 16, 64).clone() for _ in range(2))
        k0 = k.clone()
        new_lens, err = up([CANARY] * len(lens)), up([0])
        d = [up(x) for x in (kept, n_kept, off, lens, bt)]
        h.tree_keep(d[0].data_ptr(), len(kept[0]), d[1].data_ptr(), d[2].data_ptr(), d[3].data_ptr(), d[4].data_ptr(), len(lens), k.data_ptr(),
                    v.data_ptr(), new_lens.data_ptr(), err.data_ptr(), stream())
        assert torch.equal(k, v)
        return int(err), new_lens.cpu().tolist(), sorted(set((k != k0).any(-1).any(1).nonzero()[:, 0].tolist()))

    bt = [[0, 1, 2, 3], [4, 5, 6, 7]]
    good = [1, 3, 0]
    for bad, n in (([3, 1, 0], 2), ([1, 1, 0], 2), ([-1, 2, 0], 2), ([2, 5, 0], 2), ([0, 1, 2], 4), ([0, 1, 2], -1)):
        assert call([bad, good], [n, 2], [0, 5, 10], [25, 25], bt) == (lib.ERR_BAD_TREE, [25, 22], [5])
    assert call([good, good], [2, 2], [0, 5, 10], [3, 25], bt) == (lib.ERR_BAD_LENGTH, [3, 22], [5])
    assert call([good, good], [2, 2], [0, 5, 10], [65, 25], bt) == (lib.ERR_PLAN_OVERFLOW, [65, 22], [5])
    assert call([good, good], [2, 2], [0, 5, 10], [25, 25], [[0, 40, 2, 3], bt[1]]) == (lib.ERR_BAD_PAGE_ID, [22, 22], [5])
    one = up([0]).data_ptr()
    good = [one, 1, one, one, one, one, 1, one & ~15, one & ~15, 0, one, 0]
    for i, bad in [(0, 0), (1, 0), (2, 0), (3, 0), (4, 0), (5, 0), (6, -1), (6, 9), (7, 0), (8, (one & ~15) + 8), (9, one), (10, 0)]:
        args = list(good)
        args[i] = bad
        assert lib.lib.libra_tree_keep(h._h, *[x or None if j not in (1, 6) else x for j, x in enumerate(args)]) == lib.INVALID_ARGUMENT, i
    for args in ((one, one, one, 1, 1, one, 0, 0, one), (one, one, one, 1, 1, one, -1, 0, one), (one, one, one, 9, 1, one, 1, 0, one),
                 (one, one, one, 1, -1, one, 1, 0, one), (one + 1, one, one, 1, 1, one, 1, 0, one)):
        assert lib.lib.libra_tree_mask(h._h, *args, None) == lib.INVALID_ARGUMENT
    assert lib.lib.libra_tree_mask(h._h, one, one, one, 1, 1, one, 33, 0, one, None) == lib.UNSUPPORTED_SHAPE
    h.close()


# ---------------------------------------------------------------------------------------------------- a whole step
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_drafted_steps_together(lib, kv):
    """Steps as a server makes them: pages, tree, append, attention, accepted rows, pages back; then one decode step on what is left.
    Attention is checked on the pools as they were written, the pools against the norm and rotation of what went in."""
    import torch
    rng = np.random.default_rng(3)
    B, hq, hkv, dim, page, ld, pool = 5, 8, 2, 128, 16, 20, 60
    h = lib.Handle(hq, hkv, dim, pool, B, ld, page_size=page)
    scales = (None, None)
    if kv == "e4m3":
        scales = (0.03125, 0.0625)
        h.set_kv_dtype(lib.KV_E4M3, *scales)
    kind = torch.bfloat16 if kv == "bf16" else torch.uint8
    k, v = (torch.full((pool, hkv, page, dim), float("nan") if kv == "bf16" else 0x7F, dtype=kind, device="cuda") for _ in range(2))
    bt, lens, free, count = up(np.full((B, ld), -1)), up([0] * B), up(rng.permutation(pool)), up([pool])
    off, err = up([0] * (B + 1)), up([0])
    rope, turns = rope_of(lib, dim), K.rope_turns(dim, 10000.0)
    wq, wk = (torch.from_numpy(1 + 0.25 * rng.standard_normal(dim)).to(torch.bfloat16).cuda() for _ in range(2))
    model = [[] for _ in range(B)]          # (position, normalised and rotated k with its bound, v) of every cached token
    for step in range(4):
        new = [int(x) for x in rng.integers(1, 60 if step == 0 else 25, B)]
        if step == 2:
            new[1] = 0
        had = [len(m) for m in model]
        parents = [draw_parents(rng, n, "chain" if step == 0 else "tree") for n in new]
        rows, words_ld = sum(new), 2
        proj = torch.from_numpy(rng.standard_normal((rows, hq + 2 * hkv, dim))).to(torch.bfloat16).cuda()
        pos, slots = (torch.empty(rows, dtype=torch.int32, device="cuda") for _ in range(2))
        mask = torch.empty((rows, words_ld), dtype=torch.int32, device="cuda")
        q_rot, out = (torch.empty((rows, hq, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        dn, dp = up(new), up(sum(parents, []))
        st = stream()
        h.cache_extend(dn.data_ptr(), lens.data_ptr(), bt.data_ptr(), B, free.data_ptr(), count.data_ptr(), off.data_ptr(), 0, slots.data_ptr(), rows,
                       err.data_ptr(), st)
        h.tree_mask(dp.data_ptr(), off.data_ptr(), lens.data_ptr(), B, rows, mask.data_ptr(), words_ld, pos.data_ptr(), err.data_ptr(), st)
        q, kn, vn = proj[:, :hq], proj[:, hq:hq + hkv], proj[:, hq + hkv:]
        h.norm_rope_append(rope, wq.data_ptr(), wk.data_ptr(), EPS, q.data_ptr(), q.stride(0), q_rot.data_ptr(), q_rot.stride(0), kn.data_ptr(),
                           vn.data_ptr(), kn.stride(0), pos.data_ptr(), slots.data_ptr(), off.data_ptr() + 4 * B, rows, k.data_ptr(), v.data_ptr(),
                           err.data_ptr(), st)
        seq = [a + n for a, n in zip(had, new)]
        ws = torch.empty(h.chunk_workspace_size(rows), dtype=torch.uint8, device="cuda")
        h.chunk_plan(np.array(new, np.int32), np.array(seq, np.int32), ws.data_ptr(), ws.numel(), st)
        h.tree_attn(q_rot.data_ptr(), q_rot.stride(0), k.data_ptr(), v.data_ptr(), bt.data_ptr(), mask.data_ptr(), words_ld, out.data_ptr(), 0,
                    err.data_ptr(), st)
        torch.cuda.synchronize()
        assert int(err) == 0 and lens.cpu().tolist() == seq
        table = bt.cpu().numpy()
        kh, vh = (x.view(torch.int16).cpu().numpy().view(np.uint16) if kv == "bf16" else x.cpu().numpy() for x in (k, v))
        kt, vt = (K.sequence_tokens(x, table, seq, "HND", s) for x, s in zip((kh, vh), scales))
        sees = [ancestors(p) for p in parents]
        positions = np.concatenate([a + s.sum(1) - 1 for a, s in zip(had, sees)])
        ky, ke = forward(f64(kn), f64(wk), K.rope_angles(positions, turns), K.HALF, 1.0, float(np.float32(EPS)))
        qy, qe = forward(f64(q), f64(wq), K.rope_angles(positions, turns), K.HALF, 1.0, float(np.float32(EPS)))
        assert np.all(np.abs(f64(q_rot) - qy) <= rounded(qy, qe, "bf16"))
        r = 0
        for b in range(B):
            for i in range(new[b]):
                model[b].append((ky[r], ke[r], f64(vn[r:r + 1])[0]))
                r += 1
            for t, (y, e, x) in enumerate(model[b]):
                # half a step of the type: bf16 2^-8; E4M3 2^-4, below its normal numbers half of 2^-9 times the scale
                half, tiny = (2.0 ** -8, 2.0 ** -134) if kv == "bf16" else (2.0 ** -4 + 2.0 ** -21, 0.0)
                ks, vs = (0.0, 0.0) if kv == "bf16" else (2.0 ** -10 * scales[0], 2.0 ** -10 * scales[1])
                assert np.all(np.abs(kt[b][:, t] - y) <= e + half * (np.abs(y) + e) + tiny + ks), (step, b, t)
                assert np.all(np.abs(vt[b][:, t] - x) <= (0.0 if kv == "bf16" else half * np.abs(x) + vs))
        # the attention, from the pools as they are
        got, r = f64(out), 0
        for b in range(B):
            L, n = seq[b], new[b]
            for i in range(n):
                seen = np.concatenate([np.ones(L - n, bool), sees[b][i]])
                s = np.einsum("hgd,htd->hgt", f64(q_rot[r]).reshape(hkv, -1, dim), kt[b][:, seen]) / math.sqrt(dim)
                p = np.exp(s - s.max(-1, keepdims=True))
                p /= p.sum(-1, keepdims=True)
                ref, spread = (np.einsum("hgt,htd->hgd", p, x[:, seen]).reshape(hq, dim) for x in (vt[b], np.abs(vt[b])))
                # |q . k| over channels is below 2^9 here, times dim 2^-23 and the scale: below 2^-10 of a score, twice that of a weight
                e = spread * (2.0 ** -8 + 2.0 ** -9)
                assert np.all(np.abs(got[r] - ref) <= e + 2.0 ** -8 * (np.abs(ref) + e) + L * 2.0 ** -25 * np.abs(vt[b]).max()), (step, b, i)
                r += 1
        # accept a path (the whole prompt at first), move its rows together, give the pages back
        kept, at = [], 0
        for p in parents:
            i, path = (len(p) - 1 if step == 0 else int(rng.integers(-1, len(p)))) if p else -1, []
            while i >= 0:
                path.append(i)
                i = p[i]
            kept.append(path[::-1])
        table_kept = np.zeros((B, 64), np.int32)
        for b, path in enumerate(kept):
            table_kept[b, :len(path)] = path
        dk, dn2, new_lens = up(table_kept), up([len(x) for x in kept]), up([0] * B)
        h.tree_keep(dk.data_ptr(), 64, dn2.data_ptr(), off.data_ptr(), lens.data_ptr(), bt.data_ptr(), B, k.data_ptr(), v.data_ptr(), new_lens.data_ptr(),
                    err.data_ptr(), st)
        h.cache_trim(new_lens.data_ptr(), lens.data_ptr(), bt.data_ptr(), B, free.data_ptr(), count.data_ptr(), err.data_ptr(), st)
        torch.cuda.synchronize()
        model = [m[:a] + [m[a + j] for j in path] for m, a, path in zip(model, had, kept)]
        assert int(err) == 0 and lens.cpu().tolist() == [len(m) for m in model]
        assert int(count) == pool - sum(-(-len(m) // page) for m in model)
    # a decode step over what was kept reads the same rows
    seq = np.array([len(m) for m in model], np.int32)
    ws = torch.empty(h.workspace_size(), dtype=torch.uint8, device="cuda")
    q1, out = (torch.randn((B, hq, dim), device="cuda").to(torch.bfloat16) for _ in range(2))
    h.plan(seq, ws.data_ptr(), ws.numel(), stream())
    h.decode_attn(q1.data_ptr(), k.data_ptr(), v.data_ptr(), bt.data_ptr(), lens.data_ptr(), out.data_ptr(), stream())
    torch.cuda.synchronize()
    assert h.debug_error_word() == 0
    kh, vh = (x.view(torch.int16).cpu().numpy().view(np.uint16) if kv == "bf16" else x.cpu().numpy() for x in (k, v))
    kt, vt = (K.sequence_tokens(x, bt.cpu().numpy(), seq, "HND", s) for x, s in zip((kh, vh), scales))
    for b in range(B):
        for t, (y, e, x) in enumerate(model[b]):
            half = 2.0 ** -8 if kv == "bf16" else 2.0 ** -4 + 2.0 ** -21
            ks = 2.0 ** -134 if kv == "bf16" else 2.0 ** -10 * scales[0]
            assert np.all(np.abs(kt[b][:, t] - y) <= e + half * (np.abs(y) + e) + ks)
        s = np.einsum("hgd,htd->hgt", f64(q1[b]).reshape(hkv, -1, dim), kt[b]) / math.sqrt(dim)
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        ref = np.einsum("hgt,htd->hgd", p, vt[b]).reshape(hq, dim)
        assert np.all(np.abs(f64(out[b]) - ref) <= 1e-2 + 1e-2 * np.abs(ref))
    h.close()
