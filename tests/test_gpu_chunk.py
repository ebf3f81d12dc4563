"""Causal attention of packed chunks over the pages, on the GPU against the float64 oracle.

Tolerance.  A score is a sum of d exact products accumulated in fp32 (taken as truncating): off by at most
e_s = d * 2^-23 * max (|q| . |k|) * scale, which is also the relative error of a probability, to which the exponential adds
2^-21.  Probabilities are rounded to 16 bits: h = 2^-8 relative (bf16 pools) or 2^-11 (E4M3 pools, fp16), the latter with steps of
2^-24 below 2^-14 where the largest probability is at least 1: n * 2^-25 * max |v| for a row that sees n tokens.  Their sum is
not rounded.  With spread = sum_t p_t |v_t|:
    |out - ref| <= spread * (h + 2 (e_s + 2^-21) + 2^-20) + [fp16] n 2^-25 max |v|,  then half a bf16 step, 2^-8 of the value.
lse: e_s + 2^-20 (1 + |lse|).
"""
import math

import numpy as np
import pytest

from oracle import attention_oracle as O
from oracle import chunk_oracle as K
from paper_2606_03077_b200 import workloads as W

from test_gpu_rope import bound as rope_bound

pytestmark = pytest.mark.gpu


class Case:
    """Host inputs, their copies on the device and a handle."""

    def __init__(self, lib, q_lens, seq_lens, hq=4, hkv=1, dim=64, page=16, order="HND", kv="bf16", seed=0, sm_scale=0.0, gap=0,
                 q_values=None, k_values=None, max_batch=None):
        import torch
        self.torch, self.lib = torch, lib
        self.q_lens, self.seq_lens = np.asarray(q_lens, np.int32), np.asarray(seq_lens, np.int32)
        self.hq, self.hkv, self.dim, self.page, self.order, self.kv, self.sm_scale = hq, hkv, dim, page, order, kv, sm_scale
        B, rng = len(q_lens), np.random.default_rng(seed)
        if kv == "bf16":
            _, self.bt, _, k, v = W.random_case(seed, B, hq, hkv, dim, self.seq_lens, page_size=page)
            if k_values is not None:
                k = self._put(k, k_values)
            dead = k == W.f32_to_bf16_bits(np.array([W.POISON_F32]))[0]
            k[dead], v[dead] = 0x7FC0, 0xFFC0            # NaN where no token lives
            self.scales = (None, None)
        else:
            _, self.bt, _, k, v = W.random_case_e4m3(seed, B, hq, hkv, dim, self.seq_lens, page_size=page)
            self.scales = (0.37, 1.7)
        self.kh, self.vh = k, v
        rows = int(self.q_lens.sum())
        self.qh = W.f32_to_bf16_bits(rng.standard_normal((rows, hq, dim), dtype=np.float32) if q_values is None else q_values)
        if order == "NHD":
            k, v = (np.ascontiguousarray(x.transpose(0, 2, 1, 3)) for x in (k, v))
        view = (lambda x: torch.from_numpy(x.view(np.int16)).cuda()) if kv == "bf16" else (lambda x: torch.from_numpy(x).cuda())
        self.k, self.v = view(k), view(v)
        wide = torch.full((max(rows, 1), hq * dim + gap), 0x7FC0, dtype=torch.int16, device="cuda")
        wide[:rows, :hq * dim] = torch.from_numpy(self.qh.view(np.int16)).cuda().view(rows, hq * dim)
        self.q = wide
        self.dbt = torch.from_numpy(self.bt).cuda()
        self.out = torch.full((max(rows, 1), hq, dim), 0x7FC0, dtype=torch.int16, device="cuda")
        self.lse = torch.full((max(rows, 1), hq), float("nan"), device="cuda")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        strides = (0, 0, 0) if order == "HND" else (page * hkv * dim, dim, hkv * dim)
        self.h = lib.Handle(hq, hkv, dim, k.shape[0], max_batch or max(B, 1), self.bt.shape[1], page_size=page, kv_strides=strides,
                            sm_scale=sm_scale)
        if kv == "e4m3":
            self.h.set_kv_dtype(lib.KV_E4M3, *self.scales)
        self.ws = torch.full((self.h.chunk_workspace_size(rows),), 0xEE, dtype=torch.uint8, device="cuda")
        self.rows = rows

    def _put(self, pages, values):
        """values[b]: float32 [Hkv, L, d] into the pages (HND)."""
        for b, x in enumerate(values):
            for t in range(x.shape[1]):
                pages[self.bt[b, t // self.page], :, t % self.page] = W.f32_to_bf16_bits(x[:, t])
        return pages

    def plan(self):
        self.h.chunk_plan(self.q_lens, self.seq_lens, self.ws.data_ptr(), self.ws.numel(), self.torch.cuda.current_stream().cuda_stream)

    def attn(self, lse=True):
        self.h.chunk_attn(self.q.data_ptr(), self.q.stride(0), self.k.data_ptr(), self.v.data_ptr(), self.dbt.data_ptr(),
                          self.out.data_ptr(), self.lse.data_ptr() if lse else 0, self.err.data_ptr(),
                          self.torch.cuda.current_stream().cuda_stream)

    def reference(self):
        q = O.bf16_bits_to_f64(self.qh)
        kt, vt = (K.sequence_tokens(x, self.bt, self.seq_lens, "HND", s) for x, s in zip((self.kh, self.vh), self.scales))
        return K.packed_chunk_attention(q, kt, vt, self.q_lens, self.seq_lens, self.sm_scale or None), (q, kt, vt)

    def check(self):
        """Every element of out and lse against the oracle, within the bound above."""
        (ref, lse, spread), (q, kt, vt) = self.reference()
        got = O.bf16_bits_to_f64(self.out.cpu().numpy().view(np.uint16))[:self.rows]
        scale = self.sm_scale or 1 / math.sqrt(self.dim)
        r, G = 0, self.hq // self.hkv
        for b, (n, L) in enumerate(zip(self.q_lens, self.seq_lens)):
            if n == 0:
                continue
            aq = np.abs(q[r:r + n]).reshape(n, self.hkv, G, self.dim)
            s_abs = scale * np.einsum("nhgd,htd->nhgt", aq, np.abs(kt[b])).max(axis=-1).reshape(n, self.hq, 1) if L else 0.0
            e_s = self.dim * 2.0 ** -23 * s_abs
            tiny = 0.0 if self.kv == "bf16" or not L else L * 2.0 ** -25 * np.abs(vt[b]).max()
            e = spread[r:r + n] * ((2.0 ** -8 if self.kv == "bf16" else 2.0 ** -11) + 2 * (e_s + 2.0 ** -21) + 2.0 ** -20) + tiny
            tol = e + 2.0 ** -8 * (np.abs(ref[r:r + n]) + e) + 2.0 ** -134
            err = np.abs(got[r:r + n] - ref[r:r + n])
            assert np.all(err <= tol), (b, float(np.nanmax(err / tol)), np.argwhere(~(err <= tol))[:4])
            g, w = self.lse.double().cpu().numpy()[r:r + n], lse[r:r + n]
            seen = np.isfinite(w)
            assert np.array_equal(np.isneginf(g), ~seen)
            bound = np.broadcast_to((e_s + 2.0 ** -20)[..., 0] if L else 0.0, w.shape) + 2.0 ** -20 * np.abs(np.where(seen, w, 0))
            assert np.all(np.abs(g[seen] - w[seen]) <= bound[seen]), float((np.abs(g[seen] - w[seen]) / bound[seen]).max())
            r += n

    def run(self):
        self.plan()
        self.attn()
        self.torch.cuda.synchronize()
        assert int(self.err) == 0
        self.check()
        self.h.close()


def test_one_token(lib):
    Case(lib, [1], [1]).run()


def test_one_full_tile(lib):
    Case(lib, [128], [128], hq=1, hkv=1).run()


def test_two_row_tiles(lib):
    Case(lib, [256], [256], hq=1, hkv=1, dim=128).run()


BATCHES = {
    "ragged": ([1, 0, 5, 130, 64, 33, 0], [1, 7, 5, 300, 1000, 40, 0]),
    "edges": ([16, 17, 127, 128, 129, 1, 31], [128, 129, 127, 256, 257, 128, 32]),
    "longer than the sequence": ([9, 3, 140], [4, 0, 130]),
    "one long": ([70], [2500]),
    "single tokens": ([1] * 6, [700, 1, 128, 129, 1500, 64]),
}


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("batch", list(BATCHES))
@pytest.mark.parametrize("hq,hkv,dim,page,order", [(4, 1, 64, 16, "HND"), (8, 2, 128, 16, "HND"), (10, 2, 128, 32, "NHD"),
                                                   (16, 1, 64, 64, "NHD"), (2, 2, 128, 64, "HND"), (7, 1, 128, 16, "NHD")])
def test_shapes(lib, hq, hkv, dim, page, order, batch, kv):
    q, L = BATCHES[batch]
    Case(lib, q, L, hq, hkv, dim, page, order, kv, seed=hq + dim, gap=8 if page == 32 else 0).run()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_scale_is_an_argument(lib, kv):
    Case(lib, [40, 3], [200, 150], 8, 2, 128, kv=kv, sm_scale=0.25, seed=3).run()


@pytest.mark.parametrize("dim", [64, 128])
def test_maximum_grows_all_along(lib, dim):
    """Scores that rise by far more than the slack of the running maximum from step to step, and fall again."""
    rng = np.random.default_rng(5)
    L, n = 900, 150
    q = np.ones((n, 2, dim), np.float32) * 0.25
    for up in (1, -1):
        ramp = (np.arange(L)[:: up] / 16).astype(np.float32)
        k = np.repeat(ramp[None, :, None], dim, axis=2) * 0.25 + 0.01 * rng.standard_normal((1, L, dim)).astype(np.float32)
        Case(lib, [n], [L], 2, 1, dim, q_values=q, k_values=[k], seed=6).run()


def test_one_dominant_key_around_every_limit(lib):
    """A key that outweighs all others at each position about a row's limit: only rows that see it return its value."""
    n, L, dim = 40, 300, 64
    for at in (0, 127, 128, 259, 260, 261, 298, 299):
        k = np.zeros((1, L, dim), np.float32)
        k[0, at, 0] = 64.0
        q = np.zeros((n, 1, dim), np.float32)
        q[:, 0, 0] = 64.0
        c = Case(lib, [n], [L], 1, 1, dim, q_values=q, k_values=[k], seed=at)
        c.plan(); c.attn()
        got = O.bf16_bits_to_f64(c.out.cpu().numpy().view(np.uint16))[:, 0]
        v = K.sequence_tokens(c.vh, c.bt, c.seq_lens)[0][0, at]
        sees = np.arange(n) + L - n >= at
        assert np.array_equal(got[sees], np.broadcast_to(v, (int(sees.sum()), dim))) and not np.any(np.all(got[~sees] == v, axis=-1))
        c.check(); c.h.close()


def test_same_bits_every_time_and_no_lse(lib):
    c = Case(lib, [40, 200, 3], [3000, 200, 2500], 8, 2, 128, seed=8)
    plan = lib.libra_chunk_plan_host(148, 8, 2, c.q_lens, c.seq_lens)
    assert len(plan["merges"]) > 0
    c.plan(); c.attn()
    first, lse = c.out.clone(), c.lse.clone()
    c.check()
    c.lse.fill_(7.0)
    for _ in range(20):
        c.out.fill_(0x7FC0)
        c.attn(lse=False)
        assert c.torch.equal(c.out, first)
    assert bool((c.lse == 7.0).all())
    c.plan(); c.attn()
    assert c.torch.equal(c.out, first) and c.torch.equal(c.lse, lse)
    c.h.close()


def test_agrees_with_the_decode_step(lib):
    """One new token per sequence: the decode step's result, within both roundings; several: libra_decode_attn_multi's."""
    import torch
    for n in (1, 3):
        c = Case(lib, [n] * 5, [900, 3, 64, 1, 2000], 8, 2, 128, seed=9)
        c.run()
        h = lib.Handle(8, 2, 128, c.kh.shape[0], 5, c.bt.shape[1])
        h.set_max_query_tokens(n)
        ws = torch.empty(h.workspace_size(), dtype=torch.uint8, device="cuda")
        out = torch.empty_like(c.out)
        lens = torch.from_numpy(c.seq_lens).cuda()
        st = torch.cuda.current_stream().cuda_stream
        h.plan(c.seq_lens, ws.data_ptr(), ws.numel(), st)
        h.decode_attn_multi(c.q.data_ptr(), n, c.k.data_ptr(), c.v.data_ptr(), c.dbt.data_ptr(), lens.data_ptr(), out.data_ptr(), st)
        a, b = (x.view(torch.bfloat16).double().cpu().numpy() for x in (c.out, out))
        (_, _, spread), _ = c.reference()
        assert np.all(np.abs(a - b) <= 2.0 ** -7 * np.abs(b) + 2.0 ** -7 * spread)
        h.close()


def test_prompt_tool_return_and_decode_together(lib):
    """As a rollout uses them: a prompt and a tool return are rotated, appended and attended to, then one token is decoded; all
    against float64: the rows and the cache from the projections, the attention from the rows and the cache."""
    import torch
    hq, hkv, dim, page = 8, 2, 64, 16
    rng = np.random.default_rng(10)
    rope = lib.libra_rope_init(64, lib.ROPE_HALF, 10000.0, lib.ROPE_SCALE_LINEAR, 2.0)
    turns = K.rope_turns(64, 10000.0, "linear", 2.0)
    phases = [[100, 33, 0], [20, 0, 77], [1, 1, 1]]
    total = [sum(p[b] for p in phases) for b in range(3)]
    pages = [-(-L // page) for L in total]
    bt = np.full((3, max(pages)), -1, np.int32)
    ids = rng.permutation(sum(pages) + 3)
    for b in range(3):
        bt[b, :pages[b]] = ids[sum(pages[:b]):sum(pages[:b + 1])]
    k, v = (torch.full((len(ids), hkv, page, dim), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    h = lib.Handle(hq, hkv, dim, len(ids), 3, bt.shape[1])
    dbt, err = torch.from_numpy(bt).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    dws = torch.empty(h.workspace_size(), dtype=torch.uint8, device="cuda")
    lens = np.zeros(3, np.int32)
    seen = {b: [] for b in range(3)}
    for step, n in enumerate(phases):
        lens = lens + np.asarray(n, np.int32)
        rows = sum(n)
        proj = torch.from_numpy(rng.standard_normal((rows, hq + 2 * hkv, dim))).to(torch.bfloat16).cuda()
        q, kn, vn = proj[:, :hq], proj[:, hq:hq + hkv], proj[:, hq + hkv:]
        off = torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32, device="cuda")
        dl = torch.from_numpy(lens.copy()).cuda()
        rot, out = (torch.empty((rows, hq, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        h.rope_append(rope, q.data_ptr(), q.stride(0), rot.data_ptr(), rot.stride(0), kn.data_ptr(), vn.data_ptr(), kn.stride(0),
                      off.data_ptr(), dl.data_ptr(), dbt.data_ptr(), 3, rows, k.data_ptr(), v.data_ptr(), err.data_ptr(), st)
        if step < 2:
            ws = torch.empty(h.chunk_workspace_size(rows), dtype=torch.uint8, device="cuda")
            h.chunk_plan(np.asarray(n, np.int32), lens, ws.data_ptr(), ws.numel(), st)
            h.chunk_attn(rot.data_ptr(), rot.stride(0), k.data_ptr(), v.data_ptr(), dbt.data_ptr(), out.data_ptr(), 0, err.data_ptr(), st)
        else:
            h.plan(lens, dws.data_ptr(), dws.numel(), st)
            h.decode_attn(rot.data_ptr(), k.data_ptr(), v.data_ptr(), dbt.data_ptr(), dl.data_ptr(), out.data_ptr(), st)
        torch.cuda.synchronize()
        assert int(err) == 0
        # the rotated rows, and every cached token so far, against the projections
        ang = K.rope_angles(K.row_positions(n, lens), turns)
        x = proj.double().cpu().numpy()
        rq, rk = K.rotate(x[:, :hq], ang, K.HALF), K.rotate(x[:, hq:hq + hkv], ang, K.HALF)
        gq = rot.double().cpu().numpy()
        assert np.all(np.abs(gq - rq) <= rope_bound(x[:, :hq], rq, 64, K.HALF, 1.0, "bf16"))
        kb = rope_bound(x[:, hq:hq + hkv], rk, 64, K.HALF, 1.0, "bf16")
        r = 0
        for b in range(3):
            seen[b] += [(rk[i], kb[i], x[i, hq + hkv:]) for i in range(r, r + n[b])]
            r += n[b]
        kt, vt = (K.sequence_tokens(t.view(torch.int16).cpu().numpy().view(np.uint16), bt, lens) for t in (k, v))
        for b in range(3):
            for t, (want, tol, value) in enumerate(seen[b]):
                assert np.all(np.abs(kt[b][:, t] - want) <= tol) and np.array_equal(vt[b][:, t], value)
        # the attention, from the rows and pages as they are
        ref, _, spread = K.packed_chunk_attention(gq, kt, vt, n, lens)
        got = out.double().cpu().numpy()
        assert np.all(np.abs(got - ref) <= (2.0 ** -8 + 2.0 ** -14) * spread * 1.01 + 2.0 ** -8 * np.abs(ref))
    h.close()


def test_recorded_and_replayed(lib):
    """New q and new cache contents in the same buffers; then another plan in the workspace: flagged, nothing written."""
    import torch
    c = Case(lib, [40, 3], [3000, 90], 8, 2, 128, seed=11)
    side = torch.cuda.Stream()
    c.plan(); c.attn(); torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        c.attn()
        with pytest.raises(lib.LibraError) as e:
            c.plan()                 # not while the stream is being recorded
        assert e.value.status == lib.INVALID_ARGUMENT
    rng = np.random.default_rng(12)
    c.qh = W.f32_to_bf16_bits(rng.standard_normal(c.qh.shape, dtype=np.float32))
    c.q[:, :8 * 128] = torch.from_numpy(c.qh.view(np.int16)).cuda().view(c.rows, -1)
    c.vh = np.where(c.vh == 0xFFC0, c.vh, c.vh ^ 0x8000).astype(np.uint16)
    c.v.copy_(torch.from_numpy(c.vh.view(np.int16)))
    c.out.fill_(0x7FC0)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert int(c.err) == 0
    c.check()
    c.h.chunk_plan(np.array([1, 1], np.int32), np.array([9, 9], np.int32), c.ws.data_ptr(), c.ws.numel(), torch.cuda.current_stream().cuda_stream)
    c.out.fill_(0x7FC0)
    g.replay(); torch.cuda.synchronize()
    assert int(c.err) == lib.ERR_PLAN_CHANGED and bool((c.out == 0x7FC0).all())
    c.err.zero_()
    c.plan(); c.attn(); torch.cuda.synchronize()
    assert int(c.err) == 0
    c.check()
    del g
    c.h.close()


def test_two_handles_on_two_streams(lib):
    import torch
    a = Case(lib, [300, 7], [2000, 3000], 8, 2, 128, seed=13)
    b = Case(lib, [64] * 4, [500, 64, 900, 1200], 10, 2, 128, seed=14, kv="e4m3")
    a.plan(); b.plan(); a.attn(); b.attn()
    torch.cuda.synchronize()
    a.check(); b.check()
    want = a.out.clone(), b.out.clone()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(10):
        a.out.fill_(0x7FC0); b.out.fill_(0x7FC0)
        torch.cuda.synchronize()
        for _ in range(3):
            with torch.cuda.stream(sa):
                a.plan(); a.attn()
            with torch.cuda.stream(sb):
                b.plan(); b.attn()
        torch.cuda.synchronize()
        assert torch.equal(a.out, want[0]) and torch.equal(b.out, want[1])
    a.h.close(); b.h.close()


def test_bad_page_reads_as_zeros(lib):
    """An id outside the pool: flagged; its tokens count as zero keys and values, nothing else changes."""
    for bad in (-5, None, 2 ** 31 - 1):
        c = Case(lib, [20], [200], 4, 2, 64, seed=15)
        at = int(c.bt[0, 3])
        c.dbt[0, 3] = bad if bad is not None else c.kh.shape[0]
        c.plan(); c.attn()
        assert int(c.err) == lib.ERR_BAD_PAGE_ID
        c.kh[at], c.vh[at] = 0, 0
        c.check(); c.h.close()


def test_writes_stay_in_bounds(lib):
    """out, lse and the workspace between bands of known bytes; rows behind the batch stay."""
    import torch
    band = 4096
    for q, L in (([40, 3], [3000, 90]), ([130, 1], [140, 5])):
        c = Case(lib, q, L, 10, 2, 128, seed=16, kv="bf16")
        n_ws = c.h.chunk_workspace_size(c.rows)
        sizes = (c.rows * 10 * 128 * 2, c.rows * 10 * 4, n_ws)
        bufs = [torch.full((band + -(-n // 256) * 256 + band,), 0x5A, dtype=torch.uint8, device="cuda") for n in sizes]
        st = torch.cuda.current_stream().cuda_stream
        c.h.chunk_plan(c.q_lens, c.seq_lens, bufs[2].data_ptr() + band, n_ws, st)
        c.h.chunk_attn(c.q.data_ptr(), c.q.stride(0), c.k.data_ptr(), c.v.data_ptr(), c.dbt.data_ptr(), bufs[0].data_ptr() + band,
                       bufs[1].data_ptr() + band, c.err.data_ptr(), st)
        torch.cuda.synchronize()
        for buf, n in zip(bufs, sizes):
            assert bool((buf[:band] == 0x5A).all()) and bool((buf[band + n:] == 0x5A).all())
        c.out.view(torch.uint8).view(-1)[:sizes[0]] = bufs[0][band:band + sizes[0]]
        c.lse.view(torch.uint8).view(-1)[:sizes[1]] = bufs[1][band:band + sizes[1]]
        assert int(c.err) == 0
        c.check(); c.h.close()


def test_far_into_a_large_pool(lib):
    """Pages whose offsets pass 2^31 elements and 2^32 bytes."""
    import torch
    hkv, dim, page, L, n = 8, 128, 64, 150, 20
    pages = (1 << 31) // (hkv * dim * page) + 40
    k, v = (torch.zeros((pages, hkv, page, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bt = np.array([[pages - 1, 2, pages - 7]], np.int32)
    for x in (k, v):
        x[bt[0].tolist()] = torch.randn((3, hkv, page, dim), device="cuda").to(torch.bfloat16)
    h = lib.Handle(8, 8, dim, pages, 1, 3, page_size=page)
    q = torch.randn((n, 8, dim), device="cuda").to(torch.bfloat16)
    out, err = torch.empty_like(q), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(h.chunk_workspace_size(n), dtype=torch.uint8, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    h.chunk_plan(np.array([n], np.int32), np.array([L], np.int32), ws.data_ptr(), ws.numel(), st)
    dbt = torch.from_numpy(bt).cuda()
    h.chunk_attn(q.data_ptr(), q.stride(0), k.data_ptr(), v.data_ptr(), dbt.data_ptr(), out.data_ptr(), 0, err.data_ptr(), st)
    assert int(err) == 0
    kt, vt = (x[bt[0].tolist()].double().cpu().numpy().transpose(1, 0, 2, 3).reshape(hkv, -1, dim)[:, :L] for x in (k, v))
    ref, _, spread = K.packed_chunk_attention(q.double().cpu().numpy(), [kt], [vt], [n], [L])
    assert np.all(np.abs(out.double().cpu().numpy() - ref) <= (2.0 ** -8 + 2.0 ** -14) * spread * 1.01 + 2.0 ** -8 * np.abs(ref))
    h.close()


def test_sequences_that_share_pages(lib):
    """A common beginning held once: both block tables name the same pages."""
    c = Case(lib, [30, 7], [100, 100], 8, 2, 128, seed=18)
    c.bt[1, :4] = c.bt[0, :4]
    c.dbt.copy_(c.torch.from_numpy(c.bt))
    c.run()


def test_launches_that_are_not_dependent_give_the_same_bits(lib):
    c = Case(lib, [40, 3], [3000, 90], 8, 2, 128, seed=19)
    c.plan(); c.attn()
    want = c.out.clone()
    c.h.set_dependent_launch(False)
    c.out.fill_(0x7FC0)
    c.attn()
    assert c.torch.equal(c.out, want)
    c.check(); c.h.close()


def test_more_items_than_a_grid_dimension_holds(lib):
    """70,000 sequences of one token: each row of out is its value row."""
    import torch
    n = 70000
    k, v, q = (torch.randn((n, 1, 16, 64), device="cuda").to(torch.bfloat16) for _ in range(3))
    k[:, :, 1:], v[:, :, 1:] = float("nan"), float("nan")
    h = lib.Handle(1, 1, 64, n, n, 1)
    bt = torch.randperm(n, device="cuda").to(torch.int32)
    ws = torch.empty(h.chunk_workspace_size(n), dtype=torch.uint8, device="cuda")
    out, err = torch.empty((n, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    h.chunk_plan(np.ones(n, np.int32), np.ones(n, np.int32), ws.data_ptr(), ws.numel(), st)
    rows = q[:, 0, 0].contiguous()
    h.chunk_attn(rows.data_ptr(), 64, k.data_ptr(), v.data_ptr(), bt.data_ptr(), out.data_ptr(), 0, err.data_ptr(), st)
    assert int(err) == 0 and torch.equal(out, v[bt.long(), 0, 0])
    h.close()


def test_pools_of_the_other_type_after_the_plan(lib):
    """The plan does not depend on the pools' type: one plan, attention over E4M3 pools and then over bf16 ones."""
    c8 = Case(lib, [20, 3], [300, 90], 8, 2, 128, seed=20, kv="e4m3")
    c16 = Case(lib, [20, 3], [300, 90], 8, 2, 128, seed=20)
    c8.h.close()
    c8.h = c16.h
    assert c8.kh.shape == c16.kh.shape
    c16.plan()
    c8.h.set_kv_dtype(lib.KV_E4M3, *c8.scales)
    c8.attn()
    c8.check()
    c16.h.set_kv_dtype(lib.KV_BF16)
    c16.attn()
    c16.check()
    assert int(c8.err) == 0 and int(c16.err) == 0
    c16.h.close()


def test_refusals(lib):
    c = Case(lib, [4, 2], [30, 9], 4, 2, 64, seed=17)
    good = dict(q_ptr=c.q.data_ptr(), q_stride=256, k_ptr=c.k.data_ptr(), v_ptr=c.v.data_ptr(), block_table_ptr=c.dbt.data_ptr(),
                out_ptr=c.out.data_ptr(), lse_ptr=0, error_word_ptr=c.err.data_ptr(), stream=0)
    with pytest.raises(lib.LibraError) as e:
        c.h.chunk_attn(**good)
    assert e.value.status == lib.NOT_PLANNED
    ws, n = c.ws.data_ptr(), c.ws.numel()
    a32 = lambda *x: np.asarray(x, np.int32)
    for args, status in [((a32(4, 2), a32(30, -1), ws, n, 0), lib.INVALID_ARGUMENT), ((a32(-4, 2), a32(30, 9), ws, n, 0), lib.INVALID_ARGUMENT),
                         ((a32(4, 2), a32(33, 9), ws, n, 0), lib.INVALID_ARGUMENT), ((a32(4, 2, 1), a32(30, 9, 9), ws, n, 0), lib.INVALID_ARGUMENT),
                         ((a32(4, 2), a32(30, 9), 0, n, 0), lib.INVALID_ARGUMENT), ((a32(4, 2), a32(30, 9), ws + 16, n, 0), lib.INVALID_ARGUMENT),
                         ((a32(4, 2), a32(30, 9), ws, 256, 0), lib.WORKSPACE_TOO_SMALL)]:
        with pytest.raises(lib.LibraError) as e:
            c.h.chunk_plan(*args)
        assert e.value.status == status
    c.plan()
    for kw in (dict(q_ptr=0), dict(k_ptr=0), dict(v_ptr=0), dict(block_table_ptr=0), dict(out_ptr=0), dict(error_word_ptr=0), dict(q_stride=248),
               dict(q_stride=260), dict(q_ptr=c.q.data_ptr() + 8), dict(k_ptr=c.k.data_ptr() + 8), dict(out_ptr=c.out.data_ptr() + 8),
               dict(lse_ptr=c.lse.data_ptr() + 2)):
        with pytest.raises(lib.LibraError) as e:
            c.h.chunk_attn(**{**good, **kw})
        assert e.value.status == lib.INVALID_ARGUMENT, kw
    with pytest.raises(lib.LibraError):
        c.h.chunk_workspace_size(-1)
    # a batch without new tokens, an empty batch: nothing to do
    for q, L in ((a32(0, 0), a32(30, 9)), (a32(), a32())):
        c.h.chunk_plan(q, L, ws, n, 0)
        c.h.chunk_attn(**good)
    assert bool((c.out == 0x7FC0).all())
    c.h.close()
