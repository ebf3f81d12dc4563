"""Rotary positions and the append with rotation on the GPU against the float64 oracle.

Tolerance of a rotated value y = m (u cos a - v sin a): the angle is off by at most 2^-32 turn (cut phase) plus half a unit of
a float32 of at most an eighth of a turn, below 2^-24 rad together; sincospif is off by at most 2 units in the last place,
2^-23 for values up to 1; the magnitude and the two products round three times by 2^-24 of each term and the sum once: below
2^-21.2 (|u| + |v|) m altogether, taken as 2^-21.  Then one rounding to the type: half a step relative to the value, and half
of its smallest step near zero."""
import numpy as np
import pytest

from oracle import attention_oracle as O
from oracle import chunk_oracle as K

from test_rope import SCALINGS, rope_of

pytestmark = pytest.mark.gpu

HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
TINY = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25, "f32": 2.0 ** -150}


def types(torch):
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def bound(x, ref, rotary, layout, magnitude, dtype):
    """Per element: the arithmetic above on the pair the element belongs to, then the rounding; channels that pass: 0."""
    n = rotary // 2
    s = np.abs(x)
    b = np.zeros_like(ref)
    for i in range(n):
        a, c = (i, i + n) if layout == K.HALF else (2 * i, 2 * i + 1)
        e = 2.0 ** -21 * magnitude * (s[..., a] + s[..., c])
        for k in (a, c):
            b[..., k] = e + HALF_STEP[dtype] * (np.abs(ref[..., k]) + e) + TINY[dtype]
    return b


def apply(lib, rope, x, out, positions, dtype, direction):
    import torch
    lib.libra_rope_apply(0, rope, x.data_ptr(), out.data_ptr(), {"bf16": lib.ROPE_BF16, "f16": lib.ROPE_F16, "f32": lib.ROPE_F32}[dtype],
                         positions.data_ptr(), x.shape[0], x.shape[1], x.shape[2], x.stride(0), x.stride(1), out.stride(0),
                         out.stride(1), direction, torch.cuda.current_stream().cuda_stream)


@pytest.mark.parametrize("gradient", [False, True])
@pytest.mark.parametrize("layout", [K.HALF, K.INTERLEAVED])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens,heads,dim,rotary,scaling", [
    (1, 1, 2, 2, "none"), (1, 32, 128, 128, "none"), (7, 3, 80, 80, "linear"), (37, 5, 96, 32, "base"), (130, 2, 64, 64, "bands"),
    (3, 1, 256, 256, "ramp"), (5, 4, 66, 10, "ramp"), (1200, 1, 64, 24, "none"), (2500, 2, 8, 8, "none"), (3, 2, 1024, 250, "none"), (700, 3, 1024, 256, "linear")])
def test_apply(lib, tokens, heads, dim, rotary, scaling, dtype, layout, gradient):
    import torch
    rope = rope_of(lib, rotary, layout, 10000.0, scaling)
    rng = np.random.default_rng(tokens * 1000 + dim)
    x = torch.from_numpy(rng.standard_normal((tokens, heads, dim))).to("cuda").to(types(torch)[dtype])
    pos = rng.integers(0, 1 << 20, tokens).astype(np.int32)
    pos[0] = 0 if tokens > 1 else 2 ** 31 - 1
    if tokens > 4:
        pos[1:5] = [2 ** 31 - 1, -1, -2 ** 31, 1]
    out = torch.full_like(x, float("nan"))
    apply(lib, rope, x, out, torch.from_numpy(pos).cuda(), dtype, lib.ROPE_GRADIENT if gradient else lib.ROPE_FORWARD)
    xs = x.double().cpu().numpy()
    a = K.rope_angles(pos, K.rope_turns(rotary, 10000.0, scaling, **SCALINGS[scaling]))
    ref = K.rotate(xs, -a if gradient else a, layout, float(rope.magnitude))
    err = np.abs(out.double().cpu().numpy() - ref)
    assert np.all(err <= bound(xs, ref, rotary, layout, float(rope.magnitude), dtype))


@pytest.mark.parametrize("layout", [K.HALF, K.INTERLEAVED])
def test_apply_strided_in_place_and_unaligned(lib, layout):
    """Rows inside a wider buffer: what lies between them stays; in place equals out of place; rows off any 16-byte boundary."""
    import torch
    rng = np.random.default_rng(7)
    tokens, heads, dim, rotary = 19, 3, 64, 32
    rope = rope_of(lib, rotary, layout)
    pos = torch.from_numpy(rng.integers(0, 5000, tokens).astype(np.int32)).cuda()
    for off, gap in ((0, 0), (0, 8), (1, 0), (3, 5)):
        wide = torch.from_numpy(rng.standard_normal((tokens + 1, (heads + 2) * (dim + gap) + 7))).to(torch.bfloat16).cuda()
        stride = wide.shape[1]
        view = torch.as_strided(wide, (tokens, heads, dim), (stride, dim + gap, 1), off)
        before, out = wide.clone(), torch.empty((tokens, heads, dim), dtype=torch.bfloat16, device="cuda")
        apply(lib, rope, view, out, pos, "bf16", lib.ROPE_FORWARD)
        assert torch.equal(wide, before)
        ref = K.rotate(view.double().cpu().numpy(), K.rope_angles(pos.cpu().numpy(), K.rope_turns(rotary, 10000.0)), layout)
        assert np.all(np.abs(out.double().cpu().numpy() - ref) <= bound(view.double().cpu().numpy(), ref, rotary, layout, 1.0, "bf16"))
        apply(lib, rope, view, view, pos, "bf16", lib.ROPE_FORWARD)
        assert torch.equal(view, out)
        keep = torch.ones_like(wide, dtype=torch.bool)
        torch.as_strided(keep, (tokens, heads, dim), (stride, dim + gap, 1), off).fill_(False)
        assert torch.equal(wide[keep], before[keep])


def test_apply_on_head_major_rows_and_another_stream(lib):
    """[heads, tokens, channels], as attention over dense keys wants it, from and into; the call on a side stream."""
    import torch
    rng = np.random.default_rng(9)
    tokens, heads, dim = 50, 6, 64
    rope, pos = rope_of(lib, 64), torch.from_numpy(rng.integers(0, 5000, 50).astype(np.int32)).cuda()
    x = torch.from_numpy(rng.standard_normal((heads, tokens, dim))).to(torch.bfloat16).cuda()
    out = torch.full_like(x, float("nan"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        apply(lib, rope, x.transpose(0, 1), out.transpose(0, 1), pos, "bf16", lib.ROPE_FORWARD)
    side.synchronize()
    xs = x.transpose(0, 1).double().cpu().numpy()
    ref = K.rotate(xs, K.rope_angles(pos.cpu().numpy(), K.rope_turns(64, 10000.0)), K.HALF)
    assert np.all(np.abs(out.transpose(0, 1).double().cpu().numpy() - ref) <= bound(xs, ref, 64, K.HALF, 1.0, "bf16"))


@pytest.mark.parametrize("layout", [K.HALF, K.INTERLEAVED])
def test_gradient_against_differences(lib, layout):
    """The map is linear: <g, f(x + d) - f(x)> = <gradient(g), d>; each side's terms are off by 2^-20 of their size."""
    import torch
    rng = np.random.default_rng(8)
    tokens, heads, dim, rotary = 33, 4, 96, 64
    rope = rope_of(lib, rotary, layout, scaling="ramp")
    pos = torch.from_numpy(rng.integers(0, 1 << 17, tokens).astype(np.int32)).cuda()
    x, d, g = (torch.from_numpy(rng.standard_normal((tokens, heads, dim))).float().cuda() for _ in range(3))
    fx, fxd, gg = (torch.empty_like(x) for _ in range(3))
    xd = x + d
    apply(lib, rope, x, fx, pos, "f32", lib.ROPE_FORWARD)
    apply(lib, rope, xd, fxd, pos, "f32", lib.ROPE_FORWARD)
    apply(lib, rope, g, gg, pos, "f32", lib.ROPE_GRADIENT)
    left = (g.double() * (fxd.double() - fx.double())).sum(-1)
    right = (gg.double() * (xd.double() - x.double())).sum(-1)
    size = 2.0 ** -20 * rope.magnitude * 4 * (g.abs().double().sum(-1) * (xd.abs() + x.abs()).double().amax(-1))
    assert bool(((left - right).abs() <= size).all())


# ----------------------------------------------------------------------------------------------------------------- append
class Batch:
    """Packed new tokens and their pages."""

    def __init__(self, lib, q_lens, seq_lens, hq=4, hkv=2, dim=64, page=16, order="HND", kv="bf16", seed=0, extra_rows=0, fused=False,
                 ld=None):
        import torch
        rng = np.random.default_rng(seed)
        self.q_lens, self.seq_lens, self.kv, self.order, self.page = list(q_lens), list(seq_lens), kv, order, page
        B, rows = len(q_lens), int(sum(q_lens))
        self.rows, self.max_rows = rows, rows + extra_rows
        pages = [-(-L // page) for L in seq_lens]
        self.ld = max(1, max(pages)) if ld is None else ld
        self.pool_pages = sum(pages) + 2
        ids = rng.permutation(self.pool_pages)[:sum(pages)]
        self.bt = np.full((B, self.ld), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(pages):
            m = min(n, self.ld)
            self.bt[b, :m] = ids[at:at + m]
            at += n
        shape = (self.pool_pages, hkv, page, dim) if order == "HND" else (self.pool_pages, page, hkv, dim)
        if kv == "bf16":
            pools = [torch.from_numpy(rng.integers(0, 1 << 15, shape).astype(np.int16)).cuda() for _ in range(2)]
        else:
            pools = [torch.from_numpy(rng.integers(0, 256, shape).astype(np.uint8)).cuda() for _ in range(2)]
        self.k, self.v = pools
        self.k0, self.v0 = self.k.clone(), self.v.clone()
        proj = torch.from_numpy(rng.standard_normal((self.max_rows, hq + 2 * hkv, dim))).to(torch.bfloat16).cuda()
        self.q, self.kn, self.vn = proj[:, :hq], proj[:, hq:hq + hkv], proj[:, hq + hkv:]
        if not fused:
            self.q, self.kn, self.vn = (x.contiguous() for x in (self.q, self.kn, self.vn))
        self.q_out = torch.full((self.max_rows, hq, dim), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.off = torch.tensor(np.concatenate([[0], np.cumsum(q_lens)]), dtype=torch.int32, device="cuda")
        self.lens = torch.tensor(seq_lens, dtype=torch.int32, device="cuda")
        self.dbt = torch.from_numpy(self.bt).cuda()
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        strides = (0, 0, 0) if order == "HND" else (page * hkv * dim, dim, hkv * dim)
        self.h = lib.Handle(hq, hkv, dim, self.pool_pages, max(B, 1), self.ld, page_size=page, kv_strides=strides)
        self.scales = (1.0, 1.0)
        if kv == "e4m3":
            self.scales = (0.0371, 0.25)
            self.h.set_kv_dtype(lib.KV_E4M3, *self.scales)

    def append(self, rope, q=True, in_place=False):
        import torch
        out = self.q if in_place else self.q_out
        args = (self.q.data_ptr(), self.q.stride(0), out.data_ptr(), out.stride(0)) if q else (0, 0, 0, 0)
        self.h.rope_append(rope, *args, self.kn.data_ptr(), self.vn.data_ptr(), self.kn.stride(0), self.off.data_ptr(),
                           self.lens.data_ptr(), self.dbt.data_ptr(), len(self.q_lens), self.max_rows, self.k.data_ptr(),
                           self.v.data_ptr(), self.err.data_ptr(), torch.cuda.current_stream().cuda_stream)

    def check(self, rotary, layout, turns, magnitude=1.0, q=True, skip=()):
        """q_out and both pools, every element: new slots within the bound, all others as they were."""
        pos = K.row_positions(self.q_lens, self.seq_lens)
        ang = K.rope_angles(pos, turns)
        r = self.rows
        qx, kx, vx = (x[:r].double().cpu().numpy() for x in (self.q, self.kn, self.vn))
        if q:
            ref = K.rotate(qx, ang, layout, magnitude)
            got = self.q_out.double().cpu().numpy()
            assert np.all(np.abs(got[:r] - ref) <= bound(qx, ref, rotary, layout, magnitude, "bf16"))
            assert np.all(np.isnan(got[r:]))
        for pool, before, x, turn, scale in ((self.k, self.k0, kx, True, self.scales[0]), (self.v, self.v0, vx, False, self.scales[1])):
            now, was = pool.cpu().numpy(), before.cpu().numpy().copy()
            if self.order == "HND":
                now, was = now.transpose(0, 2, 1, 3), was.transpose(0, 2, 1, 3)
            y = K.rotate(x, ang, layout, magnitude) if turn else x
            e = bound(x, y, rotary, layout, magnitude, "f32") if turn else np.zeros_like(y)
            row = 0
            for b, (n, L) in enumerate(zip(self.q_lens, self.seq_lens)):
                for t in range(L - n, L):
                    if t >= 0 and (b, t) not in skip:
                        at = self.bt[b, t // self.page], t % self.page
                        if self.kv == "bf16":
                            got = O.bf16_bits_to_f64(now[at].view(np.uint16))
                            # a value that is only copied comes back as it was
                            assert np.all(np.abs(got - y[row]) <= np.where(e[row] > 0, e[row] + 2.0 ** -8 * (np.abs(y[row]) + e[row]) + 2.0 ** -134, 0.0))
                        else:
                            # between the codes of the two ends of what the float32 value, times the rounded reciprocal, may be
                            z, ez = y[row] / scale, e[row] / scale + 2.0 ** -22 * np.abs(y[row] / scale)
                            lo, hi = (K.e4m3_values()[K.e4m3_encode(z + s * ez)] for s in (-1, 1))
                            got = K.e4m3_values()[now[at]]
                            assert np.all((got >= lo) & (got <= hi))
                        was[at] = now[at]
                    row += 1
            assert np.array_equal(now, was)
        self.h.close()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("order", ["HND", "NHD"])
@pytest.mark.parametrize("layout", [K.HALF, K.INTERLEAVED])
@pytest.mark.parametrize("page,dim,rotary,scaling", [(16, 64, 64, "none"), (32, 128, 64, "ramp"), (64, 128, 128, "bands"),
                                                     (16, 64, 24, "linear"), (16, 128, 10, "none")])
def test_append(lib, page, dim, rotary, scaling, layout, order, kv):
    """Ragged batch: no new tokens, one, a chunk over several pages, a whole prompt, a chunk longer than its sequence."""
    rope = rope_of(lib, rotary, layout, scaling=scaling)
    b = Batch(lib, [1, 0, 37, 20, 0, 5, 1, 0], [1, 40, 100, 20, 0, 3, 65, 9], dim=dim, page=page, order=order, kv=kv, extra_rows=9,
              fused=page == 16, seed=page + dim)
    b.append(rope)
    assert int(b.err) == 0
    b.check(rotary, layout, K.rope_turns(rotary, 10000.0, scaling, **SCALINGS[scaling]), float(rope.magnitude))


def test_append_single_tokens_many_sequences(lib):
    """One token each (a decode step) of 300 sequences, five query heads per KV head."""
    rng = np.random.default_rng(4)
    b = Batch(lib, [1] * 300, [int(x) for x in rng.integers(1, 200, 300)], hq=10, hkv=2, dim=128)
    b.append(rope_of(lib, 128))
    assert int(b.err) == 0
    b.check(128, K.HALF, K.rope_turns(128, 10000.0))


def test_append_in_place_without_q_and_without_rotation(lib):
    import torch
    rope, turns = rope_of(lib, 64), K.rope_turns(64, 10000.0)
    a, b = (Batch(lib, [3, 18], [19, 18], seed=5) for _ in range(2))
    a.append(rope)
    q0 = b.q.clone()
    b.append(rope, in_place=True)
    assert torch.equal(b.q, a.q_out) and torch.equal(a.k, b.k) and torch.equal(a.v, b.v) and not torch.equal(b.q, q0)
    a.check(64, K.HALF, turns)
    c = Batch(lib, [3, 18], [19, 18], seed=5)
    c.append(rope, q=False)
    assert torch.equal(c.k, b.k) and bool(torch.isnan(c.q_out).all())
    d = Batch(lib, [3, 18], [19, 18], seed=5)
    d.append(None)
    assert torch.equal(d.q_out, d.q)
    d.check(2, K.HALF, [0])
    b.h.close(); c.h.close()


def test_append_bad_pages_and_short_tables(lib):
    """A page id outside the pool and a token past the table are flagged and not stored; all else is."""
    rope, turns = rope_of(lib, 64), K.rope_turns(64, 10000.0)
    for bad in (-1, None):
        b = Batch(lib, [20, 40], [50, 40], seed=6)
        b.bt[1, 1] = bad if bad is not None else b.pool_pages
        b.dbt.copy_(__import__("torch").from_numpy(b.bt))
        b.append(rope)
        assert int(b.err) == lib.ERR_BAD_PAGE_ID
        b.check(64, K.HALF, turns, skip={(1, t) for t in range(16, 32)})
    b = Batch(lib, [20, 40], [50, 40], ld=3, seed=6)
    b.append(rope)
    assert int(b.err) == lib.ERR_PLAN_OVERFLOW
    b.check(64, K.HALF, turns, skip={(0, 48), (0, 49)})


def test_append_recorded_and_replayed_with_fewer_tokens(lib):
    """A graph recorded for 24 rows of 4 sequences, replayed after offsets and lengths changed in their buffers."""
    import torch
    rope, turns = rope_of(lib, 64), K.rope_turns(64, 10000.0)
    b = Batch(lib, [8, 8, 8, 0], [30, 8, 9, 0], seed=7)
    side = torch.cuda.Stream()
    b.append(rope); torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        b.append(rope)
    b.q_out.fill_(float("nan")); b.k.copy_(b.k0); b.v.copy_(b.v0)
    b.q_lens, b.seq_lens, b.rows = [2, 0, 9, 0], [29, 8, 9, 0], 11
    b.off.copy_(torch.tensor([0, 2, 2, 11, 11], dtype=torch.int32)); b.lens.copy_(torch.tensor(b.seq_lens, dtype=torch.int32))
    g.replay(); torch.cuda.synchronize()
    assert int(b.err) == 0
    b.check(64, K.HALF, turns)
    del g


def test_append_far_into_a_large_pool(lib):
    """Slots whose offsets pass 2^31 elements and 2^32 bytes."""
    import torch
    hkv, dim, page = 8, 128, 64
    pages = (1 << 31) // (hkv * dim * page) + 40                  # 2.15e9 elements, 4.3 GB a pool
    k, v = (torch.zeros((pages, hkv, page, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    h = lib.Handle(8, 8, dim, pages, 1, 2, page_size=page)
    bt = torch.tensor([[pages - 1, 3]], dtype=torch.int32, device="cuda")
    off, lens = torch.tensor([0, 66], dtype=torch.int32, device="cuda"), torch.tensor([66], dtype=torch.int32, device="cuda")
    kn, vn = (torch.randn((66, hkv, dim), device="cuda").to(torch.bfloat16) for _ in range(2))
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    h.rope_append(None, 0, 0, 0, 0, kn.data_ptr(), vn.data_ptr(), hkv * dim, off.data_ptr(), lens.data_ptr(), bt.data_ptr(), 1, 66,
                  k.data_ptr(), v.data_ptr(), err.data_ptr(), torch.cuda.current_stream().cuda_stream)
    for pool, x in ((k, kn), (v, vn)):
        assert torch.equal(pool[pages - 1], x[:64].transpose(0, 1)) and torch.equal(pool[3, :, :2], x[64:].transpose(0, 1))
        assert int((pool != 0).sum()) == int((x != 0).sum())
    assert int(err) == 0
    h.close()


def test_append_refusals(lib):
    b = Batch(lib, [2], [2])
    rope = rope_of(lib, 64)
    good = dict(rope=rope, q_ptr=b.q.data_ptr(), q_stride=256, q_out_ptr=b.q_out.data_ptr(), q_out_stride=256, k_new_ptr=b.kn.data_ptr(),
                v_new_ptr=b.vn.data_ptr(), kv_stride=128, q_offsets_ptr=b.off.data_ptr(), seq_lens_ptr=b.lens.data_ptr(),
                block_table_ptr=b.dbt.data_ptr(), batch=1, max_rows=2, k_ptr=b.k.data_ptr(), v_ptr=b.v.data_ptr(),
                error_word_ptr=b.err.data_ptr(), stream=0)
    for kw, status in [
        (dict(q_ptr=0), lib.INVALID_ARGUMENT), (dict(q_out_ptr=0), lib.INVALID_ARGUMENT), (dict(k_new_ptr=0), lib.INVALID_ARGUMENT),
        (dict(v_ptr=0), lib.INVALID_ARGUMENT), (dict(error_word_ptr=0), lib.INVALID_ARGUMENT), (dict(batch=2), lib.INVALID_ARGUMENT),
        (dict(batch=-1), lib.INVALID_ARGUMENT), (dict(max_rows=-1), lib.INVALID_ARGUMENT), (dict(q_stride=248), lib.INVALID_ARGUMENT),
        (dict(kv_stride=132), lib.INVALID_ARGUMENT), (dict(q_out_stride=260), lib.INVALID_ARGUMENT),
        (dict(q_out_ptr=b.q.data_ptr(), q_out_stride=264), lib.INVALID_ARGUMENT), (dict(k_new_ptr=b.kn.data_ptr() + 2), lib.INVALID_ARGUMENT),
        (dict(rope=lib.Rope()), lib.INVALID_ARGUMENT), (dict(rope=rope_of(lib, 128)), lib.UNSUPPORTED_SHAPE),
    ]:
        with pytest.raises(lib.LibraError) as e:
            b.h.rope_append(**{**good, **kw})
        assert e.value.status == status, kw
    b.h.rope_append(**{**good, "batch": 0})
    b.h.rope_append(**{**good, "max_rows": 0})
    b.h.close()
