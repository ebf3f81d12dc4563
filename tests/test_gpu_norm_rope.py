"""Norms of the heads of q and k with the rotation, their gradient and the append by slots, on the GPU against float64.

Tolerances, with u = 2^-24 (half a float32 step, relative).  The sum of D squares is off by at most D u of itself, r by half of
that, u of its own rounding and another u of the mean's product and sum: er = D u / 2 + 2 u.  A normalised channel n = w x r adds two
products: en = er + 2 u, relative.  The rotation adds 2^-21 m (|a| + |b|) for the pair (a, b) it turns (derived in test_gpu_rope.py),
and carries the errors of the pair's normalised channels with it.  Then half a step of the type.

Gradient: g, the pair turned back, is off by eg = 2^-21 m (|dy_a| + |dy_b|), 0 where channels pass.  With A = |w g|,
eA = |w| eg + u A, and S = r sum |w g x| / D: eS = r sum(eA |x|) / D + (D u + 3 u + er) S;  dx = r (w g - n mean) is off by
r (eA + |n| eS + S en |n| + 2 u (A + |n| S)) + (er + u) r (A + |n| S), n = x r.  dw = sum g n over N rows: sum of eg |n| + en |g n|, and
N u sum |g n| for the additions."""
import numpy as np
import pytest

from oracle import attention_oracle as O
from oracle import chunk_oracle as K

from test_gpu_rope import HALF_STEP, TINY, types
from test_rope import SCALINGS, rope_of

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-6


def pairs_of(dim, rotary, layout):
    """Partner of every channel (itself where it passes)."""
    p = np.arange(dim)
    for i in range(rotary // 2):
        a, c = (i, i + rotary // 2) if layout == K.HALF else (2 * i, 2 * i + 1)
        p[a], p[c] = c, a
    return p


def forward(x, w, angles, layout, magnitude, eps=EPS, normed=True):
    """float64 reference and the bound before the last rounding; x [tokens, heads, dim]."""
    D = x.shape[-1]
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps) if normed else 1.0
    n = x * r * (w if normed else 1.0)
    y = K.rotate(n, angles, layout, magnitude)
    other = pairs_of(D, 2 * angles.shape[1], layout)
    turned = other != np.arange(D)
    en = (D * U / 2 + 4 * U) if normed else 0.0
    both = np.abs(n) + np.abs(n[..., other])
    e = np.where(turned, (2.0 ** -21 + en) * magnitude * both, en * np.abs(n))
    return y, e


def gradient(x, dy, w, angles, layout, magnitude, eps=EPS):
    """float64 dx, dw and their bounds before the last rounding."""
    D = x.shape[-1]
    g = K.rotate(dy, -angles, layout, magnitude)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r
    mean = (w * g * n).mean(-1, keepdims=True)
    dx, dw = r * (w * g - n * mean), (g * n).sum((0, 1))
    other = pairs_of(D, 2 * angles.shape[1], layout)
    eg = np.where(other != np.arange(D), 2.0 ** -21 * magnitude * (np.abs(dy) + np.abs(dy[..., other])), 0.0)
    er = D * U / 2 + 2 * U
    A = np.abs(w * g)
    eA = np.abs(w) * eg + U * A
    S = np.abs(w * g * n).mean(-1, keepdims=True)
    eS = (eA * np.abs(n)).mean(-1, keepdims=True) + (D * U + 3 * U + er) * S
    an = np.abs(n)
    e = r * (eA + an * eS + S * (er + 2 * U) * an + 2 * U * (A + an * S)) + (er + U) * r * (A + an * S)
    N = x.shape[0] * x.shape[1]
    ew = (eg * an + (er + 2 * U) * np.abs(g) * an).sum((0, 1)) + N * U * (np.abs(g) * an).sum((0, 1))
    return dx, dw, e, ew


def rounded(ref, e, dtype):
    return e + HALF_STEP[dtype] * (np.abs(ref) + e) + TINY[dtype]


def dtype_of(lib, dtype):
    return {"bf16": lib.ROPE_BF16, "f16": lib.ROPE_F16, "f32": lib.ROPE_F32}[dtype]


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def make(tokens, heads, dim, dtype, rng, gap=0, off=0, scale=1.5):
    """Rows within a wider array, `off` elements into it; the array and the rows."""
    import torch
    pitch = heads * dim + gap
    wide = torch.from_numpy(rng.standard_normal(tokens * pitch + off + 16) * scale).to(types(torch)[dtype]).cuda()
    return wide, torch.as_strided(wide, (tokens, heads, dim), (pitch, dim, 1), off)


def f64(t):
    return t.double().cpu().numpy()


SHAPES = [  # tokens, q heads, k heads, head_dim, rotary_dim
    (1, 1, 0, 64, 64), (5, 4, 1, 128, 128), (33, 5, 2, 128, 64), (7, 3, 1, 80, 80), (9, 8, 8, 96, 48), (3, 2, 1, 256, 256), (4, 1, 3, 256, 64),
    (6, 2, 2, 80, 40), (3, 5, 1, 24, 24), (2, 3, 1, 30, 10), (2, 2, 1, 1024, 256), (3, 2, 1, 512, 128), (2, 1, 1, 2, 2), (2, 2, 1, 64, 0), (1, 70, 1, 128, 32)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("layout", [K.HALF, K.INTERLEAVED])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_apply_and_gradient(lib, shape, layout, dtype):
    import torch
    tokens, hq, hk, dim, rotary = shape
    rng = np.random.default_rng(dim + rotary + tokens)
    scaling = "ramp" if rotary > 2 else "none"
    rope = rope_of(lib, rotary, layout, scaling=scaling) if rotary else None
    magnitude = float(rope.magnitude) if rope else 1.0
    pos = rng.integers(0, 1 << 20, tokens).astype(np.int32)
    pos[0] = 2 ** 31 - 1 if tokens > 2 else 0
    angles = K.rope_angles(pos, K.rope_turns(rotary, 10000.0, scaling, **SCALINGS[scaling])) if rotary else np.zeros((tokens, 0))
    dpos = torch.from_numpy(pos).cuda()
    xs, gs, ws, outs, gouts, gws = [], [], [], [], [], []
    for h in (hq, hk):
        if not h:
            continue
        xs.append(make(tokens, h, dim, dtype, rng, gap=8 * (dim % 16 == 0))[1])
        gs.append(make(tokens, h, dim, dtype, rng)[1])
        ws.append(torch.from_numpy(1 + 0.5 * rng.standard_normal(dim)).to(types(torch)[dtype]).cuda())
        outs.append(torch.full((tokens, h, dim), float("nan"), dtype=types(torch)[dtype], device="cuda"))
        gouts.append(torch.full_like(outs[-1], float("nan")))
        gws.append(torch.full((dim,), float("nan"), device="cuda"))
    if tokens > 3:
        xs[0][1] = 0.0          # a token of zeros
        xs[0][2] *= 2.0 ** -12
    n = len(xs)
    rows = [lib.NormRows.of(x, w, o) for x, w, o in zip(xs, ws, outs)] + [None]
    lib.libra_norm_rope_apply(0, rope, rows[0], rows[1], dtype_of(lib, dtype), dpos.data_ptr(), tokens, dim, EPS, stream())
    ws_bytes = lib.libra_norm_rope_workspace_size(0, dim)
    space = torch.full((ws_bytes,), 0xEE, dtype=torch.uint8, device="cuda")
    grads = [lib.NormGrads.of(x, g, w, o, gw) for x, g, w, o, gw in zip(xs, gs, ws, gouts, gws)] + [None]
    lib.libra_norm_rope_gradient(0, rope, grads[0], grads[1], dtype_of(lib, dtype), dpos.data_ptr(), tokens, dim, EPS, space.data_ptr(),
                                 ws_bytes, stream())
    eps = float(np.float32(EPS))
    for i in range(n):
        x, g, w = f64(xs[i]), f64(gs[i]), f64(ws[i])
        ref, e = forward(x, w, angles, layout, magnitude, eps)
        assert np.all(np.abs(f64(outs[i]) - ref) <= rounded(ref, e, dtype)), i
        dx, dw, e, ew = gradient(x, g, w, angles, layout, magnitude, eps)
        err = np.abs(f64(gouts[i]) - dx)
        assert np.all(err <= rounded(dx, e, dtype)), (i, float((err / rounded(dx, e, dtype)).max()))
        assert np.all(np.abs(f64(gws[i]) - dw) <= ew + U * np.abs(dw) + 2.0 ** -126), i


def test_the_reference_against_differences():
    """The formula's gradient is that of the forward map, in float64; central differences of step 2^-17."""
    rng = np.random.default_rng(3)
    tokens, heads, dim = 3, 2, 16
    x, dy, w = rng.standard_normal((tokens, heads, dim)), rng.standard_normal((tokens, heads, dim)), rng.standard_normal(dim)
    angles = rng.standard_normal((tokens, 4))
    for layout in (K.HALF, K.INTERLEAVED):
        f = lambda a, b: (forward(a, b, angles, layout, 1.25)[0] * dy).sum()
        dx, dw = gradient(x, dy, w, angles, layout, 1.25)[:2]
        h = 2.0 ** -17
        for at in np.ndindex(x.shape):
            d = np.zeros_like(x)
            d[at] = h
            assert abs((f(x + d, w) - f(x - d, w)) / (2 * h) - dx[at]) < 1e-7
        for c in range(dim):
            d = np.zeros(dim)
            d[c] = h
            assert abs((f(x, w + d) - f(x, w - d)) / (2 * h) - dw[c]) < 1e-7


@pytest.mark.parametrize("layout", [K.HALF, K.INTERLEAVED])
@pytest.mark.parametrize("dim,rotary", [(64, 32), (128, 128)])
def test_strides_in_place_and_unaligned(lib, dim, rotary, layout):
    """Rows inside wider buffers, on and off 16-byte boundaries: the same bits out of place and in place, what lies between stays."""
    import torch
    rng = np.random.default_rng(dim)
    tokens, heads = 19, 3
    rope, pos = rope_of(lib, rotary, layout), torch.from_numpy(rng.integers(0, 5000, tokens).astype(np.int32)).cuda()
    angles = K.rope_angles(pos.cpu().numpy(), K.rope_turns(rotary, 10000.0))
    ws = torch.empty(lib.libra_norm_rope_workspace_size(0, dim), dtype=torch.uint8, device="cuda")
    for off, gap in ((0, 0), (0, 24), (1, 0), (3, 5), (8, 8)):
        wide, x = make(tokens, heads, dim, "bf16", rng, gap, off)
        gwide, g = make(tokens, heads, dim, "bf16", rng, gap, off)
        w = torch.from_numpy(rng.standard_normal(dim + 1)).to(torch.bfloat16).cuda()[off % 2:][:dim]
        before, gbefore = wide.clone(), gwide.clone()
        keep = torch.ones_like(wide, dtype=torch.bool)
        torch.as_strided(keep, x.shape, x.stride(), off).fill_(False)
        out, gout = (torch.full((tokens, heads, dim), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        gw = torch.empty(dim, device="cuda")
        apply = lambda o: lib.libra_norm_rope_apply(0, rope, lib.NormRows.of(x, w, o), None, lib.ROPE_BF16, pos.data_ptr(), tokens, dim, EPS, stream())
        back = lambda o: lib.libra_norm_rope_gradient(0, rope, lib.NormGrads.of(x, g, w, o, gw), None, lib.ROPE_BF16, pos.data_ptr(), tokens, dim,
                                                      EPS, ws.data_ptr(), ws.numel(), stream())
        apply(out)
        back(gout)
        assert torch.equal(wide, before) and torch.equal(gwide, gbefore)
        ref, e = forward(f64(x), f64(w), angles, layout, 1.0, float(np.float32(EPS)))
        assert np.all(np.abs(f64(out) - ref) <= rounded(ref, e, "bf16"))
        dx, dw, e, ew = gradient(f64(x), f64(g), f64(w), angles, layout, 1.0, float(np.float32(EPS)))
        assert np.all(np.abs(f64(gout) - dx) <= rounded(dx, e, "bf16")) and np.all(np.abs(f64(gw) - dw) <= ew + U * np.abs(dw))
        first = gw.clone()
        back(g)
        assert torch.equal(g, gout) and torch.equal(gw, first) and torch.equal(gwide[keep], gbefore[keep])
        g.copy_(torch.as_strided(gbefore, g.shape, g.stride(), off))
        apply(x)
        assert torch.equal(x, out) and torch.equal(wide[keep], before[keep])
        x.copy_(torch.as_strided(before, x.shape, x.stride(), off))
        back(x)
        assert torch.equal(x, gout) and torch.equal(gw, first)


def test_head_major_rows_on_another_stream(lib):
    import torch
    rng = np.random.default_rng(9)
    tokens, heads, dim = 50, 6, 64
    rope, pos = rope_of(lib, 64), torch.from_numpy(rng.integers(0, 5000, tokens).astype(np.int32)).cuda()
    x = torch.from_numpy(rng.standard_normal((heads, tokens, dim))).to(torch.bfloat16).cuda()
    w, out = torch.ones(dim, dtype=torch.bfloat16, device="cuda"), torch.full_like(x, float("nan"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lib.libra_norm_rope_apply(0, rope, lib.NormRows.of(x.transpose(0, 1), w, out.transpose(0, 1)), None, lib.ROPE_BF16, pos.data_ptr(), tokens,
                                  dim, EPS, stream())
    side.synchronize()
    ref, e = forward(f64(x.transpose(0, 1)), np.ones(dim), K.rope_angles(pos.cpu().numpy(), K.rope_turns(64, 10000.0)), K.HALF, 1.0)
    assert np.all(np.abs(f64(out.transpose(0, 1)) - ref) <= rounded(ref, e, "bf16"))


@pytest.mark.parametrize("dim", [128, 40])
def test_many_rows_the_same_bits_and_recorded(lib, dim):
    """More rows than the device holds at once, through both kinds of kernels; two graphs with a workspace each, replayed together."""
    import torch
    rng = np.random.default_rng(dim)
    tokens, hq, hk = 4001, 8, 3
    rope, pos = rope_of(lib, dim), torch.from_numpy(rng.integers(0, 5000, tokens).astype(np.int32)).cuda()
    x, g = ([torch.from_numpy(rng.standard_normal((tokens, h, dim)).astype(np.float32)).cuda() for h in (hq, hk)] for _ in range(2))
    w = [torch.from_numpy(rng.standard_normal(dim).astype(np.float32)).cuda() for _ in range(2)]

    def call(o, gw, ws):
        q, k = (lib.NormGrads.of(*a) for a in zip(x, g, w, o, gw))
        lib.libra_norm_rope_gradient(0, rope, q, k, lib.ROPE_F32, pos.data_ptr(), tokens, dim, EPS, ws.data_ptr(), ws.numel(), stream())

    sets = [([torch.empty_like(t) for t in x], [torch.empty_like(t) for t in w],
             torch.empty(lib.libra_norm_rope_workspace_size(0, dim), dtype=torch.uint8, device="cuda")) for _ in range(3)]
    call(*sets[0])
    for i in range(2):   # against the same formula in 64 bits, the whole batch at once
        xd, gd, wd = x[i].double(), g[i].double(), w[i].double()
        angle = torch.from_numpy(K.rope_angles(np.arange(5000), K.rope_turns(dim, 10000.0))).cuda()[pos.long()][:, None]
        a, b = gd[..., :dim // 2], gd[..., dim // 2:]
        t = torch.cat((a * angle.cos() + b * angle.sin(), b * angle.cos() - a * angle.sin()), -1)
        r = (xd.square().mean(-1, keepdim=True) + float(np.float32(EPS))).rsqrt()
        n = xd * r
        dx = r * (wd * t - n * (wd * t * n).mean(-1, keepdim=True))
        assert float((sets[0][0][i].double() - dx).abs().max()) <= 2.0 ** -17 * float(dx.abs().max())
        size = (t.abs() * n.abs()).sum((0, 1))
        # 2^-20 of a term for the rotation, the norm and the product; additions: under 2^9 one after another in any of the stages
        assert bool(((sets[0][1][i].double() - (t * n).sum((0, 1))).abs() <= (2.0 ** -20 + 2.0 ** -14) * size).all())
    graphs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    for s, st in zip(sets[1:], streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            call(*s)
        graphs.append(graph)
    for _ in range(5):
        for s in sets[1:]:
            for t in s[0] + s[1]:
                t.fill_(float("nan"))
        torch.cuda.synchronize()
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
        torch.cuda.synchronize()
        for s in sets[1:]:
            assert all(torch.equal(a, b) for a, b in zip(s[0] + s[1], sets[0][0] + sets[0][1]))
    del graphs


def torch_forward(x, w, pos, rotary, layout, eps=EPS):
    """The forward map in float64 on the device, and the bound before the last rounding."""
    import torch
    x, w = x.double(), w.double()
    r = (x.square().mean(-1, keepdim=True) + float(np.float32(eps))).rsqrt()
    n, D = x * r * w, x.shape[-1]
    theta = torch.tensor([10000.0 ** (-2.0 * i / rotary) for i in range(rotary // 2)], dtype=torch.float64, device=x.device)
    a = pos.double()[:, None, None] * theta
    h = rotary // 2
    u, v = (n[..., :h], n[..., h:rotary]) if layout == K.HALF else (n[..., 0:rotary:2], n[..., 1:rotary:2])
    yu, yv, both = u * a.cos() - v * a.sin(), u * a.sin() + v * a.cos(), u.abs() + v.abs()
    y, e = n.clone(), (D * U / 2 + 4 * U) * n.abs()
    for at, val in ((0, yu), (1, yv)):
        sl = slice(at * h, at * h + h) if layout == K.HALF else slice(at, rotary, 2)
        # float64 angles of up to 2^13 radians are right to 2^-39
        y[..., sl], e[..., sl] = val, (2.0 ** -21 + D * U / 2 + 4 * U + 2.0 ** -38) * both
    return y, e


@pytest.mark.parametrize("layout", [K.HALF, K.INTERLEAVED])
@pytest.mark.parametrize("dim,rotary", [(128, 128), (80, 40), (256, 64), (48, 12)])
@pytest.mark.parametrize("hq,hk", [(24, 5), (7, 7), (33, 0)])
def test_runs_that_begin_anywhere(lib, hq, hk, dim, rotary, layout):
    """More steps than warps, so that the warps' runs begin and end within a token, a kind and a group of heads."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(dim + hq)
    tokens = 2503
    draw = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    rope, pos = rope_of(lib, rotary, layout), torch.randint(0, 8000, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    xs, ws = [draw(tokens, h, dim) for h in (hq, hk) if h], [draw(dim) for _ in range(2)]
    outs = [torch.full_like(x, float("nan")) for x in xs]
    rows = [lib.NormRows.of(x, w, o) for x, w, o in zip(xs, ws, outs)] + [None]
    lib.libra_norm_rope_apply(0, rope, rows[0], rows[1], lib.ROPE_BF16, pos.data_ptr(), tokens, dim, EPS, stream())
    for x, w, o in zip(xs, ws, outs):
        ref, e = torch_forward(x, w, pos, rotary, layout)
        assert bool(((o.double() - ref).abs() <= e + HALF_STEP["bf16"] * (ref.abs() + e) + TINY["bf16"]).all())


@pytest.mark.parametrize("order", ["HND", "NHD"])
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_append_of_many_rows(lib, kv, order):
    import torch
    rows, hq, hkv, dim, page = 3001, 40, 8, 128, 32
    a = Append(lib, rows, hq, hkv, dim, page, order, kv, seed=7, dead={17: -1})
    a.n[0] = rows - 3
    a.pos %= 8000
    a.dpos.copy_(torch.from_numpy(a.pos))
    a.call(rope_of(lib, dim))
    n = rows - 3
    ref, e = torch_forward(a.q[:n], a.w[0], a.dpos[:n], dim, K.HALF)
    assert bool(((a.out[:n].double() - ref).abs() <= e + HALF_STEP["bf16"] * (ref.abs() + e) + TINY["bf16"]).all())
    assert bool(torch.isnan(a.out[n:]).all()) and int(a.err) == 0
    ky, ke = torch_forward(a.kn[:n], a.w[1], a.dpos[:n], dim, K.HALF)
    live = torch.from_numpy(a.slots[:n] >= 0).cuda()
    s = a.dslots[:n].long()[live]
    for pool, before, y, e, scale in ((a.k, a.k0, ky, ke, a.scales[0]), (a.v, a.v0, a.vn[:n].double(), torch.zeros_like(ky), a.scales[1])):
        now, was = (x if order == "NHD" else x.transpose(1, 2) for x in (pool, before.clone()))
        got = now[s // page, s % page]
        was[s // page, s % page] = got
        assert torch.equal(now, was)      # every other slot as it was
        if kv == "bf16":
            got, half, least = got.view(torch.bfloat16).double(), 2.0 ** -8, 2.0 ** -134
        else:
            # the float32 product with the rounded reciprocal: 2^-22; half a step of E4M3, or of its smallest numbers
            got, half, least = got.view(torch.float8_e4m3fn).double() * scale, 2.0 ** -4 + 2.0 ** -21, 2.0 ** -10 * scale
            y = y.clamp(-448 * scale, 448 * scale)
        y, e = y[live], e[live]
        assert bool(((got - y).abs() <= e + half * (y.abs() + e) + least).all())
    a.h.close()


def test_rows_far_apart_and_more_steps_than_31_bits_count(lib):
    """Tokens 2.4 GB from one another; and 1.1e9 tokens of one broadcast row, of q and of k."""
    import torch
    dim, far = 128, 1_200_000_000
    wide = torch.zeros(2 * far + 4 * dim, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(wide, (3, 2, dim), (far, 2 * dim, 1), 0)
    x.copy_(torch.randn((3, 2, dim), device="cuda"))
    w, pos = torch.ones(dim, dtype=torch.bfloat16, device="cuda"), torch.tensor([5, 6, 7], dtype=torch.int32, device="cuda")
    near, dense = x.contiguous(), torch.empty((3, 2, dim), dtype=torch.bfloat16, device="cuda")
    rope = rope_of(lib, dim)
    lib.libra_norm_rope_apply(0, rope, lib.NormRows.of(near, w, dense), None, lib.ROPE_BF16, pos.data_ptr(), 3, dim, EPS, stream())
    lib.libra_norm_rope_apply(0, rope, lib.NormRows.of(x, w, x), None, lib.ROPE_BF16, pos.data_ptr(), 3, dim, EPS, stream())
    assert torch.equal(x, dense)
    del wide, x
    tokens, dim = 1_100_000_000, 8
    row = torch.randn((1, 1, dim), device="cuda").to(torch.bfloat16)
    w, outs = torch.ones(dim, dtype=torch.bfloat16, device="cuda"), [torch.zeros((tokens, 1, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    q, k = (lib.NormRows.of(row.expand(tokens, 1, dim), w, o) for o in outs)
    assert q.x_stride_token == 0
    lib.libra_norm_rope_apply(0, None, q, k, lib.ROPE_BF16, 0, tokens, dim, EPS, stream())
    for o in outs:
        words = o.view(torch.int64).view(-1, 2)
        for at in range(0, tokens, 1 << 27):
            part = words[at:at + (1 << 27)]
            assert bool((part == words[0]).all())
    assert float(outs[0][0].abs().max()) > 0 and torch.equal(outs[0][0], outs[1][0])


def test_recorded_where_the_kernel_needs_more_shared_memory_than_the_default(lib):
    """Heads of 1022 channels in float32 through shared memory, gradient of q and k, first call within the recording."""
    import torch
    rng = np.random.default_rng(2)
    x, g = ([torch.from_numpy(rng.standard_normal((5, h, 1022)).astype(np.float32)).cuda() for h in (2, 1)] for _ in range(2))
    w = [torch.from_numpy(rng.standard_normal(1022).astype(np.float32)).cuda() for _ in range(2)]
    o, gw = [torch.empty_like(t) for t in x], [torch.empty_like(t) for t in w]
    pos = torch.arange(5, dtype=torch.int32, device="cuda")
    ws = torch.empty(lib.libra_norm_rope_workspace_size(0, 1022), dtype=torch.uint8, device="cuda")
    q, k = (lib.NormGrads.of(*a) for a in zip(x, g, w, o, gw))
    rope = rope_of(lib, 254)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.libra_norm_rope_gradient(0, rope, q, k, lib.ROPE_F32, pos.data_ptr(), 5, 1022, EPS, ws.data_ptr(), ws.numel(), stream())
    graph.replay()
    angles = K.rope_angles(pos.cpu().numpy(), K.rope_turns(254, 10000.0))
    for i in range(2):
        dx, dw, e, ew = gradient(f64(x[i]), f64(g[i]), f64(w[i]), angles, K.HALF, 1.0, float(np.float32(EPS)))
        assert np.all(np.abs(f64(o[i]) - dx) <= rounded(dx, e, "f32")) and np.all(np.abs(f64(gw[i]) - dw) <= ew + U * np.abs(dw))
    del graph


def test_no_tokens(lib):
    import torch
    x, w = torch.zeros((1, 2, 64), device="cuda"), torch.ones(64, device="cuda")
    gw = torch.full((64,), float("nan"), device="cuda")
    ws = torch.empty(lib.libra_norm_rope_workspace_size(0, 64), dtype=torch.uint8, device="cuda")
    lib.libra_norm_rope_apply(0, None, lib.NormRows.of(x, w, x), None, lib.ROPE_F32, 0, 0, 64, EPS, stream())
    lib.libra_norm_rope_gradient(0, None, lib.NormGrads.of(x, x, w, x, gw), None, lib.ROPE_F32, 0, 0, 64, EPS, ws.data_ptr(), ws.numel(), stream())
    assert bool((gw == 0).all())


def test_a_row_that_is_not_finite_stays_alone(lib):
    import torch
    x = torch.ones((6, 4, 128), dtype=torch.bfloat16, device="cuda")
    x[2, 1, 5], x[4, 3, 127] = float("nan"), float("inf")
    w, out = torch.ones(128, dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
    lib.libra_norm_rope_apply(0, None, lib.NormRows.of(x, w, out), None, lib.ROPE_BF16, 0, 6, 128, EPS, stream())
    bad = torch.isnan(out).any(-1)
    assert bool(bad[2, 1]) and bool(bad[4, 3]) and int(bad.sum()) == 2
    assert bool(torch.isnan(out[2, 1]).all()) and int(torch.isnan(out[4, 3]).sum()) == 1 and float(out[4, 3, 0]) == 0.0


# ----------------------------------------------------------------------------------------------------------------- append
class Append:
    """New rows with positions and slots of their own."""

    def __init__(self, lib, rows, hq=4, hkv=2, dim=64, page=16, order="HND", kv="bf16", seed=0, fused=True, norm=True, pool=None, dead=()):
        import torch
        self.lib, self.kv, self.order, self.page, self.rows, self.norm = lib, kv, order, page, rows, norm
        rng = np.random.default_rng(seed)
        self.pool = pool or rows // page + 3
        shape = (self.pool, hkv, page, dim) if order == "HND" else (self.pool, page, hkv, dim)
        top, kind = (1 << 15, np.int16) if kv == "bf16" else (256, np.uint8)
        self.k, self.v = (torch.from_numpy(rng.integers(0, top, shape).astype(kind)).cuda() for _ in range(2))
        self.k0, self.v0 = self.k.clone(), self.v.clone()
        proj = torch.from_numpy(rng.standard_normal((rows, hq + 2 * hkv, dim))).to(torch.bfloat16).cuda()
        parts = proj[:, :hq], proj[:, hq:hq + hkv], proj[:, hq + hkv:]
        self.q, self.kn, self.vn = parts if fused else tuple(x.contiguous() for x in parts)
        self.w = [torch.from_numpy(1 + 0.5 * rng.standard_normal(dim)).to(torch.bfloat16).cuda() for _ in range(2)]
        self.pos = rng.integers(0, 1 << 17, rows).astype(np.int32)
        self.slots = rng.permutation(self.pool * page)[:rows].astype(np.int32)
        for i, s in dict(dead).items():
            self.slots[i] = s
        self.dpos, self.dslots = torch.from_numpy(self.pos).cuda(), torch.from_numpy(self.slots).cuda()
        self.out = torch.full((rows, hq, dim), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.n = torch.tensor([rows], dtype=torch.int32, device="cuda")
        strides = (0, 0, 0) if order == "HND" else (page * hkv * dim, dim, hkv * dim)
        self.h = lib.Handle(hq, hkv, dim, self.pool, 1, 4, page_size=page, kv_strides=strides)
        self.scales = (1.0, 1.0)
        if kv == "e4m3":
            self.scales = (0.0371, 0.25)
            self.h.set_kv_dtype(lib.KV_E4M3, *self.scales)

    def call(self, rope, n_rows=True, q=True, out=None):
        out = self.out if out is None else out
        args = (self.q.data_ptr(), self.q.stride(0), out.data_ptr(), out.stride(0)) if q else (0, 0, 0, 0)
        w = [x.data_ptr() if self.norm else 0 for x in self.w]
        self.h.norm_rope_append(rope, *w, EPS, *args, self.kn.data_ptr(), self.vn.data_ptr(), self.kn.stride(0), self.dpos.data_ptr() if rope else 0,
                                self.dslots.data_ptr(), self.n.data_ptr() if n_rows else 0, self.rows, self.k.data_ptr(), self.v.data_ptr(),
                                self.err.data_ptr(), stream())

    def check(self, rotary, layout, turns, magnitude=1.0, rows=None, q=True):
        """q and both pools, every element: named slots within the bound, all others as they were."""
        rows = self.rows if rows is None else rows
        angles = K.rope_angles(self.pos[:rows], turns) if rotary else np.zeros((rows, 0))
        qx, kx, vx = (f64(x[:rows]) for x in (self.q, self.kn, self.vn))
        eps = float(np.float32(EPS))
        if q:
            ref, e = forward(qx, f64(self.w[0]), angles, layout, magnitude, eps, self.norm)
            got = f64(self.out)
            assert np.all(np.abs(got[:rows] - ref) <= rounded(ref, e, "bf16"))
            assert np.all(np.isnan(got[rows:]))
        ky, ke = forward(kx, f64(self.w[1]), angles, layout, magnitude, eps, self.norm)
        for pool, before, y, e, scale in ((self.k, self.k0, ky, ke, self.scales[0]), (self.v, self.v0, vx, np.zeros_like(vx), self.scales[1])):
            now, was = pool.cpu().numpy(), before.cpu().numpy().copy()
            if self.order == "HND":
                now, was = now.transpose(0, 2, 1, 3), was.transpose(0, 2, 1, 3)
            for row, slot in enumerate(self.slots[:rows]):
                if 0 <= slot < self.pool * self.page:
                    at = slot // self.page, slot % self.page
                    if self.kv == "bf16":
                        got = O.bf16_bits_to_f64(now[at].view(np.uint16))
                        assert np.all(np.abs(got - y[row]) <= np.where(e[row] > 0, rounded(y[row], e[row], "bf16"), 0.0))
                    else:   # between the codes of the two ends of what the float32 value, times the rounded reciprocal, may be
                        z, ez = y[row] / scale, (e[row] + 2.0 ** -22 * np.abs(y[row])) / scale
                        lo, hi = (K.e4m3_values()[K.e4m3_encode(z + s * ez)] for s in (-1, 1))
                        got = K.e4m3_values()[now[at]]
                        assert np.all((got >= lo) & (got <= hi))
                    was[at] = now[at]
            assert np.array_equal(now, was)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("order", ["HND", "NHD"])
@pytest.mark.parametrize("layout", [K.HALF, K.INTERLEAVED])
@pytest.mark.parametrize("page,dim,rotary,scaling,norm", [(16, 64, 64, "none", True), (32, 128, 64, "ramp", True), (64, 128, 128, "bands", False),
                                                          (16, 64, 24, "linear", True), (16, 128, 10, "none", True)])
def test_append(lib, page, dim, rotary, scaling, norm, layout, order, kv):
    rope = rope_of(lib, rotary, layout, scaling=scaling)
    a = Append(lib, 61, 10 if page == 32 else 4, 2, dim, page, order, kv, seed=page + dim, fused=page == 16, norm=norm, dead={3: -1, 60: -1})
    a.call(rope)
    assert int(a.err) == 0
    a.check(rotary, layout, K.rope_turns(rotary, 10000.0, scaling, **SCALINGS[scaling]), float(rope.magnitude))
    a.h.close()


def test_append_without_q_rotation_and_count(lib):
    import torch
    rope, turns = rope_of(lib, 64), K.rope_turns(64, 10000.0)
    a = Append(lib, 30, seed=2)
    a.call(rope, n_rows=False, q=False)
    a.check(64, K.HALF, turns, q=False)
    assert bool(torch.isnan(a.out).all())
    b = Append(lib, 30, seed=2)
    b.call(None)
    b.check(0, K.HALF, [])
    c = Append(lib, 30, seed=2)
    c.n[0] = 11
    c.call(rope)
    c.check(64, K.HALF, turns, rows=11)
    d = Append(lib, 30, seed=2, fused=False)
    d.call(rope, out=d.q)
    assert torch.equal(d.k, a.k)
    e = Append(lib, 30, seed=2)
    e.call(rope)
    assert torch.equal(d.q, e.out)
    for x in (a, b, c, d, e):
        x.h.close()


def test_append_without_norms_is_the_append_of_the_chunk_operators(lib):
    """The same bits as libra_rope_append where positions are the slots' own."""
    import torch
    rope = rope_of(lib, 128)
    for kv in ("bf16", "e4m3"):
        a, b = (Append(lib, 50, 8, 2, 128, kv=kv, seed=4, norm=False, pool=4) for _ in range(2))
        a.pos = np.arange(7, 57).astype(np.int32)
        table = np.array([[2, 0, 3, 1]], np.int32)
        a.slots = (table[0, a.pos // 16] * 16 + a.pos % 16).astype(np.int32)
        a.dpos.copy_(torch.from_numpy(a.pos)); a.dslots.copy_(torch.from_numpy(a.slots))
        a.call(rope)
        dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        off, lens, bt = dev([0, 50]), dev([57]), dev(table)
        b.h.rope_append(rope, b.q.data_ptr(), b.q.stride(0), b.out.data_ptr(), b.out.stride(0), b.kn.data_ptr(), b.vn.data_ptr(), b.kn.stride(0),
                        off.data_ptr(), lens.data_ptr(), bt.data_ptr(), 1, 50, b.k.data_ptr(), b.v.data_ptr(), b.err.data_ptr(), stream())
        assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v) and torch.equal(a.out, b.out)
        a.h.close(); b.h.close()


def test_append_slots_outside_the_pool(lib):
    a = Append(lib, 20, seed=5, dead={0: -2, 7: 2 ** 31 - 1, 19: -1})
    a.slots[8] = a.pool * a.page
    a.dslots[8] = a.pool * a.page
    a.call(rope_of(lib, 64))
    assert int(a.err) == lib.ERR_BAD_PAGE_ID
    a.check(64, K.HALF, K.rope_turns(64, 10000.0))
    a.h.close()


def test_append_at_the_far_end_of_a_large_pool(lib):
    """Slots past 2^32 bytes into the pools."""
    import torch
    pages = 300000   # 300000 x 1 x 64 x 128 x 2 bytes = 4.9 GB each
    h = lib.Handle(2, 1, 128, pages, 1, 4, page_size=64)
    k, v = (torch.zeros((pages, 1, 64, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x = torch.randn((3, 4, 128), device="cuda").to(torch.bfloat16)
    slots = torch.tensor([pages * 64 - 1, 5, 270000 * 64 + 13], dtype=torch.int32, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.empty((3, 2, 128), dtype=torch.bfloat16, device="cuda")
    h.norm_rope_append(None, 0, 0, EPS, x.data_ptr(), x.stride(0), out.data_ptr(), out.stride(0), x[:, 2:].data_ptr(), x[:, 3:].data_ptr(), x.stride(0), 0,
                       slots.data_ptr(), 0, 3, k.data_ptr(), v.data_ptr(), err.data_ptr(), stream())
    s = slots.long()
    assert int(err) == 0 and torch.equal(out, x[:, :2])
    assert torch.equal(k[s // 64, 0, s % 64], x[:, 2]) and torch.equal(v[s // 64, 0, s % 64], x[:, 3])
    assert int((k != 0).any(-1).sum()) == 3 and int((v != 0).any(-1).sum()) == 3
    h.close()


def test_append_refused(lib):
    a = Append(lib, 20)
    p = lambda x: x.data_ptr()
    rope = rope_of(lib, 64)
    good = [rope, p(a.w[0]), p(a.w[1]), EPS, p(a.q), a.q.stride(0), p(a.out), a.out.stride(0), p(a.kn), p(a.vn), a.kn.stride(0), p(a.dpos), p(a.dslots),
            p(a.n), 20, p(a.k), p(a.v), p(a.err), 0]
    for i, bad in [(3, 0.0), (3, -1e-6), (3, float("nan")), (3, 1e-42), (4, 0), (6, 0), (8, 0), (9, 0), (11, 0), (12, 0), (15, 0), (16, 0), (17, 0),
                   (14, -1), (1, p(a.w[0]) + 2), (5, 100), (5, 257), (10, 100), (10, 129), (4, p(a.q) + 2), (12, p(a.dslots) + 1)]:
        args = list(good)
        args[i] = bad
        with pytest.raises(lib.LibraError) as e:
            a.h.norm_rope_append(*args)
        assert e.value.status == lib.INVALID_ARGUMENT, i
    args = list(good)
    args[0] = rope_of(lib, 128)
    with pytest.raises(lib.LibraError) as e:
        a.h.norm_rope_append(*args)
    assert e.value.status == lib.UNSUPPORTED_SHAPE
    a.h.set_kv_dtype(lib.KV_E4M3, 1e-40, 1.0)
    with pytest.raises(lib.LibraError) as e:
        a.h.norm_rope_append(*good)
    assert e.value.status == lib.INVALID_ARGUMENT
    a.h.close()


@pytest.mark.parametrize("dim", [128, 24])
def test_small_rows_and_a_small_epsilon(lib, dim):
    """Rows far below the square root of epsilon, and an epsilon of 2^-100: r is up to 2^50, what is returned is no more than that."""
    import torch
    rng = np.random.default_rng(dim)
    x = torch.from_numpy((rng.standard_normal((6, 4, dim)) * np.array([1, 2.0 ** -30, 2.0 ** -52, 2.0 ** -60, 0, 2.0 ** 40])[:, None, None]).astype(np.float32)).cuda()
    g, w = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda() for s in ((6, 4, dim), (dim,)))
    pos, rope = torch.arange(6, dtype=torch.int32, device="cuda"), rope_of(lib, dim)
    out, gx, gw = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w)
    ws = torch.empty(lib.libra_norm_rope_workspace_size(0, dim), dtype=torch.uint8, device="cuda")
    angles = K.rope_angles(np.arange(6), K.rope_turns(dim, 10000.0))
    for eps in (1e-6, 2.0 ** -100):
        lib.libra_norm_rope_apply(0, rope, lib.NormRows.of(x, w, out), None, lib.ROPE_F32, pos.data_ptr(), 6, dim, eps, stream())
        lib.libra_norm_rope_gradient(0, rope, lib.NormGrads.of(x, g, w, gx, gw), None, lib.ROPE_F32, pos.data_ptr(), 6, dim, eps, ws.data_ptr(), ws.numel(), stream())
        e64 = float(np.float32(eps))
        ref, e = forward(f64(x), f64(w), angles, K.HALF, 1.0, e64)
        assert np.all(np.abs(f64(out) - ref) <= rounded(ref, e, "f32"))
        dx, dw, e, ew = gradient(f64(x), f64(g), f64(w), angles, K.HALF, 1.0, e64)
        assert np.all(np.abs(f64(gx) - dx) <= rounded(dx, e, "f32")) and np.all(np.abs(f64(gw) - dw) <= ew + U * np.abs(dw))
