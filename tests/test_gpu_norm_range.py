"""Norms at the ends of what float32 holds: epsilons next to the smallest normal number, squares whose sum has no place in
float32, gradients whose product with x has none although every term of the result has one.  Bounds as derived in
test_gpu_norm_rope.py; rows held by a group of lanes (64 channels) and through shared memory (30 channels)."""
import numpy as np
import pytest

from oracle import chunk_oracle as K

from test_gpu_norm_rope import U, dtype_of, f64, forward, gradient, rounded, stream
from test_rope import rope_of

pytestmark = pytest.mark.gpu


def run(lib, x, g, w, dtype, eps):
    import torch
    T = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    tokens, heads, dim = x.shape
    x, g, w = (torch.from_numpy(a).to(T).cuda() for a in (x, g, w))
    pos, rope = torch.arange(tokens, dtype=torch.int32, device="cuda"), rope_of(lib, dim)
    angles = K.rope_angles(np.arange(tokens), K.rope_turns(dim, 10000.0))
    out, gx, gw = torch.empty_like(x), torch.empty_like(x), torch.empty(dim, device="cuda")
    ws = torch.empty(lib.libra_norm_rope_workspace_size(0, dim), dtype=torch.uint8, device="cuda")
    kind = dtype_of(lib, dtype)
    lib.libra_norm_rope_apply(0, rope, lib.NormRows.of(x, w, out), None, kind, pos.data_ptr(), tokens, dim, eps, stream())
    lib.libra_norm_rope_gradient(0, rope, lib.NormGrads.of(x, g, w, gx, gw), None, kind, pos.data_ptr(), tokens, dim, eps, ws.data_ptr(), ws.numel(),
                                 stream())
    e64 = float(np.float32(eps))
    ref, e = forward(f64(x), f64(w), angles, K.HALF, 1.0, e64)
    assert np.all(np.abs(f64(out) - ref) <= rounded(ref, e, dtype))
    dx, dw, e, ew = gradient(f64(x), f64(g), f64(w), angles, K.HALF, 1.0, e64)
    assert np.all(np.isfinite(dx)) and np.abs(dx).max() > 2.0 ** -100
    assert np.all(np.abs(f64(gx) - dx) <= rounded(dx, e, dtype))
    assert np.all(np.abs(f64(gw) - dw) <= ew + U * np.abs(dw) + 2.0 ** -126)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 30])
@pytest.mark.parametrize("eps", [2.0 ** -126, 1.5 * 2.0 ** -126, 2.0 ** -125, 2.0 ** -124])
def test_the_smallest_epsilons(lib, eps, dim, dtype):
    rng = np.random.default_rng(dim)
    x, g, w = rng.standard_normal((6, 3, dim)), rng.standard_normal((6, 3, dim)), rng.standard_normal(dim)
    # zeros; rows whose squares count as zero beside epsilon; rows that decide alone
    x *= np.array([0.0, 2.0 ** -80, 1.0, 0.0, 2.0 ** -40, 2.0 ** 40])[:, None, None]
    run(lib, x, g, w, dtype, eps)


@pytest.mark.parametrize("dim", [64, 30])
def test_rows_whose_squares_have_no_sum(lib, dim):
    """Zeros for the row, which adds nothing to the weight's gradient, NaN for a channel that is infinite, and its own row alone."""
    import torch
    x, g = (torch.ones((3, 4, dim), device="cuda") for _ in range(2))
    x[0, 2], x[2, 0], x[2, 1] = 2.0 ** 70, 2.0 ** 62.5, -2.0 ** 63      # the means of the last two have a place in float32
    w, out, gx, gw = torch.ones(dim, device="cuda"), torch.empty_like(x), torch.empty_like(x), torch.empty(dim, device="cuda")
    ws = torch.empty(lib.libra_norm_rope_workspace_size(0, dim), dtype=torch.uint8, device="cuda")
    lib.libra_norm_rope_apply(0, None, lib.NormRows.of(x, w, out), None, lib.ROPE_F32, 0, 3, dim, 1e-6, stream())
    lib.libra_norm_rope_gradient(0, None, lib.NormGrads.of(x, g, w, gx, gw), None, lib.ROPE_F32, 0, 3, dim, 1e-6, ws.data_ptr(), ws.numel(), stream())
    past = x.abs()[..., 0] > 1
    assert bool((out[past] == 0).all()) and bool((gx[past] == 0).all())
    # 1 / sqrt(1 + 1e-6) = 1 - 5e-7 for the others, each of them g x r; steps of 2^-24 (dim / 2 of them at most, and nine additions)
    assert bool(((out[~past] - 1).abs() <= 1e-6 + dim * U).all()) and bool(((gw - 9).abs() <= 9 * (1e-6 + dim * U)).all())
    x[1, 3, 5], x[0, 0, 7] = float("inf"), float("nan")
    lib.libra_norm_rope_apply(0, None, lib.NormRows.of(x, w, out), None, lib.ROPE_F32, 0, 3, dim, 1e-6, stream())
    bad = torch.isnan(out)
    assert bad[1, 3].tolist() == [c == 5 for c in range(dim)] and bool((out[1, 3][~bad[1, 3]] == 0).all())
    assert bool(bad[0, 0].all()) and int(bad.sum()) == dim + 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 30])
@pytest.mark.parametrize("x_scale,g_scale,w_scale", [(-50, -80, 0), (-50, -99, 0), (58, 75, 0), (60, 90, -5), (20, 110, 3), (-40, -60, -25), (0, 0, 0)])
def test_gradients_far_from_one(lib, x_scale, g_scale, w_scale, dim, dtype):
    rng = np.random.default_rng(100 + dim - x_scale)
    x, g, w = (rng.standard_normal(s) * 2.0 ** k for s, k in (((5, 3, dim), x_scale), ((5, 3, dim), g_scale), (dim, w_scale)))
    if g_scale + w_scale < 70:   # dx of a row of zeros is 2^50 w g: 2^125 and more at the others' scales, of which elements pass 2^128
        x[1, 1] = 0.0
    run(lib, x, g, w, dtype, 2.0 ** -100)
