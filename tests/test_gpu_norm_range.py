"""Norms at the ends of what float32 holds: epsilons next to the smallest normal number.  Bounds as derived in test_gpu_norm_rope.py; rows
held by a group of lanes (64 channels) and through shared memory (30 channels)."""
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
