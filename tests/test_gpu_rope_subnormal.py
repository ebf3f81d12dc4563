"""Rotary positions and append on numbers below the smallest normal float32, within the bounds of test_gpu_rope, and what append
copies: the same bits."""
import numpy as np
import pytest

from oracle import chunk_oracle as K

from test_gpu_rope import Batch, apply, bound, types
from test_rope import rope_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("direction", ["forward", "gradient"])
@pytest.mark.parametrize("layout", [K.HALF, K.INTERLEAVED])
@pytest.mark.parametrize("dtype,size", [("f32", 2.0 ** -130), ("f32", 2.0 ** -126), ("bf16", 2.0 ** -128), ("f16", 2.0 ** -20)])
@pytest.mark.parametrize("rotary", [64, 10])
def test_small_numbers(lib, rotary, dtype, size, layout, direction):
    import torch
    rng = np.random.default_rng(51)
    rope = rope_of(lib, rotary, layout)
    x = torch.from_numpy(rng.standard_normal((40, 3, 64)) * size).to("cuda").to(types(torch)[dtype])
    pos = rng.integers(0, 5000, 40).astype(np.int32)
    out = torch.full_like(x, float("nan"))
    apply(lib, rope, x, out, torch.from_numpy(pos).cuda(), dtype, lib.ROPE_GRADIENT if direction == "gradient" else lib.ROPE_FORWARD)
    xs, a = x.double().cpu().numpy(), K.rope_angles(pos, K.rope_turns(rotary, 10000.0))
    assert np.any(xs != 0)
    ref = K.rotate(xs, -a if direction == "gradient" else a, layout)
    tol = bound(xs, ref, rotary, layout, 1.0, dtype)
    # the products and the sum round by half of the smallest step too, 2^-150 each
    tol = np.where(tol > 0, tol + 3 * 2.0 ** -150 * (1 + 2.0 ** -8), 0.0)
    assert np.all(np.abs(out.double().cpu().numpy() - ref) <= tol)


@pytest.mark.parametrize("layout", [K.HALF, K.INTERLEAVED])
@pytest.mark.parametrize("rotary", [64, 32, 10])
def test_append_copies_every_bit_pattern(lib, rotary, layout):
    """v, and the channels of q and k that pass: all 65536 bf16 patterns but for the payload of a NaN."""
    import torch
    b = Batch(lib, [512, 1], [512, 1], hq=2, hkv=2, dim=64, seed=52)
    patterns = torch.arange(65536, dtype=torch.int32).to(torch.int16).cuda().view(torch.bfloat16)
    b.vn[:512] = patterns.view(512, 2, 64)
    b.q[:512, :, rotary:] = patterns.view(512, 2, 64)[:, :, rotary:]
    b.append(rope_of(lib, rotary, layout))
    assert int(b.err) == 0
    v = torch.cat([b.v.view(torch.bfloat16)[int(p)].transpose(0, 1) for p in b.bt[0, :32]])
    for got, ref in ((v, b.vn[:512]), (b.q_out[:512, :, rotary:], b.q[:512, :, rotary:])):
        nan = torch.isnan(ref)
        assert torch.equal(torch.isnan(got), nan)
        assert torch.equal(got.contiguous().view(torch.int16)[~nan], ref.contiguous().view(torch.int16)[~nan])
    b.h.close()
