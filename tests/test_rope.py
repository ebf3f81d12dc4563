"""Rotary positions on the CPU: the table that libra_rope_init makes against the oracle, the oracle's own pins, and what
the entry points refuse before they touch a GPU."""
import math

import numpy as np
import pytest

from oracle import attention_oracle as O
from oracle import chunk_oracle as K

SCALINGS = {
    "none": dict(),
    "linear": dict(factor=4.0),
    "base": dict(factor=8.0),
    "bands": dict(factor=8.0, low=1.0, high=4.0, original_len=8192),
    "ramp": dict(factor=4.0, low=1.0, high=32.0, original_len=4096),
}


def rope_of(lib, rotary, layout=K.HALF, base=10000.0, scaling="none", magnitude=0.0):
    kind = {"none": lib.ROPE_SCALE_NONE, "linear": lib.ROPE_SCALE_LINEAR, "base": lib.ROPE_SCALE_BASE, "bands": lib.ROPE_SCALE_BANDS,
            "ramp": lib.ROPE_SCALE_RAMP}[scaling]
    return lib.libra_rope_init(rotary, lib.ROPE_HALF if layout == K.HALF else lib.ROPE_INTERLEAVED, base, kind,
                               magnitude=magnitude, **SCALINGS[scaling])


@pytest.mark.parametrize("scaling", list(SCALINGS))
@pytest.mark.parametrize("rotary,base", [(128, 10000.0), (64, 500000.0), (256, 1e6), (10, 10000.0), (2, 10000.0)])
def test_table_equals_the_oracle(lib, rotary, base, scaling):
    if rotary == 2 and scaling == "base":
        with pytest.raises(lib.LibraError):
            rope_of(lib, rotary, base=base, scaling=scaling)
        return
    r = rope_of(lib, rotary, base=base, scaling=scaling)
    want = K.rope_turns(rotary, base, scaling, **SCALINGS[scaling])
    assert r.rotary_dim == rotary and r.layout == lib.ROPE_HALF
    for i, w in enumerate(want):
        # the library works in long double: a few units of 2^-64 relative to turns below one
        assert abs(r.turns[i] - (w >> 64)) <= 64, (i, r.turns[i], w >> 64)
    assert all(r.turns[i] == 0 for i in range(len(want), lib.ROPE_MAX_PAIRS))
    assert r.magnitude == np.float32(0.1 * math.log(4.0) + 1.0 if scaling == "ramp" else 1.0)
    assert rope_of(lib, rotary, base=base, scaling=scaling, magnitude=0.5).magnitude == 0.5


def test_whole_turns_per_position_change_nothing(lib):
    # base below one: angles of more than a turn per position
    r = lib.libra_rope_init(4, lib.ROPE_HALF, 1e-4)
    w = K.rope_turns(4, 1e-4)
    assert w[1] > 1 << 128
    assert abs(r.turns[1] - ((w[1] % (1 << 128)) >> 64)) <= 4096


def test_refusals_of_init(lib):
    bad = [
        (dict(rotary_dim=0), lib.INVALID_ARGUMENT), (dict(rotary_dim=3), lib.INVALID_ARGUMENT),
        (dict(rotary_dim=258), lib.UNSUPPORTED_SHAPE), (dict(rotary_dim=64, layout=2), lib.INVALID_ARGUMENT),
        (dict(rotary_dim=64, base=0.0), lib.INVALID_ARGUMENT), (dict(rotary_dim=64, base=float("nan")), lib.INVALID_ARGUMENT),
        (dict(rotary_dim=64, base=float("inf")), lib.INVALID_ARGUMENT), (dict(rotary_dim=64, scaling=5), lib.INVALID_ARGUMENT),
        (dict(rotary_dim=64, scaling=lib.ROPE_SCALE_LINEAR, factor=0.5), lib.INVALID_ARGUMENT),
        (dict(rotary_dim=64, scaling=lib.ROPE_SCALE_LINEAR, factor=float("nan")), lib.INVALID_ARGUMENT),
        (dict(rotary_dim=64, scaling=lib.ROPE_SCALE_BANDS, factor=2.0, low=4.0, high=4.0, original_len=8), lib.INVALID_ARGUMENT),
        (dict(rotary_dim=64, scaling=lib.ROPE_SCALE_BANDS, factor=2.0, low=1.0, high=4.0), lib.INVALID_ARGUMENT),
        (dict(rotary_dim=64, scaling=lib.ROPE_SCALE_RAMP, factor=2.0, low=1.0, high=32.0, original_len=8, base=1.0),
         lib.INVALID_ARGUMENT),
        (dict(rotary_dim=64, magnitude=-1.0), lib.INVALID_ARGUMENT),
    ]
    for kw, status in bad:
        with pytest.raises(lib.LibraError) as e:
            lib.libra_rope_init(**kw)
        assert e.value.status == status, kw
    assert lib.lib.libra_rope_init(None, 64, 0, 10000.0, None) == lib.INVALID_ARGUMENT


def test_refusals_of_apply_and_append_before_a_gpu_is_touched(lib):
    import ctypes as C
    rope = lib.libra_rope_init(64)
    good = dict(device=0, rope=rope, x_ptr=256, out_ptr=4096, dtype=lib.ROPE_BF16, positions_ptr=256, n_tokens=0, n_heads=2,
                head_dim=64, x_stride_token=128, x_stride_head=64, out_stride_token=128, out_stride_head=64,
                direction=lib.ROPE_FORWARD, stream=0)
    lib.libra_rope_apply(**good)          # no tokens: nothing to do
    for kw, status in [
        (dict(device=-1), lib.INVALID_ARGUMENT), (dict(x_ptr=0), lib.INVALID_ARGUMENT), (dict(out_ptr=0), lib.INVALID_ARGUMENT),
        (dict(positions_ptr=0), lib.INVALID_ARGUMENT), (dict(n_tokens=-1), lib.INVALID_ARGUMENT),
        (dict(n_heads=0), lib.INVALID_ARGUMENT), (dict(head_dim=0), lib.INVALID_ARGUMENT), (dict(head_dim=63), lib.UNSUPPORTED_SHAPE),
        (dict(head_dim=1026, n_heads=1), lib.UNSUPPORTED_SHAPE), (dict(head_dim=32), lib.UNSUPPORTED_SHAPE), (dict(dtype=3), lib.INVALID_ARGUMENT),
        (dict(direction=2), lib.INVALID_ARGUMENT), (dict(x_stride_token=-128), lib.INVALID_ARGUMENT),
        (dict(n_tokens=2, out_stride_token=32), lib.INVALID_ARGUMENT), (dict(out_stride_head=32), lib.INVALID_ARGUMENT),
        (dict(n_tokens=2, out_stride_token=64), lib.INVALID_ARGUMENT), (dict(n_tokens=3, out_stride_token=64, out_stride_head=128), lib.INVALID_ARGUMENT),
        (dict(n_heads=16385), lib.UNSUPPORTED_SHAPE),
        (dict(x_ptr=4096, x_stride_token=256), lib.INVALID_ARGUMENT), (dict(x_ptr=257), lib.INVALID_ARGUMENT),
        (dict(x_ptr=258, dtype=lib.ROPE_F32), lib.INVALID_ARGUMENT), (dict(rope=lib.Rope()), lib.INVALID_ARGUMENT),
    ]:
        with pytest.raises(lib.LibraError) as e:
            lib.libra_rope_apply(**{**good, **kw})
        assert e.value.status == status, kw
    assert lib.lib.libra_rope_append(None, C.byref(rope), None, 0, None, 0, None, None, 0, None, None, None, 0, 0,
                                     None, None, None, None) == lib.INVALID_ARGUMENT


# ------------------------------------------------------------------------------------------------ pins of the oracle
def test_oracle_turns_by_a_quarter():
    # theta_0 = 1: position pi/2 is no integer, so pin by composition: turning by a then b = turning by a + b
    t = K.rope_turns(8, 10000.0)
    x = np.random.default_rng(0).standard_normal((1, 3, 10))
    for layout in (K.HALF, K.INTERLEAVED):
        one = K.rotate(K.rotate(x, K.rope_angles([5], t), layout), K.rope_angles([37], t), layout)
        assert np.allclose(one, K.rotate(x, K.rope_angles([42], t), layout), atol=1e-14)
        back = K.rotate(one, K.rope_angles([-42], t), layout)
        assert np.allclose(back, x, atol=1e-14)
        assert np.array_equal(one[:, :, 8:], x[:, :, 8:])
    # position 1 turns pair 0 by one radian: (1, 0) -> (cos 1, sin 1)
    e = np.zeros((1, 1, 8)); e[0, 0, 0] = 1
    y = K.rotate(e, K.rope_angles([1], t), K.HALF)[0, 0]
    assert abs(y[0] - math.cos(1)) < 1e-15 and abs(y[4] - math.sin(1)) < 1e-15
    y = K.rotate(e, K.rope_angles([1], t), K.INTERLEAVED)[0, 0]
    assert abs(y[0] - math.cos(1)) < 1e-15 and abs(y[1] - math.sin(1)) < 1e-15


def test_oracle_scores_depend_on_the_distance_alone():
    t = K.rope_turns(64, 10000.0, "bands", **SCALINGS["bands"])
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 64))
    dots = [float((K.rotate(q, K.rope_angles([p + 11], t), K.HALF) * K.rotate(k, K.rope_angles([p], t), K.HALF)).sum())
            for p in (0, 1, 1000, 2 ** 30)]
    assert np.allclose(dots, dots[0], atol=1e-12)


def test_oracle_e4m3():
    v = K.e4m3_values()
    finite = np.flatnonzero(~np.isnan(v))
    assert len(finite) == 254 and v[0x7E] == 448 and v[1] == 2.0 ** -9 and v[0x38] == 1.0
    assert np.array_equal(K.e4m3_encode(v[finite]), finite)         # -0.0 keeps its sign
    assert K.e4m3_encode(1e9) == 0x7E and K.e4m3_encode(-np.inf) == 0xFE and K.e4m3_encode(np.nan) == 0x7F
    assert v[K.e4m3_encode(1.0625)] == 1.0 and v[K.e4m3_encode(1.1875)] == 1.25   # ties to even
    assert v[K.e4m3_encode(2.0 ** -10)] == 0.0 and v[K.e4m3_encode(1.01 * 2.0 ** -10)] == 2.0 ** -9


def test_oracle_chunk_attention_is_the_multi_token_one():
    from paper_2606_03077_b200 import workloads as W
    lens, bt, q, k, v = W.random_case(5, 3, 4, 2, 64, [40, 3, 17])
    n = 5
    q5 = W.f32_to_bf16_bits(np.random.default_rng(3).standard_normal((3, n, 4, 64), dtype=np.float32))
    want, want_lse = O.paged_multi_token_attention(q5, k, v, bt, lens)
    out, lse, spread = K.packed_chunk_attention(O.bf16_bits_to_f64(q5).reshape(3 * n, 4, 64), K.sequence_tokens(k, bt, lens),
                                                K.sequence_tokens(v, bt, lens), [n] * 3, lens)
    assert np.allclose(out.reshape(want.shape), want, atol=1e-13)
    seen = np.isfinite(lse)
    assert np.allclose(lse[seen], want_lse.reshape(lse.shape)[seen], atol=1e-13) and np.all(spread >= np.abs(out) - 1e-13)
    assert np.array_equal(np.isfinite(want_lse.reshape(lse.shape)), seen) and not seen.all()
