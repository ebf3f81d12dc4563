"""What the norms of q and k refuse before they touch a GPU."""
import ctypes as C

import numpy as np
import pytest

from test_rope import rope_of


class Fake:
    """An address and strides."""

    def __init__(self, address, tokens=4, heads=2, dim=64, strides=None):
        self.address, self.shape, self.strides = address, (tokens, heads, dim), strides or (heads * dim, dim)

    def data_ptr(self):
        return self.address

    def stride(self):
        return self.strides


def x(**kw):
    return Fake(1 << 20, **kw)


W = Fake(1 << 12)


def status(lib, call):
    try:
        call()
    except lib.LibraError as e:
        return e.status
    return lib.OK


def apply(lib, q, k=None, rope=None, dtype=0, positions=1 << 10, tokens=4, dim=64, eps=1e-6, device=0):
    return status(lib, lambda: lib.libra_norm_rope_apply(device, rope, q, k, dtype, positions, tokens, dim, eps, 0))


def test_apply(lib):
    of, bad, shape = lib.NormRows.of, lib.INVALID_ARGUMENT, lib.UNSUPPORTED_SHAPE
    good, out = of(x(), W, Fake(1 << 24)), Fake(1 << 24)
    assert apply(lib, None) == bad
    for q in (of(Fake(0), W, out), of(x(), Fake(0), out), of(x(), W, Fake(0)), of(x(heads=0), W, out), of(Fake((1 << 20) + 1), W, out),
              of(x(), Fake(4097), out), of(x(strides=(-128, 64)), W, out), of(x(), W, Fake(1 << 24, strides=(64, 64))),
              of(x(), W, Fake(1 << 24, strides=(128, 32))), of(x(), W, Fake(1 << 20, strides=(256, 64)))):
        assert apply(lib, q) == bad
        assert apply(lib, good, q) == bad
    assert apply(lib, of(x(heads=16385), W, Fake(1 << 24, heads=16385))) == shape
    rope = rope_of(lib, 128)
    assert apply(lib, good, rope=rope) == shape                  # rotary_dim past the head
    assert apply(lib, good, rope=rope_of(lib, 64), positions=0) == bad
    assert apply(lib, good, positions=1025) == bad
    for kw in (dict(dtype=3), dict(dtype=-1), dict(tokens=-1), dict(dim=0), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("inf")),
               dict(eps=float("nan")), dict(eps=1e-40), dict(device=-1)):
        assert apply(lib, good, **kw) == bad, kw
    far = of(x(dim=2048, strides=(4096, 2048)), W, Fake(1 << 24, dim=2048, strides=(4096, 2048)))
    for kw in (dict(dim=63), dict(tokens=1 << 31), dict(q=far, dim=1026)):
        assert apply(lib, **{"q": good, **kw}) == shape, kw
    r = rope_of(lib, 64)
    r.rotary_dim = 63
    assert apply(lib, good, rope=r) == bad
    assert apply(lib, good, tokens=0) == lib.OK                  # nothing to do, no device needed


def test_gradient(lib):
    of, bad = lib.NormGrads.of, lib.INVALID_ARGUMENT
    g, o, gw = Fake(1 << 22), Fake(1 << 24), Fake(1 << 14)
    call = lambda q, k=None, ws=1 << 26, n=1 << 30, **kw: status(lib, lambda: lib.libra_norm_rope_gradient(
        kw.get("device", 0), kw.get("rope"), q, k, kw.get("dtype", 0), kw.get("positions", 1 << 10), 4, 64, kw.get("eps", 1e-6), ws, n, 0))
    good = of(x(), g, W, o, gw)
    assert call(None) == bad and call(good, ws=0) == bad and call(good, ws=(1 << 26) + 8) == bad and call(good, eps=0.0) == bad
    for q in (of(Fake(0), g, W, o, gw), of(x(), Fake(0), W, o, gw), of(x(), g, Fake(0), o, gw), of(x(), g, W, Fake(0), gw), of(x(), g, W, o, Fake(0)),
              of(x(), g, W, o, Fake(4098)), of(x(), Fake(1 << 22, strides=(-1, 64)), W, o, gw), of(x(), g, W, Fake(1 << 24, strides=(64, 64)), gw),
              of(x(), g, W, Fake(1 << 20, strides=(256, 64)), gw), of(x(), g, W, Fake(1 << 22, strides=(256, 64)), gw), of(x(heads=0), g, W, o, gw)):
        assert call(q) == bad
        assert call(good, q) == bad
    n = C.c_size_t(0)
    f = lib.lib.libra_norm_rope_workspace_size
    assert f(0, 0, C.byref(n)) == bad and f(-1, 64, C.byref(n)) == bad and f(0, 64, None) == bad and f(0, 1026, C.byref(n)) == lib.UNSUPPORTED_SHAPE


def test_null_handles(lib):
    f = lib.lib
    one = np.zeros(4, np.int32).ctypes.data
    assert f.libra_cache_extend(None, one, one, one, 1, one, one, one, None, None, 1, one, None) == lib.INVALID_ARGUMENT
    assert f.libra_cache_trim(None, one, one, one, 1, one, one, one, None) == lib.INVALID_ARGUMENT
    assert f.libra_tree_mask(None, one, one, one, 1, 1, one, 1, None, one, None) == lib.INVALID_ARGUMENT
    assert f.libra_tree_keep(None, one, 1, one, one, one, one, 1, one, one, None, one, None) == lib.INVALID_ARGUMENT
    assert f.libra_tree_attn(None, one, 128, one, one, one, one, 1, one, None, one, None) == lib.INVALID_ARGUMENT
    assert f.libra_norm_rope_append(None, None, None, None, 1e-6, None, 0, None, 0, one, one, 64, None, one, None, 1, one, one, one,
                                    None) == lib.INVALID_ARGUMENT
