"""Results of q and of k in the same place are refused, before a GPU is touched."""
from test_norm_refused import Fake, W, apply, status, x


def test_apply(lib):
    a, b = (lib.NormRows.of(x(), W, Fake(at)) for at in (1 << 24, 1 << 25))
    assert apply(lib, a, a) == lib.INVALID_ARGUMENT
    assert apply(lib, a, b, tokens=0) == lib.OK


def test_gradient(lib):
    g, o, ok, gw, gwk = Fake(1 << 22), Fake(1 << 24), Fake(1 << 25), Fake(1 << 14), Fake(1 << 15)
    call = lambda *a: status(lib, lambda: lib.libra_norm_rope_gradient(0, None, *(lib.NormGrads.of(x(), g, W, *t) for t in a), 0, 0, 4, 64, 1e-6, 1 << 26,
                                                                       1 << 30, 0))
    assert call((o, gw), (ok, gw)) == lib.INVALID_ARGUMENT    # the sums of both in one array
    assert call((o, gw), (o, gwk)) == lib.INVALID_ARGUMENT
