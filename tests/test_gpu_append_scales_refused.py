"""Append into E4M3 pools multiplies by the scales' reciprocals: scales whose reciprocal is no normal float32 are refused."""
import pytest

from test_gpu_rope import Batch
from test_rope import rope_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scales", [(1e-39, 1.0), (1.0, 1e-39), (3e38, 1.0), (1.0, 2.0 ** 127)])
def test_refused_and_nothing_stored(lib, scales):
    import torch
    b = Batch(lib, [3, 18], [19, 18], kv="e4m3", seed=43)
    b.h.set_kv_dtype(lib.KV_E4M3, *scales)
    with pytest.raises(lib.LibraError) as e:
        b.append(rope_of(lib, 64))
    assert e.value.status == lib.INVALID_ARGUMENT
    assert torch.equal(b.k, b.k0) and torch.equal(b.v, b.v0) and bool(torch.isnan(b.q_out).all())
    b.h.close()


@pytest.mark.parametrize("scale", [2.0 ** -126, 2.0 ** 126])
def test_the_ends_of_the_range_are_taken(lib, scale):
    """Zeros stay zeros, everything else goes to the end of the codes that it belongs to."""
    import torch
    b = Batch(lib, [3, 18], [19, 18], kv="e4m3", seed=44)
    b.h.set_kv_dtype(lib.KV_E4M3, scale, scale)
    b.vn[:, :, :8] = 0.0
    b.append(None)
    assert int(b.err) == 0
    page, at = int(b.bt[1, 0]), 5
    got = b.v[page, :, at].cpu()
    x = b.vn[3 + at].float().cpu()
    want = torch.where(x < 0, 0x80, 0).to(torch.uint8) + (0x7E if scale < 1 else 0)
    want[x == 0] = 0
    assert torch.equal(got, want.to(torch.uint8))
    b.h.close()
