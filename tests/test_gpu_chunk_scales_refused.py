"""Chunk attention with scales that are no normal float32 once they are combined: refused, not computed with."""
import numpy as np
import pytest

from test_gpu_chunk import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sm_scale", [1e-39, 2.0 ** -127, 3.3e38])
def test_chunk_attention_score_scale(lib, sm_scale):
    """sm_scale * log2(e) below the smallest normal float32, or beyond the largest."""
    c = Case(lib, [4, 2], [30, 9], 4, 2, 64, seed=41, sm_scale=sm_scale)
    c.plan()
    with pytest.raises(lib.LibraError) as e:
        c.attn()
    assert e.value.status == lib.INVALID_ARGUMENT
    assert bool((c.out == 0x7FC0).all())
    c.h.close()


@pytest.mark.parametrize("scales,ok", [((1e-37, 1.0), True), ((5e-38, 1.0), False), ((1e-39, 1.0), False), ((1.0, 1e-39), False), ((2.0 ** -122, 2.0 ** -126), True)])
def test_chunk_attention_pool_scales(lib, scales, ok):
    """k_scale * sm_scale * log2(e) and v_scale.  2^-122 * 0.1803 = 2^-124.5 and 1e-37 * 0.1803 = 1.8e-38 are still
    normal numbers (the smallest is 1.18e-38), whose scores weigh all tokens alike; 5e-38 * 0.1803 = 9e-39 is not."""
    c = Case(lib, [4, 2], [30, 9], 4, 2, 64, seed=42, kv="e4m3")
    c.scales = scales
    c.h.set_kv_dtype(lib.KV_E4M3, *scales)
    c.plan()
    if ok:
        c.attn()
        assert int(c.err) == 0
        lse = c.lse.double().cpu().numpy()
        want = np.log([27, 28, 29, 30, 8, 9])[:, None]
        assert np.all(np.abs(lse - want) <= 2.0 ** -20 * (1 + want))
    else:
        with pytest.raises(lib.LibraError) as e:
            c.attn()
        assert e.value.status == lib.INVALID_ARGUMENT
        assert bool((c.out == 0x7FC0).all())
    c.h.close()
