"""The factor on the rotated channels is kept as a float32: one that no normal float32 holds is refused."""
import pytest


@pytest.mark.parametrize("magnitude", [1e39, 3.5e38, 1e-39, 1e-300, 1e300])
def test_refused(lib, magnitude):
    with pytest.raises(lib.LibraError) as e:
        lib.libra_rope_init(64, magnitude=magnitude)
    assert e.value.status == lib.INVALID_ARGUMENT


def test_the_ends_of_the_range_are_taken(lib):
    for magnitude in (2.0 ** -126, 3.0e38):
        assert lib.libra_rope_init(64, magnitude=magnitude).magnitude > 0
    assert lib.libra_rope_init(64, scaling=lib.ROPE_SCALE_RAMP, factor=1e300, low=1.0, high=32.0, original_len=4096).magnitude < 1e3
