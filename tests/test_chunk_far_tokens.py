"""Sequences whose last steps would count past 32 bits are refused by the chunk planner: the kernel's token numbers run up to
two steps past a sequence's end."""
import pytest

LIMIT = 2 ** 31 - 512


@pytest.mark.parametrize("seq_len", [LIMIT + 1, 2 ** 31 - 128, 2 ** 31 - 1])
@pytest.mark.parametrize("q_len", [0, 1, 300])
def test_refused(lib, seq_len, q_len):
    with pytest.raises(lib.LibraError) as e:
        lib.libra_chunk_plan_host(148, 8, 2, [q_len, 1], [seq_len, 5])
    assert e.value.status == lib.UNSUPPORTED_SHAPE


def test_the_longest_one_is_planned(lib):
    items = lib.libra_chunk_plan_host(148, 8, 2, [1], [LIMIT])["items"]
    ranges = sorted((int(r[4]), int(r[5])) for r in items)
    assert ranges[0][0] == 0 and ranges[-1][1] == LIMIT and all(a[1] == b[0] for a, b in zip(ranges, ranges[1:]))
    for begin, end in ranges:
        steps = -(-(end - begin) // 128)
        assert begin + (steps + 1) * 128 + 127 < 2 ** 31 and end - begin + 127 < 2 ** 31
