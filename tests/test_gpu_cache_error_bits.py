"""The error word of refused calls that hand pages out or take them back, bit for bit as the header lists them."""
import numpy as np
import pytest

from test_gpu_cache_tables import Tables

pytestmark = pytest.mark.gpu


def unchanged(t):
    assert np.array_equal(t.d_lens.cpu().numpy(), t.lens) and int(t.d_count) == t.count
    assert np.array_equal(t.d_table.cpu().numpy(), t.table) and np.array_equal(t.d_stack.cpu().numpy(), t.stack)


@pytest.mark.parametrize("length,keep,bits", [(97, 1, "PLAN_OVERFLOW"), (2 ** 31 - 1, 0, "PLAN_OVERFLOW"), (97, 97, "PLAN_OVERFLOW"),
                                              (97, 98, "BAD_LENGTH PLAN_OVERFLOW"), (97, -1, "BAD_LENGTH PLAN_OVERFLOW"), (-1, 0, "BAD_LENGTH"),
                                              (96, 97, "BAD_LENGTH"), (96, 96, "")])
def test_trim_past_the_end_of_a_row(lib, length, keep, bits):
    """A row of the table describes 6 x 16 = 96 tokens."""
    t = Tables(lib, [5, 96, 40], 6, spare=3)
    t.d_lens[1] = length
    t.lens[1] = length
    t.trim([5, keep, 40])
    assert int(t.err) == sum(getattr(lib, "ERR_" + b) for b in bits.split())
    unchanged(t)
    t.h.close()


@pytest.mark.parametrize("new,count,bits", [([0, 0, 0], -1, "BAD_LENGTH"), ([1, 1, 1], -1, "BAD_LENGTH"), ([30, 30, 0], -2 ** 31, "BAD_LENGTH"),
                                            ([12, 33, 0], 1000, "BAD_LENGTH"), ([12, 33, 1], None, "NO_PAGES"), ([0, 0, 57], None, "PLAN_OVERFLOW"),
                                            ([11, 20, 30], None, "PLAN_OVERFLOW"), ([1, -1, 1], None, "BAD_LENGTH"),
                                            ([2 ** 31 - 1] * 3, None, "PLAN_OVERFLOW"), ([-1, 0, 57], None, "BAD_LENGTH PLAN_OVERFLOW")])
def test_extend(lib, new, count, bits):
    t = Tables(lib, [5, 16, 40], 6, spare=3)
    t.rows_for(60)
    if count is not None:
        t.d_count[0] = t.count = count
    t.extend(new)
    assert int(t.err) == sum(getattr(lib, "ERR_" + b) for b in bits.split())
    unchanged(t)
    assert t.q_off[:4].tolist() == [0, 0, 0, 0]
    t.h.close()
