"""Page ids outside the pool, in the stack of free pages or in a block table: the slots of such a page are below -1, whatever the
id, so that the append by slots reports every row and stores none."""
import numpy as np
import pytest

from test_gpu_cache_tables import CANARY, Tables

pytestmark = pytest.mark.gpu


def ids_outside(pool, page):
    """The first id past the pool, -1, and ids whose first slot, counted in 32 bits, is 0, page or the sign bit alone."""
    return [pool, -1, -2, 2 ** 32 // page, 2 ** 32 // page + 1, 2 ** 31 // page, 2 ** 31 - 1, -2 ** 31, -2 ** 31 + 1]


def wrapped(x):
    return int(np.array(x, np.int64).astype(np.int32))


@pytest.mark.parametrize("many", [False, True], ids=["a row a thread", "eight rows a thread"])
@pytest.mark.parametrize("page", [16, 32, 64])
def test_slots_of_pages_outside_the_pool(lib, page, many):
    new = [3 * page, 2 * page + 5, 7] + ([200 * page + 3] * 2 if many else [0, 1])
    lens = [page - 1, 0, page + page // 2, 0, 0]
    ld = 210
    t0 = Tables(lib, lens, ld, page, spare=450)
    t0.h.close()
    for k, bad in enumerate(ids_outside(t0.pool, page)):
        bad = wrapped(bad)
        t = Tables(lib, lens, ld, page, spare=450)
        t.table[0, 0] = bad                       # a page that the sequence has: one token of it is new
        t.table[2, 1] = bad
        t.stack[t.count - 2] = bad                # the second page that is handed out: sequence 0's
        t.stack[t.count - 5 - k % 2] = bad        # sequence 1's
        for dev, host in ((t.d_table, t.table), (t.d_stack, t.stack)):
            dev.copy_(t.torch.from_numpy(host))
        t.rows_for(sum(new))
        t.extend(new)
        off, pos, _ = t.model_extend(new)
        owner = np.repeat(np.arange(len(new)), new)
        ids = t.table[owner, pos // page].astype(np.int64)
        outside = (ids < 0) | (ids >= t.pool)
        assert outside.sum() >= 13 + page
        got = t.slots.cpu().numpy()[t.off:t.off + len(pos)]
        assert np.all(got[outside] < -1)
        t.check_rows(off, pos, np.where(outside, got, ids * page + pos % page))
        t.check_state()                           # the ids themselves are handed on as they are
        assert int(t.err) == 0
        t.h.close()


@pytest.mark.parametrize("bad", [-1, 2 ** 32 // 16])
def test_their_rows_are_reported_and_not_stored(lib, bad):
    import torch
    t = Tables(lib, [10], 4, spare=4)
    t.table[0, 0] = wrapped(bad)
    t.stack[t.count - 2] = wrapped(bad)
    t.d_table.copy_(torch.from_numpy(t.table)); t.d_stack.copy_(torch.from_numpy(t.stack))
    new = 6 + 16 + 16 + 3                         # the rest of a bad page, a good one, a bad one, 3 tokens of a good one
    t.rows_for(new)
    t.extend([new])
    t.model_extend([new])
    k, v = (torch.zeros((t.pool, 2, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x = torch.ones((new, 4, 64), dtype=torch.bfloat16, device="cuda")

    def append(slots, rows):
        t.err.zero_()
        t.h.norm_rope_append(None, 0, 0, 1e-6, 0, 0, 0, 0, x.data_ptr(), x[:, 2:].data_ptr(), x.stride(0), 0, slots.data_ptr(), 0, rows, k.data_ptr(),
                             v.data_ptr(), t.err.data_ptr(), torch.cuda.current_stream().cuda_stream)
        return int(t.err)

    assert append(t.slots, new) == lib.ERR_BAD_PAGE_ID
    for pool in (k, v):
        rows = pool[:, 0, :, 0].float().cpu().numpy()
        want = np.zeros((t.pool, 16))
        want[t.table[0, 1]] = 1.0
        want[t.table[0, 3], :3] = 1.0
        assert np.array_equal(rows, want)
    for row in [*range(6), *range(22, 38)]:       # each of them by itself
        assert append(t.slots[row:], 1) == lib.ERR_BAD_PAGE_ID, row
    t.h.close()
