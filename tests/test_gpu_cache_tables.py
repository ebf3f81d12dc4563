"""Pages and slots handed out on the GPU against a list of free pages on the host; integers, every one of them compared."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

CANARY = -77


class Tables:
    """A pool's bookkeeping on the device and its model on the host."""

    def __init__(self, lib, lens, ld, page=16, spare=0, seed=0, off=0):
        import torch
        self.torch, self.lib, self.page, self.ld = torch, lib, page, ld
        rng = np.random.default_rng(seed)
        B = len(lens)
        owned = [-(-int(L) // page) for L in lens]
        self.pool = sum(owned) + spare
        ids = rng.permutation(self.pool).astype(np.int32)
        self.table = np.full((B, ld), CANARY, np.int32)
        at = 0
        for b, n in enumerate(owned):
            self.table[b, :n] = ids[at:at + n]
            at += n
        self.stack = np.full(self.pool, CANARY, np.int32)
        self.count = self.pool - at
        self.stack[:self.count] = ids[at:]
        self.lens = np.asarray(lens, np.int32).copy()
        up = lambda a: torch.from_numpy(a.copy()).cuda()
        self.d_table, self.d_stack, self.d_lens = up(self.table), up(self.stack), up(self.lens)
        self.d_count = torch.tensor([self.count], dtype=torch.int32, device="cuda")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.h = lib.Handle(8, 2, 64, max(self.pool, 1), max(B, 1), ld, page_size=page)
        self.off = off   # of positions and slots within their arrays
        self.change = torch.zeros(max(B, 1), dtype=torch.int32, device="cuda")

    def rows_for(self, max_rows):
        full = lambda n: self.torch.full((n + self.off,), CANARY, dtype=self.torch.int32, device="cuda")
        self.pos, self.slots = full(max_rows + 5), full(max_rows + 5)
        self.q_off = full(len(self.lens) + 2)
        self.max_rows = max_rows

    def extend(self, new, positions=True, slots=True):
        if new is not None:
            self.change[:len(new)] = self.torch.tensor(np.asarray(new, np.int32))
        self.h.cache_extend(self.change.data_ptr(), self.d_lens.data_ptr(), self.d_table.data_ptr(), len(self.lens),
                            self.d_stack.data_ptr(), self.d_count.data_ptr(), self.q_off.data_ptr(),
                            self.pos[self.off:].data_ptr() if positions else 0, self.slots[self.off:].data_ptr() if slots else 0,
                            self.max_rows, self.err.data_ptr(), self.torch.cuda.current_stream().cuda_stream)

    def trim(self, keep):
        if keep is not None:
            self.change[:len(keep)] = self.torch.tensor(np.asarray(keep, np.int32))
        self.h.cache_trim(self.change.data_ptr(), self.d_lens.data_ptr(), self.d_table.data_ptr(), len(self.lens),
                          self.d_stack.data_ptr(), self.d_count.data_ptr(), self.err.data_ptr(),
                          self.torch.cuda.current_stream().cuda_stream)

    def model_extend(self, new):
        """Row offsets, positions and slots."""
        off, pos, slots = [0], [], []
        for b, n in enumerate(int(x) for x in new):
            L = int(self.lens[b])
            for i in range(-(-L // self.page), -(-(L + n) // self.page)):
                self.count -= 1
                self.table[b, i] = self.stack[self.count]
            t = np.arange(L, L + n)
            pos.append(t)
            slots.append(self.table[b, t // self.page].astype(np.int64) * self.page + t % self.page)
            off.append(off[-1] + n)
            self.lens[b] += n
        return np.array(off), np.concatenate(pos + [np.zeros(0, int)]), np.concatenate(slots + [np.zeros(0, int)])

    def model_trim(self, keep):
        for b in range(len(self.lens) - 1, -1, -1):
            for i in range(-(-int(self.lens[b]) // self.page) - 1, -(-int(keep[b]) // self.page) - 1, -1):
                self.stack[self.count] = self.table[b, i]
                self.count += 1
            self.lens[b] = keep[b]

    def check_state(self):
        assert np.array_equal(self.d_lens.cpu().numpy(), self.lens) and int(self.d_count) == self.count
        assert np.array_equal(self.d_table.cpu().numpy(), self.table)
        assert np.array_equal(self.d_stack.cpu().numpy()[:self.count], self.stack[:self.count])

    def check_rows(self, off, pos, slots):
        B, n = len(self.lens), len(pos)
        got = self.q_off.cpu().numpy()
        assert np.array_equal(got[:B + 1], off) and np.all(got[B + 1:] == CANARY)
        for have, want in ((self.pos, pos), (self.slots, slots)):
            have = have.cpu().numpy()
            assert np.array_equal(have[self.off:self.off + n], want)
            assert np.all(have[:self.off] == CANARY) and np.all(have[self.off + n:] == CANARY)


SIZES = {"one": (1, 1), "three": (3, 7), "a step": (64, 1), "returns": (40, 300), "many": (1025, 9), "most": (4096, 40), "prompts": (5, 20000)}


@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("size", list(SIZES))
def test_grow_shrink_and_end(lib, size, page):
    """Rounds of extending and trimming: lengths on and off page borders, sequences without new tokens, ones that end."""
    B, most = SIZES[size]
    rng = np.random.default_rng(B + page)
    lens = rng.integers(0, 3 * page, B)
    lens[rng.random(B) < 0.3] = page
    ld = -(-(int(lens.max()) + 3 * most + 1) // page)
    t = Tables(lib, lens, ld, page, spare=int(B * (3 * most / page + 2)) + 1, seed=B, off=page == 32)
    for turn in range(3):
        new = rng.integers(0, most + 1, B)
        new[rng.random(B) < 0.2] = 0
        t.rows_for(int(new.sum()) + (turn if turn < 2 else 0))
        t.extend(new)
        want = t.model_extend(new)
        t.check_rows(*want)
        t.check_state()
        keep = np.where(rng.random(B) < 0.4, t.lens, rng.integers(0, t.lens + 1))
        keep[rng.random(B) < 0.2] = 0
        t.trim(keep)
        t.model_trim(keep)
        t.check_state()
    assert int(t.err) == 0
    t.h.close()


def test_trim_undoes_extend(lib):
    t = Tables(lib, [5, 16, 0, 31], 12, spare=30)
    before, count = t.stack.copy(), t.count
    t.rows_for(200)
    for new in ([1, 1, 1, 1], [0, 0, 0, 0], [100, 0, 33, 2]):
        lens = t.lens.copy()
        t.extend(new)
        t.model_extend(new)
        t.check_state()
        t.trim(lens)
        t.model_trim(lens)
        t.check_state()
        assert t.count == count and np.array_equal(t.d_stack.cpu().numpy()[:count], before[:count])
    t.h.close()


def test_every_page_of_the_pool(lib):
    """The last page is handed out, and taken back into a full stack."""
    t = Tables(lib, [0, 0], 4, spare=7)
    t.rows_for(112)
    t.extend([64, 48])
    t.check_rows(*t.model_extend([64, 48]))
    t.check_state()
    assert t.count == 0
    t.trim([0, 0])
    t.model_trim([0, 0])
    t.check_state()
    assert int(t.err) == 0 and t.count == t.pool
    t.h.close()


def test_outputs_that_are_not_wanted(lib):
    t = Tables(lib, [5, 16], 4, spare=6)
    t.rows_for(40)
    t.extend([20, 3], positions=False)
    off, pos, slots = t.model_extend([20, 3])
    t.check_state()
    assert np.all(t.pos.cpu().numpy() == CANARY) and np.array_equal(t.slots.cpu().numpy()[:23], slots)
    t.slots.fill_(CANARY)
    t.extend([0, 4], slots=False)
    off, pos, slots = t.model_extend([0, 4])
    t.check_state()
    assert np.all(t.slots.cpu().numpy() == CANARY) and np.array_equal(t.pos.cpu().numpy()[:4], pos)
    t.extend([1, 1], positions=False, slots=False)   # the block table and the lengths are written all the same
    t.model_extend([1, 1])
    t.check_state()
    t.h.close()


def test_no_sequences(lib):
    t = Tables(lib, [7], 4, spare=3)
    t.rows_for(4)
    t.h.cache_extend(t.change.data_ptr(), t.d_lens.data_ptr(), t.d_table.data_ptr(), 0, t.d_stack.data_ptr(), t.d_count.data_ptr(),
                     t.q_off.data_ptr(), 0, 0, 4, t.err.data_ptr(), t.torch.cuda.current_stream().cuda_stream)
    assert int(t.err) == 0 and t.q_off.cpu().tolist() == [0, CANARY, CANARY]
    t.check_state()
    t.h.close()


def test_no_sequences_and_no_rows(lib):
    t = Tables(lib, [7], 4, spare=3)
    t.rows_for(0)
    for batch, offsets in ((0, [0, CANARY, CANARY]), (1, [0, 0, CANARY])):
        t.h.cache_extend(t.change.data_ptr(), t.d_lens.data_ptr(), t.d_table.data_ptr(), batch, t.d_stack.data_ptr(), t.d_count.data_ptr(),
                         t.q_off.data_ptr(), 0, 0, 0, t.err.data_ptr(), t.torch.cuda.current_stream().cuda_stream)
        assert int(t.err) == 0 and t.q_off.cpu().tolist() == offsets
        t.h.cache_trim(t.d_lens.clone().data_ptr(), t.d_lens.data_ptr(), t.d_table.data_ptr(), batch, t.d_stack.data_ptr(), t.d_count.data_ptr(),
                       t.err.data_ptr(), t.torch.cuda.current_stream().cuda_stream)
        t.check_state()
    assert int(t.err) == 0
    t.h.close()


@pytest.mark.parametrize("what", ["pages", "row of the table", "rows", "negative", "negative length", "count", "huge"])
def test_extend_refused_on_the_device(lib, what):
    """Nothing changes but the error word, and the batch has no new rows."""
    t = Tables(lib, [5, 16, 40], 6, spare=3)
    t.rows_for(60)
    new, bit = {"pages": ([12, 33, 1], lib.ERR_NO_PAGES), "row of the table": ([0, 0, 57], lib.ERR_PLAN_OVERFLOW),
                "rows": ([11, 20, 30], lib.ERR_PLAN_OVERFLOW), "negative": ([1, -1, 1], lib.ERR_BAD_LENGTH),
                "negative length": ([1, 1, 1], lib.ERR_BAD_LENGTH), "count": ([1, 1, 1], lib.ERR_BAD_LENGTH),
                "huge": ([2 ** 31 - 1] * 3, lib.ERR_PLAN_OVERFLOW)}[what]
    if what == "negative length":
        t.d_lens[1] = t.lens[1] = -3
    if what == "count":
        t.d_count[0] = t.count = t.pool + 1
    t.extend(new)
    assert int(t.err) & bit
    assert np.array_equal(t.d_lens.cpu().numpy(), t.lens) and int(t.d_count) == t.count
    assert np.array_equal(t.d_table.cpu().numpy(), t.table) and np.array_equal(t.d_stack.cpu().numpy(), t.stack)
    assert t.q_off.cpu().tolist() == [0, 0, 0, 0, CANARY]
    assert np.all(t.pos.cpu().numpy() == CANARY) and np.all(t.slots.cpu().numpy() == CANARY)
    t.h.close()


@pytest.mark.parametrize("what", ["more than there is", "negative", "stack"])
def test_trim_refused_on_the_device(lib, what):
    t = Tables(lib, [5, 16, 40], 6, spare=3)
    keep = {"more than there is": [6, 0, 0], "negative": [0, -1, 0], "stack": [0, 0, 0]}[what]
    if what == "stack":
        t.d_count[0] = t.count = t.pool - 4   # 1 + 1 + 3 pages would go back, one more than there is room for
    t.trim(keep)
    assert int(t.err) == lib.ERR_BAD_LENGTH
    assert np.array_equal(t.d_lens.cpu().numpy(), t.lens) and int(t.d_count) == t.count
    assert np.array_equal(t.d_table.cpu().numpy(), t.table) and np.array_equal(t.d_stack.cpu().numpy(), t.stack)
    t.h.close()


def test_recorded_and_replayed(lib):
    """One recording of both calls, replayed while the numbers of tokens change in their buffer; on a side stream."""
    import torch
    t = Tables(lib, [3, 20, 0, 15], 40, spare=60)
    t.rows_for(300)
    keep = torch.zeros(4, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        t.extend(None)
        t.h.cache_trim(keep.data_ptr(), t.d_lens.data_ptr(), t.d_table.data_ptr(), 4, t.d_stack.data_ptr(), t.d_count.data_ptr(),
                       t.err.data_ptr(), torch.cuda.current_stream().cuda_stream)
    rng = np.random.default_rng(1)
    for _ in range(5):
        new = rng.integers(0, 75, 4)
        left = np.minimum(t.lens + new, rng.integers(0, 120, 4))
        t.change.copy_(torch.tensor(new.astype(np.int32)))
        keep.copy_(torch.tensor(left.astype(np.int32)))
        t.pos.fill_(CANARY); t.slots.fill_(CANARY)
        g.replay()
        torch.cuda.synchronize()
        t.check_rows(*t.model_extend(new))
        t.model_trim(left)
        t.check_state()
    assert int(t.err) == 0
    del g
    t.h.close()


def test_recorded_with_as_many_sequences_as_there_can_be(lib):
    """The prefix sums of 4096 sequences need more shared memory than the default; the first call is within the recording."""
    import torch
    rng = np.random.default_rng(4)
    lens = rng.integers(0, 40, 4096)
    t = Tables(lib, lens, 6, spare=4096 * 2)
    new = rng.integers(0, 30, 4096)
    t.change.copy_(torch.tensor(new.astype(np.int32)))
    t.rows_for(int(new.sum()))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        t.extend(None)
    g.replay()
    torch.cuda.synchronize()
    assert int(t.err) == 0
    t.check_rows(*t.model_extend(new))
    t.check_state()
    del g
    t.h.close()


def test_a_table_row_of_2_to_the_31_tokens(lib):
    """Lengths next to the largest one; a sequence of 2^31 - 1 tokens cannot grow."""
    import torch
    h = lib.Handle(8, 2, 64, 2 ** 25 - 1, 2, 2 ** 25, page_size=64)   # one page more would be refused
    table = torch.zeros((2, 2 ** 25), dtype=torch.int32, device="cuda")
    last = 2 ** 31 - 1
    lens = torch.tensor([last - 65, last], dtype=torch.int32, device="cuda")
    free, count = torch.arange(100, 110, dtype=torch.int32, device="cuda").repeat(2 ** 22)[:2 ** 25].contiguous(), torch.tensor([10], dtype=torch.int32, device="cuda")
    off, pos, slots, err = (torch.full((n,), CANARY, dtype=torch.int32, device="cuda") for n in (3, 70, 70, 1))
    err.zero_()

    def extend(new):
        change = torch.tensor(new, dtype=torch.int32, device="cuda")
        h.cache_extend(change.data_ptr(), lens.data_ptr(), table.data_ptr(), 2, free.data_ptr(), count.data_ptr(), off.data_ptr(), pos.data_ptr(),
                       slots.data_ptr(), 70, err.data_ptr(), torch.cuda.current_stream().cuda_stream)
        return int(err)

    assert extend([65, 1]) == lib.ERR_PLAN_OVERFLOW and off.tolist() == [0, 0, 0] and lens.tolist() == [last - 65, last]
    err.zero_()
    assert extend([65, 0]) == 0 and lens.tolist() == [last, last] and int(count) == 9
    assert pos[:65].tolist() == list(range(last - 65, last)) and int(table[0, 2 ** 25 - 1]) == 109
    old, new = [0 * 64 + i for i in range(62, 64)], [109 * 64 + i for i in range(63)]
    assert slots[:65].tolist() == old + new
    h.close()


def test_refused_by_the_host(lib):
    import torch
    t = Tables(lib, [5, 16], 6, spare=3)
    t.rows_for(10)
    a = lambda x: x.data_ptr()
    good = [a(t.change), a(t.d_lens), a(t.d_table), 2, a(t.d_stack), a(t.d_count), a(t.q_off), a(t.pos), a(t.slots), 10, a(t.err), 0]
    for i, bad in [(0, 0), (1, 0), (2, 0), (4, 0), (5, 0), (6, 0), (10, 0), (3, -1), (3, 3), (9, -1), (0, a(t.change) + 2), (7, a(t.pos) + 1),
                   (0, a(t.d_lens)), (6, a(t.d_lens)), (6, a(t.change))]:
        args = list(good)
        args[i] = bad or None
        assert lib.lib.libra_cache_extend(t.h._h, *args) == lib.INVALID_ARGUMENT, i
    good = [a(t.change), a(t.d_lens), a(t.d_table), 2, a(t.d_stack), a(t.d_count), a(t.err), 0]
    for i, bad in [(0, 0), (1, 0), (2, 0), (4, 0), (5, 0), (6, 0), (3, -1), (3, 3), (0, a(t.d_lens))]:
        args = list(good)
        args[i] = bad or None
        assert lib.lib.libra_cache_trim(t.h._h, *args) == lib.INVALID_ARGUMENT, i
    h = lib.Handle(8, 2, 64, 100, 5000, 6)
    with pytest.raises(lib.LibraError) as e:
        h.cache_extend(a(t.change), a(t.d_lens), a(t.d_table), 4097, a(t.d_stack), a(t.d_count), a(t.q_off), 0, 0, 10, a(t.err), 0)
    assert e.value.status == lib.UNSUPPORTED_SHAPE
    h.close()
    h = lib.Handle(8, 2, 64, 2 ** 27, 2, 6)   # more slots than 31 bits count
    with pytest.raises(lib.LibraError) as e:
        h.cache_trim(a(t.change), a(t.d_lens), a(t.d_table), 2, a(t.d_stack), a(t.d_count), a(t.err), 0)
    assert e.value.status == lib.UNSUPPORTED_SHAPE
    torch.cuda.synchronize()
    assert np.array_equal(t.d_lens.cpu().numpy(), t.lens)
    h.close(); t.h.close()
