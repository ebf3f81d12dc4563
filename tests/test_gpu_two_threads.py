"""Calls from two host threads at once whose kernels need different amounts of shared memory: neither is refused."""
import threading

import pytest

pytestmark = pytest.mark.gpu


def together(*calls, turns=4000):
    import torch
    torch.cuda.synchronize()
    failed, start = [], threading.Barrier(len(calls))

    def work(call):
        start.wait()
        try:
            for _ in range(turns):
                call()
        except Exception as e:   # handed to the test
            failed.append(e)

    threads = [threading.Thread(target=work, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed


def test_extend_of_two_long_batches(lib):
    import torch
    keep, calls = [], []
    for batch in (4096, 3500):
        h = lib.Handle(8, 2, 64, 100, 4096, 4)
        z = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
        new, lens, table, free, count, off, err, st = z(batch), z(batch), z(batch * 4), z(100), z(1), z(batch + 1), z(1), torch.cuda.Stream()
        args = [batch, free.data_ptr(), count.data_ptr(), off.data_ptr(), 0, 0, 0, err.data_ptr(), st.cuda_stream]
        keep.append((h, new, lens, table, free, count, off, err, st))
        calls.append(lambda h=h, a=[new.data_ptr(), lens.data_ptr(), table.data_ptr()] + args: h.cache_extend(*a))
    together(*calls)
    for k in keep:
        assert int(k[7]) == 0
        k[0].close()
