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


def test_gradients_through_shared_memory(lib):
    import torch
    keep, calls = [], []
    for dim in (1022, 702):   # rows that no 16-byte vector divides; q and k
        x, g, o = (torch.ones((3, 1, dim), device="cuda") for _ in range(3))
        k_out, w, gw, gw_k = torch.ones((3, 1, dim), device="cuda"), *(torch.ones(dim, device="cuda") for _ in range(3))
        ws, st = torch.empty(lib.libra_norm_rope_workspace_size(0, dim), dtype=torch.uint8, device="cuda"), torch.cuda.Stream()
        q, k = lib.NormGrads.of(x, g, w, o, gw), lib.NormGrads.of(x, g, w, k_out, gw_k)
        keep.append((x, g, o, k_out, w, gw, gw_k, ws, st))
        calls.append(lambda q=q, k=k, dim=dim, ws=ws, st=st: lib.libra_norm_rope_gradient(
            0, None, q, k, lib.ROPE_F32, 0, 3, dim, 1e-6, ws.data_ptr(), ws.numel(), st.cuda_stream))
    together(*calls)
