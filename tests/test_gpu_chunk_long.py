"""Chunk attention against the float64 oracle on caches longer than those of test_gpu_chunk, with 16 query heads per KV head
over cut ranges, and the same bits from call to call, plan to plan and handle to handle."""
import numpy as np
import pytest

from test_gpu_chunk import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("hq,hkv,dim,page,order", [(16, 1, 128, 16, "HND"), (16, 1, 64, 32, "NHD"), (5, 1, 128, 64, "NHD"), (8, 2, 64, 64, "HND")])
def test_long_caches(lib, hq, hkv, dim, page, order, kv):
    q, L = [3, 1, 17], [40000, 12345, 20001]
    assert len(lib.libra_chunk_plan_host(148, hq, hkv, q, L)["merges"]) > 0
    Case(lib, q, L, hq, hkv, dim, page, order, kv, seed=61 + hq).run()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q,L", [([40, 200, 3], [3000, 200, 2500]), ([1] * 6, [700, 1, 128, 129, 1500, 64]), ([300] * 8, [300, 400, 500, 600, 700, 800, 900, 1000])])
def test_the_same_bits_from_every_call(lib, q, L, dim, kv):
    import torch
    want = None
    for k in range(3):
        c = Case(lib, q, L, 8, 2, dim, kv=kv, seed=62)
        for _ in range(2):
            c.plan()
            for _ in range(10):
                c.out.fill_(0x7FC0); c.lse.fill_(float("nan"))
                c.attn()
                got = c.out.clone(), c.lse.clone()
                want = want or got
                assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert int(c.err) == 0
        c.h.close()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("order", ["heads, pages, tokens", "tokens, pages, heads", "pages, tokens, heads, with gaps"])
def test_other_orders_of_the_pools(lib, order, kv):
    """Pools whose pages are not one piece, or have gaps: append and attention write and read the same bits as in the usual order."""
    import torch
    hq, hkv, dim, page = 8, 2, 64, 16
    q_lens, seq_lens = np.array([20, 3, 1], np.int32), np.array([300, 40, 1], np.int32)
    a = Case(lib, q_lens, seq_lens, hq, hkv, dim, page, kv=kv, seed=63)
    a.plan(); a.attn()
    a.check()
    pages = a.kh.shape[0]
    permute = {"heads, pages, tokens": (1, 0, 2, 3), "tokens, pages, heads": (2, 0, 1, 3), "pages, tokens, heads, with gaps": (0, 2, 1, 3)}[order]
    gap = 16 if "gaps" in order else 0

    def other(x):   # the same pool in the other order, as a view in the usual one
        y = x.permute(permute)
        wide = torch.full(y.shape[:3] + (dim + gap,), 0x7F, dtype=x.dtype, device="cuda")
        wide[..., :dim] = y
        back = [permute.index(i) for i in range(4)]
        return wide[..., :dim].permute(back)

    k, v = other(a.k), other(a.v)
    assert k.stride(3) == 1 and not k.is_contiguous() and torch.equal(k, a.k)
    h = lib.Handle(hq, hkv, dim, pages, 3, a.bt.shape[1], page_size=page, kv_strides=(k.stride(0), k.stride(1), k.stride(2)))
    if kv == "e4m3":
        h.set_kv_dtype(lib.KV_E4M3, *a.scales)
    st = torch.cuda.current_stream().cuda_stream
    out, lse, err = torch.zeros_like(a.out), torch.zeros_like(a.lse), torch.zeros(1, dtype=torch.int32, device="cuda")
    h.chunk_plan(q_lens, seq_lens, a.ws.data_ptr(), a.ws.numel(), st)
    h.chunk_attn(a.q.data_ptr(), a.q.stride(0), k.data_ptr(), v.data_ptr(), a.dbt.data_ptr(), out.data_ptr(), lse.data_ptr(), err.data_ptr(), st)
    assert int(err) == 0 and torch.equal(out, a.out) and torch.equal(lse, a.lse)
    # append through both handles
    rope = lib.libra_rope_init(dim)
    new = torch.randn((24, hkv, dim), device="cuda").to(torch.bfloat16)
    off, lens = torch.tensor([0, 20, 23, 24], dtype=torch.int32, device="cuda"), torch.from_numpy(seq_lens).cuda()
    for handle, kk, vv in ((a.h, a.k, a.v), (h, k, v)):
        handle.rope_append(rope, 0, 0, 0, 0, new.data_ptr(), new.data_ptr(), hkv * dim, off.data_ptr(), lens.data_ptr(), a.dbt.data_ptr(), 3, 24,
                           kk.data_ptr(), vv.data_ptr(), err.data_ptr(), st)
    assert int(err) == 0 and torch.equal(k, a.k) and torch.equal(v, a.v)
    if gap:
        rest = torch.as_strided(k, k.shape[:3] + (gap,), k.stride(), k.storage_offset() + dim)
        assert bool((rest == 0x7F).all())
    a.h.close(); h.close()
