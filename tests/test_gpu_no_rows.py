"""Calls without tokens, rows or sequences take the empty arrays that a program has then: those know no address."""
import pytest

from test_rope import rope_of

pytestmark = pytest.mark.gpu

EPS = 1e-6


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("dim", [64, 30])
@pytest.mark.parametrize("rotary", [0, 10])
def test_norms(lib, dim, rotary):
    import torch
    empty = lambda h: torch.empty((0, h, dim), device="cuda")
    assert empty(2).data_ptr() == 0
    rope, pos, w = rope_of(lib, rotary) if rotary else None, torch.empty(0, dtype=torch.int32, device="cuda"), torch.ones(dim, device="cuda")
    fused = empty(6)
    q, k = lib.NormRows.of(fused[:, :4], w, empty(4)), lib.NormRows.of(fused[:, 4:5], w, empty(1))
    lib.libra_norm_rope_apply(0, rope, q, k, lib.ROPE_F32, pos.data_ptr(), 0, dim, EPS, stream())
    gw = [torch.full((dim,), float("nan"), device="cuda") for _ in range(2)]
    q, k = (lib.NormGrads.of(fused[:, :h], empty(h), w, empty(h + 1)[:, :h], g) for h, g in zip((4, 1), gw))
    ws = torch.empty(lib.libra_norm_rope_workspace_size(0, dim), dtype=torch.uint8, device="cuda")
    lib.libra_norm_rope_gradient(0, rope, q, k, lib.ROPE_F32, pos.data_ptr(), 0, dim, EPS, ws.data_ptr(), ws.numel(), stream())
    assert all(bool((g == 0).all()) for g in gw)


def test_append(lib):
    import torch
    h = lib.Handle(4, 2, 64, 3, 1, 4)
    kv = torch.full((3, 2, 16, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    x, i, err = torch.empty((0, 8, 64), dtype=torch.bfloat16, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    w, out = torch.ones(64, dtype=torch.bfloat16, device="cuda"), torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    for rope in (None, rope_of(lib, 64)):
        h.norm_rope_append(rope, w.data_ptr(), w.data_ptr(), EPS, x.data_ptr(), x.stride(0), out.data_ptr(), out.stride(0), x.data_ptr(), x.data_ptr(),
                           x.stride(0), i.data_ptr(), i.data_ptr(), 0, 0, kv.data_ptr(), kv.data_ptr(), err.data_ptr(), stream())
    assert int(err) == 0 and bool((kv == 7).all())
    h.close()


def test_tables(lib):
    import torch
    h = lib.Handle(4, 2, 64, 3, 1, 4)
    none, one = torch.empty(0, dtype=torch.int32, device="cuda").data_ptr(), torch.zeros(4, dtype=torch.int32, device="cuda")
    free, count, off = torch.arange(3, dtype=torch.int32, device="cuda"), torch.tensor([3], dtype=torch.int32, device="cuda"), torch.full((2,), -7, dtype=torch.int32, device="cuda")
    h.cache_extend(none, none, none, 0, free.data_ptr(), count.data_ptr(), off.data_ptr(), none, none, 0, one.data_ptr(), stream())
    assert off.tolist() == [0, -7] and int(count) == 3
    h.cache_trim(none, none, none, 0, free.data_ptr(), count.data_ptr(), one.data_ptr(), stream())
    assert int(count) == 3 and one.tolist() == [0] * 4 and free.tolist() == [0, 1, 2]
    h.close()


def test_trees(lib):
    import torch
    h = lib.Handle(4, 2, 64, 3, 2, 4)
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    kv, err, none = torch.full((3, 2, 16, 64), 7.0, dtype=torch.bfloat16, device="cuda"), z(1), torch.empty(0, dtype=torch.int32, device="cuda").data_ptr()
    p, s = kv.data_ptr(), stream()
    # sequences without new tokens
    off, lens, bt = z(3), torch.tensor([5, 9], dtype=torch.int32, device="cuda"), z(2, 4)
    h.tree_mask(none, off.data_ptr(), lens.data_ptr(), 2, 0, none, 1, none, err.data_ptr(), s)
    ws = torch.empty(h.chunk_workspace_size(1), dtype=torch.uint8, device="cuda")
    h.chunk_plan([0, 0], [5, 9], ws.data_ptr(), ws.numel(), s)
    h.tree_attn(none, 256, p, p, bt.data_ptr(), none, 1, none, none, err.data_ptr(), s)
    # no sequences
    h.tree_mask(none, z(1).data_ptr(), none, 0, 0, none, 1, none, err.data_ptr(), s)
    h.tree_keep(none, 1, none, z(1).data_ptr(), none, none, 0, p, p, none, err.data_ptr(), s)
    h.chunk_plan([], [], ws.data_ptr(), ws.numel(), s)
    h.tree_attn(none, 256, p, p, none, none, 1, none, none, err.data_ptr(), s)
    assert int(err) == 0 and bool((kv == 7).all())
    h.close()
