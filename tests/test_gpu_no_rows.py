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
