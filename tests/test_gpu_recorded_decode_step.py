"""A decode step that never asks the host: pages and slots, norm + rotation + append, plan on the device, attention, sequences that end,
recorded once and replayed over changing lengths.  The pools are compared with the norm and rotation of what went in (bounds of
test_gpu_norm_rope.py), the attention with float64 on the pools as they are (tight gate)."""
import math

import numpy as np
import pytest

from oracle import chunk_oracle as K

import gates
from test_gpu_norm_rope import EPS, f64, forward, rounded
from test_rope import rope_of

pytestmark = pytest.mark.gpu

B, HQ, HKV, DIM, PAGE, LD, LAYERS = 6, 8, 2, 128, 16, 40, 2


def up(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


class Step:
    def __init__(self, lib, pool, lens):
        import torch
        self.torch, self.lib, self.pool = torch, lib, pool
        rng = self.rng = np.random.default_rng(pool)
        self.h = lib.Handle(HQ, HKV, DIM, pool, B, LD, page_size=PAGE)
        kv = lambda: torch.full((pool, HKV, PAGE, DIM), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.pools = [(kv(), kv()) for _ in range(LAYERS)]
        self.rope, self.turns = rope_of(lib, DIM), K.rope_turns(DIM, 10000.0)
        self.w = [torch.from_numpy(1 + 0.25 * rng.standard_normal(DIM)).to(torch.bfloat16).cuda() for _ in range(2)]
        ids, at = rng.permutation(pool), 0
        table = np.full((B, LD), -1, np.int32)
        for b, n in enumerate(lens):
            table[b, :-(-n // PAGE)] = ids[at:at - (-n // PAGE)]
            at += -(-n // PAGE)
        self.bt, self.lens, self.count = up(table), up(lens), up([pool - at])
        stack = np.full(pool, -1, np.int32)
        stack[:pool - at] = ids[at:]
        self.free, self.new, self.keep = up(stack), up([1] * B), up([0] * B)
        self.off, self.pos, self.slots, self.err = up([0] * (B + 1)), up([0] * B), up([0] * B), up([0])
        self.proj = [torch.empty((B, HQ + 2 * HKV, DIM), dtype=torch.bfloat16, device="cuda") for _ in range(LAYERS)]
        self.q, self.out = ([torch.empty((B, HQ, DIM), dtype=torch.bfloat16, device="cuda") for _ in range(LAYERS)] for _ in range(2))
        self.ws = torch.empty(self.h.workspace_size(), dtype=torch.uint8, device="cuda")
        # what the sequences have, in every layer
        self.model = [[[(rng.standard_normal((HKV, DIM)), np.zeros((HKV, DIM)), rng.standard_normal((HKV, DIM))) for _ in range(n)] for n in lens]
                      for _ in range(LAYERS)]
        for (k, v), m in zip(self.pools, self.model):
            for b, rows in enumerate(m):
                for t, (y, e, x) in enumerate(rows):
                    page = int(table[b, t // PAGE])
                    k[page, :, t % PAGE], v[page, :, t % PAGE] = (torch.from_numpy(z).to(torch.bfloat16).cuda() for z in (y, x))
                    rows[t] = (f64(k[page, :, t % PAGE]), e, f64(v[page, :, t % PAGE]))

    def calls(self):
        h, p, st = self.h, lambda x: x.data_ptr(), self.torch.cuda.current_stream().cuda_stream
        h.cache_trim(p(self.keep), p(self.lens), p(self.bt), B, p(self.free), p(self.count), p(self.err), st)
        h.cache_extend(p(self.new), p(self.lens), p(self.bt), B, p(self.free), p(self.count), p(self.off), p(self.pos), p(self.slots), B, p(self.err), st)
        h.plan_device(p(self.lens), B, p(self.ws), self.ws.numel(), st)
        for (k, v), x, q, out in zip(self.pools, self.proj, self.q, self.out):
            h.norm_rope_append(self.rope, p(self.w[0]), p(self.w[1]), EPS, p(x), x.stride(0), p(q), q.stride(0), p(x[:, HQ:]), p(x[:, HQ + HKV:]),
                               x.stride(0), p(self.pos), p(self.slots), p(self.off) + 4 * B, B, p(k), p(v), p(self.err), st)
            h.decode_attn(p(q), p(k), p(v), p(self.bt), p(self.lens), p(out), st)

    def inputs(self, keep):
        self.keep.copy_(up(keep))
        for x, q, out in zip(self.proj, self.q, self.out):
            x.copy_(self.torch.from_numpy(self.rng.standard_normal(x.shape)).to(x.dtype))
            out.fill_(float("nan"))

    def check(self, keep):
        """After a step that was not refused."""
        lens = self.lens.cpu().numpy()
        assert int(self.err) == 0 and self.h.debug_error_word() == 0 and lens.tolist() == [n + 1 for n in keep]
        assert int(self.count) == self.pool - sum(-(-int(n) // PAGE) for n in lens)
        table = self.bt.cpu().numpy()
        angles = K.rope_angles(np.array(keep), self.turns)
        for (k, v), x, q, out, m in zip(self.pools, self.proj, self.q, self.out, self.model):
            qy, qe = forward(f64(x[:, :HQ]), f64(self.w[0]), angles, K.HALF, 1.0, float(np.float32(EPS)))
            assert np.all(np.abs(f64(q) - qy) <= rounded(qy, qe, "bf16"))
            ky, ke = forward(f64(x[:, HQ:HQ + HKV]), f64(self.w[1]), angles, K.HALF, 1.0, float(np.float32(EPS)))
            vn = f64(x[:, HQ + HKV:])
            bits = lambda t: t.view(self.torch.int16).cpu().numpy().view(np.uint16)
            kt, vt = (K.sequence_tokens(bits(t), table, lens, "HND", None) for t in (k, v))
            for b in range(B):
                m[b] = m[b][:keep[b]] + [(ky[b], ke[b], vn[b])]
                for t, (y, e, z) in enumerate(m[b]):
                    assert np.all(np.abs(kt[b][:, t] - y) <= np.where(e > 0, rounded(y, e, "bf16"), 0.0)) and np.array_equal(vt[b][:, t], z)
                s = np.einsum("hgd,htd->hgt", f64(q[b]).reshape(HKV, -1, DIM), kt[b]) / math.sqrt(DIM)
                w = np.exp(s - s.max(-1, keepdims=True))
                ref = np.einsum("hgt,htd->hgd", w / w.sum(-1, keepdims=True), vt[b]).reshape(HQ, DIM)
                assert gates.tight_violations(f64(out[b]), ref) == 0


def test_replayed_over_changing_lengths(lib):
    import torch
    lens = [30, 0, 15, 500, 16, 300]
    s = Step(lib, 90, lens)
    side = torch.cuda.Stream()
    s.inputs(lens)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):   # one step that is not recorded
        s.calls()
    torch.cuda.synchronize()
    s.check(lens)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        s.calls()
    for step in range(6):
        had = s.lens.cpu().tolist()
        keep = [0 if (step, b) in ((1, 3), (2, 0), (4, 4)) else (n // 2 if (step, b) == (3, 5) else n) for b, n in enumerate(had)]   # some end, one goes back
        s.inputs(keep)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        s.check(keep)
    del g
    s.h.close()


def test_a_step_without_pages_leaves_the_cache_as_it_is(lib):
    """No page left: the error word says so, no row is stored, and the attention runs over what was there before."""
    import torch
    lens = [16, 32, 5, 48, 7, 20]
    s = Step(lib, 1 + 2 + 1 + 3 + 1 + 2 + 2, lens)      # three sequences need a page, two are free
    g = torch.cuda.CUDAGraph()
    s.inputs(lens)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):   # sets up the workspace outside the recording
        s.h.plan_device(s.lens.data_ptr(), B, s.ws.data_ptr(), s.ws.numel(), side.cuda_stream)
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        s.calls()
    before = [t.clone() for kv in s.pools for t in kv]
    g.replay()
    torch.cuda.synchronize()
    assert int(s.err) == lib.ERR_NO_PAGES and s.lens.cpu().tolist() == lens and int(s.count) == 2 and s.off.cpu().tolist() == [0] * (B + 1)
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(before, [t for kv in s.pools for t in kv]))
    assert s.h.debug_error_word() == 0
    s.err.zero_()
    keep = [16, 0, 5, 48, 7, 20]                          # one sequence ends: its two pages are enough now
    s.inputs(keep)
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    s.check(keep)
    del g
    s.h.close()
