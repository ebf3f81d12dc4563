"""The operators that write and read the paged KV cache for chunks of new tokens, as cases that can be timed and compared:
rotary positions (``rope``), rotation and append of new tokens to the pages (``append``), and causal attention of the new
tokens over the pages (``chunk``).

With ``own`` false, ``run`` computes them from elementary torch operations in 32 bits (angles in 64); with ``own`` true
it makes the library's calls.  ``exact`` is the definition in 64 bits.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
POISON = 1.0e30   # what the slots that no token owns hold (E4M3 pools: the NaN code)


# ---------------------------------------------------------------------------------------------------------- the cases
def _rope(**kw):
    d = dict(op="rope", tokens=64, heads=32, dim=128, rotary=128, layout="half", scaling="none", factor=1.0, dtype="bf16",
             fused=0, gradient=False, far=4096)
    d.update(kw)
    return d


def _append(**kw):
    d = dict(op="append", batch=64, hq=32, hkv=8, dim=128, page=16, new_lo=1, new_hi=1, ctx_lo=512, ctx_hi=4096, mix=1,
             kv="bf16", layout="half", scaling="none", factor=1.0, fused=False, order="HND")
    d.update(kw)
    return d


def _chunk(**kw):
    d = dict(op="chunk", batch=32, hq=32, hkv=8, dim=128, page=16, new_lo=1, new_hi=256, ctx_lo=128, ctx_hi=4096, mix=1,
             kv="bf16", order="HND")
    d.update(kw)
    return d


def listed():
    return [
        # q of one decode step of 64 sequences: the call is its latency
        _rope(name="rope_step_b64"),
        # a prompt's q, half of each head rotated in pairs of neighbours, positions of a long context
        _rope(name="rope_prompt_partial", tokens=8191, heads=40, rotary=64, layout="interleaved", scaling="ramp", factor=4.0,
              far=32768),
        # the gradient of the rotation in 32 bits, heads of 64, rows inside a wider projection
        _rope(name="rope_gradient_f32", tokens=16384, heads=16, dim=64, rotary=64, scaling="bands", factor=8.0, dtype="f32",
              fused=1, gradient=True, far=131072),
        # one decode step of 64 sequences: rotate q and k, append k and v
        _append(name="append_step_b64"),
        # tool returns of 1 to 256 tokens for 128 sequences, q, k, v in one projection
        _append(name="append_returns", batch=128, hq=40, new_hi=256, fused=True),
        # a prompt into an 8-bit cache of 64-token pages
        _append(name="append_prompt_e4m3", batch=2, hq=64, new_lo=8000, new_hi=8200, ctx_lo=0, ctx_hi=0, page=64, kv="e4m3",
                scaling="linear", factor=4.0),
        # single tokens of a small model: the call is its latency
        _chunk(name="chunk_single_tiny", batch=4, hq=4, hkv=1, dim=64, new_hi=1, ctx_lo=0, ctx_hi=300),
        # three drafted tokens on eight long trajectories: bound by the read of the cache
        _chunk(name="chunk_draft_long", batch=8, hq=64, new_lo=3, new_hi=3, ctx_lo=32000, ctx_hi=32765),
        # tool returns of 1 to 256 tokens on 32 trajectories
        _chunk(name="chunk_returns"),
        # the same on an 8-bit cache, five query heads per KV head
        _chunk(name="chunk_returns_e4m3", hq=40, batch=16, new_hi=500, ctx_hi=8192, kv="e4m3"),
        # four prompts at once, nothing cached before, heads of 64
        _chunk(name="chunk_prompts_d64", batch=4, hq=16, hkv=4, dim=64, new_lo=1000, new_hi=2047, ctx_lo=0, ctx_hi=0, page=32,
               order="NHD"),
        # a chunk of a long prompt: bound by arithmetic
        _chunk(name="chunk_prompt_long", batch=1, hq=64, new_lo=4096, new_hi=4096, ctx_lo=12288, ctx_hi=12288, page=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "chunk"])
    scaling = rng.choice(["none", "linear", "base", "bands", "ramp"])
    factor = 1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0])
    layout = rng.choice(["half", "interleaved"])
    if op == "rope":
        dim = rng.choice([64, 80, 96, 128, 256])
        dtype = rng.choice(["bf16", "f16", "f32"])
        heads = _log(rng, 1, 64)
        most = (16384 * 64 * 16 * 4) // (heads * dim * (4 if dtype == "f32" else 2))
        return _rope(tokens=_log(rng, 1, min(32768, most)), heads=heads, dim=dim, rotary=rng.choice([dim, dim // 2, 32]),
                     layout=layout, scaling=scaling, factor=factor, dtype=dtype, fused=rng.choice([0, 1, 2]),
                     gradient=rng.random() < 0.4, far=_log(rng, 64, 1 << 20))
    hq, hkv, dim = rng.choice([(32, 8, 128), (64, 8, 128), (40, 8, 128), (16, 4, 64), (4, 1, 64), (16, 1, 128), (8, 8, 128)])
    kv, page, order = rng.choice(["bf16", "bf16", "e4m3"]), rng.choice([16, 32, 64]), rng.choice(["HND", "NHD"])
    shape = dict(hq=hq, hkv=hkv, dim=dim, page=page, kv=kv, order=order, mix=rng.randrange(1, 1 << 20))
    if op == "append":
        batch = _log(rng, 1, 256)
        hi = _log(rng, 1, max(1, 16384 // batch))
        return _append(batch=batch, new_lo=rng.choice([1, hi]), new_hi=hi, ctx_lo=0, ctx_hi=_log(rng, 1, max(1, 131072 // batch)),
                       layout=layout, scaling=scaling, factor=factor, fused=rng.random() < 0.5, **shape)
    batch = _log(rng, 1, 64)
    most = 64 * 4096 * 16384 // (4 * hq * batch)          # new tokens x context of the largest sequence
    hi = _log(rng, 1, min(4096, max(1, int(math.sqrt(most)))))
    ctx = _log(rng, 1, max(1, min(32768, 400000 // batch, most // hi) - hi))
    return _chunk(batch=batch, new_lo=rng.choice([1, max(1, hi // 2), hi]), new_hi=hi, ctx_lo=rng.choice([0, ctx // 2, ctx]),
                  ctx_hi=ctx, **shape)


def _lens(c):
    """New tokens and length (new ones included) of each sequence: a part of the case, not of the seed."""
    rng = random.Random(c["mix"])
    new = [rng.randint(c["new_lo"], c["new_hi"]) for _ in range(c["batch"])]
    return new, [n + rng.randint(c["ctx_lo"], c["ctx_hi"]) for n in new]


def work(c):
    if c["op"] == "rope":
        n = c["tokens"] * c["heads"]
        return {"bytes": 2 * n * c["dim"] * (4 if c["dtype"] == "f32" else 2) + 4 * c["tokens"], "flops": 3 * n * c["rotary"]}
    new, lens = _lens(c)
    eb = 1 if c["kv"] == "e4m3" else 2
    rows = sum(new)
    if c["op"] == "append":
        kv = 2 * c["hkv"] * c["dim"]
        return {"bytes": rows * (2 * c["hq"] * c["dim"] * 2 + kv * 2 + kv * eb) + 4 * sum(-(-n // c["page"]) for n in new),
                "flops": 3 * rows * (c["hq"] + c["hkv"]) * c["dim"]}
    seen = sum(n * (L - n) + n * (n + 1) // 2 for n, L in zip(new, lens))
    return {"bytes": rows * c["hq"] * (c["dim"] * 4 + 4) + 2 * sum(lens) * c["hkv"] * c["dim"] * eb,
            "flops": 4 * c["dim"] * c["hq"] * seen}


# --------------------------------------------------------------------------------------------------------- the inputs
BAND_LOW, BAND_HIGH, RAMP_LOW, RAMP_HIGH, BASE = 1.0, 4.0, 1.0, 32.0, 500000.0


def _original(c):
    return 8192


def _frequencies(c, rotary):
    """Angle per position of each pair, in float64, and the factor on the result."""
    i = np.arange(rotary // 2, dtype=np.float64)
    f, base = c["factor"], BASE
    if c["scaling"] == "base":
        base = BASE * f ** (rotary / (rotary - 2))
    theta = base ** (-2.0 * i / rotary)
    if c["scaling"] == "linear":
        theta = theta / f
    if c["scaling"] == "bands":
        turns = _original(c) * theta / (2 * np.pi)            # turns within the length that was trained on
        keep = np.clip((turns - BAND_LOW) / (BAND_HIGH - BAND_LOW), 0.0, 1.0)
        theta = theta * keep + theta / f * (1 - keep)
    if c["scaling"] == "ramp":
        at = [rotary * math.log(_original(c) / (b * 2 * math.pi)) / (2 * math.log(BASE)) for b in (RAMP_HIGH, RAMP_LOW)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rotary - 1)
        gone = np.clip((i - lo) / max(hi - lo, 0.001), 0.0, 1.0)
        theta = theta * (1 - gone) + theta / f * gone
    return theta, (0.1 * math.log(f) + 1.0 if c["scaling"] == "ramp" else 1.0)


def _own_rope(b, c, rotary):
    kind = {"none": b.ROPE_SCALE_NONE, "linear": b.ROPE_SCALE_LINEAR, "base": b.ROPE_SCALE_BASE, "bands": b.ROPE_SCALE_BANDS,
            "ramp": b.ROPE_SCALE_RAMP}[c["scaling"]]
    low, high = {"bands": (BAND_LOW, BAND_HIGH), "ramp": (RAMP_LOW, RAMP_HIGH)}.get(c["scaling"], (0.0, 0.0))
    return b.libra_rope_init(rotary, b.ROPE_HALF if c["layout"] == "half" else b.ROPE_INTERLEAVED, BASE, kind, c["factor"], low,
                             high, _original(c))


def prepare(case, seed):
    c, dev = case, torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    s = {"case": c}
    if c["op"] == "rope":
        # rows of a projection that holds `fused` more groups of heads behind these
        wide = torch.randn((c["tokens"], (1 + c["fused"]) * c["heads"], c["dim"]), generator=g, device=dev).to(DTYPES[c["dtype"]])
        s["x"] = wide[:, :c["heads"]]
        s["positions"] = torch.randint(0, c["far"], (c["tokens"],), generator=g, device=dev, dtype=torch.int32)
        s["out"] = torch.empty((c["tokens"], c["heads"], c["dim"]), dtype=DTYPES[c["dtype"]], device=dev)
        theta, s["magnitude"] = _frequencies(c, c["rotary"])
        s["theta"] = torch.from_numpy(theta).to(dev)
        if own:
            from paper_2606_03077_b200 import binding
            s["b"], s["rope"] = binding, _own_rope(binding, c, c["rotary"])
            s["dtype"] = {"bf16": binding.ROPE_BF16, "f16": binding.ROPE_F16, "f32": binding.ROPE_F32}[c["dtype"]]
        return s

    new, lens = _lens(c)
    B, hq, hkv, D, P = c["batch"], c["hq"], c["hkv"], c["dim"], c["page"]
    rows, pages = sum(new), [-(-n // P) for n in lens]
    need, ld = sum(pages), max(1, max(pages))
    pool = need + max(1, need // 8)
    place = torch.randperm(pool, generator=g, device=dev)[:need].to(torch.int32).cpu().numpy()
    table, at = np.full((B, ld), -1, dtype=np.int32), 0
    for b, n in enumerate(pages):
        table[b, :n] = place[at:at + n]
        at += n
    s["block_table"] = torch.from_numpy(table).to(dev)
    s["seq_lens"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    s["q_offsets"] = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device=dev)
    shape = (pool, hkv, P, D) if c["order"] == "HND" else (pool, P, hkv, D)
    kinds = torch.bfloat16 if c["kv"] == "bf16" else torch.float8_e4m3fn

    def draw_pool():
        x = torch.empty(shape, dtype=kinds, device=dev)
        for p0 in range(0, pool, 4096):
            x[p0:p0 + 4096] = torch.randn((min(4096, pool - p0),) + shape[1:], generator=g, device=dev).to(kinds)
        return x

    s["k"], s["v"] = draw_pool(), draw_pool()
    s["k_scale"], s["v_scale"] = (1.0, 1.0) if c["kv"] == "bf16" else (0.0625, 0.03125)
    s["rows"], s["most_new"], s["most"] = rows, max(new), max(lens)
    proj = torch.randn((rows, hq + 2 * hkv, D), generator=g, device=dev).to(torch.bfloat16)
    s["q"] = proj[:, :hq]
    s["error"] = torch.zeros(1, dtype=torch.int32, device=dev)
    if c["op"] == "append":
        s["k_new"], s["v_new"] = proj[:, hq:hq + hkv], proj[:, hq + hkv:]
        if not c["fused"]:
            s["q"], s["k_new"], s["v_new"] = (x.contiguous() for x in (s["q"], s["k_new"], s["v_new"]))
        theta, s["magnitude"] = _frequencies(c, D)
        s["theta"] = torch.from_numpy(theta).to(dev)
    else:
        s["q"] = s["q"].contiguous()
        poison = POISON if c["kv"] == "bf16" else float("nan")
        for b, L in enumerate(lens):      # what lies behind a sequence's end in its last page may be anything
            if L % P:
                last = int(table[b, L // P])
                for x in (s["k"], s["v"]):
                    (x[last].transpose(0, 1) if c["order"] == "HND" else x[last])[L % P:] = poison
        s["lse"] = torch.empty((rows, hq), dtype=torch.float32, device=dev)
    s["out"] = torch.empty((rows, hq, D), dtype=torch.bfloat16, device=dev)
    if own:
        from paper_2606_03077_b200 import binding
        s["b"] = binding
        strides = (0, 0, 0) if c["order"] == "HND" else (P * hkv * D, D, hkv * D)
        h = s["handle"] = binding.Handle(hq, hkv, D, pool, B, ld, page_size=P, kv_strides=strides)
        if c["kv"] == "e4m3":
            h.set_kv_dtype(binding.KV_E4M3, s["k_scale"], s["v_scale"])
        if c["op"] == "append":
            s["rope"] = _own_rope(binding, c, D)
        else:
            s["workspace"] = torch.empty(h.chunk_workspace_size(rows), dtype=torch.uint8, device=dev)
            h.chunk_plan(np.asarray(new, dtype=np.int32), np.asarray(lens, dtype=np.int32), s["workspace"].data_ptr(),
                         s["workspace"].numel(), torch.cuda.current_stream().cuda_stream)
    return s


# ------------------------------------------------------------------------------------------------------ the operators
def _rotate(x, positions, theta, magnitude, layout, gradient=False):
    """x: float32 [tokens, heads, channels]; the first 2 * len(theta) channels are rotated."""
    n = theta.numel()
    angle = positions.double()[:, None] * theta
    cos, sin = ((f * magnitude).float()[:, None] for f in (angle.cos(), angle.sin()))
    if gradient:
        sin = -sin
    r, rest = x[..., :2 * n], x[..., 2 * n:]
    a, b = (r[..., :n], r[..., n:]) if layout == "half" else (r[..., 0::2], r[..., 1::2])
    ya, yb = a * cos - b * sin, a * sin + b * cos
    y = torch.cat((ya, yb), dim=-1) if layout == "half" else torch.stack((ya, yb), dim=-1).flatten(-2)
    return torch.cat((y, rest), dim=-1)


def _plain_append(s):
    c = s["case"]
    row = torch.arange(s["rows"], device=s["q"].device, dtype=torch.int32)
    b = torch.searchsorted(s["q_offsets"], row, right=True) - 1
    pos = s["seq_lens"][b] - s["q_offsets"][b + 1] + row
    q = _rotate(s["q"].float(), pos, s["theta"], s["magnitude"], c["layout"]).to(torch.bfloat16)
    k = _rotate(s["k_new"].float(), pos, s["theta"], s["magnitude"], c["layout"])
    v = s["v_new"].float()
    if c["kv"] == "e4m3":
        k, v = ((x / f).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8) for x, f in ((k, s["k_scale"]), (v, s["v_scale"])))
        pools = s["k"].view(torch.uint8), s["v"].view(torch.uint8)
    else:
        k, v, pools = k.to(torch.bfloat16), v.to(torch.bfloat16), (s["k"], s["v"])
    page, slot = s["block_table"][b, pos // c["page"]].long(), (pos % c["page"]).long()
    if c["order"] == "HND":
        pools[0][page, :, slot], pools[1][page, :, slot] = k, v
    else:
        pools[0][page, slot], pools[1][page, slot] = k, v
    return {"q": q, "k": s["k"], "v": s["v"]}


def _plain_chunk(s):
    c = s["case"]
    B, hq, hkv, D, P = c["batch"], c["hq"], c["hkv"], c["dim"], c["page"]
    dev, G, N, T = s["q"].device, c["hq"] // c["hkv"], s["most_new"], s["most"]
    new = s["q_offsets"][1:] - s["q_offsets"][:-1]
    table = s["block_table"].clamp(min=0).long()
    t = torch.arange(table.shape[1] * P, device=dev)

    def tokens(pool, scale):
        x = pool.view(torch.uint8)[table].view(pool.dtype).float() * scale
        x = x.transpose(1, 2) if c["order"] == "HND" else x.permute(0, 3, 1, 2, 4)
        x = x.reshape(B, hkv, -1, D)
        return torch.where((t < s["seq_lens"][:, None])[:, None, :, None], x, 0.0)[:, :, :T]

    k, v = tokens(s["k"], s["k_scale"]), tokens(s["v"], s["v_scale"])
    i = torch.arange(N, device=dev)
    live = i < new[:, None]                                                         # [B, N]
    row = torch.where(live, s["q_offsets"][:-1, None] + i, 0)
    q = s["q"][row].float().view(B, N, hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, hkv, N * G, D)
    p = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(D)).view(B, hkv, N, G, T)
    seen = t[:T] < (s["seq_lens"] - new)[:, None, None] + i[:, None] + 1                # [B, N, T]
    p.masked_fill_(~seen[:, None, :, None, :], float("-inf"))
    m = p.amax(dim=-1, keepdim=True)
    p.sub_(torch.where(m > float("-inf"), m, 0.0)).exp_()
    z = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p.view(B, hkv, N * G, T), v).view(B, hkv, N, G, D)
    o = torch.where(z > 0, o / z, 0.0)
    lse = (m + z.log()).squeeze(-1)
    o = o.permute(0, 2, 1, 3, 4).reshape(B, N, hq, D)[live].to(torch.bfloat16)
    return {"out": o, "lse": lse.permute(0, 2, 1, 3).reshape(B, N, hq)[live]}


def run(state):
    s = state
    c = s["case"]
    if not own:
        if c["op"] == "rope":
            return _rotate(s["x"].float(), s["positions"], s["theta"], s["magnitude"], c["layout"], c["gradient"]).to(s["x"].dtype)
        return _plain_append(s) if c["op"] == "append" else _plain_chunk(s)
    b, stream = s["b"], torch.cuda.current_stream().cuda_stream
    if c["op"] == "rope":
        x, out = s["x"], s["out"]
        b.libra_rope_apply(0, s["rope"], x.data_ptr(), out.data_ptr(), s["dtype"], s["positions"].data_ptr(), c["tokens"],
                           c["heads"], c["dim"], x.stride(0), x.stride(1), out.stride(0), out.stride(1),
                           b.ROPE_GRADIENT if c["gradient"] else b.ROPE_FORWARD, stream)
        return out
    h = s["handle"]
    if c["op"] == "append":
        h.rope_append(s["rope"], s["q"].data_ptr(), s["q"].stride(0), s["out"].data_ptr(), s["out"].stride(0),
                      s["k_new"].data_ptr(), s["v_new"].data_ptr(), s["k_new"].stride(0), s["q_offsets"].data_ptr(),
                      s["seq_lens"].data_ptr(), s["block_table"].data_ptr(), c["batch"], s["rows"], s["k"].data_ptr(),
                      s["v"].data_ptr(), s["error"].data_ptr(), stream)
        return {"q": s["out"], "k": s["k"], "v": s["v"]}
    h.chunk_attn(s["q"].data_ptr(), s["q"].stride(0), s["k"].data_ptr(), s["v"].data_ptr(), s["block_table"].data_ptr(),
                 s["out"].data_ptr(), s["lse"].data_ptr(), s["error"].data_ptr(), stream)
    return {"out": s["out"], "lse": s["lse"]}


# ------------------------------------------------------------------------------------------------------ in 64 bits
def _exact_rotate(x, positions, theta, magnitude, layout, gradient):
    """The rotation as a product of complex numbers."""
    x, n = x.double(), theta.numel()
    turn = torch.polar(torch.full_like(theta, magnitude).expand(len(positions), n), positions.double()[:, None] * theta)[:, None]
    turn = turn.conj() if gradient else turn
    y = x.clone()
    even, odd = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    z = torch.complex(x[..., even], x[..., odd]) * turn
    y[..., even], y[..., odd] = z.real, z.imag
    return y


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "rope":
        return _exact_rotate(s["x"], s["positions"], s["theta"], s["magnitude"], c["layout"], c["gradient"])
    new, lens = _lens(c)
    first = [0] + list(np.cumsum(new))
    P, G = c["page"], c["hq"] // c["hkv"]
    if c["op"] == "append":
        pos = torch.tensor([L - n + i for n, L in zip(new, lens) for i in range(n)], device=s["q"].device)
        q = _exact_rotate(s["q"], pos, s["theta"], s["magnitude"], c["layout"], False)
        pools = []
        k_new = _exact_rotate(s["k_new"], pos, s["theta"], s["magnitude"], c["layout"], False) / s["k_scale"]
        for pool, x in ((s["k"], k_new), (s["v"], s["v_new"].double() / s["v_scale"])):
            y = pool.double()
            y = y.transpose(1, 2) if c["order"] == "HND" else y             # [page, slot, head, channel]
            for b in range(c["batch"]):
                at = pos[first[b]:first[b + 1]]
                y[s["block_table"][b, at // P].long(), at % P] = x[first[b]:first[b + 1]]
            y = y.transpose(1, 2) if c["order"] == "HND" else y
            pools.append(y.clamp(-448.0, 448.0) if c["kv"] == "e4m3" else y)
        return {"q": q, "k": pools[0], "v": pools[1]}
    out = torch.zeros((s["rows"], c["hq"], c["dim"]), dtype=torch.float64, device=s["q"].device)
    lse = torch.full((s["rows"], c["hq"]), float("-inf"), dtype=torch.float64, device=s["q"].device)
    for b, (n, L) in enumerate(zip(new, lens)):
        ids = s["block_table"][b, :-(-L // P)].long()
        for g in range(c["hkv"]):
            k, v = ((x[ids, g] if c["order"] == "HND" else x[ids, :, g]).double().flatten(0, 1)[:L] * f
                    for x, f in ((s["k"], s["k_scale"]), (s["v"], s["v_scale"])))
            for h in range(g * G, (g + 1) * G):
                a = s["q"][first[b]:first[b + 1], h].double() @ k.T / math.sqrt(c["dim"])
                a = a + torch.triu(torch.full_like(a, float("-inf")), diagonal=L - n + 1)
                z = torch.logsumexp(a, dim=-1)
                lse[first[b]:first[b + 1], h] = z
                out[first[b]:first[b + 1], h] = torch.exp(a - z[:, None]) @ v
    return {"out": out, "lse": lse}
