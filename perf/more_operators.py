"""The operators of a step over the paged KV cache that takes drafted tokens, as cases that can be timed and compared: pages and
slots handed out on the GPU (``tables``), norms of the heads of q and k with the rotation by position (``norm``), the same with the
append to the pages (``append``), and attention of trees of drafted tokens over the pages (``tree``).

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
BASE, EPS = 500000.0, 1.0e-6


# ---------------------------------------------------------------------------------------------------------- the cases
def _tables(**kw):
    d = dict(op="tables", batch=64, page=16, new_lo=1, new_hi=1, ctx_lo=1, ctx_hi=8192, mix=1, drafts="none", hkv=8, dim=128,
             kv="bf16", order="HND")
    d.update(kw)
    return d


def _norm(**kw):
    d = dict(op="norm", tokens=64, hq=32, hkv=8, dim=128, rotary=128, layout="half", dtype="bf16", fused=False, gradient=False,
             far=4096)
    d.update(kw)
    return d


def _append(**kw):
    d = dict(op="append", batch=64, hq=32, hkv=8, dim=128, rotary=128, page=16, new_lo=1, new_hi=1, ctx_lo=512, ctx_hi=4096, mix=1,
             kv="bf16", layout="half", drafts="none", fused=True, order="HND")
    d.update(kw)
    return d


def _tree(**kw):
    d = dict(op="tree", batch=32, hq=32, hkv=8, dim=128, page=16, new_lo=16, new_hi=16, ctx_lo=128, ctx_hi=4096, mix=1,
             drafts="bushy", kv="bf16", order="HND")
    d.update(kw)
    return d


def listed():
    return [
        # one decode step of 64 sequences: a page for those whose last one is full, the slots of the step, and back
        _tables(name="tables_step_b64"),
        # prompts and tool returns of 256 sequences in one step
        _tables(name="tables_prompts", batch=256, new_lo=1, new_hi=900, ctx_lo=0),
        # the bookkeeping of a step that verifies trees of up to 32 drafted tokens for 64 sequences, one layer's rows moved
        _tables(name="tables_drafts_b64", new_lo=8, new_hi=32, ctx_hi=2048, drafts="bushy"),
        # q and k of one decode step of 64 sequences: the call is its latency
        _norm(name="norm_step_b64"),
        # q and k of a prompt in fp16, half of each head rotated in pairs of neighbours, rows inside the layer's projection
        _norm(name="norm_prompt_f16", tokens=8191, hq=40, rotary=64, layout="interleaved", dtype="f16", fused=True, far=32768),
        # the gradient for a training batch: of q, k and both weights, rows inside the gradient of the projection
        _norm(name="norm_gradient", tokens=16384, fused=True, gradient=True, far=16384),
        # the gradient in 32 bits, heads of 64
        _norm(name="norm_gradient_f32", tokens=4001, hq=16, hkv=4, dim=64, rotary=64, dtype="f32", gradient=True, far=131072),
        # trees of 1 to 32 drafted tokens for 128 sequences, positions by depth, q, k, v in one projection
        _append(name="append_drafts", batch=128, hq=40, new_hi=32, drafts="bushy"),
        # two prompts into an 8-bit cache of 64-token pages
        _append(name="append_prompt_e4m3", batch=2, hq=64, new_lo=8000, new_hi=8200, ctx_lo=0, ctx_hi=0, page=64, kv="e4m3"),
        # a few drafted tokens of a small model: the call is its latency
        _tree(name="tree_small", batch=4, hq=4, hkv=1, dim=64, new_lo=2, new_hi=7, ctx_lo=0, ctx_hi=300),
        # trees of 16 on eight long trajectories: bound by the read of the cache
        _tree(name="tree_long", batch=8, hq=64, ctx_lo=32000, ctx_hi=32752),
        # trees of 16 to 64 for 32 sequences over an 8-bit cache, five query heads per KV head
        _tree(name="tree_wide_e4m3", hq=40, new_hi=64, ctx_hi=8192, kv="e4m3", page=32, order="NHD"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "norm", "append", "tree"])
    layout = rng.choice(["half", "interleaved"])
    if op == "norm":
        dim = rng.choice([64, 80, 96, 128, 256])
        dtype = rng.choice(["bf16", "f16", "f32"])
        hkv = rng.choice([0, 1, 2, 4, 8])
        hq = max(1, hkv) * rng.choice([1, 4, 5, 8])
        gradient = rng.random() < 0.5
        most = 16384 * 40 * 128 * 2 // ((hq + hkv) * dim * (4 if dtype == "f32" else 2))
        return _norm(tokens=_log(rng, 1, min(32768, most)), hq=hq, hkv=hkv, dim=dim, rotary=rng.choice([dim, dim // 2, 32]),
                     layout=layout, dtype=dtype, fused=rng.random() < 0.5, gradient=gradient, far=_log(rng, 64, 1 << 20))
    hq, hkv, dim = rng.choice([(32, 8, 128), (64, 8, 128), (40, 8, 128), (16, 4, 64), (4, 1, 64), (16, 1, 128), (8, 8, 128)])
    kv, page, order = rng.choice(["bf16", "bf16", "e4m3"]), rng.choice([16, 32, 64]), rng.choice(["HND", "NHD"])
    drafts = rng.choice(["chain", "bushy", "wide"])
    shape = dict(hkv=hkv, dim=dim, page=page, kv=kv, order=order, mix=rng.randrange(1, 1 << 20))
    if op == "tables":
        batch = _log(rng, 1, 512)
        if rng.random() < 0.5:
            hi = _log(rng, 1, min(64, max(1, 4096 // batch)))
            return _tables(batch=batch, new_lo=rng.choice([1, hi]), new_hi=hi, ctx_lo=0, ctx_hi=_log(rng, 1, max(1, 65536 // batch)),
                           drafts=drafts, **shape)
        hi = _log(rng, 1, max(1, 131072 // batch))
        return _tables(batch=batch, new_lo=rng.choice([0, 1, hi]), new_hi=hi, ctx_lo=0, ctx_hi=_log(rng, 1, max(1, 1 << 20) // batch),
                       **shape)
    if op == "append":
        batch = _log(rng, 1, 256)
        hi = _log(rng, 1, max(1, 16384 // batch))
        trees = hi <= 64 and rng.random() < 0.5
        return _append(batch=batch, hq=hq, rotary=rng.choice([dim, dim // 2, 32]), new_lo=rng.choice([1, hi]), new_hi=hi, ctx_lo=0,
                       ctx_hi=_log(rng, 1, max(1, 131072 // batch)), layout=layout, drafts=drafts if trees else "none",
                       fused=rng.random() < 0.5, **shape)
    batch = _log(rng, 1, 64)
    hi = _log(rng, 1, max(1, min(128, 2048 // batch)))
    ctx = _log(rng, 1, max(1, min(32768 - hi, 262144 // batch)))
    return _tree(batch=batch, hq=hq, new_lo=rng.choice([1, max(1, hi // 2), hi]), new_hi=hi, ctx_lo=rng.choice([0, ctx // 2, ctx]),
                 ctx_hi=ctx, drafts=drafts, **shape)


def _lens(c):
    """New tokens and cached ones of each sequence: a part of the case, not of the seed."""
    rng = random.Random(c["mix"])
    new = [rng.randint(c["new_lo"], c["new_hi"]) for _ in range(c["batch"])]
    return new, [rng.randint(c["ctx_lo"], c["ctx_hi"]) for _ in new]


def _parents(c, new):
    """Of every drafted token its parent's place among its sequence's, -1: it follows the last cached token."""
    rng, out = random.Random(c["mix"] + 1), []
    for n in new:
        for i in range(n):
            lo = {"chain": i - 1, "bushy": max(-1, i // 2 - 1), "wide": -1}[c["drafts"]]
            out.append(rng.randint(lo, {"chain": i - 1, "bushy": i - 1, "wide": min(i - 1, 1)}[c["drafts"]]))
    return out


def _accepted(c, new, parents):
    """A path from the root of each tree, as places in ascending order.  Cut short so that no token of it stands where another one
    goes: moving its rows together twice is then the same as once."""
    rng, out, at = random.Random(c["mix"] + 2), [], 0
    for n in new:
        path, i = [], rng.randrange(-1, n)
        while i >= 0:
            path.append(i)
            i = parents[at + i]
        path.reverse()
        m = len(path)
        while any(j != i and j < m for i, j in enumerate(path[:m])):
            m -= 1
        out.append(path[:m])
        at += n
    return out


def _words(c):
    """32-bit words of a row of the mask."""
    return -(-c["new_hi"] // 32)


def work(c):
    if c["op"] == "norm":
        n, eb = c["tokens"] * (c["hq"] + c["hkv"]) * c["dim"], 4 if c["dtype"] == "f32" else 2
        return {"bytes": (3 if c["gradient"] else 2) * n * eb + 4 * c["tokens"], "flops": (14 if c["gradient"] else 7) * n}
    new, ctx = _lens(c)
    rows, eb, P = sum(new), 1 if c["kv"] == "e4m3" else 2, c["page"]
    if c["op"] == "tables":
        pages = sum(-(-(n + L) // P) - -(-L // P) for n, L in zip(new, ctx))
        moved = 0
        if c["drafts"] != "none":
            moved = sum(i != j for p in _accepted(c, new, _parents(c, new)) for i, j in enumerate(p))
        row = 8 if c["drafts"] == "none" else 20 + 4 * _words(c)
        return {"bytes": 28 * c["batch"] + 16 * pages + row * rows + moved * 4 * c["hkv"] * c["dim"] * eb, "flops": 8 * rows}
    if c["op"] == "append":
        kv = 2 * c["hkv"] * c["dim"]
        return {"bytes": rows * (2 * c["hq"] * c["dim"] * 2 + kv * 2 + kv * eb + 8), "flops": 7 * rows * (c["hq"] + c["hkv"]) * c["dim"]}
    seen, at, parents = 0, 0, _parents(c, new)
    for n, L in zip(new, ctx):
        depth = []
        for i in range(n):
            p = parents[at + i]
            depth.append(1 + (depth[p] if p >= 0 else 0))
        seen += n * L + sum(depth)
        at += n
    return {"bytes": rows * (c["hq"] * (c["dim"] * 4 + 4) + 4 * _words(c)) + 2 * (sum(ctx) + rows) * c["hkv"] * c["dim"] * eb,
            "flops": 4 * c["dim"] * c["hq"] * seen}


# --------------------------------------------------------------------------------------------------------- the inputs
def _theta(rotary):
    return BASE ** (-2.0 * np.arange(rotary // 2, dtype=np.float64) / rotary)


def _own_rope(b, c):
    return b.libra_rope_init(c["rotary"], b.ROPE_HALF if c["layout"] == "half" else b.ROPE_INTERLEAVED, BASE)


def _stream():
    return torch.cuda.current_stream().cuda_stream


def prepare(case, seed):
    c, dev = case, torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    s = {"case": c}
    randn = lambda *shape: torch.randn(shape, generator=g, device=dev)
    if c["op"] == "norm":
        t, kinds = c["tokens"], DTYPES[c["dtype"]]

        def heads(extra=0):   # q and k: rows of a projection that holds v (or its gradient) too, or arrays of their own
            wide = (randn(t, c["hq"] + 2 * c["hkv"], c["dim"]) * 1.5).to(kinds)
            parts = wide[:, :c["hq"]], wide[:, c["hq"]:c["hq"] + c["hkv"]]
            return parts if c["fused"] else tuple(x.contiguous() for x in parts)

        s["x"] = heads()
        s["weight"] = tuple((1.0 + 0.25 * randn(c["dim"])).to(kinds) for _ in range(2))
        s["positions"] = torch.randint(0, c["far"], (t,), generator=g, device=dev, dtype=torch.int32)
        s["theta"] = torch.from_numpy(_theta(c["rotary"])).to(dev)
        if c["gradient"]:
            s["grad"] = heads()
            s["grad_weight"] = tuple(torch.empty(c["dim"], dtype=torch.float32, device=dev) for _ in range(2))
        s["out"] = heads()   # overwritten
        if own:
            from paper_2606_03077_b200 import binding
            s["b"], s["rope"] = binding, _own_rope(binding, c)
            s["dtype"] = {"bf16": binding.ROPE_BF16, "f16": binding.ROPE_F16, "f32": binding.ROPE_F32}[c["dtype"]]
            if c["gradient"]:
                n = binding.libra_norm_rope_workspace_size(0, c["dim"])
                s["workspace"] = torch.empty(n, dtype=torch.uint8, device=dev)
        return s

    new, ctx = _lens(c)
    B, hkv, D, P = c["batch"], c["hkv"], c["dim"], c["page"]
    lens = [n + L for n, L in zip(new, ctx)]
    rows, pages = sum(new), [-(-n // P) for n in (ctx if c["op"] == "tables" else lens)]
    need, ld = sum(-(-n // P) for n in lens), max(1, max(-(-n // P) for n in lens))
    pool = need + max(1, need // 8)
    order = torch.randperm(pool, generator=g, device=dev).to(torch.int32)
    place, owned = order.cpu().numpy(), sum(pages)
    table, at = np.full((B, ld), -1, dtype=np.int32), 0
    for b, n in enumerate(pages):
        table[b, :n] = place[at:at + n]
        at += n
    s["block_table"] = torch.from_numpy(table).to(dev)
    s["q_offsets"] = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device=dev)
    s["rows"], s["most_new"], s["most"] = rows, max(new), max(lens)
    s["error"] = torch.zeros(1, dtype=torch.int32, device=dev)
    if c["drafts"] != "none":
        parents = _parents(c, new)
        s["parents"] = torch.tensor(parents, dtype=torch.int32, device=dev)
        s["mask"] = torch.empty((rows, _words(c)), dtype=torch.int32, device=dev)
    pools = c["op"] != "tables" or c["drafts"] != "none"
    if pools:
        shape = (pool, hkv, P, D) if c["order"] == "HND" else (pool, P, hkv, D)
        kinds = torch.bfloat16 if c["kv"] == "bf16" else torch.float8_e4m3fn

        def draw_pool():
            x = torch.empty(shape, dtype=kinds, device=dev)
            for p0 in range(0, pool, 4096):
                x[p0:p0 + 4096] = randn(min(4096, pool - p0), *shape[1:]).to(kinds)
            return x

        s["k"], s["v"] = draw_pool(), draw_pool()
        s["k_scale"], s["v_scale"] = (1.0, 1.0) if c["kv"] == "bf16" else (0.0625, 0.03125)
    if own:
        from paper_2606_03077_b200 import binding
        s["b"] = binding
        strides = (0, 0, 0) if c["order"] == "HND" else (P * hkv * D, D, hkv * D)
        h = s["handle"] = binding.Handle(c.get("hq", hkv), hkv, D, pool, B, ld, page_size=P, kv_strides=strides)
        if c["kv"] == "e4m3":
            h.set_kv_dtype(binding.KV_E4M3, s["k_scale"] if pools else 1.0, s["v_scale"] if pools else 1.0)

    if c["op"] == "tables":
        s["seq_lens"] = torch.tensor(ctx, dtype=torch.int32, device=dev)
        s["keep"] = s["seq_lens"].clone()          # what is kept at the end of the pass: nothing of what is new
        s["new"] = torch.tensor(new, dtype=torch.int32, device=dev)
        s["free"] = torch.zeros(pool, dtype=torch.int32, device=dev)
        s["free"][:pool - owned] = order[owned:]
        s["free_count"] = torch.tensor([pool - owned], dtype=torch.int32, device=dev)
        s["positions"], s["slots"] = (torch.empty(rows, dtype=torch.int32, device=dev) for _ in range(2))
        if c["drafts"] != "none":
            accepted = _accepted(c, new, parents)
            kept = np.zeros((B, max(1, max(len(p) for p in accepted))), dtype=np.int32)
            for b, p in enumerate(accepted):
                kept[b, :len(p)] = p
            s["kept"] = torch.from_numpy(kept).to(dev)
            s["n_kept"] = torch.tensor([len(p) for p in accepted], dtype=torch.int32, device=dev)
            s["new_lens"] = torch.empty(B, dtype=torch.int32, device=dev)
        return s

    hq = c["hq"]
    s["seq_lens"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    proj = randn(rows, hq + 2 * hkv, D).to(torch.bfloat16)
    s["q"] = proj[:, :hq]
    s["out"] = torch.empty((rows, hq, D), dtype=torch.bfloat16, device=dev)
    if c["op"] == "append":
        s["k_new"], s["v_new"] = proj[:, hq:hq + hkv], proj[:, hq + hkv:]
        if not c["fused"]:
            s["q"], s["k_new"], s["v_new"] = (x.contiguous() for x in (s["q"], s["k_new"], s["v_new"]))
        s["weight"] = tuple((1.0 + 0.25 * randn(D)).to(torch.bfloat16) for _ in range(2))
        s["theta"] = torch.from_numpy(_theta(c["rotary"])).to(dev)
        position, slot, at = [], [], 0
        for b, (n, L) in enumerate(zip(new, ctx)):
            depth = list(range(n))
            if c["drafts"] != "none":
                for i in range(n):
                    depth[i] = 1 + depth[parents[at + i]] if parents[at + i] >= 0 else 0
            position += [L + d for d in depth]
            slot += [int(table[b, (L + i) // P]) * P + (L + i) % P for i in range(n)]
            at += n
        s["positions"], s["slots"] = (torch.tensor(x, dtype=torch.int32, device=dev) for x in (position, slot))
        if own:
            s["rope"] = _own_rope(binding, c)
        return s
    s["q"] = s["q"].contiguous()
    poison = POISON if c["kv"] == "bf16" else float("nan")
    for b, L in enumerate(lens):      # what lies behind a sequence's end in its last page may be anything
        if L % P:
            last = int(table[b, L // P])
            for x in (s["k"], s["v"]):
                (x[last].transpose(0, 1) if c["order"] == "HND" else x[last])[L % P:] = poison
    s["lse"] = torch.empty((rows, hq), dtype=torch.float32, device=dev)
    if own:   # the plan and the mask serve all layers of a step
        s["workspace"] = torch.empty(h.chunk_workspace_size(rows), dtype=torch.uint8, device=dev)
        h.chunk_plan(np.asarray(new, dtype=np.int32), np.asarray(lens, dtype=np.int32), s["workspace"].data_ptr(),
                     s["workspace"].numel(), _stream())
        h.tree_mask(s["parents"].data_ptr(), s["q_offsets"].data_ptr(), s["seq_lens"].data_ptr(), B, rows, s["mask"].data_ptr(),
                    _words(c), 0, s["error"].data_ptr(), _stream())
    else:
        s["mask"] = _plain_mask(s)[0]
    return s


# ------------------------------------------------------------------------------------------------------ the operators
def _row_owner(counts, total):
    return torch.repeat_interleave(torch.arange(counts.numel(), device=counts.device), counts.long(), output_size=total)


def _plain_mask(s):
    """Each drafted token's ancestors and itself as bits, and how many ancestors it has."""
    c, rows, words = s["case"], s["rows"], _words(s["case"])
    off, parents = s["q_offsets"].long(), s["parents"].long()
    b = _row_owner(off[1:] - off[:-1], rows)
    first = off[b]
    own_place = torch.arange(rows, device=off.device) - first
    mask = torch.zeros((rows, words), dtype=torch.int64, device=off.device)
    depth = torch.full((rows,), -1, dtype=torch.int64, device=off.device)
    at = own_place
    word = torch.arange(words, device=off.device)
    for _ in range(s["most_new"]):
        live = at >= 0
        bit = torch.where(live[:, None] & (word == (at >> 5)[:, None]), (1 << (at & 31).clamp(min=0))[:, None], 0)
        mask = mask + bit                  # an ancestor is met once
        depth = depth + live
        at = torch.where(live, parents[(first + at).clamp(min=0)], -1)
    mask = torch.where(mask >= 1 << 31, mask - (1 << 32), mask)
    return mask.to(torch.int32), depth


def _plain_tables(s):
    c, P, rows = s["case"], s["case"]["page"], s["rows"]
    table, lens, new = s["block_table"], s["seq_lens"], s["new"]
    had = (lens + P - 1) // P
    want = (lens + new + P - 1) // P - had
    off = torch.cumsum(torch.cat((torch.zeros_like(new[:1]), new)), 0).to(torch.int32)
    b = _row_owner(new, rows)
    pos = lens[b] + torch.arange(rows, device=lens.device, dtype=torch.int32) - off[b]
    begins = torch.cumsum(want, 0) - want
    page = pos // P
    fresh = page >= had[b]
    taken = s["free"][(s["free_count"] - 1 - begins[b] - (page - had[b])).clamp(min=0).long()]
    ids = torch.where(fresh, taken, table[b, page.long()])
    table[b, page.long()] = ids
    s["slots"].copy_(ids * P + pos % P)
    s["positions"].copy_(pos)
    s["q_offsets"].copy_(off)
    lens += new
    s["free_count"] -= want.sum().to(torch.int32)
    out = {"q_offsets": s["q_offsets"], "positions": s["positions"], "slots": s["slots"], "block_table": table}
    if c["drafts"] != "none":
        s["mask"], depth = _plain_mask(s)
        ctx = lens - new
        s["positions"].copy_(ctx[b] + depth)
        # the rows of the kept tokens, moved together at the end of what was cached
        i = torch.arange(s["kept"].shape[1], device=lens.device)
        live = i < s["n_kept"][:, None]
        frm, to = (ctx[:, None] + x for x in (torch.where(live, s["kept"], 0), torch.where(live, i, 0)))
        frm, to = (torch.gather(table, 1, (x // P).long()).long() * P + x % P for x in (frm, to))
        live, frm, to = live.flatten(), frm.flatten(), to.flatten()
        frm, to = frm[live], to[live]
        for pool in (s["k"], s["v"]):
            x = pool.view(torch.uint8) if c["kv"] == "e4m3" else pool
            if c["order"] == "HND":
                x[to // P, :, to % P] = x[frm // P, :, frm % P]
            else:
                x[to // P, to % P] = x[frm // P, frm % P]
        s["new_lens"].copy_(ctx + s["n_kept"])
        out.update(mask=s["mask"], new_lens=s["new_lens"], k=s["k"], v=s["v"])
    # back: the pages behind what is kept, those of the first sequence last
    keep = s["keep"]
    had, left = (lens + P - 1) // P, (keep + P - 1) // P
    gone = had - left
    begins, count = torch.cumsum(gone, 0) - gone, gone.sum()
    j = torch.arange(table.shape[1], device=lens.device)
    freed = (j >= left[:, None]) & (j < had[:, None])
    k = (begins[:, None] + j - left[:, None])[freed]
    s["free"][(s["free_count"] + count - 1 - k).long()] = table[freed]
    s["free_count"] += count.to(torch.int32)
    lens.copy_(keep)
    out.update(seq_lens=lens, free=s["free"], free_count=s["free_count"])
    return out


def _rotate(x, positions, theta, layout, back=False):
    """x: float32 [tokens, heads, channels]; the first 2 * len(theta) channels are rotated."""
    n = theta.numel()
    angle = positions.double()[:, None] * theta
    cos, sin = (f.float()[:, None] for f in (angle.cos(), angle.sin()))
    if back:
        sin = -sin
    r, rest = x[..., :2 * n], x[..., 2 * n:]
    a, b = (r[..., :n], r[..., n:]) if layout == "half" else (r[..., 0::2], r[..., 1::2])
    ya, yb = a * cos - b * sin, a * sin + b * cos
    y = torch.cat((ya, yb), dim=-1) if layout == "half" else torch.stack((ya, yb), dim=-1).flatten(-2)
    return torch.cat((y, rest), dim=-1)


def _plain_norm(x, weight):
    x = x.float()
    return x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS), weight.float()


def _plain_norm_gradient(s):
    c, out = s["case"], []
    for x, g, w in zip(s["x"], s["grad"], s["weight"]):
        if x.shape[1] == 0:
            continue
        x, w = x.float(), w.float()
        r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
        n = x * r
        g = _rotate(g.float(), s["positions"], s["theta"], c["layout"], back=True)
        gw = (g.double() * n).sum(dim=(0, 1)).float()
        g = g * w
        out += [(r * (g - n * (g * n).mean(dim=-1, keepdim=True))).to(DTYPES[c["dtype"]]), gw]
    return out


def _plain_append(s):
    c = s["case"]
    q, k = (_rotate(n * w, s["positions"], s["theta"], c["layout"]) for n, w in
            (_plain_norm(x, w) for x, w in zip((s["q"], s["k_new"]), s["weight"])))
    q, v = q.to(torch.bfloat16), s["v_new"].float()
    if c["kv"] == "e4m3":
        k, v = ((x / f).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8) for x, f in ((k, s["k_scale"]), (v, s["v_scale"])))
        pools = s["k"].view(torch.uint8), s["v"].view(torch.uint8)
    else:
        k, v, pools = k.to(torch.bfloat16), v.to(torch.bfloat16), (s["k"], s["v"])
    page, slot = (s["slots"] // c["page"]).long(), (s["slots"] % c["page"]).long()
    if c["order"] == "HND":
        pools[0][page, :, slot], pools[1][page, :, slot] = k, v
    else:
        pools[0][page, slot], pools[1][page, slot] = k, v
    return {"q": q, "k": s["k"], "v": s["v"]}


def _plain_tree(s):
    c = s["case"]
    B, hq, hkv, D, P = c["batch"], c["hq"], c["hkv"], c["dim"], c["page"]
    dev, G, N, T = s["q"].device, c["hq"] // c["hkv"], s["most_new"], s["most"]
    new = s["q_offsets"][1:] - s["q_offsets"][:-1]
    ctx = s["seq_lens"] - new
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
    row = torch.where(live, s["q_offsets"][:-1, None] + i, 0).long()
    q = s["q"][row].float().view(B, N, hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, hkv, N * G, D)
    p = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(D)).view(B, hkv, N, G, T)
    j = t[:T] - ctx[:, None]                                                         # [B, T]: place among the drafted tokens
    at = j.clamp(0, 32 * _words(c) - 1)
    words = torch.gather(s["mask"][row], 2, (at >> 5)[:, None].expand(B, N, T))
    seen = torch.where(j[:, None] < 0, True, ((words >> (at & 31)[:, None]) & 1) == 1) & (j[:, None] <= i[:, None])
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
        if c["op"] == "tables":
            return _plain_tables(s)
        if c["op"] == "norm":
            if c["gradient"]:
                return _plain_norm_gradient(s)
            return [_rotate(n * w, s["positions"], s["theta"], c["layout"]).to(x.dtype)
                    for x, (n, w) in ((x, _plain_norm(x, w)) for x, w in zip(s["x"], s["weight"]) if x.shape[1])]
        return _plain_append(s) if c["op"] == "append" else _plain_tree(s)
    b, stream = s["b"], _stream()
    if c["op"] == "norm":
        t, dim = c["tokens"], c["dim"]
        if c["gradient"]:
            q, k = (b.NormGrads.of(x, g, w, o, gw) if x.shape[1] else None
                    for x, g, w, o, gw in zip(s["x"], s["grad"], s["weight"], s["out"], s["grad_weight"]))
            b.libra_norm_rope_gradient(0, s["rope"], q, k, s["dtype"], s["positions"].data_ptr(), t, dim, EPS,
                                       s["workspace"].data_ptr(), s["workspace"].numel(), stream)
            return [y for x, o, gw in zip(s["x"], s["out"], s["grad_weight"]) if x.shape[1] for y in (o, gw)]
        q, k = (b.NormRows.of(x, w, o) if x.shape[1] else None for x, w, o in zip(s["x"], s["weight"], s["out"]))
        b.libra_norm_rope_apply(0, s["rope"], q, k, s["dtype"], s["positions"].data_ptr(), t, dim, EPS, stream)
        return [o for x, o in zip(s["x"], s["out"]) if x.shape[1]]
    h, B, error = s["handle"], c["batch"], s["error"].data_ptr()
    table, lens, off = s["block_table"].data_ptr(), s["seq_lens"].data_ptr(), s["q_offsets"].data_ptr()
    if c["op"] == "tables":
        trees = c["drafts"] != "none"
        h.cache_extend(s["new"].data_ptr(), lens, table, B, s["free"].data_ptr(), s["free_count"].data_ptr(), off,
                       0 if trees else s["positions"].data_ptr(), s["slots"].data_ptr(), s["rows"], error, stream)
        out = {"q_offsets": s["q_offsets"], "positions": s["positions"], "slots": s["slots"], "block_table": s["block_table"]}
        if trees:
            h.tree_mask(s["parents"].data_ptr(), off, lens, B, s["rows"], s["mask"].data_ptr(), s["mask"].shape[1],
                        s["positions"].data_ptr(), error, stream)
            h.tree_keep(s["kept"].data_ptr(), s["kept"].shape[1], s["n_kept"].data_ptr(), off, lens, table, B, s["k"].data_ptr(),
                        s["v"].data_ptr(), s["new_lens"].data_ptr(), error, stream)
            out.update(mask=s["mask"], new_lens=s["new_lens"], k=s["k"], v=s["v"])
        h.cache_trim(s["keep"].data_ptr(), lens, table, B, s["free"].data_ptr(), s["free_count"].data_ptr(), error, stream)
        out.update(seq_lens=s["seq_lens"], free=s["free"], free_count=s["free_count"])
        return out
    if c["op"] == "append":
        h.norm_rope_append(s["rope"], s["weight"][0].data_ptr(), s["weight"][1].data_ptr(), EPS, s["q"].data_ptr(), s["q"].stride(0),
                           s["out"].data_ptr(), s["out"].stride(0), s["k_new"].data_ptr(), s["v_new"].data_ptr(),
                           s["k_new"].stride(0), s["positions"].data_ptr(), s["slots"].data_ptr(), off + 4 * B, s["rows"],
                           s["k"].data_ptr(), s["v"].data_ptr(), error, stream)
        return {"q": s["out"], "k": s["k"], "v": s["v"]}
    h.tree_attn(s["q"].data_ptr(), s["q"].stride(0), s["k"].data_ptr(), s["v"].data_ptr(), table, s["mask"].data_ptr(),
                s["mask"].shape[1], s["out"].data_ptr(), s["lse"].data_ptr(), error, stream)
    return {"out": s["out"], "lse": s["lse"]}


# ------------------------------------------------------------------------------------------------------ in 64 bits
def _exact_rotate(x, positions, theta, layout):
    """The rotation as a product of complex numbers; differentiable."""
    n = theta.numel()
    turn = torch.polar(torch.ones_like(theta).expand(len(positions), n), positions.double()[:, None] * theta)[:, None]
    r = x[..., :2 * n]
    z = torch.complex(r[..., :n], r[..., n:]) if layout == "half" else torch.view_as_complex(r.unflatten(-1, (n, 2)).contiguous())
    z = z * turn
    y = torch.cat((z.real, z.imag), -1) if layout == "half" else torch.view_as_real(z).flatten(-2)
    return torch.cat((y, x[..., 2 * n:]), dim=-1)


def _exact_norm(x, weight, positions, theta, layout):
    return _exact_rotate(x / torch.sqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * weight, positions, theta, layout)


def _exact_tables(s):
    """Page by page, as a list of free pages is used."""
    c, P = s["case"], s["case"]["page"]
    new, ctx = _lens(c)
    table = s["block_table"].cpu().numpy().copy()
    free = s["free"].cpu().numpy().copy()
    count, offsets, position, slot = int(s["free_count"]), [0], [], []
    for b, (n, L) in enumerate(zip(new, ctx)):
        for page in range(-(-L // P), -(-(L + n) // P)):
            count -= 1
            table[b, page] = free[count]
        t = np.arange(L, L + n)
        position.append(t)
        slot.append(table[b, t // P] * P + t % P)
        offsets.append(offsets[-1] + n)
    out = {"q_offsets": offsets, "positions": np.concatenate(position), "slots": np.concatenate(slot), "block_table": table}
    if c["drafts"] != "none":
        parents, at, k, v = _parents(c, new), 0, s["k"].double(), s["v"].double()
        bits, kept = np.zeros((s["rows"], _words(c) * 32), dtype=np.int64), _accepted(c, new, parents)
        for b, (n, L) in enumerate(zip(new, ctx)):
            for i in range(n):
                p = parents[at + i]
                if p >= 0:
                    bits[at + i] = bits[at + p]
                out["positions"][at + i] = L + bits[at + i].sum()
                bits[at + i, i] = 1
            for i, j in enumerate(kept[b]):
                (f, fs), (t, ts) = ((int(table[b, (L + x) // P]), (L + x) % P) for x in (j, i))
                for x in (k, v):
                    if c["order"] == "HND":
                        x[t, :, ts] = x[f, :, fs]
                    else:
                        x[t, ts] = x[f, fs]
            at += n
        words = (bits.reshape(s["rows"], -1, 32) << np.arange(32)).sum(-1)
        out.update(mask=words.astype(np.uint32).view(np.int32).reshape(s["rows"], -1),
                   new_lens=[L + len(p) for L, p in zip(ctx, kept)], k=k, v=v)
    for b in range(c["batch"] - 1, -1, -1):
        for page in range(-(-(ctx[b] + new[b]) // P) - 1, -(-ctx[b] // P) - 1, -1):
            free[count] = table[b, page]
            count += 1
    out.update(seq_lens=ctx, free=free, free_count=[count])
    return {n: x if torch.is_tensor(x) else torch.from_numpy(np.asarray(x).astype(np.int32)) for n, x in out.items()}


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "tables":
        return _exact_tables(s)
    if c["op"] == "norm":
        out = []
        for i, x in enumerate(s["x"]):
            if x.shape[1] == 0:
                continue
            x, w = x.double().requires_grad_(), s["weight"][i].double().requires_grad_()
            y = _exact_norm(x, w, s["positions"], s["theta"], c["layout"])
            out += list(torch.autograd.grad(y, (x, w), s["grad"][i].double())) if c["gradient"] else [y.detach()]
        return out
    new, ctx = _lens(c)
    first = [0] + list(np.cumsum(new))
    P, G = c["page"], c["hq"] // c["hkv"]
    if c["op"] == "append":
        q, k_new = (_exact_norm(x.double(), w.double(), s["positions"], s["theta"], c["layout"])
                    for x, w in zip((s["q"], s["k_new"]), s["weight"]))
        pools, slots = [], s["slots"].long()
        for pool, x in ((s["k"], k_new / s["k_scale"]), (s["v"], s["v_new"].double() / s["v_scale"])):
            y = pool.double()
            (y.transpose(1, 2) if c["order"] == "HND" else y)[slots // P, slots % P] = x
            pools.append(y.clamp(-448.0, 448.0) if c["kv"] == "e4m3" else y)
        return {"q": q, "k": pools[0], "v": pools[1]}
    out = torch.zeros((s["rows"], c["hq"], c["dim"]), dtype=torch.float64, device=s["q"].device)
    lse = torch.full((s["rows"], c["hq"]), float("-inf"), dtype=torch.float64, device=s["q"].device)
    parents = _parents(c, new)
    for b, (n, L) in enumerate(zip(new, ctx)):
        hidden = np.ones((n, n), dtype=bool)
        for i in range(n):
            j = i
            while j >= 0:
                hidden[i, j] = False
                j = parents[first[b] + j]
        hidden = torch.from_numpy(hidden).to(out.device)
        ids = s["block_table"][b, :-(-(L + n) // P)].long()
        for g in range(c["hkv"]):
            k, v = ((x[ids, g] if c["order"] == "HND" else x[ids, :, g]).double().flatten(0, 1)[:L + n] * f
                    for x, f in ((s["k"], s["k_scale"]), (s["v"], s["v_scale"])))
            for h in range(g * G, (g + 1) * G):
                a = s["q"][first[b]:first[b + 1], h].double() @ k.T / math.sqrt(c["dim"])
                a[:, L:][hidden] = float("-inf")
                z = torch.logsumexp(a, dim=-1)
                lse[first[b]:first[b + 1], h] = z
                out[first[b]:first[b + 1], h] = torch.exp(a - z[:, None]) @ v
    return {"out": out, "lse": lse}
