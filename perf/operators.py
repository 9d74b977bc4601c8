"""Cases for the operators of a decode step that stays on the device: block tables and slots from request lengths,
rotary positions with the append to the paged cache, and attention of one new token per request over that cache.

`run` computes an operator in its plain form (elementary torch operations) or, with `own` set, through the library's
entry points.  Sizes: head counts, head sizes, block sizes and context ranges of the workloads in
paper_2512_12928_b200/workloads.py, and generic ones around them.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # a decode batch: every request gets one token, a sixteenth of them a new block
        {"name": "slots_decode", "op": "slots", "rows": 64, "lo": 1024, "hi": 4096, "prefill": 0, "chunk": 0, "ends": 0,
         "block": 16, "slack": 64},
        # a mixed batch: decode rows, prompt chunks of up to 2048 tokens, requests that end, padding behind the tokens
        {"name": "slots_mixed", "op": "slots", "rows": 256, "lo": 0, "hi": 8192, "prefill": 24, "chunk": 2048, "ends": 17,
         "block": 16, "slack": 701},
        # many prompts at once, odd block size
        {"name": "slots_prompts", "op": "slots", "rows": 1000, "lo": 0, "hi": 600, "prefill": 1000, "chunk": 509, "ends": 0,
         "block": 24, "slack": 0},
        # one token of one request: latency
        {"name": "rope_one", "op": "rope", "tokens": 1, "pad": 0, "hq": 32, "hkv": 8, "dim": 128, "rot": 128, "axes": 1,
         "neighbours": False, "inverse": False, "append": True, "block": 16, "far": 4096, "dtype": "bf16"},
        # a decode batch behind images or video: three axes, padded to the captured batch
        {"name": "rope_batch_axes", "op": "rope", "tokens": 200, "pad": 56, "hq": 28, "hkv": 4, "dim": 128, "rot": 128, "axes": 3,
         "neighbours": False, "inverse": False, "append": True, "block": 16, "far": 100000, "dtype": "fp16"},
        # a prompt chunk of the 64-query-head shape
        {"name": "rope_prompt", "op": "rope", "tokens": 8192, "pad": 0, "hq": 64, "hkv": 8, "dim": 128, "rot": 128, "axes": 1,
         "neighbours": False, "inverse": False, "append": True, "block": 16, "far": 131072, "dtype": "bf16"},
        # patches of a video: time, height, width, a part of each head rotated, neighbours paired; the gradient's direction
        {"name": "rope_video_grad", "op": "rope", "tokens": 5003, "pad": 0, "hq": 16, "hkv": 16, "dim": 80, "rot": 48, "axes": 3,
         "neighbours": True, "inverse": True, "append": False, "block": 16, "far": 2000, "dtype": "fp16"},
        # one short request: latency
        {"name": "attn_one", "op": "attn", "rows": 1, "lo": 300, "hi": 300, "long": 0, "hq": 32, "hkv": 8, "dim": 128, "block": 16,
         "window": 0, "dtype": "bf16"},
        # the 8B-shaped decode batch
        {"name": "attn_batch", "op": "attn", "rows": 64, "lo": 1024, "hi": 4096, "long": 0, "hq": 32, "hkv": 8, "dim": 128,
         "block": 16, "window": 0, "dtype": "bf16"},
        # ragged rows from empty to 4500 tokens, four KV heads, sliding window, odd block size
        {"name": "attn_window_ragged", "op": "attn", "rows": 33, "lo": 0, "hi": 4500, "long": 0, "hq": 28, "hkv": 4, "dim": 128,
         "block": 24, "window": 1000, "dtype": "fp16"},
        # one very long request, all query heads on one KV head of 64
        {"name": "attn_long_shared", "op": "attn", "rows": 1, "lo": 131071, "hi": 131071, "long": 0, "hq": 16, "hkv": 1, "dim": 64,
         "block": 16, "window": 0, "dtype": "bf16"},
        # a decode batch with one long request in it, 64 query heads, blocks of 32
        {"name": "attn_batch_and_long", "op": "attn", "rows": 65, "lo": 4096, "hi": 4096, "long": 32768, "hq": 64, "hkv": 8,
         "dim": 128, "block": 32, "window": 0, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["slots", "rope", "attn"])
    if op == "slots":
        rows = _log(rng, 1, 1500)
        block = rng.choice([1, 8, 16, 16, 24, 32, 64, 100])
        hi = _log(rng, 1, min(8192, 2000000 * block // rows))
        prefill = rng.choice([0, rows, rng.randint(0, rows)])
        chunk = _log(rng, 1, max(1, min(2048, 260000 // max(1, prefill)))) if prefill else 0
        return {"op": op, "rows": rows, "lo": rng.choice([0, hi // 2]), "hi": hi, "prefill": prefill, "chunk": chunk,
                "ends": rng.choice([0, rng.randint(0, rows - prefill)]), "block": block,
                "slack": rng.choice([0, 1, rng.randint(0, 2000)])}
    if op == "rope":
        hkv = rng.choice([1, 2, 4, 8, 8, 16])
        dim = rng.choice([64, 80, 96, 128, 128, 256])
        hq = hkv * rng.choice([1, 2, 4, 5, 7, 8])
        tokens = _log(rng, 1, min(8192, 8192 * 80 * 128 // ((hq + 2 * hkv) * dim)))
        return {"op": op, "tokens": tokens, "pad": rng.choice([0, 0, rng.randint(0, 64)]), "hq": hq, "hkv": hkv, "dim": dim,
                "rot": rng.choice([dim, dim, dim // 2, dim // 4 // 2 * 2]), "axes": rng.choice([1, 1, 2, 3, 4]),
                "neighbours": rng.random() < 0.3, "inverse": rng.random() < 0.2, "append": rng.random() < 0.8,
                "block": rng.choice([1, 8, 16, 16, 24, 32, 64]), "far": _log(rng, 64, 1 << 20),
                "dtype": rng.choice(["bf16", "bf16", "fp16"])}
    hkv, dim = rng.choice([1, 2, 3, 4, 5, 8, 8, 8]), rng.choice([64, 128, 128])
    hq = hkv * rng.choice([1, 2, 3, 4, 4, 7, 8, 8, 16, 20])
    rows = _log(rng, 1, 200)
    # the plain form holds the padded batch in 32 bits: rows * longest * width is kept below the largest listed case's
    most = int(min(131072, 6e8 / (rows * (hkv * dim + hq))))
    hi = _log(rng, 1, max(1, most // 2))
    long = rng.choice([0, 0, rng.randint(1, max(1, most))])
    return {"op": op, "rows": rows, "lo": rng.choice([0, hi // 4, hi]), "hi": hi, "long": long, "hq": hq, "hkv": hkv, "dim": dim,
            "block": rng.choice([1, 8, 16, 16, 16, 24, 32, 64, 100]), "window": rng.choice([0, 0, 0, _log(rng, 1, 4096)]),
            "dtype": rng.choice(["bf16", "bf16", "fp16"])}


# --------------------------------------------------------------------------------------------- inputs

def _lengths(case, g):
    """Context lengths of the rows, the same on every call with the same generator state; a range from zero gets its ends."""
    n = torch.randint(case["lo"], case["hi"] + 1, (case["rows"],), generator=g, dtype=torch.int64)
    if case["rows"] > 2 and case["lo"] < case["hi"]:
        n[0], n[1] = case["lo"], case["hi"]
    return n


def _tables(n_blocks, stride, pool_blocks, g):
    """Block tables of rows with n_blocks blocks each out of a shuffled pool; entries behind a row's blocks are zero.
    Also the ids that no row holds, in shuffled order."""
    order = torch.randperm(pool_blocks, generator=g)
    at = torch.cumsum(n_blocks, 0) - n_blocks
    col = torch.arange(stride)[None, :]
    mine = col < n_blocks[:, None]
    ids = torch.where(mine, order[torch.where(mine, at[:, None] + col, 0)], 0)
    return ids.to(torch.int32), order[int(n_blocks.sum()):].to(torch.int32)


def _token_room(case):
    """Tokens that the slot map has room for: the most that the rows can bring, as a captured step is sized, and some more."""
    return case["prefill"] * case["chunk"] + case["rows"] - case["prefill"] + case["slack"]


def prepare(case, seed):
    g = torch.Generator().manual_seed(seed)
    dev = torch.device("cuda")
    gd = torch.Generator(device=dev).manual_seed(seed + 1)
    s = {"case": case}
    S = case["block"]
    if case["op"] == "slots":
        rows = case["rows"]
        ctx = _lengths(case, g)
        new = torch.ones(rows, dtype=torch.int64)
        who = torch.randperm(rows, generator=g)
        pre, ends = who[: case["prefill"]], who[case["prefill"]: case["prefill"] + case["ends"]]
        if case["prefill"]:
            new[pre] = torch.randint(0, case["chunk"] + 1, (case["prefill"],), generator=g)
        new[ends] = -1
        old = (ctx + S - 1) // S
        after = torch.where(new < 0, 0, (ctx + new.clamp(min=0) + S - 1) // S)
        stride = (case["hi"] + max(1, case["chunk"]) + S - 1) // S
        pool = case["rows"] * stride
        tables, free = _tables(old, stride, pool, g)
        ids = torch.zeros(pool, dtype=torch.int32)
        ids[: len(free)] = free
        cap = _token_room(case)
        s.update(ctx=ctx.to(torch.int32).to(dev), new=new.to(torch.int32).to(dev), tables=tables.to(dev), free_ids=ids.to(dev),
                 free_count=torch.tensor([len(free)], dtype=torch.int32, device=dev),
                 slots=torch.zeros(cap, dtype=torch.int64, device=dev), positions=torch.zeros(cap, dtype=torch.int32, device=dev),
                 start=torch.zeros(rows + 1, dtype=torch.int32, device=dev), ctx_out=torch.zeros(rows, dtype=torch.int32, device=dev),
                 free_out=torch.zeros(1, dtype=torch.int32, device=dev), pool=pool)
        return s
    dt = DTYPES[case["dtype"]]
    hq, hkv, D = case["hq"], case["hkv"], case["dim"]
    if case["op"] == "rope":
        T = case["tokens"] + case["pad"]
        # queries, keys and values lie in one buffer, as a fused projection leaves them
        qkv = torch.randn((T, (hq + 2 * hkv) * D), device=dev, dtype=dt, generator=gd)
        q = qkv[:, : hq * D].view(T, hq, D)
        k = qkv[:, hq * D: (hq + hkv) * D].view(T, hkv, D)
        v = qkv[:, (hq + hkv) * D:].view(T, hkv, D)
        pos = torch.randint(0, case["far"], (case["axes"], T), device=dev, dtype=torch.int32, generator=gd)
        half = case["rot"] // 2
        inv = (10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)).to(torch.float32).to(dev)
        axis = sorted(i % case["axes"] for i in range(half))     # each axis has a run of the frequencies
        s.update(q=q, k=k, v=v, pos=pos, inv=inv, axis=axis, axis_d=torch.tensor(axis, device=dev), q_out=torch.zeros((T, hq, D), device=dev, dtype=dt))
        if case["append"]:
            nb = (T + S - 1) // S + 8
            slots = torch.randperm(nb * S, generator=g)[:T]
            slots[case["tokens"]:] = -1
            s.update(slots=slots.to(dev), kpool=torch.randn((nb, S, hkv, D), device=dev, dtype=dt, generator=gd),
                     vpool=torch.randn((nb, S, hkv, D), device=dev, dtype=dt, generator=gd))
        else:
            s.update(k_out=torch.zeros((T, hkv, D), device=dev, dtype=dt))
        return s
    ctx = _lengths(case, g)
    if case["long"]:
        ctx[-1] = case["long"]
    n = (ctx + S - 1) // S
    pool = int(n.sum()) + 16
    tables, _ = _tables(n, max(1, int(n.max())), pool, g)
    s.update(ctx=ctx.to(torch.int32).to(dev), tables=tables.to(dev),
             kpool=torch.randn((pool, S, hkv, D), device=dev, dtype=dt, generator=gd),
             vpool=torch.randn((pool, S, hkv, D), device=dev, dtype=dt, generator=gd),
             q=torch.randn((case["rows"], hq, D), device=dev, dtype=dt, generator=gd),
             out=torch.zeros((case["rows"], hq, D), device=dev, dtype=dt),
             lse=torch.zeros((case["rows"], hq), device=dev, dtype=torch.float32), longest=max(1, int(ctx.max())))
    return s


# ------------------------------------------------------------------------------------------ plain forms

def _plain_slots(s):
    S = s["case"]["block"]
    ctx, new, tables, ids = s["ctx"].long(), s["new"].long(), s["tables"].long(), s["free_ids"].long()
    dev = ctx.device
    ends, add = new < 0, new.clamp(min=0)
    old = (ctx + S - 1) // S
    ctx_out = torch.where(ends, 0, ctx + add)
    after = (ctx_out + S - 1) // S
    need = torch.where(ends, 0, after - old)
    back = torch.where(ends, old, 0)
    back_end, need_end, tok_end = torch.cumsum(back, 0), torch.cumsum(need, 0), torch.cumsum(add, 0)
    count, R, N = s["free_count"].long(), back_end[-1], need_end[-1]
    free_out = count + R - N

    def stack(i):
        """Entry i of the stack after the ended rows' blocks went onto it."""
        r = (i - count).clamp(min=0)
        row = torch.searchsorted(back_end, r, right=True).clamp(max=len(ctx) - 1)
        returned = tables[row, (r - (back_end - back)[row]).clamp(0, tables.shape[1] - 1)]
        return torch.where(i < count, ids[i.clamp(0, len(ids) - 1)], returned)

    col = torch.arange(tables.shape[1], device=dev)[None, :]
    fresh = (col >= old[:, None]) & (col < after[:, None])
    rank = (need_end - need)[:, None] + col - old[:, None]
    tables_out = torch.where(fresh, stack((count + R - 1 - rank).clamp(min=0)), tables)
    i = torch.arange(len(ids), device=dev)
    ids_out = torch.where((i >= count) & (i < count + R), stack(i), ids)   # what was popped again stays above the new top
    t = torch.arange(len(s["slots"]), device=dev)
    row = torch.searchsorted(tok_end, t, right=True).clamp(max=len(ctx) - 1)
    p = ctx[row] + t - (tok_end - add)[row]
    live = t < tok_end[-1]
    slots = torch.where(live, tables_out[row, torch.where(live, p // S, 0)] * S + p % S, -1)
    start = torch.cat([torch.zeros(1, dtype=torch.int64, device=dev), tok_end])
    return (tables_out.int(), slots, torch.where(live, p, 0).int(), start.int(), ctx_out.int(), free_out.int(), ids_out.int())


def _turn(x, cos, sin, rot, neighbours):
    """The rotation of the first rot dims of x [T, heads, D] in 32 bits."""
    x = x.float()
    r = x[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if neighbours else (r[..., : rot // 2], r[..., rot // 2:])
    c, s = cos[:, None, :], sin[:, None, :]
    a, b = a * c - b * s, b * c + a * s
    r = torch.stack([a, b], -1).flatten(-2) if neighbours else torch.cat([a, b], -1)
    return torch.cat([r, x[..., rot:]], -1)


def _plain_rope(s):
    case, dt = s["case"], s["q"].dtype
    # angles of far positions need 64 bits
    angle = s["pos"].double()[s["axis_d"]].T * s["inv"].double()
    sign = -1.0 if case["inverse"] else 1.0
    cos, sin = torch.cos(angle).float(), (sign * torch.sin(angle)).float()
    q = _turn(s["q"], cos, sin, case["rot"], case["neighbours"]).to(dt)
    k = _turn(s["k"], cos, sin, case["rot"], case["neighbours"]).to(dt)
    if not case["append"]:
        return q, k
    live = s["slots"] >= 0
    at = s["slots"][live]
    s["kpool"].view(-1, *k.shape[1:])[at] = k[live]
    s["vpool"].view(-1, *k.shape[1:])[at] = s["v"][live]
    return torch.where(live[:, None, None], q, 0), s["kpool"], s["vpool"]


def _plain_attn(s):
    case = s["case"]
    rows, hq, D = s["q"].shape
    S, hkv = case["block"], case["hkv"]
    ctx = s["ctx"].long()
    t = torch.arange(s["longest"], device=ctx.device)
    seen = t[None, :] < ctx[:, None]
    if case["window"]:
        seen &= t[None, :] >= ctx[:, None] - case["window"]
    token = s["tables"].long()[:, t // S] * S + (t % S)[None, :]
    k = s["kpool"].view(-1, hkv, D)[token].float()
    q = s["q"].float().view(rows, hkv, hq // hkv, D)
    x = torch.matmul(q, k.permute(0, 2, 3, 1)) / math.sqrt(D)
    del k
    x = torch.where(seen[:, None, None, :], x, -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    v = s["vpool"].view(-1, hkv, D)[token].float()
    out = torch.matmul(p, v.permute(0, 2, 1, 3)) / torch.where(total > 0, total, 1.0)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)
    return out.reshape(rows, hq, D).to(s["q"].dtype), lse.reshape(rows, hq)


# ------------------------------------------------------------------------------------------------ run

def _did(answer):
    if answer[0]:
        raise RuntimeError(answer[1])


def run(state):
    s, case = state, state["case"]
    if case["op"] == "slots":
        if own:
            from paper_2512_12928_b200 import binding as B
            _did(B.ps_build_slots(s["ctx"], s["new"], s["tables"], s["slots"], s["positions"], s["start"], s["ctx_out"],
                                  block_size=case["block"], num_gpu_blocks=s["pool"], free_ids=s["free_ids"],
                                  free_count=s["free_count"], free_count_out=s["free_out"]))
            return s["tables"], s["slots"], s["positions"], s["start"], s["ctx_out"], s["free_out"], s["free_ids"]
        return _plain_slots(s)
    if case["op"] == "rope":
        if own:
            from paper_2512_12928_b200 import binding as B
            _did(B.ps_rope_append(s["q"], s["k"], s["q_out"], s.get("k_out"), s["pos"], s["inv"], v=s["v"] if case["append"] else None,
                                  kpool=s.get("kpool"), vpool=s.get("vpool"), slots=s.get("slots"), freq_axis=s["axis"],
                                  neighbours=case["neighbours"], inverse=case["inverse"]))
            return (s["q_out"], s["kpool"], s["vpool"]) if case["append"] else (s["q_out"], s["k_out"])
        return _plain_rope(s)
    if own:
        from paper_2512_12928_b200 import binding as B
        _did(B.ps_paged_attn(s["kpool"], s["vpool"], s["q"], s["out"], s["tables"], s["ctx"], lse=s["lse"], window=case["window"]))
        return s["out"], s["lse"]
    return _plain_attn(s)


# ----------------------------------------------------------------------------------------------- work

def work(case):
    if case["op"] == "slots":
        mean = (case["lo"] + case["hi"]) / 2
        tokens = case["prefill"] * case["chunk"] / 2 + case["rows"] - case["prefill"] - case["ends"]
        fresh = tokens / case["block"] + case["ends"] * mean / case["block"]
        return {"bytes": 16.0 * case["rows"] + 12.0 * _token_room(case) + 8.0 * fresh + 8, "flops": 0}
    if case["op"] == "rope":
        row = (case["hq"] + 2 * case["hkv"]) if case["append"] else case["hq"] + case["hkv"]
        per = 2 * row * case["dim"] * 2 + 4 * case["axes"] + (8 if case["append"] else 0)
        return {"bytes": float(case["tokens"] * per), "flops": float(case["tokens"] * (case["hq"] + case["hkv"]) * case["rot"] * 3)}
    mean = (case["lo"] + case["hi"]) / 2
    seen = case["rows"] * mean
    if case["window"]:   # of a length that is uniform in the range
        w, lo, hi = case["window"], case["lo"], case["hi"]
        mean = min(w, lo) if hi == lo else (hi - w) / (hi - lo) * w + (w - lo) / (hi - lo) * (w + lo) / 2 if lo < w < hi else min(w, mean)
        seen = case["rows"] * mean
    if case["long"]:
        seen += (min(case["window"], case["long"]) if case["window"] else case["long"]) - mean
    kv = seen * case["hkv"] * case["dim"]
    return {"bytes": 4 * kv + case["rows"] * case["hq"] * (case["dim"] * 4 + 4), "flops": 4 * kv * case["hq"] / case["hkv"]}


# ---------------------------------------------------------------------------------------------- exact

def _exact_rope(s):
    case = s["case"]
    T, half = s["q"].shape[0], case["rot"] // 2
    turn = torch.zeros((T, half), dtype=torch.float64, device=s["q"].device)
    for i in range(half):
        turn[:, i] = s["pos"][s["axis"][i]].double() * s["inv"][i].double()
    if case["inverse"]:
        turn = -turn
    z = torch.polar(torch.ones_like(turn), turn)

    def rotate(x):
        y = x.double().clone()
        if case["neighbours"]:
            w = torch.view_as_complex(y[..., : 2 * half].reshape(*y.shape[:2], half, 2).contiguous()) * z[:, None]
            y[..., : 2 * half] = torch.view_as_real(w).reshape(*y.shape[:2], 2 * half)
        else:
            w = torch.complex(y[..., :half].contiguous(), y[..., half: 2 * half].contiguous()) * z[:, None]
            y[..., :half], y[..., half: 2 * half] = w.real, w.imag
        return y

    q, k = rotate(s["q"]), rotate(s["k"])
    if not case["append"]:
        return q, k
    n = case["tokens"]
    q[n:] = 0
    kp, vp = (s[x].double().flatten(0, 1) for x in ("kpool", "vpool"))
    kp.index_copy_(0, s["slots"][:n], k[:n])
    vp.index_copy_(0, s["slots"][:n], s["v"][:n].double())
    return q, kp.view(s["kpool"].shape), vp.view(s["vpool"].shape)


def _exact_attn(s):
    case = s["case"]
    rows, hq, D = s["q"].shape
    hkv, S = case["hkv"], case["block"]
    out = torch.zeros((rows, hq, D), dtype=torch.float64, device=s["q"].device)
    lse = torch.full((rows, hq), -math.inf, dtype=torch.float64, device=s["q"].device)
    for b, n in enumerate(s["ctx"].tolist()):
        if n == 0:
            continue
        ids = s["tables"][b, : (n + S - 1) // S].long()
        first = max(0, n - case["window"]) if case["window"] else 0
        for h in range(hkv):
            heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            k = s["kpool"][ids, :, h].flatten(0, 1)[first:n].double()
            v = s["vpool"][ids, :, h].flatten(0, 1)[first:n].double()
            x = s["q"][b, heads].double() @ k.T * D ** -0.5
            lse[b, heads] = torch.logsumexp(x, -1)
            out[b, heads] = torch.softmax(x, -1) @ v
    return out, lse


def exact(case, seed):
    if case["op"] == "slots":
        return None     # whole numbers: they have to be equal
    s = prepare(case, seed)
    return _exact_rope(s) if case["op"] == "rope" else _exact_attn(s)
