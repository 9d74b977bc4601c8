"""Cases for the operators of a paged KV cache that is held in 8 bits, with a 32-bit scale for each block of tokens and
KV head: keys and values quantised as they are written, tokens read back, and attention of one new token per request.

`run` computes an operator in its plain form (elementary torch operations) or, with `own` set, through the library's
entry points.  Sizes: head counts, head sizes, block sizes and context ranges of the workloads in
paper_2512_12928_b200/workloads.py, and generic ones around them.

A value of the cache is code * scale: code is an int8 from -127 to 127 or an e4m3 number, scale that of its block and
head.  Writing raises a block's scale to what its new tokens need (their largest magnitude / 127 or / 448) and brings
the codes that are there to the new scale; a call that writes a block's first place begins the block anew.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
CODES = {"int8": (torch.int8, 127.0), "e4m3": (torch.float8_e4m3fn, 448.0)}
LEAST_SCALE = 2.0 ** -100


# ---------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # a token is appended to one request's cache, and the cache read back: latency
        {"name": "append_one", "op": "append", "rows": 1, "lo": 1, "hi": 1, "pad": 0, "hkv": 8, "dim": 128, "block": 16, "codes": "int8",
         "dtype": "bf16"},
        # a decode batch padded to the captured size
        {"name": "append_batch", "op": "append", "rows": 200, "lo": 1, "hi": 1, "pad": 56, "hkv": 4, "dim": 128, "block": 16,
         "codes": "e4m3", "dtype": "fp16"},
        # prompt chunks of a few requests, 8192 tokens and more
        {"name": "append_prompts", "op": "append", "rows": 7, "lo": 500, "hi": 2048, "pad": 300, "hkv": 8, "dim": 128, "block": 16,
         "codes": "int8", "dtype": "bf16"},
        # many short chunks that begin and end inside blocks, odd block size and heads
        {"name": "append_ragged", "op": "append", "rows": 97, "lo": 0, "hi": 103, "pad": 0, "hkv": 16, "dim": 80, "block": 24,
         "codes": "e4m3", "dtype": "bf16"},
        # one short request's context in 16 bits: latency
        {"name": "read_one", "op": "read", "rows": 1, "lo": 300, "hi": 300, "pad": 0, "hkv": 8, "dim": 128, "block": 16, "codes": "int8",
         "dtype": "bf16"},
        # contexts that a prompt chunk attends, several requests
        {"name": "read_contexts", "op": "read", "rows": 13, "lo": 0, "hi": 8192, "pad": 1000, "hkv": 8, "dim": 128, "block": 16,
         "codes": "e4m3", "dtype": "bf16"},
        # odd heads and blocks
        {"name": "read_odd", "op": "read", "rows": 5, "lo": 501, "hi": 1501, "pad": 3, "hkv": 3, "dim": 80, "block": 24, "codes": "int8",
         "dtype": "fp16"},
        # one short request: latency
        {"name": "attn_one", "op": "attn", "rows": 1, "lo": 500, "hi": 500, "long": 0, "hq": 32, "hkv": 8, "dim": 128, "block": 16,
         "window": 0, "codes": "int8", "dtype": "bf16"},
        # the 8B-shaped decode batch
        {"name": "attn_batch", "op": "attn", "rows": 64, "lo": 1024, "hi": 4096, "long": 0, "hq": 32, "hkv": 8, "dim": 128,
         "block": 16, "window": 0, "codes": "int8", "dtype": "bf16"},
        # ragged rows from empty to 4500 tokens, four KV heads, sliding window, odd block size
        {"name": "attn_window_ragged", "op": "attn", "rows": 50, "lo": 0, "hi": 4500, "long": 0, "hq": 28, "hkv": 4, "dim": 128,
         "block": 24, "window": 1500, "codes": "e4m3", "dtype": "fp16"},
        # one very long request, all query heads on one KV head of 64
        {"name": "attn_long_shared", "op": "attn", "rows": 1, "lo": 131071, "hi": 131071, "long": 0, "hq": 16, "hkv": 1, "dim": 64,
         "block": 16, "window": 0, "codes": "int8", "dtype": "fp16"},
        # a decode batch with one long request in it, 64 query heads, blocks of 32
        {"name": "attn_batch_and_long", "op": "attn", "rows": 65, "lo": 4096, "hi": 4096, "long": 32768, "hq": 64, "hkv": 8,
         "dim": 128, "block": 32, "window": 0, "codes": "e4m3", "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["append", "read", "attn"])
    codes, dtype = rng.choice(["int8", "e4m3"]), rng.choice(["bf16", "bf16", "fp16"])
    if op == "append":
        hkv, dim = rng.choice([1, 2, 3, 4, 8, 8, 16]), rng.choice([64, 80, 96, 128, 128, 256])
        rows = _log(rng, 1, 300)
        hi = rng.choice([1, _log(rng, 1, max(1, min(2048, 8192 * 1024 // (rows * hkv * dim))))])
        block = rng.choice([b for b in (1, 8, 16, 16, 24, 32, 64, 100) if rows * (hi + 2 * b) * hkv * dim <= 16384 * 1024])
        return {"op": op, "rows": rows, "lo": rng.choice([0, hi // 2, hi]), "hi": hi, "pad": rng.choice([0, 0, rng.randint(0, 64)]),
                "hkv": hkv, "dim": dim, "block": block, "codes": codes, "dtype": dtype}
    if op == "read":
        hkv, dim = rng.choice([1, 2, 3, 4, 8, 8, 16]), rng.choice([64, 80, 96, 128, 128, 256])
        rows = _log(rng, 1, 60)
        hi = _log(rng, 1, max(1, min(32768, 65536 * 1024 // (rows * hkv * dim))))
        return {"op": op, "rows": rows, "lo": rng.choice([0, hi // 2, hi]), "hi": hi, "pad": rng.choice([0, rng.randint(0, 500)]),
                "hkv": hkv, "dim": dim, "block": rng.choice([1, 8, 16, 16, 24, 32, 64, 100]), "codes": codes, "dtype": dtype}
    hkv, dim = rng.choice([1, 2, 3, 4, 5, 8, 8, 8]), rng.choice([64, 128, 128])
    hq = hkv * rng.choice([1, 2, 3, 4, 4, 7, 8, 8, 16, 20])
    rows = _log(rng, 1, 200)
    # the plain form holds the padded batch in 32 bits: rows * longest * width is kept below the largest listed case's
    most = int(min(131072, 6e8 / (rows * (hkv * dim + hq))))
    hi = _log(rng, 1, max(1, most // 2))
    long = rng.choice([0, 0, rng.randint(1, max(1, most))])
    return {"op": op, "rows": rows, "lo": rng.choice([0, hi // 4, hi]), "hi": hi, "long": long, "hq": hq, "hkv": hkv, "dim": dim,
            "block": rng.choice([1, 8, 16, 16, 16, 24, 32, 64, 100]), "window": rng.choice([0, 0, 0, _log(rng, 1, 4096)]),
            "codes": codes, "dtype": dtype}


# --------------------------------------------------------------------------------------------- inputs

def _lengths(case, g):
    """Tokens of the rows, the same on every call with the same generator state; a range gets its ends."""
    n = torch.randint(case["lo"], case["hi"] + 1, (case["rows"],), generator=g, dtype=torch.int64)
    if case["rows"] > 2 and case["lo"] < case["hi"]:
        n[0], n[1] = case["lo"], case["hi"]
    return n


def _tables(n_blocks, stride, pool_blocks, g):
    """Block tables of rows with n_blocks blocks each out of a shuffled pool; entries behind a row's blocks are zero."""
    order = torch.randperm(pool_blocks, generator=g)
    at = torch.cumsum(n_blocks, 0) - n_blocks
    col = torch.arange(stride)[None, :]
    mine = col < n_blocks[:, None]
    return torch.where(mine, order[torch.where(mine, at[:, None] + col, 0)], 0).to(torch.int32)


def _slots(tables, first, count, S, pad):
    """Slots of count[b] tokens of every row from position first[b] on, and so many of padding behind them."""
    end = torch.cumsum(count, 0)
    t = torch.arange(int(end[-1]))
    row = torch.searchsorted(end, t, right=True)
    p = first[row] + t - (end - count)[row]
    return torch.cat([tables[row, p // S].long() * S + p % S, torch.full((pad,), -1, dtype=torch.int64)])


def _cache(case, blocks, g):
    """Codes of a cache that has been written, and its scales: most blocks' largest magnitude is one that normal
    numbers reach."""
    dt, top = CODES[case["codes"]]
    shape = (blocks, case["block"], case["hkv"], case["dim"])
    x = torch.randn(shape, device="cuda", generator=g, dtype=torch.float32) * (top / 3.5)
    x = x.clamp(-top, top)
    pool = torch.round(x).to(torch.int8) if dt == torch.int8 else x.to(dt)
    scale = torch.rand(shape[0::2], device="cuda", generator=g) * (2.5 / top) + 1.5 / top
    return pool, scale


def _append_blocks(case):
    """Blocks of the pool: what a row's new tokens can touch wherever they begin."""
    return case["rows"] * ((case["hi"] + 2 * case["block"] - 2) // case["block"]) + 4


def prepare(case, seed):
    g = torch.Generator().manual_seed(seed)
    dev = torch.device("cuda")
    gd = torch.Generator(device=dev).manual_seed(seed + 1)
    dt = DTYPES[case["dtype"]]
    S, hkv, D = case["block"], case["hkv"], case["dim"]
    s = {"case": case, "dtype": dt}
    # tokens that are read come back as rows: as many with every seed
    n = _lengths(case, torch.Generator().manual_seed(case["rows"] + case["hi"]) if case["op"] == "read" else g)
    if case["op"] == "append":
        # a row has had so many tokens in its first block; only the blocks that the call touches are in the pool
        first = torch.randint(0, S, (case["rows"],), generator=g)
        nb = torch.where(n > 0, (first + n + S - 1) // S, 0)
        pool = _append_blocks(case)
        slots = _slots(_tables(nb, max(1, int(nb.max())), pool, g), first, n, S, case["pad"])
        # keys and values lie in one buffer, as a fused projection leaves them; a few channels are large, as those of keys are
        T = len(slots)
        kv = torch.randn((T, 2 * hkv * D), device=dev, generator=gd)
        kv[:, :: 61] *= 5.0
        kv = kv.to(dt)
        s.update(k=kv[:, : hkv * D].view(T, hkv, D), v=kv[:, hkv * D:].view(T, hkv, D), slots=slots.to(dev))
    elif case["op"] == "read":
        nb = (n + S - 1) // S
        pool = int(nb.sum()) + 4
        s["slots"] = _slots(_tables(nb, max(1, int(nb.max())), pool, g), torch.zeros_like(n), n, S, case["pad"]).to(dev)
    else:
        if case["long"]:
            n[-1] = case["long"]
        nb = (n + S - 1) // S
        pool = int(nb.sum()) + 16
        s.update(ctx=n.to(torch.int32).to(dev), tables=_tables(nb, max(1, int(nb.max())), pool, g).to(dev), longest=max(1, int(n.max())),
                 q=torch.randn((case["rows"], case["hq"], D), device=dev, dtype=dt, generator=gd),
                 out=torch.zeros((case["rows"], case["hq"], D), device=dev, dtype=dt),
                 lse=torch.zeros((case["rows"], case["hq"]), device=dev, dtype=torch.float32))
    s["kpool"], s["kscale"] = _cache(case, pool, gd)
    s["vpool"], s["vscale"] = _cache(case, pool, gd)
    if case["op"] == "append":
        # what the cache then holds is read into 16 bits, every place of it
        s["every"] = torch.arange(pool * S, device=dev)
    if case["op"] != "attn":
        rows = pool * S if case["op"] == "append" else len(s["slots"])
        s["k_out"], s["v_out"] = (torch.zeros((rows, hkv, D), device=dev, dtype=dt) for _ in range(2))
    return s


# ------------------------------------------------------------------------------------------ plain forms

def _codes(x, factor, dt):
    """x times factor (32 bits), as codes: whole numbers from the exact product, e4m3 from the 32-bit one."""
    if dt == torch.int8:
        return torch.round(x.double() * factor.double()).to(torch.int8)
    return (x.float() * factor).to(dt)


def _write(x, pool, scale, slots):
    S, H, D = pool.shape[1:]
    top = CODES["int8" if pool.dtype == torch.int8 else "e4m3"][1]
    live = slots >= 0
    x, at = x[live].float(), slots[live]
    block, place = at // S, at % S
    most = torch.zeros_like(scale).index_reduce_(0, block, x.abs().amax(-1), "amax")
    met = torch.zeros(len(pool), device=x.device).index_fill_(0, block, 1.0) > 0
    begun = torch.zeros(len(pool), device=x.device).index_fill_(0, block[place == 0], 1.0) > 0
    old = torch.where(begun[:, None], 0.0, scale)
    new = torch.maximum(old, most * (1.0 / top)).clamp(min=LEAST_SCALE)
    inverse = torch.ones_like(new) / new
    moves = (met & ~begun)[:, None] & (new > old)
    # (as bytes: e4m3 has no torch.where)
    bits = pool.view(torch.uint8)
    moved = _codes(pool.float(), (old * inverse)[:, None, :, None], pool.dtype).view(torch.uint8)
    bits.copy_(torch.where(moves[:, None, :, None], moved, bits))
    bits.view(-1, H, D)[at] = _codes(x, inverse[block][..., None], pool.dtype).view(torch.uint8)
    scale.copy_(torch.where(met[:, None], new, scale))


def _read(pool, scale, slots, out):
    S, H, D = pool.shape[1:]
    live = slots >= 0
    at = slots[live]
    x = pool.view(torch.uint8).view(-1, H, D)[at].view(pool.dtype).float()
    out[live] = (x * scale[at // S][..., None]).to(out.dtype)


def _plain_attn(s):
    case = s["case"]
    rows, hq, D = s["q"].shape
    S, hkv = case["block"], case["hkv"]
    ctx = s["ctx"].long()
    t = torch.arange(s["longest"], device=ctx.device)
    seen = t[None, :] < ctx[:, None]
    if case["window"]:
        seen &= t[None, :] >= ctx[:, None] - case["window"]
    block = s["tables"].long()[:, t // S]
    token = block * S + (t % S)[None, :]

    def values(pool, scale):
        x = pool.view(torch.uint8).view(-1, hkv, D)[token].view(pool.dtype).float()
        return x.mul_(scale[block][..., None])

    k = values(s["kpool"], s["kscale"])
    q = s["q"].float().view(rows, hkv, hq // hkv, D)
    x = torch.matmul(q, k.permute(0, 2, 3, 1)) / math.sqrt(D)
    del k
    x = torch.where(seen[:, None, None, :], x, -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, values(s["vpool"], s["vscale"]).permute(0, 2, 1, 3)) / torch.where(total > 0, total, 1.0)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)
    return out.reshape(rows, hq, D).to(s["q"].dtype), lse.reshape(rows, hq)


# ------------------------------------------------------------------------------------------------ run

def _did(answer):
    if answer[0]:
        raise RuntimeError(answer[1])


def run(state):
    s, case = state, state["case"]
    cache = s["kpool"], s["vpool"], s["kscale"], s["vscale"]
    if own:
        from paper_2512_12928_b200 import binding as B
    if case["op"] == "attn":
        if own:
            _did(B.ps_quant_attn(*cache, s["q"], s["out"], s["tables"], s["ctx"], lse=s["lse"], window=case["window"]))
            return s["out"], s["lse"]
        return _plain_attn(s)
    if case["op"] == "append":
        if own:
            _did(B.ps_quant_append(s["k"], s["v"], *cache, s["slots"]))
        else:
            _write(s["k"], s["kpool"], s["kscale"], s["slots"])
            _write(s["v"], s["vpool"], s["vscale"], s["slots"])
    slots = s["every"] if case["op"] == "append" else s["slots"]
    if own:
        _did(B.ps_quant_read(*cache, slots, s["k_out"], s["v_out"]))
    else:
        _read(s["kpool"], s["kscale"], slots, s["k_out"])
        _read(s["vpool"], s["vscale"], slots, s["v_out"])
    return (s["k_out"], s["v_out"]) + ((s["kscale"], s["vscale"]) if case["op"] == "append" else ())


# ----------------------------------------------------------------------------------------------- work

def work(case):
    width = case["hkv"] * case["dim"]
    mean = (case["lo"] + case["hi"]) / 2
    if case["op"] == "append":
        blocks = _append_blocks(case)
        tokens = case["rows"] * mean
        written = tokens * (2 * width * 3 + 8)
        return {"bytes": written + blocks * (case["block"] * (2 * width * 3 + 8) + 8 * case["hkv"] * 2), "flops": tokens * width * 6}
    if case["op"] == "read":
        tokens = case["rows"] * mean
        return {"bytes": tokens * (2 * width * 3 + 8 + 8 * case["hkv"] / case["block"]) + 8 * case["pad"], "flops": tokens * 2 * width}
    seen = case["rows"] * mean
    if case["window"]:   # of a length that is uniform in the range
        w, lo, hi = case["window"], case["lo"], case["hi"]
        mean = min(w, lo) if hi == lo else (hi - w) / (hi - lo) * w + (w - lo) / (hi - lo) * (w + lo) / 2 if lo < w < hi else min(w, mean)
        seen = case["rows"] * mean
    if case["long"]:
        seen += (min(case["window"], case["long"]) if case["window"] else case["long"]) - mean
    kv = seen * width
    return {"bytes": 2 * kv + 8 * seen * case["hkv"] / case["block"] + case["rows"] * case["hq"] * (case["dim"] * 4 + 4),
            "flops": 4 * kv * case["hq"] / case["hkv"]}


# ---------------------------------------------------------------------------------------------- exact

def _nearest(y, codes):
    """The code nearest to y, in 64 bits."""
    if codes == "int8":
        return torch.round(y).clamp(-127, 127)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(y / step) * step).clamp(-448, 448)


def _exact_write(x, pool, scale, slots, codes):
    """(codes, scales) of the whole cache after the write, block by block."""
    top = CODES[codes][1]
    pool, scale = pool.double(), scale.double()
    S = pool.shape[1]
    at = slots[slots >= 0]
    order = torch.argsort(at // S, stable=True)
    met, count = torch.unique_consecutive((at // S)[order], return_counts=True)
    for b, tokens in zip(met.tolist(), torch.split(order, count.tolist())):
        place, y = at[tokens] % S, x[tokens].double()
        need = (y.abs().amax(dim=(0, 2)) / top).clamp(min=LEAST_SCALE)
        if bool((place == 0).any()):
            now = need
        else:
            now = torch.maximum(scale[b], need)
            grown = (now > scale[b])[None, :, None]
            pool[b] = torch.where(grown, _nearest(pool[b] * (scale[b] / now)[None, :, None], codes), pool[b])
        scale[b] = now
        pool[b, place] = _nearest(y / now[None, :, None], codes)
    return pool, scale


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
            k, v = ((p[:, :, h].view(torch.uint8)[ids].view(p.dtype).double() * c[ids, h].double()[:, None, None]).flatten(0, 1)[first:n]
                    for p, c in ((s["kpool"], s["kscale"]), (s["vpool"], s["vscale"])))
            x = s["q"][b, heads].double() @ k.T * D ** -0.5
            lse[b, heads] = torch.logsumexp(x, -1)
            out[b, heads] = torch.softmax(x, -1) @ v
    return out, lse


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attn":
        return _exact_attn(s)
    if case["op"] == "append":
        (k, ks), (v, vs) = (_exact_write(s[x], s[x + "pool"], s[x + "scale"], s["slots"], case["codes"]) for x in ("k", "v"))
        return (k * ks[:, None, :, None]).flatten(0, 1), (v * vs[:, None, :, None]).flatten(0, 1), ks, vs
    out = []
    for pool, scale in ((s["kpool"], s["kscale"]), (s["vpool"], s["vscale"])):
        every = (pool.double() * scale.double()[:, None, :, None]).flatten(0, 1)
        rows = torch.zeros((len(s["slots"]),) + every.shape[1:], dtype=torch.float64, device=every.device)
        live = s["slots"] >= 0
        rows[live] = every[s["slots"][live]]
        out.append(rows)
    return tuple(out)
