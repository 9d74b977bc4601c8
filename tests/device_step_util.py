"""Plain 64-bit models of the calls whose lengths stay on the device, with the error that each rounding allows."""
import math

import numpy as np
import torch

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # of a rounding, relative
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}              # half of fp16's smallest step


def f64(t):
    return t.detach().double().cpu().numpy()


class SlotModel:
    """ps_build_slots one row and one id at a time."""

    def __init__(self, block_size, num_blocks, free):
        self.S, self.M, self.free = block_size, num_blocks, list(free)

    def step(self, ctx, new, tables, stride, max_tokens, pool=True):
        """(status, tables, slots, positions, start, ctx_out); the model's own stack moves."""
        S = self.S
        B = len(ctx)
        failed = (0, [list(t) for t in tables], [-1] * max_tokens, [0] * max_tokens, [0] * (B + 1), list(ctx))
        blocks = lambda n: -(-n // S)
        for c, n in zip(ctx, new):
            if c < 0 or n < -1 or c + max(n, 0) > stride * S:
                return (5,) + failed[1:]
        if sum(max(n, 0) for n in new) > max_tokens:
            return (5,) + failed[1:]
        back = sum(blocks(c) for c, n in zip(ctx, new) if n == -1)
        need = sum(blocks(c + n) - blocks(c) for c, n in zip(ctx, new) if n >= 0)
        if pool:
            if len(self.free) + back > self.M:
                return (5,) + failed[1:]
            if len(self.free) + back < need:
                return (4,) + failed[1:]
        out = [list(t) for t in tables]
        if pool:
            for b in range(B):
                if new[b] == -1:
                    self.free += out[b][: blocks(ctx[b])]
            for b in range(B):
                if new[b] >= 0:
                    for j in range(blocks(ctx[b]), blocks(ctx[b] + new[b])):
                        out[b][j] = self.free.pop()
        status, slots, pos, start = 0, [], [], [0]
        for b in range(B):
            for i in range(max(new[b], 0)):
                p = ctx[b] + i
                id_ = out[b][p // S]
                if 0 <= id_ < self.M:
                    slots.append(id_ * S + p % S)
                else:
                    slots.append(-1)
                    status = 2
                pos.append(p)
            start.append(len(slots))
        pad = max_tokens - len(slots)
        return (status, out, slots + [-1] * pad, pos + [0] * pad, start,
                [0 if n == -1 else c + n for c, n in zip(ctx, new)])


def rope_want(x, pos, inv_freq, axis, neighbours, inverse):
    """Rotation of x [T][heads][D] in 64 bits and the error a 32-bit rotation with one rounding may have.

    The angle's fraction of a turn is rounded to 32 bits (off by 2^-26 turns, 2^-23 radians), sine and cosine are off
    by a few 2^-24 and the two products and their sum by 3 roundings of 2^-24: below 2^-20 (|x1| + |x2|) together."""
    dt = x.dtype
    x = f64(x)
    T, half = x.shape[0], len(inv_freq)
    inv = f64(inv_freq)
    pos = pos.cpu().numpy().astype(np.float64).reshape(-1, T)
    ang = np.stack([pos[axis[i]] * inv[i] for i in range(half)], -1) if half else np.zeros((T, 0))
    if inverse:
        ang = -ang
    c, s = np.cos(ang)[:, None, :], np.sin(ang)[:, None, :]
    a = slice(0, 2 * half, 2) if neighbours else slice(0, half)
    b = slice(1, 2 * half, 2) if neighbours else slice(half, 2 * half)
    y, tol = x.copy(), np.zeros_like(x)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    raw = 2.0 ** -20 * (np.abs(x[..., a]) + np.abs(x[..., b]))
    tol[..., a], tol[..., b] = raw, raw
    turned = np.zeros(x.shape[-1], bool)
    turned[: 2 * half] = True
    tol = np.where(turned, tol + HALF_STEP[dt] * (np.abs(y) + tol) + TINY[dt], 0.0)   # other dims are copied
    return y, tol


def check_within(got, want, tol):
    got = f64(got)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (f"{bad.sum()} of {bad.size} values off, worst by "
                           f"{np.nanmax(np.where(bad, np.abs(got - want) / np.maximum(tol, 1e-300), 0))} times its tolerance")


def attn_want(kpool, vpool, q, tables, ctx, window=0, scale=None, weight_error=None):
    """(out, lse, tolerances of both) in 64 bits.  tables: lists of block ids per row; ids outside the pool are skipped.

    A score is a 32-bit sum of D exact products: off by at most 2^-20 sum |q k| scale (D roundings of 2^-24, and some
    room for the tensor cores' own order).  Both sides of p / sum p carry it, 2^-20 more covers exp2, the sums and
    the division.  A weight is held as the sum of two numbers of the inputs' type (a half step of a half step off), and
    the result is rounded once.  weight_error: of a kernel that rounds its weights otherwise."""
    dt = q.dtype
    B, Hq, D = q.shape
    nb, S, Hkv, _ = kpool.shape
    G = Hq // Hkv
    scale = 1 / math.sqrt(D) if scale is None else scale
    weight_error = HALF_STEP[dt] ** 2 if weight_error is None else weight_error
    out, lse = np.zeros((B, Hq, D)), np.full((B, Hq), -np.inf)
    tol, tol_lse = np.zeros((B, Hq, D)), np.zeros((B, Hq))
    qf = f64(q)
    for b in range(B):
        n = ctx[b]
        first = max(0, n - window) if window else 0
        rows = [(tables[b][t // S], t % S) for t in range(first, n)]
        rows = [r for r in rows if 0 <= r[0] < nb]
        if not rows:
            continue
        ids = torch.tensor([r[0] for r in rows], device=kpool.device)
        at = torch.tensor([r[1] for r in rows], device=kpool.device)
        K, V = f64(kpool[ids, at]), f64(vpool[ids, at])
        for h in range(Hq):
            k, v = K[:, h // G], V[:, h // G]
            s = k @ qf[b, h] * scale
            m = s.max()
            p = np.exp(s - m)
            l = p.sum()
            out[b, h] = p @ v / l
            lse[b, h] = m + math.log(l)
            ds = 2.0 ** -20 * abs(scale) * float((np.abs(k) @ np.abs(qf[b, h])).max())
            A = p @ np.abs(v) / l
            e = A * (weight_error + 2 * ds + 2.0 ** -20)
            tol[b, h] = e + HALF_STEP[dt] * (np.abs(out[b, h]) + e) + TINY[dt]
            tol_lse[b, h] = ds + 2.0 ** -20 * (1 + abs(lse[b, h]) + abs(m))
    return out, lse, tol, tol_lse


def check_attn(out, lse, want):
    o, l, tol, tol_lse = want
    check_within(out, o, tol)
    got = f64(lse)
    assert np.array_equal(np.isneginf(got), np.isneginf(l))
    fin = np.isfinite(l)
    assert (np.abs(got[fin] - l[fin]) <= tol_lse[fin]).all(), np.abs(got[fin] - l[fin]).max()


def tables_tensor(tables, stride, fill=0):
    arr = np.full((len(tables), stride), fill, np.int32)
    for i, t in enumerate(tables):
        arr[i, : len(t)] = t
    return torch.from_numpy(arr).cuda()


def make_tables(rng, ctx, S, nb):
    """Block tables of the rows out of a shuffled pool."""
    order = list(rng.permutation(nb))
    return [[int(order.pop()) for _ in range(-(-n // S))] for n in ctx]
