"""Plain models of the calls over a cache of 8 bits."""
import numpy as np
import torch

from device_step_util import attn_want, f64

CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
TOP = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}
LEAST = np.float32(2.0 ** -100)


def nearest_code(y, dt):
    """The codes nearest to y (64 bits), ties to even, as the values they are."""
    if dt == torch.int8:
        return np.clip(np.rint(y), -127, 127)
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3)
    return np.clip(np.rint(y / step) * step, -448, 448)


def bits(pool):
    return pool.view(torch.uint8) if pool.dtype != torch.uint8 else pool


def values(pool):
    """The codes of a pool as 64-bit numbers."""
    return f64(pool.float())


def codes_tensor(v, dt):
    return torch.from_numpy(np.asarray(v, np.float32)).cuda().to(dt)


class CacheModel:
    """One side of a cache, block by block with the documented 32-bit arithmetic: equal to the call's, bit for bit."""

    def __init__(self, pool, scale):
        self.dt = pool.dtype
        self.code, self.scale = values(pool), scale.detach().cpu().numpy().copy()

    def append(self, x, slots):
        """x [tokens][heads][dim] (a tensor of 16 bits), slots a list; slots outside the pool are skipped."""
        S = self.code.shape[1]
        x = f64(x)
        groups = {}
        for t, s in enumerate(slots):
            if 0 <= s < self.code.shape[0] * S:
                groups.setdefault(s // S, []).append((t, s % S))
        for b, tokens in groups.items():
            ts, places = [t for t, _ in tokens], [p for _, p in tokens]
            most = np.abs(x[ts]).max(axis=(0, 2)).astype(np.float32)
            need = most * np.float32(1.0 / TOP[self.dt])
            old = np.zeros_like(need) if 0 in places else self.scale[b]
            new = np.maximum(np.maximum(old, need), LEAST)
            inv = (np.float32(1) / new).astype(np.float32)
            if 0 not in places:
                for h in np.nonzero(new > old)[0]:
                    self.code[b, :, h] = self.round(self.code[b, :, h], old[h] * inv[h])
            self.code[b, places] = self.round(x[ts], inv[None, :, None])
            self.scale[b] = new

    def round(self, x, factor):
        if self.dt == torch.int8:
            return nearest_code(x * np.asarray(factor, np.float64), self.dt)
        return nearest_code((x.astype(np.float32) * factor).astype(np.float64), self.dt)

    def check(self, pool, scale):
        got = scale.detach().cpu().numpy()
        assert np.array_equal(got, self.scale), np.abs(got - self.scale).max()
        v = values(pool)
        assert np.array_equal(v, self.code), (np.argwhere(v != self.code)[:3], (v != self.code).sum())


def read_want(pool, scale, slots, dt):
    """Rows of the slots in 16 bits: the 32-bit product rounded once."""
    S, H, D = pool.shape[1:]
    at = torch.as_tensor(slots, device="cuda")
    x = bits(pool).reshape(-1, H, D)[at].view(pool.dtype).float()
    return (x * scale[at // S][..., None]).to(dt)


def make_cache(shape, dt, g, spread=0.5):
    """Random codes over their whole range, with scales that differ by up to 2^(2 spread) between blocks and heads."""
    x = (torch.rand(shape, device="cuda", generator=g) * 2 - 1) * TOP[dt]
    pool = torch.round(x).to(torch.int8) if dt == torch.int8 else x.to(dt)
    scale = torch.exp2((torch.rand((shape[0], shape[2]), device="cuda", generator=g) * 2 - 1) * spread) * (2.0 / TOP[dt])
    return pool, scale


def quant_attn_want(kpool, vpool, ks, vs, q, tables, ctx, window=0, scale=None):
    """attn_want over the values that the cache stands for.

    Over that, a weight times its value scale is a product in 32 bits (2^-24), held as one fp16 number for results in bf16 (off by
    2^-11 of itself) and as the sum of two for results in fp16 (2^-22), or by 2^-25 where fp16 has no smaller steps; largest weights are 2^8 or more and refer to the power of two below
    the row's largest value scale, so that the latter is 2^-33 of a token's largest possible value, times the tokens.  A score
    is multiplied by two factors (2^-23, within what attn_want gives it).  A query's values are held to 2^-21 of their head's
    largest: a score is off by that times the key's magnitudes, and a result by twice as much of its largest value."""
    K = kpool.double() * ks.double()[:, None, :, None]
    V = vpool.double() * vs.double()[:, None, :, None]
    out, lse, tol, tol_lse = attn_want(K, V, q, tables, ctx, window, scale, weight_error=2.0 ** -21 + (2.0 ** -11 if q.dtype == torch.bfloat16 else 0.0))
    nb, S = kpool.shape[:2]
    G = q.shape[1] // kpool.shape[2]
    for b, n in enumerate(ctx):
        ids = [i for i in tables[b][: -(-n // S)] if 0 <= i < nb]
        if ids:
            at = torch.tensor(ids, device="cuda")
            top = vs[at].abs().amax(0).double().cpu().numpy() * TOP[vpool.dtype]
            tol[b] += np.repeat(top, G)[:, None] * (n * 2.0 ** -33)
            ds = np.abs(f64(q[b])).max(-1) * np.repeat(K[at].abs().sum(-1).amax((0, 1)).cpu().numpy(), G) * 2.0 ** -21
            ds *= q.shape[2] ** -0.5 if scale is None else abs(scale)
            tol[b] += (2 * ds * np.repeat(V[at].abs().amax((0, 1, 3)).cpu().numpy(), G))[:, None]
            tol_lse[b] += ds
    return out, lse, tol, tol_lse
