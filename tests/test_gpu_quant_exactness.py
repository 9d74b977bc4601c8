"""How exact results over a cache of 8 bits are: that of 32-bit arithmetic, rounded once."""
import numpy as np
import pytest
import torch

from device_step_util import DTYPES, HALF_STEP, TINY, attn_want, f64
from quant_util import CODES, TOP
from test_gpu_quant import attn_case, run_attn

pytestmark = pytest.mark.gpu


def check_rounded_once(got, lse, cache, q, tables, ctx, scale=None):
    """Results against 64 bits: off by half a step of the value at hand and by what 32-bit arithmetic is off.

    Of the latter attn_want has the part of scores, exp2, sums and the division.  A weight times its value scale is a 32-bit
    product (2^-24) and held as the sum of two fp16 numbers (half a step of half a step, 2^-22): 2^-21 together.  Below fp16's
    smallest steps it is off by 2^-25, where largest weights are 2^8 or more and refer to the power of two below the row's
    largest value scale: 2^-33 of a token's largest possible value, times the tokens."""
    kp, vp, ks, vs = cache
    dt = q.dtype
    K, V = (p.double() * s.double()[:, None, :, None] for p, s in ((kp, ks), (vp, vs)))
    out, want_lse, tol, tol_lse = attn_want(K, V, q, tables, ctx, 0, scale, weight_error=2.0 ** -21)
    e = (tol - HALF_STEP[dt] * np.abs(out) - TINY[dt]) / (1 + HALF_STEP[dt])       # attn_want has half of the largest step
    S, G = kp.shape[1], q.shape[1] // kp.shape[2]
    for b, n in enumerate(ctx):
        ids = tables[b][: -(-n // S)]
        if ids:
            top = f64(vs)[ids].max(0) * TOP[vp.dtype]
            e[b] += np.repeat(top, G)[:, None] * (n * 2.0 ** -33)
    step = HALF_STEP[dt] * np.exp2(np.floor(np.log2(np.maximum(np.abs(out) + e, 2.0 ** -126)))) + TINY[dt]
    bad = ~(np.abs(f64(got) - out) <= step + e)
    assert not bad.any(), f"{bad.sum()} of {bad.size} results"
    fin = np.isfinite(want_lse)
    assert (np.abs(f64(lse) - want_lse)[fin] <= tol_lse[fin]).all(), np.abs(f64(lse) - want_lse)[fin].max()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("hq,hkv,D", [(8, 2, 128), (16, 1, 64)])
def test_weights_of_few_tokens(dtype, codes, hq, hkv, D):
    """With few tokens no rounding of a weight is averaged away: each would show in the result."""
    rng = np.random.default_rng(1)
    ctx = rng.integers(1, 7, 300).tolist()
    cache, q, tables = attn_case(rng, ctx, hq, hkv, D, 4, DTYPES[dtype], CODES[codes], spread=2.0)
    q = q * 0.125                          # scores next to one another
    check_rounded_once(*run_attn(cache, q, tables, ctx), cache, q, tables, ctx)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("hq,hkv,D,up", [(8, 2, 128, 12), (16, 1, 64, 12), (3, 3, 64, 14), (32, 2, 128, 9)])
def test_a_querys_small_values_next_to_a_large_one(dtype, codes, hq, hkv, D, up):
    """One dim of every query is 2^up and more times the others and meets codes of zero: the others decide, as in 32 bits."""
    rng = np.random.default_rng(2)
    ctx = [1, 300, 40, 900]
    cache, q, tables = attn_case(rng, ctx, hq, hkv, D, 16, DTYPES[dtype], CODES[codes])
    q[..., 5] = 2.0 ** up
    q[..., 6] *= 2.0 ** -8
    cache[0].view(torch.uint8)[..., 5] = 0
    check_rounded_once(*run_attn(cache, q, tables, ctx), cache, q, tables, ctx)
    if dtype == "bf16":                    # and further apart than fp16 reaches
        q[..., 5] *= 2.0 ** 8
        q *= 2.0 ** 60
        cache[2] *= 2.0 ** -60
        check_rounded_once(*run_attn(cache, q, tables, ctx), cache, q, tables, ctx)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("codes", ["int8", "e4m3"])
def test_infinite_queries(codes, dtype):
    """Scores that are all minus infinity give zeros, as a row without tokens does; any other infinite query gives NaN."""
    rng = np.random.default_rng(3)
    ctx = [70, 1, 2000]
    cache, q, tables = attn_case(rng, ctx, 8, 2, 64, 16, DTYPES[dtype], CODES[codes])
    codes8 = cache[0].view(torch.uint8)
    codes8[..., 5] = 0x21                  # positive in every token
    bad = q.clone()
    bad[:, 0, 5], bad[:, 3, 5], bad[:, 6, 5] = -float("inf"), float("inf"), -float("inf")
    bad[:, 6, 9] = float("inf")            # met by codes of either sign
    codes8[..., 9] |= 1
    out, lse = run_attn(cache, bad, tables, ctx)
    K = cache[0].double() * cache[2].double()[:, None, :, None]      # (the odd codes of 8-bit floats have NaN among them)
    same, same_lse = run_attn(cache, q, tables, ctx)
    seen = set()
    for b, n in enumerate(ctx):
        k = K[torch.tensor(tables[b], device="cuda")].flatten(0, 1)[:n]
        for h in range(8):
            scores = k[:, h // 4] @ bad[b, h].double()
            if torch.isneginf(scores).all():
                seen.add("zeros")
                assert not out[b, h].any() and torch.isneginf(lse[b, h])
            elif not scores.isfinite().all():
                seen.add("NaN")
                assert out[b, h].isnan().all() and lse[b, h].isnan()
            else:
                seen.add("numbers")
                assert h not in (0, 3, 6) and torch.equal(out[b, h], same[b, h]) and torch.equal(lse[b, h], same_lse[b, h])
    assert seen == {"zeros", "NaN", "numbers"}
