"""Kernels and layouts of the 8-bit cache's calls that take their own path: uneven heads in calls of many tokens, keys and values that
lie differently."""
import numpy as np
import pytest
import torch

from device_step_util import DTYPES, check_attn, tables_tensor
from paper_2512_12928_b200 import binding as B
from quant_util import CODES, CacheModel, bits, make_cache, quant_attn_want, read_want
from test_gpu_device_step import dev
from test_gpu_quant import I64, append, attn_case, gen, kv_rows, run_attn, run_slots

pytestmark = pytest.mark.gpu


def append_rule(T, H, D, S, sides=2):
    """(warps of a team, tokens of a CTA, whether rows divide a warp's lanes) of an append whose rows are read 32 bytes at a time."""
    assert D % 16 == 0
    vecs, units, team = D // 16, sides * H, 1
    while team < 8 and 32 * 4 * team < min(S, T) * vecs:
        team *= 2
    tokens = team
    while 2 * tokens <= min(S, 128 if team > 1 else 16) and T // (2 * tokens) * units * team >= 148 * 16:
        tokens *= 2
    return team, tokens, 32 % vecs == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("H,D,S,teams", [(16, 80, 24, False), (16, 48, 16, False), (9, 112, 12, False), (16, 80, 128, True), (12, 96, 100, True),
                                         (16, 112, 300, True)])
def test_append_of_many_tokens_of_uneven_heads(dtype, codes, H, D, S, teams):
    """Rows whose vectors do not divide a warp's lanes, in calls of so many tokens that CTAs have several: pieces that begin and end
    inside blocks, scales that rise by the second call and not by the third."""
    rng = np.random.default_rng(D + S)
    rows = [(int(rng.integers(0, S)), int(n)) for n in rng.integers(0, 104, 100 if not teams else 70) if n] + [(5, 700)]
    nb = sum(-(-(f + n) // S) for f, n in rows) + 3
    slots = run_slots(rng, S, nb, rows) + [-1] * 11
    team, tokens, even = append_rule(len(slots), H, D, S)
    assert not even and tokens > team and (team > 1) == teams
    (kp, ks), (vp, vs) = (make_cache((nb, S, H, D), CODES[codes], gen(D + i), spread=3.0) for i in range(2))
    mk, mv = CacheModel(kp, ks), CacheModel(vp, vs)
    for step in range(3):
        k, v = kv_rows(len(slots), H, D, DTYPES[dtype], step + D)
        k, v = (x * (1.0, 4.0, 0.25)[step] for x in (k, v))
        append(k, v, (kp, vp, ks, vs), slots)
        mk.append(k, slots)
        mv.append(v, slots)
        mk.check(kp, ks)
        mv.check(vp, vs)


def apart(cache, gaps, scale_gaps):
    """Copies of the cache's codes and scales whose blocks lie `gaps` bytes and `scale_gaps` floats further apart, keys' and values'."""
    out = []
    for x, gap in zip(cache, gaps + scale_gaps):
        nb, n = len(x), x[0].numel()
        wide = torch.zeros((nb, n + gap), device="cuda", dtype=torch.uint8 if x.element_size() == 1 else x.dtype)
        view = wide[:, :n].view(x.dtype).view(x.shape)
        (bits(view) if x.element_size() == 1 else view).copy_(bits(x) if x.element_size() == 1 else x)
        out.append(view)
    return out


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("gaps,scale_gaps", [((0, 16), (0, 0)), ((64, 0), (0, 3)), ((16, 4096), (5, 0)), ((0, 0), (1, 2))])
def test_attn_of_keys_and_values_with_strides_of_their_own(codes, gaps, scale_gaps):
    rng = np.random.default_rng(3)
    for hq, hkv, D, window in ((8, 2, 128, 0), (16, 1, 64, 100), (4, 4, 64, 0)):
        ctx = [300, 1, 0, 77, 1500]
        cache, q, tables = attn_case(rng, ctx, hq, hkv, D, 16, torch.bfloat16, CODES[codes])
        got = run_attn(apart(cache, gaps, scale_gaps), q, tables, ctx, window=window)
        check_attn(*got, quant_attn_want(*cache, q, tables, ctx, window))
        plain = run_attn(cache, q, tables, ctx, window=window)
        assert all(torch.equal(a, b) for a, b in zip(got, plain))


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("D,gaps,scale_gaps,row_gaps", [(128, (0, 32), (0, 3), (0, 64)), (64, (16, 0), (2, 0), (32, 0)), (72, (8, 24), (1, 4), (8, 24)),
                                                        (20, (1, 2), (0, 1), (3, 0))])
def test_append_and_read_of_keys_and_values_with_strides_of_their_own(codes, D, gaps, scale_gaps, row_gaps):
    H, S, T = 3, 16, 250
    rng = np.random.default_rng(4)
    slots = run_slots(rng, S, 30, [(3, 100), (0, 40), (15, 110)])
    (k0, s0), (v0, s1) = (make_cache((30, S, H, D), CODES[codes], gen(i), spread=3.0) for i in range(2))
    cache = apart((k0, v0, s0, s1), gaps, scale_gaps)
    models = CacheModel(k0, s0), CacheModel(v0, s1)
    wide = [torch.full((T, H * D + g), 3.0, device="cuda", dtype=torch.bfloat16) for g in row_gaps]
    rows = [w[:, : H * D].unflatten(1, (H, D)) for w in wide]
    for step in range(2):
        for r, x in zip(rows, kv_rows(T, H, D, torch.bfloat16, step)):
            r.copy_(x * (1 + 3 * step))
        append(*rows, cache, slots)
        for i, m in enumerate(models):
            m.append(rows[i], slots)
            m.check(cache[i], cache[2 + i])
    want = [read_want(cache[i].contiguous(), cache[2 + i], slots, torch.bfloat16) for i in range(2)]
    assert B.ps_quant_read(*cache, dev(slots, I64), *rows) == (B.PS_OK, "")
    for r, w, x, g in zip(rows, want, wide, row_gaps):
        assert torch.equal(r, w) and (x[:, H * D:] == 3.0).all()
