"""ps_quant_append, ps_quant_read and ps_quant_attn against plain models, alone and as steps over one cache."""
import numpy as np
import pytest
import torch

from device_step_util import DTYPES, check_attn, make_tables, rope_want, check_within, tables_tensor
from paper_2512_12928_b200 import binding as B
from quant_util import CODES, LEAST, TOP, CacheModel, bits, make_cache, quant_attn_want, read_want
from test_gpu_device_step import Engine, dev, engine_steps

pytestmark = pytest.mark.gpu

I32, I64 = torch.int32, torch.int64


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def kv_rows(T, H, D, dt, seed, fused=True):
    """Keys and values with a few large channels, in one buffer as a fused projection leaves them."""
    x = torch.randn((T, 2 * H * D), device="cuda", generator=gen(seed))
    x[:, ::37] *= 6
    x = x.to(dt)
    k, v = x[:, : H * D].view(T, H, D), x[:, H * D:].view(T, H, D)
    return (k, v) if fused else (k.contiguous(), v.contiguous())


def run_slots(rng, S, nb, rows):
    """Slots of rows (first place, tokens) in blocks of their own, neighbours in the call."""
    order, slots = rng.permutation(nb).tolist(), []
    for first, n in rows:
        ids = [order.pop() for _ in range(-(-(first + n) // S))]
        slots += [ids[p // S] * S + p % S for p in range(first, first + n)]
    return slots


def append(k, v, cache, slots, want_status=0):
    status = dev([0])
    rc, text = B.ps_quant_append(k, v, *cache, dev(slots, I64), status_word=status)
    assert rc == B.PS_OK, text
    torch.cuda.synchronize()
    assert status.item() == want_status


# ------------------------------------------------------------------------------------------------ append

@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("H,D,S,rows", [
    (8, 128, 16, [(3, 1)]), (8, 128, 16, [(0, 1)]), (1, 64, 1, [(0, 7)]), (4, 128, 16, [(15, 2), (0, 33), (7, 9), (5, 1)]),
    (3, 80, 24, [(0, 24), (23, 26), (1, 1), (0, 100)]), (16, 96, 7, [(6, 30), (0, 7)]), (2, 256, 100, [(99, 2), (0, 250), (50, 50)]),
    (1, 512, 16, [(2, 40)]), (5, 7, 5, [(4, 13), (0, 5)]), (2, 1, 3, [(1, 5)]), (8, 64, 32, [(i % 32, 1) for i in range(70)]),
    (1, 8, 200, [(10, 500)]), (2, 128, 16, [(0, 700)]), (9, 40, 8, [(3, 300), (0, 40)])])
def test_append(dtype, codes, H, D, S, rows):
    dt, ct = DTYPES[dtype], CODES[codes]
    rng = np.random.default_rng(H * 1000 + D)
    nb = sum(-(-(f + n) // S) for f, n in rows) + 5
    slots = run_slots(rng, S, nb, rows)
    (kp, ks), (vp, vs) = (make_cache((nb, S, H, D), ct, gen(D + i), spread=3.0) for i in range(2))
    mk, mv = CacheModel(kp, ks), CacheModel(vp, vs)
    for step in range(3):                  # the same places again: larger, then smaller values
        k, v = kv_rows(len(slots), H, D, dt, step + D)
        k, v = (x * (1.0, 4.0, 0.25)[step] for x in (k, v))
        append(k, v, (kp, vp, ks, vs), slots)
        mk.append(k, slots)
        mv.append(v, slots)
        mk.check(kp, ks)
        mv.check(vp, vs)


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
def test_append_over_the_steps_of_a_decode(codes):
    """Rows grow by a token a step and take new blocks, whose old scales (NaN among them) are nobody's; some tokens are padding."""
    H, D, S, nb, B_ = 3, 64, 4, 60, 9
    rng = np.random.default_rng(3)
    (kp, ks), (vp, vs) = (make_cache((nb, S, H, D), CODES[codes], gen(i), spread=8.0) for i in range(2))
    ks[:], vs[:] = float("nan"), 1e30
    mk, mv = CacheModel(kp, ks), CacheModel(vp, vs)
    free, ids, n = rng.permutation(nb).tolist(), [[] for _ in range(B_)], [0] * B_
    for step in range(17):
        slots = []
        for b in range(B_):
            if rng.random() < 0.2:
                slots.append(-1 - int(rng.integers(3)))
                continue
            if n[b] % S == 0:
                ids[b].append(free.pop())
            slots.append(ids[b][-1] * S + n[b] % S)
            n[b] += 1
        k, v = kv_rows(B_, H, D, torch.bfloat16, 50 + step)
        k, v = k * float(rng.uniform(0.3, 3)), v * float(rng.uniform(0.3, 3))
        append(k, v, (kp, vp, ks, vs), slots)
        mk.append(k, slots)
        mv.append(v, slots)
        np.testing.assert_array_equal(ks.cpu().numpy(), mk.scale)
        np.testing.assert_array_equal(vs.cpu().numpy(), mv.scale)
        assert np.array_equal(kp.float().cpu().numpy(), mk.code) and np.array_equal(vp.float().cpu().numpy(), mv.code)


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("T", [40, 3001])
def test_append_skips_padding_and_slots_outside_the_pool(codes, T):
    H, D, S = 2, 64, 16
    rng = np.random.default_rng(4)
    nb = T // S + 9
    rows = [(5, T - 20), (0, 20)]
    slots = run_slots(rng, S, nb, rows)
    whole = list(slots)
    for i in (0, 1, 9, 30, T - 1):
        slots[i] = -1
    for i in (12, 31):
        slots[i] = nb * S + i
    slots[33] = 1 << 45
    # a run that padding cuts in two may meet its block twice, which leaves that block undefined: its tokens become padding too
    for i in range(T):
        cut = {whole[j] // S for j in (9, 12, 30, 31, 33)}
        if whole[i] // S in cut and slots[i] >= 0 and slots[i] < nb * S:
            slots[i] = -7
    (kp, ks), (vp, vs) = (make_cache((nb, S, H, D), CODES[codes], gen(i)) for i in range(2))
    mk, mv = CacheModel(kp, ks), CacheModel(vp, vs)
    k, v = kv_rows(T, H, D, torch.float16, 8)
    append(k, v, (kp, vp, ks, vs), slots, want_status=1)
    mk.append(k, slots)
    mv.append(v, slots)
    mk.check(kp, ks)
    mv.check(vp, vs)


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
def test_append_of_a_blocks_tokens_in_any_order(codes):
    H, D, S, nb = 2, 128, 16, 12
    rng = np.random.default_rng(5)
    (kp, ks), (vp, vs) = (make_cache((nb, S, H, D), CODES[codes], gen(i), spread=4.0) for i in range(2))
    mk, mv = CacheModel(kp, ks), CacheModel(vp, vs)
    slots = []
    for b, places in ((3, range(16)), (7, [4, 2, 9]), (0, [15, 0]), (11, [8]), (5, rng.permutation(16).tolist())):
        slots += [b * S + p for p in places]
    k, v = kv_rows(len(slots), H, D, torch.bfloat16, 5)
    append(k, v, (kp, vp, ks, vs), slots)
    mk.append(k, slots)
    mv.append(v, slots)
    mk.check(kp, ks)
    mv.check(vp, vs)


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("D", [64, 72, 20])
def test_append_and_read_of_every_alignment(codes, D):
    """How wide the accesses are follows from addresses, strides and sizes; what comes out does not."""
    ct, H, S, T = CODES[codes], 3, 6, 50
    rng = np.random.default_rng(6)
    nb = 14
    slots = run_slots(rng, S, nb, [(2, 30), (0, 20)])
    first = None
    for shift, gap, rshift, rgap in ((0, 0, 0, 0), (8, 8, 4, 4), (16, 16, 8, 8), (1, 3, 0, 0), (0, 0, 1, 1), (2, 8, 2, 6)):
        (k0, s0), (v0, s1) = (make_cache((nb, S, H, D), ct, gen(i), spread=4.0) for i in range(2))
        n = S * H * D
        buf = torch.full((shift + nb * (2 * n + gap),), 77, device="cuda", dtype=torch.uint8)
        blocks = buf[shift:].view(nb, 2 * n + gap)
        kp, vp = (blocks[:, i * n: (i + 1) * n].view(ct).view(nb, S, H, D) for i in range(2))
        bits(kp).copy_(bits(k0))
        bits(vp).copy_(bits(v0))
        sbuf = torch.full((nb, 2 * H + 5), 3.0, device="cuda")
        ks, vs = sbuf[:, 1: H + 1], sbuf[:, H + 2: 2 * H + 2]
        ks.copy_(s0)
        vs.copy_(s1)
        rows = torch.full((rshift + T * (2 * H * D + rgap),), 5.0, device="cuda", dtype=torch.bfloat16)
        parts = [rows[rshift:].view(T, 2 * H * D + rgap)[:, i * H * D: (i + 1) * H * D].unflatten(1, (H, D)) for i in range(2)]
        for dst, src in zip(parts, kv_rows(T, H, D, torch.bfloat16, 9)):
            dst.copy_(src)
        was = rows.clone()
        append(*parts, (kp, vp, ks, vs), slots)
        assert torch.equal(rows, was)
        if gap:
            assert (blocks[:, 2 * n:] == 77).all()
        assert (buf[:shift] == 77).all() and (sbuf[:, [0, H + 1, 2 * H + 2]] == 3.0).all()
        wk, wv = read_want(kp, ks, slots, torch.bfloat16), read_want(vp, vs, slots, torch.bfloat16)
        rc, text = B.ps_quant_read(kp, vp, ks, vs, dev(slots, I64), *parts)
        assert rc == B.PS_OK, text
        assert torch.equal(parts[0], wk) and torch.equal(parts[1], wv)
        if rgap:
            assert (rows[rshift:].view(T, 2 * H * D + rgap)[:, 2 * H * D:] == 5.0).all()
        assert (rows[:rshift] == 5.0).all()
        got = [bits(kp).clone(), bits(vp).clone(), ks.clone(), vs.clone(), wk, wv]
        if first is None:
            first = got
            mk, mv = CacheModel(k0, s0), CacheModel(v0, s1)
            for m, x in zip((mk, mv), kv_rows(T, H, D, torch.bfloat16, 9)):
                m.append(x, slots)
            mk.check(kp, ks)
            mv.check(vp, vs)
        assert all(torch.equal(a, b) for a, b in zip(first, got))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("codes", ["int8", "e4m3"])
def test_append_of_zeros_and_of_the_smallest_and_largest_values(dtype, codes):
    H, D, S, nb = 4, 64, 4, 6
    dt = DTYPES[dtype]
    (kp, ks), (vp, vs) = (make_cache((nb, S, H, D), CODES[codes], gen(i)) for i in range(2))
    mk, mv = CacheModel(kp, ks), CacheModel(vp, vs)
    k = torch.zeros((8, H, D), device="cuda", dtype=dt)
    v = torch.zeros_like(k)
    v[0, 0, 0], v[1, 1, 1], v[2, 2] = torch.finfo(dt).tiny, torch.finfo(dt).max, -torch.finfo(dt).max
    v[3, 3] = torch.finfo(dt).smallest_normal / 2
    slots = [0, 1, 2, 3, 9, 10, 11, 16]
    append(k, v, (kp, vp, ks, vs), slots)
    mk.append(k, slots)
    mv.append(v, slots)
    mk.check(kp, ks)
    mv.check(vp, vs)
    assert (ks[0] == float(LEAST)).all() and not kp[0].float().any()


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
def test_append_of_ties_and_borders(codes):
    """Values in the middle between two codes, and next to it on either side, with scales that are powers of two."""
    ct = CODES[codes]
    H, D, S = 1, 256, 16
    top = TOP[ct]
    grid = np.arange(0, 127.25, 0.25) if codes == "int8" else np.concatenate([2.0 ** e * np.arange(8, 16, 0.25) / 8 for e in range(-10, 9)])
    grid = grid[grid <= top]
    x = np.resize(np.concatenate([grid, -grid]), (S, D))
    x[:, 0] = top                          # the block's scale is 1 then
    kp, ks = make_cache((3, S, H, D), ct, gen(1))
    m = CacheModel(kp, ks)
    for factor in (1.0, 2.0 ** -9):
        k = torch.from_numpy(x * factor).cuda().half()[:, None]
        rc, text = B.ps_quant_append(k, None, kp, None, ks, None, torch.arange(S, device="cuda") + S)
        assert rc == B.PS_OK, text
        m.append(k, list(range(S, 2 * S)))
        m.check(kp, ks)


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
def test_append_of_infinite_values_and_nan(codes):
    """A block and head that gets one has a NaN scale, and reads as NaN, until the block is begun anew; others do not notice."""
    H, D, S, nb = 2, 64, 4, 5
    (kp, ks), (vp, vs) = (make_cache((nb, S, H, D), CODES[codes], gen(i)) for i in range(2))
    mk, mv = CacheModel(kp, ks), CacheModel(vp, vs)
    slots = [4, 5, 9, 13]
    k, v = kv_rows(4, H, D, torch.bfloat16, 1, fused=False)
    good_k, good_v = k.clone(), v.clone()
    k[1, 0, 3], k[2, 1, 5], v[3, 0, 63] = float("nan"), float("inf"), -float("inf")
    append(k, v, (kp, vp, ks, vs), slots)
    mk.append(good_k, slots)
    mv.append(good_v, slots)
    bad_k, bad_v = np.isnan(ks.cpu().numpy()), np.isnan(vs.cpu().numpy())
    assert np.argwhere(bad_k).tolist() == [[1, 0], [2, 1]] and np.argwhere(bad_v).tolist() == [[3, 0]]
    for m, pool, s, bad in ((mk, kp, ks, bad_k), (mv, vp, vs, bad_v)):
        assert np.array_equal(s.cpu().numpy()[~bad], m.scale[~bad])
        same = np.broadcast_to(~bad[:, None, :, None], m.code.shape)
        assert np.array_equal(pool.float().cpu().numpy()[same], m.code[same])
    out = torch.zeros((2, H, D), device="cuda", dtype=torch.bfloat16)
    assert B.ps_quant_read(kp, None, ks, None, dev([5, 6], I64), out, None)[0] == B.PS_OK
    assert out[:, 0].isnan().all() and not out[:, 1].isnan().any()
    append(good_k[:1], good_v[:1], (kp, vp, ks, vs), [6])                 # not begun: stays NaN
    assert ks[1, 0].isnan() and not ks[1, 1].isnan()
    append(good_k[:1], good_v[:1], (kp, vp, ks, vs), [4])
    assert not ks[1].isnan().any()


def test_append_of_one_side_and_of_no_tokens():
    H, D, S, nb = 2, 64, 16, 4
    kp, ks = make_cache((nb, S, H, D), torch.int8, gen(1))
    vp, vs = make_cache((nb, S, H, D), torch.int8, gen(2))
    k, v = kv_rows(20, H, D, torch.bfloat16, 1)
    slots = list(range(20))
    m, w = CacheModel(kp, ks), CacheModel(vp, vs)
    m.append(k, slots)
    w.append(v, slots)
    assert B.ps_quant_append(k, None, kp, None, ks, None, dev(slots, I64))[0] == B.PS_OK
    assert B.ps_quant_append(None, v, None, vp, None, vs, dev(slots, I64))[0] == B.PS_OK
    torch.cuda.synchronize()
    m.check(kp, ks)
    w.check(vp, vs)
    assert B.ps_quant_append(k[:0], v[:0], kp, vp, ks, vs, dev([], I64)) == (B.PS_OK, "")
    assert B.ps_quant_read(kp, vp, ks, vs, dev([], I64), k[:0], v[:0]) == (B.PS_OK, "")
    append(k, v, (kp, vp, ks, vs), [-1] * 20)
    m.check(kp, ks)


def test_half_a_step_after_one_write_and_one_more_after_a_growth():
    """The documented error of a value: half a code's step, and half of the new one whenever the scale rises."""
    H, D, S = 1, 64, 16
    kp = torch.zeros((2, S, H, D), device="cuda", dtype=torch.int8)
    ks = torch.zeros((2, H), device="cuda")
    x = torch.randn((S, H, D), device="cuda", generator=gen(1)).bfloat16() * torch.linspace(0.5, 3, S, device="cuda")[:, None, None].bfloat16()
    room = torch.zeros(S, device="cuda", dtype=torch.float64)
    for t in range(S):
        before = ks[1, 0].item() if t else 0.0
        assert B.ps_quant_append(x[t: t + 1], None, kp, None, ks, None, dev([S + t], I64))[0] == B.PS_OK
        now = ks[1, 0].item()
        if now > before:
            room[:t] += now / 2
        room[t] = now / 2
        got = kp[1].double() * ks[1].double()[None, :, None]
        # (and the 32-bit factors: a code is up to 127 steps, each factor is off by 2^-23)
        assert ((got[: t + 1] - x[: t + 1].double()).abs().amax(dim=(1, 2)) <= room[: t + 1] + (t + 1) * 127 * now * 2.0 ** -22).all()


# -------------------------------------------------------------------------------------------------- read

@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("T,H,D,S", [(1, 8, 128, 16), (300, 8, 128, 16), (33, 3, 80, 24), (7, 1, 512, 1), (50, 5, 7, 5), (2001, 16, 64, 32),
                                     (40, 2, 72, 100), (5000, 1, 64, 16), (9, 1024, 16, 4), (20000, 4, 128, 16)])
def test_read(dtype, codes, T, H, D, S):
    dt, ct = DTYPES[dtype], CODES[codes]
    rng = np.random.default_rng(T + D)
    nb = 40
    (kp, ks), (vp, vs) = (make_cache((nb, S, H, D), ct, gen(D + i), spread=6.0) for i in range(2))
    slots = rng.integers(0, nb * S, T)               # some twice, in any order
    slots[rng.random(T) < 0.2] = -3 if T > 1 else 0
    slots[0] = nb * S - 1
    if T > 30:
        slots[[11, 17]] = [nb * S, 1 << 40]
    live = torch.from_numpy((slots >= 0) & (slots < nb * S)).cuda()
    for sides in (3, 1, 2):
        k_out, v_out = (torch.full((T, H, D), 3.0, device="cuda", dtype=dt) for _ in range(2))
        status = dev([0])
        rc, text = B.ps_quant_read(kp, vp, ks, vs, dev(slots.tolist(), I64), k_out if sides & 1 else None, v_out if sides & 2 else None,
                                   status_word=status)
        assert rc == B.PS_OK, text
        torch.cuda.synchronize()
        assert status.item() == (1 if T > 30 else 0)
        at = dev(slots.tolist(), I64)[live]
        for side, out, pool, s in ((1, k_out, kp, ks), (2, v_out, vp, vs)):
            if sides & side:
                assert torch.equal(out[live], read_want(pool, s, at, dt))
                assert (out[~live] == 3.0).all()
            else:
                assert (out == 3.0).all()


def test_read_of_every_code():
    for ct, n in ((torch.int8, 256), (torch.float8_e4m3fn, 256)):
        pool = torch.arange(n, device="cuda").to(torch.uint8).view(ct).view(4, 2, 1, 32)
        s = torch.tensor([[1.0], [0.0], [2.0 ** -130], [float("nan")]], device="cuda")
        for dt in DTYPES.values():
            out = torch.zeros((8, 1, 32), device="cuda", dtype=dt)
            assert B.ps_quant_read(pool, None, s, None, torch.arange(8, device="cuda"), out, None)[0] == B.PS_OK
            want = read_want(pool, s, torch.arange(8, device="cuda"), dt)
            assert torch.equal(out.isnan(), want.isnan()) and torch.equal(out.nan_to_num(0), want.nan_to_num(0))


def test_offsets_beyond_32_bits():
    """A pool of more than 2^32 codes: an append to its last blocks, attended and read back."""
    S, H, D = 16, 8, 128
    nb = (1 << 32) // (S * H * D) + 40
    pool = torch.empty((nb, S, H, D), device="cuda", dtype=torch.int8)
    scale = torch.zeros((nb, H), device="cuda")
    ids = [nb - 1, 3, nb - 17, (1 << 31) // (S * H * D)]
    n = 3 * S + 5
    slots = [ids[i // S] * S + i % S for i in range(n)]
    k, _ = kv_rows(n, H, D, torch.bfloat16, 1)
    assert B.ps_quant_append(k, None, pool, None, scale, None, dev(slots, I64))[0] == B.PS_OK
    out = torch.zeros((n, H, D), device="cuda", dtype=torch.bfloat16)
    assert B.ps_quant_read(pool, None, scale, None, dev(slots, I64), out, None)[0] == B.PS_OK
    assert ((out.double() - k.double()).abs() <= scale[dev(slots, I64) // S][..., None].double() * 0.5 + k.double().abs() * 2.0 ** -7).all()
    sub, sub_scale = pool[dev(ids, I64)], scale[dev(ids, I64)]
    q = torch.randn((1, 32, D), device="cuda").bfloat16()
    got, lse = torch.empty_like(q), torch.empty((1, 32), device="cuda")
    assert B.ps_quant_attn(pool, pool, scale, scale, q, got, dev([ids]), dev([n]), lse=lse)[0] == B.PS_OK
    check_attn(got, lse, quant_attn_want(sub, sub, sub_scale, sub_scale, q, [[0, 1, 2, 3]], [n]))


# --------------------------------------------------------------------------------------------- attention

def attn_case(rng, ctx, hq, hkv, D, S, dt, ct, extra=5, spread=1.0):
    nb = sum(-(-c // S) for c in ctx) + extra
    g = gen(int(rng.integers(1 << 30)))
    (kp, ks), (vp, vs) = (make_cache((nb, S, hkv, D), ct, g, spread) for _ in range(2))
    q = torch.randn((len(ctx), hq, D), device="cuda", generator=g).to(dt)
    return [kp, vp, ks, vs], q, make_tables(rng, ctx, S, nb)


def run_attn(cache, q, tables, ctx, want_status=0, stride=None, **kw):
    out = torch.full(tuple(q.shape), 9.0, device="cuda", dtype=q.dtype)
    lse = torch.full(tuple(q.shape[:2]), 9.0, device="cuda")
    status = dev([0])
    t = tables if torch.is_tensor(tables) else tables_tensor(tables, stride or max(1, max((len(t) for t in tables), default=1)))
    rc, text = B.ps_quant_attn(*cache, q, out, t, dev(list(ctx)), lse=lse, status_word=status, **kw)
    assert rc == B.PS_OK, text
    torch.cuda.synchronize()
    assert status.item() == want_status
    return out, lse


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("hq,hkv,D,S,window", [
    (32, 8, 128, 16, 0), (28, 4, 128, 24, 100), (16, 1, 64, 16, 0), (64, 1, 64, 8, 0), (5, 5, 128, 1, 0), (33, 3, 128, 100, 33), (9, 1, 128, 16, 0),
    (8, 8, 64, 32, 1), (40, 2, 64, 7, 0), (12, 6, 64, 64, 500), (1, 1, 128, 16, 0), (17, 1, 64, 5, 0)])
def test_attn(dtype, codes, hq, hkv, D, S, window):
    rng = np.random.default_rng(hq * 100 + D)
    for ctx in ([1, 0, 31, 32, 33, 700, 2], [300], [0], [5, 2500, 64, 65, 63, 1, 1, 1000]):
        cache, q, tables = attn_case(rng, ctx, hq, hkv, D, S, DTYPES[dtype], CODES[codes])
        check_attn(*run_attn(cache, q, tables, ctx, window=window), quant_attn_want(*cache, q, tables, ctx, window))


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("rows,hi", [(1, 40000), (2, 9000), (150, 300), (300, 40), (700, 3)])
def test_attn_rows_in_parts_and_in_large_numbers(codes, rows, hi):
    rng = np.random.default_rng(rows)
    ctx = rng.integers(0, hi + 1, rows).tolist()
    ctx[-1] = hi
    cache, q, tables = attn_case(rng, ctx, 4, 2, 64, 16, torch.bfloat16, CODES[codes])
    out, lse = run_attn(cache, q, tables, ctx)
    check_attn(out, lse, quant_attn_want(*cache, q, tables, ctx))
    again, lse2 = run_attn(cache, q, tables, ctx)
    assert torch.equal(out, again) and torch.equal(lse, lse2)     # no order of arrival in the results


def test_attn_strided_everything():
    """Codes and scales of a block in one buffer, gaps behind, strided queries and results, one query for all rows."""
    rng = np.random.default_rng(11)
    ctx = [50, 700, 3, 0]
    H, D, S = 2, 128, 24
    cache, _, tables = attn_case(rng, ctx, 8, H, D, S, torch.bfloat16, torch.int8)
    nb, n = len(cache[0]), S * H * D
    buf = torch.zeros((nb, 2 * n + 64), device="cuda", dtype=torch.uint8)
    views = [buf[:, :n].view(torch.int8).view(nb, S, H, D), buf[:, n: 2 * n].view(torch.int8).view(nb, S, H, D),
             buf.view(torch.float32)[:, n // 2: n // 2 + H], buf.view(torch.float32)[:, n // 2 + H: n // 2 + 2 * H]]
    for a, b in zip(views, cache):
        a.copy_(b)
    wide = torch.randn((4, 3, 8, D), device="cuda").bfloat16()
    q = wide[:, 1]
    res = torch.full((4, 2, 8, D), 5.0, device="cuda", dtype=torch.bfloat16)
    lse = torch.zeros((4, 8), device="cuda")
    rc, text = B.ps_quant_attn(*views, q, res[:, 0], tables_tensor(tables, 30), dev(ctx), lse=lse, scale=-0.3)
    assert rc == B.PS_OK, text
    check_attn(res[:, 0], lse, quant_attn_want(*cache, q, tables, ctx, scale=-0.3))
    assert (res[:, 1] == 5.0).all()
    one = q[:1].expand(4, 8, D)
    check_attn(*run_attn(views, one, tables, ctx), quant_attn_want(*cache, one, tables, ctx))
    mine = q.contiguous()
    want = quant_attn_want(*cache, mine, tables, ctx)
    l2 = torch.zeros((4, 8), device="cuda")
    assert B.ps_quant_attn(*views, mine, mine, tables_tensor(tables, 30), dev(ctx), lse=l2)[0] == B.PS_OK     # in place
    check_attn(mine, l2, want)


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
def test_attn_never_reads_what_is_not_attended_into_a_result(codes):
    """Unattended places hold the codes of the largest magnitude (e4m3: NaN too); blocks of which nothing is attended NaN scales."""
    rng = np.random.default_rng(12)
    S = 24
    for dt in DTYPES.values():
        for window in (0, 40):
            ctx = [1, 17, 100, 333, 0]
            cache, q, tables = attn_case(rng, ctx, 8, 2, 128, S, dt, CODES[codes])
            want = quant_attn_want(*cache, q, tables, ctx, window)
            kp, vp, ks, vs = cache
            seen = torch.zeros(kp.shape[:2], dtype=torch.bool, device="cuda")
            for t, n in zip(tables, ctx):
                for i in range(max(0, n - window) if window else 0, n):
                    seen[t[i // S], i % S] = True
            for code, s in ((0x7f, float("nan")), (0xff, float("inf")), (0x80, 3e38), (0x7e, -float("inf"))):
                for pool, scale in ((kp, ks), (vp, vs)):
                    b = bits(pool)
                    b[~seen] = code
                    scale[~seen.any(1)] = s
                check_attn(*run_attn(cache, q, tables, ctx, window=window), want)


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
def test_attn_of_nan_scales(codes):
    """A row and head whose attended blocks have one gives NaN, and nothing else does."""
    rng = np.random.default_rng(13)
    ctx = [100, 200, 64]
    cache, q, tables = attn_case(rng, ctx, 8, 2, 64, 16, torch.bfloat16, CODES[codes])
    want = quant_attn_want(*cache, q, tables, ctx)
    for side in (2, 3):
        c = [x.clone() for x in cache]
        c[side][tables[1][5], 1] = float("nan")
        out, lse = run_attn(c, q, tables, ctx)
        assert out[1, 4:].isnan().all()
        assert lse[1, 4:].isnan().all() if side == 2 else not lse.isnan().any()
        out[1, 4:], lse[1, 4:] = torch.from_numpy(want[0][1, 4:]), torch.from_numpy(want[1][1, 4:])
        check_attn(out, lse, want)


def test_attn_lengths_and_ids_out_of_range():
    rng = np.random.default_rng(13)
    cache, q, tables = attn_case(rng, [64, 64, 64], 8, 2, 64, 16, torch.bfloat16, torch.int8)
    out, lse = run_attn(cache, q, tables, [-5, 64, 1000], want_status=5)
    check_attn(out, lse, quant_attn_want(*cache, q, tables, [0, 64, 64]))
    tables[0][1], tables[1][3], tables[2] = -1, len(cache[0]), [1 << 30, -(1 << 31), 99999, -2]
    out, lse = run_attn(cache, q, tables, [64, 64, 64], want_status=2)
    check_attn(out, lse, quant_attn_want(*cache, q, tables, [64, 64, 64]))
    assert not out[2].any() and torch.isneginf(lse[2]).all()


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
def test_attn_queries_and_scales_of_any_size(codes):
    """Heads whose queries differ by up to 2^40, flat and peaked softmax, key scales from 2^-20 to 2^20."""
    rng = np.random.default_rng(14)
    ctx = [500, 37, 2000]
    for f, up in ((0.0, 1.0), (30.0, 1.0), (2.0 ** -30, 2.0 ** 20), (2.0 ** 60, 2.0 ** -60), (2.0 ** -90, 2.0 ** 90)):
        cache, q, tables = attn_case(rng, ctx, 8, 2, 64, 16, torch.bfloat16, CODES[codes])
        q = (q * f * torch.exp2(torch.arange(8, device="cuda") * (-5.0 if up != 1.0 else 0.0))[None, :, None]).bfloat16()
        cache[2] *= up
        check_attn(*run_attn(cache, q, tables, ctx), quant_attn_want(*cache, q, tables, ctx))


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
def test_attn_value_scales_that_differ(codes):
    """Value scales that rise and fall from block to block by up to 2^16, and are all tiny or all huge."""
    rng = np.random.default_rng(15)
    ctx = [900, 40, 3000, 17]
    for dt in DTYPES.values():
        for spread, up in ((8.0, 1.0), (0.0, 2.0 ** -90), (0.0, 2.0 ** 100), (0.0, 0.0)):
            if dt == torch.float16 and up not in (0.0, 1.0):
                continue                   # values that fp16 cannot hold
            cache, q, tables = attn_case(rng, ctx, 8, 2, 64, 16, dt, CODES[codes])
            cache[3] = (torch.exp2((torch.rand(cache[3].shape, device="cuda", generator=gen(5)) * 2 - 1) * spread) * up / 100.0).float()
            check_attn(*run_attn(cache, q, tables, ctx), quant_attn_want(*cache, q, tables, ctx))


def test_attn_small_weights():
    """4000 tokens whose weights are below fp16's smallest number next to one of weight 1: together they count."""
    D, n = 64, 4001
    kp = torch.zeros((n, 1, 1, D), device="cuda", dtype=torch.int8)
    vp = torch.full((n, 1, 1, D), 100, device="cuda", dtype=torch.int8)
    q = torch.zeros((1, 1, D), device="cuda", dtype=torch.float16)
    q[0, 0, 0], kp[0, 0, 0, 0], vp[0] = 1.0, 18, 0
    ks, vs = torch.ones((n, 1), device="cuda"), torch.full((n, 1), 10.0, device="cuda")
    cache = kp, vp, ks, vs
    check_attn(*run_attn(cache, q, [list(range(n))], [n], scale=1.0), quant_attn_want(*cache, q, [list(range(n))], [n], scale=1.0))


def test_attn_shared_blocks_more_table_rows_and_no_rows():
    rng = np.random.default_rng(15)
    cache, q, tables = attn_case(rng, [200, 200, 200], 8, 2, 128, 16, torch.float16, torch.float8_e4m3fn)
    tables = [tables[0], tables[0][:6] + tables[2], tables[1]]
    t = tables_tensor(tables + [[0]] * 4, 20, fill=-3)
    out, lse = run_attn(cache, q, t, [200, 200, 111])
    check_attn(out, lse, quant_attn_want(*cache, q, tables, [200, 200, 111]))
    run_attn(cache, q[:0], t, [])


def test_attn_own_workspace_and_its_refusal():
    rng = np.random.default_rng(16)
    ctx = [3000, 20]
    cache, q, tables = attn_case(rng, ctx, 8, 2, 128, 16, torch.bfloat16, torch.int8)
    n = B.ps_quant_attn_workspace(2, 8, 128)
    want = quant_attn_want(*cache, q, tables, ctx)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")   # NaN patterns: contents do not matter
    for _ in range(2):
        check_attn(*run_attn(cache, q, tables, ctx, workspace=ws), want)
    rc, text = B.ps_quant_attn(*cache, q, torch.empty_like(q), tables_tensor(tables, 200), dev(ctx), workspace=ws[:-256])
    assert rc == B.PS_ERR_INVALID and "workspace" in text


def test_attn_calls_on_several_streams_at_once():
    rng = np.random.default_rng(22)
    cases = []
    for i in range(4):
        ctx = rng.integers(1, 6000, 6).tolist()
        cache, q, tables = attn_case(rng, ctx, 8, 2, 128, 16, torch.bfloat16, (torch.int8, torch.float8_e4m3fn)[i % 2])
        cases.append((cache, q, tables_tensor(tables, 400), dev(ctx), torch.zeros_like(q), torch.zeros((6, 8), device="cuda"), torch.cuda.Stream(),
                      quant_attn_want(*cache, q, tables, ctx)))
    torch.cuda.synchronize()
    for _ in range(10):
        for cache, q, t, n, out, lse, s, _ in cases:
            with torch.cuda.stream(s):
                out.fill_(9.0)
                assert B.ps_quant_attn(*cache, q, out, t, n, lse=lse)[0] == B.PS_OK
    torch.cuda.synchronize()
    for *_, out, lse, s, want in cases:
        check_attn(out, lse, want)


def test_tensors_that_do_not_fit_are_refused():
    bf, f8 = torch.bfloat16, torch.float8_e4m3fn
    pool = torch.zeros((8, 16, 2, 64), device="cuda", dtype=torch.int8)
    s, rows = torch.zeros((8, 2), device="cuda"), torch.zeros((3, 2, 64), device="cuda", dtype=bf)
    sl, t, n = dev([0, 1, 2], I64), torch.zeros((3, 4), device="cuda", dtype=I32), dev([1, 1, 1])
    q = torch.zeros((3, 8, 64), device="cuda", dtype=bf)
    cache = dict(kpool=pool, vpool=pool.clone(), k_scale=s, v_scale=s.clone())
    common = [dict(vpool=pool.view(f8)), dict(vpool=pool[:4]), dict(kpool=pool.transpose(1, 2)), dict(kpool=pool.view(torch.uint8)),
              dict(k_scale=s.double()), dict(k_scale=s[:7]), dict(v_scale=s.cpu()), dict(v_scale=torch.zeros((2, 8), device="cuda").T), dict(kpool=pool.cpu()),
              dict(k_scale=None), dict(vpool=None), dict(kpool=3), dict(vpool=pool.to(bf))]
    good = dict(cache, k=rows, v=rows.clone(), slots=sl)
    assert B.ps_quant_append(**good)[0] == B.PS_OK
    for bad in common + [dict(slots=sl[:2]), dict(slots=sl.int()), dict(slots=None), dict(k=rows[:2]), dict(k=rows.float()), dict(v=rows.half()),
                         dict(k=None), dict(v=torch.zeros((3, 2, 128), device="cuda", dtype=bf)[..., ::2]), dict(v_scale=s), dict(vpool=pool)]:
        rc, text = B.ps_quant_append(**{**good, **bad})
        assert rc == B.PS_ERR_INVALID and text, bad.keys()
    good = dict(cache, slots=sl, k_out=rows, v_out=rows.clone())
    assert B.ps_quant_read(**good)[0] == B.PS_OK
    for bad in common + [dict(slots=sl[:2]), dict(slots=n), dict(k_out=rows[:1].expand(3, 2, 64)), dict(v_out=rows), dict(k_out=None, v_out=None),
                         dict(v_out=rows.half()), dict(k_out=rows.cpu())]:
        rc, text = B.ps_quant_read(**{**good, **bad})
        assert rc == B.PS_ERR_INVALID and text, bad.keys()
    good = dict(cache, q=q, out=torch.zeros_like(q), block_tables=t, ctx_lens=n)
    assert B.ps_quant_attn(**good)[0] == B.PS_OK
    for bad in common + [dict(q=q.float()), dict(q=q[:, :, ::2]), dict(q=torch.zeros((3, 8, 128), device="cuda", dtype=bf)), dict(out=q[:1].expand(3, 8, 64)),
                         dict(block_tables=t.long()), dict(block_tables=t[:2]), dict(ctx_lens=n[:2]), dict(scale=0.0), dict(window=-1), dict(window=1 << 40),
                         dict(q=torch.zeros((3, 7, 64), device="cuda", dtype=bf)), dict(lse=torch.zeros((2, 8), device="cuda")), dict(out=None)]:
        rc, text = B.ps_quant_attn(**{**good, **bad})
        assert rc == B.PS_ERR_INVALID and text, bad.keys()
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------- as a step

class QuantEngine(Engine):
    """A decode step of one layer over a cache of 8 bits, with a model of it on the host."""

    def __init__(self, *args, codes):
        super().__init__(*args)
        ct = CODES[codes]
        shape = tuple(self.kpool.shape)
        self.cache = [torch.zeros(shape, device="cuda", dtype=torch.uint8).view(ct) for _ in range(2)]
        self.cache += [torch.full((shape[0], shape[2]), float("nan"), device="cuda") for _ in range(2)]      # whatever was there
        self.k_rot = torch.zeros((self.room, self.hkv, self.D), device="cuda", dtype=self.qkv.dtype)
        self.models = [CacheModel(self.cache[i], self.cache[2 + i]) for i in range(2)]
        self.back = torch.zeros_like(self.k_rot), torch.zeros_like(self.k_rot)

    def enqueue(self):
        q, k, v = self.parts()
        assert B.ps_build_slots(self.ctx, self.new, self.tables, self.slots, self.pos, self.start, self.ctx, block_size=self.S,
                                num_gpu_blocks=self.M, free_ids=self.ids, free_count=self.count, free_count_out=self.count,
                                status_word=self.status) == (B.PS_OK, "")
        assert B.ps_rope_append(q, k, self.q_rot, self.k_rot, self.pos, self.inv, slots=self.slots, status_word=self.status) == (B.PS_OK, "")
        assert B.ps_quant_append(self.k_rot, v, *self.cache, self.slots, status_word=self.status) == (B.PS_OK, "")
        torch.index_select(self.q_rot, 0, (self.start[1:] - 1).clamp(min=0).long(), out=self.q_last)   # a row's last token
        assert B.ps_quant_attn(*self.cache, self.q_last, self.out, self.tables, self.ctx, lse=self.lse, status_word=self.status) == (B.PS_OK, "")
        assert B.ps_quant_read(*self.cache, self.slots, *self.back, status_word=self.status) == (B.PS_OK, "")

    def check(self, new, qkv):
        st, self.m_tables, slots, pos, start, self.m_ctx = self.model.step(self.m_ctx, new, self.m_tables, self.stride, self.room)
        torch.cuda.synchronize()
        assert st == 0 and self.status.item() == 0
        assert self.tables.tolist() == self.m_tables and self.ctx.tolist() == self.m_ctx and self.slots.tolist() == slots
        q, k, v = self.parts()
        n = start[-1]
        wk, tk = rope_want(k, self.pos, self.inv, [0] * (self.D // 2), False, False)
        check_within(self.k_rot[:n], wk[:n], tk[:n])
        for m, rows in zip(self.models, (self.k_rot, v)):
            m.append(rows[:n], slots[:n])
        for i in range(2):
            np.testing.assert_array_equal(self.cache[2 + i].cpu().numpy(), self.models[i].scale)
            assert np.array_equal(self.cache[i].float().cpu().numpy(), self.models[i].code)
            assert torch.equal(self.back[i][:n], read_want(self.cache[i], self.cache[2 + i], slots[:n], self.back[i].dtype))
        tables = [t[: -(-c // self.S)] for t, c in zip(self.m_tables, self.m_ctx)]
        check_attn(self.out, self.lse, quant_attn_want(*self.cache, self.q_last, tables, self.m_ctx))


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
def test_a_decode_step_over_a_cache_of_8_bits(codes):
    rng = np.random.default_rng(20)
    e = QuantEngine(rng, 9, 8, 2, 64, 4, 200, 20, 120, torch.bfloat16, codes=codes)
    for _, new, qkv in engine_steps(rng, e, 8):
        e.new.copy_(dev(new))
        e.qkv.copy_(qkv)
        e.enqueue()
        e.check(new, qkv)


def test_captured_steps_replayed_with_other_lengths():
    """Two engines' steps in two graphs, replayed on two streams at once."""
    rng = np.random.default_rng(21)
    engines = [QuantEngine(rng, 9, 8, 2, 64, 4, 200, 20, 120, torch.bfloat16, codes="int8"),
               QuantEngine(rng, 5, 4, 4, 128, 16, 64, 8, 70, torch.float16, codes="e4m3")]
    streams = [torch.cuda.Stream() for _ in engines]
    graphs = []
    for e, s in zip(engines, streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            e.enqueue()                                # with all lengths zero: changes nothing
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            e.enqueue()
        graphs.append(g)
    steps = [engine_steps(rng, e, 6) for e in engines]
    for (_, new_a, qkv_a), (_, new_b, qkv_b) in zip(*steps):
        for e, new, qkv in ((engines[0], new_a, qkv_a), (engines[1], new_b, qkv_b)):
            e.new.copy_(dev(new))
            e.qkv.copy_(qkv)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        engines[0].check(new_a, qkv_a)
        engines[1].check(new_b, qkv_b)


def test_a_context_moves_blocks_of_8_bits_with_their_scales():
    """Codes and scales of a block in one range of bytes: the context offloads and reloads them, and the reloaded request is
    appended to, attended and read back."""
    rng = np.random.default_rng(24)
    L, H, hq, D, S, nb = 2, 4, 8, 128, 16, 300
    n = S * H * D
    unit = 64 * 2                                                   # bytes of a token of one head of 64
    per = -(-(n + 4 * H) // unit)                                   # tokens of a block, to the context
    bufs = [[torch.zeros((nb, per, 1, 64), device="cuda", dtype=torch.bfloat16) for _ in range(L)] for _ in range(2)]

    def views(buf):
        raw = buf.view(nb, per * 64)
        return (raw.view(torch.int8)[:, :n].view(nb, S, H, D), raw.view(torch.float32)[:, n // 4: n // 4 + H])

    lib = B.KVSwap(num_layers=L, num_kv_heads=1, num_q_heads=1, head_dim=64, block_size=per, num_gpu_blocks=nb, max_blocks_per_req=100,
                   host_pool_bytes=64 << 20, initial_free_order=rng.permutation(nb), k_pools=bufs[0], v_pools=bufs[1])
    ctx = [1000, 40, 300]
    for r, c in enumerate(ctx):
        assert lib.kv_alloc(r, -(-(c + 1) // S) * per) == B.PS_OK   # blocks, with room for the token to come
    ids = [lib.block_table(r)[0] for r in range(3)]
    rows = [kv_rows(sum(ctx), H, D, torch.bfloat16, 40 + l) for l in range(L)]
    slots = [ids[r][p // S] * S + p % S for r in range(3) for p in range(ctx[r])]
    caches, models = [], []
    for l in range(L):
        (kp, ks), (vp, vs) = views(bufs[0][l]), views(bufs[1][l])
        caches.append((kp, vp, ks, vs))
        assert B.ps_quant_append(*rows[l], *caches[l], dev(slots, I64)) == (B.PS_OK, "")
    old = torch.tensor(ids[0], device="cuda")
    was = [[bits(c[i])[old].clone() for i in range(2)] + [c[2 + i][old].clone() for i in range(2)] for c in caches]
    assert lib.swap_out(0) == B.PS_OK and lib.sync() == B.PS_OK
    for side in bufs:
        for b in side:
            b[old] = 7.0
    assert lib.swap_in_begin(0) == B.PS_OK
    rc, _, _ = lib.step(None, None, [], -1)
    assert rc == B.PS_OK and lib.reload_fence(-1) == B.PS_OK
    ids = [lib.block_table(r)[0] for r in range(3)]
    new = torch.tensor(ids[0], device="cuda")
    for l in range(L):
        models.append([CacheModel(caches[l][i], caches[l][2 + i]) for i in range(2)])
        for i in range(2):
            assert torch.equal(bits(caches[l][i])[new], was[l][i]) and torch.equal(caches[l][2 + i][new], was[l][2 + i])
    slots = [ids[r][ctx[r] // S] * S + ctx[r] % S for r in range(3)]
    for l in range(L):
        k, v = kv_rows(3, H, D, torch.bfloat16, 60 + l)
        assert B.ps_quant_append(k, v, *caches[l], dev(slots, I64)) == (B.PS_OK, "")
        q = torch.randn((3, hq, D), device="cuda").bfloat16()
        out, lse = torch.empty_like(q), torch.empty((3, hq), device="cuda")
        assert B.ps_quant_attn(*caches[l], q, out, tables_tensor(ids, 100), dev([c + 1 for c in ctx]), lse=lse) == (B.PS_OK, "")
        torch.cuda.synchronize()
        for i, x in enumerate((k, v)):
            models[l][i].append(x, slots)
            models[l][i].check(caches[l][i], caches[l][2 + i])
        check_attn(out, lse, quant_attn_want(*caches[l], q, ids, [c + 1 for c in ctx]))
    assert lib.sync() == B.PS_OK, lib.last_error()
    lib.destroy()


# Blocks of more than a warp's registers hold: 4 times 32 vectors of 16 values, 8 of 8 or of one
@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("H,D,S,rows", [
    (8, 128, 32, [(5, 90), (31, 2), (0, 32)]), (3, 128, 64, [(0, 640), (63, 2), (17, 100), (0, 3)]),
    (2, 80, 128, [(100, 300), (0, 128), (127, 1)]), (1, 64, 256, [(0, 256), (1, 600), (200, 60), (255, 1)]),
    (5, 128, 256, [(i % 256, 1) for i in range(0, 900, 7)]), (1, 128, 1024, [(3, 2500), (0, 1024), (1000, 30)]),
    (8, 128, 64, [(i, 1 + i % 21) for i in range(50)]), (16, 128, 64, [(0, 3001)]), (7, 72, 100, [(0, 255), (99, 257), (50, 20)]),
    (3, 7, 300, [(2, 700), (0, 40)]), (1, 512, 40, [(39, 90), (0, 7)]), (2, 500, 30, [(29, 90), (0, 70)])])
def test_append_in_large_blocks(codes, H, D, S, rows):
    """A row's tokens of a block are dealt to several warps, begin and end anywhere among the 256 that a CTA looks up, and go on
    behind them; between rows stands padding, a slot behind the pool among it."""
    rng = np.random.default_rng(H + D + S)
    nb = sum(-(-(f + n) // S) for f, n in rows) + 3
    order, slots = rng.permutation(nb).tolist(), []
    for i, (first, n) in enumerate(rows):
        ids = [order.pop() for _ in range(-(-(first + n) // S))]
        slots += [ids[p // S] * S + p % S for p in range(first, first + n)] + ([-1, nb * S] if i % 3 == 1 else [])
    (kp, ks), (vp, vs) = (make_cache((nb, S, H, D), CODES[codes], gen(D + i), spread=3.0) for i in range(2))
    mk, mv = CacheModel(kp, ks), CacheModel(vp, vs)
    for step in range(3):                  # larger, then smaller values
        k, v = kv_rows(len(slots), H, D, (torch.bfloat16, torch.float16)[step % 2], step + D)
        k, v = (x * (1.0, 4.0, 0.25)[step] for x in (k, v))
        append(k, v, (kp, vp, ks, vs), slots, want_status=int(nb * S in slots))
        mk.append(k, slots)
        mv.append(v, slots)
        mk.check(kp, ks)
        mv.check(vp, vs)


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("H,D,S,B_", [(8, 128, 256, 5), (8, 128, 256, 64), (3, 80, 64, 300), (2, 72, 200, 40), (1, 7, 90, 33), (8, 128, 16, 400)])
def test_append_of_single_tokens_that_raise_the_scales_of_blocks_in_use(codes, H, D, S, B_):
    rng = np.random.default_rng(S + B_)
    nb = B_ + 2
    (kp, ks), (vp, vs) = (make_cache((nb, S, H, D), CODES[codes], gen(D + i)) for i in range(2))
    ks *= 1e-3
    vs[::2] *= 1e-3                        # some grow, some do not
    mk, mv = CacheModel(kp, ks), CacheModel(vp, vs)
    ids = rng.permutation(nb)[:B_]
    for step in range(2):
        slots = [int(i) * S + int(p) for i, p in zip(ids, rng.integers(1, S, B_))]
        k, v = (x * (1 + step) for x in kv_rows(B_, H, D, torch.bfloat16, 9 + step))
        append(k, v, (kp, vp, ks, vs), slots)
        mk.append(k, slots)
        mv.append(v, slots)
        mk.check(kp, ks)
        mv.check(vp, vs)
