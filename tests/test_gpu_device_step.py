"""ps_build_slots, ps_rope_append and ps_paged_attn against plain 64-bit models, alone and as one decode step."""
import numpy as np
import pytest
import torch

from device_step_util import (DTYPES, HALF_STEP, SlotModel, attn_want, check_attn, check_within, make_tables, rope_want, tables_tensor)
from paper_2512_12928_b200 import binding as B

pytestmark = pytest.mark.gpu

I32 = torch.int32


def dev(v, dtype=I32):
    return torch.tensor(v, dtype=dtype, device="cuda")


# ------------------------------------------------------------------------------------------------ slots

class SlotCase:
    """Device state of ps_build_slots next to the model, compared after every call."""

    def __init__(self, S, M, free, ctx, tables, stride, room, pool=True, in_place=True):
        self.S, self.M, self.stride, self.room, self.pool = S, M, stride, room, pool
        self.model = SlotModel(S, M, free)
        self.ctx = list(ctx)
        self.tables = [list(t) + [-7] * (stride - len(t)) for t in tables]
        self.d_ctx = dev(self.ctx)
        self.d_tables = dev(self.tables).view(len(ctx), stride)
        self.d_ids = dev(list(free) + [-9] * (M - len(free)))
        self.d_count = dev([len(free)])
        self.d_ctx_out = self.d_ctx if in_place else torch.full_like(self.d_ctx, 77)
        self.d_count_out = self.d_count if in_place else torch.full_like(self.d_count, 77)

    def step(self, new, want_status=0):
        n = max(self.room, 1)
        slots = torch.full((n,), 55, dtype=torch.int64, device="cuda")
        pos = torch.full((n,), 55, dtype=I32, device="cuda")
        start = torch.full((len(new) + 1,), 55, dtype=I32, device="cuda")
        status = dev([0])
        kw = dict(free_ids=self.d_ids, free_count=self.d_count, free_count_out=self.d_count_out) if self.pool else {}
        rc, text = B.ps_build_slots(self.d_ctx, dev(new), self.d_tables, slots[: self.room], pos[: self.room], start,
                                    self.d_ctx_out, block_size=self.S, num_gpu_blocks=self.M, status_word=status, **kw)
        assert rc == B.PS_OK, text
        st, tables, w_slots, w_pos, w_start, ctx = self.model.step(self.ctx, new, self.tables, self.stride, self.room, self.pool)
        torch.cuda.synchronize()
        assert status.item() == st == want_status
        assert self.d_tables.tolist() == tables
        assert slots[: self.room].tolist() == w_slots and pos[: self.room].tolist() == w_pos
        assert slots[self.room:].tolist() == [55] * (n - self.room)
        assert start.tolist() == w_start and self.d_ctx_out.tolist() == ctx
        if self.pool:
            assert self.d_count_out.item() == len(self.model.free)
            assert self.d_ids[: len(self.model.free)].tolist() == self.model.free
        self.tables, self.ctx = tables, ctx
        if self.d_ctx_out is not self.d_ctx:
            self.d_ctx.copy_(self.d_ctx_out)
            self.d_count.copy_(self.d_count_out)


def slot_case(rng, rows, S, hi, stride, M, room, **kw):
    ctx = rng.integers(0, hi + 1, rows).tolist()
    order = rng.permutation(M).tolist()
    tables = [[order.pop() for _ in range(-(-n // S))] for n in ctx]
    return SlotCase(S, M, order, ctx, tables, stride, room, **kw)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("rows,S,room", [(1, 16, 64), (1, 1, 64), (7, 16, 300), (33, 24, 5000), (300, 16, 4096), (257, 7, 6000),
                                         (1024, 16, 4097), (2500, 8, 20000),
                                         (4000, 16, 9000), (5000, 8, 6000)])
def test_slots_over_steps_with_a_stack(rows, S, room, in_place):
    rng = np.random.default_rng(rows * 100 + S)
    hi, chunk = 60, min(40, room // (rows + 1) + 1)
    stride = -(-hi * 8 // S) + 2
    c = slot_case(rng, rows, S, hi, stride, rows * stride, room, in_place=in_place)
    for step in range(4):
        new = rng.integers(0, chunk + 1, rows) if step % 2 else np.ones(rows, int)
        new[rng.random(rows) < 0.15] = -1
        new[rng.random(rows) < 0.1] = 0
        while np.maximum(new, 0).sum() > room:
            new //= 2
        c.step(new.tolist())


def test_slots_of_one_long_prompt_and_of_none():
    rng = np.random.default_rng(5)
    c = slot_case(rng, 3, 16, 40, 2100, 7000, 33000)
    c.step([32768, 0, 1])
    c.step([0, 0, 0])
    c.step([-1, 31999, -1])
    c.step([-1, -1, -1])
    c.step([1, 1, 1])


def test_slots_without_rows_or_room():
    for room in (0, 3, 5000):
        c = SlotCase(16, 4, [0, 1, 2, 3], [], [], 1, room)
        c.d_tables = torch.zeros((0, 1), dtype=I32, device="cuda")
        c.d_ctx = c.d_ctx_out = torch.zeros(0, dtype=I32, device="cuda")
        start = dev([9])
        slots = torch.full((room,), 5, dtype=torch.int64, device="cuda")
        rc, text = B.ps_build_slots(c.d_ctx, c.d_ctx, c.d_tables, slots, None, start, c.d_ctx, block_size=16, num_gpu_blocks=4,
                                    free_ids=c.d_ids, free_count=c.d_count, free_count_out=c.d_count)
        assert rc == B.PS_OK, text
        assert start.item() == 0 and slots.tolist() == [-1] * room and c.d_count.item() == 4
    c = SlotCase(16, 4, [2, 3], [16, 3], [[0], [1]], 2, 0)
    c.step([0, -1])


def test_slots_all_or_nothing():
    rng = np.random.default_rng(6)
    for room in (50, 5000):
        c = slot_case(rng, 5, 4, 20, 12, 40, room)
        free = len(c.model.free)
        c.step([30, 30, 30, 30, 30], want_status=5 if max(c.ctx) + 30 > 48 or room == 50 else 4)
        c.step([0, 0, 49, 0, 0], want_status=5)        # more than the table holds
        c.step([0, 0, -2, 0, 0], want_status=5)
        assert len(c.model.free) == free
        c.step([1, 1, 1, 1, 1])
    c = SlotCase(4, 8, [5], [4, 4], [[0], [1]], 8, 64)
    c.step([5, 4], want_status=4)                       # three blocks, one free
    c.step([5, -1])                                     # the second row's block makes it two
    assert c.tables[0][:3] == [0, 1, 5]
    c = SlotCase(4, 4, [3, 2, 1], [8, 0], [[0, 1], []], 4, 64)
    c.step([-1, 0], want_status=5)                      # more ids than the pool has: the stack would overflow
    c = SlotCase(4, 4, [3], [-1, 4], [[], [0]], 4, 64)
    c.step([1, 1], want_status=5)


def test_slots_of_tables_that_hold_the_blocks():
    rng = np.random.default_rng(7)
    for rows, room in ((6, 100), (6, 5000)):
        S, stride, M = 16, 6, 64
        tables = [rng.permutation(M)[:stride].tolist() for _ in range(rows)]
        c = SlotCase(S, M, [], [0, 1, 15, 16, 17, 50], tables, stride, room, pool=False)
        c.step([3, 15, 1, 16, 0, 1])
        c.step([1, 1, 1, 1, -1, 1])
        c.step([1, 1, 200, 1, 1, 1], want_status=5)
        tables[0][0], tables[1][2] = -1, M              # ids outside the pool
        c = SlotCase(S, M, [], [0, 30, 0, 0, 0, 0], tables, stride, room, pool=False)
        c.step([20, 4, 1, 1, 1, 1], want_status=2)


def test_slots_are_what_the_host_calls_give():
    """The same free order, endings and growth through ps_kv_free and ps_kv_alloc on a bookkeeping context."""
    rng = np.random.default_rng(8)
    S, M, rows, stride = 16, 400, 24, 40
    order = rng.permutation(M).tolist()
    host = B.KVSwap(num_layers=1, num_kv_heads=8, num_q_heads=8, head_dim=64, block_size=S, num_gpu_blocks=M,
                    max_blocks_per_req=stride, initial_free_order=order, flags=B.PS_FLAG_BOOKKEEPING_ONLY)
    # the host hands out order[0] first: its top
    c = SlotCase(S, M, order[::-1], [0] * rows, [[] for _ in range(rows)], stride, 2000)
    for step in range(12):
        new = rng.integers(0, 50, rows)
        new[rng.random(rows) < 0.3] = -1
        new[[x + max(n, 0) > stride * S for x, n in zip(c.ctx, new)]] = -1
        for b in range(rows):
            if new[b] == -1 and c.ctx[b] > 0:
                assert host.kv_free(b) == B.PS_OK
        before = list(c.ctx)
        c.step(new.tolist())
        for b in range(rows):
            if new[b] >= 0 and before[b] + new[b] > 0:
                assert host.kv_alloc(b, before[b] + int(new[b])) == B.PS_OK
        for b in range(rows):
            if c.ctx[b]:
                assert host.block_table(b)[0] == c.tables[b][: -(-c.ctx[b] // S)]
        assert host.num_free_blocks() == c.d_count.item()


# ------------------------------------------------------------------------------------------------- rope

def rope_inputs(T, hq, hkv, D, dt, rng_seed, fused=True):
    g = torch.Generator(device="cuda").manual_seed(rng_seed)
    n = hq + 2 * hkv
    if fused:
        x = torch.randn((T, n * D), device="cuda", generator=g).to(dt)
        return x[:, : hq * D].view(T, hq, D), x[:, hq * D: (hq + hkv) * D].view(T, hkv, D), x[:, (hq + hkv) * D:].view(T, hkv, D)
    return tuple(torch.randn((T, h, D), device="cuda", generator=g).to(dt) for h in (hq, hkv, hkv))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T,hq,hkv,D,rot,axes,neighbours,S", [
    (1, 32, 8, 128, 128, 1, False, 16), (5, 28, 4, 128, 64, 3, False, 24), (77, 4, 2, 64, 64, 2, True, 1), (3, 3, 1, 80, 48, 3, True, 8),
    (9, 2, 2, 96, 24, 1, False, 16), (13, 5, 5, 80, 20, 4, True, 7), (6, 4, 1, 256, 256, 3, False, 32), (4, 1, 1, 512, 512, 8, False, 16),
    (2, 3, 3, 10, 6, 2, False, 5), (1030, 8, 2, 64, 32, 3, False, 16), (11, 7, 1, 128, 0, 1, False, 16), (8, 2, 1, 6, 2, 1, True, 3),
    (4700, 2, 1, 64, 32, 3, False, 16), (9001, 3, 1, 64, 64, 1, True, 7), (2500, 2, 2, 128, 64, 2, False, 64), (4730, 1, 1, 512, 16, 1, False, 16)])
def test_rope_and_append(dtype, T, hq, hkv, D, rot, axes, neighbours, S):
    dt = DTYPES[dtype]
    rng = np.random.default_rng(T * 1000 + D)
    q, k, v = rope_inputs(T, hq, hkv, D, dt, T + D)
    pos = torch.from_numpy(rng.integers(-50, 1 << 20, (axes, T)).astype(np.int32)).cuda()
    half = rot // 2
    inv = torch.from_numpy((10000.0 ** (-np.arange(half) / max(half, 1))).astype(np.float32)).cuda()
    axis = rng.integers(0, axes, half).tolist()
    nb = T // S + 9
    slots = rng.permutation(nb * S)[:T]
    slots[rng.random(T) < 0.2] = -1 if T > 1 else 0
    kpool = torch.randn((nb, S, hkv, D), device="cuda").to(dt)
    vpool = torch.randn((nb, S, hkv, D), device="cuda").to(dt)
    for inverse in (False, True):
        kp, vp = kpool.clone(), vpool.clone()
        q_out = torch.full((T, hq, D), 3.0, device="cuda", dtype=dt)
        k_out = torch.full((T, hkv, D), 3.0, device="cuda", dtype=dt) if inverse else None
        status = dev([0])
        rc, text = B.ps_rope_append(q, k, q_out, k_out, pos if rot else None, inv if rot else None, v=v, kpool=kp, vpool=vp,
                                    slots=dev(slots.tolist(), torch.int64), freq_axis=axis if rot else None, neighbours=neighbours,
                                    inverse=inverse, status_word=status)
        assert rc == B.PS_OK, text
        torch.cuda.synchronize()
        assert status.item() == 0
        live = torch.from_numpy(slots >= 0).cuda()
        at = dev(slots[slots >= 0].tolist(), torch.int64)
        wq, tq = rope_want(q, pos, inv, axis, neighbours, inverse)
        wk, tk = rope_want(k, pos, inv, axis, neighbours, inverse)
        ln = live.cpu().numpy()
        check_within(q_out[live], wq[ln], tq[ln])
        assert (q_out[~live] == 3.0).all()               # padding is left as it was
        check_within(kp.view(-1, hkv, D)[at], wk[ln], tk[ln])
        assert torch.equal(vp.view(-1, hkv, D)[at], v[live])
        if k_out is not None:
            assert torch.equal(k_out[live], kp.view(-1, hkv, D)[at]) and (k_out[~live] == 3.0).all()
        rest = torch.ones(nb * S, dtype=torch.bool, device="cuda")
        rest[at] = False
        for now, was in ((kp, kpool), (vp, vpool)):      # foreign rows too
            assert torch.equal(now.view(-1, hkv, D)[rest], was.view(-1, hkv, D)[rest])


@pytest.mark.parametrize("D,rot,neighbours", [
    (512, 4, True), (512, 2, True), (512, 4, False), (512, 504, False), (510, 510, True), (80, 40, False), (80, 20, False), (96, 24, False),
    (64, 64, True), (64, 64, False), (12, 12, True), (20, 8, False), (34, 18, False), (7, 4, True)])
@pytest.mark.parametrize("T", [6, 2600])
def test_rope_rows_of_every_alignment(T, D, rot, neighbours):
    """How wide the accesses are follows from addresses, strides and sizes; what comes out does not."""
    hq, hkv, S = 3, 2, 4
    nb = T // S + 3
    q, k, v = rope_inputs(T, hq, hkv, D, torch.bfloat16, D + T, fused=False)
    pos = torch.arange(T, device="cuda", dtype=torch.int32) * 7
    inv = torch.rand(rot // 2, device="cuda")
    axis = [0] * (rot // 2)
    slots = torch.randperm(nb * S, device="cuda")[:T]
    (wq, tq), (wk, tk) = rope_want(q, pos[None], inv, axis, neighbours, False), rope_want(k, pos[None], inv, axis, neighbours, False)
    n = hq + 2 * hkv
    first = None
    for shift, gap in ((0, 0), (1, 0), (2, 0), (4, 8), (0, 1), (0, 2), (8, 4)):
        x = torch.full((T * (n * D + gap) + shift,), 5.0, device="cuda", dtype=torch.bfloat16)
        rows = x[shift:].view(T, n * D + gap)
        parts = [rows[:, a * D: b * D].view(T, b - a, D) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, n))]
        for dst, src in zip(parts, (q, k, v)):
            dst.copy_(src)
        kp, vp = (torch.zeros(nb * S * hkv * D + shift, device="cuda", dtype=torch.bfloat16)[shift:].view(nb, S, hkv, D) for _ in range(2))
        rc, text = B.ps_rope_append(parts[0], parts[1], parts[0], None, pos, inv, v=parts[2], kpool=kp, vpool=vp, slots=slots,
                                    neighbours=neighbours)
        assert rc == B.PS_OK, text
        got = parts[0].clone(), kp.clone(), vp.clone()
        assert torch.equal(parts[1], k) and torch.equal(parts[2], v)
        assert (rows[:, n * D:] == 5.0).all() and (x[:shift] == 5.0).all()
        if first is None:
            first = got
            check_within(got[0], wq, tq)
            check_within(kp.view(-1, hkv, D)[slots], wk, tk)
            assert torch.equal(vp.view(-1, hkv, D)[slots], v)
        assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_rope_in_place_alone_and_of_keys_alone():
    T, hq, hkv, D = 19, 6, 2, 128
    q, k, _ = rope_inputs(T, hq, hkv, D, torch.bfloat16, 1)
    pos = dev(list(range(T)))
    inv = torch.from_numpy((500000.0 ** (-np.arange(64) / 64)).astype(np.float32)).cuda()
    wq, tq = rope_want(q, pos, inv, [0] * 64, False, False)
    wk, tk = rope_want(k, pos, inv, [0] * 64, False, False)
    k_out = torch.empty((T, hkv, D), device="cuda", dtype=torch.bfloat16)
    assert B.ps_rope_append(None, k, None, k_out, pos, inv)[0] == B.PS_OK
    check_within(k_out, wk, tk)
    assert B.ps_rope_append(q, k, q, k, pos, inv)[0] == B.PS_OK      # strided, in place
    check_within(q, wq, tq)
    check_within(k, wk, tk)


def test_rope_text_uses_one_row_of_positions_for_all_axes():
    T = 6
    q, k, _ = rope_inputs(T, 4, 2, 64, torch.float16, 2)
    pos = dev([7, 0, 3, 9, 100, 5])
    inv = torch.rand(32, device="cuda")
    a, b = torch.empty((T, 4, 64), device="cuda", dtype=torch.float16), torch.empty((T, 4, 64), device="cuda", dtype=torch.float16)
    axis = [i % 3 for i in range(32)]
    assert B.ps_rope_append(q, None, a, None, pos.expand(3, T), inv, freq_axis=axis)[0] == B.PS_OK
    assert B.ps_rope_append(q, None, b, None, pos, inv)[0] == B.PS_OK
    assert torch.equal(a, b)


def test_rope_of_no_tokens():
    q, k, v = rope_inputs(0, 4, 2, 64, torch.float16, 5, fused=False)
    pool = torch.zeros((2, 16, 2, 64), device="cuda", dtype=torch.float16)
    inv, none = torch.rand(32, device="cuda"), dev([], torch.int64)
    for kw in (dict(), dict(v=v, kpool=pool, vpool=pool.clone(), slots=none)):
        assert B.ps_rope_append(q, k, torch.empty_like(q), torch.empty_like(k), dev([]), inv, **kw) == (B.PS_OK, "")
    torch.cuda.synchronize()
    assert not pool.any()


def test_rope_slots_outside_the_pool_are_reported_and_skipped():
    T, hkv, D = 4, 2, 64
    q, k, v = rope_inputs(T, 2, hkv, D, torch.bfloat16, 3)
    kp, vp = (torch.zeros((3, 4, hkv, D), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    out, status = torch.zeros((T, 2, D), device="cuda", dtype=torch.bfloat16), dev([0])
    slots = dev([11, 12, 1 << 40, 2], torch.int64)
    assert B.ps_rope_append(q, k, out, None, None, None, v=v, kpool=kp, vpool=vp, slots=slots, status_word=status)[0] == B.PS_OK
    torch.cuda.synchronize()
    assert status.item() == 1
    assert torch.equal(out, q) and torch.equal(kp.view(-1, hkv, D)[[11, 2]], k[[0, 3]]) and torch.equal(vp.view(-1, hkv, D)[[11, 2]], v[[0, 3]])
    kp.view(-1, hkv, D)[[11, 2]] = 0
    assert not kp.any()


def test_rope_gradient():
    """The inverse turn is the gradient: against the formula's transpose and against differences of the forward call."""
    T, h, D, rot = 5, 3, 64, 48
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((T, h, D), device="cuda", generator=g).half()
    dy = torch.randn((T, h, D), device="cuda", generator=g).half()
    pos = torch.randint(0, 500, (3, T), device="cuda", dtype=I32, generator=g)
    inv = torch.rand(rot // 2, device="cuda", generator=g)
    axis = sorted(i % 3 for i in range(rot // 2))
    for nbr in (False, True):
        y, dx = torch.empty_like(x), torch.empty_like(x)
        assert B.ps_rope_append(x, None, y, None, pos, inv, freq_axis=axis, neighbours=nbr)[0] == B.PS_OK
        assert B.ps_rope_append(dy, None, dx, None, pos, inv, freq_axis=axis, neighbours=nbr, inverse=True)[0] == B.PS_OK
        w, tol = rope_want(dy, pos, inv, axis, nbr, True)
        check_within(dx, w, tol)
        # the rotation is linear, so a difference quotient is exact up to the roundings: of a step along e at (t, i, d),
        # y changes by R e, and dy . R e has to be dx there.  Each of the two outputs of a pair is rounded (2^-11).
        e = torch.zeros_like(x)
        rng = np.random.default_rng(9)
        for _ in range(8):
            t, i, d = int(rng.integers(T)), int(rng.integers(h)), int(rng.integers(D))
            e.zero_()
            e[t, i, d] = 1.0
            ye = torch.empty_like(x)
            assert B.ps_rope_append(e, None, ye, None, pos, inv, freq_axis=axis, neighbours=nbr)[0] == B.PS_OK
            got = float((ye.double() * dy.double()).sum())
            room = 2.0 ** -10 * float(dy[t, i].abs().max()) * 2 + 2.0 ** -11 * abs(float(dx[t, i, d])) + 2.0 ** -16
            assert abs(got - float(dx[t, i, d])) <= room


# -------------------------------------------------------------------------------------------- attention

def attn_case(rng, ctx, hq, hkv, D, S, dt, extra=5, gap=0):
    n = [-(-c // S) for c in ctx]
    nb = sum(n) + extra
    tables = make_tables(rng, ctx, S, nb)
    g = torch.Generator(device="cuda").manual_seed(int(rng.integers(1 << 30)))
    if gap:    # K and V of a block side by side in one buffer, with a gap behind
        buf = torch.randn((nb, 2 * S * hkv * D + gap), device="cuda", generator=g).to(dt)
        kp = buf[:, : S * hkv * D].view(nb, S, hkv, D)
        vp = buf[:, S * hkv * D: 2 * S * hkv * D].view(nb, S, hkv, D)
    else:
        kp = torch.randn((nb, S, hkv, D), device="cuda", generator=g).to(dt)
        vp = torch.randn((nb, S, hkv, D), device="cuda", generator=g).to(dt)
    q = torch.randn((len(ctx), hq, D), device="cuda", generator=g).to(dt)
    return kp, vp, q, tables


def run_attn(kp, vp, q, tables, ctx, want_status=0, stride=None, **kw):
    out = torch.full(tuple(q.shape), 9.0, device="cuda", dtype=q.dtype)
    lse = torch.full(tuple(q.shape[:2]), 9.0, device="cuda")
    status = dev([0])
    t = tables if torch.is_tensor(tables) else tables_tensor(tables, stride or max(1, max((len(t) for t in tables), default=1)))
    rc, text = B.ps_paged_attn(kp, vp, q, out, t, dev(list(ctx)), lse=lse, status_word=status, **kw)
    assert rc == B.PS_OK, text
    torch.cuda.synchronize()
    assert status.item() == want_status
    return out, lse


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("hq,hkv,D,S,window", [
    (32, 8, 128, 16, 0), (64, 8, 128, 32, 0), (28, 4, 128, 24, 100), (8, 8, 64, 16, 0), (4, 2, 64, 1, 33), (16, 1, 64, 16, 0),
    (20, 1, 128, 8, 0), (64, 1, 128, 16, 700), (9, 3, 64, 100, 0), (10, 10, 128, 16, 0), (77, 11, 64, 7, 1), (34, 2, 128, 64, 0)])
def test_attn_shapes(dtype, hq, hkv, D, S, window):
    rng = np.random.default_rng(hq * 100 + S)
    ctx = [0, 1, 2, 15, 16, 17, 31, 33, 100, 128, 129, 1000, 0, 2049, 5]
    kp, vp, q, tables = attn_case(rng, ctx, hq, hkv, D, S, DTYPES[dtype])
    out, lse = run_attn(kp, vp, q, tables, ctx, window=window)
    check_attn(out, lse, attn_want(kp, vp, q, tables, ctx, window))


@pytest.mark.parametrize("rows,hi", [(1, 20000), (2, 9000), (200, 60), (600, 9), (149, 0), (3, 131072)])
def test_attn_batches(rows, hi):
    """One long row cut into many parts, many rows of a tile, many empty rows."""
    rng = np.random.default_rng(rows)
    ctx = rng.integers(0, hi + 1, rows).tolist()
    ctx[-1] = hi
    kp, vp, q, tables = attn_case(rng, ctx, 4, 2, 64, 16, torch.bfloat16)
    out, lse = run_attn(kp, vp, q, tables, ctx)
    check_attn(out, lse, attn_want(kp, vp, q, tables, ctx))
    again, lse2 = run_attn(kp, vp, q, tables, ctx)
    assert torch.equal(out, again) and torch.equal(lse, lse2)     # no order of arrival in the results


def test_attn_strided_everything():
    rng = np.random.default_rng(11)
    ctx = [50, 700, 3, 0]
    for gap in (8, 4096):
        kp, vp, _, tables = attn_case(rng, ctx, 8, 2, 128, 24, torch.bfloat16, gap=gap)
        wide = torch.randn((4, 3, 8, 128), device="cuda").bfloat16()
        q = wide[:, 1]
        res = torch.full((4, 2, 8, 128), 5.0, device="cuda", dtype=torch.bfloat16)
        lse = torch.zeros((4, 8), device="cuda")
        rc, text = B.ps_paged_attn(kp, vp, q, res[:, 0], tables_tensor(tables, 30), dev(ctx), lse=lse, scale=-0.3)
        assert rc == B.PS_OK, text
        check_attn(res[:, 0], lse, attn_want(kp, vp, q, tables, ctx, scale=-0.3))
        assert (res[:, 1] == 5.0).all()
        one = q[:1].expand(4, 8, 128)                              # one query for all rows
        out, l = run_attn(kp, vp, one, tables, ctx)
        check_attn(out, l, attn_want(kp, vp, one, tables, ctx))


def test_attn_never_reads_what_is_not_attended_into_a_result():
    rng = np.random.default_rng(12)
    for dt in DTYPES.values():
        for window in (0, 40):
            ctx = [1, 17, 100, 333, 0]
            kp, vp, q, tables = attn_case(rng, ctx, 8, 2, 128, 24, dt)
            want = attn_want(kp, vp, q, tables, ctx, window)
            seen = torch.zeros(kp.shape[:2], dtype=torch.bool, device="cuda")
            for t, n in zip(tables, ctx):
                for i in range(max(0, n - window) if window else 0, n):
                    seen[t[i // 24], i % 24] = True
            for value in (float("nan"), float("inf"), -float("inf")):
                kp[~seen] = value
                vp[~seen] = value
                check_attn(*run_attn(kp, vp, q, tables, ctx, window=window), want)


def test_attn_lengths_and_ids_out_of_range():
    rng = np.random.default_rng(13)
    kp, vp, q, tables = attn_case(rng, [64, 64, 64], 8, 2, 64, 16, torch.bfloat16)
    out, lse = run_attn(kp, vp, q, tables, [-5, 64, 1000], want_status=5)
    check_attn(out, lse, attn_want(kp, vp, q, tables, [0, 64, 64]))
    tables[0][1], tables[1][3], tables[2] = -1, kp.shape[0], [1 << 30, -(1 << 31), 99999, -2]
    out, lse = run_attn(kp, vp, q, tables, [64, 64, 64], want_status=2)
    check_attn(out, lse, attn_want(kp, vp, q, tables, [64, 64, 64]))
    assert not out[2].any() and torch.isneginf(lse[2]).all()


def test_attn_scores_of_any_size():
    """Flat and peaked softmax, scores in the hundreds and far below the lowest starting value a maximum could have."""
    rng = np.random.default_rng(14)
    ctx = [500, 37, 3000]
    for dt, factors in ((torch.bfloat16, (0.0, 1.0, 30.0)), (torch.float16, (0.0, 1.0, 30.0))):
        for f in factors:
            kp, vp, q, tables = attn_case(rng, ctx, 8, 2, 64, 16, dt)
            q = (q * f).to(dt)
            out, lse = run_attn(kp, vp, q, tables, ctx)
            check_attn(out, lse, attn_want(kp, vp, q, tables, ctx))
    kp, vp, q, tables = attn_case(rng, ctx, 8, 2, 64, 16, torch.bfloat16)
    kp.fill_(-2.0 ** 60)
    q.fill_(2.0 ** 60)                                             # every score is -2^126 * 8
    out, lse = run_attn(kp, vp, q, tables, ctx, scale=1.0 / 8)
    for b, n in enumerate(ctx):
        v = vp[torch.tensor(tables[b], device="cuda")].double().view(-1, 2, 64)[:n].mean(0)
        # equal scores: p = 1, exactly; the mean is rounded once, its sum of n values n times in 32 bits
        err = (out[b].view(2, 4, 64).double() - v[:, None]).abs()
        assert (err <= 2.0 ** -8 * v[:, None].abs() + n * 2.0 ** -22).all()


def test_attn_small_weights_in_fp16():
    """4000 tokens whose weights are below fp16's smallest number next to one of weight 1: together they count."""
    D, n = 64, 4001
    kp = torch.zeros((n, 1, 1, D), device="cuda", dtype=torch.float16)
    vp = torch.ones((n, 1, 1, D), device="cuda", dtype=torch.float16)
    q = torch.zeros((1, 1, D), device="cuda", dtype=torch.float16)
    q[0, 0, 0] = 1.0
    kp[0, 0, 0, 0] = 18.0                                          # e^-18 = 1.5e-8 for the others
    vp[0] = 0.0
    vp[1:] = 1000.0
    out, lse = run_attn(kp, vp, q, [list(range(n))], [n], scale=1.0)
    check_attn(out, lse, attn_want(kp, vp, q, [list(range(n))], [n], scale=1.0))


def test_attn_offsets_beyond_32_bits():
    """A pool of more than 2^32 elements, rows in its last blocks; and slots there through the append."""
    S, hkv, D = 16, 8, 128
    nb = (1 << 32) // (S * hkv * D) + 40
    pool = torch.empty((nb, S, hkv, D), device="cuda", dtype=torch.bfloat16)
    ids = [nb - 1, 3, nb - 17, nb - 2, (1 << 31) // (S * hkv * D)]
    pool[torch.tensor(ids, device="cuda")] = torch.randn((5, S, hkv, D), device="cuda").bfloat16()
    ctx = [77]
    q = torch.randn((1, 32, D), device="cuda").bfloat16()
    T = 3
    rows = torch.randn((T, hkv, D), device="cuda").bfloat16()
    slots = dev([(nb - 1) * S + 4, ids[4] * S + 12, 3 * S], torch.int64)
    assert B.ps_rope_append(None, rows, None, None, None, None, v=rows, kpool=pool, vpool=pool, slots=slots)[0] == B.PS_OK
    torch.cuda.synchronize()
    for t, (blk, at) in enumerate(((nb - 1, 4), (ids[4], 12), (3, 0))):
        assert torch.equal(pool[blk, at], rows[t])
    out, lse = run_attn(pool, pool, q, [ids], ctx)
    check_attn(out, lse, attn_want(pool, pool, q, [ids], ctx))


def test_attn_shared_blocks_more_table_rows_and_no_rows():
    rng = np.random.default_rng(15)
    kp, vp, q, tables = attn_case(rng, [200, 200, 200], 8, 2, 128, 16, torch.float16)
    tables = [tables[0], tables[0][:6] + tables[2], tables[1]]
    t = tables_tensor(tables + [[0]] * 4, 20, fill=-3)
    out, lse = run_attn(kp, vp, q, t, [200, 200, 111])
    check_attn(out, lse, attn_want(kp, vp, q, tables, [200, 200, 111]))
    run_attn(kp, vp, q[:0], t, [])


def test_attn_own_workspace_and_its_refusal():
    rng = np.random.default_rng(16)
    ctx = [3000, 20]
    kp, vp, q, tables = attn_case(rng, ctx, 8, 2, 128, 16, torch.bfloat16)
    n = B.ps_paged_attn_workspace(2, 8, 128)
    want = attn_want(kp, vp, q, tables, ctx)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")   # NaN patterns: contents do not matter
    for _ in range(2):
        check_attn(*run_attn(kp, vp, q, tables, ctx, workspace=ws), want)
    rc, text = B.ps_paged_attn(kp, vp, q, torch.empty_like(q), tables_tensor(tables, 200), dev(ctx), workspace=ws[:-256])
    assert rc == B.PS_ERR_INVALID and "workspace" in text
    big = torch.empty(n + 64, dtype=torch.uint8, device="cuda")
    rc, text = B.ps_paged_attn(kp, vp, q, torch.empty_like(q), tables_tensor(tables, 200), dev(ctx), workspace=big[64:])
    assert rc == B.PS_ERR_INVALID and "boundary" in text


def test_tensors_that_do_not_fit_are_refused():
    bf, h = torch.bfloat16, torch.float16
    kp = torch.zeros((8, 16, 2, 64), device="cuda", dtype=bf)
    q = torch.zeros((3, 8, 64), device="cuda", dtype=bf)
    t, n = torch.zeros((3, 4), device="cuda", dtype=I32), dev([1, 1, 1])
    good = dict(kpool=kp, vpool=kp, q=q, out=torch.zeros_like(q), block_tables=t, ctx_lens=n)
    assert B.ps_paged_attn(**good)[0] == B.PS_OK
    for bad in (dict(vpool=kp.to(h)), dict(vpool=kp[:4]), dict(kpool=kp.transpose(1, 2)), dict(q=q.float()), dict(q=q[:, :, ::2]),
                dict(out=torch.zeros((3, 8, 128), device="cuda", dtype=bf)[:, :, 1:65]), dict(out=q[:1].expand(3, 8, 64)),
                dict(block_tables=t.long()), dict(block_tables=t[:2]), dict(block_tables=t[:, :2]), dict(ctx_lens=n[:2]), dict(ctx_lens=n.cpu()),
                dict(lse=torch.zeros((3, 8), device="cuda", dtype=bf)), dict(lse=torch.zeros((2, 8), device="cuda")), dict(scale=0.0),
                dict(scale=float("nan")), dict(scale="a"), dict(window=-1), dict(window=1 << 40), dict(window=1 << 70), dict(window=None),
                dict(q=None), dict(out=None), dict(ctx_lens=None), dict(block_tables=None), dict(kpool=[1]), dict(q=torch.zeros((3, 7, 64), device="cuda", dtype=bf)),
                dict(kpool=kp.view(-1)[4:4 + 7 * 16 * 128].view(7, 16, 2, 64), vpool=kp[:7])):
        rc, text = B.ps_paged_attn(**{**good, **bad})
        assert rc == B.PS_ERR_INVALID and text, bad.keys()
    k = torch.zeros((3, 2, 64), device="cuda", dtype=bf)
    inv, pos, sl = torch.zeros(32, device="cuda"), dev([0, 0, 0]), dev([0, 1, 2], torch.int64)
    good = dict(q=q, k=k, q_out=torch.zeros_like(q), k_out=None, positions=pos, inv_freq=inv, v=k, kpool=kp, vpool=kp.clone(), slots=sl)
    assert B.ps_rope_append(**good)[0] == B.PS_OK
    for bad in (dict(q_out=None), dict(v=None), dict(slots=None), dict(slots=pos), dict(slots=sl[:2]), dict(positions=None),
                dict(positions=pos[:2]), dict(positions=pos.long()), dict(inv_freq=inv.double()), dict(inv_freq=torch.zeros(33, device="cuda")),
                dict(vpool=None), dict(kpool=None), dict(kpool=kp.to(h)), dict(k=k[:2]), dict(v=k.to(h)), dict(freq_axis=[0] * 31),
                dict(freq_axis=[1] * 32), dict(freq_axis=[-1] * 32), dict(freq_axis=[0.5] * 32), dict(freq_axis=[1 << 80] * 32), dict(freq_axis=3), dict(q_out=q[:1].expand(3, 8, 64)), dict(k=None)):
        rc, text = B.ps_rope_append(**{**good, **bad})
        assert rc == B.PS_ERR_INVALID and text, bad.keys()
    ids, cnt = dev([0] * 8), dev([8])
    good = dict(ctx_lens=n, new_lens=n, block_tables=t, slots=sl, positions=pos, token_start=dev([0] * 4), ctx_lens_out=n, block_size=16,
                num_gpu_blocks=8, free_ids=ids, free_count=cnt, free_count_out=cnt)
    assert B.ps_build_slots(**good)[0] == B.PS_OK
    for bad in (dict(new_lens=n[:2]), dict(ctx_lens=n.long()), dict(block_tables=t[:2]), dict(block_tables=t[0]), dict(slots=pos),
                dict(positions=pos[:2]), dict(token_start=n), dict(free_ids=ids[:7]), dict(free_count=None), dict(free_count_out=None),
                dict(block_size=0), dict(block_size=1 << 70), dict(block_size=1.5), dict(new_lens=None), dict(token_start=None), dict(ctx_lens_out=n.cpu()), dict(slots=sl.cpu())):
        rc, text = B.ps_build_slots(**{**good, **bad})
        assert rc == B.PS_ERR_INVALID and text, bad.keys()
    assert B.ps_build_slots(**{**good, "block_size": np.int64(16)})[0] == B.PS_OK
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------- as a step

class Engine:
    """A decode step of one layer whose lengths stay on the device, with a model of it on the host."""

    def __init__(self, rng, rows, hq, hkv, D, S, M, stride, room, dt):
        self.rows, self.hq, self.hkv, self.D, self.S, self.M, self.stride, self.room = rows, hq, hkv, D, S, M, stride, room
        free = rng.permutation(M).tolist()
        self.model = SlotModel(S, M, free)
        self.m_ctx, self.m_tables = [0] * rows, [[0] * stride for _ in range(rows)]
        self.ids, self.count = dev(free), dev([M])
        self.ctx, self.tables = dev([0] * rows), torch.zeros((rows, stride), device="cuda", dtype=I32)
        self.new = dev([0] * rows)
        self.slots = torch.zeros(room, device="cuda", dtype=torch.int64)
        self.pos = torch.zeros(room, device="cuda", dtype=I32)
        self.start = torch.zeros(rows + 1, device="cuda", dtype=I32)
        self.kpool, self.vpool = (torch.zeros((M, S, hkv, D), device="cuda", dtype=dt) for _ in range(2))
        self.qkv = torch.zeros((room, (hq + 2 * hkv) * D), device="cuda", dtype=dt)
        self.q_rot = torch.zeros((room, hq, D), device="cuda", dtype=dt)
        self.q_last = torch.zeros((rows, hq, D), device="cuda", dtype=dt)
        self.out = torch.zeros((rows, hq, D), device="cuda", dtype=dt)
        self.lse = torch.zeros((rows, hq), device="cuda")
        self.status = dev([0])
        self.inv = torch.from_numpy((10000.0 ** (-np.arange(D // 2) / (D // 2))).astype(np.float32)).cuda()
        self.m_k, self.m_v = self.kpool.clone(), self.vpool.clone()

    def parts(self):
        a, b = self.hq * self.D, (self.hq + self.hkv) * self.D
        n = self.room
        return self.qkv[:, :a].view(n, self.hq, self.D), self.qkv[:, a:b].view(n, self.hkv, self.D), self.qkv[:, b:].view(n, self.hkv, self.D)

    def enqueue(self):
        q, k, v = self.parts()
        assert B.ps_build_slots(self.ctx, self.new, self.tables, self.slots, self.pos, self.start, self.ctx, block_size=self.S,
                                num_gpu_blocks=self.M, free_ids=self.ids, free_count=self.count, free_count_out=self.count,
                                status_word=self.status) == (B.PS_OK, "")
        assert B.ps_rope_append(q, k, self.q_rot, None, self.pos, self.inv, v=v, kpool=self.kpool, vpool=self.vpool, slots=self.slots,
                                status_word=self.status) == (B.PS_OK, "")
        torch.index_select(self.q_rot, 0, (self.start[1:] - 1).clamp(min=0).long(), out=self.q_last)   # a row's last token
        assert B.ps_paged_attn(self.kpool, self.vpool, self.q_last, self.out, self.tables, self.ctx, lse=self.lse,
                               status_word=self.status) == (B.PS_OK, "")

    def check(self, new, qkv):
        st, self.m_tables, slots, pos, start, self.m_ctx = self.model.step(self.m_ctx, new, self.m_tables, self.stride, self.room)
        torch.cuda.synchronize()
        assert st == 0 and self.status.item() == 0
        assert self.tables.tolist() == self.m_tables and self.ctx.tolist() == self.m_ctx and self.slots.tolist() == slots
        q, k, v = self.parts()
        wk, tk = rope_want(k, self.pos, self.inv, [0] * (self.D // 2), False, False)
        wq, tq = rope_want(q, self.pos, self.inv, [0] * (self.D // 2), False, False)
        n = start[-1]
        at = dev(slots[:n], torch.int64)
        check_within(self.kpool.view(-1, self.hkv, self.D)[at], wk[:n], tk[:n])
        check_within(self.q_rot[:n], wq[:n], tq[:n])
        self.m_k.view(-1, self.hkv, self.D)[at] = self.kpool.view(-1, self.hkv, self.D)[at]
        self.m_v.view(-1, self.hkv, self.D)[at] = v[:n]
        assert torch.equal(self.kpool, self.m_k) and torch.equal(self.vpool, self.m_v)
        tables = [t[: -(-c // self.S)] for t, c in zip(self.m_tables, self.m_ctx)]
        check_attn(self.out, self.lse, attn_want(self.m_k, self.m_v, self.q_last, tables, self.m_ctx))


def engine_steps(rng, e, steps):
    for step in range(steps):
        new = rng.integers(0, 12, e.rows) if step % 3 == 0 else np.ones(e.rows, int)
        new[rng.random(e.rows) < 0.2] = -1
        yield step, new.tolist(), torch.randn(tuple(e.qkv.shape), device="cuda").to(e.qkv.dtype)


def test_a_decode_step_on_the_device():
    rng = np.random.default_rng(20)
    e = Engine(rng, 9, 8, 2, 64, 4, 200, 20, 120, torch.bfloat16)
    for _, new, qkv in engine_steps(rng, e, 8):
        e.new.copy_(dev(new))
        e.qkv.copy_(qkv)
        e.enqueue()
        e.check(new, qkv)


def test_a_captured_decode_step_replayed_with_other_lengths():
    """Two engines' steps in two graphs, replayed on two streams at once."""
    rng = np.random.default_rng(21)
    engines = [Engine(rng, 9, 8, 2, 64, 4, 200, 20, 120, torch.bfloat16), Engine(rng, 5, 4, 4, 128, 16, 64, 8, 70, torch.float16)]
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


def test_a_captured_step_with_room_for_prompts():
    """Lengths, stack and tables updated in place by the whole chip, and attended right behind it, over many replays."""
    rng = np.random.default_rng(25)
    e = Engine(rng, 40, 4, 2, 64, 16, 2400, 60, 5000, torch.bfloat16)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        e.enqueue()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        e.enqueue()
    for step in range(12):
        new = rng.integers(0, 120, e.rows) if step % 3 == 0 else np.ones(e.rows, int)
        new[rng.random(e.rows) < 0.1] = -1
        new[[c + max(n, 0) > e.stride * e.S for c, n in zip(e.m_ctx, new)]] = -1
        qkv = torch.randn(tuple(e.qkv.shape), device="cuda").to(e.qkv.dtype)
        e.new.copy_(dev(new.tolist()))
        e.qkv.copy_(qkv)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            g.replay()
        torch.cuda.synchronize()
        e.check(new.tolist(), qkv)


def test_calls_on_several_streams_at_once():
    rng = np.random.default_rng(22)
    cases = []
    for i in range(4):
        ctx = rng.integers(1, 6000, 6).tolist()
        kp, vp, q, tables = attn_case(rng, ctx, 8, 2, 128, 16, torch.bfloat16)
        t = tables_tensor(tables, 400)
        cases.append((kp, vp, q, t, dev(ctx), torch.zeros_like(q), torch.zeros((6, 8), device="cuda"), torch.cuda.Stream(),
                      attn_want(kp, vp, q, tables, ctx)))
    torch.cuda.synchronize()
    for _ in range(10):
        for kp, vp, q, t, n, out, lse, s, _ in cases:
            with torch.cuda.stream(s):
                out.fill_(9.0)
                assert B.ps_paged_attn(kp, vp, q, out, t, n, lse=lse)[0] == B.PS_OK
    torch.cuda.synchronize()
    for *_, out, lse, s, want in cases:
        check_attn(out, lse, want)


def test_attention_next_to_a_contexts_own():
    """The pools and tables of a context: append through its tables, then both attentions on the same cache."""
    rng = np.random.default_rng(23)
    L, hkv, hq, D, S, nb = 1, 8, 32, 128, 16, 300
    kp, vp = (torch.randn((L, nb, S, hkv, D), device="cuda").bfloat16() for _ in range(2))
    lib = B.KVSwap(num_layers=L, num_kv_heads=hkv, num_q_heads=hq, head_dim=D, block_size=S, num_gpu_blocks=nb, max_blocks_per_req=100,
                   max_batch=8, host_pool_bytes=1 << 20, initial_free_order=rng.permutation(nb), k_pools=[kp[0]], v_pools=[vp[0]])
    before = [100, 1, 777, 15, 16]
    reqs = list(range(5))
    for r in reqs:
        assert lib.kv_alloc(r, before[r] + 1) == B.PS_OK
    tables = tables_tensor([lib.block_table(r)[0] for r in reqs], 100)
    ctx, start = dev(before), torch.zeros(6, device="cuda", dtype=I32)
    slots, pos = torch.zeros(5, device="cuda", dtype=torch.int64), torch.zeros(5, device="cuda", dtype=I32)
    assert B.ps_build_slots(ctx, dev([1] * 5), tables, slots, pos, start, ctx, block_size=S, num_gpu_blocks=nb)[0] == B.PS_OK
    q, k, v = rope_inputs(5, hq, hkv, D, torch.bfloat16, 23)
    inv = torch.rand(64, device="cuda")
    q_rot = torch.empty((5, hq, D), device="cuda", dtype=torch.bfloat16)
    assert B.ps_rope_append(q, k, q_rot, None, pos, inv, v=v, kpool=kp[0], vpool=vp[0], slots=slots)[0] == B.PS_OK
    a, b = torch.empty_like(q_rot), torch.empty_like(q_rot)
    la, lb = torch.empty((5, hq), device="cuda"), torch.empty((5, hq), device="cuda")
    assert B.ps_paged_attn(kp[0], vp[0], q_rot, a, tables, ctx, lse=la)[0] == B.PS_OK
    assert lib.decode_attn(0, q_rot, b, reqs, lb) == B.PS_OK
    assert lib.sync() == B.PS_OK
    args = kp[0], vp[0], q_rot, [lib.block_table(r)[0] for r in reqs], [n + 1 for n in before]
    check_attn(a, la, attn_want(*args))
    check_attn(b, lb, attn_want(*args, weight_error=HALF_STEP[torch.bfloat16]))   # rounds a weight once
    lib.destroy()


def test_attention_over_a_request_that_was_offloaded_and_reloaded():
    """The context moves a request out and back; behind the fence the device-side step appends to it and attends it."""
    rng = np.random.default_rng(24)
    L, hkv, hq, D, S, nb = 2, 4, 8, 64, 16, 500
    kp, vp = (torch.randn((L, nb, S, hkv, D), device="cuda").bfloat16() for _ in range(2))
    lib = B.KVSwap(num_layers=L, num_kv_heads=hkv, num_q_heads=hq, head_dim=D, block_size=S, num_gpu_blocks=nb, max_blocks_per_req=200,
                   max_batch=8, host_pool_bytes=256 << 20, initial_free_order=rng.permutation(nb), k_pools=[kp[l] for l in range(L)],
                   v_pools=[vp[l] for l in range(L)])
    ctx = [1500, 40, 900]
    for r, n in enumerate(ctx):
        assert lib.kv_alloc(r, n + 1) == B.PS_OK                   # with room for the token to come
    old = lib.block_table(0)[0]
    K, V = kp[:, torch.tensor(old, device="cuda")].clone(), vp[:, torch.tensor(old, device="cuda")].clone()
    assert lib.swap_out(0) == B.PS_OK and lib.sync() == B.PS_OK
    kp[:, torch.tensor(old, device="cuda")] = 0
    vp[:, torch.tensor(old, device="cuda")] = 0
    assert lib.swap_in_begin(0) == B.PS_OK
    rc, _, _ = lib.step(None, None, [], -1)                        # the whole reload, asynchronously
    assert rc == B.PS_OK and lib.reload_fence(-1) == B.PS_OK
    ids = [lib.block_table(r)[0] for r in range(3)]
    tables = tables_tensor(ids, 200)
    d_ctx, start = dev(ctx), torch.zeros(4, device="cuda", dtype=I32)
    slots, pos = torch.zeros(3, device="cuda", dtype=torch.int64), torch.zeros(3, device="cuda", dtype=I32)
    assert B.ps_build_slots(d_ctx, dev([1] * 3), tables, slots, pos, start, d_ctx, block_size=S, num_gpu_blocks=nb) == (B.PS_OK, "")
    outs = []
    for l in range(L):
        q, k, v = rope_inputs(3, hq, hkv, D, torch.bfloat16, 30 + l)
        assert B.ps_rope_append(None, k, None, None, None, None, v=v, kpool=kp[l], vpool=vp[l], slots=slots) == (B.PS_OK, "")
        out, lse = torch.empty((3, hq, D), device="cuda", dtype=torch.bfloat16), torch.empty((3, hq), device="cuda")
        assert B.ps_paged_attn(kp[l], vp[l], q, out, tables, d_ctx, lse=lse) == (B.PS_OK, "")
        outs.append((q, k, v, out, lse))
    assert lib.sync() == B.PS_OK, lib.last_error()
    new = torch.tensor(ids[0], device="cuda")
    for l, (q, k, v, out, lse) in enumerate(outs):
        for pool, was, row in ((kp, K, k), (vp, V, v)):            # the reloaded bytes, and the appended row
            want = was[l].clone()
            want.view(-1, hkv, D)[ctx[0]] = row[0]
            assert torch.equal(pool[l, new], want)
        check_attn(out, lse, attn_want(kp[l], vp[l], q, ids, [n + 1 for n in ctx]))
    lib.destroy()
