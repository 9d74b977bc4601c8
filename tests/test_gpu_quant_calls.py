"""Calls over a cache of 8 bits that its other tests do not make: README's loop, a process's first calls in a capture, heads in
large numbers, pools that span more than 32 bits of 16-byte steps."""
import ctypes as C
import os
import re
import subprocess
import sys

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)                                            # as a script too
from device_step_util import check_attn, tables_tensor
from paper_2512_12928_b200 import binding as B
from quant_util import CacheModel, make_cache, quant_attn_want, read_want
from test_gpu_device_step import Engine, dev
from test_gpu_quant import I64, QuantEngine, attn_case, gen, kv_rows, run_attn

pytestmark = pytest.mark.gpu


def test_readmes_loop():
    """README's step over a cache of 8 bits as it stands there, with the slots and tables of its first loop."""
    text = open(os.path.join(ROOT, "README.md")).read()
    blocks = re.findall(r"```python\n(.*?)```", text, re.S)
    code, = [c for c in blocks if "ps_quant_append" in c]
    begin, = [c for c in blocks if "cache = [" in c]
    rng = np.random.default_rng(30)
    rows, L, hq, hkv, D, S, M = 6, 2, 8, 2, 64, 16, 60
    e = Engine(rng, rows, hq, hkv, D, S, M, 12, 40, torch.bfloat16)
    ns = dict(torch=torch, B=B, L=L, M=M, q_rot=e.q_rot, out=e.out, inv_freq=e.inv, ctx_lens=e.ctx, tables=e.tables, slots=e.slots,
              positions=e.pos, block_size=S, num_kv_heads=hkv, head_dim=D)
    ns["q"], ns["k"], ns["v"] = e.parts()
    exec(begin, ns)
    models = [[CacheModel(c[i], c[2 + i]) for i in range(2)] for c in ns["cache"]]
    for new in ([5] * 6, [1, 1, 0, 1, 1, 1], [1, -1, 1, 0, 1, 1], [20, 1, -1, -1, 0, 1], [0, 1, 1, 0, -1, 1]):
        e.new.copy_(dev(new))
        e.qkv.copy_(torch.randn(tuple(e.qkv.shape), device="cuda"))
        assert B.ps_build_slots(e.ctx, e.new, e.tables, e.slots, e.pos, e.start, e.ctx, block_size=S, num_gpu_blocks=M, free_ids=e.ids,
                                free_count=e.count, free_count_out=e.count) == (B.PS_OK, "")
        ns["last"] = (e.start[1:] - 1).clamp(min=0)
        exec(code, ns)
        assert ns["rc"] == B.PS_OK, ns["err"]
        torch.cuda.synchronize()
        st, e.m_tables, slots, _, start, e.m_ctx = e.model.step(e.m_ctx, new, e.m_tables, 12, 40)
        assert st == 0 and e.slots.tolist() == slots
        n = start[-1]
        caches = ns["cache"]
        for c, pair in zip(caches, models):
            for i, (m, x) in enumerate(zip(pair, (ns["k_rot"], ns["v"]))):
                m.append(x[:n], slots[:n])
                m.check(c[i], c[2 + i])
        live = [b for b in range(rows) if new[b] > 0]
        own = e.q_rot[dev([start[b + 1] - 1 for b in live], I64)]
        tables = [e.m_tables[b][: -(-e.m_ctx[b] // S)] for b in live]
        w, _, tol, _ = quant_attn_want(*caches[-1], own, tables, [e.m_ctx[b] for b in live])
        got = e.out[dev(live, I64)].double().cpu().numpy()
        assert (np.abs(got - w) <= tol).all()
        assert torch.equal(ns["k_back"][:n], read_want(caches[-1][0], caches[-1][2], slots[:n], torch.bfloat16))


@pytest.mark.parametrize("codes", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("hq,hkv,D,ctx", [(9, 9, 64, [40, 700]), (1024, 1024, 64, [1, 70]), (34, 17, 128, [500, 33, 0]), (2048, 32, 64, [45]),
                                          (100, 5, 128, [300, 2000]), (192, 3, 64, [1500])])
def test_attn_many_heads(codes, hq, hkv, D, ctx):
    rng = np.random.default_rng(hq)
    for dt in (torch.bfloat16, torch.float16):
        cache, q, tables = attn_case(rng, ctx, hq, hkv, D, 16, dt, codes)
        check_attn(*run_attn(cache, q, tables, ctx), quant_attn_want(*cache, q, tables, ctx))


@pytest.mark.parametrize("codes", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_attn_of_queries_that_are_not_finite(codes, dt):
    """A head with a NaN has NaN results; one with an infinite value has no finite ones; other heads do not notice."""
    rng = np.random.default_rng(3)
    ctx = [100, 40]
    cache, q, tables = attn_case(rng, ctx, 8, 2, 128, 16, dt, codes)
    want = quant_attn_want(*cache, q, tables, ctx)
    bad = q.clone()
    bad[0, 1, 17], bad[1, 6, 127], bad[1, 2, 0] = float("nan"), float("inf"), -float("inf")
    out, lse = run_attn(cache, bad, tables, ctx)
    assert out[0, 1].isnan().all() and lse[0, 1].isnan()
    for b, h in ((1, 6), (1, 2)):
        assert not out[b, h].isfinite().any() and not lse[b, h].isfinite()
    for b, h in ((0, 1), (1, 6), (1, 2)):
        out[b, h], lse[b, h] = torch.from_numpy(want[0][b, h]), float(want[1][b, h])
    check_attn(out, lse, want)


def test_attn_of_the_largest_and_smallest_queries():
    """Heads of the types' largest and smallest values, and of zeros, next to ordinary ones."""
    rng = np.random.default_rng(4)
    ctx = [70]
    for codes in (torch.int8, torch.float8_e4m3fn):
        for dt in (torch.bfloat16, torch.float16):
            cache, q, tables = attn_case(rng, ctx, 8, 2, 64, 16, dt, codes)
            big, small = torch.finfo(dt).max, torch.finfo(dt).smallest_normal
            q[0, 0], q[0, 1], q[0, 5] = 0, q[0, 1].sign() * small, q[0, 5].sign() * big
            q[0, 6, 1:] = q[0, 6, 1:].sign() * small              # next to one ordinary value
            q[0, 2] = q[0, 2].sign() * small / 4
            cache[2] *= 2.0 ** -40 if dt == torch.float16 else 2.0 ** -140      # so that the large head's scores are finite
            cache[2].clamp_(min=0)
            check_attn(*run_attn(cache, q, tables, ctx, scale=1.0), quant_attn_want(*cache, q, tables, ctx, scale=1.0))


@pytest.mark.parametrize("codes", [torch.int8, torch.float8_e4m3fn])
def test_attn_of_a_pool_that_counts_more_blocks_than_it_uses(codes):
    """A pool said to have so many blocks that its 16-byte steps need more than 32 bits is addressed in 64; the tables name the
    blocks that are there."""
    rng = np.random.default_rng(5)
    ctx = [333, 1, 64]
    for D in (64, 128):
        cache, q, tables = attn_case(rng, ctx, 8, 2, D, 16, torch.bfloat16, codes)
        want = quant_attn_want(*cache, q, tables, ctx)
        check_attn(*run_attn(cache, q, tables, ctx), want)
        block = 16 * 2 * D
        out, lse = torch.empty_like(q), torch.empty((3, 8), device="cuda")
        t, n = tables_tensor(tables, 30), dev(ctx)
        ws = torch.empty(B.ps_quant_attn_workspace(2, 8, D), device="cuda", dtype=torch.uint8)
        c = B.PsQuantCache(*[x.data_ptr() for x in cache], block, block, 2, 2, (1 << 36) // block + 1, 16, 2, D, 0 if codes == torch.int8 else 1)
        a = B.PsQuantAttnArgs(c, q.data_ptr(), out.data_ptr(), lse.data_ptr(), t.data_ptr(), n.data_ptr(), None, ws.data_ptr(), ws.numel(), 8 * D,
                              8 * D, 3, 30, 8, 0, 0.0, 0)
        err = C.create_string_buffer(256)
        assert B.load().ps_quant_attn(C.byref(a), torch.cuda.current_stream().cuda_stream, err, 256) == B.PS_OK, err.value
        check_attn(out, lse, want)


def test_blocks_far_apart():
    """Blocks 2^35 bytes apart, the last one 2^36 behind the first: written, attended and read back."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 70 GB of device memory")
    S, H, D = 16, 2, 64
    n = S * H * D
    buf = torch.empty((1 << 36) + 2 * n + 64, device="cuda", dtype=torch.uint8)
    kp, vp = (buf[i * n:].as_strided((3, n), (1 << 35, 1), i * n).view(torch.int8).unflatten(1, (S, H, D)) for i in range(2))
    scales = torch.zeros((2, 3, H), device="cuda")
    slots = [2 * S + i for i in range(S)] + [S + i for i in range(S)] + list(range(7))
    k, v = kv_rows(len(slots), H, D, torch.bfloat16, 1)
    cache = kp, vp, scales[0], scales[1]
    assert B.ps_quant_append(k, v, *cache, dev(slots, I64)) == (B.PS_OK, "")
    near = [torch.empty((3, S, H, D), device="cuda", dtype=torch.int8) for _ in range(2)] + [torch.zeros((3, H), device="cuda") for _ in range(2)]
    assert B.ps_quant_append(k, v, *near, dev(slots, I64)) == (B.PS_OK, "")
    for c in (2, 1, 0):
        for far, close in zip(cache, near):
            places = slice(0, 7) if c == 0 and far.dim() == 4 else slice(None)
            assert torch.equal(far[c][places], close[c][places])
    q = torch.randn((1, 8, D), device="cuda").bfloat16()
    ctx, tables = [2 * S + 7], [[2, 1, 0]]
    check_attn(*run_attn(cache, q, tables, ctx), quant_attn_want(*near, q, tables, ctx))
    back = [torch.zeros_like(k) for _ in range(2)]
    assert B.ps_quant_read(*cache, dev(slots, I64), *back) == (B.PS_OK, "")
    assert torch.equal(back[0], read_want(near[0], near[2], slots, torch.bfloat16)) and torch.equal(back[1], read_want(near[1], near[3], slots, torch.bfloat16))
    del buf, kp, vp, cache
    torch.cuda.empty_cache()


def test_two_appends_and_attention_behind_each_other():
    """Many dependent calls on one stream without a wait: each sees what the one before it wrote."""
    H, D, S, nb, B_ = 2, 64, 8, 64, 5
    rng = np.random.default_rng(9)
    for codes in (torch.int8, torch.float8_e4m3fn):
        (kp, ks), (vp, vs) = (make_cache((nb, S, H, D), codes, gen(i)) for i in range(2))
        ids = rng.permutation(nb)[: B_ * 5].reshape(B_, 5).tolist()
        t = tables_tensor(ids, 5)
        mk, mv = CacheModel(kp, ks), CacheModel(vp, vs)
        outs, steps = [], []
        for n in range(36):
            slots = [ids[b][n // S] * S + n % S for b in range(B_)]
            k, v = (x * (1.0 + n % 5) for x in kv_rows(B_, H, D, torch.bfloat16, n, fused=False))
            q = torch.randn((B_, 4, D), device="cuda", generator=gen(n)).bfloat16()
            steps.append((slots, k, v, q, dev(slots, I64), dev([n + 1] * B_)))
            outs.append((torch.empty_like(q), torch.empty((B_, 4), device="cuda")))
        torch.cuda.synchronize()
        for (slots, k, v, q, d_slots, d_ctx), (out, lse) in zip(steps, outs):
            assert B.ps_quant_append(k, v, kp, vp, ks, vs, d_slots)[0] == B.PS_OK
            assert B.ps_quant_attn(kp, vp, ks, vs, q, out, t, d_ctx, lse=lse)[0] == B.PS_OK
        torch.cuda.synchronize()
        for n, ((slots, k, v, q, *_), (out, lse)) in enumerate(zip(steps, outs)):
            mk.append(k, slots)
            mv.append(v, slots)
            if n % 7 == 0 or n == 35:
                c = [torch.from_numpy(m.code).cuda() for m in (mk, mv)] + [torch.from_numpy(m.scale).cuda() for m in (mk, mv)]
                c[1] = c[1].float().to(codes)                      # (the model's tolerance goes by the codes' type)
                check_attn(out, lse, quant_attn_want(*c, q, ids, [n + 1] * B_))
        mk.check(kp, ks)
        mv.check(vp, vs)


def first_calls_captured():
    """A process's first calls, inside a capture that a side stream's kernels feed."""
    rng = np.random.default_rng(34)
    e = QuantEngine(rng, 7, 8, 2, 64, 16, 200, 60, 5000, torch.bfloat16, codes="int8")          # 903 tokens in the longest row
    base = torch.randn(tuple(e.qkv.shape), device="cuda").to(e.qkv.dtype)
    new_in, factor = torch.zeros_like(e.new), torch.ones((), device="cuda", dtype=e.qkv.dtype)
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        here = torch.cuda.current_stream()
        side.wait_stream(here)
        with torch.cuda.stream(side):
            for _ in range(20):
                torch.mul(base, factor, out=e.qkv)
            e.new.copy_(new_in)
        here.wait_stream(side)
        e.enqueue()
    for step in range(6):
        new = [40, 1, 0, 300, 1, 1, 17] if step % 2 == 0 else [1, -1, 1, 1, 0, -1, 1]
        new_in.copy_(dev(new))
        factor.fill_(float(step + 1))
        torch.cuda.synchronize()
        g.replay()
        e.check(new, None)


def test_first_calls_of_a_process_captured_behind_another_stream():
    p = subprocess.run([sys.executable, os.path.abspath(__file__), "captured"], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stdout[-2000:] + p.stderr[-2000:]


if __name__ == "__main__":
    first_calls_captured()
