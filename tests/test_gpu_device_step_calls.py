"""Calls of the device-side step that its other tests do not make: row counts around the kernels' limits, README's loop."""
import os
import re
import subprocess
import sys

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)                                            # as a script too
from device_step_util import attn_want, check_attn, check_within, rope_want, tables_tensor
from paper_2512_12928_b200 import binding as B
from test_gpu_device_step import Engine, attn_case, dev, run_attn, slot_case

pytestmark = pytest.mark.gpu


def slots_steps(rows, in_place):
    """Three steps of a batch with room for 9000 tokens against the model."""
    rng = np.random.default_rng(rows)
    c = slot_case(rng, rows, 16, 40, 6, rows * 6, 9000, in_place=in_place)
    for _ in range(3):
        new = rng.integers(0, 4, rows)
        new[rng.random(rows) < 0.1] = -1
        c.step(new.tolist())


@pytest.mark.parametrize("rows,in_place", [(3024, False), (3025, False), (3050, True), (3071, False), (4096, False), (4097, True)])
def test_slots_as_a_process_first_call(rows, in_place):
    """The rows' scanned counts take 16 bytes of shared memory each: around what a kernel has without asking for more, the
    call may not depend on what an earlier call of the process has asked for."""
    p = subprocess.run([sys.executable, os.path.abspath(__file__), str(rows), str(int(in_place))], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stdout[-2000:] + p.stderr[-2000:]


def test_readmes_loop_with_requests_that_end_and_pause():
    """README's step as it stands there, in a batch where tokens and rows are not numbered alike: a row that ended and one
    without a new token have no query among the tokens."""
    text = open(os.path.join(ROOT, "README.md")).read()
    code, = [c for c in re.findall(r"```python\n(.*?)```", text, re.S) if "ps_build_slots" in c]
    rng = np.random.default_rng(30)
    rows, L, hq, hkv, D, S, M = 6, 2, 8, 2, 64, 16, 60
    e = Engine(rng, rows, hq, hkv, D, S, M, 12, rows, torch.bfloat16)       # the room of a captured decode step
    K, V = (torch.zeros((L, M, S, hkv, D), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    q, k, v = e.parts()
    ns = dict(torch=torch, B=B, L=L, M=M, K=K, V=V, q=q, k=k, v=v, q_rot=e.q_rot, out=e.out, inv_freq=e.inv, ctx_lens=e.ctx, new_lens=e.new,
              tables=e.tables, slots=e.slots, positions=e.pos, token_start=e.start, stack=e.ids, top=e.count)
    for new in ([1] * 6, [1, 1, 0, 1, 1, 1], [1, -1, 1, 0, 1, 1], [1, 1, -1, -1, 0, 1], [0, 1, 1, 0, -1, 1]):
        e.new.copy_(dev(new))
        e.qkv.copy_(torch.randn(tuple(e.qkv.shape), device="cuda"))
        e.q_rot.fill_(7.0)
        exec(code, ns)
        assert ns["rc"] == B.PS_OK, ns["err"]
        torch.cuda.synchronize()
        st, e.m_tables, slots, pos, start, e.m_ctx = e.model.step(e.m_ctx, new, e.m_tables, 12, rows)
        assert st == 0 and e.slots.tolist() == slots and e.start.tolist() == start and e.ctx.tolist() == e.m_ctx
        wq, tq = rope_want(q, e.pos, e.inv, [0] * (D // 2), False, False)
        check_within(e.q_rot[: start[-1]], wq[: start[-1]], tq[: start[-1]])
        live = [b for b in range(rows) if new[b] > 0]
        own = e.q_rot[dev([start[b] for b in live], torch.int64)]           # a row's token is its query
        tables = [e.m_tables[b][: -(-e.m_ctx[b] // S)] for b in live]
        o, _, tol, _ = attn_want(K[L - 1], V[L - 1], own, tables, [e.m_ctx[b] for b in live])
        check_within(e.out[dev(live, torch.int64)], o, tol)
        assert not e.out[dev([b for b in range(rows) if new[b] < 0], torch.int64)].any()


def test_rope_outputs_between_the_inputs_rows():
    """Outputs in the gaps of the inputs' buffer: one stride for all, and keys whose rows lie twice as far apart."""
    T, hq, hkv, D = 9, 3, 2, 64
    buf = torch.randn((2 * T, 12 * D), device="cuda").bfloat16()
    part = lambda rows, at, heads: rows[:, at * D: (at + heads) * D].view(T, heads, D)
    q, q_out, k = part(buf[:T], 0, hq), part(buf[:T], 3, hq), part(buf[:T], 6, hkv)
    far = part(buf[::2], 8, hkv)
    pos, inv = dev(list(range(T))), torch.rand(D // 2, device="cuda")
    (wq, tq), (wk, tk) = rope_want(q, pos, inv, [0] * 32, False, False), rope_want(k, pos, inv, [0] * 32, False, False)
    was = buf.clone()
    assert B.ps_rope_append(q, k, q_out, far, pos, inv) == (B.PS_OK, "")
    check_within(q_out, wq, tq)
    check_within(far, wk, tk)
    q_out.copy_(part(was[:T], 3, hq))
    far.copy_(part(was[::2], 8, hkv))
    assert torch.equal(buf, was)
    rc, text = B.ps_rope_append(q, k, part(buf[:T], 1, hq), None, pos, inv, v=k, kpool=buf[:4].view(-1)[: 4 * hkv * D].view(1, 4, hkv, D),
                                vpool=buf[4:8].view(-1)[: 4 * hkv * D].view(1, 4, hkv, D), slots=dev([-1] * T, torch.int64))
    assert rc == B.PS_ERR_INVALID and "overlap" in text
    torch.cuda.synchronize()
    assert torch.equal(buf, was)


@pytest.mark.parametrize("hq,hkv,D,ctx", [
    (1024, 1024, 64, [0, 1, 40, 200]), (1040, 130, 128, [700, 3]), (65 * 33, 65, 64, [5, 300, 0]), (576, 9, 128, [33] * 40 + [900])])
def test_attn_many_heads(hq, hkv, D, ctx):
    """Rows whose heads are many CTAs' work, up to the 1024 KV heads that are accepted."""
    rng = np.random.default_rng(hq)
    kp, vp, q, tables = attn_case(rng, ctx, hq, hkv, D, 16, torch.bfloat16)
    out, lse = run_attn(kp, vp, q, tables, ctx)
    check_attn(out, lse, attn_want(kp, vp, q, tables, ctx))


@pytest.mark.parametrize("hq,hkv,D,ctx", [(32, 8, 128, [300]), (32, 8, 128, [0, 5000, 17, 900]), (16, 1, 64, [60000]), (64, 1, 128, [700] * 9),
                                          (24, 24, 64, [1] * 30 + [4000] + [90] * 200)])
def test_attn_in_place(hq, hkv, D, ctx):
    """out may be q, whether a row is one CTA's or cut."""
    rng = np.random.default_rng(hq + D)
    kp, vp, q, tables = attn_case(rng, ctx, hq, hkv, D, 16, torch.bfloat16)
    out, lse = run_attn(kp, vp, q, tables, ctx)
    t = tables_tensor(tables, max(1, max(len(x) for x in tables)))
    for _ in range(20):
        rows = torch.full((len(ctx), hq + 2, D), 3.0, device="cuda", dtype=torch.bfloat16)
        own, own_lse = rows[:, 1: 1 + hq], torch.empty_like(lse)
        own.copy_(q)
        assert B.ps_paged_attn(kp, vp, own, own, t, dev(ctx), lse=own_lse) == (B.PS_OK, "")
        assert torch.equal(own, out) and torch.equal(own_lse, lse)
        assert (rows[:, 0] == 3.0).all() and (rows[:, -1] == 3.0).all()


def test_attn_infinite_values():
    """Of an infinite value among the attended ones its own dims are not finite and no others; scores of -inf have no weight."""
    rng = np.random.default_rng(31)
    ctx = [40, 700]
    for dt in (torch.bfloat16, torch.float16):
        kp, vp, q, tables = attn_case(rng, ctx, 8, 2, 64, 16, dt)
        want = attn_want(kp, vp, q, tables, ctx)
        vp[tables[1][3], 5, 1, 7] = float("inf")
        out, lse = run_attn(kp, vp, q, tables, ctx)
        hit = torch.zeros_like(out, dtype=torch.bool)
        hit[1, 4:, 7] = True
        assert not torch.isfinite(out[hit]).any()
        o, l, tol, tol_lse = want
        o[hit.cpu().numpy()], tol[hit.cpu().numpy()] = 0.0, 0.0
        check_attn(torch.where(hit, 0.0, out), lse, (o, l, tol, tol_lse))


def test_attn_very_many_rows():
    """More rows than a CTA's threads read in a few rounds, some empty, in blocks that rows share."""
    rows, S, hq, hkv, D, nb = 40001, 16, 4, 2, 64, 50
    g = torch.Generator(device="cuda").manual_seed(33)
    kp, vp = (torch.randn((nb, S, hkv, D), device="cuda", generator=g).bfloat16() for _ in range(2))
    q = torch.randn((rows, hq, D), device="cuda", generator=g).bfloat16()
    tables = torch.randint(0, nb, (rows, 3), device="cuda", generator=g, dtype=torch.int32)
    ctx = torch.randint(0, 3 * S + 1, (rows,), device="cuda", generator=g, dtype=torch.int32)
    out, lse = run_attn(kp, vp, q, tables, ctx.tolist())
    some = list(range(0, rows, 397)) + [rows - 1]
    check_attn(out[some], lse[some], attn_want(kp, vp, q[some], tables[some].tolist(), ctx[some].tolist()))
    t = torch.arange(3 * S, device="cuda")                              # all rows, loosely: a half step of the result and some room
    at = tables.long()[:, t // S] * S + t % S
    x = torch.einsum("bhgd,bthd->bhgt", q.view(rows, hkv, 2, D).float(), kp.view(-1, hkv, D)[at].float()) / 8
    p = torch.softmax(x.masked_fill(t >= ctx[:, None, None, None], -1e30), -1) * (ctx > 0)[:, None, None, None]
    want = torch.einsum("bhgt,bthd->bhgd", p, vp.view(-1, hkv, D)[at].float()).reshape(rows, hq, D)
    assert ((out.float() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all()


def first_calls_captured():
    """A process's first calls, inside a capture that a side stream's kernels feed."""
    rng = np.random.default_rng(34)
    e = Engine(rng, 7, 8, 2, 64, 16, 200, 60, 5000, torch.bfloat16)          # 903 tokens in the longest row
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
        assert torch.equal(e.qkv, base * factor)


def test_first_calls_of_a_process_captured_behind_another_stream():
    p = subprocess.run([sys.executable, os.path.abspath(__file__), "captured"], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stdout[-2000:] + p.stderr[-2000:]


if __name__ == "__main__":
    if sys.argv[1] == "captured":
        first_calls_captured()
    else:
        slots_steps(int(sys.argv[1]), bool(int(sys.argv[2])))
