"""Argument errors of the calls over a cache of 8 bits come back before anything is enqueued: no GPU."""
import ctypes as C

import pytest
import torch

from paper_2512_12928_b200 import binding as B
from test_device_step_refusals import refused

A = 1 << 40   # addresses that no refused call reads, far from one another
K, V, KS, VS, KP, VP, Q, OUT, T, WS = (A + (i << 32) for i in range(10))
BLOCK = 16 * 8 * 128


def cache(**kw):
    base = dict(kpool=KP, vpool=VP, k_scale=KS, v_scale=VS, k_block_stride=BLOCK, v_block_stride=BLOCK, k_scale_stride=8, v_scale_stride=8,
                num_gpu_blocks=64, block_size=16, num_kv_heads=8, head_dim=128, codes=0)
    return B.PsQuantCache(**{**base, **{k: v for k, v in kw.items() if k in base}}), {k: v for k, v in kw.items() if k not in base}


def append_args(**kw):
    c, rest = cache(**kw)
    return B.PsQuantAppendArgs(**{**dict(cache=c, k=K, v=V, slots=T, k_stride=1024, v_stride=1024, tokens=5), **rest})


def read_args(**kw):
    c, rest = cache(**kw)
    return B.PsQuantReadArgs(**{**dict(cache=c, k_out=K, v_out=V, slots=T, k_out_stride=1024, v_out_stride=1024, tokens=5), **rest})


def attn_args(**kw):
    c, rest = cache(**kw)
    return B.PsQuantAttnArgs(**{**dict(cache=c, q=Q, out=OUT, block_tables=T, ctx_lens=T, workspace=WS, workspace_bytes=1 << 40, q_stride=4096,
                                       out_stride=4096, batch=2, table_stride=4, num_q_heads=32), **rest})


CACHE = [dict(num_gpu_blocks=0), dict(num_gpu_blocks=-1), dict(block_size=0), dict(num_kv_heads=0), dict(num_kv_heads=1025), dict(head_dim=0),
         dict(codes=2), dict(codes=-1), dict(dtype=2), dict(dtype=-1), dict(kpool=None), dict(vpool=None), dict(k_scale=None), dict(v_scale=None),
         dict(k_block_stride=BLOCK - 1), dict(v_block_stride=0), dict(k_scale_stride=7), dict(v_scale_stride=0), dict(k_scale=KS + 2)]


@pytest.mark.parametrize("kw", CACHE + [
    dict(head_dim=513), dict(tokens=-1), dict(tokens=(1 << 31) - 100), dict(k_stride=1 << 31), dict(k=None), dict(v=None), dict(slots=None), dict(k=K + 1),
    dict(block_size=1 << 24, num_gpu_blocks=1 << 16, k_block_stride=1 << 36, v_block_stride=1 << 36),
    dict(k=None, v=None, kpool=None, vpool=None, k_scale=None, v_scale=None),
    dict(vpool=KP), dict(vpool=KP + BLOCK - 1), dict(v_scale=KS), dict(v_scale=KS + 4 * 7), dict(k_scale=KP + 64), dict(k=KP), dict(k=KS - 2),
    dict(kpool=K + 2 * 1023), dict(kpool=KP, vpool=KP + BLOCK, k_block_stride=2 * BLOCK - 1, v_block_stride=2 * BLOCK - 1)])
def test_append_refuses(kw):
    assert refused(B.load().ps_quant_append, append_args(**kw)).startswith("ps_quant_append: ")


@pytest.mark.parametrize("kw", CACHE + [
    dict(head_dim=513), dict(tokens=-1), dict(tokens=(1 << 31) - 100), dict(v_out_stride=-(1 << 31) - 1), dict(k_out=None, v_out=None), dict(slots=None), dict(v_out=K), dict(v_out=K + 2 * 1023),
    dict(k_out_stride=1023), dict(v_out_stride=0), dict(k_out=KP + 100), dict(v_out=KS), dict(k_out=K + 1)])
def test_read_refuses(kw):
    assert refused(B.load().ps_quant_read, read_args(**kw)).startswith("ps_quant_read: ")


@pytest.mark.parametrize("kw", CACHE + [
    dict(num_q_heads=0), dict(num_q_heads=33), dict(num_kv_heads=1, num_q_heads=65), dict(head_dim=96), dict(head_dim=80), dict(batch=-1),
    dict(table_stride=0), dict(window=-1), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(out=None),
    dict(block_tables=None), dict(ctx_lens=None), dict(workspace=None), dict(v_block_stride=BLOCK + 8), dict(kpool=KP + 8), dict(q=Q + 8),
    dict(q_stride=4100), dict(out=OUT + 2), dict(out_stride=2048), dict(out=Q, out_stride=4096 + 8), dict(out=Q + 32), dict(table_stride=1 << 30, batch=1 << 20),
    dict(k_block_stride=1 << 36), dict(v_scale_stride=1 << 30)])
def test_attn_refuses(kw):
    assert refused(B.load().ps_quant_attn, attn_args(**kw)).startswith("ps_quant_attn: ")


def test_null_arguments():
    lib = B.load()
    for fn in (lib.ps_quant_append, lib.ps_quant_read, lib.ps_quant_attn):
        refused(fn, None)
    assert lib.ps_quant_attn_workspace(8, 32, 128, None) == B.PS_ERR_INVALID
    n = C.c_int64(7)
    assert lib.ps_quant_attn_workspace(8, 31, 128, C.byref(n)) == B.PS_ERR_INVALID and n.value == 7
    assert lib.ps_quant_attn_workspace(8, 32, 80, C.byref(n)) == B.PS_ERR_INVALID and n.value == 7


def test_nothing_to_do_needs_no_device():
    lib = B.load()
    err = C.create_string_buffer(64)
    assert lib.ps_quant_append(C.byref(append_args(tokens=0, k=None, v=None)), None, err, 64) == B.PS_OK
    assert lib.ps_quant_read(C.byref(read_args(tokens=0, k_out=None)), None, err, 64) == B.PS_OK
    assert lib.ps_quant_attn(C.byref(attn_args(batch=0)), None, err, 64) == B.PS_OK


def test_tensors_on_the_host_are_refused():
    x = torch.zeros((2, 8, 64), dtype=torch.bfloat16)
    pool, scale = torch.zeros((4, 16, 8, 64), dtype=torch.int8), torch.zeros((4, 8))
    slots, i = torch.zeros(2, dtype=torch.int64), torch.zeros(2, dtype=torch.int32)
    for rc, text in (B.ps_quant_append(x, x, pool, pool, scale, scale, slots), B.ps_quant_read(pool, pool, scale, scale, slots, x, x),
                     B.ps_quant_attn(pool, pool, scale, scale, x, x, torch.zeros((2, 2), dtype=torch.int32), i),
                     B.ps_quant_append(None, None, pool, pool, scale, scale, slots), B.ps_quant_read(pool, pool, scale, scale, slots, None, None)):
        assert rc == B.PS_ERR_INVALID and text
