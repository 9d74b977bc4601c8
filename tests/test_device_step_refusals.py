"""Argument errors of ps_build_slots, ps_rope_append and ps_paged_attn come back before anything is enqueued: no GPU."""
import ctypes as C

import pytest
import torch

from paper_2512_12928_b200 import binding as B

A = 1 << 20   # an address that no refused call reads


def slots_args(**kw):
    base = dict(ctx_lens=A, new_lens=A, block_tables=A, free_ids=A, free_count=A, free_count_out=A, slots=A, positions=A,
                token_start=A, ctx_lens_out=A, batch=4, table_stride=8, block_size=16, num_gpu_blocks=64, max_tokens=16)
    return B.PsSlotsArgs(**{**base, **kw})


def rope_args(**kw):
    base = dict(q=A, k=A, v=A, q_out=A, kpool=A, vpool=A, slots=A, positions=A, inv_freq=A, q_stride=4096, k_stride=1024,
                v_stride=1024, q_out_stride=4096, k_block_stride=16 * 1024, v_block_stride=16 * 1024, tokens=3, num_q_heads=32,
                num_kv_heads=8, head_dim=128, rot_dim=128, num_axes=1, block_size=16, num_gpu_blocks=64)
    return B.PsRopeArgs(**{**base, **kw})


def attn_args(**kw):
    base = dict(kpool=A, vpool=A, q=A, out=A, block_tables=A, ctx_lens=A, workspace=A, workspace_bytes=1 << 40,
                k_block_stride=16 * 1024, v_block_stride=16 * 1024, q_stride=4096, out_stride=4096, batch=2, table_stride=4,
                num_kv_heads=8, num_q_heads=32, head_dim=128, block_size=16, num_gpu_blocks=64)
    return B.PsPagedAttnArgs(**{**base, **kw})


def refused(fn, args):
    err = C.create_string_buffer(256)
    rc = fn(C.byref(args) if args is not None else None, None, err, 256)
    assert rc == B.PS_ERR_INVALID and err.value
    assert fn(C.byref(args) if args is not None else None, None, None, 0) == B.PS_ERR_INVALID   # no text asked for
    return err.value.decode()


@pytest.mark.parametrize("kw", [
    dict(batch=-1), dict(max_tokens=-1), dict(block_size=0), dict(num_gpu_blocks=0), dict(table_stride=0),
    dict(ctx_lens=None), dict(new_lens=None), dict(block_tables=None), dict(ctx_lens_out=None), dict(token_start=None),
    dict(slots=None), dict(free_count=None), dict(free_count_out=None)])
def test_build_slots_refuses(kw):
    assert refused(B.load().ps_build_slots, slots_args(**kw)).startswith("ps_build_slots: ")


@pytest.mark.parametrize("kw", [
    dict(tokens=-1), dict(num_q_heads=-1), dict(num_kv_heads=-1), dict(head_dim=0), dict(head_dim=514), dict(rot_dim=-2),
    dict(rot_dim=130), dict(rot_dim=63), dict(dtype=2), dict(dtype=-1), dict(flags=4), dict(q_out=None), dict(kpool=None),
    dict(vpool=None), dict(k=None), dict(v=None), dict(slots=None), dict(block_size=0), dict(num_gpu_blocks=0),
    dict(k_block_stride=16 * 1024 - 1), dict(v_block_stride=0), dict(kpool=None, vpool=None), dict(inv_freq=None),
    dict(num_axes=0), dict(num_axes=9), dict(positions=None)])
def test_rope_append_refuses(kw):
    assert refused(B.load().ps_rope_append, rope_args(**kw)).startswith("ps_rope_append: ")


def test_rope_append_refuses_an_axis_that_is_not_there():
    for axis in (3, 255):
        arr = (C.c_uint8 * 256)(*([0] * 63 + [axis]))
        assert "axis" in refused(B.load().ps_rope_append, rope_args(num_axes=3, freq_axis=arr))


@pytest.mark.parametrize("kw", [
    dict(num_kv_heads=0), dict(num_q_heads=0), dict(num_q_heads=33), dict(num_kv_heads=1, num_q_heads=65), dict(head_dim=96),
    dict(num_kv_heads=1025, num_q_heads=1025), dict(batch=-1), dict(block_size=0), dict(num_gpu_blocks=0), dict(table_stride=0),
    dict(window=-1), dict(dtype=2), dict(scale=float("nan")), dict(scale=float("inf")), dict(kpool=None), dict(vpool=None),
    dict(q=None), dict(out=None), dict(block_tables=None), dict(ctx_lens=None), dict(workspace=None),
    dict(k_block_stride=1024), dict(v_block_stride=16 * 1024 + 4), dict(kpool=A + 8), dict(q=A + 8), dict(q_stride=4100),
    dict(out=A + 2), dict(out_stride=2048)])
def test_paged_attn_refuses(kw):
    assert refused(B.load().ps_paged_attn, attn_args(**kw)).startswith("ps_paged_attn: ")


def test_null_arguments():
    lib = B.load()
    for fn in (lib.ps_build_slots, lib.ps_rope_append, lib.ps_paged_attn):
        refused(fn, None)
    assert lib.ps_paged_attn_workspace(8, 32, 128, None) == B.PS_ERR_INVALID
    n = C.c_int64(7)
    assert lib.ps_paged_attn_workspace(8, 31, 128, C.byref(n)) == B.PS_ERR_INVALID and n.value == 7


def test_nothing_to_do_needs_no_device():
    lib = B.load()
    err = C.create_string_buffer(64)
    assert lib.ps_rope_append(C.byref(rope_args(tokens=0)), None, err, 64) == B.PS_OK
    assert lib.ps_rope_append(C.byref(rope_args(q=None, k=None, v=None, kpool=None, vpool=None)), None, err, 64) == B.PS_OK
    assert lib.ps_paged_attn(C.byref(attn_args(batch=0)), None, err, 64) == B.PS_OK


def test_tensors_on_the_host_are_refused():
    """The binding checks tensors before it hands addresses on."""
    i = torch.zeros(4, dtype=torch.int32)
    rc, text = B.ps_build_slots(i, i, torch.zeros((4, 2), dtype=torch.int32), torch.zeros(4, dtype=torch.int64), i,
                                torch.zeros(5, dtype=torch.int32), i, block_size=16, num_gpu_blocks=8)
    assert rc == B.PS_ERR_INVALID and "device" in text
    x = torch.zeros((2, 8, 64), dtype=torch.bfloat16)
    rc, text = B.ps_rope_append(x, None, x, None, None, None)
    assert rc == B.PS_ERR_INVALID and text
    pool = torch.zeros((4, 16, 8, 64), dtype=torch.bfloat16)
    rc, text = B.ps_paged_attn(pool, pool, x, x, torch.zeros((2, 2), dtype=torch.int32), i[:2])
    assert rc == B.PS_ERR_INVALID and text
