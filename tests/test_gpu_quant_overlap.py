"""Results of ps_quant_attn that lie in the cache are refused; those between its blocks are not."""
import numpy as np
import pytest
import torch

from device_step_util import check_attn, tables_tensor
from paper_2512_12928_b200 import binding as B
from quant_util import quant_attn_want
from test_gpu_device_step import dev
from test_gpu_quant import attn_case

pytestmark = pytest.mark.gpu


def interleaved(gap):
    """A case whose blocks' codes and scales lie in one buffer, `gap` bytes apart: (buffer, cache, a copy of it, q, tables, lengths)."""
    rng = np.random.default_rng(1)
    ctx, H, D, S = [40, 17, 3], 2, 64, 16
    cache, q, tables = attn_case(rng, ctx, 8, H, D, S, torch.bfloat16, torch.int8)
    nb, n = len(cache[0]), S * H * D
    buf = torch.zeros((nb, 2 * n + 16 + gap), device="cuda", dtype=torch.uint8)
    views = [buf[:, :n].view(torch.int8).view(nb, S, H, D), buf[:, n: 2 * n].view(torch.int8).view(nb, S, H, D),
             buf.view(torch.float32)[:, n // 2: n // 2 + H], buf.view(torch.float32)[:, n // 2 + H: n // 2 + 2 * H]]
    for a, b in zip(views, cache):
        a.copy_(b)
    return buf, views, cache, q, tables, ctx


def test_results_in_the_cache_are_refused():
    buf, cache, _, q, tables, ctx = interleaved(2048)
    was = buf.clone()
    flat, t, n = buf.view(-1), tables_tensor(tables, 4), dev(ctx)
    row, width = buf.shape[1], 8 * 64
    as_out = lambda at, stride: flat.view(torch.bfloat16).as_strided((3, 8, 64), (stride // 2, 64, 1), at // 2)
    free = torch.zeros_like(q)
    for at, stride in ((0, 2 * width), (2 * row + 2048, row), (4096 + 16 - 2 * width + 16, row), (row - 16 - 2 * width + 32, row), (row - 2 * width, 2 * width)):
        rc, text = B.ps_quant_attn(*cache, q, as_out(at, stride), t, n)
        assert rc == B.PS_ERR_INVALID and "out overlaps the cache" in text, (at, stride)
    floats = flat.view(torch.float32)
    for at in (0, (row + 2048) // 4, 4096 // 4 + 3 - 23, 4096 // 4):
        rc, text = B.ps_quant_attn(*cache, q, free, t, n, lse=floats[at: at + 24].view(3, 8))
        assert rc == B.PS_ERR_INVALID and "lse overlaps the cache" in text, at
    torch.cuda.synchronize()
    assert torch.equal(buf, was)


def test_results_between_the_blocks_are_not():
    buf, cache, same, q, tables, ctx = interleaved(2048)
    row, flat = buf.shape[1], buf.view(-1)
    at = 4096 + 16
    out = flat.view(torch.bfloat16).as_strided((3, 8, 64), (row // 2, 64, 1), at // 2)
    lse = flat.view(torch.float32)[(at + 1024) // 4: (at + 1024) // 4 + 24].view(3, 8)
    rc, text = B.ps_quant_attn(*cache, q, out, tables_tensor(tables, 4), dev(ctx), lse=lse)
    assert rc == B.PS_OK, text
    check_attn(out, lse, quant_attn_want(*same, q, tables, ctx))
