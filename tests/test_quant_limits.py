"""Limits of the calls over a cache of 8 bits at their borders, through the C ABI: no GPU."""
import ctypes as C

import pytest
import torch

from paper_2512_12928_b200 import binding as B
from test_quant_refusals import append_args, read_args, refused

MOST = (1 << 31) - 1 - 4096


def one_large_block(size):
    return dict(block_size=size, num_gpu_blocks=1, num_kv_heads=1, head_dim=1, k_block_stride=size, v_block_stride=size, k_scale_stride=1,
                v_scale_stride=1, k_stride=1, v_stride=1)


@pytest.mark.parametrize("over", [1, 3000, 4096])
def test_blocks_whose_places_would_wrap_in_32_bits_are_refused(over):
    kw = one_large_block(MOST + over)
    assert "block_size" in refused(B.load().ps_quant_append, append_args(**kw))
    kw["k_out_stride"], kw["v_out_stride"] = kw.pop("k_stride"), kw.pop("v_stride")
    assert "block_size" in refused(B.load().ps_quant_read, read_args(**kw))


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are nobody's")
def test_the_largest_block_is_not_refused():
    err = C.create_string_buffer(256)
    args = append_args(**{**one_large_block(MOST), "v": None, "vpool": None, "v_scale": None})
    assert B.load().ps_quant_append(C.byref(args), None, err, 256) == B.PS_ERR_CUDA     # no device, but nothing wrong
