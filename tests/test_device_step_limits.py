"""How long the tables of ps_paged_attn may be: what the header promises is accepted, what does not fit is refused, both
before the device is asked for anything.  No GPU, and none used: the workspace of every call here is too small."""
import ctypes as C

import pytest

from paper_2512_12928_b200 import binding as B

A = 1 << 20                      # an address that no refused call reads
INT_MAX = (1 << 31) - 1


def too_long(batch, stride, block, hkv, group, dim):
    """Whether the call is refused because of its tables' length."""
    args = B.PsPagedAttnArgs(kpool=A, vpool=A, q=A, out=A, block_tables=A, ctx_lens=A, workspace=A, workspace_bytes=0,
                             k_block_stride=block * hkv * dim, v_block_stride=block * hkv * dim, q_stride=hkv * group * dim,
                             out_stride=hkv * group * dim, batch=batch, table_stride=stride, num_kv_heads=hkv, num_q_heads=hkv * group,
                             head_dim=dim, block_size=block, num_gpu_blocks=64)
    err = C.create_string_buffer(256)
    rc = B.load().ps_paged_attn(C.byref(args), None, err, 256)
    text = err.value.decode()
    if rc == B.PS_ERR_INVALID and "2^30 tiles" in text:
        return True
    assert rc == B.PS_ERR_CUDA or (rc == B.PS_ERR_INVALID and "workspace" in text), (rc, text)   # no device, or one
    return False


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group", [1, 4, 8, 16, 17, 32, 33, 48, 64])
@pytest.mark.parametrize("hkv", [1, 2, 3, 5, 8, 9, 13, 128, 1024])
def test_what_the_header_promises_is_accepted(hkv, group, dim):
    """Tables with room for up to 2^34 tokens times KV heads, counting 1024 tokens more for every row."""
    for batch in (1, 2, 3, 5, 8, 16, 17, 64, 1000, 65536, 1 << 20):
        room = min(INT_MAX, (1 << 34) // (batch * hkv) - 1024)
        if room > 0:
            assert not too_long(batch, room, 1, hkv, group, dim)
            assert not too_long(batch, max(1, room // 16), 16, hkv, group, dim)
    assert not too_long(1, INT_MAX, 1024, 1, group, dim)        # of a row, tokens beyond 2^31 - 1025 are not counted


@pytest.mark.parametrize("batch,stride,block,hkv,group,dim", [
    (64, 1 << 22, 16, 8, 64, 128),      # 2^35 tokens times KV heads, in 32 units of 16 query heads
    (4096, 1 << 19, 16, 1, 64, 128), (2048, 1 << 20, 24, 3, 33, 128), (64, INT_MAX, 1, 8, 4, 128), (INT_MAX, 1, 1, 1, 1, 64),
    (1 << 20, 1 << 20, 16, 1024, 64, 64)])
def test_what_does_not_fit_is_refused(batch, stride, block, hkv, group, dim):
    assert too_long(batch, stride, block, hkv, group, dim)
