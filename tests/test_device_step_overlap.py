"""Outputs of ps_rope_append and ps_paged_attn that share elements with what they read or write elsewhere are refused: no GPU.

Every call here is refused: those whose rows are apart lack positions, or a workspace, which is found out last."""
import ctypes as C
import random

import pytest

from paper_2512_12928_b200 import binding as B

A = 1 << 30                      # an address that no refused call reads
T, HQ, HKV, D = 7, 3, 2, 8
QW, KW = HQ * D, HKV * D


def answer(rows, tokens=T, append=True, **kw):
    """rows: name -> (element offset, stride).  Which complaint comes back: 'overlap', or 'positions' for rows that are apart."""
    f = dict(q=None, k=None, v=None, q_out=None, k_out=None)
    for name, (at, stride) in rows.items():
        f[name] = A + 2 * at
        f[name + "_stride"] = stride
    if append:
        f.update(kpool=A << 2, vpool=A << 3, slots=A << 4, block_size=4, num_gpu_blocks=8, k_block_stride=4 * KW, v_block_stride=4 * KW)
    f.update(dict(tokens=tokens, num_q_heads=HQ, num_kv_heads=HKV, head_dim=D, rot_dim=D, num_axes=1, inv_freq=A << 5, positions=None), **kw)
    err = C.create_string_buffer(256)
    assert B.load().ps_rope_append(C.byref(B.PsRopeArgs(**f)), None, err, 256) == B.PS_ERR_INVALID
    text = err.value.decode()
    assert text.startswith("ps_rope_append: ") and ("overlap" in text) != ("positions" in text), text
    return "overlap" if "overlap" in text else "positions"


FUSED = QW + 2 * KW              # q, k and v side by side
BASE = dict(q=(0, FUSED), k=(QW, FUSED), v=(QW + KW, FUSED), q_out=(5000, QW), k_out=(9000, KW))


@pytest.mark.parametrize("change,want", [
    (dict(), "positions"),
    (dict(q_out=(0, FUSED)), "positions"), (dict(k_out=(QW, FUSED)), "positions"),                 # in place
    (dict(q_out=(0, FUSED), k_out=(QW, FUSED)), "positions"),
    (dict(q_out=(0, QW)), "overlap"), (dict(q_out=(0, FUSED + 1)), "overlap"),                     # q by another stride
    (dict(q_out=(1, FUSED)), "overlap"), (dict(q_out=(D, FUSED)), "overlap"),                      # a part of q, of k
    (dict(q_out=(FUSED, FUSED)), "overlap"), (dict(q_out=((T - 1) * FUSED, FUSED)), "overlap"),    # a token later, the last
    (dict(q_out=(T * FUSED, FUSED)), "positions"), (dict(q_out=(QW, FUSED)), "overlap"),
    (dict(k_out=(0, FUSED)), "overlap"), (dict(k_out=(QW + KW, FUSED)), "overlap"),                # q, v
    (dict(k_out=(5000, KW)), "overlap"), (dict(k_out=(5000 + QW * T - 1, KW)), "overlap"), (dict(k_out=(5000 + QW * T, KW)), "positions"),
    (dict(q_out=(5000, QW - 1)), "overlap"), (dict(q_out=(5000, 0)), "overlap"), (dict(k_out=(9000, -KW + 1)), "overlap"),
    (dict(q=(0, 0), q_out=(0, 0)), "overlap"), (dict(q=(0, 0)), "positions"), (dict(q=(0, 0), q_out=(0, QW)), "overlap"),
    (dict(q=(3 * FUSED, -FUSED), q_out=(3 * FUSED, -FUSED)), "positions"),
])
def test_layouts(change, want):
    assert answer({**BASE, **change}) == want


def test_what_is_not_read_does_not_count():
    """v without pools, one token's strides."""
    assert answer({**BASE, "k_out": (QW + KW, FUSED)}, append=False) == "positions"
    assert answer({**BASE, "q_out": (0, 5)}, tokens=1) == "positions"
    assert answer({**BASE, "q_out": (QW - 1, 5)}, tokens=1) == "overlap"
    assert answer(dict(q=(0, QW), q_out=(0, QW)), append=False) == "positions"
    assert answer(dict(q=(0, QW), q_out=(1, QW)), append=False) == "overlap"
    assert answer(dict(k=(0, KW), k_out=(2 * KW, 3 * KW)), append=False) == "overlap"
    assert answer(dict(k=(0, 3 * KW), k_out=(KW, 3 * KW)), append=False) == "positions"


def test_against_sets_of_elements():
    rng = random.Random(1)
    seen = {"overlap": 0, "positions": 0}
    for _ in range(6000):
        tokens = rng.choice([1, 2, 3, 5, 9])
        width = dict(q=QW, k=KW, v=KW, q_out=QW, k_out=KW)
        one = rng.choice([QW, FUSED, 4 * FUSED])
        rows = {}
        for name in width:
            stride = one if rng.random() < 0.7 else rng.choice([0, 1, KW, QW, FUSED, 2 * FUSED, -FUSED, rng.randint(-300, 300)])
            rows[name] = (rng.choice([rng.randint(2000, 2600), 2000 + rng.randint(0, 40) * KW, rng.randint(2000, 9000)]), stride)
        if rng.random() < 0.3:
            rows["q_out"] = rows["q"]
        if rng.random() < 0.3:
            rows["k_out"] = rows["k"]
        if rng.random() < 0.2:
            del rows["k_out"]

        def elements(name):
            at, stride = rows[name]
            return [at + t * stride + e for t in range(tokens) for e in range(width[name])]

        bad = False
        for out in ("q_out", "k_out"):
            if out in rows:
                el = elements(out)
                bad |= len(set(el)) < len(el)
                own = {"q_out": "q", "k_out": "k"}[out]
                for other in rows:
                    same = other == own and rows[own][0] == rows[out][0] and (rows[own][1] == rows[out][1] or tokens == 1)
                    if other != out and not same:
                        bad |= not set(el).isdisjoint(elements(other))
        want = "overlap" if bad else "positions"
        seen[want] += 1
        assert answer(rows, tokens) == want, rows
    assert min(seen.values()) > 500, seen


@pytest.mark.parametrize("batch,q,out,want", [
    (3, (0, 512), (1536, 512), False), (3, (0, 512), (1528, 512), True), (3, (0, 512), (0, 512), False), (3, (0, 512), (0, 520), True),
    (3, (0, 512), (8, 512), True), (3, (0, 1024), (512, 1024), False), (3, (0, 1024), (504, 1024), True), (3, (0, 0), (512, 512), False),
    (3, (0, 0), (0, 512), True), (1, (0, 8), (0, 16), False), (1, (0, 8), (504, 512), True), (40, (512, 2048), (0, 512), True),
    (3, (512, 1536), (1024, 1536), False)])
def test_attention_in_place_and_beside(batch, q, out, want):
    a = B.PsPagedAttnArgs(kpool=A << 1, vpool=A << 2, q=A + 2 * q[0], out=A + 2 * out[0], q_stride=q[1], out_stride=out[1], block_tables=A, ctx_lens=A,
                          workspace=A, workspace_bytes=0, k_block_stride=1 << 14, v_block_stride=1 << 14, batch=batch, table_stride=4,
                          num_kv_heads=2, num_q_heads=4, head_dim=128, block_size=16, num_gpu_blocks=4)
    err = C.create_string_buffer(256)
    rc = B.load().ps_paged_attn(C.byref(a), None, err, 256)
    text = err.value.decode()
    assert (rc == B.PS_ERR_INVALID and "overlaps q" in text) == want
    if not want:
        assert rc == B.PS_ERR_CUDA or "workspace" in text, text          # no device, or one
