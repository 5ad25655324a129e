"""What the entry points of 4-bit caches and block tables refuse, on the host: the addresses are never read.  No GPU needed."""
import ctypes as C

import pytest

from paper_2605_23258_amd import binding as vb

SOME = 4096                                            # an address that nothing may use
ARG, SHAPE, WORKSPACE, DTYPE = vb.VECTOR_ERR_ARG, vb.VECTOR_ERR_SHAPE, vb.VECTOR_ERR_WORKSPACE, vb.VECTOR_ERR_DTYPE


def shape(**kw):
    s = dict(n_q_heads=4, n_kv_heads=2, head_dim=128, seq_len=100, window=1, pool_kernel=1, dtype=vb.VECTOR_BF16)
    s.update(kw)
    return vb.Shape(**s)


def test_struct_layouts():
    assert C.sizeof(vb.Blocks) == 6 * 4 + 4 * 8
    assert C.sizeof(vb.CacheFp4) == 8 * 4 + 8 * 8 + 4 * 8 + 8 + 4 * 4


def blocks(**kw):
    b = dict(batch=3, n_kv_heads=2, block_rows=16, blocks_per_seq=8, n_free=10, len=SOME, free_blocks=SOME)
    b.update(kw)
    return vb.Blocks(**b)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), SHAPE), (dict(batch=4097), SHAPE), (dict(n_kv_heads=0), SHAPE), (dict(n_kv_heads=65536), SHAPE), (dict(block_rows=8), ARG),
    (dict(block_rows=24), ARG), (dict(block_rows=-16), ARG), (dict(blocks_per_seq=0), ARG), (dict(n_free=-1), ARG), (dict(len=None), ARG),
    (dict(batch=4096, n_kv_heads=1024, blocks_per_seq=512), SHAPE), (dict(len=2 * SOME), ARG), (dict(len_held=2 * SOME), ARG),
    (dict(n_used=SOME), ARG), (dict(batch=4096, n_kv_heads=16385, blocks_per_seq=1), SHAPE)])
def test_block_tables(kw, code):
    assert vb.lib().vector_block_tables(C.byref(blocks(**kw)), SOME, 2 * SOME, None, 0, SOME, None) == code


@pytest.mark.parametrize("at,value", [(0, None), (1, None), (4, None), (3, -1), (3, 2 ** 31 - 1)])
def test_block_tables_outputs(at, value):
    args = [SOME, 2 * SOME, SOME, 5, SOME]
    args[at] = value
    assert vb.lib().vector_block_tables(C.byref(blocks()), *args, None) == ARG
    assert vb.lib().vector_block_tables(None, SOME, 2 * SOME, SOME, 5, SOME, None) == ARG
    assert vb.lib().vector_block_tables(C.byref(blocks()), SOME, 2 * SOME, None, 5, SOME, None) == ARG       # columns of no map


@pytest.mark.parametrize("kw,code", [(dict(head_dim=96), SHAPE), (dict(dtype=2), DTYPE), (dict(n_kv_heads=0), SHAPE), (dict(seq_len=0), SHAPE),
                                     (dict(k_stride_tok=130), SHAPE), (dict(v_stride_tok=64), SHAPE), (dict(k_stride_head=-8), SHAPE)])
def test_shapes_of_rows(kw, code):
    L = vb.lib()
    assert L.vector_compact_fp4(C.byref(shape(**kw)), SOME, SOME, SOME, SOME, 1, 1, *([SOME] * 6), 1, None) == code
    assert L.vector_store_fp4(C.byref(shape(**kw)), SOME, SOME, SOME, 10, *([SOME] * 4), None) == code


def test_compact():
    L, s = vb.lib(), shape()
    call = lambda n_r, n_a, cap, args: L.vector_compact_fp4(C.byref(s), *args[:4], n_r, n_a, *args[4:], cap, None)
    good = [SOME] * 10
    for n_r, n_a, cap in ((-1, 0, 5), (0, -1, 5), (10, 5, 9), (60, 41, 60)):
        assert call(n_r, n_a, cap, good) == ARG
    for i in range(10):
        for bad in (None, SOME + 8):
            if i in (2, 3) and bad:                     # the lists need no alignment
                continue
            args = list(good)
            args[i] = bad
            assert call(5, 5, 5, args) == ARG, i
    assert L.vector_compact_fp4(None, *([SOME] * 4), 1, 1, *([SOME] * 6), 1, None) == ARG


def test_store():
    L, s = vb.lib(), shape(seq_len=1 << 22)            # longer than one sequence may be
    good = [SOME, SOME, SOME, 10, SOME, SOME, SOME, SOME]
    for i, bad in [(0, None), (0, SOME + 2), (1, SOME + 2), (1, None), (2, None), (3, -1), (4, None), (4, SOME + 4), (5, None), (6, None), (7, SOME + 1)]:
        args = list(good)
        args[i] = bad
        assert L.vector_store_fp4(C.byref(s), *args, None) == ARG, (i, bad)
    assert L.vector_store_fp4(None, *good, None) == ARG
    assert L.vector_store_fp4(C.byref(shape(seq_len=(1 << 28) + 1)), *good, None) == SHAPE


def test_load():
    L = vb.lib()
    good = [5, 128, vb.VECTOR_BF16, SOME, SOME, 10, None, SOME]
    for i, bad, code in [(0, -1, ARG), (0, (1 << 29) + 1, SHAPE), (1, 32, SHAPE), (2, 2, DTYPE), (3, None, ARG), (3, SOME + 4, ARG), (4, None, ARG), (4, SOME + 4, ARG), (5, -1, ARG),
                         (7, None, ARG), (7, SOME + 8, ARG)]:
        args = list(good)
        args[i] = bad
        assert L.vector_load_fp4(*args, None) == code, (i, bad)
    assert L.vector_load_fp4(0, *good[1:], None) == 0   # nothing to do


def cache(**kw):
    c = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=vb.VECTOR_BF16, cap_retain=10, n_approx=5, len_retain=SOME, k_ret=SOME,
             k_ret_scale=SOME, v_ret=SOME, v_ret_scale=SOME, k_apx=SOME, k_apx_scale=SOME, W=SOME)
    c.update(kw)
    return vb.CacheFp4(**c)


def attn(c, q=SOME, scale=1.0, out=SOME, flags=0, ws=SOME, ws_bytes=1 << 40, rope=None):
    return vb.lib().vector_decode_attn_fp4(C.byref(c) if c else None, C.byref(rope) if rope else None, q, scale, out, flags, ws, ws_bytes, None)


def step(c, k_new=SOME, v_new=SOME):
    return vb.lib().vector_decode_step_fp4(C.byref(c), None, SOME, k_new, v_new, 1.0, SOME, 0, SOME, 1 << 40, None)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), SHAPE), (dict(batch=65536), SHAPE), (dict(n_q_heads=9), SHAPE), (dict(n_q_heads=22), SHAPE), (dict(n_q_heads=1), SHAPE), (dict(head_dim=96), SHAPE),
    (dict(dtype=3), DTYPE), (dict(cap_retain=-1), ARG), (dict(n_approx=-1), ARG),
    (dict(cap_retain=(1 << 30) + 1), SHAPE), (dict(n_approx=(1 << 30) + 1), SHAPE)])
def test_cache_shapes(kw, code):
    c = cache(**kw)
    assert attn(c) == code and step(c) == code and vb.vector_decode_fp4_workspace_bytes(c) == 0


@pytest.mark.parametrize("name", ["len_retain", "k_ret", "k_ret_scale", "v_ret", "v_ret_scale", "k_apx", "k_apx_scale", "W"])
def test_cache_memory(name):
    assert attn(cache(**{name: None})) == ARG
    if name != "len_retain":
        assert attn(cache(**{name: SOME + 8})) == ARG


def test_decode_arguments():
    assert attn(None) == ARG
    for kw in (dict(q=None), dict(out=None), dict(q=SOME + 4), dict(out=SOME + 4), dict(flags=4), dict(flags=-1 & ~1), dict(scale=float("nan"))):
        assert attn(cache(), **kw) == ARG, kw
    assert attn(cache(), flags=vb.VECTOR_DECODE_LITERAL) == DTYPE
    need = vb.vector_decode_fp4_workspace_bytes(cache())
    assert need > 0 and attn(cache(), ws_bytes=need - 1) == WORKSPACE and attn(cache(), ws=None) == WORKSPACE and attn(cache(), ws=SOME + 16) == WORKSPACE
    for kw in (dict(k_new=None), dict(v_new=None), dict(k_new=SOME + 2), dict(v_new=SOME + 2)):
        assert step(cache(), **kw) == ARG
    assert step(cache(cap_retain=0)) == ARG


def test_layouts():
    arrays = dict(cap_retain_seq=SOME, n_approx_seq=SOME, ret_row_start=SOME, apx_row_start=SOME)
    for name in arrays:
        assert attn(cache(**{k: v for k, v in arrays.items() if k != name})) == ARG
    paged = dict(ret_block_table=SOME, ret_block_rows=16, ret_blocks_per_seq=4, n_blocks=8)
    for bad in (dict(ret_block_rows=8), dict(ret_block_rows=20), dict(ret_blocks_per_seq=0), dict(n_blocks=-1), dict(cap_retain=65), arrays):
        assert attn(cache(**{**paged, **bad})) == ARG, bad


def test_rotary_arguments():
    rope, keep = vb.make_rope([1.0] * 64)
    bad = vb.Rope()
    assert attn(cache(), rope=bad) == ARG
    rope.pos_offset = 1 << 24
    assert attn(cache(), rope=rope) == ARG
    rope, keep = vb.make_rope([float("nan")] * 64)
    assert attn(cache(), rope=rope) == ARG
