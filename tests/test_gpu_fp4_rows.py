"""Rows into 4 bits and back against the oracle, bit for bit: codes and scales are whole numbers."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import fp4_oracle as fo
from paper_2605_23258_amd import binding as vb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def host_rows(rng, shape, spread=6.0):
    """Rows whose blocks differ by many octaves, with what is special planted."""
    x = (rng.standard_normal(shape) * 2.0 ** rng.uniform(-spread, spread, shape[:-1] + (1,))).astype(np.float32)
    flat = x.reshape(-1, shape[-1])
    n = len(flat)
    flat[0, :8] = [0.25, -0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0]
    flat[0, 8:] = 0.0
    flat[n // 3] = 0.0
    flat[n // 2, :32] *= np.float32(2.0 ** -100)
    flat[n // 2, 3] = 1e-40
    flat[2 * n // 3, 32:64] = 3e38
    flat[n - 1, 5] = np.inf
    flat[n // 4, 40] = np.nan
    return x


def to_dtype(x, dtype):
    t = torch.from_numpy(x).to(DEV)
    return t.bfloat16() if dtype == "bf16" else t


def wide(t):
    return t.float().cpu().numpy().astype(np.float64)


def vdt(dtype):
    return vb.VECTOR_BF16 if dtype == "bf16" else vb.VECTOR_F32


def bytes_full(*shape):
    return torch.full(shape, 0xA5, dtype=torch.uint8, device=DEV)


def check_rows(codes, scales, ref, what):
    want_codes, want_scales = fo.quantise(ref)
    assert np.array_equal(scales, want_scales), f"{what}: scales"
    assert np.array_equal(codes, want_codes), f"{what}: codes"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,H,n,n_r,n_a,room", [(128, 2, 300, 77, 51, 5), (64, 3, 131, 40, 0, 0), (128, 1, 1, 1, 0, 3), (64, 2, 77, 0, 33, 2), (128, 8, 2049, 333, 700, 1)])
def test_compact(dtype, d, H, n, n_r, n_a, room):
    rng = np.random.default_rng(d + n)
    k, v = (to_dtype(host_rows(rng, (H, n, d)), dtype) for _ in range(2))
    lists = np.argsort(rng.random((H, n)), axis=1).astype(np.int32)
    idx_r, idx_a = np.sort(lists[:, :n_r], 1), np.sort(lists[:, n_r:n_r + n_a], 1)
    cap = n_r + room
    out = {x: (bytes_full(H, max(rows, 1), d // 2), bytes_full(H, max(rows, 1), d // 32)) for x, rows in (("k_ret", cap), ("v_ret", cap), ("k_apx", n_a))}
    shape = vb.Shape(n_q_heads=H, n_kv_heads=H, head_dim=d, seq_len=n, window=1, pool_kernel=1, dtype=vdt(dtype))
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV) if x.size else None
    vb.vector_compact_fp4(shape, k, v, dev(idx_r), dev(idx_a), n_r, n_a, *out["k_ret"], *out["v_ret"], *out["k_apx"], cap)
    torch.cuda.synchronize()
    at = np.arange(H)[:, None]
    for x, src, idx in (("k_ret", k, idx_r), ("v_ret", v, idx_r), ("k_apx", k, idx_a)):
        codes, scales = (t.cpu().numpy() for t in out[x])
        m = idx.shape[1]
        if m:
            check_rows(codes[:, :m], scales[:, :m], wide(src)[at, idx], x)
        assert (codes[:, m:] == 0xA5).all() and (scales[:, m:] == 0xA5).all(), f"{x}: rows behind the last were touched"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_compact_reads_strided_rows_and_passes_over_foreign_indices(dtype, d):
    rng = np.random.default_rng(5)
    H, n, n_r = 2, 50, 9
    packed = to_dtype(host_rows(rng, (n, 3, H, d)), dtype)            # tokens first, [q, k, v] side by side
    k, v = packed[:, 1], packed[:, 2]
    idx = np.sort(np.argsort(rng.random((H, n)), 1)[:, :n_r].astype(np.int32), 1)
    idx[0, 4], idx[1, 0] = n, -1
    shape = vb.Shape(n_q_heads=H, n_kv_heads=H, head_dim=d, seq_len=n, window=1, pool_kernel=1, dtype=vdt(dtype),
                     k_stride_head=d, k_stride_tok=3 * H * d, v_stride_head=d, v_stride_tok=3 * H * d)
    out = [bytes_full(H, n_r, d // 2), bytes_full(H, n_r, d // 32), bytes_full(H, n_r, d // 2), bytes_full(H, n_r, d // 32)]
    vb.vector_compact_fp4(shape, k, v, torch.from_numpy(idx).to(DEV), None, n_r, 0, *out, None, None, n_r)
    torch.cuda.synchronize()
    codes, scales = out[2].cpu().numpy(), out[3].cpu().numpy()
    there = (idx >= 0) & (idx < n)
    rows = wide(v).transpose(1, 0, 2)[np.arange(H)[:, None], np.clip(idx, 0, n - 1)]
    want_codes, want_scales = fo.quantise(rows)
    assert np.array_equal(codes[there], want_codes[there]) and np.array_equal(scales[there], want_scales[there])
    assert (codes[~there] == 0xA5).all() and (scales[~there] == 0xA5).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,H,T,with_v", [(128, 2, 1, True), (64, 3, 100, True), (128, 1, 517, False), (64, 1, 2, False), (128, 8, 33, True)])
def test_store_and_load(dtype, d, H, T, with_v):
    rng = np.random.default_rng(T)
    rows = H * T + 40
    k, v = (to_dtype(host_rows(rng, (H, T, d)), dtype) for _ in range(2))
    slots = rng.permutation(rows)[:H * T].reshape(H, T).astype(np.int64)
    if T > 2:                                           # no slot: padding, behind the pool, far out
        slots[0, 1], slots[-1, T - 1], slots[0, 0] = -1, rows, 1 << 40
    pools = [bytes_full(rows, d // 2), bytes_full(rows, d // 32), bytes_full(rows, d // 2), bytes_full(rows, d // 32)]
    shape = vb.Shape(n_q_heads=H, n_kv_heads=H, head_dim=d, seq_len=T, window=1, pool_kernel=1, dtype=vdt(dtype))
    at = torch.from_numpy(slots).to(DEV)
    vb.vector_store_fp4(shape, k, v if with_v else None, at, rows, *(pools if with_v else pools[:2]))
    torch.cuda.synchronize()
    ok = (slots >= 0) & (slots < rows)
    untouched = np.setdiff1d(np.arange(rows), slots[ok])
    for src, codes, scales in ((k, pools[0], pools[1]), (v, pools[2], pools[3])):
        c, s = codes.cpu().numpy(), scales.cpu().numpy()
        if src is v and not with_v:
            assert (c == 0xA5).all() and (s == 0xA5).all()
            continue
        check_rows(c[slots[ok]], s[slots[ok]], wide(src)[ok], "pool")
        assert (c[untouched] == 0xA5).all() and (s[untouched] == 0xA5).all()
        # and back, in either type, zeros where there is no row
        ref = np.zeros((H, T, d))
        ref[ok] = fo.values(c[slots[ok]], s[slots[ok]])
        for out_type in ("bf16", "f32"):
            out = to_dtype(np.full((H, T, d), 7.0, np.float32), out_type)
            vb.vector_load_fp4(H * T, d, vdt(out_type), codes, scales, rows, at, out)
            torch.cuda.synchronize()
            np.testing.assert_array_equal(wide(out), ref)


@pytest.mark.parametrize("d", [64, 128])
def test_load_gives_every_code_under_every_scale(d):
    """All 16 codes under all 256 scale bytes, NaN and the largest and smallest among them."""
    codes = np.tile(np.arange(d // 2, dtype=np.uint8) % 16 * 17 ^ 0x50, (256, 1))
    codes[:, :16] = np.arange(16, dtype=np.uint8) | (15 - np.arange(16, dtype=np.uint8)) << 4
    scales = np.tile(np.arange(256, dtype=np.uint8)[:, None], (1, d // 32))
    out = torch.full((256, d), 7.0, device=DEV)
    vb.vector_load_fp4(256, d, vb.VECTOR_F32, torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV), 256, None, out)
    torch.cuda.synchronize()
    with np.errstate(over="ignore"):
        want = fo.values(codes, scales).astype(np.float32)      # 2^127 times 2 and more is infinite in 32 bits
    np.testing.assert_array_equal(out.cpu().numpy(), want)


def test_rows_far_into_a_pool():
    """Offsets beyond 2^32 bytes: a pool of 2^26 + 8 rows of 128 elements has 4 GiB of codes."""
    d, rows = 128, (1 << 26) + 8
    codes, scales = torch.zeros(rows, d // 2, dtype=torch.uint8, device=DEV), torch.zeros(rows, d // 32, dtype=torch.uint8, device=DEV)
    x = torch.randn(1, 3, d, device=DEV)
    slots = torch.tensor([[rows - 1, 5, 1 << 26]], device=DEV)
    shape = vb.Shape(n_q_heads=1, n_kv_heads=1, head_dim=d, seq_len=3, window=1, pool_kernel=1, dtype=vb.VECTOR_F32)
    vb.vector_store_fp4(shape, x, None, slots, rows, codes, scales)
    out = torch.empty(3, d, device=DEV)
    vb.vector_load_fp4(3, d, vb.VECTOR_F32, codes, scales, rows, slots, out)
    torch.cuda.synchronize()
    want = fo.quantise(wide(x)[0])
    np.testing.assert_array_equal(wide(out), fo.values(*want))
    assert np.array_equal(codes[slots[0]].cpu().numpy(), want[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_store_reads_strided_rows(dtype, d):
    """Tokens first, queries, keys and values of a token side by side."""
    rng = np.random.default_rng(6)
    H, T = 3, 41
    packed = to_dtype(host_rows(rng, (T, 3, H, d)), dtype)
    shape = vb.Shape(n_q_heads=H, n_kv_heads=H, head_dim=d, seq_len=T, window=1, pool_kernel=1, dtype=vdt(dtype),
                     k_stride_head=d, k_stride_tok=3 * H * d, v_stride_head=d, v_stride_tok=3 * H * d)
    slots = rng.permutation(H * T).reshape(H, T)
    pools = [bytes_full(H * T, d // 2), bytes_full(H * T, d // 32), bytes_full(H * T, d // 2), bytes_full(H * T, d // 32)]
    vb.vector_store_fp4(shape, packed[:, 1], packed[:, 2], torch.from_numpy(slots).to(DEV), H * T, *pools)
    torch.cuda.synchronize()
    for src, codes, scales in ((packed[:, 1], *pools[:2]), (packed[:, 2], *pools[2:])):
        check_rows(codes.cpu().numpy()[slots], scales.cpu().numpy()[slots], wide(src).transpose(1, 0, 2), "pool")


def test_load_to_bf16_is_exact_under_every_scale():
    codes = torch.arange(32, dtype=torch.uint8, device=DEV).repeat(256, 1) * 8 + 3
    scales = torch.arange(256, dtype=torch.uint8, device=DEV)[:, None].repeat(1, 2)
    out = torch.full((256, 64), 7.0, device=DEV, dtype=torch.bfloat16)
    vb.vector_load_fp4(256, 64, vb.VECTOR_BF16, codes, scales, 256, None, out)
    torch.cuda.synchronize()
    with np.errstate(over="ignore"):
        want = fo.values(codes.cpu().numpy(), scales.cpu().numpy()).astype(np.float32)
    np.testing.assert_array_equal(out.float().cpu().numpy(), want)


def test_as_many_rows_as_a_call_takes():
    """2^28 tokens (32 GiB of keys), 2^29 rows read back (64 GiB); few of them are somewhere."""
    d, T, rows = 64, 1 << 28, 100
    k = torch.zeros(1, T, d, dtype=torch.bfloat16, device=DEV)
    slots = torch.full((1, T), -1, dtype=torch.int64, device=DEV)
    some = torch.tensor([0, 31, 12345, (1 << 25) + 7, 1 << 27, T - 33, T - 1], device=DEV)
    k[0, some] = torch.randn(len(some), d, device=DEV).bfloat16()
    slots[0, some] = torch.arange(len(some), device=DEV) * 3
    codes, scales = bytes_full(rows, d // 2), bytes_full(rows, d // 32)
    shape = vb.Shape(n_q_heads=1, n_kv_heads=1, head_dim=d, seq_len=T, window=1, pool_kernel=1, dtype=vb.VECTOR_BF16)
    vb.vector_store_fp4(shape, k, None, slots, rows, codes, scales)
    torch.cuda.synchronize()
    at = np.arange(len(some)) * 3
    values = wide(k[0, some])
    check_rows(codes.cpu().numpy()[at], scales.cpu().numpy()[at], values, "pool")
    rest = np.setdiff1d(np.arange(rows), at)
    assert (codes.cpu().numpy()[rest] == 0xA5).all()
    del k
    back = torch.full((2, T), -1, dtype=torch.int64, device=DEV)
    back[1] = slots[0]
    out = torch.full((2, T, d), 7.0, dtype=torch.bfloat16, device=DEV)
    vb.vector_load_fp4(2 * T, d, vb.VECTOR_BF16, codes, scales, rows, back, out)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(wide(out[1, some]), fo.values(codes.cpu().numpy()[at], scales.cpu().numpy()[at]))
    out[1, some] = 0
    assert all(not bool(part.any()) for part in out.view(-1, 1 << 24))
