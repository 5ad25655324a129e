"""Decode attention over caches held in 4 bits where a wave takes several tiles of a piece, all of them complete, or paged ones of which not every block exists.

24 sequences of 8 KV heads are cut into four pieces each, three or four steps of 128 rows long, so that every wave has three or four tiles: complete ones, and then one
behind whose rows the table ends, or names no block.  Tolerances as in test_gpu_decode_fp4.py.  Before every call the same launch runs over empty
caches: its workgroups leave zeros and minus infinities in LDS, which read as a mask of rows would drop live ones."""
import itertools

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import fp4_oracle as fo
from paper_2605_23258_amd import binding as vb
from paper_2605_23258_amd import datagen as dg
from paper_2605_23258_amd import pipeline as pl
from test_gpu_decode_fp4 import NEAR, U, Problem, dev, unrotate

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = [("bf16", 128, 4), ("bf16", 64, 2), ("bf16", 128, 7), ("bf16", 64, 16), ("f32", 128, 3), ("f32", 64, 1)]      # type, dims, query heads per KV head
B, H = 24, 8
LOW_HIGH = np.array(fo.MAGNITUDES + tuple(-m for m in fo.MAGNITUDES))[np.arange(256)[:, None] >> [0, 4] & 15]      # the two elements of a byte of codes


def values(rows):
    """fo.values by a table: (codes [n, d / 2], scales [n, d / 32]) -> [n, d]."""
    codes, scales = rows
    return (LOW_HIGH[codes].reshape(-1, fo.BLOCK) * np.ldexp(1.0, scales.reshape(-1, 1).astype(int) - 127)).reshape(len(codes), 2 * codes.shape[1])


def to_dev(x, dtype):
    return dev(x) if dtype == "f32" else dev(dg.f32_to_bf16_bits(x).view(np.int16)).view(torch.bfloat16)


def wide(x, dtype):
    return x.astype(np.float64) if dtype == "f32" else dg.widen(dg.f32_to_bf16_bits(x))


class Long(Problem):
    """24 sequences of `lens` live rows, paged or one block of `cap` rows after the other; every row of the pools has values, those that are no row's as well."""

    def __init__(self, lens, cap, block_rows, dtype, d, G, n_apx=0, seed=0, layout="paged", turned=None):
        rng = np.random.default_rng(seed)
        self.B, self.H, self.G, self.d, self.dtype, self.layout, self.rope, self.block_rows = B, H, G, d, dtype, layout, None, block_rows
        self.lens, self.caps, self.n_apx, self.scale = np.array(lens, dtype=np.int32), [cap] * B, n_apx, 1.0 / np.sqrt(d)
        per_seq = -(-cap // block_rows) if layout == "paged" else 0
        self.n_blocks = B * H * per_seq + 3
        self.table = rng.permutation(self.n_blocks)[:B * H * per_seq].reshape(B, H, per_seq).astype(np.int32)
        self.ret0, self.apx0 = [b * H * cap for b in range(B)], [b * H * n_apx for b in range(B)]
        n_rows = self.n_blocks * block_rows if layout == "paged" else B * H * cap
        rnd = lambda *s: rng.standard_normal(s).astype(np.float32)
        q, W, kn, vn = rnd(B, H * G, d), rnd(H, d, d) / np.float32(np.sqrt(d)), rnd(B, H, d), 3 * rnd(B, H, d)
        self.q_dev, self.W_dev, self.k_new, self.v_new = (to_dev(x, dtype) for x in (q, W, kn, vn))
        self.q, self.W = wide(q, dtype), wide(W, dtype)
        self.new = [fo.quantise(wide(x, dtype)) for x in (kn, vn)]
        some = lambda n: (rng.integers(0, 256, (n, d // 2), dtype=np.uint8), rng.integers(124, 128, (n, d // 32), dtype=np.uint8))
        self.rows = [some(n_rows), some(n_rows), some(max(B * H * n_apx, 1))]
        self.pools = [(dev(c), dev(s)) for c, s in self.rows]
        self.live, self.table_dev = dev(self.lens), dev(self.table)
        c = self.cache = vb.CacheFp4(batch=B, n_q_heads=H * G, n_kv_heads=H, head_dim=d, dtype=vb.VECTOR_BF16 if dtype == "bf16" else vb.VECTOR_F32, cap_retain=cap, n_approx=n_apx)
        c.len_retain, c.W = self.live.data_ptr(), self.W_dev.data_ptr()
        (c.k_ret, c.k_ret_scale), (c.v_ret, c.v_ret_scale), (c.k_apx, c.k_apx_scale) = ((a.data_ptr(), s.data_ptr()) for a, s in self.pools)
        if layout == "paged":
            c.ret_block_table, c.ret_block_rows, c.ret_blocks_per_seq, c.n_blocks = self.table_dev.data_ptr(), block_rows, per_seq, self.n_blocks
        if layout == "sequences":
            self.keep = [dev(np.array(x, dtype=t)) for x, t in ((self.caps, np.int32), ([n_apx] * B, np.int32), (self.ret0, np.int64), (self.apx0, np.int64))]
            c.cap_retain_seq, c.n_approx_seq, c.ret_row_start, c.apx_row_start = (x.data_ptr() for x in self.keep)
        if turned:
            self.interleaved, self.inv_freq = turned == "next", dg.rotary_inv_freq(d, 500000.0)
            pos = np.sort(rng.integers(0, 60000, (B, H, n_apx)), -1).astype(np.int32) if turned != "in order" else np.tile(np.arange(n_apx, dtype=np.int32), (B, H, 1))
            self.pos, self.pos_dev = pos + 5, dev(pos)
            self.rope, self.freq = vb.make_rope(self.inv_freq, None if turned == "in order" else self.pos_dev, self.interleaved, 5)
        self.ws = pl.alloc_workspace(vb.vector_decode_fp4_workspace_bytes(c))

    def set_table(self):
        self.table_dev.copy_(dev(self.table))

    def expected(self, step=False):
        """(result, how far it may be off), [B, Hq, d]: the rows of blocks that exist."""
        H, G, d = self.H, self.G, self.d
        out, tol = np.zeros((B, H, G, d)), np.zeros((B, H, G, d))
        for b, h in itertools.product(range(B), range(H)):
            at = np.arange(self.lens[b])
            ids = self.table[b, h, at // self.block_rows] if self.layout == "paged" else 0 * at
            at = self.pool_rows(b, h, at)[(ids >= 0) & (ids < self.n_blocks)]
            k, v = (values((c[at], s[at])) for c, s in self.rows[:2])
            if step:
                k, v = (np.concatenate((x, values((c[b, h][None], s[b, h][None])))) for x, (c, s) in zip((k, v), self.new))
            own = (b * H + h) * self.n_apx + np.arange(self.n_apx)
            ka = values((self.rows[2][0][own], self.rows[2][1][own]))
            k = np.concatenate((k, ka))
            if self.rope is not None:
                ka = unrotate(ka, self.pos[b, h], self.inv_freq, self.interleaved)
            size = np.abs(ka) @ np.abs(self.W[h])
            turned = np.concatenate((0 * v, size if self.rope is not None else 0 * size))
            size, v = np.concatenate((np.abs(v), size)), np.concatenate((v, ka @ self.W[h]))
            n = len(k)
            if n == 0:
                continue
            q = self.q[b, h * G:(h + 1) * G]
            s = self.scale * (q @ k.T)
            p = np.exp(s - s.max(axis=1, keepdims=True))
            p /= p.sum(axis=1, keepdims=True)
            A = self.scale * (np.abs(q) @ np.abs(k).T).max(axis=1, keepdims=True)
            rel = 2 * (d * U * A + 4 * U * 3 * A * 1.45 + 2 * U) + (2.0 ** -16 if self.dtype == "bf16" else 2.0 ** -22) + (n + 2 * d) * U
            out[b, h], tol[b, h] = p @ v, rel * (p @ size) + (2.0 ** -17 + (2.0 ** -8 + NEAR if self.dtype == "bf16" else 0)) * (p @ turned) + 1e-37
        return out.reshape(B, H * G, d), tol.reshape(B, H * G, d)

    def check(self, step):
        """The result, and that no row but the stored tokens' has changed."""
        self.live.zero_()
        self.call()
        self.live.copy_(dev(self.lens))
        got = self.call(step).cpu().numpy()
        want, tol = self.expected(step)
        bad = ~(np.abs(got - want) <= tol)
        assert not bad.any(), f"{bad.any(axis=(1, 2)).sum()} sequences off, the first {np.argmax(bad.any(axis=(1, 2)))}, worst {np.nanmax(np.abs(got - want) / tol):.3g} of the tolerance"
        stored = {}
        if step:
            assert np.array_equal(self.live.cpu().numpy(), np.minimum(self.lens + 1, self.caps))
            for b, h in itertools.product(range(B), range(H)):
                if self.lens[b] < self.caps[b] and (self.layout != "paged" or 0 <= self.table[b, h, self.lens[b] // self.block_rows] < self.n_blocks):
                    stored[int(self.pool_rows(b, h, np.array([self.lens[b]]))[0])] = (b, h)
        at = np.array(sorted(stored), dtype=np.int64)
        for i, (rows, pool) in enumerate(zip(self.rows, self.pools)):
            for j in range(2):
                want_rows = rows[j].copy()
                if i < 2 and len(at):
                    want_rows[at] = [self.new[i][j][stored[r]] for r in at]
                assert np.array_equal(want_rows, pool[j].cpu().numpy()), "rows that were none of the step's changed, or the token is not there"


def lengths(*ends):
    """Sequences that end as asked for, one after the other, and three short ones."""
    lens = [ends[i % len(ends)] for i in range(B)]
    lens[5], lens[6], lens[7] = 0, 1, 77
    return lens


@pytest.mark.parametrize("dtype,d,G", KINDS)
@pytest.mark.parametrize("step", [False, True])
def test_an_odd_number_of_small_blocks_in_use_to_the_last(dtype, d, G, step):
    """101 blocks of 16 rows: the last tile begins in the last block, and its second half is behind the table."""
    Long(lengths(1610, 1601, 1615, 1600, 1584, 1593), 1616, 16, dtype, d, G, seed=1).check(step)


@pytest.mark.parametrize("dtype,d,G", KINDS)
@pytest.mark.parametrize("block_rows", [16, 32, 64])
@pytest.mark.parametrize("step", [False, True])
def test_a_table_with_no_ids_behind_the_live_rows(dtype, d, G, block_rows, step):
    """As a table is that begins as -1 everywhere and whose requests ask for the blocks they need."""
    p = Long(lengths(1610, 1553, 1500, 1425, 1039, 1535), 2048, block_rows, dtype, d, G, seed=2)
    for b in range(B):
        p.table[b, :, -(-(p.lens[b] + step) // block_rows):] = -1
    p.set_table()
    p.check(step)


@pytest.mark.parametrize("dtype,d,G", KINDS)
@pytest.mark.parametrize("block_rows", [16, 32, 128])
def test_a_block_that_is_missing_in_the_middle_of_a_piece(dtype, d, G, block_rows):
    p = Long(lengths(1600, 1511, 1311), 1664, block_rows, dtype, d, G, n_apx=40, seed=3)
    rng = np.random.default_rng(block_rows)
    for b, h in itertools.product(range(0, B, 2), range(0, H, 3)):
        p.table[b, h, rng.choice(1300 // block_rows, 2, replace=False)] = -1, p.n_blocks
    p.set_table()
    p.check(False)


@pytest.mark.parametrize("dtype,d,G", KINDS)
@pytest.mark.parametrize("block_rows,cap", [(16, 1600), (16, 1616), (16, 1607), (64, 1600), (32, 1568), (128, 1536)])
def test_a_step_on_full_caches(dtype, d, G, block_rows, cap):
    """The token is attended, behind the table or between the capacity and the end of its block, and not stored."""
    Long(lengths(cap, cap, cap - 1, cap - 32), cap, block_rows, dtype, d, G, seed=4).check(True)


@pytest.mark.parametrize("dtype,d,G", KINDS)
@pytest.mark.parametrize("block_rows", [16, 32, 64])
def test_a_step_whose_token_has_no_block(dtype, d, G, block_rows):
    """As after a request for a block that was refused: the token is the first row of a block that the table does not name."""
    p = Long(lengths(1536, 1408 + block_rows, 1216, 1343), 1600, block_rows, dtype, d, G, seed=5)
    for b in range(B):
        p.table[b, :, -(-p.lens[b] // block_rows):] = -1
    p.set_table()
    p.check(True)


@pytest.mark.parametrize("dtype,d,G", KINDS[:2] + KINDS[4:5])
def test_prompts_and_refused_steps_on_a_table_that_begins_without_ids(dtype, d, G):
    """Tables from vector_block_tables on a table of -1, blocks of 16 rows, until the free list is used up; rows by the slots."""
    R, per_seq = 16, 101
    p = Long(lengths(1504, 1600, 1488, 1567), per_seq * R, R, dtype, d, G, seed=6)
    need, T = H * sum(-(-int(n) // R) for n in p.lens), int(p.lens.sum())
    free = dev(np.random.default_rng(6).permutation(p.n_blocks).astype(np.int32))[:need + 5 * H]        # five of the sequences that ask for a block get one
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)
    held, live, grown, counts, slots = i32(B), i32(B), i32(B), i32(3), torch.empty(H, T, dtype=torch.int64, device=DEV)
    p.table_dev.fill_(-1)
    vb.vector_block_tables(vb.make_blocks(p.live, H, R, per_seq, free, held=held), p.table_dev, live, slots, counts)
    assert counts.tolist() == [need, need, T] and torch.equal(live, p.live)
    # rows by their slots: of values of the format, which stay what they are
    shape = vb.Shape(n_q_heads=H, n_kv_heads=H, head_dim=d, seq_len=T, window=1, pool_kernel=1, dtype=p.cache.dtype)
    rng = np.random.default_rng(7)
    k, v = (to_dev(rng.standard_normal((H, T, d)).astype(np.float32), dtype) for _ in range(2))
    vb.vector_store_fp4(shape, k, v, slots, p.n_blocks * R, *p.pools[0], *p.pools[1])
    p.rows = [(c.cpu().numpy(), s.cpu().numpy()) for c, s in p.pools]
    first = int(p.lens[:9].sum())
    rows = slots[3, first:first + int(p.lens[9])].cpu().numpy()
    codes, scales = fo.quantise(k[3, first:first + int(p.lens[9])].double().cpu().numpy())
    assert np.array_equal(p.rows[0][0][rows], codes) and np.array_equal(p.rows[0][1][rows], scales)
    # the next token of every sequence
    used, wanted = counts[:1].clone(), live + 1
    vb.vector_block_tables(vb.make_blocks(wanted, H, R, per_seq, free, held=live, used=used), p.table_dev, grown, None, counts)
    assert counts[0].item() == 5 * H and int((grown == live).sum()) >= 4
    p.table = p.table_dev.cpu().numpy()
    p.check(True)


@pytest.mark.parametrize("dtype,d,G", KINDS)
@pytest.mark.parametrize("layout", ["blocks", "sequences", "paged"])
@pytest.mark.parametrize("step", [False, True])
def test_complete_tiles(dtype, d, G, layout, step):
    """Of retained rows and of approximated ones; lengths that end in every wave's tile, 16-row blocks."""
    Long(lengths(1610, 1601, 1535, 1500, 1472, 1441), 1664, 16, dtype, d, G, n_apx=[1000, 777][step], seed=8, layout=layout).check(step)


@pytest.mark.parametrize("dtype,d,G", KINDS)
@pytest.mark.parametrize("turned", ["apart", "next", "in order"])
def test_complete_tiles_of_keys_turned_back(dtype, d, G, turned):
    Long(lengths(400, 333), 512, 16, dtype, d, G, n_apx=1100, seed=9, layout=["blocks", "paged"][G % 2], turned=turned).check(False)


PEAKS = {                                              # magnitudes of every element of the keys that stand out, by the step of 128 rows that they are in
    "first": {0: 1.5, 3: 1.5, 6: 1.5, 9: 1.5},         # of every piece: no score behind it comes near
    "last": {2: 1.5, 5: 1.5, 8: 1.5, 12: 1.5},
    "growing": {0: 1.0, 1: 2.0, 2: 4.0, 4: 1.5, 5: 3.0, 7: 2.0, 8: 4.0, 10: 2.0, 11: 4.0, 12: 6.0},
    "falling": {0: 6.0, 1: 4.0, 2: 2.0, 3: 3.0, 4: 1.5, 9: 4.0, 10: 2.0},
}


@pytest.mark.parametrize("dtype,d,G", KINDS)
@pytest.mark.parametrize("peaks", PEAKS)
@pytest.mark.parametrize("layout", ["blocks", "paged"])
def test_largest_scores_in_one_tile_or_another(dtype, d, G, peaks, layout):
    """Every wave has a row in the tiles named whose score lies 12 (17 powers of two) above the others for every 1.5 of its key's magnitude, so that sums that are
    there already are weighted anew, in the first tile, the last one or each.  Their values are 0: the result is what is left of the others' sums."""
    p = Long([1610] * B, 1616, 16, dtype, d, G, seed=10, layout=layout)
    signs = np.sign(np.random.default_rng(11).standard_normal((B, H, 1, d)))
    p.q = (np.abs(p.q.reshape(B, H, G, d)) * signs).reshape(B, H * G, d)     # (the values stay those of the type)
    p.q_dev = to_dev(p.q.astype(np.float32), dtype)
    p.scale = float(np.float32(12.0 / 1.5 / np.abs(p.q).sum(axis=-1).mean()))
    (codes, scales), (v_codes, _) = p.rows[:2]
    scales -= 3
    for b, h in itertools.product(range(B), range(H)):
        half = np.where(signs[b, h, 0] < 0, 8, 0)
        for at, size in PEAKS[peaks].items():
            x = half | fo.MAGNITUDES.index(size)
            rows = p.pool_rows(b, h, np.array([r for r in 128 * at + 32 * np.arange(4) + 7 if r < 1610]))
            codes[rows], scales[rows], v_codes[rows] = x[0::2] | x[1::2] << 4, 127, 0
    for to, x in zip(p.pools[0] + p.pools[1][:1], (codes, scales, v_codes)):
        to.copy_(dev(x))
    p.check(False)
