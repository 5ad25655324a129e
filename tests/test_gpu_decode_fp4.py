"""Decode attention over caches held in 4 bits against the 64-bit oracle on the values that the codes stand for.

How far the fp32 result may be off, per element, by arithmetic (u = 2^-24, half a step of fp32; B = sum_t p_t |v_t|, for approximated rows
with |k| |W| in the place of |v|; n rows; all first-order, worst case):
  scores    sums of d products in fp32: d u A with A the largest |scale| sum |q k| of a row; times log2(e) and the difference from the
            reference round once each: 4 u (A + spread), spread <= 2 A; exp2 of the hardware is good to 2 u.  A weight is off by
            twice that in the worst case, since numerator and sum may go apart
  weights   bf16: two parts of 8 bits, 2^-16; fp32: three, 2^-22 (their exponents end at 2^-126, far below)
  sums      fp32 over n rows, and d products with W: (n + 2 d) u
  turned    keys un-rotated: angle and hardware sine and cosine 2^-17 together; bf16: rounded to 8 bits on the way, 2^-8
A bf16 output is the rounding of the fp32 one, bit for bit."""
import itertools

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import fp4_oracle as fo
from paper_2605_23258_amd import binding as vb
from paper_2605_23258_amd import datagen as dg
from paper_2605_23258_amd import pipeline as pl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


# bf16: turns of a row from those of one near it, 64 away at most.  The difference to a whole turn is taken in numbers below 128, off by 2^-18, and the
# frequency is a float, off by 2^-25 of itself, 2^-19 in 64 turns: together 2 pi (2^-18 + 2^-19) of the pair's length
NEAR = 2 * np.pi * (2.0 ** -18 + 2.0 ** -19)


class Problem:
    """Caches of `lens` live retained rows and n_apx approximated rows per sequence in one of three layouts, with junk (NaN blocks
    among it) in every row that is none."""

    def __init__(self, lens, n_apx, H=2, G=4, d=128, dtype="bf16", layout="blocks", room=3, block_rows=16, rope=False, interleaved=False, positions=True, spread=None, seed=0,
                 q_size=1.0, scale=None, caps=None):
        rng = np.random.default_rng(seed)
        self.B, self.H, self.G, self.d, self.dtype, self.layout = len(lens), H, G, d, dtype, layout
        B = self.B
        self.lens = np.array(lens, dtype=np.int32)
        apx = list(n_apx) if layout == "sequences" else [n_apx] * B
        if caps is None:
            caps = [n + room for n in lens] if layout == "sequences" else [max(lens) + room] * B
        self.caps, self.apx = caps, apx
        self.scale = scale if scale is not None else 1.0 / np.sqrt(d)
        half = dg.f32_to_bf16_bits
        t = lambda x: dev(x) if dtype == "f32" else dev(half(x).view(np.int16)).view(torch.bfloat16)
        w = lambda x: x.astype(np.float64) if dtype == "f32" else dg.widen(half(x))
        rnd = lambda *s: rng.standard_normal(s).astype(np.float32)
        q = rnd(B, H * G, d) * np.float32(q_size)
        W = rnd(H, d, d) / np.float32(np.sqrt(d))
        self.q_dev, self.W_dev, self.q, self.W = t(q), t(W), w(q), w(W)
        kn, vn = rnd(B, H, d), rnd(B, H, d) * 3
        self.k_new, self.v_new = t(kn), t(vn)
        self.new = [fo.quantise(w(x)) for x in (kn, vn)]
        # rows of the segments, sequence by sequence
        rows = lambda n: [fo.quantise(rnd(H, n, d) * np.where(rng.random((H, n, 1)) < 0.05, 4, 1) * 2.0 ** rng.uniform(-2, 2, (H, n, 1))) for _ in range(2)]
        self.ret = [rows(n) for n in lens]
        self.kapx = [rows(n)[0] for n in apx]
        junk = lambda n: (rng.integers(0, 256, (n, d // 2), dtype=np.uint8), np.where(rng.random((n, d // 32)) < 0.5, 255, rng.integers(0, 255, (n, d // 32))).astype(np.uint8))
        self.table = None
        if layout == "paged":
            per_seq = -(-caps[0] // block_rows) if caps[0] else 1
            n_blocks = B * H * per_seq + 3
            self.table = rng.permutation(n_blocks)[:B * H * per_seq].reshape(B, H, per_seq).astype(np.int32)
            self.block_rows, self.n_blocks = block_rows, n_blocks
            n_rows = n_blocks * block_rows
        else:
            n_rows = max(H * sum(caps), 1)
        self.ret0, self.apx0 = [H * sum(caps[:b]) for b in range(B)], [H * sum(apx[:b]) for b in range(B)]
        pools = [junk(n_rows), junk(n_rows), junk(max(H * sum(apx), 1))]
        for b in range(B):
            for h in range(H):
                at = self.pool_rows(b, h, np.arange(lens[b]))
                for pool, part in zip(pools, self.ret[b]):
                    pool[0][at], pool[1][at] = part[0][h], part[1][h]
                at = self.apx0[b] + h * apx[b] + np.arange(apx[b])
                pools[2][0][at], pools[2][1][at] = self.kapx[b][0][h], self.kapx[b][1][h]
        self.pools = [(dev(c), dev(s)) for c, s in pools]
        self.live = dev(self.lens)
        c = vb.CacheFp4(batch=B, n_q_heads=H * G, n_kv_heads=H, head_dim=d, dtype=vb.VECTOR_BF16 if dtype == "bf16" else vb.VECTOR_F32, cap_retain=max(caps), n_approx=max(apx))
        c.len_retain, c.W = self.live.data_ptr(), self.W_dev.data_ptr()
        (c.k_ret, c.k_ret_scale), (c.v_ret, c.v_ret_scale), (c.k_apx, c.k_apx_scale) = ((a.data_ptr(), s.data_ptr()) for a, s in self.pools)
        self.keep = []
        if layout == "sequences":
            self.keep = [dev(np.array(x, dtype=np.int32)) for x in (caps, apx)] + [dev(np.array(x, dtype=np.int64)) for x in (self.ret0, self.apx0)]
            c.cap_retain_seq, c.n_approx_seq, c.ret_row_start, c.apx_row_start = (x.data_ptr() for x in self.keep)
        if layout == "paged":
            self.table_dev = dev(self.table)
            c.ret_block_table, c.ret_block_rows, c.ret_blocks_per_seq, c.n_blocks = self.table_dev.data_ptr(), block_rows, self.table.shape[2], self.n_blocks
        self.cache = c
        self.rope = self.inv_freq = self.pos = None
        self.interleaved = interleaved
        if rope:
            self.inv_freq = dg.rotary_inv_freq(d, 500000.0)
            offset = 5
            pos = [np.sort(rng.integers(0, 60000, (H, n)), -1).astype(np.int32) if positions else np.tile(np.arange(n, dtype=np.int32), (H, 1)) for n in apx]
            if spread:
                pos = [np.stack([spread(rng, n) for _ in range(H)]).astype(np.int32) for n in apx]
            self.pos = [x + offset for x in pos]
            flat = dev(np.concatenate([x.reshape(-1) for x in pos])) if positions and sum(apx) else None
            self.rope, keep = vb.make_rope(self.inv_freq, flat, interleaved, offset)
            self.keep.append((keep, flat))
        self.ws = pl.alloc_workspace(vb.vector_decode_fp4_workspace_bytes(c))

    def pool_rows(self, b, h, at):
        if self.layout == "paged":
            return self.table[b, h, at // self.block_rows].astype(np.int64) * self.block_rows + at % self.block_rows
        return self.ret0[b] + h * self.caps[b] + at

    def expected(self, step=False):
        """(result, how far it may be off), [B, Hq, d]."""
        H, G, d = self.H, self.G, self.d
        out, tol = np.zeros((self.B, H * G, d)), np.zeros((self.B, H * G, d))
        bf16 = self.dtype == "bf16"
        for b in range(self.B):
            for h in range(H):
                k, v = (fo.values(c[h], s[h]) for c, s in self.ret[b])
                if step:
                    k, v = (np.concatenate((x, fo.values(c[b, h], s[b, h])[None])) for x, (c, s) in zip((k, v), self.new))
                ka = fo.values(self.kapx[b][0][h], self.kapx[b][1][h])
                n = len(k) + len(ka)
                if n == 0:
                    continue
                k = np.concatenate((k, ka))
                if self.rope is not None and len(ka):
                    ka = unrotate(ka, self.pos[b][h], self.inv_freq, self.interleaved)
                va = ka @ self.W[h]
                size = np.concatenate((np.abs(v), np.abs(ka) @ np.abs(self.W[h])))
                turned = np.concatenate((np.zeros_like(v), np.abs(ka) @ np.abs(self.W[h]))) if self.rope is not None else 0 * size
                v = np.concatenate((v, va))
                for g in range(G):
                    q = self.q[b, h * G + g]
                    s = (k @ q) * self.scale
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    A = np.abs(self.scale) * (np.abs(k) @ np.abs(q)).max()
                    rel = 2 * (d * U * A + 4 * U * 3 * A * 1.45 + 2 * U) + (2.0 ** -16 if bf16 else 2.0 ** -22) + (n + 2 * d) * U
                    out[b, h * G + g] = p @ v
                    tol[b, h * G + g] = rel * (p @ size) + (2.0 ** -17 + (2.0 ** -8 + NEAR if bf16 else 0)) * (p @ turned) + 1e-37
        return out, tol

    def call(self, step=False, out=None, flags=vb.VECTOR_DECODE_OUT_F32, stream=None):
        f32 = self.dtype == "f32" or flags & vb.VECTOR_DECODE_OUT_F32
        out = torch.full((self.B, self.H * self.G, self.d), 7.0, dtype=torch.float32 if f32 else torch.bfloat16, device=DEV) if out is None else out
        if step:
            vb.vector_decode_step_fp4(self.cache, self.q_dev, self.k_new, self.v_new, self.scale, out, self.ws, rope=self.rope, flags=flags, stream=stream)
        else:
            vb.vector_decode_attn_fp4(self.cache, self.q_dev, self.scale, out, self.ws, rope=self.rope, flags=flags, stream=stream)
        return out

    def check(self, step=False, what=""):
        before = [x.clone() for pair in self.pools for x in pair]
        got = self.call(step).cpu().numpy()
        torch.cuda.synchronize()
        want, tol = self.expected(step)
        err = np.abs(got - want)
        assert (err <= tol).all(), f"{what}: {np.sum(~(err <= tol))} of {err.size} off, worst {np.nanmax(err / tol):.2f} of the tolerance"
        after = [x.cpu().numpy() for pair in self.pools for x in pair]
        if step:
            # the new row is in the cache, nothing else has changed, the lengths have grown where there was room
            for b in range(self.B):
                if self.lens[b] < self.caps[b]:
                    for h in range(self.H):
                        at = self.pool_rows(b, h, np.array([self.lens[b]]))[0]
                        for i, (c, s) in enumerate(self.new):
                            assert np.array_equal(after[2 * i][at], c[b, h]) and np.array_equal(after[2 * i + 1][at], s[b, h]), what
                            before[2 * i][at], before[2 * i + 1][at] = dev(c[b, h]), dev(s[b, h])
            assert np.array_equal(self.live.cpu().numpy(), np.minimum(self.lens + 1, self.caps)), what
        for x, y in zip(after, before):
            assert np.array_equal(x, y.cpu().numpy()), f"{what}: rows that were none of the step's changed"
        if self.dtype == "bf16":
            if step:
                self.live.copy_(dev(self.lens))
            bits = pl.to_host(self.call(step, flags=0))
            assert np.array_equal(bits, dg.f32_to_bf16_bits(got)), f"{what}: the bf16 output is not the rounding of the fp32 one"
        return got


def unrotate(k, pos, inv_freq, interleaved):
    """Rows k [n, d] turned back by their positions."""
    n, d = k.shape
    z = (k[:, 0::2] + 1j * k[:, 1::2]) if interleaved else (k[:, :d // 2] + 1j * k[:, d // 2:])
    z = z * np.exp(-1j * pos[:, None].astype(np.float64) * inv_freq[None])
    out = np.empty_like(k)
    if interleaved:
        out[:, 0::2], out[:, 1::2] = z.real, z.imag
    else:
        out[:, :d // 2], out[:, d // 2:] = z.real, z.imag
    return out


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 255, 300, 511, 640]


@pytest.mark.parametrize("dtype,d", itertools.product(["bf16", "f32"], [64, 128]))
@pytest.mark.parametrize("layout,block_rows", [("blocks", 0), ("sequences", 0), ("paged", 16), ("paged", 32), ("paged", 128)])
@pytest.mark.parametrize("step", [False, True])
def test_lengths(dtype, d, layout, block_rows, step):
    """Twenty sequences of every kind of length at once, retained rows alone and with approximated ones."""
    apx = [0, 1, 31, 32, 33, 64, 100] * 3
    for some in (False, True):
        n_apx = (apx[:20] if some else [0] * 20) if layout == "sequences" else (45 if some else 0)
        Problem(LENGTHS, n_apx, dtype=dtype, d=d, G=3, layout=layout, block_rows=block_rows, seed=d + some).check(step, f"approximated {some}")


@pytest.mark.parametrize("dtype,d", itertools.product(["bf16", "f32"], [64, 128]))
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 16])
def test_query_heads(dtype, d, G):
    Problem([150, 33, 0], 70, G=G, dtype=dtype, d=d, seed=G).check(True)


@pytest.mark.parametrize("dtype,d", itertools.product(["bf16", "f32"], [64, 128]))
@pytest.mark.parametrize("interleaved,positions", [(False, True), (True, True), (False, False)])
@pytest.mark.parametrize("G", [4, 12])
def test_keys_turned_back(dtype, d, interleaved, positions, G):
    kw = dict(dtype=dtype, d=d, G=G, rope=True, interleaved=interleaved, positions=positions)
    Problem([40, 3], 130, **kw).check()
    Problem([40, 0, 77], [33, 200, 0], layout="sequences", **kw).check(True)
    Problem([40, 3], 0, **kw).check()                    # nothing to turn back


SPREADS = {
    "dense": lambda rng, n: np.sort(rng.choice(4 * n, n, replace=False)),
    "one in thirty": lambda rng, n: 30 * np.arange(n) + rng.integers(0, 30, n),      # about as far as near goes
    "jumps": lambda rng, n: np.arange(n) + (np.arange(n) // 37) * 100_000,           # most tiles near, some not
    "any order": lambda rng, n: rng.permutation(n),
    "the same": lambda rng, n: np.full(n, 777),
    "far": lambda rng, n: np.sort(rng.integers(0, 2 ** 24 - 6, n)),
    "far and dense": lambda rng, n: np.arange(2 ** 24 - 6 - n, 2 ** 24 - 6),
}


@pytest.mark.parametrize("dtype,d", itertools.product(["bf16", "f32"], [64, 128]))
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("spread", SPREADS)
def test_positions_near_and_far(dtype, d, interleaved, spread):
    kw = dict(dtype=dtype, d=d, rope=True, interleaved=interleaved, spread=SPREADS[spread])
    Problem([40, 3], 300, G=4, **kw).check()
    Problem([5, 0], [77, 260], G=2, layout="sequences", **kw).check(True)


@pytest.mark.parametrize("dtype,G", [("bf16", 4), ("bf16", 16), ("f32", 3)])
def test_one_map_for_all_heads(dtype, G):
    p = Problem([40, 3], 90, H=3, G=G, dtype=dtype)
    p.W[1:] = p.W[0]
    p.W_dev = p.W_dev[:1].contiguous()
    p.cache.W, p.cache.w_shared = p.W_dev.data_ptr(), 1
    p.check(True)


@pytest.mark.parametrize("d", [64, 128])
def test_many_splits(d):
    """One pair of long segments cut into many pieces, and many pairs."""
    Problem([5000], 3001, H=1, G=4, d=d).check(True)
    Problem([700, 20] * 20, 300, H=3, G=2, d=d).check()


@pytest.mark.parametrize("layout", ["blocks", "sequences", "paged"])
def test_full_blocks(layout):
    """A block that is full: the token is attended, not stored, and the length stays."""
    lens = [48, 17, 0]
    p = Problem(lens, [5, 0, 9] if layout == "sequences" else 9, layout=layout, caps=[48, 18, 0] if layout == "sequences" else [48] * 3)
    p.check(True)


def test_nothing_cached_gives_zeros():
    for kw in (dict(n_apx=0), dict(n_apx=[0, 0], layout="sequences"), dict(n_apx=0, layout="paged")):
        p = Problem([0, 0], caps=[0, 0] if kw.get("layout") != "paged" else [32, 32], **kw)
        assert (p.call().cpu().numpy() == 0).all()
    got = Problem([0, 5], 0).check()
    assert (got[0] == 0).all()


def test_blocks_that_do_not_exist_hold_no_rows():
    """Entries below zero and beyond the pool: their rows take no part, a step's token in one is attended and not stored."""
    for block_rows in (16, 64):
        p = Problem([300, 64, 130], 20, layout="paged", block_rows=block_rows, room=70)
        gone = []
        for b, h, c in ((0, 0, 0), (0, 1, 2), (2, 0, 1), (1, 1, 64 // block_rows)):
            p.table[b, h, c] = -1 if c % 2 else p.n_blocks
            gone.append((b, h, c))
        p.table_dev.copy_(dev(p.table))
        real = [[tuple(list(x) for x in pair) for pair in seg] for seg in p.ret]
        for b, h, c in gone:
            rows = np.arange(p.lens[b])
            keep = (rows // block_rows) != c
            for i in range(2):
                codes, scales = real[b][i]
                real[b][i] = ([x if hh != h else x[keep] for hh, x in enumerate(codes)], [x if hh != h else x[keep] for hh, x in enumerate(scales)])
        p.ret = real
        before = [x.clone() for pair in p.pools for x in pair]
        got = p.call(True).cpu().numpy()
        torch.cuda.synchronize()
        want, tol = p.expected(True)
        assert (np.abs(got - want) <= tol).all()
        # the token of (1, 1) had no block: its row is in none
        new = p.new[0][0][1, 1]
        assert not (p.pools[0][0].cpu().numpy() == new).all(-1).any() and (p.pools[0][0].cpu().numpy() == p.new[0][0][1, 0]).all(-1).any()
        assert sum(int((x != y).any(-1).sum()) for x, y in zip(before[:1], [p.pools[0][0]])) <= 2 * 3 - 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sizes_of_scores(dtype):
    """Peaked and flat rows: scores far apart (a row's largest comes late, or first), all alike, all below zero by far."""
    for q_size, scale in ((40.0, None), (1e-3, None), (1.0, 0.0), (1.0, -3.0), (300.0, 0.01)):
        Problem([333, 40], 100, dtype=dtype, q_size=q_size, scale=scale).check(False, f"{q_size} {scale}")


def test_a_nan_block_reaches_its_own_head_only():
    p = Problem([100, 70], 30)
    p.pools[1][1][p.pool_rows(0, 1, np.array([57]))[0], 2] = 255        # values, dims 64 .. 95
    p.pools[0][1][p.pool_rows(1, 0, np.array([3]))[0], 0] = 255         # a key: every score of it
    got = p.call().cpu().numpy().reshape(2, 2, 4, 128)
    want, tol = p.expected()
    nan = np.zeros(got.shape, bool)
    nan[0, 1, :, 64:96] = True
    nan[1, 0] = True
    assert np.isnan(got[nan]).all() and (np.abs(got - want.reshape(got.shape)) <= tol.reshape(got.shape))[~nan].all()


def test_the_same_bits_every_time_and_on_another_stream():
    p = Problem([500, 33, 1200], 700, G=5)
    first = p.call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = p.call(stream=side)
    side.synchronize()
    assert torch.equal(first, second)


def test_step_is_store_and_attend():
    """The step gives what storing the row and attending give, bit for bit where the work is cut alike."""
    p = Problem([63, 100], 40, room=5)
    got = p.call(True)
    shape = vb.Shape(n_q_heads=2, n_kv_heads=2, head_dim=128, seq_len=2, window=1, pool_kernel=1, dtype=vb.VECTOR_BF16)
    r = Problem([63, 100], 40, room=5)
    slots = np.array([[r.pool_rows(b, h, np.array([r.lens[b]]))[0] for b in range(2)] for h in range(2)], dtype=np.int64)
    k, v = (x.transpose(0, 1).contiguous() for x in (r.k_new, r.v_new))
    vb.vector_store_fp4(shape, k, v, dev(slots), r.pools[0][0].shape[0], *r.pools[0], *r.pools[1])
    r.live.add_(1)
    again = r.call()
    torch.cuda.synchronize()
    assert torch.equal(p.pools[0][0], r.pools[0][0]) and torch.equal(p.pools[1][1], r.pools[1][1])
    assert torch.equal(got, again)


def test_captured_steps():
    """A captured step is replayed; every replay is held against the eager step."""
    make = lambda: Problem([30, 0, 95], 20, layout="paged", block_rows=32, room=10)
    eager, graphed = make(), make()
    rng = np.random.default_rng(9)
    tokens = [[dev(rng.standard_normal(x.shape).astype(np.float32)).bfloat16() for x in (eager.q_dev, eager.k_new, eager.v_new)] for _ in range(5)]
    out = torch.empty(3, 8, 128, device=DEV)
    warm = make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm.call(True, out=out, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.call(True, out=out, stream=torch.cuda.current_stream())
    for i, new in enumerate(tokens):
        for p in (eager, graphed):
            for to, x in zip((p.q_dev, p.k_new, p.v_new), new):
                to.copy_(x)
        want = eager.call(True)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), f"replay {i}"
        assert torch.equal(eager.live, graphed.live)
        for x, y in zip(eager.pools, graphed.pools):
            assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])


def test_serving_from_prompts_to_steps():
    """The operators one after the other, as a serving loop has them: blocks for the prompts, their rows by the slots, steps whose tokens get
    their blocks on the GPU; against attention over the rounded rows in 64 bits."""
    rng = np.random.default_rng(2)
    H, G, d, R, per_seq, B, steps = 2, 4, 128, 16, 8, 3, 20
    lens = np.array([37, 16, 90], dtype=np.int32)
    half = lambda *s: dev(dg.f32_to_bf16_bits(rng.standard_normal(s).astype(np.float32)).view(np.int16)).view(torch.bfloat16)
    T = int(lens.sum())
    n_blocks = B * H * per_seq
    pool = [torch.full((n_blocks * R, n), 255, dtype=torch.uint8, device=DEV) for n in (d // 2, d // 32, d // 2, d // 32)]
    free = dev(rng.permutation(n_blocks).astype(np.int32))
    table, live = torch.zeros(B, H, per_seq, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    counts, wanted, slots = torch.zeros(3, dtype=torch.int32, device=DEV), dev(lens), torch.empty(H, T, dtype=torch.int64, device=DEV)
    vb.vector_block_tables(vb.make_blocks(wanted, H, R, per_seq, free), table, live, slots, counts)
    k, v = half(H, T, d), half(H, T, d)
    shape = vb.Shape(n_q_heads=H, n_kv_heads=H, head_dim=d, seq_len=T, window=1, pool_kernel=1, dtype=vb.VECTOR_BF16)
    vb.vector_store_fp4(shape, k, v, slots, n_blocks * R, *pool)
    start = np.concatenate(([0], np.cumsum(lens)))
    rounded = lambda x: fo.values(*fo.quantise(x.float().cpu().numpy()))
    rows = [[[rounded(x[:, start[b]:start[b + 1]])[h] for h in range(H)] for x in (k, v)] for b in range(B)]
    cache = vb.CacheFp4(batch=B, n_q_heads=H * G, n_kv_heads=H, head_dim=d, dtype=vb.VECTOR_BF16, cap_retain=per_seq * R, n_approx=0)
    (cache.k_ret, cache.k_ret_scale, cache.v_ret, cache.v_ret_scale) = (x.data_ptr() for x in pool)
    cache.ret_block_table, cache.ret_block_rows, cache.ret_blocks_per_seq, cache.n_blocks = table.data_ptr(), R, per_seq, n_blocks
    ws = pl.alloc_workspace(vb.vector_decode_fp4_workspace_bytes(cache))
    out = torch.empty(B, H * G, d, device=DEV)
    taken = counts[0].item()
    grown, held = live.clone(), torch.zeros_like(live)
    for s in range(steps):
        # the next token of every sequence: its block first, then the step, which advances `live` itself
        held.copy_(live)
        torch.add(live, 1, out=wanted)
        vb.vector_block_tables(vb.make_blocks(wanted, H, R, per_seq, free[taken:], held=held), table, grown, None, counts)
        taken += counts[0].item()
        cache.len_retain = live.data_ptr()
        q, kn, vn = half(B, H * G, d), half(B, H, d), half(B, H, d)
        vb.vector_decode_step_fp4(cache, q, kn, vn, 1 / np.sqrt(d), out, ws, flags=vb.VECTOR_DECODE_OUT_F32)
        torch.cuda.synchronize()
        assert torch.equal(live, grown)
        got = out.cpu().numpy()
        for b in range(B):
            for i, new in enumerate((rounded(kn), rounded(vn))):
                rows[b][i] = [np.concatenate((rows[b][i][h], new[b, h][None])) for h in range(H)]
            for h in range(H):
                kk, vv = rows[b][0][h], rows[b][1][h]
                for g in range(G):
                    x = kk @ q[b, h * G + g].double().cpu().numpy() / np.sqrt(d)
                    p = np.exp(x - x.max())
                    p /= p.sum()
                    assert (np.abs(got[b, h * G + g] - p @ vv) <= 2.0 ** -14 * (p @ np.abs(vv)) + 1e-30).all(), f"step {s}"
    assert taken == H * sum(-(-(n + steps) // R) for n in lens) and live.tolist() == (lens + steps).tolist()


@pytest.mark.parametrize("d,G,rope", [(128, 4, False), (128, 4, True), (64, 2, False), (64, 5, True), (128, 16, False), (128, 10, True)])
@pytest.mark.parametrize("layout", ["blocks", "sequences", "paged16", "paged64"])
def test_sequences_of_different_lengths(d, G, rope, layout):
    """Enough rows by the capacities for the cuts that the device makes; the live lengths are anything."""
    rng = np.random.default_rng(d + G)
    lens = [int(x) for x in rng.integers(0, 700, 24)]
    lens[3], lens[4], lens[11], lens[23] = 0, 1, 1500, 0
    apx = [int(x) for x in rng.integers(0, 90, 24)]
    apx[0], apx[4], apx[23] = 0, 200, 0
    kw = dict(H=8, G=G, d=d, rope=rope, interleaved=G == 10, layout="paged" if layout.startswith("paged") else layout, room=100, block_rows=64 if layout == "paged64" else 16)
    p = Problem(lens, apx if layout == "sequences" else 40, **kw)
    if layout == "sequences":
        p.cache.cap_retain, p.cache.n_approx = 1 << 20, max(apx)
    p.check(True, layout)


def test_queries_that_are_not_finite_stay_in_their_head():
    for bad in (float("inf"), float("nan"), float("-inf")):
        for d, G in ((128, 4), (128, 7), (128, 12), (64, 4)):
            p = Problem([60, 5], 40, d=d, G=G)
            p.q_dev[1, G + 1, 17] = bad
            got = p.call().cpu().numpy()
            want, tol = p.expected()
            assert np.isnan(got[1, G + 1]).all()
            got[1, G + 1] = want[1, G + 1]
            assert (np.abs(got - want) <= tol).all()


def test_rows_far_into_a_pool():
    """Pools of 2^26 + 64 rows, 4 GiB of codes each: blocks that begin beyond 2^32 bytes, and the step's row among them."""
    small = Problem([70, 33], 0, layout="paged", block_rows=32, room=20)
    rows = (1 << 26) + 64 * 8
    big = Problem([70, 33], 0, layout="paged", block_rows=32, room=20)
    first = (1 << 26) // 32 - 6
    pools = []
    for codes, scales in small.pools[:2]:
        c, s = torch.zeros(rows, 64, dtype=torch.uint8, device=DEV), torch.zeros(rows, 4, dtype=torch.uint8, device=DEV)
        at = slice(first * 32, first * 32 + codes.shape[0])
        c[at], s[at] = codes, scales
        pools.append((c, s))
    big.table_dev.copy_(dev(small.table + first))
    big.cache.n_blocks = rows // 32
    (big.cache.k_ret, big.cache.k_ret_scale), (big.cache.v_ret, big.cache.v_ret_scale) = ((c.data_ptr(), s.data_ptr()) for c, s in pools)
    want, got = small.call(True), big.call(True)
    torch.cuda.synchronize()
    assert torch.equal(want, got)
    for (c, s), (c2, s2) in zip(small.pools[:2], pools):
        at = slice(first * 32, first * 32 + c.shape[0])
        assert torch.equal(c, c2[at]) and torch.equal(s, s2[at])
    # the same rows in one contiguous segment that begins beyond 2^32 bytes
    far = Problem([70], [0], H=1, layout="sequences", caps=[100])
    start = (1 << 26) + 7
    moved = []
    for codes, scales in far.pools[:2]:
        c, s = torch.zeros(rows, 64, dtype=torch.uint8, device=DEV), torch.zeros(rows, 4, dtype=torch.uint8, device=DEV)
        c[start:start + 100], s[start:start + 100] = codes, scales
        moved.append((c, s))
    want = far.call()
    far.keep[2].fill_(start)
    (far.cache.k_ret, far.cache.k_ret_scale), (far.cache.v_ret, far.cache.v_ret_scale) = ((c.data_ptr(), s.data_ptr()) for c, s in moved)
    assert torch.equal(want, far.call())


def test_a_captured_serving_loop_without_the_host():
    """Blocks for the next tokens and the step over them in one graph, replayed: lengths, tables and the place in the free list advance on the
    GPU.  Against the same calls made eagerly."""
    rng = np.random.default_rng(4)
    H, G, d, R, per_seq, B, steps = 2, 4, 128, 16, 6, 5, 24
    half = lambda *s: dev(dg.f32_to_bf16_bits(rng.standard_normal(s).astype(np.float32)).view(np.int16)).view(torch.bfloat16)
    n_blocks = B * H * per_seq
    free = dev(rng.permutation(n_blocks).astype(np.int32))
    tokens = [(half(B, H * G, d), half(B, H, d), half(B, H, d)) for _ in range(steps)]

    class Loop:
        def __init__(self):
            i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)
            self.pool = [torch.full((n_blocks * R, n), 255, dtype=torch.uint8, device=DEV) for n in (d // 2, d // 32, d // 2, d // 32)]
            self.table, self.live, self.held, self.wanted, self.grown, self.counts, self.used = i32(B, H, per_seq), i32(B), i32(B), i32(B), i32(B), i32(3), i32(1)
            self.q, self.k, self.v = (torch.zeros_like(x) for x in tokens[0])
            self.out = torch.zeros(B, H * G, d, device=DEV)
            c = self.cache = vb.CacheFp4(batch=B, n_q_heads=H * G, n_kv_heads=H, head_dim=d, dtype=vb.VECTOR_BF16, cap_retain=per_seq * R, n_approx=0)
            c.k_ret, c.k_ret_scale, c.v_ret, c.v_ret_scale = (x.data_ptr() for x in self.pool)
            c.len_retain, c.ret_block_table, c.ret_block_rows, c.ret_blocks_per_seq, c.n_blocks = self.live.data_ptr(), self.table.data_ptr(), R, per_seq, n_blocks
            self.ws = pl.alloc_workspace(vb.vector_decode_fp4_workspace_bytes(c))
            self.blocks = vb.make_blocks(self.wanted, H, R, per_seq, free, held=self.held, used=self.used)

        def step(self, stream):
            self.held.copy_(self.live)
            torch.add(self.live, 1, out=self.wanted)
            vb.vector_block_tables(self.blocks, self.table, self.grown, None, self.counts, stream=stream)
            self.used.add_(self.counts[:1])
            vb.vector_decode_step_fp4(self.cache, self.q, self.k, self.v, 1 / np.sqrt(d), self.out, self.ws, flags=vb.VECTOR_DECODE_OUT_F32, stream=stream)

    eager, graphed, warm = Loop(), Loop(), Loop()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm.step(side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step(torch.cuda.current_stream())
    for i, token in enumerate(tokens):
        for loop in (eager, graphed):
            for to, x in zip((loop.q, loop.k, loop.v), token):
                to.copy_(x)
        eager.step(None)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name in ("out", "live", "table", "used", "grown"):
            assert torch.equal(getattr(eager, name), getattr(graphed, name)), f"step {i}: {name}"
        assert eager.live.tolist() == [i + 1] * B and eager.used.item() == B * H * (-(-(i + 1) // R))
