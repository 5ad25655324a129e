"""Block tables and slot maps against the oracle, entry by entry."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import fp4_oracle as fo
from paper_2605_23258_amd import binding as vb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def dev(x, dtype=torch.int32):
    return None if x is None else torch.as_tensor(np.asarray(x), dtype=dtype, device=DEV)


def run(length, H, R, per_seq, free, n_slots, held, table, stream=None):
    B = len(length)
    d_len, d_free, d_held = dev(length), dev(free if len(free) else [0])[:len(free)], dev(held)
    out = torch.full((B, H, per_seq), -77, dtype=torch.int32, device=DEV) if table is None else dev(table)
    live, counts = torch.full((B,), -77, dtype=torch.int32, device=DEV), torch.full((3,), -77, dtype=torch.int32, device=DEV)
    slots = None if n_slots is None else torch.full((H, n_slots), -77, dtype=torch.int64, device=DEV)
    b = vb.make_blocks(d_len, H, R, per_seq, d_free, held=d_held)
    vb.vector_block_tables(b, out, live, slots, counts, stream)
    torch.cuda.synchronize()
    return out.cpu().numpy(), live.cpu().numpy(), None if slots is None else slots.cpu().numpy(), tuple(counts.tolist())


def check(length, H, R, per_seq, free, n_slots=None, held=None, table=None):
    got = run(length, H, R, per_seq, free, n_slots, held, table)
    want = fo.block_tables(length, H, R, per_seq, free, n_slots=n_slots, held=held, table=table)
    for g, w, what in zip(got, want, ("table", "live", "slots", "counts")):
        if w is None:
            continue
        assert np.array_equal(np.asarray(g), np.asarray(w)), what


@pytest.mark.parametrize("B,H,R,per_seq", [(1, 1, 16, 1), (1, 8, 64, 300), (7, 2, 16, 40), (63, 3, 32, 11), (64, 8, 64, 5), (65, 1, 16, 9), (256, 2, 16, 20), (257, 2, 128, 3),
                                           (1000, 1, 16, 4), (4096, 2, 16, 3)])
@pytest.mark.parametrize("new", [True, False])
@pytest.mark.parametrize("supply", ["enough", "short", "none"])
def test_batches(B, H, R, per_seq, new, supply):
    rng = np.random.default_rng(B * 7 + per_seq)
    most = per_seq * R
    length = rng.integers(0, most + 1, B)
    length[rng.random(B) < 0.1] = 0
    length[rng.random(B) < 0.1] = most
    held = table = None
    if not new:
        held = np.minimum(length, rng.integers(0, most + 1, B))
        same = rng.random(B) < 0.3
        held[same] = length[same]
        table = rng.integers(5000, 9000, (B, H, per_seq)).astype(np.int32)
    wanted = fo.block_tables(length, H, R, per_seq, range(1 << 24), held=held, table=table)[3][1]
    free = rng.permutation(wanted + 9)[:{"enough": wanted, "short": wanted * 2 // 3, "none": 0}[supply]] + 100
    tokens = int((length - (0 if held is None else held)).sum())
    for n_slots in (None, tokens, tokens + 37, tokens // 2, 0):
        if n_slots is not None and H * n_slots > 3_000_000:
            continue
        check(length, H, R, per_seq, free, n_slots, held, table)


def test_lengths_that_ask_for_nothing_or_too_much():
    # below zero, below what is held, longer than the table, as long as the table
    free = list(range(50, 90))
    check([-5, 3, 1000, 64, 2 ** 31 - 1, 17, 0], 2, 16, 4, free, n_slots=100)
    table = np.arange(7 * 2 * 4, dtype=np.int32).reshape(7, 2, 4)
    check([-5, 3, 1000, 64, 2 ** 31 - 1, 17, 0], 2, 16, 4, free, n_slots=200, held=[0, 20, 5, 63, 16, -3, 12], table=table)
    # slots for the first requests only, then a request without new tokens
    check([20, 20, 10], 2, 16, 4, free, n_slots=30, held=[0, 0, 10], table=table[:3])
    # one request at the end of the longest table, a token at a time
    check([2 ** 20], 1, 16, 2 ** 16, list(range(3, 9)), n_slots=1, held=[2 ** 20 - 1], table=np.arange(2 ** 16, dtype=np.int32).reshape(1, 1, -1))


def test_free_blocks_in_order():
    """Without a list the free blocks are 0, 1, 2, .."""
    length = dev([40, 3, 0, 33])
    b = vb.Blocks(batch=4, n_kv_heads=2, block_rows=16, blocks_per_seq=4, n_free=12, len=length.data_ptr())
    table, live, counts = torch.full((4, 2, 4), -7, dtype=torch.int32, device=DEV), torch.empty(4, dtype=torch.int32, device=DEV), torch.empty(3, dtype=torch.int32, device=DEV)
    slots = torch.empty(2, 76, dtype=torch.int64, device=DEV)
    vb.vector_block_tables(b, table, live, slots, counts)
    torch.cuda.synchronize()
    want = fo.block_tables([40, 3, 0, 33], 2, 16, 4, range(12), n_slots=76)
    for g, w in zip((table, live, slots), want):
        assert np.array_equal(g.cpu().numpy(), w)
    assert tuple(counts.tolist()) == want[3]


def test_ids_whose_rows_pass_32_bits():
    """Slots are 64-bit: block 2^30 of 128 rows begins at row 2^37."""
    got = run([5], 1, 128, 1, [1 << 30], 5, None, None)
    assert got[2].tolist() == [[(1 << 37) + i for i in range(5)]]


def test_longest_slot_map():
    """As many columns as there may be, 16 GiB of them; a request that does not fit the last two."""
    n_slots, R = 2 ** 31 - 2, 1 << 20
    length = dev([2 ** 30, 2 ** 30 - 7, 3, 5])
    table, live, counts = torch.full((4, 1, 1024), -7, dtype=torch.int32, device=DEV), torch.empty(4, dtype=torch.int32, device=DEV), torch.empty(3, dtype=torch.int32, device=DEV)
    slots = torch.full((1, n_slots), -7, dtype=torch.int64, device=DEV)
    vb.vector_block_tables(vb.make_blocks(length, 1, R, 1024, 3000), table, live, slots, counts)
    torch.cuda.synchronize()
    assert live.tolist() == [2 ** 30, 2 ** 30 - 7, 3, 0] and counts.tolist() == [2049, 2050, 2 ** 31 - 1]
    full, part = 2 ** 31 - 7, 1 << 28
    for a in range(0, full, part):
        b = min(a + part, full)
        assert bool((slots[0, a:b] == torch.arange(a, b, device=DEV)).all()), a
    assert slots[0, full:].tolist() == [2 ** 31, 2 ** 31 + 1, 2 ** 31 + 2, -1, -1]


def test_replays_and_another_stream():
    """A captured call reads the lengths that the buffers hold then."""
    B, H, R, per_seq = 50, 4, 16, 12
    rng = np.random.default_rng(1)
    free = dev(rng.permutation(4000))
    length, held = dev(np.zeros(B)), dev(np.zeros(B))
    table, live, counts = torch.zeros(B, H, per_seq, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    slots = torch.zeros(H, B * per_seq * R, dtype=torch.int64, device=DEV)
    b = vb.make_blocks(length, H, R, per_seq, free, held=held)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        vb.vector_block_tables(b, table, live, slots, counts, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vb.vector_block_tables(b, table, live, slots, counts, stream=torch.cuda.current_stream())
    for rep in range(4):
        old = rng.integers(0, per_seq * R // 2, B)
        new = old + rng.integers(0, per_seq * R // 2, B)
        start = rng.integers(0, 4000, (B, H, per_seq)).astype(np.int32)
        length.copy_(dev(new)); held.copy_(dev(old)); table.copy_(dev(start))
        slots.fill_(5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = fo.block_tables(new, H, R, per_seq, free.tolist(), n_slots=slots.shape[1], held=old, table=start)
        for g, w in zip((table, live, slots), want):
            assert np.array_equal(g.cpu().numpy(), w)
        assert tuple(counts.tolist()) == want[3]


@pytest.mark.parametrize("listed", [True, False])
def test_blocks_taken_before(listed):
    """Ids from behind those that calls before have taken; a number out of range is the nearest one in it."""
    for used, start in ((0, 0), (5, 5), (12, 12), (40, 30), (-3, 0)):
        ids = list(range(900, 930)) if listed else list(range(30))
        length, n_used = dev([40, 3, 0, 33]), dev([used])
        free = dev(ids)
        b = vb.make_blocks(length, 2, 16, 4, free, used=n_used)
        if not listed:
            b.free_blocks = None
        table, live, counts = torch.full((4, 2, 4), -7, dtype=torch.int32, device=DEV), torch.empty(4, dtype=torch.int32, device=DEV), torch.empty(3, dtype=torch.int32, device=DEV)
        slots = torch.empty(2, 76, dtype=torch.int64, device=DEV)
        vb.vector_block_tables(b, table, live, slots, counts)
        torch.cuda.synchronize()
        want = fo.block_tables([40, 3, 0, 33], 2, 16, 4, ids[start:], n_slots=76)
        for g, w in zip((table, live, slots), want):
            assert np.array_equal(g.cpu().numpy(), w)
        assert tuple(counts.tolist()) == want[3] and n_used.tolist() == [used]
