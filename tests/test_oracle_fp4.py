"""Pins of the oracle of 4-bit rows and block tables: hand-computed codes, the rules by exhaustive search, what the format promises.
No GPU needed."""
import numpy as np
import pytest

from oracle import fp4_oracle as fo


def row(*first):
    x = np.zeros(32)
    x[:len(first)] = first
    return x


def test_codes_by_hand():
    codes, scales = fo.quantise(row(6.0, -0.5, 0.25, 0.26, 1.0, -1.5, 2.5, 5.0))
    # 6 <= 7: scale 1.  0.25 lies between 0 and 0.5 and goes to the even code 0, 2.5 to 2, 5 to 4
    assert scales.tolist() == [127]
    assert codes[:4].tolist() == [7 | 9 << 4, 0 | 1 << 4, 2 | 11 << 4, 4 | 6 << 4]
    np.testing.assert_array_equal(fo.values(codes, scales)[:8], [6.0, -0.5, 0.0, 0.5, 1.0, -1.5, 2.0, 4.0])


@pytest.mark.parametrize("top,byte", [(7.0, 127), (7.0000005, 128), (3.5, 126), (14.0, 128), (0.0, 1), (1e-45, 1), (7 * 2.0 ** -126, 1),
                                      (8 * 2.0 ** -126, 2), (3.4e38, 252), (2.9e38, 252), (np.inf, 255), (np.nan, 255)])
def test_scale_bytes_by_hand(top, byte):
    assert fo.quantise(row(0.0, -top))[1].tolist() == [byte]


def test_against_exhaustive_search():
    """Every code is the nearest one, every scale the smallest that holds, in exact arithmetic."""
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((40, 64)) * 10.0 ** rng.uniform(-30, 30, (40, 1))).astype(np.float32)
    x[0, :8] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0]            # every border, at scale 1
    x[0, 8:32] = 0
    codes, scales = fo.quantise(x)
    half = np.stack((codes & 15, codes >> 4), -1).reshape(x.shape)
    for r in range(x.shape[0]):
        for b in range(2):
            part = x[r, 32 * b:32 * b + 32].astype(np.float64)
            e = fo.scale_exponent(np.abs(part).max())
            assert scales[r, b] == e + 127
            for i, v in enumerate(part):
                assert half[r, 32 * b + i] & 7 == fo.nearest_code(abs(v) * 2.0 ** -e)
                assert half[r, 32 * b + i] >> 3 == np.signbit(v)


def test_what_is_off_by_how_much():
    x = np.random.default_rng(1).standard_normal((200, 128)) * np.exp(np.random.default_rng(2).uniform(-9, 9, (200, 1)))
    codes, scales = fo.quantise(x)
    y = fo.values(codes, scales)
    unit = np.repeat(2.0 ** (scales.astype(float) - 127), 32, axis=-1)
    assert (np.abs(y - x) <= unit).all()                                # at most one unit
    small = np.abs(x) <= 2 * unit
    assert (np.abs(y - x)[small] <= 0.25 * unit[small]).all()           # codes below 2 lie half a unit apart
    again = fo.quantise(y)
    np.testing.assert_array_equal(fo.values(*again), y)                 # a value of the format stays what it is
    assert (fo.quantise(-x)[0] == codes ^ 0x88).all()                   # symmetric


def test_a_block_with_an_infinity_is_nan_and_its_neighbours_are_not():
    x = np.ones(128)
    x[40] = -np.inf
    y = fo.values(*fo.quantise(x))
    assert np.isnan(y[32:64]).all() and (y[:32] == 1).all() and (y[64:] == 1).all()


def test_tables_by_hand():
    # blocks of 16 rows, two heads: 17 tokens need 2 blocks a head, 16 need 1, 0 none, 40 need 3 (6: too many of the 7 left are gone)
    table, live, slots, counts = fo.block_tables([17, 16, 0, 40, 5], 2, 16, 4, list(range(100, 109)), n_slots=80)
    assert table[0].tolist() == [[100, 101, 0, 0], [102, 103, 0, 0]] and table[1, :, 0].tolist() == [104, 105]
    assert live.tolist() == [17, 16, 0, 0, 0] and counts == (6, 14, 78)
    assert slots[0, :18].tolist() == list(range(1600, 1616)) + [1616, 1664] and slots[1, 17] == 1680
    assert (slots[:, 33:] == -1).all()
    # the next token of the second request needs a block, that of the first does not
    grown, live, slots, counts = fo.block_tables([18, 17], 2, 16, 4, [7, 8, 9], n_slots=2, held=[17, 16], table=table[:2])
    assert grown[1].tolist() == [[104, 7, 0, 0], [105, 8, 0, 0]] and (grown[0] == table[0]).all()
    assert slots.tolist() == [[101 * 16 + 1, 7 * 16], [103 * 16 + 1, 8 * 16]] and counts == (2, 2, 2) and live.tolist() == [18, 17]


def test_no_block_is_handed_out_twice():
    rng = np.random.default_rng(3)
    for _ in range(30):
        B, H, R = int(rng.integers(1, 9)), int(rng.integers(1, 4)), int(rng.choice([16, 32]))
        held = rng.integers(0, 60, B)
        free = rng.permutation(60)[:int(rng.integers(0, 60))] + 1000
        table = np.arange(B * H * 8, dtype=np.int32).reshape(B, H, 8)
        out, live, slots, (taken, wanted, tokens) = fo.block_tables(held + rng.integers(0, 70, B), H, R, 8, free, n_slots=500, held=held, table=table)
        new = out[out >= 1000]
        assert len(set(new.tolist())) == len(new) == taken <= min(wanted, len(free)) and set(new) == set(free[:taken])
        used = slots[slots >= 0]
        assert len(set(used.tolist())) == len(used) == H * (live - held).sum()
