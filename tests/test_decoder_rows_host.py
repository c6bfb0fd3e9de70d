"""Block tables of steps by sequences, on the CPU."""
import numpy as np
import pytest

from paper_2607_16184_amd.decoder import BlockTables


def _rows(t, *args):
    r = t.rows(*args, device="cpu")
    assert list(r) == ["block_table", "lens", "slots", "starts", "positions"]
    return [x.numpy() for x in r.values()]


def test_rows_agree_with_single_rows():
    a, b = (BlockTables(n_blocks=9, block_tokens=32, sequences=3, max_len=120) for _ in range(2))
    for seqs, counts in [([0, 2], [40, 3]), ([1], [33]), ([2, 0, 1], [1, 5, 7])]:
        table, lens, slots = (t.numpy() for t in a.step(seqs, counts, device="cpu"))
        rt, rl, rs, starts, pos = _rows(b, seqs, counts)
        assert [t.dtype for t in (rt, rl, rs, starts, pos)] == [np.int32, np.int32, np.int64, np.int32, np.int32]
        assert np.array_equal(rs, slots) and np.array_equal(pos, lens - 1)
        assert starts.tolist() == np.cumsum([0] + counts).tolist()
        assert np.array_equal(np.repeat(rt, counts, 0), table)
        assert rl.tolist() == [lens[e - 1] for e in starts[1:]]


def test_positions_of_trees():
    t = BlockTables(8, 32, 2, 100)
    t.rows([0, 1], [30, 7], device="cpu")
    _, lens, slots, starts, pos = _rows(t, [1, 0], [4, 3], [[0, 0, 1, 2], [0, 1, 1]])
    assert pos.tolist() == [7, 7, 8, 9, 30, 31, 31] and lens.tolist() == [11, 33] and starts.tolist() == [0, 4, 7]
    assert [int(s) % 32 for s in slots] == [7, 8, 9, 10, 30, 31, 0]


def test_truncation_gives_blocks_back():
    t = BlockTables(6, 32, 2, 160)
    t.rows([0, 1], [100, 32], device="cpu")
    held = t.table[0].copy()
    t.truncate(0, 65)
    assert t.length[0] == 65 and np.array_equal(t.table[0, :3], held[:3]) and (t.table[0, 3:] == -1).all()
    assert sorted(t.free) == sorted(set(range(6)) - set(held[:3]) - {int(t.table[1, 0])})
    t.truncate(0, 64)
    assert (t.table[0, 2:] == -1).all() and len(t.free) == 3
    t.truncate(0, 64)
    t.truncate(1, 0)
    assert len(t.free) == 4 and (t.table[1] == -1).all()
    for s, n in ((0, 65), (0, -1), (2, 0), (-1, 0)):
        with pytest.raises(ValueError):
            t.truncate(s, n)


def test_refused_rows_change_nothing():
    t = BlockTables(3, 32, 2, 96)
    t.rows([0], [40], device="cpu")
    before = t.table.copy(), t.length.copy(), list(t.free)
    for error, args in ((ValueError, ([0, 0], [1, 1])), (ValueError, ([0], [1, 2])), (ValueError, ([0], [60])), (ValueError, ([5], [1])),
                        (MemoryError, ([0, 1], [30, 33])), (ValueError, ([0], [-1])), (ValueError, ([0], [2], [[0]])),
                        (ValueError, ([0], [2], [[0, -1]]))):
        with pytest.raises(error):
            t.rows(*args, device="cpu")
    assert np.array_equal(t.table, before[0]) and np.array_equal(t.length, before[1]) and t.free == before[2]


def test_empty_steps():
    t = BlockTables(2, 32, 2, 64)
    table, lens, slots, starts, pos = _rows(t, [], [])
    assert table.shape == (0, 2) and lens.size == slots.size == pos.size == 0 and starts.tolist() == [0]
    assert _rows(t, [1], [0])[3].tolist() == [0, 0]
