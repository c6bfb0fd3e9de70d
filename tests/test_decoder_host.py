"""Block tables of the decoder block, on the CPU."""
import numpy as np
import pytest

from paper_2607_16184_amd.decoder import BlockTables


def test_slots_follow_the_table():
    t = BlockTables(n_blocks=7, block_tokens=32, sequences=3, max_len=100)
    seen = {}
    for step in ([(0, 40), (2, 1)], [(2, 31)], [(0, 24), (1, 5), (2, 1)], [(0, 1)]):
        before = t.length.copy()
        table, lens, slots = (x.numpy() for x in t.step(*zip(*step), device="cpu"))
        assert table.dtype == np.int32 and lens.dtype == np.int32 and slots.dtype == np.int64
        i = 0
        for s, n in step:
            for k in range(n):
                pos = int(before[s]) + k
                assert lens[i] == pos + 1 and slots[i] == table[i, pos // 32] * 32 + pos % 32
                assert slots[i] not in seen and np.array_equal(table[i], t.table[s])
                seen[int(slots[i])] = (s, pos)
                i += 1
        assert i == len(lens)
    held = t.table[t.table >= 0]
    assert len(set(held)) == len(held) and not set(held) & set(t.free) and len(held) + len(t.free) == 7


def test_blocks_come_back():
    t = BlockTables(4, 32, 2, 128)
    t.step([0], [128], device="cpu")
    with pytest.raises(MemoryError):
        t.step([1], [1], device="cpu")
    assert t.length[1] == 0 and (t.table[1] == -1).all()
    t.release(0)
    assert sorted(t.free) == [0, 1, 2, 3]
    t.step([1], [97], device="cpu")
    assert len(t.free) == 0


def test_refusals():
    t = BlockTables(4, 32, 2, 50)
    with pytest.raises(ValueError):
        t.step([0], [51], device="cpu")
    with pytest.raises(ValueError):
        t.step([0, 0], [1, 1], device="cpu")
    with pytest.raises(MemoryError):
        BlockTables(3, 32, 2, 100).step([0, 1], [64, 64], device="cpu")
    assert len(t.free) == 4 and not t.length.any()


@pytest.mark.parametrize("sequences,tokens,error", [
    ([0, 1], [10, 51], ValueError),          # the second would pass max_len
    ([1, 0], [3, 50], ValueError),           # the second would, with what it has
    ([0, 1], [10], ValueError), ([0], [10, 10], ValueError),
    ([0, 1], [10, -1], ValueError), ([1], [-2], ValueError),
    ([0, 3], [10, 1], ValueError), ([2, -1], [10, 1], ValueError),
    ([0, 1, 2], [49, 50, 50], MemoryError)])
def test_a_refused_step_changes_nothing(sequences, tokens, error):
    """Also where the fault lies with a later sequence of the step."""
    t = BlockTables(5, 32, 3, 50)
    t.step([0, 1], [1, 2], device="cpu")
    t.release(1)
    table, length, free = t.table.copy(), t.length.copy(), list(t.free)
    with pytest.raises(error):
        t.step(sequences, tokens, device="cpu")
    assert np.array_equal(t.table, table) and np.array_equal(t.length, length) and t.free == free
    for s, n in zip(sequences, tokens):
        if n < 0:
            with pytest.raises(error):
                t.extend(s, n)
            assert np.array_equal(t.table, table) and np.array_equal(t.length, length) and t.free == free
