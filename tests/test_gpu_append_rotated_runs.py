"""The rotated append by runs of positions, at head sizes and rotations of its own forms
and on both sides of where it begins, against the definition in 64 bits."""
import pytest

from test_gpu_heads import BF, FP, _append, _runs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act,bits", [(BF, 16), (FP, 16), (BF, 8), (FP, 8)])
@pytest.mark.parametrize("D,dims,inter,norm", [(192, 192, False, True), (192, 64, False, False), (192, 128, False, True), (192, 96, True, True),
                                               (256, 256, False, True), (256, 128, False, True), (256, 0, False, True), (128, 64, False, True),
                                               (64, 0, False, False)])
def test_forms(D, dims, inter, norm, act, bits):
    """2218 tokens of 8 key heads (17744 heads)."""
    lengths = [700, 1, 31, 33, 7, 8, 9, 64, 500, 100, 3, 5, 150, 600]
    slots = _runs(lengths, 64, 60, D)
    assert len(slots) * 8 >= 16384
    _append(len(slots), 2, 8, D, dims, act, bits, inter, norm, P=64, slots=slots, n_blocks=60, seed=D + dims)


@pytest.mark.parametrize("T", [511, 512, 1023, 1024, 1025])
@pytest.mark.parametrize("bits", [16, 8])
def test_where_it_begins(T, bits):
    """16 key heads: 1024 tokens are 16384 heads. In runs, and in no order."""
    slots = _runs([T - 12, 1, 11], 32, T // 32 + 5, T)
    _append(len(slots), 1, 16, 64, 64, BF, bits, P=32, slots=slots, n_blocks=T // 32 + 5, seed=T)
    _append(T, 1, 16, 64, 64, BF, bits, P=32, seed=T)
