"""Whole numbers past 32 bits, which a foreign-function call would cut down without a
word: refused by the operators on tensors (no GPU is needed)."""
import pytest

from paper_2607_16184_amd import ops
from test_ops_devices import ATTN, _make, gpu  # noqa: F401
from test_rows_host import APPEND_T, HEADS_T, KEEP_T, ROWS_T, _kv, _rotation, calls  # noqa: F401

WRAPS = [(1 << 32) + 5, 1 << 31, -(1 << 31) - 1, 1 << 40]


@pytest.mark.parametrize("offset", WRAPS)
def test_offsets(calls, offset):  # noqa: F811
    t = _make(HEADS_T, 0)
    with pytest.raises(ValueError):
        ops.norm_rotate(t["q"], t["k"], t["pos"], _rotation(t), out=(t["qo"], t["ko"]), offset=offset)
    t = _make(APPEND_T, 0)
    with pytest.raises(ValueError):
        _kv(t).append_rotated(t["k"], t["v"], t["slots"], t["pos"], _rotation(t), t["q"], q_out=t["qo"], offset=offset)
    assert not calls


@pytest.mark.parametrize("offset", [(1 << 31) - 1, -(1 << 31)])
def test_offsets_at_the_ends(calls, offset):  # noqa: F811
    t = _make(HEADS_T, 0)
    ops.norm_rotate(t["q"], t["k"], t["pos"], _rotation(t), out=(t["qo"], t["ko"]), offset=offset)
    assert len(calls) == 1


@pytest.mark.parametrize("window", WRAPS)
def test_windows(calls, window):  # noqa: F811
    t = _make(ROWS_T, 0)
    with pytest.raises(ValueError):
        _kv(t).attend_rows(t["q"], t["starts"], t["table"], t["lens"], 100, window=window, out=t["out"])
    t = _make(ATTN, 0)
    with pytest.raises(ValueError):
        _kv(t).attend(t["q"], t["table"], t["lens"], 100, window=window, out=t["out"])
    assert not calls


def test_lengths(calls):  # noqa: F811
    """Blocks so long that the table covers a bound of more than 2^32 tokens."""
    t, d = _make(ROWS_T + KEEP_T[-2:], 0), _make(ATTN, 0)
    kv = _kv(t)
    kv.block_tokens = 1 << 31
    for call in (lambda: kv.attend_rows(t["q"], t["starts"], t["table"], t["lens"], (1 << 32) + 100, out=t["out"]),
                 lambda: kv.attend(d["q"], d["table"], d["lens"], (1 << 32) + 100, out=d["out"]),
                 lambda: kv.keep(t["starts"], t["table"], t["lens"], (1 << 32) + 100, t["chosen"], out=t["new"])):
        with pytest.raises(ValueError):
            call()
    assert not calls
