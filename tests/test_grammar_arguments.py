"""What a Grammar is made from: tables of other shapes and of numbers that 32 bits do not hold.  No GPU: what reaches the library is looked
at on its way there."""
import ctypes

import numpy as np
import pytest

import paper_2603_02597_amd as B
from paper_2603_02597_amd import binding


class _Reached(Exception):
    pass


@pytest.fixture
def built(monkeypatch):
    """Calls Grammar and returns the table that it hands to bpe_grammar_build."""
    seen = []

    class Library:
        def bpe_grammar_build(self, transitions, accepting, n_states, out):
            at = ctypes.cast(transitions, ctypes.POINTER(ctypes.c_int32))
            seen.append(np.ctypeslib.as_array(at, (n_states, 256)).copy())
            raise _Reached

    monkeypatch.setattr(binding, "load_library", Library)

    def call(table):
        with pytest.raises(_Reached):
            B.Grammar(table)
        return seen.pop()

    return call


@pytest.mark.parametrize("dtype", [np.int8, np.uint8, np.int16, np.uint16, np.int32, np.uint32, np.int64, np.uint64, np.float32, np.float64, bool])
def test_tables_of_every_type(built, dtype):
    table = np.arange(512).reshape(2, 256) % 2
    assert np.array_equal(built(table.astype(dtype)), table)
    assert np.array_equal(built(table.astype(dtype).reshape(-1)), table)
    assert np.array_equal(built(table.astype(dtype).tolist()), table)


@pytest.mark.parametrize("end", [-1, -7, -2**31, -2**32, -2**40, np.iinfo(np.int64).min])
def test_any_negative_number_ends_a_walk(built, end):
    table = np.zeros((3, 256), dtype=np.int64)
    table[1, 5] = end
    got = built(table)
    assert got[1, 5] < 0 and (np.delete(got.reshape(-1), 261) == 0).all()


@pytest.mark.parametrize("state", [2**31, 2**32, 2**32 + 1, 2**40 + 1])
def test_numbers_that_are_no_states_stay_none(built, state):
    for dtype in (np.int64, np.uint64, np.float32):
        table = np.zeros((3, 256), dtype=dtype)
        table[1, 5] = state
        assert built(table)[1, 5] >= 3                   # (which the library refuses)


def test_tables_that_are_none():
    for table in (np.zeros((4, 128), dtype=np.int32), np.zeros((1, 512), dtype=np.int32), np.full((2, 256), 0.5), np.full((2, 256), np.nan)):
        with pytest.raises(ValueError):
            B.Grammar(table)
