"""Integer list arguments of the binding: any sequence of numbers, converted as ctypes converts them."""
import ctypes

import numpy as np
import pytest

from paper_2608_21719_amd import binding as B
from tests.kv8_helpers import shape


@pytest.mark.parametrize("seq", [
    [], [1, 2, 3], (4, -5), range(6), np.array([7, 8], dtype=np.int64), np.array([9], dtype=np.uint8), [np.int32(3), 4],
    [1.9, -1.9], np.array([2.5, 3.5]), b"\x01\x02\x03", bytearray(8), "123", {5: 0, 6: 0}, [True, False],
    [2 ** 31, -2 ** 31 - 1, 2 ** 32 + 5, -1], [2 ** 70 + 1], [1, 2.5, 2 ** 40]])
def test_as_ctypes_converts(seq):
    want = (ctypes.c_int32 * len(seq))(*[int(x) for x in seq])
    got = B.ints(seq)
    assert list(got) == list(want)
    got = ctypes.cast(got, ctypes.POINTER(ctypes.c_int32))  # what a call receives
    assert [got[i] for i in range(len(seq))] == list(want)


def test_a_number_past_32_bits_is_refused_by_the_library():
    cfg = B.make_cfg(shape(4, 2, 64))
    kv = B.KV8(cfg, 1, 8, 2, 4, 0x100000)  # host calls only: the pool is not touched
    s = kv.open()
    kv.alloc(s, 32)
    with pytest.raises(B.PsError) as e:
        kv.commit([s], [2 ** 31])
    assert e.value.code == B.PS_E_INVALID
    with pytest.raises(B.PsError):
        kv.commit([2 ** 31 + 7], [1])
    assert kv.seq_len(s) == 0
