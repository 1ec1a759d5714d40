"""The references of append and read back at table entries that are no page of the pool."""
import numpy as np
import pytest

import oracle
from oracle import cache as C


@pytest.mark.parametrize("entry", [-1, 3, 2 ** 31 - 1])
def test_a_token_without_a_page_goes_nowhere(entry):
    rng = np.random.default_rng(3)
    k, v = rng.integers(0, 1 << 15, (2, 3, 4, 2, 64)).astype(np.uint16)
    new = rng.integers(0, 0x7F80, (1, 6, 2, 64)).astype(np.uint16)
    table, lens = np.array([[2, entry, 0]], np.int32), np.array([10], np.int32)  # tokens 4 to 9: pages 1 and 2
    for got, old in zip(oracle.kv_append(k, v, new, new, table, lens), (k, v)):
        want = old.copy()
        want[0, :2] = new[0, 4:]
        assert np.array_equal(got, want)
    codes, scales = C.kv4_cache(k)
    c, s = C.kv4_append(codes, scales, new, table, lens)
    assert np.array_equal(c[1:], codes[1:]) and np.array_equal(s[1:], scales[1:])
    back = C.kv4_read(c, s, 6, table, lens)
    assert (back[0, :4] == 0).all()
    assert np.array_equal(back[0, 4:], C.kv4_values(*C.kv4_quantise(new[0, 4:])).reshape(2, 2, 64))
