"""The oracle of 8-bit caches with a scale per block where something is not finite, against codes written out by hand."""
import numpy as np
import pytest

from oracle import cache_blocks_ref


@pytest.mark.parametrize("dtype", [np.int8, np.uint8])  # two's complement, e4m3
def test_what_is_not_finite(dtype):
    inf, nan = np.inf, np.nan
    most, least, none = (127, -127, 0) if dtype == np.int8 else (0x7e, 0xfe, 0x7f)

    def one(row, code=0x31, scale=7.0, first=0):
        codes, scales = np.full((1, 1, 8, 4), code, dtype), np.full((1, 1, 1), scale, np.float32)
        cache_blocks_ref.append(codes, scales, np.array(row, np.float32).reshape(1, 1, 4), [0], first, 8)
        return codes[0, 0], scales[0, 0, 0]

    codes, scale = one([inf, -inf, nan, 1])
    assert list(codes[0]) == [most, least, none, most] and scale == np.float32(1) * (np.float32(1) / np.float32(127 if dtype == np.int8 else 448))
    codes, scale = one([inf, -0.0, nan, -inf])  # nothing that is finite and not 0, in a block without a scale
    assert list(codes[0]) == [0, 0, none, 0] and scale == 0
    codes, scale = one([inf, 0, nan, 0], first=3)  # the same under a scale that is there
    assert list(codes[3]) == [most, 0, none, 0] and scale == 7 and (codes[:3] == 0x31).all()
    for bad in (0, -1, inf, -inf, nan):  # scales that are none: what was held under them is 0
        codes, scale = one([inf, 0, 0, 0], code=0x7f, scale=bad, first=3)
        assert not codes[:4].any() and (codes[4:] == 0x7f).all() and scale == 0
