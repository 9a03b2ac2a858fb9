"""A decode wave's steps through the longest rows that pages can hold, without a GPU."""
import ctypes

import pytest

atf = pytest.importorskip("paper_2608_02947_amd")


@pytest.mark.parametrize("t_end", [1, 128, 129, 2 ** 31 - 128, 2 ** 31 - 97, 2 ** 31 - 32, 2 ** 31 - 1])
def test_no_step_past_the_end(t_end):
    """From every block of the last steps, of each of a workgroup's 4 waves: 128 tokens on, or the end."""
    f = ctypes.CDLL(atf.LIB_PATH)["_ZN3atf11decode_nextEiii"]
    f.restype, f.argtypes = ctypes.c_int32, [ctypes.c_int32] * 3
    for t0 in range(max(0, (t_end - 1) // 128 * 128 - 256), t_end, 32):
        assert f(t0, t_end, 128) == min(t0 + 128, t_end)
