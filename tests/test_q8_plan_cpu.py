"""The ragged plan of the decode over 8-bit caches at the longest rows, without a GPU: where a
workgroup's tokens begin, by the plan's own arithmetic, and where its waves' blocks do."""
import ctypes

import numpy as np
import pytest

atf = pytest.importorskip("paper_2608_02947_amd")

STEP = 256  # tokens of a step of the plan
_i32 = ctypes.c_int32


def _first():
    f = ctypes.CDLL(atf.LIB_PATH)["_ZN3atf15decode_q8_firstEiii"]
    f.restype, f.argtypes = _i32, [_i32] * 3
    return f


def plan(keys, splits):
    """[(row, first token, end)] of the items of a ragged batch whose rows reach `keys`: the device's
    steps, its sums and quotients in 32-bit floats."""
    f = np.float32
    steps = [-(-n // STEP) for n in keys]
    alive = sum(n > 0 for n in steps)
    total = f(0)
    for r0 in range(0, len(steps), 64):
        total = f(total + f(sum(steps[r0:r0 + 64])))
    many = 4 * alive > 3 * splits
    if total >= f(16777216):
        total = f(total * f(1.0002))
    span = max(1, int(min(np.ceil(f(total / f(splits if many else splits - alive // 2))), f(8388608))))
    for _ in range(0 if many else 8):
        items = sum(-(-n // span) for n in steps)
        if items <= splits:
            break
        span = max(span + 1, int(f(f(f(span) * f(items)) / f(splits))))
    return [(r, i * span * STEP, min(n, (i + 1) * span * STEP))
            for r, n in enumerate(keys) for i in range(-(-steps[r] // span))]


def test_waves_begin_inside_the_longest_rows():
    """A row of 2^31 - 32 keys (of shared pages) among others whose lengths make the plan cut it after
    2^23 - 1 steps: the last item begins at 2^31 - 256, and the sums of its 8 waves' blocks would
    pass 2^31.  One KV head of 17 to 32 query heads: 256 slots."""
    keys = [2 ** 31 - 32] + [7317721 * STEP] * 4 + [7487071 * STEP]
    items = plan(keys, 256)
    assert len(items) <= 256 and (0, 2 ** 31 - 256, 2 ** 31 - 32) in items
    for r, n in enumerate(keys):  # every key once
        own = [i for i in items if i[0] == r]
        assert own[0][1] == 0 and own[-1][2] == n and all(a[2] == b[1] for a, b in zip(own, own[1:]))
    first = _first()
    for _, begin, end in items:
        for wave in range(8):
            assert first(begin, end, wave) == min(begin + 64 * wave, end)


@pytest.mark.parametrize("begin,end", [(0, 0), (0, 1), (0, 64), (0, 65), (256, 700), (2 ** 31 - 256, 2 ** 31 - 1),
                                       (2 ** 31 - 512, 2 ** 31 - 1), (0, 2 ** 31 - 1)])
def test_first_block_of_a_wave(begin, end):
    first = _first()
    assert [first(begin, end, w) for w in range(8)] == [min(begin + 64 * w, end) for w in range(8)]
