"""Workspaces of the operators over blocks, sized once for calls of several sizes, on the host."""
import ctypes
import random

import pytest

import test_blocks_cpu as C
from test_blocks_plan_cpu import Plan

atf = pytest.importorskip("paper_2608_02947_amd")

_fit = ctypes.CDLL(atf.LIB_PATH)["_ZN3atf11attend_planElll"]
_fit.restype, _fit.argtypes = Plan, [ctypes.c_int64] * 3
_plan = ctypes.CDLL(atf.LIB_PATH)["_ZN3atf11attend_planEll"]
_plan.restype, _plan.argtypes = Plan, [ctypes.c_int64] * 2


def test_attention_splits_no_further_than_its_room():
    rng = random.Random(2)
    for _ in range(20000):
        groups, tiles, room = int(2 ** rng.uniform(0, 9)), int(2 ** rng.uniform(0, 14)), rng.choice([0, 1, 2, 7, 30, 300])
        p, whole = _fit(groups, tiles, room), _plan(groups, tiles)
        assert 1 <= p.splits <= max(1, min(room, 256 // groups, tiles // 8))
        assert p.waves == whole.waves and p.splits * p.split_tiles >= tiles > (p.splits - 1) * p.split_tiles
        if room >= tiles:
            assert (p.splits, p.split_tiles) == (whole.splits, whole.split_tiles)


def test_attention_workspace_that_serves_every_call():
    """The bound that atf.h names."""
    for h_q, h_kv, d in ((32, 4, 128), (14, 2, 64), (40, 1, 64), (72, 1, 128), (16, 16, 64), (300, 300, 64)):
        most = 256 * (h_q // h_kv) * (4 * d + 8) + 768
        for n in list(range(1, 300)) + [900, 5000]:
            for top, bt in ((1, 32), (16, 32), (27, 32), (64, 64), (300, 32), (4096, 128)):
                assert 256 <= atf.atf_attend_workspace_bytes(n, h_q, h_kv, top, bt, d) <= most


@pytest.mark.parametrize("size", [0, 255])
def test_attention_workspaces_below_the_least_are_refused(size):
    fn, make = C.CALLS["attend"]
    assert fn(*make(bytes=size).values()) == atf.ATF_EWORKSPACE
    assert atf.atf_last_error()


def test_selection_workspace_serves_smaller_calls():
    """Fewer tokens and fewer keys take no more; what the tokens of one launch need is there: 12 bytes a block
    for as many tokens as 256 MB hold."""
    for h_q, h_kv, bt, d in ((6, 2, 64, 128), (32, 8, 64, 128), (64, 64, 32, 128), (40, 2, 32, 64), (3000, 3000, 64, 64)):
        rng = random.Random(h_q)
        tokens = sorted({0, 1, 2, 64} | {int(2 ** rng.uniform(0, 11)) for _ in range(20)})
        keys = sorted({1, 500000, 1 << 20, 2000000, 6 << 20, 2 ** 31 - 1} | {int(2 ** rng.uniform(0, 31)) for _ in range(40)})
        size = [[atf.atf_select_workspace_bytes(n, h_q, h_kv, k, bt, d) for k in keys] for n in tokens]
        for i, n in enumerate(tokens):
            for j, k in enumerate(keys):
                assert size[i][j] >= size[max(i - 1, 0)][j] and size[i][j] >= size[i][max(j - 1, 0)]
                each = 12 * h_kv * -(-k // (16 * bt)) * 16
                assert size[i][j] >= each * max(1, min(n, 65535 // h_kv, (1 << 28) // (2 * each)))
