"""The rule that shares the tiles of listed blocks out over waves and workgroups, on the host."""
import ctypes
import random

import pytest

atf = pytest.importorskip("paper_2608_02947_amd")


class Plan(ctypes.Structure):
    _fields_ = [("waves", ctypes.c_int32), ("splits", ctypes.c_int32), ("split_tiles", ctypes.c_int32)]


_plan = ctypes.CDLL(atf.LIB_PATH)["_ZN3atf11attend_planEll"]
_plan.restype, _plan.argtypes = Plan, [ctypes.c_int64, ctypes.c_int64]


@pytest.mark.parametrize("groups,tiles,waves,splits", [
    # a wave a tile at most; waves by the groups
    (1, 1, 1, 1), (2, 4, 4, 1), (4, 16, 8, 1), (256, 128, 8, 1), (257, 128, 4, 1), (640, 128, 4, 1), (641, 128, 2, 1),
    (2048, 128, 2, 1), (2049, 128, 1, 1), (100000, 3, 1, 1),
    # split where that saves 20 tiles of a workgroup's
    (4, 32, 8, 4), (8, 24, 8, 1), (4, 23, 8, 1), (4, 26, 8, 1), (4, 30, 8, 3), (128, 32, 8, 1), (128, 128, 8, 2), (64, 32, 8, 4), (4, 512, 8, 64), (1, 4096, 8, 256),
    (0, 100, 8, 12)])
def test_attend_plan(groups, tiles, waves, splits):
    p = _plan(groups, tiles)
    assert (p.waves, p.splits) == (waves, splits)


def test_attend_plans_cover_every_tile_and_leave_no_split_empty():
    rng = random.Random(1)
    for _ in range(20000):
        groups, tiles = int(2 ** rng.uniform(0, 23)), int(2 ** rng.uniform(0, 26))
        p = _plan(groups, tiles)
        assert p.waves in (1, 2, 4, 8) and p.waves < 2 * tiles
        assert p.splits * p.split_tiles >= tiles > (p.splits - 1) * p.split_tiles
        assert p.splits == 1 or (p.waves == 8 and groups * p.splits * 8 <= 2048 and p.split_tiles >= 8)


def test_workspaces_hold_the_splits():
    for T, h_q, h_kv, top, bt, d in ((1, 14, 2, 16, 64, 64), (4, 32, 4, 64, 64, 128), (3, 40, 1, 300, 32, 128), (900, 32, 4, 64, 64, 128)):
        groups = T * h_kv * -(-(h_q // h_kv) // 32)
        p = _plan(groups, top * bt // 32)
        need = T * h_q * p.splits * (d + 2) * 4 if p.splits > 1 else 0
        assert need <= atf.atf_attend_workspace_bytes(T, h_q, h_kv, top, bt, d) <= need + 1024
