"""Refusals of the operators over pages and blocks (no call reaches a launch), and their plain forms on
cases worked out by hand."""
import ctypes
import math

import numpy as np
import pytest
import torch

import blocksref as R

atf = pytest.importorskip("paper_2608_02947_amd")

LIB = atf.library()
A = 1 << 20  # addresses that are never dereferenced, far apart


def addr(i):
    return ctypes.c_void_p(A * 1024 * (i + 1))


KEPT = []  # the arrays that the windows below point to


def window(d=128, **kw):
    w, arrays = atf.Window(d, 1e4, 2.0, **kw).as_c()
    KEPT.append(arrays)
    return w


def plan_args(**kw):
    a = dict(block_table=addr(0), max_pages=10, page_tokens=64, free_pages=addr(1), free_capacity=100,
             free_count=addr(2), batch=4, n_k_rows=addr(3), n_new_rows=addr(4), n_k_out=addr(5), row_starts=addr(6),
             max_tokens=100, slots=addr(7), token_rows=addr(8), positions=addr(9), counts=addr(10), stream=None)
    a.update(kw)
    return a


def slots_args(**kw):
    a = dict(k_new=addr(0), v_new=addr(1), k_pages=addr(2), v_pages=addr(3), slots=addr(4), n_tokens=5, num_pages=7,
             page_tokens=64, h_kv=2, head_dim=64, stream=None)
    a.update(kw)
    return a


def turned_args(**kw):
    a = dict(k_new=addr(0), v_new=addr(1), k_pages=addr(2), v_pages=addr(3), slots=addr(4), positions=addr(5),
             n_tokens=5, num_pages=7, page_tokens=64, h_kv=2, w=window(64), inv_freq=None, stream=None)
    a.update(kw)
    return a


def bounds_args(**kw):
    a = dict(k_pages=addr(0), bounds=addr(1), block_table=addr(2), max_pages=10, num_pages=7, page_tokens=64,
             block_tokens=32, batch=4, n_k_rows=addr(3), n_new_rows=addr(4), max_new=5, h_kv=2, head_dim=64, stream=None)
    a.update(kw)
    return a


def select_args(**kw):
    a = dict(q=addr(0), bounds=addr(1), blocks=addr(2), n_tokens=5, block_table=addr(3), max_pages=10, num_pages=7,
             page_tokens=64, block_tokens=32, batch=4, token_rows=addr(4), positions=addr(5), n_k_rows=addr(6),
             max_n_k=640, top=8, first=1, last=2, h_q=6, h_kv=2, w=window(), workspace=addr(7), bytes=1 << 29, stream=None)
    a.update(kw)
    return a


def attend_args(**kw):
    a = dict(q=addr(0), k_pages=addr(1), v_pages=addr(2), o=addr(3), lse=addr(4), n_tokens=5, block_table=addr(5),
             max_pages=10, num_pages=7, page_tokens=64, block_tokens=32, batch=4, token_rows=addr(6), positions=addr(7),
             n_k_rows=addr(8), blocks=addr(9), top=8, h_q=6, h_kv=2, w=window(), scale=0.0, workspace=addr(10),
             bytes=1 << 29, stream=None)
    a.update(kw)
    return a


CALLS = {"plan": (LIB.atf_plan_pages, plan_args), "slots": (LIB.atf_cache_append_slots, slots_args),
         "turned": (LIB.atf_cache_append_slots_rotated, turned_args), "bounds": (LIB.atf_block_bounds, bounds_args),
         "select": (LIB.atf_select_blocks, select_args), "attend": (LIB.atf_attend_blocks, attend_args)}
EINVAL, EUNSUPPORTED, EWORKSPACE = atf.ATF_EINVAL, atf.ATF_EUNSUPPORTED, atf.ATF_EWORKSPACE

BAD = [("plan", dict(page_tokens=48), EINVAL), ("plan", dict(page_tokens=0), EINVAL), ("plan", dict(max_pages=0), EINVAL),
       ("plan", dict(max_pages=1 << 26), EINVAL), ("plan", dict(batch=0), EINVAL), ("plan", dict(batch=(1 << 20) + 1), EINVAL),
       ("plan", dict(free_capacity=-1), EINVAL), ("plan", dict(max_tokens=-1), EINVAL),
       ("plan", dict(max_tokens=(1 << 30) + 1), EINVAL), ("plan", dict(n_k_out=addr(4)), EINVAL),
       ("plan", dict(slots=ctypes.c_void_p(addr(7).value + 4)), EINVAL),
       ("plan", dict(counts=ctypes.c_void_p(addr(10).value + 2)), EINVAL), ("plan", dict(token_rows=addr(9)), EINVAL),
       ("plan", dict(row_starts=ctypes.c_void_p(addr(3).value - 4)), EINVAL),
       ("slots", dict(head_dim=96), EUNSUPPORTED), ("slots", dict(n_tokens=-1), EINVAL), ("slots", dict(h_kv=0), EINVAL),
       ("slots", dict(page_tokens=16), EINVAL), ("slots", dict(num_pages=0), EINVAL),
       ("slots", dict(n_tokens=(1 << 28) + 1), EINVAL), ("slots", dict(k_pages=addr(3)), EINVAL),
       ("slots", dict(slots=ctypes.c_void_p(addr(4).value + 4)), EINVAL),
       ("slots", dict(k_new=ctypes.c_void_p(addr(0).value + 8)), EINVAL), ("slots", dict(v_new=addr(3)), EINVAL),
       ("turned", dict(w=None), EINVAL), ("turned", dict(w=window(32)), EUNSUPPORTED),
       ("turned", dict(w=window(64, inv_freq=[-1.0] * 32)), EINVAL),
       ("turned", dict(positions=addr(2)), EINVAL), ("turned", dict(positions=ctypes.c_void_p(addr(5).value + 2)), EINVAL),
       ("bounds", dict(head_dim=80), EUNSUPPORTED), ("bounds", dict(block_tokens=48), EINVAL),
       ("bounds", dict(block_tokens=128), EINVAL), ("bounds", dict(block_tokens=0), EINVAL), ("bounds", dict(batch=0), EINVAL),
       ("bounds", dict(h_kv=0), EINVAL), ("bounds", dict(max_new=-1), EINVAL), ("bounds", dict(bounds=addr(0)), EINVAL),
       ("bounds", dict(num_pages=0), EINVAL), ("bounds", dict(bounds=ctypes.c_void_p(addr(1).value + 8)), EINVAL),
       ("select", dict(w=None), EINVAL), ("select", dict(w=window(32)), EUNSUPPORTED), ("select", dict(top=0), EINVAL),
       ("select", dict(top=4097), EINVAL), ("select", dict(first=-1), EINVAL), ("select", dict(last=-1), EINVAL),
       ("select", dict(first=7), EINVAL), ("select", dict(first=2 ** 31 - 1, last=2 ** 31 - 1), EINVAL),
       ("select", dict(h_q=7), EINVAL), ("select", dict(h_kv=0), EINVAL), ("select", dict(n_tokens=-1), EINVAL),
       ("select", dict(n_tokens=(1 << 23) // 6 + 1), EINVAL), ("select", dict(max_n_k=641), EINVAL),
       ("select", dict(max_n_k=0), EINVAL), ("select", dict(bytes=16), EWORKSPACE), ("select", dict(workspace=None), EWORKSPACE),
       ("select", dict(workspace=ctypes.c_void_p(addr(7).value + 8)), EINVAL), ("select", dict(block_tokens=96), EINVAL),
       ("select", dict(blocks=addr(0)), EINVAL), ("select", dict(workspace=addr(0)), EINVAL),
       ("select", dict(page_tokens=33, block_tokens=33), EINVAL), ("select", dict(w=atf.Window(128, 0.5, 2.0).as_c()[0]), EINVAL),
       ("attend", dict(w=None), EINVAL), ("attend", dict(w=window(32)), EUNSUPPORTED), ("attend", dict(top=0), EINVAL),
       ("attend", dict(top=4097), EINVAL), ("attend", dict(h_q=5), EINVAL), ("attend", dict(scale=math.nan), EINVAL),
       ("attend", dict(scale=math.inf), EINVAL), ("attend", dict(bytes=0), EWORKSPACE), ("attend", dict(workspace=None), EWORKSPACE),
       ("attend", dict(o=addr(0)), EINVAL), ("attend", dict(lse=addr(9)), EINVAL), ("attend", dict(n_tokens=-1), EINVAL),
       ("attend", dict(batch=0), EINVAL), ("attend", dict(lse=ctypes.c_void_p(addr(4).value + 2)), EINVAL),
       ("attend", dict(top=4096, page_tokens=1 << 19, block_tokens=1 << 19), EINVAL),
       ("attend", dict(page_tokens=(1 << 26) + 32, block_tokens=32, max_pages=1), EUNSUPPORTED),
       ("bounds", dict(page_tokens=32, max_pages=(1 << 26) - 1, h_kv=9), EINVAL),
       ("attend", dict(k_pages=ctypes.c_void_p(addr(1).value + 8)), EINVAL), ("attend", dict(num_pages=0), EINVAL)]
BAD += [(call, {name: None}, EINVAL) for call, (_, make) in CALLS.items() for name, value in make().items()
        if isinstance(value, ctypes.c_void_p) and name != "workspace"]


@pytest.mark.parametrize("call,change,code", BAD, ids=lambda x: str(x) if not isinstance(x, dict) else "-".join(x))
def test_refused(call, change, code):
    fn, make = CALLS[call]
    assert fn(*make(**change).values()) == code
    assert atf.atf_last_error()


@pytest.mark.parametrize("call", ["slots", "turned", "select", "attend"])
def test_calls_without_tokens_do_nothing(call):
    fn, make = CALLS[call]
    assert fn(*make(n_tokens=0).values()) == 0
    none = {x: None for x in ("q", "k_new", "v_new", "slots", "positions", "token_rows", "blocks", "o", "lse") if x in make()}
    assert fn(*make(n_tokens=0, **none).values()) == 0


def test_bounds_of_no_tokens_do_nothing():
    assert LIB.atf_block_bounds(*bounds_args(max_new=0).values()) == 0


def test_workspace_sizes():
    assert atf.atf_select_workspace_bytes(0, 6, 2, 100, 32, 128) > 0
    one = atf.atf_select_workspace_bytes(1, 6, 2, 1 << 20, 64, 128)
    assert one >= 2 * (1 << 14) * 4
    assert atf.atf_select_workspace_bytes(1 << 20, 6, 2, 1 << 20, 64, 128) <= 1 << 29
    assert atf.atf_attend_workspace_bytes(5, 6, 2, 16, 32, 64) > 0
    for bad in (dict(n=-1), dict(h_q=5), dict(h_kv=0), dict(bt=48), dict(d=32), dict(n=1 << 23)):
        a = dict(n=4, h_q=6, h_kv=2, x=100, bt=32, d=128)
        a.update(bad)
        assert atf.atf_select_workspace_bytes(*a.values()) == 0
        assert atf.atf_attend_workspace_bytes(*a.values()) == 0
    assert atf.atf_select_workspace_bytes(4, 6, 2, 0, 32, 128) == 0
    assert atf.atf_attend_workspace_bytes(4, 6, 2, 4097, 32, 128) == 0


def test_tensors_that_are_not_on_the_gpu_are_refused():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        atf.atf_plan_pages(i32(2, 4), 32, i32(8), i32(1), i32(2), i32(2), i32(2), i32(3),
                           torch.zeros(5, dtype=torch.int64), i32(5), i32(5), i32(3))
    with pytest.raises(ValueError, match="shapes"):
        bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
        atf.atf_cache_append_slots(bf(5, 2, 64), bf(5, 2, 64), bf(3, 2, 4, 32, 16), bf(3, 2, 1, 64, 16),
                                   torch.zeros(5, dtype=torch.int64))
    with pytest.raises(ValueError, match="bounds"):
        atf.atf_select_blocks(bf(2, 4, 64), bf(3, 2, 5, 4, 2, 16), i32(2, 2, 4), i32(1, 3), 32, i32(2), i32(2), i32(1), 64,
                              atf.Window(64, 1e4, 2.0), torch.zeros(8, dtype=torch.uint8))


# ---- the plain forms

def test_plain_plan_by_hand():
    # page of 32 tokens; row 0 ends (2 pages back), row 1 grows by a page, row 2 idles, row 3 starts with 2
    got = R.plan([[4, 5, -1], [6, -1, -1], [7, -1, -1], [-1, -1, -1]], 32, [1, 2, 0, 0, 0], 2, [40, 30, 3, 0],
                 [-1, 5, 0, 33], 50)
    assert got["free_pages"].tolist() == [1, 2, 4, 5, 0]
    assert got["block_table"].tolist() == [[4, 5, -1], [6, 5, -1], [7, -1, -1], [4, 2, -1]]
    assert got["n_k_out"].tolist() == [0, 35, 3, 33] and got["counts"].tolist() == [1, 38, 0]
    assert got["row_starts"].tolist() == [0, 0, 5, 5, 38]
    assert got["slots"][:6].tolist() == [6 * 32 + 30, 6 * 32 + 31, 5 * 32, 5 * 32 + 1, 5 * 32 + 2, 4 * 32]
    assert got["slots"][37:].tolist() == [2 * 32] + [-1] * 12
    # row 0 would outgrow its three pages (97 tokens), which stops no other; then it lacks one, which does
    long = R.plan([[4, 5, -1], [6, -1, -1]], 32, [1], 1, [64, 30], [33, 5], 50)
    assert long["n_k_out"].tolist() == [64, 35] and long["counts"].tolist() == [0, 38, 1]
    short = R.plan([[4, -1, -1], [6, -1, -1]], 32, [1], 1, [32, 30], [33, 5], 50)
    assert short["n_k_out"].tolist() == [32, 30] and short["counts"].tolist() == [1, 38, 2]


def test_plain_scores_bound_every_key():
    rng = np.random.default_rng(3)
    for trial in range(40):
        d, bt, n = 64, 32, int(rng.integers(1, 130))
        pt, W = 64, np.sort(rng.integers(0, 150, d // 2))
        kpool = rng.standard_normal((3, 1, d // 16, pt, 16))
        table = np.array([[2, 0, 1]])
        b = R.bounds(kpool, np.zeros((3, 1, pt // bt, d // 16, 2, 16)), table, [n], [n], n, pt, bt)
        p = int(rng.integers(0, n + 20))
        last = min(p, n - 1)
        q = rng.standard_normal((2, d))
        s = R.scores(q, b, table[0], p, last, W, pt, bt)
        k = R.row_keys(kpool, table[0], pt, n)[:last + 1, 0]
        keep = (p - np.arange(last + 1))[:, None] <= W
        x = (np.concatenate([keep, keep], axis=1) * k) @ q.T
        for j in range(s.shape[1]):
            assert x[j * bt:(j + 1) * bt].max() <= s[0, j] + 1e-12
