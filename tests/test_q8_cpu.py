"""The normed appends, the 8-bit caches and decode over them without a GPU: the plain forms the
GPU tests use against torch's own conversions, and every refusal before anything is launched
(the C calls get placeholder pointers; none passes validation except the no-ops)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import q8ref as R

atf = pytest.importorskip("paper_2608_02947_amd")
EINVAL, EUNSUP, EWS, OK = atf.ATF_EINVAL, atf.ATF_EUNSUPPORTED, atf.ATF_EWORKSPACE, atf.ATF_OK


def test_plain_e4m3_is_torchs():
    assert len(R.E4M3) == 127 and R.E4M3[-1] == 448.0
    allb = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(allb, R.E4M3)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.uniform(-448, 448, 4000), rng.normal(0, 2.0 ** -7, 4000), R.E4M3,
                        (R.E4M3[1:] + R.E4M3[:-1]) / 2])  # ties too
    x = x.astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(R.e4m3_round(x.astype(np.float64)), want)


def test_plain_exponent():
    for a, e in [(0.0, -60), (448.0, 0), (449.0, 1), (448.0 * 2.0 ** -60, -60), (1e-30, -60),
                 (447.0 * 2.0 ** 119, 119), (3.3e38, 119), (1.0, -8), (1.75, -8), (1.7578125, -7)]:
        assert R.exponent(np.array(a)) == e, a


def test_plain_decode_is_softmax():
    rng = np.random.default_rng(1)
    q, k, v = rng.normal(size=(4, 64)), rng.normal(size=(2, 9, 64)), rng.normal(size=(2, 9, 64))
    o, lse, _, _ = R.decode(q, k, v, 20, R.thresholds(64, 1e4, math.inf), 0.125)
    s = np.einsum("hd,htd->ht", q, k[[0, 0, 1, 1]]) * 0.125
    p = np.exp(s) / np.exp(s).sum(1, keepdims=True)
    assert np.allclose(o, np.einsum("ht,htd->hd", p, v[[0, 0, 1, 1]]))
    assert np.allclose(lse, np.log(np.exp(s).sum(1)))


def _window(d=128):
    return atf.Window(d, 1e4, 2.0).as_c()


BIG = 1 << 34  # placeholders far apart


@pytest.mark.parametrize("scaled", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("pages", [False, True], ids=["contiguous", "paged"])
def test_append_refusals(scaled, pages):
    lib = atf.library()

    def call(d=128, window=True, freq=None, **kw):
        a = dict(q=BIG, k=2 * BIG, v=3 * BIG, qo=4 * BIG, kc=5 * BIG, ks=6 * BIG, vc=7 * BIG, vs=8 * BIG,
                 table=9 * BIG, max_pages=4, num_pages=8, pt=64, batch=2, n=10, pos0=0, rows=None, h_q=8,
                 h_kv=2, cap=256, qw=None, kw=None, eps=1e-6)
        a.update(kw)
        w, keep = _window(d)
        f = None
        if freq is not None:
            arr = (ctypes.c_double * len(freq))(*freq)
            f = ctypes.cast(arr, ctypes.c_void_p)
        cache = [a["kc"], a["ks"], a["vc"], a["vs"]] if scaled else [a["kc"], a["vc"]]
        place = [a["table"], a["max_pages"], a["num_pages"], a["pt"]] if pages else []
        tail = [] if pages else [a["cap"]]
        name = "atf_cache_append_" + ("paged_" if pages else "") + ("q8" if scaled else "normed")
        rc = getattr(lib, name)(a["q"], a["k"], a["v"], a["qo"], *cache, *place, a["batch"], a["n"],
                                a["pos0"], a["rows"], a["h_q"], a["h_kv"], *tail,
                                ctypes.byref(w) if window else None, f, a["qw"], a["kw"], a["eps"], None)
        if rc != OK:
            assert name[4:] in atf.atf_last_error()
        return rc

    assert call(n=0) == OK and call(n=0, q=None, qo=None, h_q=0) == OK
    assert call(n=0, qo=BIG) == OK                       # in place
    assert call(n=0, q=None, qo=None, k=None, v=None) == OK  # tensors without elements
    for bad in (dict(window=False), dict(batch=0), dict(h_kv=0), dict(h_q=0), dict(n=-1), dict(pos0=-1),
                dict(q=None), dict(qo=None), dict(k=None), dict(v=None), dict(kc=None), dict(vc=None),
                dict(k=2 * BIG + 8), dict(qo=4 * BIG + 2), dict(kc=5 * BIG + 4), dict(eps=-1.0),
                dict(eps=math.inf), dict(eps=math.nan), dict(rows=3), dict(qw=2), dict(kw=1),
                dict(pos0=250), dict(rows=1 << 12, pos0=1), dict(n=2 ** 31, rows=1 << 12),
                dict(batch=2 ** 20, n=2 ** 12, rows=1 << 12), dict(freq=[-1.0] * 64),
                dict(freq=[math.nan] * 64), dict(qo=BIG + 16), dict(kc=2 * BIG), dict(vc=5 * BIG + 256),
                dict(qo=7 * BIG)):
        assert call(**bad) == EINVAL, bad
    assert call(d=80) == EUNSUP and call(h_q=70000) == EUNSUP
    if scaled:
        for bad in (dict(ks=None), dict(vs=None), dict(ks=6 * BIG + 8), dict(vs=6 * BIG), dict(ks=5 * BIG + 16)):
            assert call(**bad) == EINVAL, bad
    if pages:
        for bad in (dict(table=None), dict(table=9 * BIG + 2), dict(pt=48), dict(pt=0), dict(num_pages=0),
                    dict(max_pages=0), dict(max_pages=2 ** 26, pt=64)):
            assert call(**bad) == EINVAL, bad
    else:
        assert call(cap=0) == EINVAL and call(cap=2 ** 31) == EINVAL


def test_largest_capacity():
    """Scales of the longest caches, 2^31 a head, are counted as such: buffers apart are accepted."""
    lib, far = atf.library(), 1 << 44
    (w, keep), cap = _window(64), 2 ** 31 - 1
    at = [None] + [far * i for i in (1, 2)] + [None] + [far * i for i in (3, 4, 5, 6)]
    assert lib.atf_cache_append_q8(*at, 1, 0, 0, None, 0, 1, cap, ctypes.byref(w), None, None, None, 1e-6, None) == OK
    assert lib.atf_cache_read_q8(*[far * i for i in range(1, 7)], 1, 0, cap, 1, 64, cap, cap, None) == OK
    # the same buffers nearer than a head's 2^31 scales
    at[5], at[7] = far, far + 2 ** 31 - 16
    assert lib.atf_cache_append_q8(*at, 1, 0, 0, None, 0, 1, cap, ctypes.byref(w), None, None, None, 1e-6, None) == EINVAL


@pytest.mark.parametrize("pages", [False, True], ids=["contiguous", "paged"])
def test_read_refusals(pages):
    lib = atf.library()

    def call(**kw):
        a = dict(k=BIG, ks=2 * BIG, v=3 * BIG, vs=4 * BIG, table=9 * BIG, max_pages=4, num_pages=8, pt=64,
                 kc=5 * BIG, vc=6 * BIG, batch=2, n=100, pos0=0, h_kv=2, d=128, src=256, cap=300)
        a.update(kw)
        src = [a["k"], a["ks"], a["v"], a["vs"]]
        if pages:
            return lib.atf_cache_read_paged_q8(*src, a["table"], a["max_pages"], a["num_pages"], a["pt"],
                                               a["kc"], a["vc"], a["batch"], a["n"], a["pos0"], a["h_kv"],
                                               a["d"], a["cap"], None)
        return lib.atf_cache_read_q8(*src, a["kc"], a["vc"], a["batch"], a["n"], a["pos0"], a["h_kv"], a["d"],
                                     a["src"], a["cap"], None)

    assert call(n=0) == OK and call(n=0, pos0=256) == OK
    for bad in (dict(k=None), dict(ks=None), dict(v=None), dict(vs=None), dict(kc=None), dict(vc=None),
                dict(k=BIG + 8), dict(vs=4 * BIG + 4), dict(vc=6 * BIG + 2), dict(batch=0), dict(h_kv=0),
                dict(n=-1), dict(pos0=-1), dict(n=257), dict(pos0=157), dict(cap=99), dict(cap=0),
                dict(cap=2 ** 31), dict(kc=BIG), dict(vc=5 * BIG + 64), dict(kc=4 * BIG + 16)):
        assert call(**bad) == EINVAL, bad
    assert call(d=80) == EUNSUP and call(batch=40000) == EUNSUP
    if pages:
        for bad in (dict(table=None), dict(pt=40), dict(num_pages=0), dict(max_pages=0)):
            assert call(**bad) == EINVAL, bad
    else:
        assert call(src=0) == EINVAL and call(src=2 ** 31) == EINVAL


@pytest.mark.parametrize("form", ["uniform", "ragged", "paged"])
def test_decode_refusals(form):
    lib = atf.library()
    need = atf.atf_decode_workspace_bytes(2, 24, 8, 256, 128)

    def call(d=128, window=True, **kw):
        a = dict(q=BIG, k=2 * BIG, ks=3 * BIG, v=4 * BIG, vs=5 * BIG, o=6 * BIG, lse=7 * BIG, batch=2, n=256,
                 q_pos=255, nk=1 << 13, qp=1 << 14, table=9 * BIG, max_pages=4, num_pages=8, pt=64, h_q=24,
                 h_kv=8, cap=256, scale=0.0, ws=8 * BIG, size=16)
        a.update(kw)
        w, keep = _window(d)
        pre = [a["q"], a["k"], a["ks"], a["v"], a["vs"], a["o"], a["lse"], a["batch"]]
        post = [ctypes.byref(w) if window else None, a["scale"], a["ws"], a["size"], None]
        if form == "uniform":
            return lib.atf_decode_q8(*pre, a["n"], a["q_pos"], a["h_q"], a["h_kv"], a["cap"], *post)
        if form == "ragged":
            return lib.atf_decode_ragged_q8(*pre, a["nk"], a["qp"], a["n"], a["h_q"], a["h_kv"], a["cap"], *post)
        return lib.atf_decode_paged_q8(*pre, a["table"], a["max_pages"], a["num_pages"], a["pt"], a["nk"],
                                       a["qp"], a["n"], a["h_q"], a["h_kv"], *post)

    assert call() == EWS and call(ws=None, size=need) == EWS     # all else valid
    for bad in (dict(window=False), dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(lse=None),
                dict(q=BIG + 8), dict(lse=7 * BIG + 2), dict(batch=0), dict(n=0), dict(h_q=0), dict(h_kv=0),
                dict(h_kv=5), dict(scale=math.inf), dict(scale=math.nan), dict(size=need, ws=8 * BIG + 8),
                dict(size=need, ks=None), dict(size=need, vs=None), dict(size=need, ks=3 * BIG + 8),
                dict(size=need, vs=5 * BIG + 1)):
        assert call(**bad) == EINVAL, bad
    assert call(d=96) == EUNSUP
    if form == "uniform":
        assert call(q_pos=-1) == EINVAL and call(q_pos=2 ** 31 - 1) == EINVAL and call(cap=255) == EINVAL
    else:
        for bad in (dict(nk=None), dict(qp=None), dict(nk=(1 << 13) + 1), dict(qp=(1 << 14) + 2), dict(n=257)):
            assert call(**bad) == EINVAL, bad
    if form == "paged":
        for bad in (dict(table=None), dict(table=9 * BIG + 1), dict(pt=48), dict(num_pages=0), dict(max_pages=0)):
            assert call(**bad) == EINVAL, bad


def test_binding_refuses_shapes_types_and_host_tensors():
    B, n, h_q, h_kv, d, cap = 2, 3, 4, 2, 64, 40
    bf = torch.bfloat16
    win = atf.Window(d, 1e4, 2.0)
    q, k = torch.zeros(B, n, h_q, d, dtype=bf), torch.zeros(B, n, h_kv, d, dtype=bf)
    kc, vc = torch.zeros(atf.kcache_shape(B, cap, h_kv, d), dtype=bf), torch.zeros(atf.vcache_shape(B, cap, h_kv, d), dtype=bf)
    with pytest.raises(ValueError, match="on the GPU"):
        atf.atf_cache_append_normed(q, k, k, q, kc, vc, 0, win)
    with pytest.raises(ValueError, match="together"):
        atf.atf_cache_append_normed(None, k, k, q, kc, vc, 0, win)
    with pytest.raises(ValueError, match="inconsistent"):
        atf.atf_cache_append_normed(None, k, k[:, :2], None, kc, vc, 0, win)
    with pytest.raises(ValueError, match="inconsistent"):
        atf.atf_cache_append_normed(q[:1], k, k, q[:1], kc, vc, 0, win)
    with pytest.raises(ValueError, match="inconsistent"):
        atf.atf_cache_append_normed(q, k, k, q, kc, vc, 0, atf.Window(128, 1e4, 2.0))
    assert atf.qscale_shape(2, 40, 3) == (2, 3, 48) and atf.qscale_shape(5, 64, 1) == (5, 1, 64)
    k8, v8 = kc.to(torch.float8_e4m3fn), vc.to(torch.float8_e4m3fn)
    sc = torch.zeros(atf.qscale_shape(B, cap, h_kv), dtype=torch.uint8).view(torch.float8_e8m0fnu)
    o, lse, ws = q[:, 0].contiguous(), torch.zeros(B, h_q), torch.zeros(1, dtype=torch.uint8)
    with pytest.raises(ValueError, match="qscale_shape"):
        atf.atf_cache_read_q8(k8, sc[:, :, :40], v8, sc, kc, vc, 8)
    with pytest.raises(ValueError, match="inconsistent"):
        atf.atf_cache_read_q8(k8, sc, v8, sc, kc, vc[:, :, :2], 8)
    with pytest.raises(ValueError, match="inconsistent"):
        atf.atf_decode_q8(o, k8, sc, v8, sc, o, lse[:1], 5, win, ws)
    with pytest.raises(ValueError):
        atf.atf_decode_paged_q8(o, k8[0], sc, v8, sc, o, lse, torch.zeros(B, 2, dtype=torch.int32),
                                torch.zeros(B, dtype=torch.int32), torch.zeros(B, dtype=torch.int32), 5, win, ws)


def _rule(name, restype, *argtypes):
    f = getattr(ctypes.CDLL(atf.LIB_PATH), name)
    f.restype, f.argtypes = restype, argtypes
    return f


_i32, _i64, _bool = ctypes.c_int32, ctypes.c_int64, ctypes.c_bool
_direct = _rule("_ZN3atf16decode_q8_directEliilb", _bool, _i64, _i32, _i32, _i64, _bool)
_waves = _rule("_ZN3atf15decode_q8_wavesEillbb", _i32, _i32, _i64, _i64, _bool, _bool)
_slots = _rule("_ZN3atf15decode_q8_slotsEiii", _i32, _i32, _i32, _i32)
_splits = _rule("_ZN3atf16decode_q8_splitsElll", _i64, _i64, _i64, _i64)
_room = _rule("_ZN3atf13decode_splitsEiil", _i32, _i32, _i32, _i64)


def test_decode_plan_rules():
    """Whole rows or splits, 4 or 8 waves: both sides of the rules' borders."""
    assert _direct(8, 128, 1, 800, False) and not _direct(8, 128, 1, 801, False)
    assert _direct(200, 128, 1, 10 ** 6, False) and not _direct(300, 128, 1, 1501, False)
    assert _direct(512, 128, 2, 10 ** 6, False) and not _direct(128, 64, 2, 1801, False)
    assert _direct(64, 64, 1, 1100, True) and not _direct(64, 64, 1, 1101, True)
    assert _direct(100, 128, 1, 1200, True) and not _direct(100, 128, 1, 1201, True)
    assert _direct(200, 128, 2, 1920, True) and not _direct(160, 128, 2, 1281, True)
    assert _direct(4096, 128, 1, 4800, True) and not _direct(4096, 128, 1, 4801, True)
    assert _waves(1, 256, 1000, False, True) == 8 and _waves(1, 257, 1000, False, True) == 4
    assert _waves(1, 4, 24000, False, False) == 8 and _waves(1, 4, 23999, False, False) == 4
    assert _waves(1, 5, 10 ** 6, False, False) == 4 and _waves(2, 5, 10 ** 6, False, False) == 8
    assert _waves(2, 128, 500, True, False) == 8 and _waves(2, 129, 500, True, False) == 4
    assert _waves(1, 2, 96000, True, False) == 8 and _waves(1, 2, 95999, True, False) == 4


def test_decode_splits_fit_the_workspace():
    """Splits and the states they write: within the workspace's room, none without keys."""
    for d in (64, 128):
        for tiles in (1, 2):
            for waves in (4, 8):
                slots = _slots(d, tiles, waves)
                for batch in (1, 2, 3, 7, 16, 36, 100, 400, 5000):
                    for h_kv in (1, 2, 5, 8, 64):
                        for n in (1, 255, 256, 257, 5000, 131072, 10 ** 6, 2 ** 31 - 2):
                            steps = -(-n // 256)
                            room = min(_room(batch, h_kv, n), steps)
                            s = _splits(batch * h_kv, slots, room)
                            assert 1 <= s <= room
                            per = -(-steps // s)
                            used = -(-steps // per)
                            assert used <= s and (used - 1) * per * 256 < n <= used * per * 256
