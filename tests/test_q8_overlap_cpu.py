"""Appends with norms and reads of 8-bit caches refuse written buffers that overlap what the call reads
beside its tensors: weights, rows' positions and block tables.  No GPU: placeholder pointers."""
import ctypes

import pytest

atf = pytest.importorskip("paper_2608_02947_amd")
BIG = 1 << 34


@pytest.mark.parametrize("scaled", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("pages", [False, True], ids=["contiguous", "paged"])
def test_appends(scaled, pages):
    lib = atf.library()
    name = "atf_cache_append_" + ("paged_" if pages else "") + ("q8" if scaled else "normed")
    w, keep = atf.Window(128, 1e4, 2.0).as_c()
    batch, n, h_q, h_kv = 2, 10, 8, 2

    def call(n=n, **kw):
        a = dict(qo=4 * BIG, kc=5 * BIG, ks=6 * BIG, vc=7 * BIG, vs=8 * BIG, table=9 * BIG, rows=10 * BIG, qw=11 * BIG,
                 kw=12 * BIG)
        a.update(kw)
        cache = [a["kc"], a["ks"], a["vc"], a["vs"]] if scaled else [a["kc"], a["vc"]]
        place = [a["table"], 4, 8, 64] if pages else []
        tail = [] if pages else [256]
        return getattr(lib, name)(BIG, 2 * BIG, 3 * BIG, a["qo"], *cache, *place, batch, n, 0, a["rows"], h_q, h_kv, *tail,
                                  ctypes.byref(w), None, a["qw"], a["kw"], 1e-6, None)

    assert call(n=0) == atf.ATF_OK  # all apart, and nothing to do
    q_bytes = batch * n * h_q * 128 * 2
    sizes = dict(qw=512, kw=512, rows=4 * batch, **(dict(table=batch * 4 * 4) if pages else {}))
    written = ["qo", "kc", "vc"] + (["ks", "vs"] if scaled else [])
    start = dict(qo=4, kc=5, ks=6, vc=7, vs=8)
    for what, size in sizes.items():
        for at in written:
            assert call(**{what: start[at] * BIG}) == atf.ATF_EINVAL, (what, at)
            assert call(**{what: start[at] * BIG - size + 4}) == atf.ATF_EINVAL, (what, at)
        assert call(**{what: 4 * BIG + q_bytes - 4}) == atf.ATF_EINVAL, what
        assert "overlap" in atf.atf_last_error()
        assert call(n=0, **{what: 5 * BIG - size}) == atf.ATF_OK, what  # up to a buffer's start
    assert call(n=0, qw=11 * BIG, kw=11 * BIG) == atf.ATF_OK  # the same weights twice are only read


def test_reads_of_pages():
    lib = atf.library()

    def call(table, n):
        return lib.atf_cache_read_paged_q8(BIG, 2 * BIG, 3 * BIG, 4 * BIG, table, 4, 8, 64, 5 * BIG, 6 * BIG, 2, n, 0, 2, 128,
                                           300, None)

    assert call(9 * BIG, 0) == atf.ATF_OK and call(5 * BIG - 32, 0) == atf.ATF_OK
    for table in (5 * BIG, 6 * BIG + 1000, 5 * BIG - 28):
        assert call(table, 100) == atf.ATF_EINVAL and "overlap" in atf.atf_last_error()
