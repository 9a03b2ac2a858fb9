"""The appends with norms, the 8-bit caches, reading them back and decode over them on the GPU,
against the plain 64-bit forms of q8ref.py; tolerances are derived there."""
import math

import numpy as np
import pytest
import torch

import q8ref as R
from conftest import gpu_available
from parity import note

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]

DEV, BF, E4, E8 = "cuda", torch.bfloat16, torch.float8_e4m3fn, torch.float8_e8m0fnu
EPS = 1e-6
SENTINEL = 0x5A  # byte of every slot that no call writes


def randn(shape, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(BF)


class Case:
    """An append: inputs on the host, caches full of the sentinel on the GPU, and what came out."""

    def __init__(self, d, h_q, h_kv, B, n, q8, pos, cap=100, pages=0, norm=True, base=1e4, seed=0, q=True,
                 tweak=None, pos0=None):
        import paper_2608_02947_amd as atf
        self.d, self.h_kv, self.B, self.n, self.q8, self.cap, self.pages = d, h_kv, B, n, q8, cap, pages
        self.pos = np.array(pos if pos0 is None else [pos0] * B)
        self.q = randn((B, n, h_q, d), seed + 1) if q else None
        self.k, self.v = randn((B, n, h_kv, d), seed + 2, 2.0), randn((B, n, h_kv, d), seed + 3)
        if tweak is not None:
            tweak(self)
        g = torch.Generator().manual_seed(seed + 4)
        self.qw = 1 + 0.3 * torch.randn(d, generator=g) if norm else None
        self.kw = 1 + 0.3 * torch.randn(d, generator=g) if norm else None
        self.theta = R.theta(d, base)
        lead, T = B, cap
        self.table = None
        if pages:
            width = -(-cap // pages)
            lead, T = B * width + 3, pages
            self.table = torch.randperm(lead, generator=g)[: B * width].view(B, width).to(torch.int32)
        fill = lambda shape, dt: torch.full(shape + ((1 if q8 else 2),), SENTINEL, dtype=torch.uint8,
                                            device=DEV).view(dt).view(shape)
        dt = E4 if q8 else BF
        self.kc, self.vc = fill(atf.kcache_shape(lead, T, h_kv, d), dt), fill(atf.vcache_shape(lead, T, h_kv, d), dt)
        if q8:
            one = lambda: torch.full(atf.qscale_shape(lead, T, h_kv), SENTINEL, dtype=torch.uint8, device=DEV).view(E8)
            self.ks, self.vs = one(), one()
        self.pos0 = pos0

    def run(self, in_place=False, stream=None):
        import paper_2608_02947_amd as atf
        dev = lambda t: None if t is None else t.to(DEV)
        q = dev(self.q)
        self.q_out = q if in_place or q is None else torch.full_like(q, 7.0)
        win = atf.Window(self.d, 1e4, 2.0)
        more = dict(q_weight=dev(self.qw), k_weight=dev(self.kw), eps=EPS, rope_inv_freq=self.theta, stream=stream)
        if self.pos0 is None:
            more["pos_rows"] = torch.tensor(self.pos, dtype=torch.int32, device=DEV)
        args = [q, dev(self.k), dev(self.v), self.q_out]
        args += [self.kc, self.ks, self.vc, self.vs] if self.q8 else [self.kc, self.vc]
        if self.pages:
            args.append(dev(self.table))
        name = "atf_cache_append_" + ("paged_" if self.pages else "") + ("q8" if self.q8 else "normed")
        getattr(atf, name)(*args, self.pos0 or 0, win, **more)
        torch.cuda.synchronize()
        return self

    def tokens(self):
        """Bytes of the caches as tokens: k and v [lead, h, T, d] of unsigned numbers, scales."""
        raw = lambda t: t.cpu().view(torch.uint8 if self.q8 else torch.int16).numpy()
        T = self.kc.shape[3]
        k, v = R.k_tokens(raw(self.kc)), R.v_tokens(raw(self.vc), not self.q8)[:, :, :T]
        sc = [t.cpu().view(torch.uint8).numpy()[:, :, :T] for t in (self.ks, self.vs)] if self.q8 else [None, None]
        return k, v, sc[0], sc[1]

    def check(self):
        k, v, ks, vs = self.tokens()
        touched = np.zeros(k.shape[:3], bool)
        q_out = None if self.q is None else R.f64(self.q_out)
        for b in range(self.B):
            first = int(self.pos[b])
            if first < 0:
                if self.q is not None:
                    assert (q_out[b] == 7.0).all()
                continue
            pos = first + np.arange(self.n, dtype=np.int64)
            if self.q is not None:
                want, err = R.norm_rotate(R.f64(self.q[b]), None if self.qw is None else R.f64(self.qw), EPS, pos, self.theta)
                bad = ~np.isfinite(want)
                assert np.array_equal(bad, ~np.isfinite(q_out[b]))
                d = np.abs(q_out[b] - want)
                assert (d <= R.BF16_HALF * np.abs(want) + err + 2.0 ** -133)[~bad].all()
            kw, kerr = R.norm_rotate(R.f64(self.k[b]), None if self.kw is None else R.f64(self.kw), EPS, pos, self.theta)
            vw = R.f64(self.v[b])
            for t in range(self.n):
                p = first + t
                if p >= (self.cap if not self.pages else self.pages * self.table.shape[1]):
                    continue
                e, s = (b, p) if not self.pages else (int(self.table[b, p // self.pages]), p % self.pages)
                if e < 0 or e >= k.shape[0]:
                    continue
                touched[e, :, s] = True
                if self.q8:
                    self.check_row(k[e, :, s], ks[e, :, s], kw[t], kerr[t])
                    num, ex = R.quantise(vw[t])
                    got = torch.from_numpy(v[e, :, s].copy()).view(E4).float().numpy().astype(np.float64)
                    assert np.array_equal(vs[e, :, s].astype(int) - 127, ex)
                    assert np.array_equal(got, num, equal_nan=True)
                else:
                    got = (k[e, :, s].astype(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)
                    bad = ~np.isfinite(kw[t])
                    assert np.array_equal(bad, ~np.isfinite(got))
                    assert (np.abs(got - kw[t]) <= R.BF16_HALF * np.abs(kw[t]) + kerr[t] + 2.0 ** -133)[~bad].all()
                    assert np.array_equal(v[e, :, s], self.v[b, t].view(torch.int16).numpy())
        rest = SENTINEL if self.q8 else SENTINEL * 257
        assert (k[~touched] == rest).all() and (v[~touched] == rest).all()
        if self.q8:
            assert (ks[~touched] == SENTINEL).all() and (vs[~touched] == SENTINEL).all()

    def check_row(self, byte, scale, want, err):
        """Keys of one token, [h, d]: the power is that of the largest, or, where that is nearer
        to a border than its own error, the next; numbers within half a step of the power."""
        got = torch.from_numpy(byte.copy()).view(E4).float().numpy().astype(np.float64)
        fin = np.isfinite(want)
        assert np.array_equal(fin, np.isfinite(got))
        a = np.where(fin, np.abs(want), 0.0)
        e = scale.astype(int) - 127
        slack = np.where(fin, err, 0.0).max(-1)
        assert (e >= R.exponent(np.maximum(a.max(-1) - slack, 0.0))).all()
        assert (e <= R.exponent(a.max(-1) + slack)).all()
        power = 2.0 ** e[:, None].astype(np.float64)
        off = np.abs(np.where(fin, got * power, 0.0) - np.where(fin, np.clip(want, -448 * power, 448 * power), 0.0))
        assert (off <= np.maximum(R.E4M3_HALF * a, R.E4M3_TINY * power) * (1 + 2.0 ** -10) + np.where(fin, err, 0.0)).all()


APPENDS = [  # d, h_q, h_kv, B, n, positions, cap, pages
    (64, 3, 1, 1, 1, [0], 1, 0),
    (64, 14, 2, 3, 1, [17, -1, 63], 64, 32),
    (128, 8, 2, 5, 1, [0, 15, 16, -1, 99], 100, 0),
    (128, 4, 4, 2, 3, [30, 95], 100, 0),             # past the end of one row
    (64, 2, 2, 2, 16, [0, 13], 40, 0),
    (128, 5, 1, 3, 33, [0, 7, 31], 100, 96),
    (64, 1, 3, 2, 67, [2, 5], 77, 0),
    (128, 6, 2, 1, 100, [0], 100, 32),
    (128, 28, 4, 2, 131, [16, 3], 150, 0),
    (64, 14, 2, 3, 48, [17, -1, 63], 120, 32),
    (64, 16, 16, 3, 4001, [-1, 5, 300], 4200, 0),    # more heads of a wave than it loads at once
    (128, 40, 2, 2, 1701, [9, 100], 1790, 64),       # queries past the L2s
]


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("norm", [True, False], ids=["normed", "plain"])
@pytest.mark.parametrize("i", range(len(APPENDS)))
def test_append(i, norm, q8):
    d, h_q, h_kv, B, n, pos, cap, pages = APPENDS[i]
    note(f"append {APPENDS[i]} norm={norm} q8={q8}")
    Case(d, h_q, h_kv, B, n, q8, pos, cap, pages, norm, seed=10 * i).run().check()


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("d", [64, 128])
def test_append_one_position_for_all_rows(d, q8):
    note(f"append pos0 {d} {q8}")
    Case(d, 4, 2, 3, 21, q8, None, 60, 0, pos0=39).run().check()
    Case(d, 4, 2, 3, 21, q8, None, 64, 32, pos0=0, q=False).run().check()


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("d,h_kv,B,n", [(64, 1, 1, 1), (128, 3, 2, 50), (64, 5, 3, 17), (128, 1, 1, 7)])
def test_append_without_queries(d, h_kv, B, n, q8):
    """Waves of the last workgroup without work, and no queries that they could take."""
    note(f"append no queries {d} {h_kv} {B} {n} {q8}")
    Case(d, 1, h_kv, B, n, q8, None, 60, 0, pos0=5, q=False).run().check()


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_append_in_place_far_positions_and_streams(q8):
    """Queries far past the cache (their keys are not stored) and written over themselves, on
    another stream."""
    note(f"append far q8={q8}")
    st = torch.cuda.Stream()
    c = Case(128, 6, 2, 2, 5, q8, [2 ** 30 + 5, 3], 20, 0, base=1e7)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        c.run(in_place=True, stream=st)
    c.check()
    note(f"append at the end of the positions q8={q8}")
    c = Case(64, 2, 1, 2, 2, q8, [2 ** 31 - 2, 4], 20, 0)  # the second token is past 2^31 - 2
    got = c.run().q_out.cpu()
    assert (got[0, 1] == 7.0).all() and (got[0, 0] != 7.0).any()


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_append_bad_pages_are_skipped(q8):
    note(f"append bad pages q8={q8}")
    c = Case(64, 2, 2, 2, 70, q8, [0, 20], 96, 32)
    c.table[0, 1], c.table[1, 2] = -1, c.kc.shape[0]
    c.run().check()


@pytest.mark.parametrize("n", [1, 16, 37])
def test_append_q8_numbers_at_the_edges(n):
    """Rows of zeros, infinities and NaN, the largest and the smallest magnitudes."""
    note(f"append edges n={n}")

    def tweak(c):
        for x in (c.k, c.v):
            x[0, 0, 0] = 0.0
            x[0, 0, 1, 3], x[0, 0, 1, 7], x[0, 0, 1, 9] = math.inf, -math.inf, math.nan
            x[1, 0, 0] *= 2.0 ** 126
            x[1, 0, 1] *= 2.0 ** -80
            x[2, 0, 0] *= 2.0 ** -130
            x[2, 0, 1] = math.nan
            x[3, 0, 0, 5] = 2.0 ** 40
    c = Case(64, 1, 2, 4, n, True, [0, 3, 16, 20], 60, 0, norm=False, tweak=tweak)
    # (the keys' turn adds pairs: only those that stay finite in fp32 have a value to compare)
    c.theta = np.zeros(32)
    c.run().check()


def test_append_normed_zero_rows_and_nan():
    note("append normed zeros")

    def tweak(c):
        c.q[0, 0, 0] = 0.0
        c.k[0, 0, 0] = 0.0
        c.k[1, 0, 0, 3] = math.nan
    c = Case(128, 2, 2, 2, 2, True, [0, 0], 20, 0, tweak=tweak).run()
    k, _, ks, _ = c.tokens()
    assert (c.q_out[0, 0, 0] == 0).all() and (k[0, 0, 0] & 127 == 0).all() and ks[0, 0, 0] == 67
    assert ((k[1, 0, 0] & 127) == 127).all() and ks[1, 0, 0] == 67  # the norm makes all of them NaN
    assert ((k[1, 1, 0] & 127) != 127).all()


@pytest.mark.parametrize("d,h_kv,cap,n,pos0,pages", [
    (64, 1, 1, 1, 0, 0), (128, 3, 50, 33, 9, 0), (64, 2, 64, 64, 0, 32), (128, 2, 100, 3, 95, 0),
    (64, 5, 130, 77, 50, 96), (128, 4, 200, 200, 0, 0), (64, 2, 40, 16, 16, 0)])
def test_read_back(d, h_kv, cap, n, pos0, pages):
    import paper_2608_02947_amd as atf
    note(f"read {d} {h_kv} {cap} {n} {pos0} {pages}")
    c = Case(d, 1, h_kv, 2, cap, True, None, cap, pages, pos0=0, q=False).run()
    out = cap + 7
    full = lambda shape: torch.full(shape, -7.0, dtype=BF, device=DEV)
    kc, vc = full(atf.kcache_shape(2, out, h_kv, d)), full(atf.vcache_shape(2, out, h_kv, d))
    src = (c.kc, c.ks, c.vc, c.vs)
    if pages:
        atf.atf_cache_read_paged_q8(*src, c.table.to(DEV), kc, vc, n, pos0)
    else:
        atf.atf_cache_read_q8(*src, kc, vc, n, pos0)
    torch.cuda.synchronize()
    k, v, ks, vs = c.tokens()
    for got, x, s in ((R.k_tokens(R.f64(kc)), k, ks), (R.v_tokens(R.f64(vc), True), v, vs)):
        x = torch.from_numpy(np.ascontiguousarray(x)).view(E4).float().numpy() * np.exp2(s.astype(np.float64) - 127)[..., None]
        for b in range(2):
            row = x[b] if not pages else R.paged(x, c.table.numpy(), b, pages, cap)
            assert np.array_equal(got[b, :, pos0:pos0 + n], row[:, pos0:pos0 + n])
            assert (got[b, :, :pos0] == -7.0).all() and (got[b, :, pos0 + n:] == -7.0).all()


# ---- decode

def q8_caches(B, h_kv, T, d, seed, spread=0):
    """Random 8-bit caches: (numbers k, v [B, h, T, d] and exponents [B, h, T], as arrays)."""
    rng = np.random.default_rng(seed)
    out = []
    for _ in "kv":  # (rows out of a pool of them)
        pool = rng.normal(size=(2048, d)) * 2.0 ** rng.integers(-spread, spread + 1, (2048, 1))
        x, e = R.quantise(pool)
        at = rng.integers(0, 2048, (B, h_kv, T))
        out += [x[at], e[at]]
    return out


def to_layout(x, e, v, pages=0):
    """[lead, h, T, d] numbers and exponents -> the K (or V) cache and its scales, on the GPU; slots
    past T hold NaN."""
    lead, h, T, d = x.shape
    T16 = (T + 15) // 16 * 16
    b = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(E4).view(torch.uint8)
    if v:
        full = torch.full((lead, h, T16, d), 0x7F, dtype=torch.uint8)
        full[:, :, :T] = b
        c = full.view(lead, h, T16 // 16, 16, d).transpose(3, 4)
    else:
        c = b[..., torch.from_numpy(R.dims(d))].permute(0, 1, 3, 2, 4)
    s = torch.full((lead, h, T16), 0xFF, dtype=torch.uint8)
    s[:, :, :T] = torch.from_numpy(e + 127).to(torch.uint8)
    return c.contiguous().to(DEV).view(E4), s.to(DEV).view(E8)


def value(x, e):
    return x * 2.0 ** e[..., None].astype(np.float64)


def workspace(B, h_q, h_kv, n, d):
    import paper_2608_02947_amd as atf
    size = atf.atf_decode_workspace_bytes(B, h_q, h_kv, n, d)
    return torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV)  # NaN states


def sample(B):
    """All rows of a small batch; of a large one every seventh and the last (each is a loop here)."""
    return range(B) if B <= 16 else [*range(0, B - 1, 7), B - 1]


def judge(o, lse, want):
    o, lse = R.f64(o), lse.cpu().numpy().astype(np.float64)
    for b, (wo, wl, oe, le) in zip(sample(len(o)), want):
        inf = np.isinf(wl)
        assert np.array_equal(inf, np.isinf(lse[b])), b
        assert (o[b][inf] == 0).all()
        assert (np.abs(o[b] - wo) <= oe)[~inf].all(), (b, np.max(np.abs(o[b] - wo) / np.maximum(oe, 1e-300)))
        assert (np.abs(lse[b][~inf] - wl[~inf]) <= le[~inf]).all(), b


def window(kind, d, base=1e4):
    """(window, thresholds) independently on both sides."""
    import paper_2608_02947_amd as atf
    if kind == "off":
        return atf.Window(d, base, math.inf), R.thresholds(d, base, math.inf)
    if kind == "sliding":  # every pair ends at 40: cells beyond have score 0
        return (atf.Window(d, base, 1.0, k_profile=[0.0] * (d // 2), beta=40.0, cap=40.0),
                np.full(d // 2, 40, dtype=np.int64))
    if kind == "rounded":
        W = R.thresholds(d, base, 2.0)
        return atf.Window(d, base, 2.0, slice_pairs=8), W.reshape(-1, 8)[:, 7].repeat(8)
    return atf.Window(d, base, 2.0), R.thresholds(d, base, 2.0)


DECODES = [  # d, h_q, h_kv, B, n_k, q_pos, cap
    (64, 1, 1, 1, 1, 0, 1), (128, 4, 2, 2, 1, 5, 3), (64, 7, 1, 1, 63, 62, 63), (128, 3, 1, 3, 64, 64, 70),
    (64, 16, 1, 1, 65, 70, 65), (128, 17, 1, 2, 255, 254, 256), (64, 40, 2, 1, 257, 300, 260),
    (128, 28, 4, 2, 1000, 999, 1003), (64, 33, 1, 1, 700, 699, 700), (128, 16, 16, 1, 513, 400, 600),
    (128, 8, 1, 1, 5001, 5000, 5001), (64, 5, 5, 2, 2049, 2100, 2050),
    (64, 4, 4, 80, 70, 69, 70), (128, 2, 2, 150, 33, 40, 48),   # more rows than a round of workgroups
    (64, 1, 1, 1, 40000, 39999, 40000), (128, 40, 1, 1, 20000, 20010, 20001),  # merges of 8 and 16 waves
    (64, 3, 1, 260, 1530, 1529, 1530),                          # few splits of many rows
    # split over workgroups of 8 waves
    (128, 4, 2, 1, 50011, 50010, 50020), (64, 2, 1, 1, 96005, 97000, 96010), (128, 20, 1, 1, 97000, 96999, 97000),
]


@pytest.mark.parametrize("i,kind", [(i, kind) for i in range(len(DECODES)) for kind in
                                    (["exact", "off", "sliding", "rounded"] if i < 12 else ["exact", "off"])])
def test_decode(i, kind):
    import paper_2608_02947_amd as atf
    d, h_q, h_kv, B, n_k, q_pos, cap = DECODES[i]
    note(f"decode {DECODES[i]} {kind}")
    k, ke, v, ve = q8_caches(B, h_kv, n_k, d, 100 + i, spread=3)
    pad = lambda x: np.concatenate([x, np.zeros((B, h_kv, cap - n_k) + x.shape[3:])], axis=2)
    kc, ks = to_layout(pad(k), pad(ke).astype(int), False)
    vc, vs = to_layout(pad(v), pad(ve).astype(int), True)
    # slots past n_k hold NaN, their powers are no numbers
    kc.view(torch.uint8)[:, :, :, n_k:] = 0x7F
    T16 = vs.shape[2]
    flat = vc.view(torch.uint8).transpose(3, 4).reshape(B, h_kv, T16, d)
    flat[:, :, n_k:] = 0x7F
    vc = flat.view(B, h_kv, T16 // 16, 16, d).transpose(3, 4).contiguous().view(E4)
    for s in (ks, vs):
        s.view(torch.uint8)[:, :, n_k:] = 0xFF
    win, W = window(kind, d)
    q = randn((B, h_q, d), 7 + i)
    o, lse = torch.empty_like(q, device=DEV), torch.empty((B, h_q), device=DEV)
    args = (q.to(DEV), kc, ks, vc, vs, o, lse, q_pos, win, workspace(B, h_q, h_kv, n_k, d))
    atf.atf_decode_q8(*args, n_k=n_k)
    torch.cuda.synchronize()
    want = [R.decode(R.f64(q[b]), value(k, ke)[b], value(v, ve)[b], q_pos, W, d ** -0.5) for b in sample(B)]
    judge(o, lse, want)
    first = o.clone(), lse.clone()
    atf.atf_decode_q8(*args, n_k=n_k)
    assert torch.equal(first[0], o) and torch.equal(first[1], lse)


RAGGED = [  # d, h_q, h_kv, lengths, query positions less lengths, pages
    (64, 14, 2, [0, 1, 300, 64], 0), (128, 24, 8, [77, 0, 0, 513, 2, 1200], 0), (128, 20, 1, [400, 31, 0], 32),
    (64, 16, 16, [65, 129, 1, 1000], 96), (128, 32, 4, [1, 2048, 33], 64), (64, 2, 1, [5] * 70, 32),
    (64, 3, 1, [(37 * i) % 2300 for i in range(130)], 0), (128, 2, 1, [4000 - 900 * i for i in range(5)] + [3] * 90, 32),
    (64, 20, 2, [3000, 0, 1, 2999], 0),
    (64, 4, 1, [96001, 700], 0), (64, 17, 1, [(53 * i) % 2500 for i in range(132)], 0),
]


@pytest.mark.parametrize("kind", ["exact", "off"])
@pytest.mark.parametrize("i", range(len(RAGGED)))
def test_decode_rows_of_their_own(i, kind):
    import paper_2608_02947_amd as atf
    d, h_q, h_kv, lens, pages = RAGGED[i]
    note(f"decode ragged {RAGGED[i]} {kind}")
    B, top = len(lens), max(lens)
    k, ke, v, ve = q8_caches(B, h_kv, top, d, 200 + i)
    q_pos = [max(n - 1 + (b % 3) - 1, 0) for b, n in enumerate(lens)]  # before, at and past the last key
    win, W = window(kind, d)
    q = randn((B, h_q, d), 17 + i)
    o, lse = torch.empty_like(q, device=DEV), torch.empty((B, h_q), device=DEV)
    rows = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in (lens, q_pos)]
    ws = workspace(B, h_q, h_kv, top, d)
    if pages:
        width = -(-top // pages) + 1
        pool = B * width + 2
        table = torch.randperm(pool, generator=torch.Generator().manual_seed(i))[: B * width].view(B, width).to(torch.int32)
        put = lambda x: _into_pages(x, table, pool, pages)
        (kc, ks), (vc, vs) = to_layout(put(k), put(ke), False), to_layout(put(v), put(ve), True)
        for b, n in enumerate(lens):  # entries no key needs: any number
            table[b, -(-n // pages):] = (-5, pool + 9)[b % 2]
        atf.atf_decode_paged_q8(q.to(DEV), kc, ks, vc, vs, o, lse, table.to(DEV), *rows, top, win, ws)
    else:
        kc, ks = to_layout(k, ke, False)
        vc, vs = to_layout(v, ve, True)
        atf.atf_decode_ragged_q8(q.to(DEV), kc, ks, vc, vs, o, lse, *rows, top, win, ws)
    torch.cuda.synchronize()
    want = [R.decode(R.f64(q[b]), value(k, ke)[b, :, : lens[b]], value(v, ve)[b, :, : lens[b]], q_pos[b], W, d ** -0.5)
            for b in sample(B)]
    judge(o, lse, want)


def _into_pages(x, table, pool, pages):
    """[B, h, T, ..] -> [pool, h, pages, ..]; what no row uses is 0."""
    out = np.zeros((pool, x.shape[1], pages) + x.shape[3:], x.dtype)
    for b in range(x.shape[0]):
        for j in range(-(-x.shape[2] // pages)):
            part = x[b, :, j * pages:(j + 1) * pages]
            out[int(table[b, j]), :, : part.shape[1]] = part
    return out


def test_decode_clamps_rows():
    """Lengths and positions outside their ranges read nothing outside the caches."""
    import paper_2608_02947_amd as atf
    note("decode clamps")
    d, T = 64, 50
    k, ke, v, ve = q8_caches(3, 1, T, d, 5)
    (kc, ks), (vc, vs) = to_layout(k, ke, False), to_layout(v, ve, True)
    q = randn((3, 2, d), 3)
    o, lse = torch.empty_like(q, device=DEV), torch.empty((3, 2), device=DEV)
    rows = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([-4, 10 ** 6, 20], [3, 2 ** 31 - 1, -7])]
    win, W = window("off", d)
    atf.atf_decode_ragged_q8(q.to(DEV), kc, ks, vc, vs, o, lse, *rows, T, win, workspace(3, 2, 1, T, d))
    torch.cuda.synchronize()
    lens, pos = [0, T, 20], [3, 2 ** 31 - 3, 0]
    judge(o, lse, [R.decode(R.f64(q[b]), value(k, ke)[b, :, : lens[b]], value(v, ve)[b, :, : lens[b]], pos[b], W, d ** -0.5)
                   for b in range(3)])


def test_decode_scale_and_large_scores():
    """A given softmax scale, and scores that leave one key with all the weight."""
    import paper_2608_02947_amd as atf
    note("decode scale")
    d, T = 128, 300
    k, ke, v, ve = q8_caches(1, 2, T, d, 6)
    ke = ke + 3
    (kc, ks), (vc, vs) = to_layout(k, ke, False), to_layout(v, ve, True)
    q = randn((1, 6, d), 3)
    win, W = window("exact", d)
    for scale in (0.01, 1.5):
        o, lse = torch.empty_like(q, device=DEV), torch.empty((1, 6), device=DEV)
        atf.atf_decode_q8(q.to(DEV), kc, ks, vc, vs, o, lse, T, win, workspace(1, 6, 2, T, d), softmax_scale=scale)
        torch.cuda.synchronize()
        judge(o, lse, [R.decode(R.f64(q[0]), value(k, ke)[0], value(v, ve)[0], T, W, float(np.float32(scale)))])


def test_decode_nan_rows():
    """A key or value that is not a number reaches the rows that attend it, and no other."""
    import paper_2608_02947_amd as atf
    note("decode nan")
    d = 64
    win, _ = window("off", d)
    for T, at in ((1, 0), (40, 39), (700, 3)):
        k, ke, v, ve = q8_caches(3, 1, T, d, 9)
        k[1, 0, at, 5] = np.nan
        v[2, 0, at, 6] = np.nan
        (kc, ks), (vc, vs) = to_layout(k, ke, False), to_layout(v, ve, True)
        q = randn((3, 4, d), 3)
        o, lse = torch.empty_like(q, device=DEV), torch.empty((3, 4), device=DEV)
        atf.atf_decode_q8(q.to(DEV), kc, ks, vc, vs, o, lse, T, win, workspace(3, 4, 1, T, d))
        torch.cuda.synchronize()
        nan = torch.isnan(o).cpu()
        assert not nan[0].any() and nan[1].all() and nan[2, :, 6].all() and not nan[2, :, :6].any()
        assert torch.isnan(lse[1]).all() and torch.isfinite(lse[[0, 2]]).all()


def test_decodes_at_once_and_one_after_another():
    """Two decodes at once on two streams, each with a workspace of its own, and decodes of
    different sizes one after another in one workspace: the bits of each alone."""
    import paper_2608_02947_amd as atf
    note("decodes at once")
    d, T = 128, 3000
    win, _ = window("exact", d)
    calls, spaces, outs = [], [], []
    for i, (B, h_q, h_kv, ragged) in enumerate([(2, 8, 2, False), (3, 20, 1, True), (1, 4, 4, True)]):
        k, ke, v, ve = q8_caches(6, h_kv, 544, d, 70 + i)
        (kc, ks), (vc, vs) = to_layout(k, ke, False), to_layout(v, ve, True)
        if ragged:  # 544-token pages, the first of them in every row
            table = torch.tensor([[0, 1 + b, 2, 5, 3, 4] for b in range(B)], dtype=torch.int32, device=DEV)
            rows = [torch.tensor([T - 700 * b - x for b in range(B)], dtype=torch.int32, device=DEV) for x in (0, 1)]
        else:
            k, ke, v, ve = q8_caches(B, h_kv, T, d, 80 + i)
            (kc, ks), (vc, vs) = to_layout(k, ke, False), to_layout(v, ve, True)
        q = randn((B, h_q, d), 60 + i).to(DEV)

        def call(out, ws, stream=None, q=q, c=(kc, ks, vc, vs), more=(table, *rows) if ragged else None):
            o, lse = out
            if more is None:
                atf.atf_decode_q8(q, *c, o, lse, T - 1, win, ws, stream=stream)
            else:
                atf.atf_decode_paged_q8(q, *c, o, lse, *more, T, win, ws, stream=stream)
        calls.append(call)
        spaces.append(workspace(B, h_q, h_kv, T, d))
        outs.append((torch.zeros_like(q), torch.zeros((B, h_q), device=DEV)))

    def run(spaces, streams=(None,) * 3):
        for o, lse in outs:
            o.zero_(), lse.zero_()
        torch.cuda.synchronize()
        for call, out, ws, s in zip(calls, outs, spaces, streams):
            call(out, ws, s)
        torch.cuda.synchronize()
        return [x.clone() for out in outs for x in out]

    alone = run(spaces)
    streams = [torch.cuda.Stream() for _ in calls]
    for how in [(spaces, streams)] * 3 + [([max(spaces, key=torch.Tensor.numel)] * 3,)]:
        assert all(torch.equal(a, b) for a, b in zip(alone, run(*how)))


def test_offsets_past_32_bits():
    """Pages at the end of pools of 4.5 GiB, appended to, read back and decoded over: the bytes and
    bits of the same pages in small pools; and the end of one cache of 2^26 tokens and more."""
    import paper_2608_02947_amd as atf
    note("pools past 4 GiB")
    d, h_q, h_kv, pt, B, n = 128, 4, 2, 64, 2, 150
    win, _ = window("exact", d)
    small, large = 8, 9 * 2 ** 15
    q, k, v = (randn((B, n, h, d), 31 + h).to(DEV) for h in (h_q, h_kv, h_kv))
    got = []
    for pages in (small, large):
        table = torch.tensor([[pages - 1, pages - 4, pages - 2], [pages - 6, pages - 3, pages - 5]], dtype=torch.int32, device=DEV)
        kc = torch.zeros(atf.kpages_shape(pages, pt, h_kv, d), dtype=torch.uint8, device=DEV).view(E4)
        vc = torch.zeros(atf.vpages_shape(pages, pt, h_kv, d), dtype=torch.uint8, device=DEV).view(E4)
        ks, vs = (torch.zeros(atf.qscale_shape(pages, pt, h_kv), dtype=torch.uint8, device=DEV).view(E8) for _ in "kv")
        qo = torch.empty_like(q)
        atf.atf_cache_append_paged_q8(q, k, v, qo, kc, ks, vc, vs, table, 0, win)
        kb = torch.zeros(atf.kcache_shape(B, n, h_kv, d), dtype=BF, device=DEV)
        vb = torch.zeros(atf.vcache_shape(B, n, h_kv, d), dtype=BF, device=DEV)
        atf.atf_cache_read_paged_q8(kc, ks, vc, vs, table, kb, vb, n)
        rows = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([n, n - 1], [n - 1, n - 2])]
        o, lse = torch.empty((B, h_q, d), dtype=BF, device=DEV), torch.empty((B, h_q), device=DEV)
        atf.atf_decode_paged_q8(qo[:, -1].contiguous(), kc, ks, vc, vs, o, lse, table, *rows, n, win, workspace(B, h_q, h_kv, n, d))
        torch.cuda.synchronize()
        got.append([x[-8:].view(torch.uint8).cpu() for x in (kc, vc, ks, vs)] + [x.cpu() for x in (qo, kb, vb, o, lse)])
        assert not kc[0].view(torch.uint8).any()  # a page of no row
    assert all(torch.equal(a, b) for a, b in zip(*got))
    del kc, vc, ks, vs

    note("cache past 4 GiB")
    d, cap, n, pos0 = 64, 2 ** 26 + 1000, 101, 2 ** 26 + 77
    win, W = window("exact", d)
    k, v = (randn((1, n, 1, d), 41 + i).to(DEV) for i in range(2))
    kc = torch.zeros(atf.kcache_shape(1, cap, 1, d), dtype=torch.uint8, device=DEV).view(E4)
    vc = torch.zeros(atf.vcache_shape(1, cap, 1, d), dtype=torch.uint8, device=DEV).view(E4)
    ks, vs = (torch.full(atf.qscale_shape(1, cap, 1), 127, dtype=torch.uint8, device=DEV).view(E8) for _ in "kv")
    atf.atf_cache_append_q8(None, k, v, None, kc, ks, vc, vs, pos0, win)
    kb = torch.zeros(atf.kcache_shape(1, cap, 1, d), dtype=BF, device=DEV)
    vb = torch.zeros(atf.vcache_shape(1, cap, 1, d), dtype=BF, device=DEV)
    atf.atf_cache_read_q8(kc, ks, vc, vs, kb, vb, n, pos0)
    torch.cuda.synchronize()
    got = R.v_tokens(R.f64(vb[:, :, pos0 // 16 : (pos0 + n) // 16 + 1]), True)[0, 0, pos0 % 16 : pos0 % 16 + n]
    assert np.array_equal(got, value(*R.quantise(R.f64(v[0, :, 0]))))
    pos = pos0 + np.arange(n, dtype=np.int64)
    want, err = R.norm_rotate(R.f64(k[0]), None, 0.0, pos, R.theta(d, 1e4))
    got = R.k_tokens(R.f64(kb[:, :, :, pos0 : pos0 + n]))[0, 0]
    power = 2.0 ** (ks.view(torch.uint8)[0, 0, pos0 : pos0 + n].cpu().numpy().astype(np.float64) - 127)[:, None]
    assert (np.abs(got - want[:, 0]) <= np.maximum(R.E4M3_HALF * np.abs(want[:, 0]), R.E4M3_TINY * power) * (1 + 2.0 ** -10) + err[:, 0]).all()
    # nothing else is written
    assert not kc[0, 0, :, :pos0].view(torch.uint8).any()
    assert all((x.view(torch.uint8)[0, 0, :pos0] == 127).all() for x in (ks, vs))
    # decode over all of it: pos0 keys of score 0 with values 0, then the new ones.  The zeros' weights
    # are of one size and sum to whole multiples of it, exact below 2^24; at most 2^11 such sums are
    # joined, each with a rounding
    q = randn((1, 3, d), 43)
    o, lse = torch.empty((1, 3, d), dtype=BF, device=DEV), torch.empty((1, 3), device=DEV)
    atf.atf_decode_q8(q.to(DEV), kc, ks, vc, vs, o, lse, pos0 + n - 1, win, workspace(1, 3, 1, pos0 + n, d), n_k=pos0 + n)
    torch.cuda.synchronize()
    wo, wl, oe, le = R.decode(R.f64(q[0]), got[None], value(*R.quantise(R.f64(v[0, :, 0])))[None], n - 1, W, d ** -0.5)
    share = np.exp(wl) / (pos0 + np.exp(wl))
    off = 2.0 ** -13  # of the sum, relative
    assert (np.abs(R.f64(o[0]) - wo * share[:, None]) <= (oe + off * np.abs(wo)) * share[:, None]).all()
    assert (np.abs(lse[0].cpu().numpy() - np.log(pos0 + np.exp(wl))) <= le + off + 2.0 ** -19).all()


def test_binding_refuses_views_and_types():
    import paper_2608_02947_amd as atf
    note("views and types")
    d = 64
    win, _ = window("exact", d)
    c = Case(d, 4, 2, 2, 3, True, [0, 5], 40)
    q, k = c.q.to(DEV), c.k.to(DEV)
    good = [q, k, k.clone(), q.clone(), c.kc, c.ks, c.vc, c.vs]
    atf.atf_cache_append_q8(*good, 0, win)
    atf.atf_cache_append_q8(*[x[:, :0] for x in good[:4]], *good[4:], 40, win)  # no tokens: nothing
    for i, bad in ((0, q.transpose(0, 1).contiguous().transpose(0, 1)), (1, k.float()), (3, q.to(torch.float16)),
                   (4, c.kc.view(torch.uint8)), (5, c.ks.view(torch.uint8)), (6, c.vc.cpu())):
        with pytest.raises((TypeError, ValueError)):
            atf.atf_cache_append_q8(*[bad if j == i else x for j, x in enumerate(good)], 0, win)
    with pytest.raises((TypeError, ValueError)):
        atf.atf_cache_append_q8(*good, 0, win, q_weight=torch.ones(d, dtype=BF, device=DEV))
    with pytest.raises((TypeError, ValueError)):
        atf.atf_cache_append_q8(*good, 0, win, pos_rows=torch.zeros(2, dtype=torch.int64, device=DEV))
    torch.cuda.synchronize()


# ---- together, as a server uses them

def test_prompt_then_steps_captured():
    """A prompt enters an 8-bit paged cache in chunks, the second chunk's prefill reads the cache
    back, then rows of different lengths decode step by step, in a captured graph that is
    replayed for every step; every step against 64 bits over what the cache holds."""
    import paper_2608_02947_amd as atf
    note("together")
    d, h_q, h_kv, B, pt, width, steps = 128, 8, 2, 3, 32, 6, 5
    win, W = window("exact", d)
    qw, kw = (1 + 0.2 * randn((d,), s).float().to(DEV) for s in (1, 2))
    pool = B * width
    table = torch.randperm(pool, generator=torch.Generator().manual_seed(3)).view(B, width).to(torch.int32).to(DEV)
    kc = torch.zeros(atf.kpages_shape(pool, pt, h_kv, d), dtype=torch.uint8, device=DEV).view(E4)
    vc = torch.zeros(atf.vpages_shape(pool, pt, h_kv, d), dtype=torch.uint8, device=DEV).view(E4)
    ks, vs = (torch.zeros(atf.qscale_shape(pool, pt, h_kv), dtype=torch.uint8, device=DEV).view(E8) for _ in "kv")
    pages = (kc, ks, vc, vs)
    cap = pt * width
    kb = torch.zeros(atf.kcache_shape(B, cap, h_kv, d), dtype=BF, device=DEV)
    vb = torch.zeros(atf.vcache_shape(B, cap, h_kv, d), dtype=BF, device=DEV)

    def held(n):
        """Keys and values of all rows as tokens, from the cache's own bytes."""
        out = []
        for c, s, tok in ((kc, ks, R.k_tokens), (vc, vs, lambda x: R.v_tokens(x, False))):
            x = tok(R.f64(c)) * np.exp2(s.cpu().view(torch.uint8).numpy().astype(np.float64) - 127)[..., None]
            out.append(np.stack([R.paged(x, table.cpu().numpy(), b, pt, n) for b in range(B)]))
        return out

    # the prompt in two chunks
    lens = [61, 90, 40]
    done = 0
    for n in (33, 57):
        q, kn, vn = (randn((B, n, h, d), 50 + n + h).to(DEV) for h in (h_q, h_kv, h_kv))
        qo = torch.empty_like(q)
        atf.atf_cache_append_paged_q8(q, kn, vn, qo, *pages, table, done, win, qw, kw, EPS)
        atf.atf_cache_read_paged_q8(*pages, table, kb, vb, n, done)
        o, lse = torch.empty_like(q), torch.empty((B, h_q, n), device=DEV)
        atf.atf_prefill(qo, kb, vb, o, lse, done, win, n_k=done + n)
        torch.cuda.synchronize()
        done += n
        hk, hv = held(done)
        for b in range(B):
            for t in (0, n // 2, n - 1):
                wo, wl, oe, le = R.decode(R.f64(qo[b, t]), hk[b], hv[b], done - n + t, W, d ** -0.5)
                # the prefill's probabilities are rounded to bf16 once: 2^-8 of sum p |v|
                size = R.decode(R.f64(qo[b, t]), hk[b], np.abs(hv[b]), done - n + t, W, d ** -0.5)[0]
                assert (np.abs(R.f64(o[b, t]) - wo) <= oe + 2.0 ** -8 * size).all()
                assert (np.abs(lse[b, :, t].cpu().numpy() - wl) <= le + 2.0 ** -8).all()

    # steps: row b goes on from its own length, one slot idle in the second step
    pos = torch.tensor(lens, dtype=torch.int32, device=DEV)
    n_rows = pos + 1
    q, kn, vn = (torch.zeros((B, 1, h, d), dtype=BF, device=DEV) for h in (h_q, h_kv, h_kv))
    qo, o, lse = torch.zeros_like(q), torch.zeros((B, h_q, d), dtype=BF, device=DEV), torch.zeros((B, h_q), device=DEV)
    ws = workspace(B, h_q, h_kv, cap, d)

    def step():
        atf.atf_cache_append_paged_q8(q, kn, vn, qo, *pages, table, 0, win, qw, kw, EPS, pos_rows=pos)
        atf.atf_decode_paged_q8(qo.view(B, h_q, d), *pages, o, lse, table, n_rows, pos, cap, win, ws)

    graph = None
    for i in range(steps):
        for x, h in ((q, h_q), (kn, h_kv), (vn, h_kv)):
            x.copy_(randn((B, 1, h, d), 900 + 10 * i + h).to(DEV))
        now = [n + i for n in lens]
        idle = i == 1
        pos.copy_(torch.tensor(now if not idle else [now[0], -1, now[2]], dtype=torch.int32))
        n_rows.copy_(torch.tensor([n + 1 for n in now] if not idle else [now[0] + 1, 0, now[2] + 1], dtype=torch.int32))
        if graph is None:
            step()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone(), lse.clone()
        hk, hv = held(max(now) + 1)
        want = []
        for b in range(B):
            n = 0 if idle and b == 1 else now[b] + 1
            want.append(R.decode(R.f64(qo[b, 0]), hk[b, :, :n], hv[b, :, :n], now[b], W, d ** -0.5))
        judge(*got, want)
        step()  # eager between the replays: the same bits
        torch.cuda.synchronize()
        assert torch.equal(got[0], o) and torch.equal(got[1], lse)
        if idle:
            lens = [lens[0], lens[1] - 1, lens[2]]  # the idle row takes its token next time
