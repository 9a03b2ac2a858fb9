"""How exactly the normed and 8-bit appends turn and round, on the GPU, against forms in 64 bits and
more."""
import numpy as np
import pytest
import torch

import q8ref as R
import q8rounding as Q
import test_gpu_q8 as G
from conftest import gpu_available
from parity import note

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]


@pytest.mark.parametrize("d,base,first,n", [(128, 1e7, 1, 200), (128, 1e6, 100, 500), (64, 1e4, 1, 1500),
                                            (64, 1e4, 99990, 300), (128, 5e5, 2 ** 20 - 100, 400)])
def test_sines_next_to_nothing(d, base, first, n):
    """Queries (0, 1) and (1, 0) in every pair come out as the angle's own -sin, cos and cos, sin, the
    small ones as exactly as the large: a bf16 rounding (half a step) and 2 ulps of fp32, beside the
    angle's error, at most 2 pi pos 2^-64 (its fraction of a turn is cut there) and as much again for
    the reference's product (64 bits of fraction, below 2^20 radians a turn's 2^-42)."""
    import paper_2608_02947_amd as atf
    note(f"sines {d} {base} {first} {n}")
    theta = R.theta(d, base)
    q = torch.zeros(1, n, 2, d, dtype=torch.bfloat16)
    q[:, :, 0, d // 2:] = 1.0
    q[:, :, 1, : d // 2] = 1.0
    k = torch.zeros(1, n, 1, d, dtype=torch.bfloat16, device=G.DEV)
    out = torch.zeros_like(q, device=G.DEV)
    kc = torch.zeros(atf.kcache_shape(1, n, 1, d), dtype=torch.bfloat16, device=G.DEV)
    vc = torch.zeros(atf.vcache_shape(1, n, 1, d), dtype=torch.bfloat16, device=G.DEV)
    atf.atf_cache_append_normed(q.to(G.DEV), k, k.clone(), out, kc, vc, 0, atf.Window(d, base, 2.0),
                                pos_rows=torch.tensor([first], dtype=torch.int32, device=G.DEV), rope_inv_freq=theta)
    torch.cuda.synchronize()
    pos = first + np.arange(n)
    a = pos.astype(np.longdouble)[:, None] * theta.astype(np.longdouble)
    cos, sin = np.cos(a).astype(np.float64), np.sin(a).astype(np.float64)
    got = R.f64(out[0])
    held = 2 * 2 * np.pi * 2.0 ** -64 * pos[:, None] + 2.0 ** -63 * a.astype(np.float64)
    half = d // 2
    for h, (lo, hi) in enumerate(((-sin, cos), (cos, sin))):
        for x, want in ((got[:, h, :half], lo), (got[:, h, half:], hi)):
            assert (np.abs(x - want) <= (R.BF16_HALF + 2.0 ** -22) * np.abs(want) + held).all()


def _append(k, pos0, theta, weight=None, pos_rows=None):
    """Keys [B, n, h, d] into an 8-bit cache at positions pos0 .. (or pos_rows): numbers as they stand in
    the cache [B, h, d/16, n, 16] (uint8) and powers [B, h, n] (fp64); positions as in the cache."""
    import paper_2608_02947_amd as atf
    B, n, h, d = k.shape
    cap = n if pos_rows is None else int(pos_rows.max()) + n
    new = lambda shape, dt: torch.full(shape, G.SENTINEL, dtype=torch.uint8, device=G.DEV).view(dt)
    if pos_rows is None:
        cap += pos0
    kc, vc = new(atf.kcache_shape(B, cap, h, d), G.E4), new(atf.vcache_shape(B, cap, h, d), G.E4)
    ks, vs = (new(atf.qscale_shape(B, cap, h), G.E8) for _ in "kv")
    atf.atf_cache_append_q8(None, k, torch.ones_like(k), None, kc, ks, vc, vs, pos0, atf.Window(d, 1e4, 2.0),
                            k_weight=weight, eps=G.EPS, pos_rows=pos_rows, rope_inv_freq=theta)
    torch.cuda.synchronize()
    return kc.view(torch.uint8), ks.view(torch.uint8), vc.view(torch.uint8), vs.view(torch.uint8)


def _rows(kc, ks, pos0, n):
    """Numbers [n, d] and powers [n] (fp64) of one row of one head."""
    d = 16 * kc.shape[2]
    x = kc[0, 0, :, pos0:pos0 + n].contiguous().view(G.E4).double()  # [d/16, n, 16]
    out = torch.empty((n, d), dtype=torch.float64, device=kc.device)
    out[:, torch.from_numpy(R.dims(d)).reshape(-1).to(kc.device)] = x.transpose(0, 1).reshape(n, d)
    return out, torch.exp2(ks[0, 0, pos0:pos0 + n].double() - 127)


@pytest.mark.parametrize("normed", [False, True], ids=["plain", "normed"])
@pytest.mark.parametrize("d,n,pos0", [(64, 2 ** 23, 5), (128, 2 ** 22, 1000)])
def test_keys_round_as_the_formulas(d, n, pos0, normed):
    """537 million numbers of random keys: each other number than the formula's is one whose border is
    as near as fp32's error, and of those that are formed in 64 bits near a border at most a quarter
    of plain fp32's are left (q8rounding.py)."""
    note(f"keys round {d} {n} {normed}")
    g = torch.Generator(device=G.DEV).manual_seed(d + normed)
    k = (torch.randn((1, n, 1, d), generator=g, device=G.DEV) * 2).to(torch.bfloat16)
    w = 1 + 0.3 * torch.randn(d, generator=g, device=G.DEV) if normed else None
    theta = R.theta(d, 1e4)
    kc, ks, _, _ = _append(k, pos0, theta, w)
    bound = Q.NORMED if normed else Q.PLAIN
    rows = left = plain_rows = plain = 0
    part = 2 ** 17
    for i in range(0, n, part):
        a = torch.arange(pos0 + i, pos0 + i + part, dtype=torch.float64, device=G.DEV)[:, None] * torch.from_numpy(theta).to(G.DEV)
        cos, sin = a.cos(), a.sin()
        x = k[0, i:i + part, 0]
        want, size = Q.turned64(x, w, G.EPS, cos, sin)
        got = Q.judged(*_rows(kc, ks, pos0 + i, part), want, size, bound)
        rows, left = rows + got[0], left + got[1]
        got = Q.judged(*Q.quantised32(Q.turned32(x, w, G.EPS, cos, sin)), want, size, bound)
        plain_rows, plain = plain_rows + got[0], plain + got[1]
    note(f"  {rows} rows with another number or power, plain fp32 {plain_rows}; {left} numbers left, plain fp32 {plain}")
    assert plain >= 16 and left <= plain // 4


def test_powers_next_to_the_largest_number():
    """Keys of one pair that turn to within half an ulp of 448 times a power of two: the power, and the
    number beside it, are the formula's."""
    note("powers at borders")
    d = 64
    theta = np.ones(32)
    found = []
    for seed in range(64):
        g = torch.Generator(device=G.DEV).manual_seed(seed)
        # (the second a tenth of the first; turned, so that the border is not met exactly)
        xy = torch.randn((2, 2 ** 24), generator=g, device=G.DEV)
        xy[1] *= 0.1
        xy = xy.to(torch.bfloat16)
        pos = torch.randint(1, 4000, (2 ** 24,), generator=g, device=G.DEV)
        a = pos.double()
        x, y = xy.double()
        z = (x * a.cos() - y * a.sin()).abs()
        m, e = torch.frexp(z)
        off = (m - 0.875) * 2.0 ** 24  # in ulps
        small = (x.abs() + y.abs() <= 1.25 * z) & (z >= (y * a.cos() + x * a.sin()).abs()) & (z > 2.0 ** -20)
        at = ((off.abs() <= 0.5) & small).nonzero()[:, 0]
        found.append((xy[:, at], pos[at]))
    xy, pos = torch.cat([f[0] for f in found], 1), torch.cat([f[1] for f in found])
    n = pos.numel()
    note(f"  {n} keys")
    assert n >= 16
    k = torch.zeros((n, 1, 1, d), dtype=torch.bfloat16, device=G.DEV)
    k[:, 0, 0, 7], k[:, 0, 0, 7 + 32] = xy[0], xy[1]
    kc, ks, _, _ = _append(k, 0, theta, None, pos.to(torch.int32))
    b = torch.arange(n, device=G.DEV)
    got = kc[b, 0, :, pos].contiguous().view(G.E4).double()  # [n, d/16, 16]
    number = torch.empty((n, d), dtype=torch.float64, device=G.DEV)
    number[:, torch.from_numpy(R.dims(d)).reshape(-1).to(G.DEV)] = got.reshape(n, d)
    scale = torch.exp2(ks[b, 0, pos].double() - 127)
    a = pos.double()[:, None].expand(n, 32)
    want, size = Q.turned64(k[:, 0, 0], None, 0.0, a.cos(), a.sin())
    rows, _ = Q.judged(number, scale, want, size, Q.PLAIN)
    plain, _ = Q.judged(*Q.quantised32(Q.turned32(k[:, 0, 0], None, 0.0, a.cos(), a.sin())), want, size, Q.PLAIN)
    note(f"  {rows} rows left, plain fp32 {plain}")
    assert plain >= 4 and rows <= plain // 4


@pytest.mark.parametrize("normed", [False, True], ids=["plain", "normed"])
def test_heads_of_one_wave_and_of_many(normed):
    """128 KV heads in a call whose waves take 64 of them each: the bytes that four heads at a time
    give, whose waves take one or two."""
    note(f"heads of a wave {normed}")
    d, h, n, pos0 = 64, 128, 13400, 3
    g = torch.Generator(device=G.DEV).manual_seed(8)
    k = torch.randn((1, n, h, d), generator=g, device=G.DEV, dtype=torch.float32).to(torch.bfloat16)
    w = 1 + 0.3 * torch.randn(d, generator=g, device=G.DEV) if normed else None
    theta = R.theta(d, 1e4)
    every = _append(k, pos0, theta, w)
    for i in range(0, h, 4):
        four = _append(k[:, :, i:i + 4].contiguous(), pos0, theta, w)
        assert all(torch.equal(x[:, i:i + 4], y) for x, y in zip(every, four)), i
