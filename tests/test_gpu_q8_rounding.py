"""How exactly the normed and 8-bit appends turn and round, on the GPU, against forms in 64 bits and
more."""
import numpy as np
import pytest
import torch

import q8ref as R
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
