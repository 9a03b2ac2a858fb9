"""Decode over 8-bit caches whose keys hold numbers that are none, in pairs inside and outside the
window, on the GPU, against the plain 64-bit form of q8ref.py."""
import numpy as np
import pytest
import torch

import q8ref as R
import test_gpu_q8 as G
from conftest import gpu_available
from parity import note

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]


@pytest.mark.parametrize("half", [0, 1], ids=["first", "second"])
@pytest.mark.parametrize("d,h_q,T,r,pages", [
    (64, 3, 500, 3, 0), (64, 3, 4000, 19, 0), (64, 20, 500, 9, 32), (64, 5, 3000, 12, 96),
    (128, 2, 500, 6, 0), (128, 4, 6000, 37, 0), (128, 20, 500, 20, 0), (128, 17, 5000, 36, 64)])
def test_nan_outside_the_window_does_not_count(d, h_q, T, r, pages, half):
    """One key of each row has a NaN in pair r, whose window ends at W: at distances up to W the row
    is NaN, past it (where other pairs of its chunk are kept, or none) it is as if the number were 0."""
    import paper_2608_02947_amd as atf
    note(f"decode nan window {d} {h_q} {T} {r} {pages} {half}")
    win, W = G.window("exact", d)
    w = int(W[r])
    far = [0, w - 1, w, w + 1, w + 16, w + 65, int(W[r | 7]), int(W[r | 7]) + 1, T - 1]
    far = [z for z in far if z < T]
    assert w + 65 < T
    B = len(far)
    k, ke, v, ve = G.q8_caches(B, 1, T, d, 300 + r)
    for b, z in enumerate(far):
        k[b, 0, T - 1 - z, r + half * d // 2] = np.nan
    q = G.randn((B, h_q, d), 5)
    o, lse = torch.empty_like(q, device=G.DEV), torch.empty((B, h_q), device=G.DEV)
    ws = G.workspace(B, h_q, 1, T, d)
    if pages:
        width = -(-T // pages)
        table = torch.randperm(B * width, generator=torch.Generator().manual_seed(r)).view(B, width).to(torch.int32)
        put = lambda x: G._into_pages(x, table, B * width, pages)
        (kc, ks), (vc, vs) = G.to_layout(put(k), put(ke), False), G.to_layout(put(v), put(ve), True)
        rows = [torch.full((B,), x, dtype=torch.int32, device=G.DEV) for x in (T, T - 1)]
        atf.atf_decode_paged_q8(q.to(G.DEV), kc, ks, vc, vs, o, lse, table.to(G.DEV), *rows, T, win, ws)
    else:
        (kc, ks), (vc, vs) = G.to_layout(k, ke, False), G.to_layout(v, ve, True)
        atf.atf_decode_q8(q.to(G.DEV), kc, ks, vc, vs, o, lse, T - 1, win, ws)
    torch.cuda.synchronize()
    kept = [b for b, z in enumerate(far) if z <= w]
    out = [b for b, z in enumerate(far) if z > w]
    assert torch.isnan(o[kept]).all() and torch.isnan(lse[kept]).all()
    assert not torch.isnan(o[out]).any() and not torch.isnan(lse[out]).any()
    want = [R.decode(R.f64(q[b]), G.value(k, ke)[b], G.value(v, ve)[b], T - 1, W, d ** -0.5) for b in out]
    G.judge(o[out], lse[out], want)
