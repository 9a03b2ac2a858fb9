"""Selection of blocks and attention over them in workspaces of other sizes than the call's own."""
import numpy as np
import pytest
import torch

import test_gpu_blocks as B
from parity import note

pytestmark = B.pytestmark


class Room:
    """A workspace of `size` bytes inside a larger buffer whose other bytes are looked at."""

    def __init__(self, size):
        self.all = torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device=B.DEV)
        self.part, self.size = self.all[:size], size

    def check(self):
        assert bool((self.all[self.size:] == 0x5A).all())


@pytest.mark.parametrize("d,h_q,h_kv", [(128, 32, 4), (64, 40, 1)])
def test_attend_in_the_workspace_of_another_step(monkeypatch, d, h_q, h_kv):
    """A workspace made for a prompt's tokens serves single ones, and any size from 256 bytes on serves any call,
    without a byte written past it; the whole plan's size and the one that serves every call give the same bits."""
    import paper_2608_02947_amd as atf
    note(f"attend workspaces {d} {h_q}/{h_kv}")
    pt, bt, top = 64, 64, 64
    win, W = B.windows(d, "exact")
    for queries in ((1,), (3, 1)):
        tok = B.Tokens([4500, 3000][:len(queries)], queries, pt, 7)
        q = torch.randn((tok.T, h_q, d), generator=torch.Generator().manual_seed(7)).to(B.BF)
        kp, vp = B.random_pools(tok.P, pt, h_kv, d, 7)
        lists = B.random_lists(tok, h_kv, top, bt, 7, wild=False)
        size = lambda n: atf.atf_attend_workspace_bytes(n, h_q, h_kv, top, bt, d)
        own, prompt, every = size(tok.T), size(900), 256 * (h_q // h_kv) * (4 * d + 8) + 768
        assert prompt < own <= every
        got = {}
        attended = B.attended
        for bytes_ in (prompt, own // 5, own // 2, own - 256, own, every):
            room = Room(bytes_ // 16 * 16)
            monkeypatch.setattr(B, "attended", lambda *a: attended(*a, ws=room.part))
            got[bytes_] = B.check_attend(tok, q, kp, vp, lists, bt, win, W)
            room.check()
        monkeypatch.setattr(B, "attended", attended)
        assert all(np.array_equal(x, y) for x, y in zip(got[own], got[every]))


@pytest.mark.parametrize("what", ["random", "zeros"])
def test_select_in_the_workspace_of_longer_rows(what):
    """A workspace made for rows of 6 M keys serves rows of 1 M, whose tokens fill more of it; nothing is written
    past it."""
    import paper_2608_02947_amd as atf
    note(f"select workspace of longer rows {what}")
    d, h, pt, bt, top = 64, 64, 32, 32, 3
    win, W = B.windows(d, "exact")
    tok = B.Tokens([200, 333], [40, 22], pt, 3)
    assert tok.T == 64
    most = 1 << 20
    tok.table = np.pad(tok.table, ((0, 0), (0, most // pt - tok.table.shape[1])), constant_values=-1)
    q = torch.randn((tok.T, h, d), generator=torch.Generator().manual_seed(1)).to(B.BF)
    b = B.random_bounds(tok.P, pt, bt, h, d, 2)
    if what == "zeros":
        b.zero_()
    room = Room(atf.atf_select_workspace_bytes(tok.T, h, h, 6 * most, bt, d))
    got = B.selected(tok, q.to(B.DEV), b.to(B.DEV), bt, win, top, 1, 1, max_n_k=most, ws=room.part)
    room.check()
    want = np.full(got.shape, 777)
    B.R.select(q.double().numpy(), b.double().numpy(), tok.table, tok.rows, tok.pos, tok.lens, most, W, pt, bt, top, 1, 1, want)
    assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("T,most", [(1, 1), (1, 70000), (70, 3000), (232, 1 << 22)])
def test_select_writes_no_further_than_its_size(T, most):
    import paper_2608_02947_amd as atf
    note(f"select workspace end {T} {most}")
    d, h_q, h_kv, pt, bt = 64, 6, 2, 32, 32
    win, _ = B.windows(d, "exact")
    n = min(most, 3000)
    tok = B.Tokens([n, n], [T - T // 2, T // 2], pt, 3, pad=0)
    tok.pos = np.maximum(tok.pos, 0)
    tok.table = np.pad(tok.table, ((0, 0), (0, max(0, -(-most // pt) - tok.table.shape[1]))), constant_values=-1)
    q = torch.randn((T, h_q, d), generator=torch.Generator().manual_seed(1)).to(B.BF).to(B.DEV)
    for b in (B.random_bounds(tok.P, pt, bt, h_kv, d, 2), torch.zeros(atf.bounds_shape(tok.P, pt, bt, h_kv, d), dtype=B.BF)):
        room = Room(atf.atf_select_workspace_bytes(T, h_q, h_kv, most, bt, d))
        out = B.selected(tok, q, b.to(B.DEV), bt, win, 5, 1, 1, max_n_k=most, ws=room.part)
        room.check()
        assert torch.equal(out, B.selected(tok, q, b.to(B.DEV), bt, win, 5, 1, 1, max_n_k=most))
