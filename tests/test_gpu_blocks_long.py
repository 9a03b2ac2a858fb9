"""Selections of blocks in rows of thousands of blocks, of more heads and tokens than one pass or launch takes,
and of numbers that are none in blocks that are taken anyway; runs at once on two streams."""
import math

import numpy as np
import pytest
import torch

import blocksref as R
import test_gpu_blocks as B
from parity import note

pytestmark = B.pytestmark


def scores(q, bnd, table_row, p, last, W, bt):
    """blocksref.scores of all blocks of a row at once, summed in long doubles: [h_kv, blocks]."""
    P, h_kv, per = bnd.shape[:3]
    h_q, d = q.shape
    n, G, half = last // bt + 1, h_q // h_kv, d // 2
    j = np.arange(n)
    x = bnd[np.clip(table_row[j // per], 0, P - 1), :, j % per]  # [n, h_kv, d/16, 2, 16]
    hi, lo = R.pair_bounds(x[:, :, :, 0]), R.pair_bounds(x[:, :, :, 1])  # [n, h_kv, 2, half]
    near, far = p - np.minimum(j * bt + bt - 1, last), p - j * bt
    qs = q.reshape(h_kv, G, 2, half)
    out = np.empty((h_kv, n))
    for g in range(h_kv):
        with np.errstate(invalid="ignore"):
            s = []
            for i in range(G):
                u = np.maximum(qs[g, i], 0) * hi[:, g] + np.minimum(qs[g, i], 0) * lo[:, g]
                u = u[:, 0] + u[:, 1]
                u = np.where((W < far[:, None]) & (u < 0), 0.0, u)
                s.append(np.where(W >= near[:, None], u, 0.0).astype(np.longdouble).sum(axis=1).astype(np.float64))
            s = np.array(s)
            out[g] = np.where(np.isnan(s).any(axis=0), np.nan, s.max(axis=0))
    return out


def chosen(tok, q, bnd, bt, W, top, first, last_blocks, max_n_k=None):
    """The lists of all tokens, 777 in rows of padding."""
    h_kv = bnd.shape[1]
    most = max_n_k or max(1, int(tok.lens.max()))
    out = np.full((tok.T, h_kv, top), 777)
    for t in range(tok.T):
        b = int(tok.rows[t])
        if not 0 <= b < len(tok.lens):
            continue
        last = min(min(max(int(tok.lens[b]), 0), most) - 1, int(tok.pos[t]))
        out[t] = -1
        if last < 0:
            continue
        s = scores(q[t], bnd, tok.table[b], int(tok.pos[t]), last, W, bt)
        n = s.shape[1]
        j = np.arange(n)
        forced = (j < first) | (j >= n - last_blocks)
        for g in range(h_kv):
            none = np.isnan(s[g])
            rank = np.lexsort((j, np.where(forced | none, 0.0, -s[g]), np.where(forced, 0, np.where(none, 1, 2))))
            take = np.sort(rank[:top])
            out[t, g, :len(take)] = take
    return out


def check(tok, q, bnd, bt, win, W, top, first, last, max_n_k=None):
    got = B.selected(tok, q.to(B.DEV), bnd.to(B.DEV), bt, win, top, first, last, max_n_k).cpu().numpy()
    want = chosen(tok, q.double().numpy(), bnd.double().numpy(), bt, W, top, first, last, max_n_k)
    assert np.array_equal(got, want), np.argwhere(got != want)[:5]


def test_plain_form_is_that_of_blocksref():
    note("plain selections")
    d, h_q, h_kv, pt, bt = 64, 6, 2, 64, 32
    for kind in ("exact", "sliding", "falling"):
        _, W = B.windows(d, kind)
        tok = B.Tokens([1500, 700], [2, 2], pt, 8)
        q = torch.randn((tok.T, h_q, d), generator=torch.Generator().manual_seed(3)).double().numpy()
        b = B.random_bounds(tok.P, pt, bt, h_kv, d, 7)
        b.view(-1)[::3001] = math.nan
        want = np.full((tok.T, h_kv, 5), 777)
        R.select(q, b.double().numpy(), tok.table, tok.rows, tok.pos, tok.lens, 1500, W, pt, bt, 5, 1, 1, want)
        assert np.array_equal(chosen(tok, q, b.double().numpy(), bt, W, 5, 1, 1), want)


# blocks of a row up to which the choice has 4, 16 (256 threads), 16 (1,024 threads) in a thread's registers, and more
EDGES = [1024, 1025, 4096, 4097, 9001, 16384, 16385, 20011]


@pytest.mark.parametrize("what", ["random", "equal", "ties", "NaN", "infinite", "few"])
@pytest.mark.parametrize("n", EDGES)
def test_select_among_thousands_of_blocks(n, what):
    """equal: more blocks at the border than are listed; ties: 60 of the same score far from each other, of which
    the first ones are taken; few: scores of few values, the border in one that hundreds have."""
    note(f"select {n} blocks {what}")
    d, h_q, h_kv, pt, bt = 64, 3, 1, 64, 32
    win, W = B.windows(d, "exact" if what == "random" else "off")
    tok = B.Tokens([n * bt - 3, n * bt // 2], [1, 1], pt, n)
    g = torch.Generator().manual_seed(n)
    q = torch.randn((tok.T, h_q, d), generator=g).to(B.BF)
    b = B.random_bounds(tok.P, pt, bt, h_kv, d, n)
    top, first, last = 70, 1, 2
    if what == "equal":
        b[:] = b[:1, :, :1]
    elif what == "ties":
        best = torch.tensor([40.0, -40.0]).view(2, 1).expand(2, 16)
        for j in np.linspace(5, n // 2 - 9, 60).astype(int):
            for row in range(2):  # (the same places in both rows)
                b[tok.table[row, j * bt // pt], :, j % (pt // bt)] = best
        top = 33
    elif what == "NaN":
        b.view(-1)[torch.randint(0, b.numel(), (n // 500 + 3,), generator=g)] = math.nan
    elif what == "infinite":
        b.view(-1)[torch.randint(0, b.numel(), (40,), generator=g)] = math.inf
    elif what == "few":
        b = torch.randint(0, 2, b.shape, generator=g).to(B.BF)
        b[..., 1:, :, :] = 0
        q = (torch.arange(d) < 3).to(B.BF).expand(tok.T, h_q, d).contiguous()
    check(tok, q, b, bt, win, W, top, first, last)


@pytest.mark.parametrize("n", [4500, 9000, 20000])
def test_select_the_longest_lists(n):
    note(f"select 4096 of {n} blocks")
    d, h_q, h_kv, pt, bt = 64, 3, 1, 64, 32
    win, W = B.windows(d, "exact")
    tok = B.Tokens([n * bt, n * bt - 40], [1, 1], pt, n)
    q = torch.randn((tok.T, h_q, d), generator=torch.Generator().manual_seed(n)).to(B.BF)
    check(tok, q, B.random_bounds(tok.P, pt, bt, h_kv, d, n), bt, win, W, 4096, 1, 1)


def test_select_one_of_a_million_keys():
    """2^20 keys in blocks of 64, and one block more, 28/4 heads of 128."""
    for n in (1 << 20, (1 << 20) + 1):
        note(f"select 1 M {n}")
        d, h_q, h_kv, pt, bt = 128, 28, 4, 64, 64
        win, W = B.windows(d, "exact")
        tok = B.Tokens([n], [1], pt, 1, pad=0)
        q = torch.randn((1, h_q, d), generator=torch.Generator().manual_seed(n)).to(B.BF)
        check(tok, q, B.random_bounds(tok.P, pt, bt, h_kv, d, 1), bt, win, W, 64, 1, 2)


# ---- more heads, more tokens

@pytest.mark.parametrize("kind", ["exact", "sliding"])
@pytest.mark.parametrize("d,h_q,h_kv", [(64, 71, 1), (128, 71, 1), (128, 130, 2), (64, 200, 1)])
def test_select_and_attend_with_more_than_64_heads_to_a_kv_head(d, h_q, h_kv, kind):
    note(f"select and attend {d} {h_q}/{h_kv} {kind}")
    pt, bt = 64, 32
    win, W = B.windows(d, kind)
    tok = B.Tokens([900, 70], [3, 1], pt, 4)
    q = torch.randn((tok.T, h_q, d), generator=torch.Generator().manual_seed(d)).to(B.BF)
    check(tok, q, B.random_bounds(tok.P, pt, bt, h_kv, d, 5), bt, win, W, 6, 1, 1)
    kp, vp = B.random_pools(tok.P, pt, h_kv, d, 6)
    B.check_attend(tok, q, kp, vp, B.random_lists(tok, h_kv, 6, bt, 1), bt, win, W)


@pytest.mark.parametrize("group", [1, 3])
def test_select_more_tokens_than_a_launch_takes(group):
    """65,535 (token, KV head)s a launch: 4,095 tokens of 16 KV heads, of which 5 share a product's columns with 3
    heads a KV head, 16 with one."""
    note(f"select 4200 tokens, group {group}")
    d, h_kv, pt, bt = 64, 16, 32, 32
    win, W = B.windows(d, "exact")
    tok = B.Tokens([260, 180, 4000], [100, 100, 4000], pt, 6)
    tok.pos[200:4200] %= 230  # (many tokens of few places; not in order)
    q = torch.randn((tok.T, group * h_kv, d), generator=torch.Generator().manual_seed(2)).to(B.BF)
    check(tok, q, B.random_bounds(tok.P, pt, bt, h_kv, d, 3), bt, win, W, 3, 1, 1, max_n_k=4000)


# ---- numbers that are none

@pytest.mark.parametrize("x", [math.inf, -math.inf, math.nan, 1e38])
@pytest.mark.parametrize("queries", [(1, 1), (140, 60)])
def test_select_whatever_the_blocks_taken_anyway_hold(x, queries):
    """The first and the last blocks are taken without a look at their bounds: the same choice whatever these are."""
    note(f"select forced {x} {queries}")
    d, h, pt, bt = 64, 16, 32, 32
    win, W = B.windows(d, "exact")
    tok = B.Tokens([3000, 640], queries, pt, 9)
    q = torch.randn((tok.T, h, d), generator=torch.Generator().manual_seed(9)).to(B.BF)
    b = B.random_bounds(tok.P, pt, bt, h, d, 9)
    b[tok.table[:, 0]] = x
    b[tok.table[0, 2999 // pt], :, :, 1, 0] = x
    check(tok, q, b, bt, win, W, 7, 1, 1)


@pytest.mark.parametrize("x", [math.inf, math.nan, 1e37, 3000.0])
@pytest.mark.parametrize("n,queries", [(3000, (1, 1)), (3000, (70, 60)), (70000, (1, 1))])
def test_select_without_sums_in_64_bits_for_blocks_taken_anyway(n, queries, x):
    """What the blocks taken anyway hold, and those past a token's position that others of its row reach, leaves
    the sums in 64 bits of all other blocks undone: their place in the workspace, behind 4 bytes for each block
    and token, keeps what it holds."""
    import paper_2608_02947_amd as atf
    note(f"select forced, no sums {n} {queries} {x}")
    d, h, pt, bt = 64, 16, 32, 32
    win, W = B.windows(d, "off")
    tok = B.Tokens([n, 640], queries, pt, 9, pad=0)
    q = torch.randn((tok.T, h, d), generator=torch.Generator().manual_seed(9)).to(B.BF)
    plain = B.random_bounds(tok.P, pt, bt, h, d, 9)
    keys = tok.T * h * (-(-n // (16 * bt)) * 16)
    at = -(-4 * keys // 256) * 256
    for j, summed in ((0, False), (-1, False), (n // bt // 2, True)):
        b = plain.clone()
        for row, pos in zip(tok.rows, tok.pos):
            if j != -1:
                b[tok.table[row, j if row == 0 or not summed else 9]] = x
        if j == -1:  # the last blocks that any token of a row reaches: nobody compares them
            for row in range(2):
                last = tok.pos[tok.rows == row]
                b[tok.table[row, last.min() // bt: last.max() // bt + 1]] = x
        ws = torch.full((atf.atf_select_workspace_bytes(tok.T, h, h, n, bt, d),), 0x5A, dtype=torch.uint8, device=B.DEV)
        got = B.selected(tok, q.to(B.DEV), b.to(B.DEV), bt, win, 7, 1, 3, ws=ws).cpu().numpy()
        assert np.array_equal(got, chosen(tok, q.double().numpy(), b.double().numpy(), bt, W, 7, 1, 3))
        if summed and not math.isfinite(x):
            assert not bool((ws[at: at + 8 * keys] == 0x5A).all())
        elif not summed:
            assert bool((ws[at: at + 8 * keys] == 0x5A).all())


@pytest.mark.parametrize("kind", ["exact", "sliding"])
def test_select_for_queries_that_are_none(kind):
    """NaN and infinities in queries: scores that are none, or infinite; past its pair's window such a number does
    not count, and other tokens' choices do not see it."""
    note(f"select queries {kind}")
    d, h_q, h_kv, pt, bt = 64, 6, 2, 64, 32
    win, W = B.windows(d, kind)
    tok = B.Tokens([1500, 700], [6, 3], pt, 8)
    g = torch.Generator().manual_seed(3)
    for x in (math.nan, math.inf, -math.inf, 3e38):
        q = torch.randn((tok.T, h_q, d), generator=g).to(B.BF)
        q[1, 0, 3], q[2, 4, 33], q[4, 5, 31], q[7, 1, 0], q[7, 2, 40] = x, x, x, x, -x
        check(tok, q, B.random_bounds(tok.P, pt, bt, h_kv, d, 7), bt, win, W, 9, 1, 1)


@pytest.mark.parametrize("x", [math.inf, math.nan])
@pytest.mark.parametrize("d,h_q", [(64, 5), (128, 20)])
def test_attend_for_queries_that_are_none(d, h_q, x):
    """Such a number is its own head's and token's: all others stay within check_attend's errors of what they are
    without it (twice, once for each call: their sums may be scaled at other tiles)."""
    note(f"attend queries {d} {h_q} {x}")
    h_kv, pt, bt = 1, 64, 32
    win, W = B.windows(d, "sliding")
    tok = B.Tokens([333, 150], [1, 2], pt, 5)
    q = torch.randn((tok.T, h_q, d), generator=torch.Generator().manual_seed(1)).to(B.BF)
    kp, vp = B.random_pools(tok.P, pt, h_kv, d, 2)
    lists = B.random_lists(tok, h_kv, 4, bt, 1, wild=False)
    lists[0, 0] = [6, 7, 9, 10]  # the newest and those where the windows of 100 tokens end
    o, lse = B.check_attend(tok, q, kp, vp, lists, bt, win, W)
    wo, _, mass, size = R.attend(q.double().numpy(), kp.double().numpy(), vp.double().numpy(), tok.table, tok.rows, tok.pos,
                                 tok.lens, lists, W, pt, bt, d ** -0.5)
    bad = q.clone()
    bad[0, 1, 3] = x
    o2, lse2 = (B.to64(y)[:3] for y in B.attended(tok, bad.to(B.DEV), kp.to(B.DEV), vp.to(B.DEV), lists, bt, win))
    assert np.isnan(o2[0, 1]).all() and np.isnan(lse2[0, 1])
    e = (d + 2) * 2.0 ** -23 * size[:3] + 2.0 ** -22 * (size[:3] + 1)
    tol = 2.0 ** -7 * np.abs(wo[:3]) + 2 * (2 * e + 2.0 ** -15 + 4 * bt * 2.0 ** -23)[..., None] * mass[:3]
    rest = np.ones((3, h_q), dtype=bool)
    rest[0, 1] = False
    assert (np.abs(o2 - o) <= tol)[rest].all()
    tol_l = 2 * (e + 4 * bt * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(lse)))
    assert (np.abs(lse2 - lse) <= tol_l)[rest].all()


# ---- at once

def test_two_streams_with_their_work_queued():
    """Steps of two streams queued before either has begun, their inputs on the device: the same bits as one after
    the other.  Each has buffers and workspaces of its own."""
    note("two streams queued")
    make = lambda: B.Engine(B=6, h_q=8, h_kv=4, width=200, pages=700, T=2000, top=12)
    one, two, ref = make(), make(), make()
    news = [[500, 300, 0, 700, 40, 400], [1, 1, 900, 1, 1, 1], [1, 1, 1, -1, 0, 1], [600, 40, 1, 90, 1, 700], [1] * 6,
            [150, 0, -1, 1, 1, 800]]
    g = torch.Generator().manual_seed(1)
    inputs = [([torch.randn(x.shape, generator=g).to(B.BF).to(B.DEV) for x in (ref.q, ref.k, ref.v)], B.dev32(n)) for n in news]

    def step(e, i):
        for x, y in zip((e.q, e.k, e.v), inputs[i][0]):
            x.copy_(y)
        e.n_new.copy_(inputs[i][1])
        e.step()
    want = []
    for i in range(len(news)):
        step(ref, i)
        want.append(ref.state())
    torch.cuda.synchronize()
    streams, gate, got = [torch.cuda.Stream(), torch.cuda.Stream()], torch.randn((4096, 4096), device=B.DEV), ([], [])
    torch.cuda.synchronize()
    for _ in range(20):  # (both streams wait for this while their steps are queued)
        gate = gate @ gate * 1e-3
    begin = torch.cuda.Event()
    begin.record()
    for s in streams:
        s.wait_event(begin)
    for i in range(len(news)):
        for e, s, keep in zip((one, two), streams, got):
            with torch.cuda.stream(s):
                step(e, i)
                keep.append(e.state())
    torch.cuda.synchronize()
    for states in got:
        for i, state in enumerate(states):
            for x, y in state.items():
                assert torch.equal(y.view(torch.uint8), want[i][x].view(torch.uint8)), (i, x)
