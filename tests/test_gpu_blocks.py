"""Pages and slots, appends through slots, bounds of blocks, their selection and attention over them on the
GPU, against the plain 64-bit forms of blocksref.py."""
import math

import numpy as np
import pytest
import torch

import blocksref as R
from conftest import gpu_available
from parity import note

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]

DEV, BF = "cuda", torch.bfloat16
SENTINEL = 0x5A5A


def dev32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def to64(t):
    return t.detach().cpu().double().numpy()


def filled(shape):
    return torch.full(shape, SENTINEL, dtype=torch.int16, device=DEV).view(BF)


def bits(t):
    return t.detach().cpu().view(torch.int16)


# ---- pages and slots

class PlanState:
    def __init__(self, B, width, pt, T, seed, kind):
        rng = np.random.default_rng(seed)
        self.pt, self.T = pt, T
        cap = width * pt
        n = rng.integers(0, cap + 1, B)
        n[rng.random(B) < 0.2] = 0
        new = {"step": np.ones(B, dtype=np.int64), "idle": np.zeros(B, dtype=np.int64)}.get(
            kind, rng.integers(0, max(2, 2 * T // max(B, 1)), B))
        if kind != "idle":
            new[rng.random(B) < 0.15] = -rng.integers(1, 5)
            new[rng.random(B) < 0.1] = 0
        if kind == "fits":
            new = np.minimum(new, cap - n)
        used = -(-n // pt)
        total = int(used.sum())
        grow = np.maximum(new, 0)
        wants = int(np.where(n + grow <= cap, -(-(n + grow) // pt) - used, 0).sum())
        free = {"short": wants // 2, "none": 0}.get(kind, wants + 3)
        ids = rng.permutation(total + free + 5)
        table = np.full((B, width), -7)
        at = 0
        for b in range(B):
            table[b, :used[b]] = ids[at: at + used[b]]
            at += used[b]
        slack = 0 if kind == "tight" else total  # room for the pages that come back
        self.free = np.concatenate([ids[at: at + free], np.full(slack, -9)]).astype(np.int64)
        self.count, self.n, self.new, self.table = free, n, new, table

    def run(self, in_place=False, stream=None):
        import paper_2608_02947_amd as atf
        B, T = len(self.n), self.T
        self.t = dict(block_table=dev32(self.table), free_pages=dev32(self.free), n_k=dev32(self.n), n_new=dev32(self.new),
                      row_starts=dev32(np.full(B + 1, 77)), slots=torch.full((T,), 77, dtype=torch.int64, device=DEV),
                      token_rows=dev32(np.full(T, 77)), positions=dev32(np.full(T, 77)))
        t = self.t
        if in_place:
            t["counts"] = dev32([self.count, 55, 55])
            t["n_k_out"], count = t["n_k"], t["counts"]
        else:
            t["counts"], t["n_k_out"], count = dev32([55] * 3), dev32(np.full(B, 77)), dev32([self.count])
        call = lambda: atf.atf_plan_pages(t["block_table"], self.pt, t["free_pages"], count, t["n_k"], t["n_new"], t["n_k_out"],
                                          t["row_starts"], t["slots"], t["token_rows"], t["positions"], t["counts"],
                                          stream=stream)
        call()
        torch.cuda.synchronize()
        if not in_place:  # again: the same
            call()
            torch.cuda.synchronize()
        return self

    def check(self):
        want = R.plan(self.table, self.pt, self.free, self.count, self.n, self.new, self.T)
        for name, x in want.items():
            got = self.t[name].cpu().numpy()
            assert np.array_equal(got, x), (name, np.flatnonzero(got.reshape(-1) != x.reshape(-1))[:5])


@pytest.mark.parametrize("kind", ["step", "fits", "long", "short", "none", "tight", "idle"])
@pytest.mark.parametrize("B,width,pt,T", [(1, 1, 32, 1), (1, 700, 32, 30000), (3, 5, 64, 40), (64, 9, 32, 64), (70, 20, 96, 900),
                                          (200, 30, 64, 300), (1024, 3, 32, 1500), (1025, 3, 32, 1500), (2500, 4, 64, 2600),
                                          (24, 400, 32, 9000), (5, 3, 32, 0), (7, 40, 32, 2048), (7, 40, 32, 2049), (7, 40, 32, 8193)])
def test_plan(B, width, pt, T, kind):
    note(f"plan {B} {width} {pt} {T} {kind}")
    PlanState(B, width, pt, T, B + T, kind).run().check()


@pytest.mark.parametrize("B,T", [(3, 50), (1024, 2000), (1500, 9000), (40, 20000)])
def test_plan_in_place(B, T):
    note(f"plan in place {B} {T}")
    PlanState(B, 12, 32, T, 5, "fits").run(in_place=True).check()


def test_plan_of_values_out_of_range():
    """Lengths past the pages, a stack higher than its array, negative ones."""
    note("plan out of range")
    s = PlanState(9, 4, 32, 100, 8, "fits")
    s.n = s.n + np.array([0, 1000, -500, 0, 0, 2 ** 31 - 1 - s.n[5], 0, 0, -1 - s.n[8]])
    s.count = 10 ** 6
    s.run().check()
    s.count = -3
    s.run().check()
    s.new[:] = 2 ** 31 - 1
    s.run().check()


# ---- appends through slots

def slot_case(kind, T, pages, pt, rng):
    pool = pages * pt
    if kind == "scattered":
        x = rng.permutation(pool)[:T].astype(np.int64)
    elif kind == "runs":  # rows of any length from any place, a few tokens of padding between them
        x, at = np.full(T, -1, dtype=np.int64), 0
        free = list(rng.permutation(pages))
        while at < T and free:
            n = int(rng.integers(1, 3 * pt))
            first = int(rng.integers(0, pt))
            page, i = free.pop(), 0
            while i < n and at < T:
                p = first + i
                if p and p % pt == 0:
                    if not free:
                        break
                    page = free.pop()
                x[at] = page * pt + p % pt
                at, i = at + 1, i + 1
            at += int(rng.integers(0, 3))
    else:
        x = np.arange(T, dtype=np.int64) + 5  # one run over pages in order
    if T > 3:
        x[rng.integers(0, T)] = -1
        x[rng.integers(0, T)] = -2 ** 40
        x[rng.integers(0, T)] = pool
    return x


@pytest.mark.parametrize("kind", ["scattered", "runs", "straight"])
@pytest.mark.parametrize("d,h_kv,T,pt", [(64, 1, 1, 32), (128, 2, 3, 32), (64, 3, 37, 96), (128, 8, 300, 64), (64, 16, 700, 32),
                                         (128, 4, 2500, 128), (128, 1, 9000, 64)])
def test_append_slots(d, h_kv, T, pt, kind):
    import paper_2608_02947_amd as atf
    note(f"slots {d} {h_kv} {T} {pt} {kind}")
    rng = np.random.default_rng(T + d)
    pages = T // pt + 7
    slots = slot_case(kind, T, pages, pt, rng)
    g = torch.Generator().manual_seed(T)
    k, v = torch.randn((T, h_kv, d), generator=g).to(BF), torch.randn((T, h_kv, d), generator=g).to(BF)
    kp, vp = filled(atf.kpages_shape(pages, pt, h_kv, d)), filled(atf.vpages_shape(pages, pt, h_kv, d))
    want_k, want_v = bits(kp).numpy().copy(), bits(vp).numpy().copy()
    for t in range(T):
        if 0 <= slots[t] < pages * pt:
            R.put_k(want_k, slots[t] // pt, slots[t] % pt, bits(k[t]).numpy())
            R.put_v(want_v, slots[t] // pt, slots[t] % pt, bits(v[t]).numpy())
    atf.atf_cache_append_slots(k.to(DEV), v.to(DEV), kp, vp, torch.tensor(slots, device=DEV))
    torch.cuda.synchronize()
    assert np.array_equal(bits(kp).numpy(), want_k) and np.array_equal(bits(vp).numpy(), want_v)


@pytest.mark.parametrize("d,h_kv,n,pos0", [(64, 2, 1, 0), (128, 3, 90, 7), (128, 8, 1300, 1000001), (64, 1, 9000, 2 ** 30)])
def test_append_slots_rotated_is_the_paged_append(d, h_kv, n, pos0):
    """Keys turned to positions[t]: bit for bit what atf_cache_append_paged_rotated stores at slots of its
    own choice (the same positions, a table of its own)."""
    import paper_2608_02947_amd as atf
    note(f"slots rotated {d} {h_kv} {n} {pos0}")
    pt = 64
    first = pos0 // pt  # the table's first page in use
    pages = (pos0 + n - 1) // pt - first + 1
    win = atf.Window(d, 1e6, 2.0)
    g = torch.Generator().manual_seed(n)
    k, v = (torch.randn((n, h_kv, d), generator=g).to(BF).to(DEV) for _ in range(2))
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.zeros((1, first + pages), dtype=torch.int32)
    table[0, first:] = order
    new = lambda: (filled(atf.kpages_shape(pages, pt, h_kv, d)), filled(atf.vpages_shape(pages, pt, h_kv, d)))
    (ka, va), (kb, vb) = new(), new()
    atf.atf_cache_append_paged_rotated(k[None], v[None], ka, va, table.to(DEV), pos0, win)
    pos = torch.arange(pos0, pos0 + n)
    slots = table[0, pos // pt].long() * pt + pos % pt
    atf.atf_cache_append_slots_rotated(k, v, kb, vb, slots.to(DEV), pos.to(torch.int32).to(DEV), win)
    torch.cuda.synchronize()
    assert torch.equal(bits(ka), bits(kb)) and torch.equal(bits(va), bits(vb))


def test_append_slots_rotated_frequencies_and_any_order():
    """Positions in any order, frequencies given apart from the window, against the formula: the angle's
    error is 2^-24 turns and that of the sine and cosine, the products' 2^-23 of the pair's size, and the
    result rounds to bf16 (half a step: 2^-8)."""
    import paper_2608_02947_amd as atf
    note("slots rotated, formula")
    T, h_kv, d, pt, pages = 200, 2, 64, 32, 9
    rng = np.random.default_rng(1)
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn((T, h_kv, d), generator=g).to(BF) for _ in range(2))
    freq = rng.uniform(1e-4, 1.0, d // 2)
    slots, pos = rng.permutation(pages * pt)[:T], rng.integers(0, 100000, T)
    kp, vp = filled(atf.kpages_shape(pages, pt, h_kv, d)), filled(atf.vpages_shape(pages, pt, h_kv, d))
    atf.atf_cache_append_slots_rotated(k.to(DEV), v.to(DEV), kp, vp, torch.tensor(slots, device=DEV), dev32(pos),
                                       atf.Window(d, 1e4, 2.0), rope_inv_freq=freq)
    torch.cuda.synchronize()
    kp = to64(kp)
    x = k.double().numpy()
    z = (x[..., :d // 2] + 1j * x[..., d // 2:]) * np.exp(1j * (pos[:, None] * freq))[:, None]
    for t in range(T):
        got = R.get_k(kp, slots[t] // pt, slots[t] % pt)
        want = np.concatenate([z[t].real, z[t].imag], axis=1)
        size = np.concatenate([np.abs(z[t])] * 2, axis=1)
        assert (np.abs(got - want) <= 2 ** -8 * np.abs(want) + 2 ** -18 * size).all()


# ---- bounds of blocks

@pytest.mark.parametrize("d,h_kv,pt,bt", [(64, 1, 32, 32), (128, 3, 64, 32), (128, 2, 64, 64), (64, 5, 96, 96), (128, 4, 256, 128),
                                          (64, 2, 192, 64)])
@pytest.mark.parametrize("lens,news", [([1], [1]), ([300, 0, 31, 32, 33, 64], [1, 1, 5, 32, 2, -1]),
                                       ([257, 383, 129, 96, 2], [257, 100, 0, 1, 3])])
def test_block_bounds(d, h_kv, pt, bt, lens, news):
    import paper_2608_02947_amd as atf
    note(f"bounds {d} {h_kv} {pt} {bt} {lens}")
    rng = np.random.default_rng(d + pt + len(lens))
    B, width = len(lens), -(-384 // pt)
    P = B * width + 2
    table = rng.permutation(P)[:B * width].reshape(B, width)
    k = torch.tensor(rng.standard_normal(atf.kpages_shape(P, pt, h_kv, d)), dtype=torch.float32).to(BF)
    flat = k.view(-1)
    for x in (math.nan, math.inf, -math.inf, -0.0, 0.0, 3e38):
        flat[torch.tensor(rng.integers(0, flat.numel(), flat.numel() // 3000 + 2))] = x
    kd = k.to(DEV)
    k64 = k.double().numpy()
    for max_new in (1000, 40):
        out = filled(atf.bounds_shape(P, pt, bt, h_kv, d))
        want = R.bounds(k64, to64(out), table, lens, news, max_new, pt, bt)
        atf.atf_block_bounds(kd, out, dev32(table), dev32(lens), dev32(news), max_new)
        torch.cuda.synchronize()
        got = to64(out)
        assert np.array_equal(got, want, equal_nan=True)
        assert np.array_equal(bits(out).numpy() == SENTINEL, bits(torch.tensor(want).to(BF)).numpy() == SENTINEL)


@pytest.mark.parametrize("rows,pages,pt,h_kv", [(1, 4300, 64, 4), (1300, 3, 32, 2)])
def test_block_bounds_of_long_rows_and_many(rows, pages, pt, h_kv):
    """More blocks of a row, and more rows, than a launch has workgroups for at once."""
    import paper_2608_02947_amd as atf
    note(f"bounds {rows} rows of {pages} pages")
    d, bt, P = 64, 32, rows * pages
    k = torch.randn(atf.kpages_shape(P, pt, h_kv, d), generator=torch.Generator().manual_seed(rows)).to(BF)
    x = k.view(P, h_kv, d // 16, pt // bt, bt, 16).permute(0, 1, 3, 2, 4, 5)
    want = torch.stack([x.amax(dim=4), x.amin(dim=4)], dim=4)
    out = filled(atf.bounds_shape(P, pt, bt, h_kv, d))
    n = np.full(rows, pages * pt)
    atf.atf_block_bounds(k.to(DEV), out, dev32(np.arange(P).reshape(rows, pages)), dev32(n), dev32(n), pages * pt)
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), want)


def test_block_bounds_nan_of_either_sign():
    import paper_2608_02947_amd as atf
    note("bounds of NaNs")
    k = torch.zeros(atf.kpages_shape(1, 32, 1, 64), dtype=BF)
    raw = k.view(torch.int16)
    raw[0, 0, 0, 3, 2], raw[0, 0, 1, 31, 5], raw[0, 0, 2, 0, 0], raw[0, 0, 3, 1, 15] = 0x7F81, -1, -128 + 1, 0x7FFF
    out = filled(atf.bounds_shape(1, 32, 32, 1, 64))
    atf.atf_block_bounds(k.to(DEV), out, dev32([[0]]), dev32([32]), dev32([32]), 32)
    got = out.cpu().float()[0, 0, 0]
    want = torch.zeros_like(got)
    want[0, :, 2] = want[1, :, 5] = want[2, :, 0] = want[3, :, 15] = math.nan
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(), want.nan_to_num())


# ---- selection

def windows(d, kind):
    import paper_2608_02947_amd as atf
    w = {"exact": lambda: atf.Window(d, 1e4, 2.0), "off": lambda: atf.Window(d, 1e4, math.inf),
         "rounded": lambda: atf.Window(d, 1e4, 2.0, slice_pairs=8),
         "sliding": lambda: atf.Window(d, 1e4, 0.0, beta=100.0, cap=100.0),
         "falling": lambda: atf.Window(d, 1e4, 1.0, inv_freq=np.geomspace(1e-3, 0.5, d // 2))}[kind]()
    return w, atf.atf_window_table(w).astype(np.int64)


class Tokens:
    """Rows, lengths and packed query tokens: `queries` of each row, the last of them at its end or at
    `shift` from it, and padding."""

    def __init__(self, lens, queries, pt, seed, shift=0, pad=2, shared=0):
        rng = np.random.default_rng(seed)
        self.pt, self.lens = pt, np.array(lens)
        need = np.maximum(1, -(-self.lens // pt))
        width = int(need.max()) + 1
        self.P = int(need.sum()) + 2
        order = rng.permutation(self.P)
        self.table = np.full((len(lens), width), -1)
        at = 0
        for b in range(len(lens)):
            self.table[b, :need[b]] = order[at: at + need[b]]
            at += need[b]
        for b in range(1, len(lens)):  # a prefix that rows share
            m = min(shared, need[b] - 1, need[0] - 1)
            self.table[b, :max(m, 0)] = self.table[0, :max(m, 0)]
        rows, pos = [], []
        for b, n in enumerate(lens):
            for i in range(queries[b]):
                rows.append(b)
                pos.append(n - queries[b] + i + shift)
        rows += [-1, len(lens)][:pad]
        pos += [-1, 3][:pad]
        self.rows, self.pos = np.array(rows), np.array(pos)
        self.T = len(rows)


def selected(tok, q, bnd, bt, win, top, first, last, max_n_k=None, ws=None, stream=None, out=None):
    import paper_2608_02947_amd as atf
    h_q, d, h_kv = q.shape[1], q.shape[2], bnd.shape[1]
    max_n_k = max_n_k or max(1, int(tok.lens.max()))
    if out is None:
        out = torch.full((tok.T, h_kv, top), 777, dtype=torch.int32, device=DEV)
    if ws is None:
        ws = torch.empty(atf.atf_select_workspace_bytes(tok.T, h_q, h_kv, max_n_k, bt, d), dtype=torch.uint8, device=DEV)
    atf.atf_select_blocks(q, bnd, out, dev32(tok.table), tok.pt, dev32(tok.rows), dev32(tok.pos), dev32(tok.lens), max_n_k,
                          win, ws, first_blocks=first, last_blocks=last, stream=stream)
    torch.cuda.synchronize()
    return out


def random_bounds(P, pt, bt, h_kv, d, seed):
    import paper_2608_02947_amd as atf
    g = torch.Generator().manual_seed(seed)
    shape = list(atf.bounds_shape(P, pt, bt, h_kv, d))
    shape[4] = 1
    mid, reach = 0.4 * torch.randn(shape, generator=g), 1.5 + 0.5 * torch.randn(shape, generator=g).abs()
    return torch.cat([mid + reach, mid - reach], dim=4).to(BF)


def check_select(tok, q, bnd, bt, win, W, top, first, last, max_n_k=None):
    got = selected(tok, q.to(DEV), bnd.to(DEV), bt, win, top, first, last, max_n_k)
    want = np.full(got.shape, 777)
    R.select(q.double().numpy(), bnd.double().numpy(), tok.table, tok.rows, tok.pos, tok.lens,
             max_n_k or max(1, int(tok.lens.max())), W, tok.pt, bt, top, first, last, want)
    assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("kind", ["exact", "off", "rounded", "sliding", "falling"])
@pytest.mark.parametrize("d,h_q,h_kv,pt,bt,top,first,last", [
    (64, 2, 2, 32, 32, 4, 1, 1), (128, 14, 2, 64, 32, 7, 0, 0), (128, 20, 1, 64, 64, 5, 1, 2), (64, 40, 2, 96, 32, 12, 2, 3),
    (128, 8, 8, 128, 128, 3, 3, 0), (64, 6, 2, 192, 64, 1, 0, 1), (128, 33, 1, 64, 32, 9, 1, 1)])
def test_select(d, h_q, h_kv, pt, bt, top, first, last, kind):
    note(f"select {d} {h_q}/{h_kv} {pt} {bt} {top} {kind}")
    win, W = windows(d, kind)
    for seed, (lens, queries, shift) in enumerate([([1, 0, 700, 33, 64], [1, 1, 1, 1, 1], 0), ([900, 500], [5, 3], 0),
                                                   ([321, 640], [3, 1], -200), ([400, 250], [1, 2], 60)]):
        tok = Tokens(lens, queries, pt, seed, shift)
        q = torch.randn((tok.T, h_q, d), generator=torch.Generator().manual_seed(seed)).to(BF)
        check_select(tok, q, random_bounds(tok.P, pt, bt, h_kv, d, seed + 9), bt, win, W, top, first, last)


@pytest.mark.parametrize("n,top,bt,pt", [(70001, 300, 32, 64), (40000, 1, 32, 32), (33000, 40, 64, 64), (9000, 4096, 32, 32)])
def test_select_long_rows(n, top, bt, pt):
    note(f"select long {n} {top} {bt}")
    d, h_q, h_kv = 64, 3, 1
    win, W = windows(d, "exact")
    tok = Tokens([n, n // 3], [2, 1], pt, n)
    q = torch.randn((tok.T, h_q, d), generator=torch.Generator().manual_seed(n)).to(BF)
    check_select(tok, q, random_bounds(tok.P, pt, bt, h_kv, d, n), bt, win, W, top, min(1, top - 1), 1)


def test_select_many_tokens():
    """More tokens than one launch may take, each with blocks of its own."""
    note("select many")
    d, h_q, h_kv, pt, bt = 64, 2, 2, 32, 32
    win, W = windows(d, "exact")
    lens, queries = [40, 65, 200, 7], [40, 65, 100, 7]
    tok = Tokens(lens, queries, pt, 3)
    q = torch.randn((tok.T, h_q, d), generator=torch.Generator().manual_seed(1)).to(BF)
    check_select(tok, q, random_bounds(tok.P, pt, bt, h_kv, d, 2), bt, win, W, 3, 1, 1)


@pytest.mark.parametrize("what", ["random", "zeros", "NaN"])
def test_select_more_tokens_than_a_workspace_holds(what):
    """Rows that may be long: the workspace holds some of the call's tokens at a time."""
    import paper_2608_02947_amd as atf
    note(f"select workspace {what}")
    d, h_q, h_kv, pt, bt = 64, 6, 2, 32, 32
    win, W = windows(d, "exact")
    tok = Tokens([600, 333], [130, 100], pt, 3)
    pages = 1 << 17
    most = pages * pt
    assert atf.atf_select_workspace_bytes(tok.T, h_q, h_kv, most, bt, d) < \
        tok.T // 2 * atf.atf_select_workspace_bytes(1, h_q, h_kv, most, bt, d)
    tok.table = np.pad(tok.table, ((0, 0), (0, pages - tok.table.shape[1])), constant_values=-1)
    q = torch.randn((tok.T, h_q, d), generator=torch.Generator().manual_seed(1)).to(BF)
    b = random_bounds(tok.P, pt, bt, h_kv, d, 2)
    if what == "zeros":
        b.zero_()
    elif what == "NaN":
        b.view(-1)[torch.arange(0, b.numel(), 3001)] = math.nan
    check_select(tok, q, b, bt, win, W, 5, 1, 1, max_n_k=most)


@pytest.mark.parametrize("what", ["random", "zeros", "NaN"])
@pytest.mark.parametrize("queries", [(1, 1), (140, 80)])
def test_select_many_picks(what, queries):
    """More than 2,048 (token, KV head)s, and few, at the same sizes: alike, and the plain form's."""
    note(f"select picks {what} {queries}")
    d, h, pt, bt = 64, 16, 64, 32
    win, W = windows(d, "exact")
    tok = Tokens([180, 130], queries, pt, 3)
    q = torch.randn((tok.T, h, d), generator=torch.Generator().manual_seed(1)).to(BF)
    b = random_bounds(tok.P, pt, bt, h, d, 2)
    if what == "zeros":
        b.zero_()
    elif what == "NaN":
        b.view(-1)[torch.arange(0, b.numel(), 4001)] = math.nan
    check_select(tok, q, b, bt, win, W, 3, 0, 1)


def test_select_many_equal_blocks_of_many_tokens():
    """More blocks at the border than are listed (64 where a wave picks, else 256), nearly all alike."""
    note("select equal, many")
    d, h, pt, bt = 64, 16, 32, 32
    win, W = windows(d, "off")
    for queries, n in (((130, 3), 4000), ((1, 1), 12000)):
        tok = Tokens([n, 90], queries, pt, 3)
        q = torch.randint(-1, 2, (tok.T, h, d), generator=torch.Generator().manual_seed(1)).to(BF)
        b = torch.ones(random_bounds(tok.P, pt, bt, h, d, 2).shape, dtype=BF)
        b[::7] = 2.0
        got = selected(tok, q.to(DEV), b.to(DEV), bt, win, 30, 1, 1).cpu().numpy()
        # one token's in the plain form; the others choose by their own queries, two of them checked
        for t in {0, min(5, tok.T - 3), tok.T - 3}:
            one = np.full((1,) + got.shape[1:], 777)
            R.select(q[t:t + 1].double().numpy(), b.double().numpy(), tok.table, tok.rows[t:t + 1], tok.pos[t:t + 1],
                     tok.lens, n, W, pt, bt, 30, 1, 1, one)
            assert np.array_equal(got[t], one[0])


@pytest.mark.parametrize("what", ["zeros", "equal", "shared", "integers", "close"])
def test_select_ties_go_to_the_lower_block(what):
    note(f"select ties {what}")
    d, h_q, h_kv, pt, bt, top = 64, 4, 2, 32, 32, 6
    win, W = windows(d, "off")
    tok = Tokens([640, 333], [2, 1], pt, 4)
    g = torch.Generator().manual_seed(6)
    q = torch.randn((tok.T, h_q, d), generator=g).to(BF)
    b = random_bounds(tok.P, pt, bt, h_kv, d, 5)
    if what == "zeros":
        b.zero_()
    elif what == "equal":
        b[:] = b[:1]
    elif what == "shared":  # half of a row's entries name one page
        tok.table[:, 3:9] = tok.table[:, 2:3]
    elif what == "integers":
        b, q = torch.randint(-2, 3, b.shape, generator=g).to(BF), torch.randint(-1, 2, q.shape, generator=g).to(BF)
    else:  # a large common part, differences that fp32 does not hold beside it
        b[:] = b[:1] * 0 + 200.0
        b[..., 0, 5] = 200.0 + torch.randint(0, 2, b[..., 0, 5].shape, generator=g).to(BF)
        q = q.abs()
        q[..., 5 + 8 * 0] = 2.0 ** -12
    check_select(tok, q, b, bt, win, W, top, 1, 1)


@pytest.mark.parametrize("kind", ["exact", "sliding"])
def test_select_numbers_that_are_none(kind):
    """Blocks with NaN in a pair that the window keeps come before all others; past its pair's window such
    a number does not count.  Infinite bounds: inf * 0 is NaN, others are infinitely large scores."""
    note(f"select NaN {kind}")
    d, h_q, h_kv, pt, bt, top = 64, 6, 2, 64, 32, 5
    win, W = windows(d, kind)
    tok = Tokens([1500, 700], [2, 2], pt, 8)
    g = torch.Generator().manual_seed(3)
    q = torch.randn((tok.T, h_q, d), generator=g).to(BF)
    rng = np.random.default_rng(4)
    for x, count in ((math.nan, 9), (math.inf, 12), (-math.inf, 12), (math.nan, 400)):
        b = random_bounds(tok.P, pt, bt, h_kv, d, 7)
        b.view(-1)[torch.tensor(rng.integers(0, b.numel(), count))] = x
        check_select(tok, q, b, bt, win, W, top, 1, 1)


@pytest.mark.parametrize("n,queries", [(640, (2, 1)), (640, (130, 9)), (9000, (1, 1)), (40000, (1, 1)), (600000, (1, 1))])
def test_select_only_what_is_taken_anyway(n, queries):
    """first_blocks + last_blocks = top_blocks: no other block, though some have scores that are none; the lists
    behind each other, so that one too long would show in the next."""
    note(f"select forced {n} {queries}")
    d, h, pt, bt = 64, 16, 64, 32
    win, W = windows(d, "off")
    tok = Tokens([n, 333], queries, pt, 4)
    q = torch.randn((tok.T, h, d), generator=torch.Generator().manual_seed(6)).to(BF)
    b = torch.full(random_bounds(1, pt, bt, h, d, 5).shape, math.nan, dtype=BF).expand(tok.P, -1, -1, -1, -1, -1)
    got = selected(tok, q.to(DEV), b.to(DEV).contiguous(), bt, win, 5, 3, 2).cpu().numpy()
    for t in range(tok.T - 2):
        last = tok.pos[t] // bt
        want = list(range(min(3, last + 1))) + list(range(max(3, last - 1), last + 1))
        want = sorted(set(want)) if last >= 5 else list(range(last + 1))
        assert (got[t] == np.array(want + [-1] * (5 - len(want)))).all(), t
    assert (got[tok.T - 2:] == 777).all()


def test_select_tiny_and_huge_numbers():
    """Denormal bounds beside queries that bring their products to size, and sums past fp32."""
    note("select tiny and huge")
    d, h_q, h_kv, pt, bt = 64, 4, 2, 32, 32
    win, W = windows(d, "off")
    tok = Tokens([640, 333], [2, 1], pt, 4)
    g = torch.Generator().manual_seed(6)
    q = torch.randn((tok.T, h_q, d), generator=g)
    b = random_bounds(tok.P, pt, bt, h_kv, d, 5).float()
    for x, y in ((2.0 ** 100, 2.0 ** -129), (2.0 ** 60, 2.0 ** 70), (2.0 ** 120, 2.0 ** -131), (2.0 ** -126, 2.0 ** 3)):
        check_select(tok, (q * x).to(BF), (b * y).to(BF), bt, win, W, 6, 1, 1)


@pytest.mark.parametrize("queries", [(2, 1), (130, 9)])
def test_select_products_below_fp32(queries):
    """Products that fp32 holds with few bits or none: the blocks are those of sums in 64 bits all the same."""
    note(f"select products below fp32 {queries}")
    d, h_q, h_kv, pt, bt = 128, 4, 2, 32, 32
    win, W = windows(d, "exact")
    tok = Tokens([3000, 700], list(queries), pt, 4)
    q = torch.randn((tok.T, h_q, d), generator=torch.Generator().manual_seed(8))
    b = random_bounds(tok.P, pt, bt, h_kv, d, 6).float()
    for e in (-66, -70, -73, -78):
        check_select(tok, (q * 2.0 ** e).to(BF), (b * 2.0 ** e).to(BF), bt, win, W, 9, 1, 1)


def test_select_of_entries_out_of_range():
    """Table entries and lengths outside their ranges are clamped."""
    note("select clamps")
    d, h_q, h_kv, pt, bt = 64, 2, 1, 32, 32
    win, W = windows(d, "exact")
    tok = Tokens([300, 200], [1, 1], pt, 2)
    tok.table[0, 2], tok.table[0, 4], tok.table[1, 1] = -5, tok.P + 100, 2 ** 31 - 1
    q = torch.randn((tok.T, h_q, d), generator=torch.Generator().manual_seed(5)).to(BF)
    b = random_bounds(tok.P, pt, bt, h_kv, d, 1)
    check_select(tok, q, b, bt, win, W, 4, 1, 1)
    tok.lens = np.array([2 ** 31 - 1, -4])
    tok.pos[0] = 2 ** 31 - 1
    check_select(tok, q, b, bt, win, W, 4, 1, 1, max_n_k=300)


# ---- attention

def attended(tok, q, kp, vp, lists, bt, win, scale=0.0, ws=None, stream=None):
    import paper_2608_02947_amd as atf
    T, h_q, d = q.shape
    h_kv, top = lists.shape[1], lists.shape[2]
    o, lse = torch.full_like(q, 7.0), torch.full((T, h_q), 7.0, device=DEV)
    if ws is None:
        ws = torch.empty(atf.atf_attend_workspace_bytes(T, h_q, h_kv, top, bt, d), dtype=torch.uint8, device=DEV)
    atf.atf_attend_blocks(q, kp, vp, o, lse, dev32(tok.table), dev32(tok.rows), dev32(tok.pos), dev32(tok.lens),
                          torch.as_tensor(lists, dtype=torch.int32, device=DEV), bt, win, ws, scale, stream=stream)
    torch.cuda.synchronize()
    return o, lse


def random_pools(P, pt, h_kv, d, seed):
    import paper_2608_02947_amd as atf
    g = torch.Generator().manual_seed(seed)
    return (1.5 * torch.randn(atf.kpages_shape(P, pt, h_kv, d), generator=g)).to(BF), \
        torch.randn(atf.vpages_shape(P, pt, h_kv, d), generator=g).to(BF)


def check_attend(tok, q, kp, vp, lists, bt, win, W, scale=0.0):
    """Errors: a score is a sum of d exact products in fp32 (each of d + 2 steps off by 2^-23 at most of the
    sum of magnitudes S, truncation allowed for), its exponent adds |score| 2^-22 and the exponential 2^-22: a
    weight is off by e = (d + 2) 2^-23 S + 2^-22 (S + 1) relative, 2^-16 more as two bf16 numbers; the output by twice that of
    the weighted magnitudes, n 2^-24 for its sums, and half a bf16 step (2^-8).  The LSE by e, n 2^-24 and 2^-22 of itself."""
    d = q.shape[2]
    o, lse = attended(tok, q.to(DEV), kp.to(DEV), vp.to(DEV), lists, bt, win, scale)
    s = scale if scale > 0 else d ** -0.5
    wo, wl, mass, size = R.attend(q.double().numpy(), kp.double().numpy(), vp.double().numpy(), tok.table, tok.rows, tok.pos,
                                  tok.lens, np.asarray(lists), W, tok.pt, bt, s)
    o, lse = to64(o), to64(lse)
    pad = np.array([not 0 <= r < len(tok.lens) for r in tok.rows])
    assert (o[pad] == 7.0).all() and (lse[pad] == 7.0).all()
    o, lse, wo, wl, mass, size = (x[~pad] for x in (o, lse, wo, wl, mass, size))
    n = np.asarray(lists).shape[2] * bt
    e = (d + 2) * 2.0 ** -23 * size + 2.0 ** -22 * (size + 1)
    tol_o = 2.0 ** -8 * np.abs(wo) + (2 * e + 2.0 ** -15 + n * 2.0 ** -23)[..., None] * mass
    bad = ~(np.abs(o - wo) <= tol_o)
    assert not bad.any(), (np.abs(o - wo)[bad].max(), tol_o[bad].min(), np.argwhere(bad)[:3])
    empty = np.isneginf(wl)
    assert np.array_equal(np.isneginf(lse), empty)
    tol_l = e + n * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(np.where(empty, 0, wl)))
    assert (np.abs(lse[~empty] - wl[~empty]) <= tol_l[~empty]).all()
    return o, lse


def random_lists(tok, h_kv, top, bt, seed, wild=True):
    """Blocks of each token in any order, with entries that name none."""
    rng = np.random.default_rng(seed)
    out = np.full((tok.T, h_kv, top), -1, dtype=np.int64)
    for t in range(tok.T):
        b = tok.rows[t]
        if not 0 <= b < len(tok.lens):
            continue
        last = min(tok.lens[b] - 1, tok.pos[t])
        if last < 0:
            continue
        for g in range(h_kv):
            x = rng.permutation(last // bt + 1)[:top]
            if not wild:
                x = np.sort(x)
            out[t, g, :len(x)] = x
            if wild and top > 2:
                out[t, g, rng.integers(0, top)] = rng.choice([-1, -2 ** 31, last // bt + 1, 2 ** 31 - 1, 2 ** 26])
                out[t, g, 0] = last // bt
    return out


SHAPES = [(64, 2, 2, 32, 32, 4), (128, 14, 2, 64, 32, 7), (128, 20, 1, 64, 64, 5), (64, 40, 2, 96, 96, 3),
          (128, 8, 8, 128, 128, 3), (64, 6, 2, 192, 64, 1), (128, 33, 1, 64, 32, 9), (128, 72, 2, 64, 64, 2),
          (64, 17, 1, 32, 32, 30)]


@pytest.mark.parametrize("kind", ["exact", "off", "rounded", "sliding", "falling"])
@pytest.mark.parametrize("d,h_q,h_kv,pt,bt,top", SHAPES)
def test_attend(d, h_q, h_kv, pt, bt, top, kind):
    note(f"attend {d} {h_q}/{h_kv} {pt} {bt} {top} {kind}")
    win, W = windows(d, kind)
    for seed, (lens, queries, shift) in enumerate([([1, 0, 700, 33, 64], [1, 1, 1, 1, 1], 0), ([900, 500], [5, 3], 0),
                                                   ([321, 640], [3, 1], -200), ([400, 250], [1, 2], 60)]):
        tok = Tokens(lens, queries, pt, seed, shift)
        q = torch.randn((tok.T, h_q, d), generator=torch.Generator().manual_seed(seed)).to(BF)
        kp, vp = random_pools(tok.P, pt, h_kv, d, seed + 9)
        check_attend(tok, q, kp, vp, random_lists(tok, h_kv, top, bt, seed), bt, win, W, 0.0 if seed != 1 else 0.3)


@pytest.mark.parametrize("n,top,tokens,d,h_q", [(40000, 300, 1, 64, 7), (9000, 4096, 1, 64, 7), (5000, 60, 2, 64, 7), (3000, 40, 70, 64, 7),
                                                (20000, 200, 1, 128, 3), (6000, 100, 1, 128, 24), (6000, 100, 3, 64, 40),
                                                (700, 9, 300, 64, 20), (700, 9, 300, 128, 20), (700, 9, 300, 128, 3)])
def test_attend_long_lists(n, top, tokens, d, h_q):
    note(f"attend long {n} {top} {tokens} {d} {h_q}")
    h_kv, pt, bt = 1, 64, 32
    win, W = windows(d, "exact")
    tok = Tokens([n, n // 2], [tokens, 1], pt, n)
    q = torch.randn((tok.T, h_q, d), generator=torch.Generator().manual_seed(n)).to(BF)
    kp, vp = random_pools(tok.P, pt, h_kv, d, n)
    check_attend(tok, q, kp, vp, random_lists(tok, h_kv, top, bt, n, wild=False), bt, win, W)


@pytest.mark.parametrize("d,h_q,h_kv", [(64, 16, 16), (128, 16, 16), (64, 17 * 5, 5), (128, 20 * 12, 12)])
def test_attend_many_heads_and_tokens(d, h_q, h_kv):
    """Workgroups of one wave, or two."""
    note(f"attend many {d} {h_q}/{h_kv}")
    pt, bt, top = 32, 32, 2
    win, W = windows(d, "exact")
    tok = Tokens([150, 90], [120, 90], pt, 3)
    q = torch.randn((tok.T, h_q, d), generator=torch.Generator().manual_seed(3)).to(BF)
    kp, vp = random_pools(tok.P, pt, h_kv, d, 3)
    check_attend(tok, q, kp, vp, random_lists(tok, h_kv, top, bt, 3), bt, win, W)


@pytest.mark.parametrize("d,h_q,h_kv", [(64, 7, 1), (128, 24, 1)])
def test_attend_a_block_named_twice_counts_twice(d, h_q, h_kv):
    note(f"attend twice {d}")
    win, W = windows(d, "exact")
    tok = Tokens([200], [1], 32, 1)
    q = torch.randn((tok.T, h_q, d), generator=torch.Generator().manual_seed(3)).to(BF)
    kp, vp = random_pools(tok.P, 32, h_kv, d, 3)
    lists = np.full((tok.T, h_kv, 6), -1)
    lists[0, :] = [3, 3, 0, 6, 3, 1]
    check_attend(tok, q, kp, vp, lists, 32, win, W)


@pytest.mark.parametrize("h_q", [5, 20])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_what_no_token_reaches_does_not_count(d, h_q):
    """NaN and infinities in slots past a row's end, past a token's position, in blocks that are not listed, and
    in pairs past their window change no bit; in a kept pair they give NaN."""
    note(f"attend garbage {d} {h_q}")
    h_kv, pt, bt = 1, 64, 32
    win, W = windows(d, "sliding")
    tok = Tokens([333, 150, 70], [1, 2, 1], pt, 5, shift=-9)
    q = torch.randn((tok.T, h_q, d), generator=torch.Generator().manual_seed(1)).to(BF)
    kp, vp = random_pools(tok.P, pt, h_kv, d, 2)
    lists = np.full((tok.T, h_kv, 4), -1)
    lists[0, 0], lists[1, 0, :2], lists[2, 0, :2], lists[3, 0, :2] = [10, 8, 1, 0], [4, 2], [2, 4], [1, 0]
    a = check_attend(tok, q, kp, vp, lists, bt, win, W)
    kn, vn = kp.clone(), vp.clone()
    used = np.zeros((tok.P, pt), dtype=bool)
    for t in range(4):
        b, last = tok.rows[t], min(tok.lens[tok.rows[t]] - 1, tok.pos[t])
        for j in lists[t, 0]:
            for x in range(j * bt, min((j + 1) * bt, last + 1)) if j >= 0 else ():
                used[tok.table[b, x // pt], x % pt] = True
    bad = (math.nan, math.inf, -math.inf)
    for i, (page, x) in enumerate(np.argwhere(~used)):
        kn[page, :, :, x] = bad[i % 3]
        vn[page, :, x // 16, :, R.v_slot(x % 16)] = bad[i % 3]
    for t in range(100):  # keys of row 0 more than 100 behind its query: no pair kept, at position 323
        kn[tok.table[0, t // pt], :, :, t % pt] = math.nan
    got = attended(tok, q.to(DEV), kn.to(DEV), vn.to(DEV), lists, bt, win)
    assert np.array_equal(to64(got[0])[:4], a[0]) and np.array_equal(to64(got[1])[:4], a[1])
    kn[tok.table[0, 320 // pt], 0, 0, 320 % pt, 0] = math.nan
    got = attended(tok, q.to(DEV), kn.to(DEV), vn.to(DEV), lists, bt, win)
    assert torch.isnan(got[0][0]).all() and torch.isnan(got[1][0]).all() and not torch.isnan(got[0][1:4]).any()


def test_attend_of_all_blocks_is_the_paged_decode():
    """Every block listed: the paged decode's output within both calls' rounding."""
    import paper_2608_02947_amd as atf
    note("attend all = decode")
    d, h_q, h_kv, pt, bt = 128, 24, 8, 64, 64
    win, _ = windows(d, "exact")
    lens = [1000, 0, 64, 517]
    tok = Tokens(lens, [1] * 4, pt, 1, pad=0)
    q = torch.randn((4, h_q, d), generator=torch.Generator().manual_seed(1)).to(BF).to(DEV)
    kp, vp = (x.to(DEV) for x in random_pools(tok.P, pt, h_kv, d, 1))
    lists = np.broadcast_to(np.arange(16), (4, h_kv, 16)).copy()
    tok.pos = np.maximum(tok.pos, 0)
    o, lse = attended(tok, q, kp, vp, lists, bt, win)
    o2, lse2 = torch.empty_like(q), torch.empty((4, h_q), device=DEV)
    ws = torch.empty(atf.atf_decode_workspace_bytes(4, h_q, h_kv, 1000, d), dtype=torch.uint8, device=DEV)
    atf.atf_decode_paged(q, kp, vp, o2, lse2, dev32(tok.table), dev32(lens), dev32(tok.pos), 1000, win, ws)
    torch.cuda.synchronize()
    # the decode holds weights as one bf16 number: 2^-8 of each
    assert (o.double() - o2.double()).abs().max() <= 2.0 ** -7 * (o2.double().abs().max() + vp.double().abs().mean())
    assert torch.equal(torch.isinf(lse), torch.isinf(lse2))
    live = ~torch.isinf(lse)
    assert (lse - lse2)[live].abs().max() <= 1e-4


def test_pages_past_32_bits():
    """Pages further on than 2^32 bytes: the same bits as in a small pool."""
    import paper_2608_02947_amd as atf
    note("pages past 32 bits")
    h_q, h_kv, d, pt, bt, T, top = 24, 8, 128, 256, 64, 700, 5
    big, width = 2 ** 32 // (h_kv * d * 2 * pt) + 40, 3
    win, _ = windows(d, "exact")
    g = torch.Generator().manual_seed(3)
    q = torch.randn((T, h_q, d), generator=g).to(BF).to(DEV)
    k, v = (torch.randn((T, h_kv, d), generator=g).to(BF).to(DEV) for _ in range(2))
    got = []
    for pages, ids in ((3, [2, 0, 1]), (big, [big - 1, big - 9, big - 17])):
        table = dev32([ids])
        kp = torch.empty(atf.kpages_shape(pages, pt, h_kv, d), dtype=BF, device=DEV)
        vp = torch.empty(atf.vpages_shape(pages, pt, h_kv, d), dtype=BF, device=DEV)
        bnd = torch.empty(atf.bounds_shape(pages, pt, bt, h_kv, d), dtype=BF, device=DEV)
        at = torch.arange(T, device=DEV)
        slots = table[0].long()[at // pt] * pt + at % pt
        pos, rows, n = dev32(np.arange(T)), dev32(np.zeros(T)), dev32([T])
        atf.atf_cache_append_slots_rotated(k, v, kp, vp, slots, pos, win)
        atf.atf_block_bounds(kp, bnd, table, n, n, T)
        blocks = dev32(np.full((T, h_kv, top), 777))
        ws = torch.empty(atf.atf_select_workspace_bytes(T, h_q, h_kv, T, bt, d), dtype=torch.uint8, device=DEV)
        atf.atf_select_blocks(q, bnd, blocks, table, pt, rows, pos, n, T, win, ws)
        o, lse = torch.empty_like(q), torch.empty((T, h_q), device=DEV)
        ws = torch.empty(atf.atf_attend_workspace_bytes(T, h_q, h_kv, top, bt, d), dtype=torch.uint8, device=DEV)
        atf.atf_attend_blocks(q, kp, vp, o, lse, table, rows, pos, n, blocks, bt, win, ws)
        torch.cuda.synchronize()
        got.append((kp[ids].cpu(), bnd[ids].cpu(), blocks.cpu(), o.cpu(), lse.cpu()))
        del kp, vp, bnd
    # (the third page's last tokens are nobody's)
    assert torch.equal(got[0][0][:2], got[1][0][:2]) and torch.equal(got[0][1][:2], got[1][1][:2])
    for x, y in zip(got[0][2:], got[1][2:]):
        assert torch.equal(x, y)


# ---- a serving step of all of them

class Engine:
    """What a user's program keeps: pools, bounds, table, lengths, and the buffers of a step."""

    def __init__(self, B=5, h_q=6, h_kv=2, d=64, pt=64, bt=32, width=12, pages=40, T=160, top=4, stream=None):
        import paper_2608_02947_amd as atf
        self.atf, self.pt, self.bt, self.B, self.T, self.top = atf, pt, bt, B, T, top
        z = lambda *s, dt=torch.int32: torch.zeros(s, dtype=dt, device=DEV)
        self.win, self.W = windows(d, "exact")
        self.h = (h_q, h_kv, d)
        self.table, self.free = z(B, width), torch.arange(pages, dtype=torch.int32, device=DEV)
        self.counts, self.n_k, self.n_new, self.starts = z(3), z(B), z(B), z(B + 1)
        self.counts[0] = pages
        self.slots, self.rows, self.pos = z(T, dt=torch.int64), z(T), z(T)
        self.kp, self.vp = z(*atf.kpages_shape(pages, pt, h_kv, d), dt=BF), z(*atf.vpages_shape(pages, pt, h_kv, d), dt=BF)
        self.bnd = z(*atf.bounds_shape(pages, pt, bt, h_kv, d), dt=BF)
        self.q, self.k, self.v = z(T, h_q, d, dt=BF), z(T, h_kv, d, dt=BF), z(T, h_kv, d, dt=BF)
        self.blocks, self.o, self.lse = z(T, h_kv, top), z(T, h_q, d, dt=BF), z(T, h_q, dt=torch.float32)
        self.most = width * pt
        u8 = lambda n: torch.empty(n, dtype=torch.uint8, device=DEV)
        self.ws = u8(atf.atf_select_workspace_bytes(T, h_q, h_kv, self.most, bt, d))
        self.ws2 = u8(atf.atf_attend_workspace_bytes(T, h_q, h_kv, top, bt, d))

    def step(self):
        a = self.atf
        a.atf_plan_pages(self.table, self.pt, self.free, self.counts, self.n_k, self.n_new, self.n_k, self.starts, self.slots,
                         self.rows, self.pos, self.counts)
        a.atf_cache_append_slots_rotated(self.k, self.v, self.kp, self.vp, self.slots, self.pos, self.win)
        a.atf_block_bounds(self.kp, self.bnd, self.table, self.n_k, self.n_new, self.T)
        a.atf_select_blocks(self.q, self.bnd, self.blocks, self.table, self.pt, self.rows, self.pos, self.n_k, self.most,
                            self.win, self.ws)
        a.atf_attend_blocks(self.q, self.kp, self.vp, self.o, self.lse, self.table, self.rows, self.pos, self.n_k, self.blocks,
                            self.bt, self.win, self.ws2)

    STEPS = [[70, 30, 0, 20, 33], [1, 1, 64, 1, 1], [1, 1, 1, -1, 0], [1, 40, 1, 90, 1], [-1, 1, 1, 1, 1], [150, 0, -1, 1, 1]]

    def feed(self, i):
        g = torch.Generator().manual_seed(i)
        for x in (self.q, self.k, self.v):
            x.copy_(torch.randn(x.shape, generator=g).to(BF))
        self.n_new.copy_(torch.tensor(self.STEPS[i], dtype=torch.int32))

    STATE = ("table", "free", "counts", "n_k", "starts", "slots", "rows", "pos", "kp", "vp", "bnd", "blocks", "o", "lse")

    def state(self):
        return {x: getattr(self, x).clone() for x in self.STATE}


def test_serving_steps_against_the_plain_forms():
    note("serving steps")
    e = Engine()
    free, table, n_k, count = e.free.cpu().numpy(), e.table.cpu().numpy(), np.zeros(e.B, dtype=int), 40
    h_q, h_kv, d = e.h
    bnd = to64(e.bnd)
    for i, new in enumerate(e.STEPS):
        e.feed(i)
        e.step()
        torch.cuda.synchronize()
        want = R.plan(table, e.pt, free, count, n_k, new, e.T)
        for name, mine in (("block_table", e.table), ("free_pages", e.free), ("n_k_out", e.n_k), ("row_starts", e.starts),
                           ("slots", e.slots), ("token_rows", e.rows), ("positions", e.pos), ("counts", e.counts)):
            assert np.array_equal(mine.cpu().numpy(), want[name]), (i, name)
        table, free, n_k, count = want["block_table"], want["free_pages"], want["n_k_out"], want["counts"][0]
        kp, vp, q = to64(e.kp), to64(e.vp), to64(e.q)
        bnd = R.bounds(kp, bnd, table, n_k, new, e.T, e.pt, e.bt)
        assert np.array_equal(to64(e.bnd), bnd)
        rows, pos = want["token_rows"], want["positions"]
        blocks = R.select(q, bnd, table, rows, pos, n_k, e.most, e.W, e.pt, e.bt, e.top, 1, 1, e.blocks.cpu().numpy().copy())
        assert np.array_equal(e.blocks.cpu().numpy(), blocks)
        wo, wl, _, size = R.attend(q, kp, vp, table, rows, pos, n_k, blocks, e.W, e.pt, e.bt, d ** -0.5)
        live = rows >= 0
        assert np.abs(to64(e.o) - wo)[live].max() <= 2.0 ** -7 * (np.abs(wo[live]).max() + 2)
        assert np.abs(to64(e.lse) - wl)[live].max() <= 1e-4


def test_serving_steps_captured():
    """A captured step replayed with other lengths, eager calls and synchronizations between the replays: the same
    bits as eager steps."""
    note("serving steps captured")
    eager, graphed = Engine(), Engine()
    want = []
    for i in range(len(Engine.STEPS)):
        eager.feed(i)
        eager.step()
        want.append(eager.state())
    torch.cuda.synchronize()
    begin = {x: getattr(graphed, x).clone() for x in Engine.STATE}
    graphed.feed(0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graphed.step()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step()
    for x, y in begin.items():
        getattr(graphed, x).copy_(y)
    for i, w in enumerate(want):
        graphed.feed(i)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in graphed.state().items():
            assert torch.equal(y.view(torch.uint8), w[x].view(torch.uint8)), (i, x)
        eager.step()  # work of the program's own between the replays


def test_two_streams_at_once():
    """The same calls on two streams, each with buffers and workspaces of its own."""
    note("two streams")
    one, two, ref = Engine(), Engine(), Engine()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for i in range(len(Engine.STEPS)):
        for e, s in zip((one, two), streams):
            with torch.cuda.stream(s):
                e.feed(i)
                e.step()
        ref.feed(i)
        ref.step()
    torch.cuda.synchronize()
    for x in Engine.STATE:
        for e in (one, two):
            assert torch.equal(getattr(e, x).view(torch.uint8), getattr(ref, x).view(torch.uint8)), x


def test_stream_argument_and_wrong_types():
    import paper_2608_02947_amd as atf
    note("stream argument")
    s = torch.cuda.Stream()
    p = PlanState(5, 6, 32, 50, 1, "fits")
    torch.cuda.synchronize()
    p.run(stream=s).check()
    with pytest.raises(ValueError, match="slots"):
        atf.atf_plan_pages(p.t["block_table"], 32, p.t["free_pages"], p.t["counts"], p.t["n_k"], p.t["n_new"], p.t["n_k_out"],
                           p.t["row_starts"], p.t["token_rows"], p.t["token_rows"], p.t["positions"], p.t["counts"])
    with pytest.raises(ValueError, match="n_new_rows"):
        atf.atf_plan_pages(p.t["block_table"], 32, p.t["free_pages"], p.t["counts"], p.t["n_k"], p.t["n_new"][:3], p.t["n_k_out"],
                           p.t["row_starts"], p.t["slots"], p.t["token_rows"], p.t["positions"], p.t["counts"])
