"""The operators of a serving step over pages whose attention is sparse, as cases to be timed and
compared: pages handed out and slots found from the requests' lengths, new tokens appended through
their slots, bounds of the keys of each block, the blocks that a query takes by those bounds, and
windowed attention over the blocks taken.

A block is `block` tokens of a row (token t is in block t / block); pages hold whole blocks.
Tokens of all rows are packed one behind the other; each has its row and its position, both -1 for
the padding at the end.

`own` false: each operator in elementary torch operations, in 32 bits, rounded once at the end
(angles, window thresholds and the blocks' scores, whose order is the result, in 64).  `own` true:
the calls of this package.  Head shapes, RoPE bases and windows are those of the benchmark's
workloads and of the tests.
"""
from __future__ import annotations

import math

import torch

own = False

# head shapes (query heads, KV heads, head dim, RoPE base, llama3 frequency scaling)
SHAPES = {
    "qwen05b": (14, 2, 64, 1e6, False),
    "llama3b": (24, 8, 128, 5e5, True),
    "qwen7b1m": (28, 4, 128, 1e7, False),
    "mha64": (16, 16, 64, 1e4, False),    # no sharing of KV heads
    "gqa8": (32, 4, 128, 1e6, False),     # a group of 8
    "gqa20": (40, 2, 128, 1e6, False),    # more heads to a KV head than a 16-column tile holds
}


def listed():
    return [
        # between two decode steps of a large serving batch: a token a row, some requests done, some
        # prompts coming in; latency is what counts
        dict(name="plan_step_b200", op="plan", batch=200, n=20000, new=1, pages=64),
        # a wave of long prompts admitted at once
        dict(name="plan_prompts_b24", op="plan", batch=24, n=5000, new=30011, pages=32),
        # the new token of every row of a decode step, keys already turned
        dict(name="slots_step_64", op="slots", shape="gqa8", batch=64, new=1, n=9000, pages=64, turn=False),
        # prompts of different lengths packed into one call, keys turned on the way
        dict(name="slots_prompts_20k", op="slots", shape="llama3b", batch=7, new=5003, n=2000, pages=64,
             turn=True),
        # the blocks that a decode step touched
        dict(name="bounds_step_64", op="bounds", shape="gqa8", batch=64, new=1, n=9000, pages=64, block=64),
        # the blocks of a long prompt
        dict(name="bounds_prompt_128k", op="bounds", shape="qwen7b1m", batch=1, new=131072, n=0, pages=128,
             block=64),
        # a token against the longest context served
        dict(name="select_1m", op="select", shape="qwen7b1m", batch=1, new=1, n=1048576, pages=64, block=64,
             top=64, window="exact"),
        # a decode step of requests of different lengths, one slot without keys
        dict(name="select_b24", op="select", shape="gqa20", batch=24, new=1, n=120011, pages=64, block=32,
             top=48, window="exact"),
        # a turn of three sessions: every token of it chooses blocks of its own
        dict(name="select_turn_3", op="select", shape="llama3b", batch=3, new=900, n=33000, pages=128,
             block=64, top=32, window="variable"),
        # a token of one request of a small model: latency and launches
        dict(name="attend_1", op="attend", shape="qwen05b", batch=1, new=1, n=20000, pages=32, block=32, top=16,
             window="exact"),
        # a decode step of a large batch
        dict(name="attend_b64", op="attend", shape="llama3b", batch=64, new=1, n=33000, pages=64, block=64,
             top=64, window="exact"),
        # a turn of three sessions
        dict(name="attend_turn_3", op="attend", shape="gqa8", batch=3, new=900, n=20011, pages=128, block=64,
             top=32, window="exact"),
    ]


MAX_SCORES = 1.1e9  # (token, query head, block, pair)s of a selection: about those of select_turn_3
MAX_KEYS = 1.5e9    # elements of the keys that the tokens attend: about those of attend_turn_3


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "slots", "bounds", "select", "select", "attend", "attend"])
    c = dict(op=op, pages=rng.choice([32, 64, 96, 128, 256]))
    if op == "plan":
        c["batch"], c["n"] = _log_int(rng, 1, 400), _log_int(rng, 20, 40000)
        c["new"] = rng.choice([1, _log_int(rng, 2, 50000)])
        c["new"] = max(1, min(c["new"], 700000 // c["batch"]))
        return c
    c["shape"] = rng.choice(list(SHAPES))
    h_q, h_kv, d, _, _ = SHAPES[c["shape"]]
    c["batch"], c["n"] = _log_int(rng, 1, 100), _log_int(rng, 50, 30000)
    c["new"] = rng.choice([1, 1, _log_int(rng, 2, 9000)])
    if op == "slots":
        c["new"] = max(1, min(c["new"], 20000 * 1024 // (c["batch"] * h_kv * d)))
        c["turn"] = rng.choice([False, True])
        return c
    if op == "bounds":
        c["block"] = rng.choice([b for b in (32, 64, 96, 128) if c["pages"] % b == 0])
        c["new"] = max(1, min(rng.choice([c["new"], 10 * c["new"]]), 131072 * 512 // (c["batch"] * h_kv * d)))
        return c
    c["block"] = rng.choice([b for b in (32, 64, 128) if c["pages"] % b == 0])
    c["top"] = _log_int(rng, 4, 128)
    c["window"] = rng.choice(["exact", "exact", "off", "variable", "rounded"])
    if rng.random() < 0.6:
        c["new"] = 1
    else:
        c["batch"], c["new"] = rng.choice([1, 1, 2, 3, 5]), _log_int(rng, 2, 900)
    T = c["batch"] * c["new"]
    if op == "select":
        if T < 20:
            c["n"] *= rng.choice([1, 10])
        c["n"] = max(1, min(c["n"], int(MAX_SCORES / (T * h_q * d / 2) * c["block"])))
    else:
        c["top"] = max(1, min(c["top"], int(MAX_KEYS / (T * h_kv * d * c["block"]))))
    return c


# ---- frequencies, thresholds, lengths

def _theta(case):
    """theta_r = base^(-2r/d), or the llama3 rule (factor 32, 1, 4, 8192) over it; fp64."""
    _, _, d, base, llama3 = SHAPES[case["shape"]]
    r = torch.arange(d // 2, dtype=torch.float64)
    th = torch.pow(torch.tensor(base, dtype=torch.float64), -2.0 * r / d)
    if not llama3:
        return th
    lam = 2.0 * math.pi / th
    s = (8192.0 / lam - 1.0) / 3.0
    mid = (1.0 - s) * th / 32.0 + s * th
    return torch.where(lam < 2048.0, th, torch.where(lam > 8192.0, th / 32.0, mid))


def _profile(case):
    half = SHAPES[case["shape"]][2] // 2
    return 16.0 - 14.0 * torch.arange(half, dtype=torch.float64) / (half - 1)


def _thresholds(case):
    """Pair r is kept at distance z iff z <= W[r]; int64 [d/2]."""
    th = _theta(case)
    if case["window"] == "off":
        return torch.full(th.shape, 2 ** 31 - 1, dtype=torch.int64)
    k = _profile(case) if case["window"] == "variable" else 2.0
    W = torch.clamp(torch.floor(k * (2.0 * math.pi / th)), max=2.0 ** 31 - 1).to(torch.int64)
    return W.view(-1, 8)[:, 7:].expand(-1, 8).reshape(-1) if case["window"] == "rounded" else W


def _spread_lengths(n, batch, seed):
    """Lengths of a batch: the longest first, a spread below it."""
    i = torch.arange(batch, dtype=torch.float64)
    return (n * torch.exp(-2.5 * ((7 * i + seed) % batch) / batch)).long()


def _rows(case):
    """(keys each row holds before the call, tokens it gets)."""
    B, new = case["batch"], case["new"]
    before, n_new = _spread_lengths(case["n"], B, 0), torch.clamp(_spread_lengths(new, B, 3), min=1)
    if case["op"] == "plan":
        b = torch.arange(B)
        if new == 1:  # a step: some requests end, some slots are idle, some prompts come in
            before[b % 11 == 7] = 0
            n_new[b % 11 == 7] = torch.clamp(_spread_lengths(900, B, 1), min=1)[b % 11 == 7]
            n_new[b % 13 == 5] = -1
        n_new[b % 17 == 9] = 0
    elif case["op"] in ("select", "attend"):
        before = torch.clamp(before - n_new, min=0)  # case["n"]: with the new ones
        if B > 1 and new == 1:
            before[B - 1] = n_new[B - 1] = 0
    return before, n_new


# ---- the states

def _most(case):
    """A bound on the rows' lengths."""
    return max(case["n"], case["new"])


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _spread(d):
    """Spread of the keys over the pairs: 0.5 at the highest frequency to 2 at the lowest."""
    sig = 0.5 + 1.5 * torch.arange(d // 2, dtype=torch.float32, device="cuda") / (d // 2 - 1)
    return torch.cat([sig, sig])


def _randn(gen, shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _table(gen, need, width, total):
    """A block table of `need` pages a row out of a shuffled pool, and the pool's other pages."""
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    at = torch.arange(width, device="cuda")[None, :]
    first = (torch.cumsum(need, 0) - need).cuda()[:, None]
    have = at < need.cuda()[:, None]
    table = torch.where(have, order[torch.where(have, first + at, torch.zeros_like(at))], torch.full_like(at, -1))
    return table.to(torch.int32), order[int(need.sum()):]


def _packed(before, n_new, pad):
    """Row and position of each packed token, -1 for the padding."""
    row = torch.repeat_interleave(torch.arange(len(n_new)), torch.clamp(n_new, min=0))
    first = torch.cumsum(torch.clamp(n_new, min=0), 0) - torch.clamp(n_new, min=0)
    pos = before[row] + torch.arange(len(row)) - first[row]
    end = torch.full((pad,), -1, dtype=torch.int64)
    return torch.cat([row, end]), torch.cat([pos, end])


def prepare(case, seed):
    B, pt, op, bf = case["batch"], case["pages"], case["op"], torch.bfloat16
    gen = _gen(seed)
    before, n_new = _rows(case)
    # which of the rows is how long goes by the seed
    shuffle = torch.randperm(B, generator=torch.Generator().manual_seed(int(seed)))
    before, n_new = before[shuffle], n_new[shuffle]
    after = before + torch.clamp(n_new, min=0)
    gpu32 = lambda x: x.to(torch.int32).cuda()
    s = {"case": case}
    if op == "plan":
        have, need = (before + pt - 1) // pt, (after + pt - 1) // pt
        width = int(need.max()) + 3
        total = int(need.sum()) + 50
        s["table"], rest = _table(gen, have, width, total)
        s["free_pages"] = torch.zeros(total, dtype=torch.int32, device="cuda")
        s["free_pages"][: len(rest)] = rest
        s["free_count"] = torch.tensor([len(rest)], dtype=torch.int32, device="cuda")
        s["n_k_rows"], s["n_new_rows"] = gpu32(before), gpu32(n_new)
        tokens = int(torch.clamp(n_new, min=0).sum())
        T = tokens + 37
        s["n_k_out"], s["row_starts"] = torch.zeros_like(s["n_k_rows"]), gpu32(torch.zeros(B + 1))
        s["counts"] = gpu32(torch.zeros(3))
        s["slots"] = torch.zeros(T, dtype=torch.int64, device="cuda")
        s["token_rows"], s["positions"] = gpu32(torch.zeros(T)), gpu32(torch.zeros(T))
        return s
    h_q, h_kv, d, _, _ = SHAPES[case["shape"]]
    need = (after + pt - 1) // pt
    width, total = max(1, int(need.max())), max(1, int(need.sum()))
    s["table"], _ = _table(gen, need, width, total)
    row, pos = _packed(before, n_new, 8 if op == "slots" else 0)
    s["token_rows"], s["positions"], s["n_k_rows"] = gpu32(row), gpu32(pos), gpu32(after)
    T = len(row)
    if op == "slots":
        page = s["table"][s["token_rows"].long().clamp(min=0), s["positions"].long().clamp(min=0) // pt].long()
        s["slots"] = torch.where(s["token_rows"] >= 0, page * pt + s["positions"] % pt, torch.full_like(page, -1))
        s["k_new"] = (_randn(gen, (T, h_kv, d)) * _spread(d)).to(bf)
        s["v_new"] = _randn(gen, (T, h_kv, d)).to(bf)
        s["k"] = torch.zeros((total, h_kv, d // 16, pt, 16), dtype=bf, device="cuda")
        s["v"] = torch.zeros((total, h_kv, pt // 16, d, 16), dtype=bf, device="cuda")
        return s
    sp = _spread(d).view(2, d // 16, 1, 8)
    chunks = torch.cat([sp[0], sp[1]], dim=-1)  # [d/16, 1, 16]
    if op in ("bounds", "attend"):
        s["k"] = (_randn(gen, (total, h_kv, d // 16, pt, 16)) * chunks).to(bf)
    bt = case["block"]
    if op == "bounds":
        s["n_new_rows"] = gpu32(n_new)
        s["bounds"] = torch.zeros((total, h_kv, pt // bt, d // 16, 2, 16), dtype=bf, device="cuda")
        return s
    s["q"] = _randn(gen, (T, h_q, d)).to(bf)
    if op == "select":
        # the middle and half the reach of a block's keys, which grows with the logarithm of their number
        shape = (total, h_kv, pt // bt, d // 16, 1, 16)
        mid = 0.3 * _randn(gen, shape) * chunks
        reach = (math.sqrt(2 * math.log(bt)) - 0.4 + 0.35 * _randn(gen, shape)).clamp(min=0.1) * chunks
        s["bounds"] = torch.cat([mid + reach, mid - reach], dim=-2).to(bf)
        s["blocks"] = torch.zeros((T, h_kv, case["top"]), dtype=torch.int32, device="cuda")
        return s
    s["v"] = _randn(gen, (total, h_kv, pt // 16, d, 16)).to(bf)
    # the blocks taken: the first, the newest, and others of those behind the query, -1 past their number
    blocks = torch.minimum(s["positions"], s["n_k_rows"][s["token_rows"].long()] - 1).long() // bt  # the newest
    most = width * pt // bt
    key = torch.rand((T, h_kv, most), generator=gen, device="cuda")
    j = torch.arange(most, device="cuda")
    key = torch.where(j == 0, torch.full_like(key, 2.0), key)
    key = torch.where(j == blocks[:, None, None], torch.full_like(key, 3.0), key)
    key = key.masked_fill(j > blocks[:, None, None], -1.0)
    if most < case["top"]:
        key = torch.cat([key, key.new_full((T, h_kv, case["top"] - most), -1.0)], dim=-1)
    val, at = torch.topk(key, case["top"], dim=-1)
    at = torch.where(val >= 0, at, torch.full_like(at, 2 ** 30)).sort(dim=-1).values
    s["blocks"] = torch.where(at < 2 ** 30, at, torch.full_like(at, -1)).to(torch.int32)
    s["o"] = torch.zeros((T, h_q, d), dtype=bf, device="cuda")
    s["lse"] = torch.zeros((T, h_q), dtype=torch.float32, device="cuda")
    return s


FIRST, LAST = 1, 2  # blocks that every selection takes: the row's first, the newest


def run(s):
    return _run_own(s) if own else PLAIN[s["case"]["op"]](s)


# ---- the framework's calls

def _kept(s):
    """What a user's program makes once: the window, and the workspaces."""
    import paper_2608_02947_amd as atf
    case = s["case"]
    if "kept" not in s:
        s["kept"] = True
        op = case["op"]
        if op != "plan":
            h_q, h_kv, d, base, llama3 = SHAPES[case["shape"]]
            th = _theta(case).tolist() if llama3 else None
            kind = case.get("window", "off")
            if kind == "variable":
                s["window"] = atf.Window(d, base, 2.0, inv_freq=th, k_profile=_profile(case).tolist())
            else:
                s["window"] = atf.Window(d, base, math.inf if kind == "off" else 2.0, inv_freq=th,
                                         slice_pairs=8 if kind == "rounded" else 0)
        size = 0
        if op == "select":
            size = atf.atf_select_workspace_bytes(s["q"].shape[0], h_q, h_kv, _most(case), case["block"], d)
        elif op == "attend":
            size = atf.atf_attend_workspace_bytes(s["q"].shape[0], h_q, h_kv, case["top"], case["block"], d)
        if size:
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return atf


def _run_own(s):
    atf = _kept(s)
    case = s["case"]
    op = case["op"]
    if op == "plan":
        atf.atf_plan_pages(s["table"], case["pages"], s["free_pages"], s["free_count"], s["n_k_rows"],
                           s["n_new_rows"], s["n_k_out"], s["row_starts"], s["slots"], s["token_rows"],
                           s["positions"], s["counts"])
        return {x: s[x] for x in ("table", "free_pages", "n_k_out", "row_starts", "slots", "token_rows",
                                  "positions", "counts")}
    if op == "slots":
        if case["turn"]:
            atf.atf_cache_append_slots_rotated(s["k_new"], s["v_new"], s["k"], s["v"], s["slots"],
                                               s["positions"], s["window"])
        else:
            atf.atf_cache_append_slots(s["k_new"], s["v_new"], s["k"], s["v"], s["slots"])
        return {"k": s["k"], "v": s["v"]}
    if op == "bounds":
        atf.atf_block_bounds(s["k"], s["bounds"], s["table"], s["n_k_rows"], s["n_new_rows"], case["new"])
        return {"bounds": s["bounds"]}
    if op == "select":
        atf.atf_select_blocks(s["q"], s["bounds"], s["blocks"], s["table"], case["pages"], s["token_rows"],
                              s["positions"], s["n_k_rows"], _most(case), s["window"], s["workspace"],
                              first_blocks=min(FIRST, case["top"]), last_blocks=min(LAST, case["top"] - 1))
        return {"blocks": s["blocks"]}
    atf.atf_attend_blocks(s["q"], s["k"], s["v"], s["o"], s["lse"], s["table"], s["token_rows"],
                          s["positions"], s["n_k_rows"], s["blocks"], case["block"], s["window"],
                          s["workspace"])
    return {"o": s["o"], "lse": s["lse"]}


# ---- the plain forms

def _plan_plain(s):
    pt, table, free = s["case"]["pages"], s["table"], s["free_pages"]
    B, width = table.shape
    T = s["slots"].shape[0]
    n = s["n_k_rows"].long().clamp(0, width * pt)
    new = s["n_new_rows"].long()
    grow = new.clamp(min=0)
    ends = torch.cumsum(grow, 0)
    have = (n + pt - 1) // pt
    fits = n + grow <= width * pt
    need = torch.where(fits, (n + grow + pt - 1) // pt - have, torch.zeros_like(n))
    back = torch.where(new < 0, have, torch.zeros_like(n))
    at = torch.arange(width, device="cuda")
    # pages of the rows that end go on top of the free ones, rows and pages in order
    f0 = s["free_count"][0].long()
    first = f0 + torch.cumsum(back, 0) - back
    b, i = (at < back[:, None]).nonzero(as_tuple=True)
    free[first[b] + i] = table[b, i]
    f1 = f0 + back.sum()
    # rows that grow take them from the top, until one finds too few
    take_end = torch.cumsum(need, 0)
    ok = fits & (take_end <= f1) & (ends <= T)
    taken = torch.where(ok, need, torch.zeros_like(need))
    b, i = (at < taken[:, None]).nonzero(as_tuple=True)
    table[b, have[b] + i] = free[f1 - 1 - (take_end - need)[b] - i]
    s["n_k_out"].copy_(torch.where(new < 0, torch.zeros_like(n), torch.where(ok, n + grow, n)))
    s["row_starts"].copy_(torch.cat([torch.zeros_like(ends[:1]), ends]).clamp(max=T))
    s["counts"].copy_(torch.stack([f1 - taken.sum(), ends[-1].clamp(max=T), ((grow > 0) & ~ok).sum()]))
    t = torch.arange(T, device="cuda")
    row = torch.searchsorted(ends, t, right=True).clamp(max=B - 1)
    inside = (t < ends[-1]) & ok[row]
    pos = n[row] + t - (ends - grow)[row]
    page = table[row, (pos // pt).clamp(0, width - 1)].long()
    none = torch.full_like(t, -1)
    s["slots"].copy_(torch.where(inside, page * pt + pos % pt, none))
    s["token_rows"].copy_(torch.where(inside, row, none))
    s["positions"].copy_(torch.where(inside, pos, none))
    return {x: s[x] for x in ("table", "free_pages", "n_k_out", "row_starts", "slots", "token_rows", "positions",
                              "counts")}


# slot 8h + 4a + b of a d-row of a V block holds token 8a + 4h + b
_SLOT = [8 * (t // 4 % 2) + 4 * (t // 8) + t % 4 for t in range(16)]


def _slots_plain(s):
    case = s["case"]
    _, h_kv, d, _, _ = SHAPES[case["shape"]]
    pt = case["pages"]
    t = (s["slots"] >= 0).nonzero()[:, 0]
    k = s["k_new"][t]
    if case["turn"]:
        ang = s["positions"][t].double()[:, None, None] * _theta(case).cuda()
        cos, sin = ang.cos().float(), ang.sin().float()
        lo, hi = k.float().chunk(2, dim=-1)
        k = torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1).to(torch.bfloat16)
    page, tok = s["slots"][t] // pt, s["slots"][t] % pt
    s["k"][page, :, :, tok] = k.view(-1, h_kv, 2, d // 16, 8).transpose(2, 3).reshape(-1, h_kv, d // 16, 16)
    s["v"][page, :, tok // 16, :, torch.tensor(_SLOT, device="cuda")[tok % 16]] = s["v_new"][t]
    return {"k": s["k"], "v": s["v"]}


def _bounds_plain(s):
    case = s["case"]
    pt, bt = case["pages"], case["block"]
    n, new = s["n_k_rows"].long(), s["n_new_rows"].long()
    blocks = torch.arange(s["table"].shape[1] * pt // bt, device="cuda")
    touched = (blocks * bt < n[:, None]) & (blocks >= ((n - new) // bt)[:, None]) & (new > 0)[:, None]
    b, j = touched.nonzero(as_tuple=True)
    page, part = s["table"][b, j // (pt // bt)].long(), j % (pt // bt)
    _, h_kv, nc, _, _ = s["k"].shape
    k = s["k"].view(-1, h_kv, nc, pt // bt, bt, 16)[page, :, :, part].float()  # [N, h, d/16, bt, 16]
    out = ((j * bt)[:, None] + torch.arange(bt, device="cuda") >= n[b][:, None])[:, None, None, :, None]
    s["bounds"][page, :, part] = torch.stack([k.masked_fill(out, -math.inf).amax(3),
                                              k.masked_fill(out, math.inf).amin(3)], dim=3).to(torch.bfloat16)
    return {"bounds": s["bounds"]}


def _slabs(T, each):
    """Tokens in slabs of about 2^27 elements."""
    step = max(1, 2 ** 27 // max(1, each))
    return [slice(t, min(T, t + step)) for t in range(0, T, step)]


def _last_key(s, t):
    """(row, position, last key of it that it reaches) of the tokens t."""
    row, pos = s["token_rows"][t].long(), s["positions"][t].long()
    return row, pos, torch.minimum(pos, s["n_k_rows"][row].long() - 1)


def _select_plain(s):
    case = s["case"]
    h_q, h_kv, d, _, _ = SHAPES[case["shape"]]
    G, half, pt, bt, top = h_q // h_kv, d // 2, case["pages"], case["block"], case["top"]
    per = pt // bt
    most = s["table"].shape[1] * per
    W = _thresholds(case).cuda()
    j = torch.arange(most, device="cuda")
    pos, neg = s["q"].double().clamp(min=0), s["q"].double().clamp(max=0)
    for t in _slabs(s["q"].shape[0], most * h_q * half):
        row, p, last = _last_key(s, t)
        bounds = s["bounds"][s["table"][row].long()].double()  # [S, P, h, per, d/16, 2, 16]
        bounds = bounds.transpose(2, 3).reshape(len(row), most, h_kv, d // 16, 2, 2, 8)
        hi, lo = (bounds[:, :, :, :, x].transpose(3, 4).reshape(len(row), most, h_kv, 1, 2, half) for x in (0, 1))
        qs = (len(row), 1, h_kv, G, 2, half)
        u = (pos[t].view(qs) * hi + neg[t].view(qs) * lo).sum(-2)  # [S, n, h, G, d/2]
        near = p[:, None] - torch.minimum((j + 1) * bt - 1, last[:, None])
        far = p[:, None] - j * bt
        part = (W >= near[..., None]) & (W < far[..., None])
        u = torch.where(part[:, :, None, None], u.clamp(min=0), u)
        u = u * (W >= near[..., None])[:, :, None, None]
        score = u.sum(-1).amax(-1).transpose(1, 2)  # [S, h, n]
        newest = (last // bt)[:, None, None]
        first, newer = min(FIRST, top), min(LAST, top - 1)
        score = score.masked_fill((j < first) | (j > newest - newer), math.inf)
        score = score.masked_fill((j * bt > last[:, None])[:, None], -math.inf)
        if most < top:
            score = torch.cat([score, score.new_full((len(row), h_kv, top - most), -math.inf)], dim=-1)
        score, at = torch.sort(score, dim=-1, descending=True, stable=True)
        at = at[..., :top].masked_fill(score[..., :top] == -math.inf, 2 ** 30).sort(dim=-1).values
        s["blocks"][t] = torch.where(at < 2 ** 30, at, torch.full_like(at, -1)).to(torch.int32)
    return {"blocks": s["blocks"]}


def _attend_plain(s):
    case = s["case"]
    h_q, h_kv, d, _, _ = SHAPES[case["shape"]]
    G, pt, bt, top = h_q // h_kv, case["pages"], case["block"], case["top"]
    W = _thresholds(case).cuda()
    slot = torch.tensor(_SLOT, device="cuda")
    head = torch.arange(h_kv, device="cuda")[None, :, None]
    for t in _slabs(s["q"].shape[0], h_kv * top * bt * d):
        row, p, last = _last_key(s, t)
        S = len(row)
        blocks = s["blocks"][t].long()
        key = (blocks[..., None] * bt + torch.arange(bt, device="cuda")).view(S, h_kv, top * bt)
        ok = (key >= 0) & (key <= last[:, None, None])
        key = torch.where(ok, key, torch.zeros_like(key))
        page = s["table"][row[:, None, None], key // pt].long().clamp(min=0)
        tok = key % pt
        k = s["k"][page, head, :, tok].float().view(S, h_kv, top * bt, d // 16, 2, 8)
        k = k.transpose(3, 4).reshape(S, h_kv, top * bt, 2, d // 2)
        k = k * ((p[:, None, None] - key)[..., None] <= W)[..., None, :]
        q = s["q"][t].float().view(S, h_kv, G, d).transpose(2, 3).contiguous()
        sc = torch.matmul(k.reshape(S, h_kv, top * bt, d), q).transpose(2, 3) / math.sqrt(d)
        sc = sc.masked_fill(~ok[:, :, None], -math.inf)
        m = sc.amax(-1, keepdim=True)
        x = torch.exp(sc - torch.where(m == -math.inf, torch.zeros_like(m), m))
        l = x.sum(-1, keepdim=True)
        v = s["v"][page, head, tok // 16, :, slot[tok % 16]].float() * ok[..., None]
        o = torch.matmul(x.contiguous(), v) / torch.where(l > 0, l, torch.ones_like(l))
        s["o"][t] = o.view(S, h_q, d).to(torch.bfloat16)
        s["lse"][t] = (m + torch.log(l)).view(S, h_q)
    return {"o": s["o"], "lse": s["lse"]}


PLAIN = {"plan": _plan_plain, "slots": _slots_plain, "bounds": _bounds_plain, "select": _select_plain,
         "attend": _attend_plain}


# ---- the work of one pass

def work(case):
    op = case["op"]
    before, n_new = _rows(case)
    grow = torch.clamp(n_new, min=0)
    after = before + grow
    tokens, pt = int(grow.sum()), case["pages"]
    if op == "plan":
        pages = int(((after + pt - 1) // pt - (before + pt - 1) // pt).sum())
        back = int(((before + pt - 1) // pt)[n_new < 0].sum())
        return {"bytes": float(16 * len(before) + 8 * (pages + back) + 16 * (tokens + 37)),
                "flops": float(4 * tokens)}
    h_q, h_kv, d, _, _ = SHAPES[case["shape"]]
    if op == "slots":
        return {"bytes": float(tokens * (8 * h_kv * d + 8)), "flops": float(3 * tokens * h_kv * d)}
    bt = case["block"]
    if op == "bounds":
        first = (after - grow) // bt
        keys = int((after - first * bt)[grow > 0].sum())
        blocks = int(((after + bt - 1) // bt - first)[grow > 0].sum())
        return {"bytes": float(h_kv * d * (2 * keys + 4 * blocks)), "flops": float(2 * keys * h_kv * d)}
    row, pos = _packed(before, n_new, 0)
    last = torch.minimum(pos, after[row] - 1)
    W, newest, T = _thresholds(case), last // bt, len(row)
    if op == "select":
        # a pair of a block is in the window up to the block that holds the key W back
        blocks = newest + 1
        first = torch.clamp(pos[:, None] - W[None, :], min=0) // bt
        pairs = torch.clamp(newest[:, None] + 1 - first, min=0)
        # the bounds of a row's blocks are read once for all of its tokens
        per_row = torch.zeros(len(after), dtype=torch.int64)
        per_row = per_row.scatter_reduce(0, row, pairs.sum(1), "amax")
        return {"bytes": float(8 * h_kv * int(per_row.sum()) + 2 * T * h_q * d + 4 * T * h_kv * case["top"]),
                "flops": float(4 * h_q * int(pairs.sum()))}
    # the blocks attended lie anywhere behind the query: their share of the pairs is the whole's
    keys = torch.minimum(last + 1, torch.tensor(case["top"] * bt))
    share = torch.minimum(last[:, None] + 1, W[None, :] + 1).sum(1) / torch.clamp(last + 1, min=1)
    pairs = float((keys * share).sum())
    # what a turn's tokens share of a row's cache is read once
    per = torch.zeros(len(after), dtype=torch.float64)
    per = per.scatter_add(0, row, keys.double())
    cached = torch.minimum(per, after.double())
    pair_bytes = 4.0 * pairs * float(cached.sum()) / max(1.0, float(per.sum()))
    return {"bytes": h_kv * (pair_bytes + 2.0 * d * float(cached.sum()) + 4.0 * T * case["top"]) +
            T * h_q * (4.0 * d + 4),
            "flops": h_q * (4.0 * pairs + 2.0 * d * float(keys.sum()))}


# ---- the same in 64 bits

def _exact_plan(s):
    pt, (B, width), T = s["case"]["pages"], s["table"].shape, s["slots"].shape[0]
    table, free = s["table"].tolist(), s["free_pages"].tolist()
    n_k, new, top = s["n_k_rows"].tolist(), s["n_new_rows"].tolist(), int(s["free_count"])
    for b in range(B):
        if new[b] < 0:
            for page in table[b][: -(-n_k[b] // pt)]:
                free[top] = page
                top += 1
    starts, tokens, full, refused, out = [0], [], False, 0, list(n_k)
    stack = free[:top]
    for b in range(B):
        more = max(new[b], 0)
        if new[b] < 0:
            out[b] = 0
        fits = n_k[b] + more <= width * pt
        need = -(-(n_k[b] + more) // pt) - -(-n_k[b] // pt) if fits else 0
        full = full or need > len(stack) or starts[-1] + more > T
        if more and fits and not full:
            for i in range(need):
                table[b][-(-n_k[b] // pt) + i] = stack.pop()
            out[b] += more
            tokens += [(table[b][p // pt] * pt + p % pt, b, p) for p in range(n_k[b], n_k[b] + more)]
        elif more:
            refused += 1
            tokens += [(-1, -1, -1)] * more
        starts.append(min(starts[-1] + more, T))
    tokens = (tokens + [(-1, -1, -1)] * T)[:T]
    tensor = lambda x: torch.tensor(x, dtype=torch.float64, device="cuda")
    slots, rows, positions = zip(*tokens)
    return {"table": tensor(table), "free_pages": tensor(free), "n_k_out": tensor(out),
            "row_starts": tensor(starts), "slots": tensor(slots), "token_rows": tensor(rows),
            "positions": tensor(positions), "counts": tensor([len(stack), starts[-1], refused])}


def _exact_slots(s):
    case = s["case"]
    _, h_kv, d, _, _ = SHAPES[case["shape"]]
    pt, half = case["pages"], d // 2
    out = {"k": s["k"].double(), "v": s["v"].double()}
    k, slots = s["k_new"].double(), s["slots"]
    if case["turn"]:
        z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                        s["positions"].double()[:, None, None] * _theta(case).cuda())
        z = torch.complex(k[..., :half], k[..., half:]) * z
        k = torch.cat([z.real, z.imag], dim=-1)
    dims = torch.arange(d, device="cuda").view(2, d // 16, 8).transpose(0, 1).reshape(d // 16, 16)
    t = torch.arange(len(slots), device="cuda")[slots >= 0]
    for tok in range(pt):  # the tokens that lie at one place of their pages
        at = t[slots[t] % pt == tok]
        page = torch.div(slots[at], pt, rounding_mode="floor")
        x = tok % 16
        x = 8 * (x // 4 % 2) + 4 * (x // 8) + x % 4
        out["k"][:, :, :, tok].index_copy_(0, page, k[at][:, :, dims])
        out["v"][:, :, tok // 16, :, x].index_copy_(0, page, s["v_new"][at].double())
    return out


def _exact_bounds(s):
    case = s["case"]
    pt, bt = case["pages"], case["block"]
    out = s["bounds"].double()
    for b, (n, new) in enumerate(zip(s["n_k_rows"].tolist(), s["n_new_rows"].tolist())):
        first = (n - new) // bt * bt
        for t in range(first, n, bt):
            page, off = int(s["table"][b, t // pt]), t % pt
            k = s["k"][page, :, :, off: off + min(bt, n - t)].double()
            out[page, :, off // bt, :, 0], out[page, :, off // bt, :, 1] = k.max(2).values, k.min(2).values
    return {"bounds": out}


def _dims(x):
    """[..., d/16, 16] of a cache as [..., d]."""
    return torch.cat([x[..., :8].flatten(-2), x[..., 8:].flatten(-2)], dim=-1)


def _exact_select(s):
    case = s["case"]
    h_q, h_kv, d, _, _ = SHAPES[case["shape"]]
    G, half, pt, bt, top = h_q // h_kv, d // 2, case["pages"], case["block"], case["top"]
    W = _thresholds(case).cuda()
    out = torch.full(s["blocks"].shape, -1, dtype=torch.float64, device="cuda")
    kept, n_k = {}, s["n_k_rows"].tolist()
    for t, (b, p) in enumerate(zip(s["token_rows"].tolist(), s["positions"].tolist())):
        last = min(p, n_k[b] - 1)
        if last < 0:
            continue
        n = last // bt + 1
        if b not in kept:
            pages = s["table"][b, : -(-n_k[b] // pt)].long()
            both = s["bounds"][pages].double().transpose(1, 2).flatten(0, 1)  # [blocks, h, d/16, 2, 16]
            kept = {b: (_dims(both[:, :, :, 0]), _dims(both[:, :, :, 1]))}
        hi, lo = (x[:n] for x in kept[b])
        j = torch.arange(n, device="cuda")
        near, far = (p - (j * bt + bt - 1).clamp(max=last))[:, None], (p - j * bt)[:, None]
        best = None
        for i in range(G):
            q = s["q"][t, i::G].double()  # head i of every group
            u = torch.where(q > 0, q * hi, q * lo)
            u = u[..., :half] + u[..., half:]
            u = torch.where((W >= far)[:, None], u, torch.where((W >= near)[:, None], u.clamp(min=0), 0.0 * u))
            u = u.sum(-1)
            best = u if best is None else torch.maximum(best, u)
        best[: min(FIRST, top)] = math.inf
        best[max(0, n - min(LAST, top - 1)):] = math.inf
        order = torch.argsort(best, dim=0, descending=True, stable=True)[:top]  # [<= top, h]
        out[t, :, : len(order)] = order.sort(dim=0).values.t().double()
    return {"blocks": out}


def _exact_attend(s):
    case = s["case"]
    h_q, h_kv, d, _, _ = SHAPES[case["shape"]]
    G, half, pt, bt = h_q // h_kv, d // 2, case["pages"], case["block"]
    W = _thresholds(case).cuda()
    T = s["q"].shape[0]
    o = torch.zeros((T, h_q, d), dtype=torch.float64, device="cuda")
    lse = torch.full((T, h_q), -math.inf, dtype=torch.float64, device="cuda")
    n_k, kept = s["n_k_rows"].tolist(), {}
    lane = torch.arange(16, device="cuda")
    lane = 8 * (lane // 4 % 2) + 4 * (lane // 8) + lane % 4
    for t, (b, p) in enumerate(zip(s["token_rows"].tolist(), s["positions"].tolist())):
        last = min(p, n_k[b] - 1)
        if last < 0:
            continue
        if b not in kept:  # the row's keys and values in order, [h, tokens, d]
            pages = s["table"][b, : -(-n_k[b] // pt)].long()
            k = _dims(s["k"][pages].permute(1, 0, 3, 2, 4)).flatten(1, 2)
            v = s["v"][pages][..., lane].permute(1, 0, 2, 4, 3).flatten(1, 3)
            kept = {b: (k, v)}
        k, v = kept[b]
        j = s["blocks"][t].long()  # [h, top]
        j = torch.where(j < 0, torch.full_like(j, last // bt + 1), j)
        key = (j[..., None] * bt + torch.arange(bt, device="cuda")).flatten(1)
        out = key > last
        key = key.clamp(max=last)[..., None].expand(-1, -1, d)
        x = torch.gather(k, 1, key).double()
        x[torch.cat([p - key[..., :half] > W] * 2, dim=-1)] = 0.0
        q = s["q"][t].double().view(h_kv, G, d) * d ** -0.5
        a = torch.bmm(q, x.transpose(1, 2).contiguous()).masked_fill(out[:, None], -math.inf)
        lse[t] = torch.logsumexp(a, -1).flatten()
        o[t] = torch.bmm(torch.softmax(a, -1), torch.gather(v, 1, key).double()).view(h_q, d)
    return {"o": o, "lse": lse}


EXACT = {"plan": _exact_plan, "slots": _exact_slots, "bounds": _exact_bounds, "select": _exact_select,
         "attend": _exact_attend}


def exact(case, seed):
    return EXACT[case["op"]](prepare(case, seed))
