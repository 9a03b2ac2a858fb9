"""The operators over normed heads and 8-bit caches, as cases to be timed and compared: queries
and keys normed per head, turned to their positions and appended in one pass (bf16 caches), the
same append into caches quantised to 8 bits, reading those back into bf16 caches, and windowed
decode over them.

An 8-bit cache holds e4m3 numbers and, for every token of every KV head, one power of two (an
e8m0 byte) that all its numbers are multiplied by, for the keys and for the values.  The power is
the smallest 2^e, e in [-60, 119], with max |x| <= 448 * 2^e (2^-60 for a row of zeros).

`own` false: each operator in elementary torch operations, in 32 bits, rounded once at the end
(angles and window thresholds in 64).  `own` true: the calls of this package.  Head shapes, RoPE
bases and windows are those of the benchmark's workloads and of the tests.
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
EPS = 1e-6
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
EXP_MIN, EXP_MAX = -60, 119


def listed():
    return [
        # a decode step of a serving batch over pages: one new token a row, at each row's own
        # position; latency is what counts
        dict(name="normed_step_b16", op="normed", shape="gqa8", batch=16, n=1, cap=9000, norm=True,
             pages=64),
        # a whole long prompt entering the caches
        dict(name="normed_prompt_16k", op="normed", shape="llama3b", batch=1, n=16384, cap=40000,
             norm=True, pages=0),
        # a turn of some sessions of a small model, each at its own place, no length round
        dict(name="normed_turn_d64", op="normed", shape="qwen05b", batch=3, n=333, cap=5001,
             norm=True, pages=0),
        # a decode step of a large batch into 8-bit pages, one slot of it idle
        dict(name="q8_step_b64", op="append_q8", shape="llama3b", batch=64, n=1, cap=4100,
             norm=True, pages=64),
        # a chunk of a chunked prefill entering an 8-bit cache
        dict(name="q8_chunk_32k", op="append_q8", shape="qwen7b1m", batch=1, n=32768, cap=65536,
             norm=True, pages=0),
        # a turn of some sessions of a model without the norms, into 8-bit pages
        dict(name="q8_turn_d64", op="append_q8", shape="mha64", batch=5, n=777, cap=4001,
             norm=False, pages=32),
        # the pages of two sessions read back for their next prefill chunk
        dict(name="read_paged_5k", op="read_q8", shape="gqa8", batch=2, n=5003, cap=6000, pages=128),
        # a long session's cache read back whole
        dict(name="read_128k", op="read_q8", shape="qwen7b1m", batch=1, n=131072, cap=131072,
             pages=0),
        # one token against a short prompt's cache: latency and launches
        dict(name="decode_q8_1k", op="decode_q8", shape="qwen05b", batch=1, n=1000, cap=1000,
             window="exact", pages=0),
        # a batch of long contexts at the same length, with the variable-k profile
        dict(name="decode_q8_b8_32k", op="decode_q8", shape="llama3b", batch=8, n=32768, cap=32800,
             window="variable", pages=0),
        # a serving batch of requests of different lengths over pages, one slot without keys
        dict(name="decode_q8_paged_b24", op="decode_ragged_q8", shape="gqa20", batch=24, n=30011,
             cap=30011, window="exact", pages=64),
        # the longest context served
        dict(name="decode_q8_1m", op="decode_q8", shape="qwen7b1m", batch=1, n=1048576, cap=1048576,
             window="exact", pages=0),
    ]


MAX_KEYS = 2 ** 29  # bytes of the keys (or of the values) of an 8-bit cache: those of decode_q8_1m
MAX_NEW = 2.2e8     # elements that an append reads: about those of q8_chunk_32k
MAX_READ = 6.8e7    # elements of the keys that are read back: about those of read_128k


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["normed", "normed", "append_q8", "append_q8", "read_q8", "decode_q8",
                     "decode_q8", "decode_ragged_q8", "decode_ragged_q8"])
    shape = rng.choice(list(SHAPES))
    h_q, h_kv, d, _, _ = SHAPES[shape]
    c = dict(op=op, shape=shape, batch=1, n=1, cap=1)
    pages = rng.choice([0, 32, 64, 128, 256])
    if op in ("normed", "append_q8"):
        c["norm"] = rng.choice([True, True, False])
        if rng.random() < 0.4:
            c["batch"] = _log_int(rng, 1, 128)
        else:
            c["batch"], c["n"] = rng.choice([1, 1, 2, 3, 5]), _log_int(rng, 2, 32768)
        c["n"] = min(c["n"], max(1, int(MAX_NEW / (c["batch"] * (h_q + 2 * h_kv) * d))))
        c["cap"] = c["n"] + _log_int(rng, 16, 8000)
    elif op == "read_q8":
        c["batch"], c["n"] = rng.choice([1, 1, 2, 4]), _log_int(rng, 100, 131072)
        c["n"] = min(c["n"], int(MAX_READ / (c["batch"] * h_kv * d)))
        c["cap"] = c["n"] + rng.choice([0, rng.randint(1, 500)])
    else:
        c["window"] = rng.choice(["exact", "exact", "off", "variable", "rounded"])
        if op == "decode_q8":
            c["batch"], c["n"] = rng.choice([1, 1, 2, 3, 8, 16, 40]), _log_int(rng, 200, 400000)
            pages = 0
        else:
            c["batch"], c["n"] = _log_int(rng, 3, 40), _log_int(rng, 500, 60000)
        c["n"] = min(c["n"], MAX_KEYS // 2 // (c["batch"] * h_kv * d))
        c["cap"] = c["n"] + rng.choice([0, rng.randint(1, 100)])
    c["pages"] = pages
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


def _lengths(case):
    """Keys of each row of a ragged batch: the longest, a spread below it, and a slot without."""
    n, B = case["n"], case["batch"]
    i = torch.arange(B, dtype=torch.float64)
    lens = torch.clamp((n * torch.exp(-3.0 * ((7 * i) % B) / B)).long(), min=1)
    lens[B - 1] = 0
    return lens


def _positions(case):
    """First position of each row's new tokens; -1 for an idle slot of a decode step."""
    B, n, room = case["batch"], case["n"], case["cap"] - case["n"]
    pos = (room - (room * torch.arange(B, dtype=torch.int64) * 5 // (8 * B)))
    if n == 1 and B > 1:
        pos[B // 2] = -1
    return pos


# ---- the states

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


def _exponent(amax):
    """The power's exponent from the row's largest magnitude, int32."""
    m, e = torch.frexp(amax)  # amax = m 2^e, m in [0.5, 1); 448 = 0.875 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.clamp(torch.where(amax > 0, e, torch.full_like(e, EXP_MIN)), EXP_MIN, EXP_MAX)


def _pow2(e):
    """2^e in fp32 of int exponents in [-126, 127], from its bits."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _pow2_64(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _fill_q8(x, dims):
    """A cache of random numbers in 8 bits: (e4m3, exponents + 127 of the rows over `dims`)."""
    e = _exponent(x.abs().amax(dim=dims, keepdim=True))
    y = (x * _pow2(-e)).to(E4M3)
    return y, (e + 127).to(torch.uint8)


def _caches_q8(gen, lead, T, h_kv, d):
    """k [lead, h, d/16, T, 16], k_scale [lead, h, T16], v [lead, h, T16/16, d, 16], v_scale."""
    T16 = (T + 15) // 16 * 16
    sp = _spread(d).view(2, d // 16, 1, 8)
    k = _randn(gen, (lead, h_kv, d // 16, T, 16))
    k *= torch.cat([sp[0], sp[1]], dim=-1)
    k, ke = _fill_q8(k, (2, 4))
    ks = torch.full((lead, h_kv, T16), 127, dtype=torch.uint8, device="cuda")
    ks[:, :, :T] = ke.view(lead, h_kv, T)
    v, ve = _fill_q8(_randn(gen, (lead, h_kv, T16 // 16, d, 16)), (3,))
    return k, ks.view(E8M0), v, ve.reshape(lead, h_kv, T16).view(E8M0)


def _table(gen, need, width):
    """A block table of `need` pages a row out of a shuffled pool, and the pool's pages."""
    total = int(need.sum())
    order = torch.randperm(total, generator=gen, device="cuda")
    at = torch.arange(width, device="cuda")[None, :]
    first = (torch.cumsum(need, 0) - need).cuda()[:, None]
    idx = torch.where(at < need.cuda()[:, None], first + at, torch.zeros_like(at))
    return order[idx].to(torch.int32), total


def prepare(case, seed):
    h_q, h_kv, d, _, _ = SHAPES[case["shape"]]
    B, n, cap, pt, op = case["batch"], case["n"], case["cap"], case["pages"], case["op"]
    gen, bf = _gen(seed), torch.bfloat16
    s = {"case": case}
    lead, T = B, cap
    if pt:
        lens = _lengths(case) if op == "decode_ragged_q8" else torch.full((B,), cap)
        need = (lens + pt - 1) // pt
        s["table"], lead = _table(gen, need, int(need.max()))
        T = pt
    if op == "normed":
        sp = _spread(d).view(2, d // 16, 1, 8)
        s["k"] = (_randn(gen, (lead, h_kv, d // 16, T, 16)) * torch.cat([sp[0], sp[1]], dim=-1)).to(bf)
        s["v"] = _randn(gen, (lead, h_kv, (T + 15) // 16, d, 16)).to(bf)
    else:
        s["k"], s["k_scale"], s["v"], s["v_scale"] = _caches_q8(gen, lead, T, h_kv, d)
    if op in ("normed", "append_q8"):
        s["q"] = _randn(gen, (B, n, h_q, d)).to(bf)
        s["k_new"] = (_randn(gen, (B, n, h_kv, d)) * _spread(d)).to(bf)
        s["v_new"] = _randn(gen, (B, n, h_kv, d)).to(bf)
        s["q_out"] = torch.zeros_like(s["q"])
        s["pos"] = _positions(case).to(torch.int32).cuda()
        for w in ("q_weight", "k_weight"):
            s[w] = 1.0 + 0.2 * _randn(gen, (d,)) if case["norm"] else None
    elif op == "read_q8":
        s["k_out"] = torch.zeros((B, h_kv, d // 16, cap, 16), dtype=bf, device="cuda")
        s["v_out"] = torch.zeros((B, h_kv, (cap + 15) // 16, d, 16), dtype=bf, device="cuda")
    else:
        s["q"] = _randn(gen, (B, h_q, d)).to(bf)
        s["o"] = torch.empty((B, h_q, d), dtype=bf, device="cuda")
        s["lse"] = torch.empty((B, h_q), dtype=torch.float32, device="cuda")
        if op == "decode_ragged_q8":
            s["n_k_rows"] = _lengths(case).to(torch.int32).cuda()
            s["q_pos_rows"] = torch.clamp(s["n_k_rows"] - 1, min=0)
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ---- the framework's calls

def _kept(s):
    """What a user's program makes once: the window, and a decode's workspace."""
    import paper_2608_02947_amd as atf
    if "window" not in s:
        case = s["case"]
        h_q, h_kv, d, base, llama3 = SHAPES[case["shape"]]
        th = _theta(case).tolist() if llama3 else None
        kind = case.get("window", "off")
        if kind == "variable":
            s["window"] = atf.Window(d, base, 2.0, inv_freq=th, k_profile=_profile(case).tolist())
        else:
            s["window"] = atf.Window(d, base, math.inf if kind == "off" else 2.0, inv_freq=th,
                                     slice_pairs=8 if kind == "rounded" else 0)
        if case["op"].startswith("decode"):
            size = atf.atf_decode_workspace_bytes(case["batch"], h_q, h_kv, case["n"], d)
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return atf, s["window"]


def _run_own(s):
    atf, window = _kept(s)
    case = s["case"]
    op, n, paged = case["op"], case["n"], case["pages"] > 0
    if op == "normed":
        more = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, pos_rows=s["pos"])
        if paged:
            atf.atf_cache_append_paged_normed(s["q"], s["k_new"], s["v_new"], s["q_out"], s["k"], s["v"],
                                              s["table"], 0, window, **more)
        else:
            atf.atf_cache_append_normed(s["q"], s["k_new"], s["v_new"], s["q_out"], s["k"], s["v"], 0,
                                        window, **more)
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    if op == "append_q8":
        more = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, pos_rows=s["pos"])
        cache = (s["k"], s["k_scale"], s["v"], s["v_scale"])
        if paged:
            atf.atf_cache_append_paged_q8(s["q"], s["k_new"], s["v_new"], s["q_out"], *cache, s["table"],
                                          0, window, **more)
        else:
            atf.atf_cache_append_q8(s["q"], s["k_new"], s["v_new"], s["q_out"], *cache, 0, window, **more)
        return {"q": s["q_out"], "k": s["k"], "k_scale": s["k_scale"], "v": s["v"], "v_scale": s["v_scale"]}
    if op == "read_q8":
        if paged:
            atf.atf_cache_read_paged_q8(s["k"], s["k_scale"], s["v"], s["v_scale"], s["table"], s["k_out"],
                                        s["v_out"], n)
        else:
            atf.atf_cache_read_q8(s["k"], s["k_scale"], s["v"], s["v_scale"], s["k_out"], s["v_out"], n)
        return {"k": s["k_out"], "v": s["v_out"]}
    cache = (s["k"], s["k_scale"], s["v"], s["v_scale"])
    if op == "decode_q8":
        atf.atf_decode_q8(s["q"], *cache, s["o"], s["lse"], n - 1, window, s["workspace"], n_k=n)
    elif paged:
        atf.atf_decode_paged_q8(s["q"], *cache, s["o"], s["lse"], s["table"], s["n_k_rows"],
                                s["q_pos_rows"], n, window, s["workspace"])
    else:
        atf.atf_decode_ragged_q8(s["q"], *cache, s["o"], s["lse"], s["n_k_rows"], s["q_pos_rows"], n,
                                 window, s["workspace"])
    return {"o": s["o"], "lse": s["lse"]}


# ---- the plain forms

# slot 8h + 4a + b of a d-row of a bf16 V block holds token 8a + 4h + b
_SLOT = [8 * (t // 4 % 2) + 4 * (t // 8) + t % 4 for t in range(16)]
_TOKEN = [8 * (x // 4 % 2) + 4 * (x // 8) + x % 4 for x in range(16)]


def _normed(x, weight):
    """The RMS norm of each head's vector, x [..., d] fp32."""
    if weight is None:
        return x
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight


def _turned(x, cos, sin):
    """x [N, h, d] turned by the angles of cos and sin [N, 1, d/2]; pairs are (r, r + d/2)."""
    lo, hi = x.chunk(2, dim=-1)
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1)


def _append_plain(s):
    case = s["case"]
    _, h_kv, d, _, _ = SHAPES[case["shape"]]
    n, pt, q8 = case["n"], case["pages"], case["op"] == "append_q8"
    at = s["pos"].long()[:, None] + torch.arange(n, device="cuda")
    b, t = (s["pos"] >= 0)[:, None].expand(-1, n).nonzero(as_tuple=True)
    p = at[b, t]
    ang = p.double()[:, None, None] * _theta(case).cuda()
    cos, sin = ang.cos().float(), ang.sin().float()
    s["q_out"][b, t] = _turned(_normed(s["q"][b, t].float(), s["q_weight"]), cos, sin).to(torch.bfloat16)
    k = _turned(_normed(s["k_new"][b, t].float(), s["k_weight"]), cos, sin)
    v = s["v_new"][b, t].float()
    row, tok = (s["table"][b, p // pt].long(), p % pt) if pt else (b, p)
    if q8:
        kb, vb = s["k"].view(torch.uint8), s["v"].view(torch.uint8)
        ke, ve = _exponent(k.abs().amax(-1)), _exponent(v.abs().amax(-1))
        s["k_scale"].view(torch.uint8)[row, :, tok] = (ke + 127).to(torch.uint8)
        s["v_scale"].view(torch.uint8)[row, :, tok] = (ve + 127).to(torch.uint8)
        k = (k * _pow2(-ke)[..., None]).to(E4M3).view(torch.uint8)
        v = (v * _pow2(-ve)[..., None]).clamp(-448, 448).to(E4M3).view(torch.uint8)
        slot = tok % 16
    else:
        kb, vb = s["k"], s["v"]
        k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
        slot = torch.tensor(_SLOT, device="cuda")[tok % 16]
    kb[row, :, :, tok] = k.view(-1, h_kv, 2, d // 16, 8).transpose(2, 3).reshape(-1, h_kv, d // 16, 16)
    vb[row, :, tok // 16, :, slot] = v
    out = {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    return dict(out, k_scale=s["k_scale"], v_scale=s["v_scale"]) if q8 else out


def _gathered(s, name, rows):
    """A cache tensor's entries, those of a paged one in each row's order: [B, pages, ...]."""
    x = s[name].view(torch.uint8)
    return (x[rows] if rows is not None else x[:, None]), s[name].dtype


def _tokens(s, rows):
    """Keys and values as tokens [B, h, T, d], fp32, from the 8-bit caches."""
    _, h_kv, d, _, _ = SHAPES[s["case"]["shape"]]
    k, e4 = _gathered(s, "k", rows)
    B, P, _, nc, T, _ = k.shape
    k = k.view(e4).float().view(B, P, h_kv, nc, T, 2, 8).permute(0, 2, 1, 4, 5, 3, 6)
    v = _gathered(s, "v", rows)[0].view(e4).float().transpose(4, 5)
    v = v.reshape(B, P, h_kv, -1, d)[:, :, :, :T].transpose(1, 2)
    ks, vs = (_pow2(_gathered(s, x, rows)[0][..., :T].transpose(1, 2).int() - 127) for x in ("k_scale", "v_scale"))
    return ((k.reshape(B, h_kv, P * T, d) * ks.reshape(B, h_kv, P * T, 1)),
            (v.reshape(B, h_kv, P * T, d) * vs.reshape(B, h_kv, P * T, 1)))


def _read_plain(s):
    case = s["case"]
    _, h_kv, d, _, _ = SHAPES[case["shape"]]
    n, bf = case["n"], torch.bfloat16
    k, v = _tokens(s, s["table"].long() if case["pages"] else None)
    B = k.shape[0]
    s["k_out"][:, :, :, :n] = k[:, :, :n].view(B, h_kv, n, 2, d // 16, 8).permute(0, 1, 4, 2, 3, 5) \
        .reshape(B, h_kv, d // 16, n, 16).to(bf)
    whole = n // 16
    order = torch.tensor(_TOKEN, device="cuda")
    s["v_out"][:, :, :whole] = v[:, :, :16 * whole].view(B, h_kv, whole, 16, d)[:, :, :, order] \
        .transpose(3, 4).to(bf)
    rest = torch.tensor(_SLOT[:n % 16], dtype=torch.long, device="cuda")
    if n % 16:
        s["v_out"][:, :, whole, :, rest] = v[:, :, 16 * whole:n].transpose(2, 3).to(bf)
    return {"k": s["k_out"], "v": s["v_out"]}


def _decode_plain(s):
    case = s["case"]
    h_q, h_kv, d, _, _ = SHAPES[case["shape"]]
    B, n = case["batch"], case["n"]
    k, v = _tokens(s, s["table"].long() if case["pages"] else None)
    T = k.shape[2]
    lens = s["n_k_rows"].long() if "n_k_rows" in s else torch.full((B,), n, device="cuda")
    t = torch.arange(T, device="cuda")
    z = (lens - 1).clamp(min=0)[:, None] - t  # the query is at the last key
    keep = z[:, :, None] <= _thresholds(case).cuda()
    k = k * torch.cat([keep, keep], dim=-1)[:, None]
    q = s["q"].float().view(B, h_kv, h_q // h_kv, d).transpose(2, 3).contiguous()
    sc = torch.matmul(k, q).transpose(2, 3) / math.sqrt(d)  # [B, h, G, T]
    inside = (t < lens[:, None])[:, None, None]
    sc = sc.masked_fill(~inside, -math.inf)
    m = sc.amax(-1, keepdim=True)
    p = torch.exp(sc - torch.where(m == -math.inf, torch.zeros_like(m), m))
    l = p.sum(-1, keepdim=True)
    v = torch.where(inside[:, :, 0, :, None], v, torch.zeros_like(v))
    o = torch.matmul(p.contiguous(), v) / torch.where(l > 0, l, torch.ones_like(l))
    s["o"].copy_(o.view(B, h_q, d))
    s["lse"].copy_((m + torch.log(l)).view(B, h_q))
    return {"o": s["o"], "lse": s["lse"]}


def _run_plain(s):
    op = s["case"]["op"]
    if op in ("normed", "append_q8"):
        return _append_plain(s)
    return _read_plain(s) if op == "read_q8" else _decode_plain(s)


# ---- the work of one pass

def work(case):
    h_q, h_kv, d, _, _ = SHAPES[case["shape"]]
    B, n, op = case["batch"], case["n"], case["op"]
    if op in ("normed", "append_q8"):
        rows = int((_positions(case) >= 0).sum()) * n
        stored = 2 * d if op == "normed" else d + 1
        turned = rows * (h_q + h_kv) * d
        return {"bytes": float(rows * (4 * d * h_q + h_kv * (4 * d + 2 * stored))),
                "flops": (3.0 + 4.0 * case["norm"]) * turned + (0 if op == "normed" else 2.0 * rows * h_kv * 2 * d)}
    if op == "read_q8":
        return {"bytes": float(B * n * h_kv * 2 * (3 * d + 1)), "flops": float(B * n * h_kv * 2 * d)}
    lens = _lengths(case) if op == "decode_ragged_q8" else torch.full((B,), n)
    W = _thresholds(case)
    pairs = int(torch.minimum(lens[:, None], W[None, :] + 1).sum())  # kept (key, pair)s of a KV head
    keys = int(lens.sum())
    return {"bytes": float(h_kv * (2 * pairs + keys * (d + 2)) + B * h_q * (4 * d + 4)),
            "flops": float(h_q * (4 * pairs + 2 * d * keys))}


# ---- the same in 64 bits

def _turn64(x, p, theta):
    half = x.shape[-1] // 2
    a = p.double()[..., None, None] * theta
    re, im = x[..., :half], x[..., half:]
    return torch.cat([re * a.cos() - im * a.sin(), im * a.cos() + re * a.sin()], dim=-1)


def _e4m3_64(x):
    """x rounded to e4m3 numbers, ties to the even one; |x| <= 448."""
    _, e = torch.frexp(x)
    step = _pow2_64(torch.clamp(e - 1, min=-6) - 3)
    return torch.round(x / step) * step


def _quantised64(x):
    """(numbers, power of each row) of x [..., d] fp64."""
    top = x.abs().amax(-1)
    e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -200) / 448.0))
    e = torch.where(top * _pow2_64(1 - e) <= 448.0, e - 1, e)
    e = torch.where(top * _pow2_64(-e) > 448.0, e + 1, e).clamp(EXP_MIN, EXP_MAX)
    return _e4m3_64((x * _pow2_64(-e)[..., None]).clamp(-448, 448)), _pow2_64(e)


def _place(s, case, b, p):
    """(entry, token) of position p of row b in the caches."""
    if not case["pages"]:
        return b, p
    return int(s["table"][b, p // case["pages"]]), p % case["pages"]


def exact(case, seed):
    h_q, h_kv, d, _, _ = SHAPES[case["shape"]]
    B, n, cap, pt, op = case["batch"], case["n"], case["cap"], case["pages"], case["op"]
    G, half = h_q // h_kv, d // 2
    s = prepare(case, seed)
    theta = _theta(case).cuda()
    dims = torch.arange(d, device="cuda").view(2, d // 16, 8).transpose(0, 1).reshape(d // 16, 16)

    def norm64(x, w):
        x = x.double()
        return x if w is None else x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / d + EPS) * w.double()

    if op in ("normed", "append_q8"):
        names = ("k", "v") if op == "normed" else ("k", "k_scale", "v", "v_scale")
        out = {x: s[x].double() for x in names}
        out["q"] = s["q_out"].double()
        for b, first in enumerate(_positions(case).tolist()):
            if first < 0:
                continue
            pos = torch.arange(first, first + n, device="cuda")
            out["q"][b] = _turn64(norm64(s["q"][b], s["q_weight"]), pos, theta)
            k = _turn64(norm64(s["k_new"][b], s["k_weight"]), pos, theta)
            v = s["v_new"][b].double()
            if op == "append_q8":
                (k, kp), (v, vp) = _quantised64(k), _quantised64(v)
            i = 0
            while i < n:  # runs of tokens that lie in one 16-token block
                p = first + i
                w = min(16 - p % 16, n - i)
                e, t = _place(s, case, b, p)
                lane = torch.arange(t % 16, t % 16 + w)
                if op == "normed":
                    lane = 8 * (lane // 4 % 2) + 4 * (lane // 8) + lane % 4
                else:
                    out["k_scale"][e, :, t:t + w] = kp[i:i + w].t()
                    out["v_scale"][e, :, t:t + w] = vp[i:i + w].t()
                out["k"][e, :, :, t:t + w] = k[i:i + w].permute(1, 0, 2)[:, :, dims].permute(0, 2, 1, 3)
                out["v"][e, :, t // 16][:, :, lane.cuda()] = v[i:i + w].permute(1, 2, 0)
                i += w
        return out

    def tokens64(b, g, count):
        """Keys and values of row b, KV head g: [count, d] each."""
        ks, vs = [], []
        for p in range(0, max(count, 1), pt if pt else cap):
            e, _ = _place(s, case, b, p)
            k, v = s["k"][e, g].double(), s["v"][e, g].double()
            T = k.shape[1]
            x = torch.empty((T, d), dtype=torch.float64, device="cuda")
            x[:, dims.reshape(-1)] = k.permute(1, 0, 2).reshape(T, d)
            ks.append(x * s["k_scale"][e, g, :T].double()[:, None])
            v = v.transpose(1, 2).reshape(-1, d)
            vs.append((v * s["v_scale"][e, g].double()[:, None])[:T])
        return torch.cat(ks)[:count], torch.cat(vs)[:count]

    if op == "read_q8":
        out = {"k": s["k_out"].double(), "v": s["v_out"].double()}
        blocks, lane = n // 16, torch.arange(16)
        src = 8 * (lane // 4 % 2) + 4 * (lane // 8) + lane % 4  # the token of each slot
        for b in range(B):
            for g in range(h_kv):
                k, v = tokens64(b, g, n)
                out["k"][b, g, :, :n] = k[:, dims].permute(1, 0, 2)
                full = v[:16 * blocks].view(blocks, 16, d)[:, src.cuda()]
                out["v"][b, g, :blocks] = full.transpose(1, 2)
                for t in range(16 * blocks, n):
                    out["v"][b, g, blocks, :, int(src[t % 16])] = v[t]
        return out

    lens = _lengths(case).tolist() if op == "decode_ragged_q8" else [n] * B
    W = _thresholds(case).tolist()
    o = torch.zeros((B, h_q, d), dtype=torch.float64, device="cuda")
    lse = torch.full((B, h_q), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        for g in range(h_kv):
            if lens[b] == 0:
                continue
            k, v = tokens64(b, g, lens[b])
            for r in range(half):  # keys further than W[r] lose pair r
                far = max(0, lens[b] - 1 - W[r])
                k[:far, r] = 0.0
                k[:far, r + half] = 0.0
            a = (s["q"][b, g * G:(g + 1) * G].double() @ k.t().contiguous()) * d ** -0.5
            lse[b, g * G:(g + 1) * G] = torch.logsumexp(a, -1)
            o[b, g * G:(g + 1) * G] = torch.softmax(a, -1) @ v
    return {"o": o, "lse": lse}
