// Windowed single-token decode over 8-bit caches (q8.hpp), gfx950: decode.hip's split-KV decode
// with the keys and values read as e4m3 numbers and widened to bf16 in registers.
//
// Caches (append_normed.hip writes them):
//   K [B][h_kv][d/16][cache_tokens][16]: chunk c of a token is 16 bytes, pairs 8c .. 8c + 7,
//     first components then second; a power per token, k_scale [B][h_kv][ceil16(cache_tokens)]
//   V [B][h_kv][ceil(cache_tokens/16)][d][16]: 16-token blocks, dim-major, tokens in order; a
//     power per token, v_scale
//
// The heads of one KV head (up to 32 a workgroup) are the columns of v_mfma_f32_16x16x32_bf16, in
// one or two tiles, a wave's block is 64 tokens, and every load of K and V is 16 bytes a lane.
// With r = lane % 16, g = lane / 16:
//   scores, tile s = 0 .. 3: A row r is token 16 (r / 4) + 4 s + r % 4, the lane's 16 bytes chunk
//     4 m + g of it: its two halves are two operands of 8 dims, for two products.  The result
//     gives the lane, for head r, tokens 16 g + 4 s + v.
//   values: the lane's 16 bytes are the 16 tokens of block g for dim 16 i + r: two operands of 8
//     tokens.  The tokens 16 g .. 16 g + 15 it needs probabilities of are those it has scores of.
// A key's power is part of its conversion (v_cvt_scalef32_pk_bf16_fp8); a value's, which differs
// along the product's sum, goes into its probability after the normaliser has taken it.
//
// A pair is kept at distance z iff z <= W_r.  Per block, two ballots give the pairs kept at some
// token and at every token: chunks without a kept pair are read from a line of zeros, queries
// lose the pairs kept nowhere, and so do the keys in chunks that hold others (a number that is none
// must not count there: 0.5 to 1 % of long rows' time); where a window ends inside the block the
// keys' bytes are masked lane by lane.
//
// Bound by HBM reads where rows are long or many: one row of 1,048,576 keys, 28/4 heads of 128 (734 MB
// of kept pairs and values) 142 us, 5.2 TB/s; 8 rows of 32,768, 24/8 heads, 433 MB in 85 (a streaming
// read reaches 5.57).  24 rows up to 30,011 of 40/2 heads, 97 MB, take 33: the first block is there
// after 10.6 us and the merge ends 7 after the last.  64 tokens a wave make the values' 16 tokens of a
// lane a block of the cache and the keys' powers 16 bytes a lane.  2 waves a SIMD: a block's
// operands, the next ones in flight, and the outputs take 208 (d = 128, one tile) to 230 registers; 4 at
// d = 64 with one tile (128 registers).
#include "atf_internal.hpp"
#include "q8.hpp"

namespace atf {

__host__ __device__ int32_t decode_q8_first(int32_t t_begin, int32_t t_end, int32_t wave) {
    return t_end - t_begin > 64 * wave ? t_begin + 64 * wave : t_end;
}

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kBlock = 64;             // tokens of a wave's block
constexpr float kRescale = 8.0f;       // lazy-rescale threshold, log2 units

// what lanes read whose chunk no token keeps, or whose tokens are past the row's keys: as long
// as the largest offset between a lane's loads
__device__ const uint32_t g_zeros[512] __attribute__((aligned(256))) = {};

__device__ __forceinline__ f32x4_t mfma16(u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                   __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// 16 bytes of global memory (an address that is either of two would be taken for a flat one), and
// what a block table holds, which nothing writes while the kernel runs (scalar loads)
__device__ __forceinline__ u32x4_t load16(uint64_t at, int offset) {
    return *((const __attribute__((address_space(1))) u32x4_t*)(at) + offset / 16);
}
typedef const __attribute__((address_space(4))) int32_t const_i32;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// 8 e4m3 numbers times a power of two as 8 bf16 numbers, exact
__device__ __forceinline__ u32x4_t widen(uint32_t a, uint32_t b, float power) {
    u32x4_t r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, power, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, power, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, power, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, power, true));
    return r;
}

// bf16 pairs whose bit is set in `mask` (bit e = pair e of the chunk)
__device__ __forceinline__ u32x4_t keep_pairs(u32x4_t x, uint32_t mask) {
    u32x4_t r;
#pragma unroll
    for (int t = 0; t < 4; ++t)
        r[t] = x[t] & (((mask >> (2 * t)) & 1u ? 0x0000FFFFu : 0u) | ((mask >> (2 * t + 1)) & 1u ? 0xFFFF0000u : 0u));
    return r;
}

// 4 bits as bytes of ones
__device__ __forceinline__ uint32_t byte_mask(uint32_t bits) { return (__umul24(bits, 0x204081u) & 0x01010101u) * 255u; }

// The sum over the wave's 64 lanes, and each lane's sum of the lanes up to it, by DPP.
template <int kCtrl, int kRows>
__device__ __forceinline__ int dpp_add(int x) {
    return x + __builtin_amdgcn_update_dpp(0, x, kCtrl, kRows, 0xF, false);
}
__device__ __forceinline__ int scan_lanes(int x) {
    x = dpp_add<0x111, 0xF>(x);  // from the lane 1, 2, 4, 8 below in the row of 16
    x = dpp_add<0x112, 0xF>(x);
    x = dpp_add<0x114, 0xF>(x);
    x = dpp_add<0x118, 0xF>(x);
    x = dpp_add<0x142, 0xA>(x);  // from the last lane of rows 0 and 2 to the rows after them
    return dpp_add<0x143, 0xC>(x);  // from that of row 1 to rows 2 and 3
}

// A row of a ragged batch: the position of its query, and the keys that it reaches, in [0, n_k].
struct Row {
    int q_pos, keys;
};
__device__ __forceinline__ Row row_of(const DecodeQ8Params& p, int r) {
    Row x = {0, 0};
    if (r < p.batch) {
        x.q_pos = min(max(p.q_pos_rows[r], 0), 0x7FFFFFFD);
        x.keys = min(min(max(p.n_k_rows[r], 0), p.n_k), x.q_pos + 1);
    }
    return x;
}

// ceil(n / span) for n and span up to 2^23, with inv near 1 / span
__device__ __forceinline__ int pieces(int n, int span, float inv) {
    const int up = n + span - 1;
    int q = int(float(up) * inv);
    const int rest = up - q * span;
    return q + (rest >= span ? 1 : 0) - (rest < 0 ? 1 : 0);
}

// The work plan of a ragged batch, the same in every wave that computes it: rows in steps of
// kDecodeQ8TokenStep tokens, cut into items of equal `tokens`, about p.splits in all: as many as
// run at once, so the span grows until they are no more than that, unless the batch has so many
// rows that their last, shorter items are a large part (p.splits + p.batch bounds them then).
// Items are numbered row by row.  Returns the row of `item` (-1 past the last), its Row and its
// first token; with `plan` set, writes the index of each row's first item and, at plan[batch],
// their number.
__device__ __forceinline__ int ragged_item(const DecodeQ8Params& p, int item, Row& out, int& t_first, int64_t& tokens,
                                           int32_t* plan) {
    const int lane = threadIdx.x & 63;
    const auto steps_of = [](const Row& x) __attribute__((always_inline)) {
        return int((uint32_t(x.keys) + kDecodeQ8TokenStep - 1) / kDecodeQ8TokenStep);
    };
    const Row own = row_of(p, lane);  // of the first 64 rows: mostly all
    const int own_steps = steps_of(own);
    const auto steps = [&](int r0) __attribute__((always_inline)) {
        return r0 == 0 ? own_steps : steps_of(row_of(p, r0 + lane));
    };
    float total = 0.f;
    int alive = 0;
    for (int r0 = 0; r0 < p.batch; r0 += 64) {
        const int n = steps(r0);
        total += float(__builtin_amdgcn_readlane(scan_lanes(n), 63));
        alive += __builtin_popcountll(__ballot(n > 0));
    }
    const bool many = 4 * alive > 3 * p.splits;
    if (total >= 16777216.f) total *= 1.0002f;  // above what it is rounded by, so that the bound holds
    // (a row's last item is half a span on average; no row has more than 2^23 steps)
    int span = max(1, int(fminf(__builtin_ceilf(total / float(many ? p.splits : p.splits - alive / 2)), 8388608.f)));
    float inv = 1.f / float(span);
    for (int round = 0; round < 8 && !many; ++round) {
        int items = 0;
        for (int r0 = 0; r0 < p.batch; r0 += 64)
            items += __builtin_amdgcn_readlane(scan_lanes(pieces(steps(r0), span, inv)), 63);
        if (items <= p.splits) break;
        span = max(span + 1, int(float(span) * float(items) / float(p.splits)));
        inv = 1.f / float(span);
    }
    int row = -1, first = 0, before = 0;
    for (int r0 = 0; r0 < p.batch; r0 += 64) {
        const int cnt = pieces(steps(r0), span, inv);
        const int incl = before + scan_lanes(cnt);
        if (plan != nullptr && r0 + lane < p.batch) plan[r0 + lane] = incl - cnt;
        const uint64_t hit = __ballot(item < incl);
        if (row < 0 && hit != 0) {
            const int l = __builtin_ctzll(hit);
            row = r0 + l;
            first = item - __builtin_amdgcn_readlane(incl - cnt, l);
            out = r0 == 0 ? Row{__builtin_amdgcn_readlane(own.q_pos, l), __builtin_amdgcn_readlane(own.keys, l)}
                          : row_of(p, row);
        }
        before = __builtin_amdgcn_readlane(incl, 63);
    }
    if (plan != nullptr && lane == 0) plan[p.batch] = before;
    tokens = int64_t(span) * kDecodeQ8TokenStep;
    t_first = int(first * tokens);
    return row;
}

// NT tiles of 16 heads share what a wave loads and widens.  NW waves: 4 or 8; with p.direct a
// workgroup takes a whole row and writes its output.
template <int D, int NT, int NW>
__global__ __launch_bounds__(NW * 64, NT == 1 && D == 64 ? 4 : 2) void decode_q8_kernel(const DecodeQ8Params p) {
    constexpr int kChunks = D / 16;
    constexpr int kHalf = D / 2;
    constexpr int kM = D / 64;   // loads of a token: 4 chunks each
    constexpr int kDB = D / 16;  // 16-dim blocks of the output
    constexpr int kOps = 2 * kM * NT;  // operands of the queries
    constexpr int kOStride = D + 4;
    __shared__ float red_m[NW][16 * NT];
    __shared__ float red_l[NW][16 * NT];
    __shared__ int s_w[kHalf];
    // the queries (and each wave's copy of them, where it is not in registers) while the waves
    // stream, then, a tile at a time, the waves' outputs [wave][head][D + 4]
    constexpr bool kQueryRegs = NT == 1 || D == 64;  // (the queries' registers: 2 tiles at d = 128 have none left)
    constexpr int kQueries = 256 * kOps * (kQueryRegs ? 1 : 1 + NW), kMerge = NW * 16 * kOStride;
    __shared__ __attribute__((aligned(16))) float shared[kQueries > kMerge ? kQueries : kMerge];

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15;
    const int g4 = lane >> 4;
    // of a ragged batch's work items the ones past the last come last, whatever the heads: they
    // would take the place of others where the chip has just one for each
    const int subgroups = p.subgroups;
    const bool items = !p.direct && p.n_k_rows != nullptr;
    const uint32_t cols = uint32_t(p.h_kv * subgroups);
    const int split = int(items ? blockIdx.x / cols : blockIdx.x);
    const int col = int(items ? blockIdx.x - split * cols : blockIdx.y);
    const int g = col / subgroups;
    const int sub = col % subgroups;
    const int hq0 = g * p.group + sub * p.heads_per_block;
    const int NH = min(p.heads_per_block, p.group - sub * p.heads_per_block);

    int my_w = lane < kHalf ? p.W[lane] : -1;
    int b, q_pos = p.q_pos, t_begin, t_end;
    int64_t slot0 = 0;
    if (p.direct) {
        b = blockIdx.x;
        t_begin = 0;
        t_end = p.n_valid;
        if (p.n_k_rows != nullptr) {
            const Row r = row_of(p, b);
            q_pos = r.q_pos;
            t_end = r.keys;
        }
    } else if (items) {
        int64_t span;
        int32_t* plan = (blockIdx.x == 0 && wave == 0) ? p.ws_plan : nullptr;
        Row r = {0, 0};
        b = ragged_item(p, split, r, t_begin, span, plan);
        if (b < 0) return;
        q_pos = r.q_pos;
        t_end = int(min(int64_t(r.keys), t_begin + span));
        slot0 = int64_t(split) * p.h_q + hq0;
    } else {
        b = blockIdx.z;
        t_begin = split * p.split_tokens;
        t_end = min(p.n_valid, t_begin + p.split_tokens);
        slot0 = (int64_t(b) * p.h_q + hq0) * p.splits + split;
    }
    b = __builtin_amdgcn_readfirstlane(b);
    q_pos = __builtin_amdgcn_readfirstlane(q_pos);
    t_begin = __builtin_amdgcn_readfirstlane(t_begin);
    t_end = __builtin_amdgcn_readfirstlane(t_end);
    const uint64_t zeros = reinterpret_cast<uint64_t>(g_zeros);
    const int tk = 16 * (r16 >> 2) + (r16 & 3);  // this lane's token of tile 0 (tile s adds 4 s)

    // a block: where its two halves of 32 tokens are (a page holds whole halves), and its pairs
    // kept at every token and at some
    struct Place {
        uint64_t k, ks, v, vs;  // of the half's first token in K chunk 0, V block, scales
    };
    struct Blk {
        Place a, b;
        uint64_t full, keep;
    };
    const int64_t cap = p.block_table != nullptr ? p.page_tokens : p.cache_tokens;
    const auto place = [&](int64_t row, int at) __attribute__((always_inline)) {
        Place x;
        x.k = reinterpret_cast<uint64_t>(p.k) + (row * kChunks * cap + at) * 16;
        x.v = reinterpret_cast<uint64_t>(p.v) + (row * ((cap + 15) / 16) * 16 + at) * D;
        x.ks = reinterpret_cast<uint64_t>(p.k_scale) + row * p.scale_tokens + at;
        x.vs = reinterpret_cast<uint64_t>(p.v_scale) + row * p.scale_tokens + at;
        return x;
    };
    const auto locate = [&](int t0) __attribute__((always_inline)) {
        Blk B;
        int64_t row = int64_t(b) * p.h_kv + g;
        if (p.block_table != nullptr) {
            const int pt = p.page_tokens, ia = t0 / pt, at = t0 - ia * pt;
            const auto* table = (const_i32*)(p.block_table + int64_t(b) * p.max_pages + ia);
            row = int64_t(min(max(table[0], 0), p.num_pages - 1)) * p.h_kv + g;
            B.a = place(row, at);
            B.b = place(row, at + 32);
            // (a row of the table has an entry for every key)
            if (at + 32 == pt && t_end - t0 > 32)
                B.b = place(int64_t(min(max(table[1], 0), p.num_pages - 1)) * p.h_kv + g, 0);
        } else {
            B.a = place(row, t0);
            B.b = place(row, t0 + 32);
        }
        return B;
    };
    const auto classify = [&](Blk& B, int t0) __attribute__((always_inline)) {
        B.full = __ballot(my_w >= q_pos - t0);
        B.keep = __ballot(my_w >= max(0, q_pos - t0 - min(kBlock, t_end - t0) + 1));
    };
    // K operands (a token past the split's end is the split's last one again)
    u32x4_t kf[4][kM], kscale;
    const int64_t k_lane = g4 * cap * 16;
    const auto load_k = [&](const Blk& B, int t0) __attribute__((always_inline)) {
        const bool hi = r16 >= 8;
        const int last = t_end - 1 - t0 - (hi ? 32 : 0);  // of the half
        const bool whole = t_end - t0 >= kBlock;
        const uint64_t at = (hi ? B.b.k : B.a.k) + k_lane;
#pragma unroll
        for (int m = 0; m < kM; ++m) {
            const int c = 4 * m + g4;
            const bool kept = last >= 0 && ((B.keep >> (8 * c)) & 0xFFull) != 0;
            const uint64_t src = kept ? at + 64 * m * cap : zeros;
            if (whole) {
#pragma unroll
                for (int s = 0; s < 4; ++s) kf[s][m] = load16(src + 16 * uint32_t(tk & 31), 64 * s);
            } else {
#pragma unroll
                for (int s = 0; s < 4; ++s) kf[s][m] = load16(src + 16 * uint32_t(max(min((tk & 31) + 4 * s, last), 0)), 0);
            }
        }
        kscale = load16(last >= (tk & 16) ? (hi ? B.b.ks : B.a.ks) + (tk & 16) : zeros, 0);
    };
    // V^T operands
    u32x4_t vf[kDB], vscale;
    const auto load_v = [&](const Blk& B, int t0) __attribute__((always_inline)) {
        const bool hi = g4 >= 2, in = 16 * g4 < t_end - t0;
        const uint64_t src = in ? (hi ? B.b.v : B.a.v) + (16 * D * (g4 & 1) + 16 * r16) : zeros;
#pragma unroll
        for (int i = 0; i < kDB; ++i) vf[i] = load16(src, 256 * i);
        vscale = load16(in ? (hi ? B.b.vs : B.a.vs) + 16 * (g4 & 1) : zeros, 0);
    };

    int t0 = decode_q8_first(t_begin, t_end, wave);
    Blk B{};
    if (t0 < t_end) {
        // (the values first: they need no window, whose table is on its way)
        B = locate(t0);
        load_v(B, t0);
    }
    if (tid < kHalf) s_w[tid] = my_w;
    asm volatile("" : "+v"(my_w));  // it has arrived: the loop need not wait for it
    if (t0 < t_end) {
        classify(B, t0);
        load_k(B, t0);
    }
    // queries: operand (tile, m, half) at 256 (2 kM tile + 2 m + half) + 4 lane
    for (int o = wave; o < kOps; o += NW) {
        const int h = 16 * (o / (2 * kM)) + r16, m = o / 2 % kM;
        u32x4_t z = {0u, 0u, 0u, 0u};
        if (h < NH)
            z = *reinterpret_cast<const u32x4_t*>(p.q + (int64_t(b) * p.h_q + hq0 + h) * D + (o & 1) * kHalf +
                                                  8 * (4 * m + g4));
        *reinterpret_cast<u32x4_t*>(&shared[256 * o + 4 * lane]) = z;
    }
    __syncthreads();
    // the queries, with the pairs outside q_keep zeroed
    uint64_t q_keep = ~0ull;
    [[maybe_unused]] u32x4_t q_regs[kQueryRegs ? kOps : 1];
    [[maybe_unused]] float* const q_lds = &shared[256 * kOps * (1 + wave) + 4 * lane];
    const auto set_query = [&](int o, u32x4_t x) __attribute__((always_inline)) {
        if constexpr (kQueryRegs)
            q_regs[o] = x;
        else
            *reinterpret_cast<u32x4_t*>(q_lds + 256 * o) = x;
    };
    const auto query = [&](int o) __attribute__((always_inline)) {
        if constexpr (kQueryRegs)
            return q_regs[o];
        else
            return *reinterpret_cast<const u32x4_t*>(q_lds + 256 * o);
    };
#pragma unroll
    for (int o = 0; o < kOps; ++o) set_query(o, *reinterpret_cast<const u32x4_t*>(&shared[256 * o + 4 * lane]));

    f32x4_t oacc[NT][kDB];
    float m_run[NT], m_thr[NT], m_neg[NT], l_run[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int i = 0; i < kDB; ++i) oacc[n][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        m_run[n] = m_thr[n] = -INFINITY;
        m_neg[n] = l_run[n] = 0.f;
    }
    const float sc = p.scale_log2;

    // (nothing in flight: the loop's waits count its own loads alone)
    asm volatile("" : "+v"(kscale), "+v"(vscale));
#pragma unroll
    for (int i = 0; i < kDB; ++i) asm volatile("" : "+v"(vf[i]));
#pragma unroll
    for (int m = 0; m < kM; ++m) asm volatile("" : "+v"(kf[0][m]), "+v"(kf[1][m]), "+v"(kf[2][m]), "+v"(kf[3][m]));
    while (t0 < t_end) {
        const uint64_t full = B.full, keep = B.keep;
        // windows that end inside the block: this lane's token and chunk, byte by byte
        if (keep & ~full) {
#pragma unroll
            for (int m = 0; m < kM; ++m) {
                int w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = s_w[8 * (4 * m + g4) + e];
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const int z = q_pos - t0 - (tk + 4 * s);
                    uint32_t lo = 0, hi = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        lo |= w[e] >= z ? 0xFFu << (8 * e) : 0u;
                        hi |= w[4 + e] >= z ? 0xFFu << (8 * e) : 0u;
                    }
                    kf[s][m] &= u32x4_t{lo, hi, lo, hi};
                }
            }
        } else {
            // chunks that hold pairs kept and pruned at all of the block's tokens: the pruned ones'
            // numbers must not count even where they are none, and 0 times NaN is NaN
#pragma unroll
            for (int m = 0; m < kM; ++m) {
                const uint32_t four = uint32_t(keep >> (32 * m));  // chunks 4 m .. 4 m + 3
                if ((four ^ (four >> 1)) & 0x7F7F7F7Fu) {
                    const uint32_t pairs = four >> (8 * g4);
                    const uint32_t lo = byte_mask(pairs & 15u), hi = byte_mask((pairs >> 4) & 15u);
#pragma unroll
                    for (int s = 0; s < 4; ++s) kf[s][m] &= u32x4_t{lo, hi, lo, hi};
                }
            }
        }
        if (keep != q_keep) {
            q_keep = keep;
#pragma unroll
            for (int o = 0; o < kOps; ++o)
                set_query(o, keep_pairs(*reinterpret_cast<const u32x4_t*>(&shared[256 * o + 4 * lane]),
                                        uint32_t(keep >> (8 * (4 * (o / 2 % kM) + g4))) & 0xFFu));
        }
        f32x4_t sacc[NT][4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const float power = q8::power((kscale[s] >> (8 * (r16 & 3))) & 255u);
#pragma unroll
            for (int m = 0; m < kM; ++m) {
                const u32x4_t k0 = widen(kf[s][m][0], kf[s][m][1], power), k1 = widen(kf[s][m][2], kf[s][m][3], power);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int o = 2 * kM * n + 2 * m;
                    sacc[n][s] = mfma16(k0, query(o), m == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : sacc[n][s]);
                    sacc[n][s] = mfma16(k1, query(o + 1), sacc[n][s]);
                }
            }
        }
        // the next block's keys, into the registers of this one's; its values follow below
        // (after the last block zeros are read, so that the loads in flight, which the waits count,
        // are the same on every path; positions reach 2^31: no sum past t_end)
        const bool more = t_end - t0 > kBlock * NW;
        const int t_next = more ? t0 + kBlock * NW : t_end;
        if (more) {
            B = locate(t_next);
            classify(B, t_next);
        }
        load_k(B, t_next);
        // tokens past the split's end: no probability, and no value that is not a number
        if (t_end - t0 < kBlock) {
            const int bound = t_end - t0 - 16 * g4;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                uint32_t msk = 0;
#pragma unroll
                for (int v = 0; v < 4; ++v) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        if (4 * s + v >= bound) sacc[n][s][v] = -INFINITY;
                    msk |= 4 * s + v < bound ? 0xFFu << (8 * v) : 0u;
                }
                vscale[s] &= msk;
#pragma unroll
                for (int i = 0; i < kDB; ++i) vf[i][s] &= msk;
            }
        }
        // P times the values' powers as two bf16 numbers, what fits and what is left over: one
        // would round every probability to 2^-9, and the output's own rounding is that size
        u32x4_t ph[NT][2], pl[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float mx = -INFINITY;
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int v = 0; v < 4; ++v) mx = fmaxf(mx, sacc[n][s][v]);
            if (__any(mx * sc > m_thr[n])) {
                mx = fmaxf(mx, __shfl_xor(mx, 16));
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                const float m_new = fmaxf(m_run[n], mx * sc);
                const float m_use = m_new == -INFINITY ? 0.f : m_new;
                const float alpha = exp2_fast(m_run[n] - m_use);
                m_run[n] = m_new;
                m_thr[n] = m_new + kRescale;
                m_neg[n] = -m_use;
                l_run[n] *= alpha;
#pragma unroll
                for (int i = 0; i < kDB; ++i)
#pragma unroll
                    for (int v = 0; v < 4; ++v) oacc[n][i][v] *= alpha;
            }
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    float x[2];
                    uint32_t h[2];
                    bf16x2_t rest;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int v = 2 * t + k;
                        const float e = exp2_fast(__builtin_fmaf(sacc[n][s][v], sc, m_neg[n]));
                        l_run[n] += e;
                        x[k] = e * q8::power((vscale[s] >> (8 * v)) & 255u);
                        h[k] = __float_as_uint(x[k]) & 0xFFFF0000u;
                        rest[k] = (__bf16)(x[k] - __uint_as_float(h[k]));
                    }
                    ph[n][s >> 1][2 * (s & 1) + t] = h[0] >> 16 | h[1];
                    pl[n][s >> 1][2 * (s & 1) + t] = __builtin_bit_cast(uint32_t, rest);
                }
        }
#pragma unroll
        for (int i = 0; i < kDB; ++i) {
            const u32x4_t v0 = widen(vf[i][0], vf[i][1], 1.f), v1 = widen(vf[i][2], vf[i][3], 1.f);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                oacc[n][i] = mfma16(v0, ph[n][0], oacc[n][i]);
                oacc[n][i] = mfma16(v1, ph[n][1], oacc[n][i]);
                oacc[n][i] = mfma16(v0, pl[n][0], oacc[n][i]);
                oacc[n][i] = mfma16(v1, pl[n][1], oacc[n][i]);
            }
        }
        load_v(B, t_next);
        t0 = t_next;
    }

    // ---- combine the waves' states (in wave order) and write the split's partial, or the output
    // of a row that is not split
    float l_lane[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        l_lane[n] = l_run[n] + __shfl_xor(l_run[n], 16);
        l_lane[n] += __shfl_xor(l_lane[n], 32);
        // every score NaN: any maximum will do for the normaliser to reach the output
        if (m_run[n] == -INFINITY && l_lane[n] != l_lane[n]) m_run[n] = 0.f;
        if (g4 == 0) {
            red_m[wave][16 * n + r16] = m_run[n];
            red_l[wave][16 * n + r16] = l_lane[n];
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        __syncthreads();  // the states are there; the queries, or the last tile, are done with
        float m_all = -INFINITY;
#pragma unroll
        for (int w = 0; w < NW; ++w) m_all = fmaxf(m_all, red_m[w][16 * n + r16]);
        const float f = m_run[n] == -INFINITY ? 0.f : exp2_fast(m_run[n] - m_all);
        const int heads = min(NH - 16 * n, 16);
        if (r16 < heads) {
#pragma unroll
            for (int i = 0; i < kDB; ++i)
                *reinterpret_cast<f32x4_t*>(&shared[(16 * wave + r16) * kOStride + 16 * i + 4 * g4]) = oacc[n][i] * f;
        }
        __syncthreads();
        for (int e = tid; e < heads * (D / 4); e += NW * 64) {
            const int r = e / (D / 4), x = 4 * (e % (D / 4)), h = 16 * n + r;
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < NW; ++w) M = fmaxf(M, red_m[w][h]);
            f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NW; ++w) o += *reinterpret_cast<const f32x4_t*>(&shared[(16 * w + r) * kOStride + x]);
            float L = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w)
                if (red_m[w][h] != -INFINITY) L += red_l[w][h] * exp2_fast(red_m[w][h] - M);
            if (p.direct) {
                const bool empty = L == 0.f;  // (as in the merge: O = 0, LSE = -inf)
                bf16x2_t lo, hi;
                lo[0] = (__bf16)(empty ? 0.f : o[0] / L);
                lo[1] = (__bf16)(empty ? 0.f : o[1] / L);
                hi[0] = (__bf16)(empty ? 0.f : o[2] / L);
                hi[1] = (__bf16)(empty ? 0.f : o[3] / L);
                const int64_t row = int64_t(b) * p.h_q + hq0 + h;
                *reinterpret_cast<uint2*>(p.o + row * D + x) =
                    make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
                if (x == 0) p.lse[row] = empty ? -INFINITY : M * 0.69314718055994531f + logf(L);
                continue;
            }
            const int64_t slot = items ? slot0 + h : slot0 + int64_t(h) * p.splits;
            if (x == 0) {
                p.ws_m[slot] = M;
                p.ws_l[slot] = L;
            }
            *reinterpret_cast<f32x4_t*>(&p.ws_o[slot * D + x]) = o;
        }
    }
}

// Merge of the split partials of one (row, head): NW waves, each over every NW-th state with a
// maximum of its own, so that no load waits for another; a lane has the same D / 64 dims of all.
template <int D, int NW>
__global__ __launch_bounds__(NW * 64) void decode_q8_merge_kernel(const DecodeQ8States p) {
    constexpr int kN = D / 64;
    constexpr int kAhead = 8;  // states in flight
    typedef float out_t __attribute__((ext_vector_type(kN)));
    __shared__ float s_o[NW][D];
    __shared__ float s_m[NW], s_l[NW];
    const int bh = blockIdx.x;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int64_t base = int64_t(bh) * p.splits, stride = 1;
    int count = p.splits;
    if (p.ws_plan != nullptr) {
        // (the clamps only restate what the plan guarantees: at most splits + batch items)
        const int b = bh / p.h_q, most = p.splits + p.batch;
        const auto* plan = (const_i32*)(p.ws_plan + b);
        const int first = min(max(plan[0], 0), most);
        count = min(max(plan[1] - first, 0), most - first);
        base = int64_t(first) * p.h_q + bh % p.h_q;
        stride = p.h_q;
    }
    float M = -INFINITY, L = 0.f;
    out_t O = {};
    for (int s0 = wave; s0 < count; s0 += NW * kAhead) {
        float m[kAhead], l[kAhead];
        out_t o[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t at = base + min(s0 + NW * i, count - 1) * stride;
            m[i] = p.ws_m[at];
            l[i] = p.ws_l[at];
            o[i] = *reinterpret_cast<const out_t*>(p.ws_o + at * D + kN * lane);
        }
        float top = M;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (s0 + NW * i >= count) m[i] = -INFINITY;
            top = fmaxf(top, m[i]);
        }
        if (top == -INFINITY) continue;  // splits without a causal key
        const float f = exp2_fast(M - top);
        M = top;
        L *= f;
        O *= f;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const float w = exp2_fast(m[i] - M);
            L += m[i] == -INFINITY ? 0.f : w * l[i];
            O += m[i] == -INFINITY ? out_t{} : w * o[i];
        }
    }
    *reinterpret_cast<out_t*>(&s_o[wave][kN * lane]) = O;
    if (lane == 0) {
        s_m[wave] = M;
        s_l[wave] = L;
    }
    __syncthreads();
    if (threadIdx.x >= D / 2) return;
    M = s_m[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) M = fmaxf(M, s_m[w]);
    L = 0.f;
    float2 o = make_float2(0.f, 0.f);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const float f = s_m[w] == -INFINITY ? 0.f : exp2_fast(s_m[w] - M);
        L += f * s_l[w];
        o.x += f * s_o[w][2 * threadIdx.x];
        o.y += f * s_o[w][2 * threadIdx.x + 1];
    }
    const bool empty = L == 0.f;  // a row without keys: O = 0, LSE = -inf
    bf16x2_t two;
    two[0] = (__bf16)(empty ? 0.f : o.x / L);
    two[1] = (__bf16)(empty ? 0.f : o.y / L);
    *reinterpret_cast<uint32_t*>(p.o + int64_t(bh) * D + 2 * threadIdx.x) = __builtin_bit_cast(uint32_t, two);
    if (threadIdx.x == 0) p.lse[bh] = empty ? -INFINITY : M * 0.69314718055994531f + logf(L);
}

template <int D, int NT>
hipError_t launch_d(const DecodeQ8Params& p, hipStream_t stream) {
    // ragged: a workgroup per possible work item (at most p.splits + batch) and KV head, or part
    const bool ragged = p.n_k_rows != nullptr, items = ragged && !p.direct;
    const int64_t cols = int64_t(p.h_kv) * p.subgroups;
    const int64_t x = p.direct ? p.batch : items ? (int64_t(p.splits) + p.batch) * cols : p.splits;
    if (x * p.waves * 64 > 0xFFFFFFFF) return hipErrorInvalidConfiguration;  // (the threads of a grid)
    const dim3 grid(unsigned(x), unsigned(items ? 1 : cols), unsigned(p.direct || ragged ? 1 : p.batch));
    if (p.waves == 8)
        hipLaunchKernelGGL((decode_q8_kernel<D, NT, 8>), grid, dim3(512), 0, stream, p);
    else
        hipLaunchKernelGGL((decode_q8_kernel<D, NT, 4>), grid, dim3(256), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.direct) return e;
    // the merge's waves by the states of a row: a ragged batch's longest rows have some times the
    // average
    const int64_t states = ragged ? 3 * int64_t(p.splits) / p.batch : p.splits;
    const dim3 heads(unsigned(p.batch * p.h_q));
    if (states > 128)
        hipLaunchKernelGGL((decode_q8_merge_kernel<D, 16>), heads, dim3(1024), 0, stream, p);
    else if (states > 32)
        hipLaunchKernelGGL((decode_q8_merge_kernel<D, 8>), heads, dim3(512), 0, stream, p);
    else
        hipLaunchKernelGGL((decode_q8_merge_kernel<D, 4>), heads, dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_decode_q8(const DecodeQ8Params& p, int head_dim, hipStream_t stream) {
    if (p.splits < 1 || p.splits > kDecodeMaxSplits || p.heads_per_block < 1 || p.heads_per_block > 32 ||
        p.subgroups < 1 || (p.subgroups - 1) * p.heads_per_block >= p.group ||
        p.subgroups * p.heads_per_block < p.group || (p.waves != 4 && p.waves != 8))
        return hipErrorInvalidValue;
    if (!p.direct && p.n_k_rows == nullptr &&
        (int64_t(p.splits) * p.split_tokens < p.n_valid || p.split_tokens % kDecodeQ8TokenStep != 0))
        return hipErrorInvalidValue;
    if (p.n_k_rows != nullptr && (p.q_pos_rows == nullptr || (!p.direct && (p.ws_plan == nullptr || p.splits > kDecodeMaxSplits - 1))))
        return hipErrorInvalidValue;
    (void)hipGetLastError();
    if (p.heads_per_block > 16)
        return head_dim == 64 ? launch_d<64, 2>(p, stream) : launch_d<128, 2>(p, stream);
    return head_dim == 64 ? launch_d<64, 1>(p, stream) : launch_d<128, 1>(p, stream);
}

}  // namespace atf
