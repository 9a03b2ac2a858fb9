// Windowed attention of query tokens over the blocks of their rows that a list names, over pages, gfx950.
//
// The heads of one KV head (up to 32 a workgroup) are the columns of v_mfma_f32_16x16x32_bf16, in one
// or two tiles; a wave's step is a tile of 32 tokens of one block.  Pages as in decode.hip.  With
// r = lane % 16, g = lane / 16:
//   scores, s = 0, 1: A row r is token 16 (r / 8) + 8 s + 4 (r / 4 % 2) + r % 4 of the tile, the lane's 16
//     bytes half g % 2 of chunk 2 m + g / 2 of it.  The result gives the lane, for head r, tokens
//     16 (g / 2) + 8 s + 4 (g % 2) + v.
//   values: the lane's 16 bytes are half g % 2 of the slots of dim 16 i + r in 16-token block g / 2: the
//     tokens whose scores it has.
//
// A pair is kept at distance z iff z <= W_r.  Per tile two ballots give the pairs kept at some token
// and at every token: chunks without a kept pair are not read, and products of two such not made;
// keys lose the pairs kept nowhere, so that a number that is none does not count there; where a window
// ends inside the tile they are masked token by token.
//
// The NW waves of a workgroup take the list's tiles in turn and join their states in LDS.  Where tokens
// are few a list is split over workgroups, whose partial states a second kernel joins.
//
// Bound by HBM reads where rows are many: 63 rows of up to 4,096 keys, 24/8 heads of 128 (813 MB), 148 us,
// 5.5 TB/s (a streaming read reaches 5.57).  Inside the CUs where many tokens read one row's: 1,460 tokens of
// 2,048 keys, 32/4 heads of 128, 219 us, and 200 with one tile's keys and values read for all (a copy of the
// kernel): 16 loads of 1 KB a tile into registers, each byte used for one token's 8 heads, and 170 vector
// instructions (ALU busy 0.51) by two waves a SIMD.  There a wave that walks its list alone and in order
// stays near the others of its XCD: 238 us with one wave a token and head, 281 with four; three waves a SIMD
// (the masks formed for each tile) take 242 for 220.  A single token's call is a launch and a chain of loads
// (token, row, list, table, keys): 7 us for 16 blocks of 32, 14/2 heads of 64.
#include "atf_internal.hpp"

namespace atf {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kTile = 32;
constexpr float kRescale = 8.0f;  // lazy-rescale threshold, log2 units

__device__ __forceinline__ f32x4_t mfma16(u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                   __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
// 16 bytes a lane at base + off (base wave-uniform), or zeros, nothing read, where off is kOutOfRange
constexpr uint32_t kOutOfRange = 0xFFFFFFFFu;
__device__ __forceinline__ u32x4_t load16(const char* base, uint32_t off, int more) {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, int(0xFFFFFFF0u), 0x00020000);
    return __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, int(off), more, 0));
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// halves of a register pair of bf16 numbers that bits 2t, 2t + 1 keep
__device__ __forceinline__ uint32_t pair_mask(uint32_t bits, int t) {
    return ((bits >> (2 * t)) & 1u ? 0x0000FFFFu : 0u) | ((bits >> (2 * t + 1)) & 1u ? 0xFFFF0000u : 0u);
}

// A lane looks up one tile of the list, 64 at a time; which of them are tokens of the row is a ballot.
struct Tile {
    int page, at;  // where its first token is
    int first;     // that token's position
};

template <int D, int NT, int NW, bool kHalves>
__global__ __launch_bounds__(NW * 64, 2) void attend_blocks_kernel(const AttendParams p) {
    constexpr int kChunks = D / 16;
    constexpr int kHalf = D / 2;
    constexpr int kM = D / 32;   // products of a score: 2 chunks each
    constexpr int kDB = D / 16;  // 16-dim blocks of the output
    constexpr int kOps = kM * NT;
    constexpr int kOStride = D + 4;
    static_assert(!kHalves || NT == 1, "8 heads are half of a tile's columns");
    __shared__ float red_m[NW][16 * NT];
    __shared__ float red_l[NW][16 * NT];
    __shared__ int s_w[kHalf];
    __shared__ u32x4_t s_masks[256];  // of each set of a chunk's pairs
    __shared__ __attribute__((aligned(16))) float s_o[NW * 16 * kOStride];

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15;
    const int g4 = lane >> 4;
    const bool rests = kHalves && r16 >= 8;  // the column has what is left over of its head's probabilities
    const int cols = p.h_kv * p.subgroups;
    const int item = int(blockIdx.x) / cols;
    const int col = int(blockIdx.x) - item * cols;
    const int t = item / p.splits, split = item - t * p.splits;
    const int g = col / p.subgroups, sub = col - g * p.subgroups;
    const int hq0 = g * p.group + sub * p.heads_per_block;
    const int NH = min(p.heads_per_block, p.group - sub * p.heads_per_block);

    const int row = __builtin_amdgcn_readfirstlane(p.token_rows[t]);
    if (row < 0 || row >= p.batch) return;  // padding: nothing of it is written
    const int q_pos = __builtin_amdgcn_readfirstlane(min(p.positions[t], 0x7FFFFFFD));
    // the last key (below 0: none)
    const int last = min(min(max(__builtin_amdgcn_readfirstlane(p.n_k_rows[row]), 0), p.max_n_k) - 1, q_pos);

    const int my_w = lane < kHalf ? p.W[lane] : -1;
    if (tid < kHalf) s_w[tid] = my_w;
    for (int e = tid; e < 256; e += NW * 64)
        s_masks[e] = u32x4_t{pair_mask(e, 0), pair_mask(e, 1), pair_mask(e, 2), pair_mask(e, 3)};

    // this wave's tiles of the split: every NW-th
    const int per = p.block_tokens / kTile;
    const int tile1 = min(p.top * per, (split + 1) * p.split_tiles);
    const int32_t* list = p.blocks + (int64_t(t) * p.h_kv + g) * p.top;
    int i0 = split * p.split_tiles + wave;
    Tile mine = {0, 0, 0};
    uint64_t found = 0;
    const auto look = [&]() __attribute__((always_inline)) {
        const int i = i0 + NW * lane;
        bool is = false;
        if (i < tile1) {
            const int k = i / per, j = list[k];
            if (j >= 0 && last >= 0 && j <= last / p.block_tokens) {
                mine.first = j * p.block_tokens + (i - k * per) * kTile;
                is = mine.first <= last;
                if (is) {
                    const int n = mine.first / p.page_tokens;
                    mine.page = min(max(p.block_table[int64_t(row) * p.max_pages + n], 0), p.num_pages - 1);
                    mine.at = mine.first - n * p.page_tokens;
                }
            }
        }
        found = __ballot(is);
        i0 += 64 * NW;
    };
    const auto next = [&](Tile& x) __attribute__((always_inline)) {
        while (found == 0) {
            if (i0 >= tile1) return false;
            look();
        }
        const int l = __builtin_ctzll(found);
        found &= found - 1;
        x.page = __builtin_amdgcn_readlane(mine.page, l);
        x.at = __builtin_amdgcn_readlane(mine.at, l);
        x.first = __builtin_amdgcn_readlane(mine.first, l);
        return true;
    };
    const int tk = 16 * (r16 >> 3) + 4 * ((r16 >> 2) & 1) + (r16 & 3);  // this lane's token of s = 0
    // (after the last tile nothing is read, but all loads are issued: those in flight, which the waits
    // count, are the same on every path)
    const uint32_t k_lane = uint32_t(g4 >> 1) * (32 * uint32_t(p.page_tokens)) + 16 * (g4 & 1);
    const uint32_t v_lane = 16 * (g4 & 1) + 32 * r16;
    u32x4_t kf[2][kM], vf[kDB];
    uint64_t full = 0, keep = 0;
    const auto load_k = [&](const Tile& x, bool is) __attribute__((always_inline)) {
        const int left = max(min(last - x.first, kTile - 1), 0);
        full = __ballot(my_w >= q_pos - x.first);
        keep = is ? __ballot(my_w >= q_pos - x.first - left) : 0ull;
        const int64_t ph = int64_t(x.page) * p.h_kv + g;
        const char* base = reinterpret_cast<const char*>(p.k_pages) + (ph * kChunks * p.page_tokens + x.at) * 32;
        const uint32_t t0 = k_lane + 32 * min(tk, left), t1 = k_lane + 32 * min(tk + 8, left);
        const uint64_t mine = keep >> (8 * (g4 >> 1));  // of this lane's chunk of each two
#pragma unroll
        for (int m = 0; m < kM; ++m) {
            const bool kept = (uint32_t(mine >> (16 * m)) & 0xFFu) != 0;
            const char* from = base + int64_t(m) * (64 * int64_t(p.page_tokens));
            kf[0][m] = load16(from, kept ? t0 : kOutOfRange, 0);
            kf[1][m] = load16(from, kept ? t1 : kOutOfRange, 0);
        }
    };
    const auto load_v = [&](const Tile& x, bool is) __attribute__((always_inline)) {
        const char* base = reinterpret_cast<const char*>(p.v_pages) +
                           ((int64_t(x.page) * p.h_kv + g) * p.page_tokens + x.at) * (2 * D);
        // (a 16-token block past the row's end is not read)
        const uint32_t off = is && 16 * (g4 >> 1) <= last - x.first ? v_lane + (g4 >> 1) * (32 * D) : kOutOfRange;
#pragma unroll
        for (int i = 0; i < kDB; ++i) vf[i] = load16(base + 512 * i, off, 0);
    };
    // they have arrived
    const auto wait_k = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < kM; ++m) asm volatile("" : "+v"(kf[0][m]), "+v"(kf[1][m]));
    };
    const auto wait_v = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kDB; ++i) asm volatile("" : "+v"(vf[i]));
    };

    Tile x = {0, 0, 0};
    bool have = next(x);
    if (have) {
        load_v(x, true);
        load_k(x, true);
    }
    // queries: operand (tile n, m).  d = 128 with two column tiles has no registers for them, nor for the
    // masks below: they are in LDS then.
    constexpr bool kCached = NT == 1 || D == 64;
    const auto query_of = [&](int o) __attribute__((always_inline)) {
        const int h = 16 * (o / kM) + (kHalves ? r16 & 7 : r16), m = o % kM;
        u32x4_t q = {0u, 0u, 0u, 0u};
        if (h < NH)
            q = *reinterpret_cast<const u32x4_t*>(p.q + (int64_t(t) * p.h_q + hq0 + h) * D + (g4 & 1) * kHalf +
                                                  8 * (2 * m + (g4 >> 1)));
        return q;
    };
    [[maybe_unused]] u32x4_t qf[kCached ? kOps : 1];
    [[maybe_unused]] u32x4_t* const s_q = reinterpret_cast<u32x4_t*>(s_o) + lane;
    if constexpr (kCached) {
#pragma unroll
        for (int o = 0; o < kOps; ++o) qf[o] = query_of(o);
    } else {
        static_assert(NW * 16 * kOStride * 4 >= kOps * 64 * 16, "the states' room holds the queries");
        for (int o = wave; o < kOps; o += NW) s_q[64 * o] = query_of(o);
    }
    __syncthreads();

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
    // masks of the pairs that are kept, and the queries so masked, of the last tile
    uint64_t q_keep = ~0ull;
    [[maybe_unused]] u32x4_t masks[kCached ? kM : 1], qm[kCached ? kOps : 1];
    if constexpr (kCached) {
#pragma unroll
        for (int m = 0; m < kM; ++m) masks[m] = u32x4_t{~0u, ~0u, ~0u, ~0u};
#pragma unroll
        for (int o = 0; o < kOps; ++o) qm[o] = qf[o];
    }

    // (nothing in flight: the loop's waits count its own loads alone)
    wait_v();
    wait_k();
    while (have) {
        wait_k();
        const int left = last - x.first;  // the tile's last token that counts, if below 31
        if (keep & ~full) {
#pragma unroll
            for (int m = 0; m < kM; ++m) {
                int w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = s_w[8 * (2 * m + (g4 >> 1)) + e];
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const int z = q_pos - x.first - (tk + 8 * s);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        kf[s][m][e] &= (w[2 * e] >= z ? 0x0000FFFFu : 0u) | (w[2 * e + 1] >= z ? 0xFFFF0000u : 0u);
                }
            }
        }
        // pairs kept nowhere in the tile: the queries and the keys (zeros in lanes whose chunk was not read)
        // lose them
        if constexpr (kCached) {
            if (keep != q_keep) {
                q_keep = keep;
#pragma unroll
                for (int m = 0; m < kM; ++m) {
                    masks[m] = s_masks[uint32_t(keep >> (16 * m + 8 * (g4 >> 1))) & 0xFFu];
#pragma unroll
                    for (int n = 0; n < NT; ++n) qm[kM * n + m] = qf[kM * n + m] & masks[m];
                }
            }
        }
        f32x4_t sacc[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) sacc[n][0] = sacc[n][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int m = 0; m < kM; ++m) {
            const uint32_t both = uint32_t(keep >> (16 * m)) & 0xFFFFu;
            if (both == 0) continue;
            if constexpr (kCached) {
                if ((both ^ (both >> 1)) & 0x7F7Fu) {
                    kf[0][m] &= masks[m];
                    kf[1][m] &= masks[m];
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int s = 0; s < 2; ++s) sacc[n][s] = mfma16(kf[s][m], qm[kM * n + m], sacc[n][s]);
            } else {
                u32x4_t mask = {~0u, ~0u, ~0u, ~0u};
                if (both != 0xFFFFu) {
                    mask = s_masks[(both >> (8 * (g4 >> 1))) & 0xFFu];
                    kf[0][m] &= mask;
                    kf[1][m] &= mask;
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const u32x4_t q = s_q[64 * (kM * n + m)] & mask;
                    sacc[n][0] = mfma16(kf[0][m], q, sacc[n][0]);
                    sacc[n][1] = mfma16(kf[1][m], q, sacc[n][1]);
                }
            }
        }
        // the next tile's keys, into the registers of this one's; its values follow below
        Tile y = x;
        have = next(y);
        load_k(y, have);
        // tokens past the row's keys: no probability, and (below) no value that is not a number
        const int bound = left - 16 * (g4 >> 1) - 4 * (g4 & 1);
        if (left < kTile - 1) {
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int v = 0; v < 4; ++v)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        if (8 * s + v > bound) sacc[n][s][v] = -INFINITY;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float mx = -INFINITY;
#pragma unroll
            for (int s = 0; s < 2; ++s)
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
            // P as two bf16 numbers, what fits and what is left over: one would round every probability
            // to 2^-9, and the output's own rounding is that size.  Up to 8 heads have a column for each.
            u32x4_t ph, pl;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    uint32_t h[2];
                    bf16x2_t two;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float w = exp2_fast(__builtin_fmaf(sacc[n][s][2 * k + e], sc, m_neg[n]));
                        l_run[n] += w;
                        h[e] = __float_as_uint(w) & 0xFFFF0000u;
                        const float rest = w - __uint_as_float(h[e]);
                        two[e] = (__bf16)(kHalves && !rests ? __uint_as_float(h[e]) : rest);
                    }
                    if constexpr (!kHalves) ph[2 * s + k] = h[0] >> 16 | h[1];
                    pl[2 * s + k] = __builtin_bit_cast(uint32_t, two);
                }
            if (n == 0) {
                wait_v();
                if (left < kTile - 1) {
                    // (value 4 s + v of the lane's 8)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t msk = 8 * (e / 4) + e % 4 <= bound ? ~0u : e & 1 ? 0x0000FFFFu : 0xFFFF0000u;
#pragma unroll
                        for (int i = 0; i < kDB; ++i) vf[i][e / 2] &= msk;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < kDB; ++i) {
                if constexpr (!kHalves) oacc[n][i] = mfma16(vf[i], ph, oacc[n][i]);
                oacc[n][i] = mfma16(vf[i], pl, oacc[n][i]);
            }
        }
        load_v(y, have);
        x = y;
    }

    // ---- combine the waves' states, in wave order, and write the output, or the split's partial
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float l_lane = l_run[n] + __shfl_xor(l_run[n], 16);
        l_lane += __shfl_xor(l_lane, 32);
        // every score NaN: any maximum will do for the normaliser to reach the output
        if (m_run[n] == -INFINITY && l_lane != l_lane) m_run[n] = 0.f;
        if (g4 == 0) {
            red_m[wave][16 * n + r16] = m_run[n];
            red_l[wave][16 * n + r16] = l_lane;
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        __syncthreads();
        float m_all = -INFINITY;
#pragma unroll
        for (int w = 0; w < NW; ++w) m_all = fmaxf(m_all, red_m[w][16 * n + r16]);
        const float f = m_run[n] == -INFINITY ? 0.f : exp2_fast(m_run[n] - m_all);
        const int heads = min(NH - 16 * n, 16);
        if ((kHalves ? r16 & 7 : r16) < heads) {
#pragma unroll
            for (int i = 0; i < kDB; ++i)
                *reinterpret_cast<f32x4_t*>(&s_o[(16 * wave + r16) * kOStride + 16 * i + 4 * g4]) = oacc[n][i] * f;
        }
        __syncthreads();
        for (int e = tid; e < heads * (D / 4); e += NW * 64) {
            const int r = e / (D / 4), d = 4 * (e % (D / 4)), h = 16 * n + r;
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < NW; ++w) M = fmaxf(M, red_m[w][h]);
            f32x4_t o = {0.f, 0.f, 0.f, 0.f};
            float L = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                o += *reinterpret_cast<const f32x4_t*>(&s_o[(16 * w + r) * kOStride + d]);
                if constexpr (kHalves) o += *reinterpret_cast<const f32x4_t*>(&s_o[(16 * w + r + 8) * kOStride + d]);
                if (red_m[w][h] != -INFINITY) L += red_l[w][h] * exp2_fast(red_m[w][h] - M);
            }
            const int64_t to = int64_t(t) * p.h_q + hq0 + h;
            if (p.splits > 1) {
                const int64_t slot = to * p.splits + split;
                if (d == 0) {
                    p.ws_m[slot] = M;
                    p.ws_l[slot] = L;
                }
                *reinterpret_cast<f32x4_t*>(&p.ws_o[slot * D + d]) = o;
                continue;
            }
            const bool empty = L == 0.f;  // no key: O = 0, LSE = -inf
            bf16x2_t lo, hi;
            lo[0] = (__bf16)(empty ? 0.f : o[0] / L);
            lo[1] = (__bf16)(empty ? 0.f : o[1] / L);
            hi[0] = (__bf16)(empty ? 0.f : o[2] / L);
            hi[1] = (__bf16)(empty ? 0.f : o[3] / L);
            *reinterpret_cast<uint2*>(p.o + to * D + d) =
                make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
            if (d == 0) p.lse[to] = empty ? -INFINITY : M * 0.69314718055994531f + logf(L);
        }
    }
}

// Joins the splits' states of one (token, head), a wave; a lane has the same D / 64 dims of all.
template <int D>
__global__ __launch_bounds__(256) void attend_join_kernel(const AttendParams p) {
    constexpr int kN = D / 64;
    constexpr int kAhead = 8;  // states in flight
    typedef float out_t __attribute__((ext_vector_type(kN)));
    const int lane = threadIdx.x & 63;
    const int64_t th = int64_t(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (th >= int64_t(p.n_tokens) * p.h_q) return;
    const int row = __builtin_amdgcn_readfirstlane(p.token_rows[th / p.h_q]);
    if (row < 0 || row >= p.batch) return;
    float M = -INFINITY, L = 0.f;
    out_t O = {};
    for (int s0 = 0; s0 < p.splits; s0 += kAhead) {
        float m[kAhead], l[kAhead];
        out_t o[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t at = th * p.splits + min(s0 + i, p.splits - 1);
            m[i] = s0 + i < p.splits ? p.ws_m[at] : -INFINITY;
            l[i] = p.ws_l[at];
            o[i] = *reinterpret_cast<const out_t*>(p.ws_o + at * D + kN * lane);
        }
        float top = M;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) top = fmaxf(top, m[i]);
        if (top == -INFINITY) continue;  // splits without a key
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
    const bool empty = L == 0.f;
    if constexpr (kN == 2) {
        bf16x2_t two;
        two[0] = (__bf16)(empty ? 0.f : O[0] / L);
        two[1] = (__bf16)(empty ? 0.f : O[1] / L);
        *reinterpret_cast<uint32_t*>(p.o + th * D + 2 * lane) = __builtin_bit_cast(uint32_t, two);
    } else {
        p.o[th * D + lane] = __builtin_bit_cast(uint16_t, (__bf16)(empty ? 0.f : O[0] / L));
    }
    if (lane == 0) p.lse[th] = empty ? -INFINITY : M * 0.69314718055994531f + logf(L);
}

template <int D, int NT, bool kHalves>
hipError_t launch_d(const AttendParams& p, hipStream_t stream) {
    const int64_t blocks = int64_t(p.n_tokens) * p.splits * p.h_kv * p.subgroups;
    if (blocks * p.waves * 64 > 0xFFFFFFFF) return hipErrorInvalidConfiguration;
    const dim3 grid(static_cast<unsigned>(blocks)), threads(unsigned(p.waves) * 64);
    if (p.waves == 1)
        hipLaunchKernelGGL((attend_blocks_kernel<D, NT, 1, kHalves>), grid, threads, 0, stream, p);
    else if (p.waves == 2)
        hipLaunchKernelGGL((attend_blocks_kernel<D, NT, 2, kHalves>), grid, threads, 0, stream, p);
    else if (p.waves == 4)
        hipLaunchKernelGGL((attend_blocks_kernel<D, NT, 4, kHalves>), grid, threads, 0, stream, p);
    else
        hipLaunchKernelGGL((attend_blocks_kernel<D, NT, 8, kHalves>), grid, threads, 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    const unsigned joins = unsigned((int64_t(p.n_tokens) * p.h_q + 3) / 4);
    hipLaunchKernelGGL(attend_join_kernel<D>, dim3(joins), dim3(256), 0, stream, p);
    return hipGetLastError();
}

template <int D>
hipError_t launch_heads(const AttendParams& p, hipStream_t stream) {
    if (p.heads_per_block > 16) return launch_d<D, 2, false>(p, stream);
    return p.heads_per_block > 8 ? launch_d<D, 1, false>(p, stream) : launch_d<D, 1, true>(p, stream);
}

}  // namespace

hipError_t launch_attend_blocks(const AttendParams& p, int head_dim, hipStream_t stream) {
    if ((p.waves != 1 && p.waves != 2 && p.waves != 4 && p.waves != 8) || p.splits < 1 || p.split_tiles < 1) return hipErrorInvalidValue;
    (void)hipGetLastError();
    return head_dim == 64 ? launch_heads<64>(p, stream) : launch_heads<128>(p, stream);
}

}  // namespace atf
