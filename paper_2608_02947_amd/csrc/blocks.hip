// Bounds of the keys of each block of a row, and the blocks that a query takes by them, gfx950.
#include "atf_internal.hpp"
#include "scan.hpp"

#include <algorithm>

namespace atf {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x2_t __attribute__((ext_vector_type(2)));

// Two bf16 numbers as two 16-bit integers in the same order (a number's negative is its bits'
// complement but for the sign; its own inverse), so that one instruction takes the larger of both
// pairs.  NaNs come outside the infinities.
__device__ __forceinline__ s16x2_t ordered(uint32_t x) {
    const s16x2_t v = __builtin_bit_cast(s16x2_t, x);
    return v ^ ((v >> 15) & short(0x7FFF));
}

// Bounds: per dim the largest and the smallest of the block's keys (those of its row), a wave per
// (row, block, KV head, 4 chunks of 8 pairs).  A lane reads 16 bytes: one half (first or second
// components) of a token's chunk, 8 loads in flight; a token past the last is the last one again.
// Lanes of equal parity then share their extremes: the smallest as the largest complement, so that
// after the first step, which leaves one in the lower lanes and the other in the upper ones, both
// go on together.
// Bound by HBM reads: 131,072 keys of 4 heads of 128 (138 MB) 26.0 us, 5.3 TB/s (a streaming read
// reaches 5.57), 30.8 with loads that stay in the caches; 2 or 8 chunks a wave 30.6 and 31.2 against 30.8.
constexpr int kBoundChunks = 4;

template <int kCtrl>
__device__ __forceinline__ s16x2_t larger_dpp(s16x2_t x) {
    return __builtin_elementwise_max(
        x, __builtin_bit_cast(s16x2_t, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), kCtrl, 0xF, 0xF, true)));
}

template <int D>
__global__ __launch_bounds__(256) void block_bounds_kernel(const BoundsParams p) {
    constexpr int kChunks = D / 16, kParts = kChunks / kBoundChunks;
    const int lane = threadIdx.x & 63;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const uint32_t units = p.row_blocks * uint32_t(p.h_kv) * kParts;
    for (int b = blockIdx.y; b < p.batch; b += gridDim.y) {
        const int64_t cap = int64_t(p.max_pages) * p.page_tokens;
        const int n = int(min(int64_t(max(p.n_k_rows[b], 0)), cap));
        const int fresh = min(min(max(p.n_new_rows[b], 0), p.max_new), n);
        if (fresh == 0) continue;
        const int j0 = (n - fresh) / p.block_tokens, j1 = (n - 1) / p.block_tokens;
        for (uint32_t unit = wave; unit < units; unit += gridDim.x * 4) {
            const int c0 = int(unit % kParts) * kBoundChunks;
            const uint32_t rest = unit / kParts;
            const uint32_t k = rest / uint32_t(p.h_kv);
            const int g = int(rest - k * uint32_t(p.h_kv));
            if (k > uint32_t(j1 - j0)) break;
            const int first = (j0 + int(k)) * p.block_tokens;
            const int last = min(p.block_tokens, n - first) - 1;
            const int page = min(max(p.block_table[int64_t(b) * p.max_pages + first / p.page_tokens], 0), p.num_pages - 1);
            const int at = first % p.page_tokens;
            const int64_t pc = (int64_t(page) * p.h_kv + g) * kChunks + c0;
            const uint16_t* src = p.k_pages + (pc * p.page_tokens + at) * 16 + (lane & 1) * 8;
            s16x2_t hi[kBoundChunks][4], lo[kBoundChunks][4];
#pragma unroll
            for (int c = 0; c < kBoundChunks; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    hi[c][e] = s16x2_t{-32768, -32768};
                    lo[c][e] = s16x2_t{32767, 32767};
                }
            for (int t0 = 0; t0 <= last; t0 += 64) {
                u32x4_t x[kBoundChunks][2];
#pragma unroll
                for (int c = 0; c < kBoundChunks; ++c)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        x[c][h] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(
                            src + (int64_t(c) * p.page_tokens + min(t0 + 32 * h + (lane >> 1), last)) * 16));
#pragma unroll
                for (int c = 0; c < kBoundChunks; ++c)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const s16x2_t v = ordered(x[c][h][e]);
                            hi[c][e] = __builtin_elementwise_max(hi[c][e], v);
                            lo[c][e] = __builtin_elementwise_min(lo[c][e], v);
                        }
            }
#pragma unroll
            for (int c = 0; c < kBoundChunks; ++c) {
                u32x4_t out, none;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    // lanes 32..63 of the largest trade places with lanes 0..31 of the complements
                    const auto sw = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, hi[c][e]),
                                                                     ~__builtin_bit_cast(uint32_t, lo[c][e]), false, false);
                    s16x2_t v = __builtin_elementwise_max(__builtin_bit_cast(s16x2_t, uint32_t(sw[0])),
                                                          __builtin_bit_cast(s16x2_t, uint32_t(sw[1])));
                    v = larger_dpp<0x4E>(v);   // lane ^ 2
                    v = larger_dpp<0x124>(v);  // 4 and 8 on in the row of 16
                    v = larger_dpp<0x128>(v);
                    const uint32_t w = __builtin_bit_cast(uint32_t, v);
                    const auto rows = __builtin_amdgcn_permlane16_swap(w, w, false, false);
                    v = __builtin_elementwise_max(__builtin_bit_cast(s16x2_t, uint32_t(rows[0])),
                                                  __builtin_bit_cast(s16x2_t, uint32_t(rows[1])));
                    // (a positive NaN shows in the largest, a negative one in the largest complement)
                    none[e] = (v[0] > 0x7F80 ? 0x7FC0u : 0u) | (v[1] > 0x7F80 ? 0x7FC00000u : 0u);
                    const uint32_t y = __builtin_bit_cast(uint32_t, v);
                    out[e] = __builtin_bit_cast(uint32_t, ordered(lane < 32 ? y : ~y));
                }
                // a key that is none: no bound either
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const auto sw = __builtin_amdgcn_permlane32_swap(none[e], none[e], false, false);
                    out[e] |= sw[0] | sw[1];
                }
                if ((lane & 31) < 2) {
                    const int64_t bc = ((int64_t(page) * p.h_kv + g) * (p.page_tokens / p.block_tokens) +
                                        at / p.block_tokens) * kChunks + c0 + c;
                    *reinterpret_cast<u32x4_t*>(p.bounds + bc * 32 + (lane >> 5) * 16 + (lane & 1) * 8) = out;
                }
            }
        }
    }
}

// ---- selection
//
// A block's score for a query head is a sum over pairs of 2 products (positive parts of the query
// with the largest, negative ones with the smallest numbers), so the scores of 16 blocks and 16 columns
// (heads of one or more tokens of a row) are products of v_mfma_f32_16x16x32_bf16, one a chunk: its 32
// numbers of a block's record are the 32 of the sum.  With r = lane % 16, g = lane / 16: A row r is block
// r of the tile, the lane's 16 bytes its largest first, largest second, smallest first, smallest second
// components (g = 0 .. 3); the result gives the lane, for column r, blocks 4 g + v.
// Pairs kept at the whole of a tile's 16 blocks go in so; a pair whose window ends in the tile (each does in one
// tile of a row) has a product of its own, of which every block and column takes what its distance
// allows; chunks without a kept pair are not read.
//
// These sums are in fp32, off by no more than their error bound: the additions that a term goes through
// (a product's 32, then one a chunk or pair), each at most 2^-23 of the sum of magnitudes, which a
// second product has, and what fp32 loses below its smallest normal number.  pick_kernel finds the
// border of the blocks taken among them (those taken anyway, first or last, are not compared, and their magnitudes
// do not count: they may be any); blocks as near to it as the bound allows, mostly the one that
// is the border, are summed again in 64 bits unless all or none of them are taken.
//
// Bound by latency for single tokens (1,048,576 keys in 16,384 blocks, 28/4 heads of 128: scores 13 us, of
// which 12 MB of bounds are 2, the choice 8.6; summing every block in 64 bits took 326 in all), by
// vector work for turns (1,460 tokens against up to 516 blocks, 24/8 heads: 59 and 22 us, 4,097 in 64 bits).
// Tokens that share the columns of a product, and 16 blocks a tile, are what keeps the vector work per
// score small; the tile's bounds stay in registers, indexed by the pair whose window ends in it (through LDS
// they took 90 us where registers took 67, at three workgroups' room a CU).  The row's last tile, where
// most windows end, shared among a workgroup's waves: 31.9 us for 30.5 (24 rows), 88 for 83 (turns).
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4_t mfma16(u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                   __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
// The same of two numbers a lane, the others 0.
typedef short bf16x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ f32x4_t mfma16_pair(uint32_t a, uint32_t b) {
    typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(bf16x4_t, u32x2_t{a, 0u}),
                                                     __builtin_bit_cast(bf16x4_t, u32x2_t{b, 0u}),
                                                     f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
}
// pairs of a chunk that bits of `bits` keep
__device__ __forceinline__ u32x4_t keep_pairs(u32x4_t x, uint32_t bits) {
    u32x4_t r;
#pragma unroll
    for (int t = 0; t < 4; ++t)
        r[t] = x[t] & (((bits >> (2 * t)) & 1u ? 0x0000FFFFu : 0u) | ((bits >> (2 * t + 1)) & 1u ? 0xFFFF0000u : 0u));
    return r;
}

// What a query token sees: its row (-1: padding), its position, and the last key that it reaches (below
// 0: none).
struct Token {
    int row, pos, last;
};
__device__ __forceinline__ Token token_of(const SelectParams& p, int t) {
    const int row = p.token_rows[t], pos = min(p.positions[t], 0x7FFFFFFD);
    const bool is = row >= 0 && row < p.batch;
    const int keys = p.n_k_rows[is ? row : 0];
    return {is ? row : -1, pos, is ? min(min(max(keys, 0), p.max_n_k) - 1, pos) : -1};
}

// The bounds of block j of a row, for KV head g: the table's entry, and where they are by it.
__device__ __forceinline__ int page_of(const SelectParams& p, int row, int j) {
    return p.block_table[int64_t(row) * p.max_pages + uint32_t(j) / uint32_t(p.page_blocks)];
}
__device__ __forceinline__ const uint16_t* bounds_of(const SelectParams& p, int page, int g, int j) {
    const uint32_t per = uint32_t(p.page_blocks);
    page = min(max(page, 0), p.num_pages - 1);
    return p.bounds + ((int64_t(page) * p.h_kv + g) * per + uint32_t(j) % per) * p.chunks * 32;
}

// fp32 numbers as integers of the same order and back; what is not finite above all
__device__ __forceinline__ int key_of(float x) {
    const int v = __float_as_int(x);
    return (v & 0x7F800000) == 0x7F800000 ? 0x7FFFFFFF : v ^ ((v >> 31) & 0x7FFFFFFF);
}
__device__ __forceinline__ float value_of(int key) { return __int_as_float(key ^ ((key >> 31) & 0x7FFFFFFF)); }

template <int kCtrl>
__device__ __forceinline__ int max_dpp(int x, int none, bool take) {
    const int y = __builtin_amdgcn_update_dpp(none, x, kCtrl, 0xF, 0xF, false);
    return take ? max(x, y) : x;
}
// The largest of a lane and the G - 1 after it in the row of 16 (for the first of them, column h = 0).
__device__ __forceinline__ int max_columns(int x, int h, int G) {
    if (G > 1) x = max_dpp<0x101>(x, INT32_MIN, h + 1 < G);
    if (G > 2) x = max_dpp<0x102>(x, INT32_MIN, h + 2 < G);
    if (G > 4) x = max_dpp<0x104>(x, INT32_MIN, h + 4 < G);
    if (G > 8) x = max_dpp<0x108>(x, INT32_MIN, h + 8 < G);
    return x;
}

// The largest of the wave's lanes.
__device__ __forceinline__ int max_lanes(int x) {
    x = max_dpp<0x111>(x, INT32_MIN, true);  // up to each lane of a row of 16, then of the wave
    x = max_dpp<0x112>(x, INT32_MIN, true);
    x = max_dpp<0x114>(x, INT32_MIN, true);
    x = max_dpp<0x118>(x, INT32_MIN, true);
    x = max(x, __builtin_amdgcn_update_dpp(INT32_MIN, x, 0x142, 0xA, 0xF, false));
    x = max(x, __builtin_amdgcn_update_dpp(INT32_MIN, x, 0x143, 0xC, 0xF, false));
    return __builtin_amdgcn_readlane(x, 63);
}

// A wave: every `ranges`-th tile of 16 blocks, for the columns of `pack` tokens (of one row each time it goes
// through the tiles) or one token's heads, 16 at a time.  The queries' operands of the first kHeld times
// 16 columns are in LDS, the next tile's bounds on their way while a tile is multiplied.
constexpr int kHeld = 4;

template <int D>
__global__ __launch_bounds__(256, 3) void scores_kernel(const SelectParams p) {
    constexpr int kChunks = D / 16, kHalf = D / 2;
    __shared__ u32x4_t s_masks[256];  // keep_pairs' of each set of pairs
    extern __shared__ u32x4_t s_query[];  // [held][kChunks][64]
    const int lane = threadIdx.x & 63, r16 = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int range = blockIdx.x * 4 + wave;
    const int g = int(blockIdx.y) % p.h_kv, t0 = int(blockIdx.y) / p.h_kv * p.pack;  // (of the slab)
    const int G = p.group, width = min(G, 16);
    const int my_w = lane < kHalf ? p.W[lane] : -1;
    // this lane's column: head h (and 16 more of its token's each time) of token t
    const int at = r16 / width, h = r16 - at * width;
    const int t = t0 + at;
    const bool is = at < p.pack && t < p.tokens;
    // operand (column tile, chunk): the positive or the negative numbers of the columns' queries
    const auto query_of = [&](int h0, int c) __attribute__((always_inline)) {
        u32x4_t x = *reinterpret_cast<const u32x4_t*>(
            p.q + (int64_t(p.first_token + (is ? t : t0)) * p.h_q + g * G + (h0 + h < G ? h0 + h : 0)) * D +
            (g4 & 1) * kHalf + 8 * c);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] &= (((x[e] >> 15) & 0x00010001u) * 0xFFFFu) ^ (g4 >= 2 ? 0u : ~0u);
        return x;
    };
    // (what the loads do not need of each other is on its way at once: the first queries, the tokens, the
    // first tile's pages by the first token's row and any number of keys)
    u32x4_t early[kChunks / 4];
#pragma unroll
    for (int i = 0; i < kChunks / 4; ++i) early[i] = query_of(0, wave + 4 * i);
    Token tok = token_of(p, p.first_token + (is ? t : t0));
    const int early_row = max(__builtin_amdgcn_readfirstlane(tok.row), 0);
    const int early_page = page_of(p, early_row, min(16 * range + r16, p.row_blocks - 1));
    if (!is) tok = {-1, 0, -1};
    // blocks that the column's choice compares, from first_blocks on
    const uint32_t compared = uint32_t(max(0, tok.last / p.block_tokens + 1 - p.last_blocks - p.first_blocks));

    const int held = min((G + 15) / 16, kHeld);
    s_masks[threadIdx.x] = keep_pairs(u32x4_t{~0u, ~0u, ~0u, ~0u}, threadIdx.x);
#pragma unroll
    for (int i = 0; i < kChunks / 4; ++i) s_query[64 * (wave + 4 * i) + lane] = early[i];
    for (int o = wave + kChunks; o < held * kChunks; o += 4) s_query[64 * o + lane] = query_of(16 * (o / kChunks), o % kChunks);
    __syncthreads();
    if (range >= p.ranges) return;
    const auto query = [&](int h0, int c) __attribute__((always_inline)) {
        return h0 < 16 * kHeld ? s_query[(h0 / 16 * kChunks + c) * 64 + lane] : query_of(h0, c);
    };

    // registers of two pairs each
    const auto query_pairs = [&](int h0, int e) __attribute__((always_inline)) {
        if (h0 < 16 * kHeld) return reinterpret_cast<const uint32_t*>(&s_query[(h0 / 16 * kChunks + e / 4) * 64 + lane])[e % 4];
        const u32x4_t x = query_of(h0, e / 4);
        return e % 4 == 0 ? x[0] : e % 4 == 1 ? x[1] : e % 4 == 2 ? x[2] : x[3];
    };

    // signs of the bounds' magnitudes: those of the queries' parts
    const uint32_t minus = g4 >= 2 ? 0x80008000u : 0u;
    bool todo = is && tok.row >= 0 && tok.last >= 0;
    float worst = 0.f;  // largest sum of magnitudes times its additions, of the blocks compared
    for (uint64_t rest = __ballot(todo); rest != 0; rest = __ballot(todo)) {
        const int row = __builtin_amdgcn_readlane(tok.row, __builtin_ctzll(rest));
        const bool mine = todo && tok.row == row;
        todo = todo && !mine;
        int first_pos = 0x7FFFFFFF, last_pos = 0, last_key = -1;
        for (uint64_t m = __ballot(mine) & 0xFFFF; m != 0; m &= m - 1) {  // (16 columns, alike in the rows of lanes)
            const int l = __builtin_ctzll(m), pos = __builtin_amdgcn_readlane(tok.pos, l);
            first_pos = min(first_pos, pos);
            last_pos = max(last_pos, pos);
            last_key = max(last_key, __builtin_amdgcn_readlane(tok.last, l));
        }
        const int n = last_key / p.block_tokens + 1, tiles = (n + 15) / 16;
        if (range >= tiles) continue;
        const auto block_of = [&](int tile) __attribute__((always_inline)) { return min(16 * tile + r16, n - 1); };
        const auto keep_of = [&](int tile) __attribute__((always_inline)) {
            const int last = min(last_key, min(16 * tile + 15, n - 1) * p.block_tokens + (p.block_tokens - 1));
            return __ballot(my_w >= max(0, first_pos - last));
        };
        // (one vector, for an index that is not known when this is compiled)
        typedef uint32_t tile_t __attribute__((ext_vector_type(4 * kChunks)));
        tile_t a = {};
        const auto chunk = [&](int c) __attribute__((always_inline)) {
            return u32x4_t{a[4 * c], a[4 * c + 1], a[4 * c + 2], a[4 * c + 3]};
        };
        const auto load = [&](int tile, int page, uint64_t keep) __attribute__((always_inline)) {
            const uint16_t* src = bounds_of(p, page, g, block_of(tile)) + 8 * g4;
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
                if ((keep >> (8 * c)) & 0xFFull) {
                    const u32x4_t x = *reinterpret_cast<const u32x4_t*>(src + 32 * c);
#pragma unroll
                    for (int e = 0; e < 4; ++e) a[4 * c + e] = x[e];
                }
        };
        uint64_t keep = keep_of(range);
        load(range, row == early_row && 16 * range + 15 < n ? early_page : page_of(p, row, block_of(range)), keep);
        // (what is not looked at before the next tile's loads is not waited for with this one's)
        int next = page_of(p, row, block_of(min(range + p.ranges, tiles - 1)));
        for (int tile = range; tile < tiles; tile += p.ranges) {
            const int j0 = 16 * tile;
            uint64_t full = __ballot(my_w >= last_pos - j0 * p.block_tokens);
            const uint64_t some = keep & ~full;  // pairs whose windows end in the tile
            int best[4] = {INT32_MIN, INT32_MIN, INT32_MIN, INT32_MIN};
            for (int h0 = 0; h0 < G; h0 += 16) {
                const bool live = mine && h0 + h < G;
                asm volatile("" : "+s"(full));  // (its chunks' parts are not kept from one time to the next)
                f32x4_t sum = {0.f, 0.f, 0.f, 0.f}, size = sum;
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    const uint32_t whole = uint32_t(full >> (8 * c)) & 0xFFu;
                    if (whole == 0) continue;
                    u32x4_t x = chunk(c), y = query(h0, c);
                    if (whole != 0xFFu) {
                        x &= s_masks[whole];
                        y &= s_masks[whole];
                    }
                    // (a sum of its own for each chunk: fewer additions to a number)
                    sum += mfma16(x, y, f32x4_t{0.f, 0.f, 0.f, 0.f});
                    size = mfma16((x & 0x7FFF7FFFu) | minus, y, size);
                }
                for (uint64_t m = some; m != 0; m &= m - 1) {
                    const int r = __builtin_ctzll(m), w = __builtin_amdgcn_readlane(my_w, r);
                    // (a pair is half a register of each lane)
                    const uint32_t half = r & 1 ? 0xFFFF0000u : 0x0000FFFFu;
                    const uint32_t x = a[r / 2] & half, y = query_pairs(h0, r / 2) & half;
                    const f32x4_t u = mfma16_pair(x, y);
                    const f32x4_t v = mfma16_pair((x & 0x7FFF7FFFu) | (minus & half), y);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        // (a tile past the row's end may reach past 2^31: wrapped, and not written)
                        const int first = int(uint32_t(j0 + 4 * g4 + i) * uint32_t(p.block_tokens));
                        const bool kept = w >= tok.pos - min(int(uint32_t(first) + uint32_t(p.block_tokens - 1)), tok.last);
                        // (a window that ends inside the block: no less than 0)
                        const float x0 = w < tok.pos - first && u[i] < 0.f ? 0.f : u[i];
                        if (kept) sum[i] += x0;
                        if (kept) size[i] += v[i];
                    }
                }
                // additions that a term goes through: those of a product of 32, the chunks', the pairs'
                const float steps = float(32 + kChunks + __builtin_popcountll(some));
                if (h0 + 16 >= G && tile + p.ranges < tiles) {  // the tile is done with
                    keep = keep_of(tile + p.ranges);
                    load(tile + p.ranges, next, keep);
                    next = page_of(p, row, block_of(min(tile + 2 * p.ranges, tiles - 1)));
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (live) best[i] = max(best[i], key_of(sum[i]));
                    if (live && uint32_t(j0 + 4 * g4 + i - p.first_blocks) < compared) worst = fmaxf(worst, size[i] * steps);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) best[i] = max_columns(best[i], h, width);
            if (mine && h == 0)
                *reinterpret_cast<int4*>(p.keys + (int64_t(t) * p.h_kv + g) * p.key_stride + j0 + 4 * g4) =
                    make_int4(best[0], best[1], best[2], best[3]);
        }
    }
    // (not less than 0: its bits are in order)
    int bound = max_columns(__float_as_int(worst), h, width);
    bound = max(bound, __shfl_xor(bound, 16));
    bound = max(bound, __shfl_xor(bound, 32));
    if (is && h == 0 && g4 == 0) p.sizes[(int64_t(t) * p.h_kv + g) * p.ranges + range] = __int_as_float(bound);
}

__device__ __forceinline__ double widen(uint16_t x) { return double(__uint_as_float(uint32_t(x) << 16)); }

// The sum over the wave's lanes.
template <int kCtrl, int kRows>
__device__ __forceinline__ double add_dpp(double x) {
    const int64_t v = __double_as_longlong(x);
    const int lo = __builtin_amdgcn_update_dpp(0, int(v), kCtrl, kRows, 0xF, false);
    const int hi = __builtin_amdgcn_update_dpp(0, int(v >> 32), kCtrl, kRows, 0xF, false);
    return x + __longlong_as_double(int64_t(hi) << 32 | uint32_t(lo));
}
__device__ __forceinline__ double add_lanes(double x) {
    x = add_dpp<0x111, 0xF>(x);  // as scan::wave
    x = add_dpp<0x112, 0xF>(x);
    x = add_dpp<0x114, 0xF>(x);
    x = add_dpp<0x118, 0xF>(x);
    x = add_dpp<0x142, 0xA>(x);
    x = add_dpp<0x143, 0xC>(x);
    return __longlong_as_double(scan::lane_of(int64_t(__double_as_longlong(x)), 63));
}

// The score of block j in 64 bits, as an integer of the same order, NaN above all; a pair a lane.
constexpr uint64_t kNaN = ~0ull;
__device__ __forceinline__ uint64_t exact_key(const SelectParams& p, const Token& tok, int t, int g, int j) {
    const int lane = threadIdx.x & 63, d = p.chunks * 16, half = d / 2;
    const int first = j * p.block_tokens;
    const int far = tok.pos - first, near = tok.pos - min(first + (p.block_tokens - 1), tok.last);
    const int w = lane < half ? p.W[lane] : -1;
    const bool kept = lane < half && w >= near;
    const uint16_t* at = bounds_of(p, page_of(p, tok.row, j), g, j) + lane / 8 * 32 + lane % 8;
    double hi0 = 0, hi1 = 0, lo0 = 0, lo1 = 0;
    if (kept) hi0 = widen(at[0]), hi1 = widen(at[8]), lo0 = widen(at[16]), lo1 = widen(at[24]);
    double best = 0;
    bool none = false;
    const int pair = min(lane, half - 1);
#pragma unroll 4
    for (int h = 0; h < p.group; ++h) {
        const uint16_t* q = p.q + (int64_t(t) * p.h_q + g * p.group + h) * d;
        const double q0 = widen(q[pair]), q1 = widen(q[pair + half]);
        double u = 0;
        if (kept) {
            // (a query that is none stays so)
            u = (q0 < 0 ? 0 : q0) * hi0 + (q0 > 0 ? 0 : q0) * lo0;
            u += (q1 < 0 ? 0 : q1) * hi1 + (q1 > 0 ? 0 : q1) * lo1;
            if (w < far && u < 0) u = 0;
        }
        u = add_lanes(u);
        none = none || u != u;
        best = h == 0 || u > best ? u : best;
    }
    if (none) return kNaN;
    const int64_t v = __double_as_longlong(best + 0.0);
    return uint64_t(v ^ ((v >> 63) & 0x7FFFFFFFFFFFFFFFll)) ^ 0x8000000000000000ull;
}

// The blocks of one token for one KV head.  A thread's kPer keys, one behind the other, stay in registers;
// 0: they are read again each time.
template <int kThreads>
struct PickShared {
    static constexpr int kBits = kThreads == 64 ? 9 : 11, kBins = 1 << kBits;
    // blocks that are ranked, or summed again, one against another
    static constexpr int kListed = kThreads < 256 ? kThreads : 256;
    int hist[kBins];
    int part[2][kThreads / 64];
    int low[kThreads / 64], high[kThreads / 64];
    float size[kThreads / 64];
    int bin, above, inside;
    int listed, sure, maybe;
    int border;
    int list[kListed], key[kListed];
    uint64_t exact[kListed];
    uint8_t win[kListed];
};

// Blocks j where take(j), in order, one behind the other: a step of kThreads blocks at a time.
template <int kThreads, typename Take>
__device__ __forceinline__ void write_taken(int32_t* out, int top, int n, PickShared<kThreads>& s, Take take) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int taken = 0;
    for (int i = 0; i * kThreads < n; ++i) {
        const int j = i * kThreads + tid;
        const bool yes = j < n && take(j);
        const uint64_t m = __ballot(yes);
        if (lane == 0) s.part[i & 1][wave] = __builtin_popcountll(m);
        __syncthreads();
        int at = taken + __builtin_popcountll(m & ((1ull << lane) - 1));
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) {
            at += w < wave ? s.part[i & 1][w] : 0;
            taken += s.part[i & 1][w];
        }
        if (yes && at < top) out[at] = j;
    }
}

// Every block's score in 64 bits, the border found 8 bits at a time: where fp32 tells nothing (numbers
// that are not finite, many equal blocks).  Bound by the latency of a wave's blocks one behind the other (16,384
// blocks of 7 heads, 16 waves: 4.2 ms).
template <int kThreads>
__device__ __forceinline__ void pick_exact(const SelectParams& p, const Token& tok, int t, int g, int n, int want,
                                                     uint64_t* keys, int32_t* out, PickShared<kThreads>& s) {
    const int tid = threadIdx.x, lane = tid & 63;
    const auto forced = [&](int j) { return j < p.first_blocks || j >= n - p.last_blocks; };
    __syncthreads();
    for (int j = __builtin_amdgcn_readfirstlane(tid >> 6); j < n; j += kThreads / 64) {
        if (forced(j)) continue;
        const uint64_t k = exact_key(p, tok, t, g, j);
        if (lane == 0) keys[j] = k;
    }
    uint64_t prefix = 0;
    int left = want;  // of the keys that begin with the prefix
    for (int shift = 56; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kThreads) s.hist[i] = 0;
        __syncthreads();
        for (int j = tid; j < n; j += kThreads)
            if (!forced(j) && (shift == 56 || (keys[j] >> (shift + 8)) == (prefix >> (shift + 8))))
                atomicAdd(&s.hist[(keys[j] >> shift) & 255], 1);
        __syncthreads();
        if (tid == 0) {
            int rest = left, v = 255;
            while (rest > s.hist[v]) rest -= s.hist[v--];
            s.bin = v;
            s.above = rest;
        }
        __syncthreads();
        prefix |= uint64_t(s.bin) << shift;
        left = s.above;
        __syncthreads();
    }
    // the equal ones from the first: their number before block j counts as it goes
    int equal = 0;
    const int wave = tid >> 6;
    int taken = 0;
    for (int j0 = 0; j0 < n; j0 += kThreads) {
        const int j = j0 + tid;
        const bool free = j < n && !forced(j), is = free && keys[j] == prefix;
        const uint64_t eq = __ballot(is);
        if (lane == 0) s.part[0][wave] = __builtin_popcountll(eq);
        __syncthreads();
        int before = equal + __builtin_popcountll(eq & ((1ull << lane) - 1));
        for (int w = 0; w < kThreads / 64; ++w) {
            before += w < wave ? s.part[0][w] : 0;
            equal += s.part[0][w];
        }
        const bool yes = j < n && (!free || keys[j] > prefix || (is && before < left));
        const uint64_t m = __ballot(yes);
        if (lane == 0) s.part[1][wave] = __builtin_popcountll(m);
        __syncthreads();
        int at = taken + __builtin_popcountll(m & ((1ull << lane) - 1));
        for (int w = 0; w < kThreads / 64; ++w) {
            at += w < wave ? s.part[1][w] : 0;
            taken += s.part[1][w];
        }
        if (yes && at < p.top) out[at] = j;
        __syncthreads();
    }
}

template <int kThreads, int kPer>
__global__ __launch_bounds__(kThreads) void pick_kernel(const SelectParams p) {
    constexpr int kWaves = kThreads / 64;
    constexpr int kBits = PickShared<kThreads>::kBits, kBins = PickShared<kThreads>::kBins;
    constexpr int kListed = PickShared<kThreads>::kListed;
    __shared__ PickShared<kThreads> s;
    __shared__ int s_scan[1][kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int slab_t = int(blockIdx.x) / p.h_kv, g = int(blockIdx.x) % p.h_kv, t = p.first_token + slab_t;
    const Token tok = token_of(p, t);
    if (tok.row < 0) return;
    int32_t* out = p.blocks + (int64_t(t) * p.h_kv + g) * p.top;
    const int n = tok.last < 0 ? 0 : tok.last / p.block_tokens + 1;
    if (n <= p.top) {
        for (int i = tid; i < p.top; i += kThreads) out[i] = i < n ? i : -1;
        return;
    }
    const int64_t at = int64_t(slab_t) * p.h_kv + g;
    const int* keys = p.keys + at * p.key_stride;
    const int want = p.top - p.first_blocks - p.last_blocks;
    // blocks that are taken anyway have the lowest key, which no score has
    const auto load = [&](int j) { return j >= p.first_blocks && j < n - p.last_blocks ? keys[j] : INT32_MIN; };
    [[maybe_unused]] int kept[kPer > 0 ? kPer : 1];
    if constexpr (kPer > 0) {
        const int j0 = tid * kPer;
        int4 x[kPer / 4] = {};
        if (j0 < n)  // (the row's keys fill up to 16)
#pragma unroll
            for (int i = 0; i < kPer / 4; ++i) x[i] = *reinterpret_cast<const int4*>(keys + j0 + 4 * i);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int j = j0 + i, k = i % 4 == 0 ? x[i / 4].x : i % 4 == 1 ? x[i / 4].y : i % 4 == 2 ? x[i / 4].z : x[i / 4].w;
            kept[i] = j >= p.first_blocks && j < n - p.last_blocks ? k : INT32_MIN;
        }
    }
    for (int i = tid; i < kBins; i += kThreads) s.hist[i] = 0;
    float size = p.sizes[at * p.ranges + min(tid, p.ranges - 1)];  // (on its way with the keys)
    const auto each = [&](auto body) __attribute__((always_inline)) {
        if constexpr (kPer > 0) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                asm volatile("" : "+v"(kept[i]));  // (its comparisons are not kept from one time to the next)
                body(tid * kPer + i, kept[i]);
            }
        } else {
            for (int j = tid; j < n; j += kThreads) body(j, load(j));
        }
    };
    // lo <= k <= hi, lo above the lowest key, in one comparison
    const auto within = [](int k, int lo, int hi) __attribute__((always_inline)) {
        return uint32_t(k) - uint32_t(lo) <= uint32_t(hi) - uint32_t(lo);
    };
    // extremes (the lowest key comes last among those so counted), and the error bound
    constexpr uint32_t kLast = 0x80000001u;
    uint32_t least = ~0u;
    int high = INT32_MIN;
    each([&](int, int k) __attribute__((always_inline)) {
        least = min(least, uint32_t(k) - kLast);
        high = max(high, k);
    });
    int low = int(least + kLast);
    if (least == ~0u) low = INT32_MAX;
    for (int i = tid + kThreads; i < p.ranges; i += kThreads) size = fmaxf(size, p.sizes[at * p.ranges + i]);
    low = ~max_lanes(~low);  // (the complement is in the opposite order)
    high = max_lanes(high);
    size = __int_as_float(max_lanes(__float_as_int(size)));
    if (lane == 0) s.low[wave] = low, s.high[wave] = high, s.size[wave] = size;
    if (tid == 0) s.listed = s.sure = s.maybe = 0;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) {
        low = min(low, s.low[w]);
        high = max(high, s.high[w]);
        size = fmaxf(size, s.size[w]);
    }
    // each addition is off by 2^-23 of the magnitudes' sum at most; that, and its product with their
    // number, by less than 2^-10; and the products and additions, fewer than 2^10, that come out below the
    // smallest normal number by no more than that, 2^-126, each
    const double error = double(size) * (0x1p-23 * (1 + 0x1p-10)) + 0x1p-115;
    bool exact = want > 0 && (high == INT32_MAX || !(error < 1e300));
    // of the keys of scores that may be as large as one of key k, the lowest; as small, the highest (the
    // numbers of fp32 next to the limits on their inner sides)
    const auto lowest_of = [&](int k) __attribute__((always_inline)) {
        const double x = double(value_of(k)) - 2 * error;
        const int y = key_of(float(x));
        return y == INT32_MAX ? INT32_MIN + 1 : y + (double(float(x)) < x);
    };
    const auto highest_of = [&](int k) __attribute__((always_inline)) {
        const double x = double(value_of(k)) + 2 * error;
        const int y = key_of(float(x));
        return y - (double(float(x)) > x && y != INT32_MAX);
    };

    int above = INT32_MAX, from = INT32_MAX;  // blocks over `above` are taken, those from `from` on maybe
    bool all = want > 0;                      // the latter all are
    if (want > 0 && !exact) {
        // the bin of the border, and so on in it until the blocks that may be at the border can be listed
        int left = want, listed;
        for (;;) {
            const uint32_t reach = uint32_t(high) - uint32_t(low);
            const int shift = max(0, 32 - kBits - __builtin_clz(reach | 1));
            each([&](int, int k) __attribute__((always_inline)) {
                if (within(k, low, high)) atomicAdd(&s.hist[(uint32_t(k) - uint32_t(low)) >> shift], 1);
            });
            __syncthreads();
            // the bin where `left` is reached, from the highest
            constexpr int kOwn = kBins / kThreads;
            int own[kOwn], sum = 0;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) sum += own[i] = s.hist[kBins - 1 - (tid * kOwn + i)];
            int upto[1] = {sum}, total[1];
            scan::block<kWaves>(upto, total, s_scan);
            int before = upto[0] - sum;
            if (before < left && left <= upto[0]) {
#pragma unroll
                for (int i = 0; i < kOwn; ++i) {
                    if (before < left && left <= before + own[i]) {
                        s.bin = kBins - 1 - (tid * kOwn + i);
                        s.above = before;
                        s.inside = own[i];
                    }
                    before += own[i];
                }
            }
            __syncthreads();
            left -= s.above;
            low = int(uint32_t(low) + (uint32_t(s.bin) << shift));
            high = min(high, int(uint32_t(low) + ((1u << shift) - 1)));
            from = lowest_of(low);
            above = highest_of(high);
            listed = s.inside;
            if (listed <= kListed) {
                int sure = 0;
                each([&](int j, int k) __attribute__((always_inline)) {
                    sure += k > above;
                    if (within(k, from, above)) {
                        const int i = atomicAdd(&s.listed, 1);
                        if (i < kListed) s.list[i] = j, s.key[i] = k;
                    }
                });
                sure = scan::lane_of(scan::wave(sure), 63);
                if (lane == 0 && sure > 0) atomicAdd(&s.sure, sure);
                __syncthreads();
                listed = s.listed;
            }
            if (listed <= kListed || shift == 0) break;
            for (int i = tid; i < kBins; i += kThreads) s.hist[i] = 0;
            __syncthreads();
            if (tid == 0) s.listed = s.sure = 0;
        }
        exact = listed > kListed;
        if (!exact) {
            // the border: the key whose place is the last one taken
            const int sure = s.sure, mine = tid < listed ? s.key[tid] : INT32_MIN;
            if (tid < listed) {
                int over = sure, same = 0;
                for (int i = 0; i < listed; ++i) {
                    over += s.key[i] > mine;
                    same += s.key[i] == mine;
                }
                if (over < want && want <= over + same) s.border = mine;
            }
            __syncthreads();
            from = lowest_of(s.border);
            above = highest_of(s.border);
            const int over = __builtin_popcountll(__ballot(tid < listed && mine > above));
            const int maybe = __builtin_popcountll(__ballot(tid < listed && within(mine, from, above)));
            if (lane == 0 && over > 0) atomicAdd(&s.sure, over);
            if (lane == 0 && maybe > 0) atomicAdd(&s.maybe, maybe);
            __syncthreads();
            const int rest = want - s.sure;
            all = s.maybe == rest;
            if (!all) {
                for (int i = wave; i < listed; i += kWaves) {
                    if (!within(__builtin_amdgcn_readfirstlane(s.key[i]), from, above)) continue;
                    const uint64_t k = exact_key(p, tok, t, g, __builtin_amdgcn_readfirstlane(s.list[i]));
                    if (lane == 0) s.exact[i] = k;
                }
                __syncthreads();
                if (tid < listed) {
                    bool win = false;
                    if (within(mine, from, above)) {
                        int better = 0;
                        for (int i = 0; i < listed; ++i)
                            better += within(s.key[i], from, above) &&
                                      (s.exact[i] > s.exact[tid] || (s.exact[i] == s.exact[tid] && s.list[i] < s.list[tid]));
                        win = better < rest;
                    }
                    s.win[tid] = win;
                }
                __syncthreads();
            }
        }
    }
    if (exact) {
        pick_exact<kThreads>(p, tok, t, g, n, want, p.exact_keys + at * p.key_stride, out, s);
        return;
    }
    if constexpr (kPer > 0) {
        // which of a thread's blocks are taken: those taken anyway, those over a limit, and the listed ones
        // that won
        const auto below = [&](int j) __attribute__((always_inline)) { return (1u << min(max(j - tid * kPer, 0), kPer)) - 1; };
        uint32_t taken = below(n) & (below(p.first_blocks) | ~below(n - p.last_blocks));
        const int limit = all ? from - 1 : above;
#pragma unroll
        for (int i = 0; i < kPer; ++i) taken |= uint32_t(kept[i] > limit) << i;
        if (!all && want > 0)
            for (int i = 0; i < s.listed; ++i) {
                const int j = s.list[i];
                if (j / kPer == tid && s.win[i]) taken |= 1u << (j % kPer);
            }
        int upto[1] = {int(__builtin_popcount(taken))}, total[1];
        int to = -upto[0];
        scan::block<kWaves>(upto, total, s_scan);
        to += upto[0];
        for (; taken != 0; taken &= taken - 1, ++to)
            if (to < p.top) out[to] = tid * kPer + __builtin_ctz(taken);
    } else {
        write_taken<kThreads>(out, p.top, n, s, [&](int j) __attribute__((always_inline)) {
            const int k = load(j);
            if (k == INT32_MIN || k > above) return true;
            bool yes = all;
            if (k >= from && !all && want > 0)
                for (int i = 0; i < s.listed; ++i) yes = yes || (s.list[i] == j && s.win[i]);
            return k >= from && yes;
        });
    }
}

}  // namespace

hipError_t launch_block_bounds(const BoundsParams& p, int head_dim, hipStream_t stream) {
    (void)hipGetLastError();
    const uint64_t units = uint64_t(p.row_blocks) * uint64_t(p.h_kv) * uint64_t(head_dim / 16 / kBoundChunks);
    if (units > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
    // (a grid has fewer than 2^32 threads)
    const dim3 grid(unsigned(std::min<uint64_t>((units + 3) / 4, 1u << 13)), unsigned(std::min(p.batch, 1 << 10)));
    if (head_dim == 64)
        hipLaunchKernelGGL(block_bounds_kernel<64>, grid, dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL(block_bounds_kernel<128>, grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_select_blocks(const SelectParams& all, hipStream_t stream) {
    (void)hipGetLastError();
    SelectParams p = all;
    for (int32_t t = 0; t < all.n_tokens; t += all.slab) {
        p.first_token = t;
        p.tokens = std::min(all.slab, all.n_tokens - t);
        const unsigned groups = unsigned((p.tokens + p.pack - 1) / p.pack) * unsigned(p.h_kv);
        const dim3 grid(unsigned((p.ranges + 3) / 4), groups);
        const size_t queries = size_t(std::min((p.group + 15) / 16, kHeld)) * size_t(p.chunks) * 1024;
        if (p.chunks == 4)
            hipLaunchKernelGGL(scores_kernel<64>, grid, dim3(256), queries, stream, p);
        else
            hipLaunchKernelGGL(scores_kernel<128>, grid, dim3(256), queries, stream, p);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        const dim3 picks(unsigned(p.tokens) * unsigned(p.h_kv));
        // A wave a pick where they are many (us of a selection, picks by 256 threads and by 64; 24/8 heads, 516
        // blocks: 1,008 picks 28.2 and 29.5, 2,040 34.2 and 33.6, 8,184 81.5 and 71.9; 94 blocks: 24.7 and 26.7,
        // 23.2 and 22.9, 53.6 and 43.0; 14/2 heads of 64, 938 blocks: 2,046 57.5 and 57.5, 4,092 79.6 and 78.6).
        // Past 16,384 blocks a row a thread's keys have no room in registers (32,768 blocks of 4 heads: 47 us; 8.5
        // for 16,384)
        if (p.row_blocks <= 1024 && picks.x > 2048)
            hipLaunchKernelGGL((pick_kernel<64, 16>), picks, dim3(64), 0, stream, p);
        else if (p.row_blocks <= 1024)
            hipLaunchKernelGGL((pick_kernel<256, 4>), picks, dim3(256), 0, stream, p);
        else if (p.row_blocks <= 4096)
            hipLaunchKernelGGL((pick_kernel<256, 16>), picks, dim3(256), 0, stream, p);
        else if (p.row_blocks <= 16384)
            hipLaunchKernelGGL((pick_kernel<1024, 16>), picks, dim3(1024), 0, stream, p);
        else
            hipLaunchKernelGGL((pick_kernel<1024, 0>), picks, dim3(1024), 0, stream, p);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace atf
