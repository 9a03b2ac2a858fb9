// Bounds of the keys of each block of a row, and the blocks that a query takes by them, gfx950.
#include "atf_internal.hpp"

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
// Bound by HBM reads.
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
                        x[c][h] = *reinterpret_cast<const u32x4_t*>(
                            src + (int64_t(c) * p.page_tokens + min(t0 + 32 * h + (lane >> 1), last)) * 16);
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

// What a query token sees: its row, its position, and the last key that it reaches (-1: none).
struct Token {
    int row, pos, last;
};
__device__ __forceinline__ Token token_of(const SelectParams& p, int t) {
    Token x = {p.token_rows[t], p.positions[t], -1};
    if (x.row < 0 || x.row >= p.batch) {
        x.row = -1;
        return x;
    }
    x.pos = min(x.pos, 0x7FFFFFFD);
    x.last = min(min(max(p.n_k_rows[x.row], 0), p.max_n_k) - 1, x.pos);
    return x;
}

// The bounds of block j of a row, for KV head g.
__device__ __forceinline__ const uint16_t* bounds_of(const SelectParams& p, int row, int g, int j) {
    const int per = p.page_tokens / p.block_tokens;
    const int page = min(max(p.block_table[int64_t(row) * p.max_pages + j / per], 0), p.num_pages - 1);
    return p.bounds + ((int64_t(page) * p.h_kv + g) * per + j % per) * p.chunks * 32;
}

__device__ __forceinline__ double widen(uint16_t x) { return double(__uint_as_float(uint32_t(x) << 16)); }

// A score as an integer of the same order: NaN above all, forced blocks above that; 0 is none.
constexpr uint64_t kForced = ~0ull, kNaN = ~0ull - 1;
__device__ __forceinline__ uint64_t key_of(double x) {
    if (x != x) return kNaN;
    const int64_t v = __double_as_longlong(x + 0.0);
    return uint64_t(v ^ ((v >> 63) & 0x7FFFFFFFFFFFFFFFll)) ^ 0x8000000000000000ull;
}

// Scores of one query token's blocks for one KV head, a block a thread, in 64 bits.
__global__ __launch_bounds__(256) void scores_kernel(const SelectParams p) {
    extern __shared__ double s_q[];  // [head][d]
    __shared__ int s_w[kMaxPairs];
    const int d = p.chunks * 16, half = d / 2;
    const int t = p.first_token + int(blockIdx.y) / p.h_kv, g = int(blockIdx.y) % p.h_kv;
    const Token tok = token_of(p, t);
    if (tok.row < 0 || tok.last < 0) return;
    const int n = tok.last / p.block_tokens + 1;
    if (int64_t(blockIdx.x) * 256 >= n) return;
    for (int i = threadIdx.x; i < p.group * d; i += 256)
        s_q[i] = widen(p.q[(int64_t(t) * p.h_q + g * p.group) * d + i]);
    if (threadIdx.x < half) s_w[threadIdx.x] = p.W[threadIdx.x];
    __syncthreads();
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j >= n) return;
    const uint16_t* bounds = bounds_of(p, tok.row, g, j);
    const int near = tok.pos - min(j * p.block_tokens + (p.block_tokens - 1), tok.last);
    const int far = tok.pos - j * p.block_tokens;
    double best = 0;
    bool none = false;
    for (int h = 0; h < p.group; ++h) {
        double sum = 0;
        for (int r = 0; r < half; ++r) {
            if (s_w[r] < near) continue;
            const uint16_t* at = bounds + (r / 8) * 32 + r % 8;
            const double q0 = s_q[h * d + r], q1 = s_q[h * d + half + r];
            double u = fmax(q0, 0.0) * widen(at[0]) + fmin(q0, 0.0) * widen(at[16]);
            u += fmax(q1, 0.0) * widen(at[8]) + fmin(q1, 0.0) * widen(at[24]);
            if (s_w[r] < far && u < 0) u = 0;  // some of the block's keys are past the pair's window
            sum += u;
        }
        none = none || sum != sum;
        best = h == 0 ? sum : fmax(best, sum);
    }
    uint64_t key = none ? kNaN : key_of(best);
    if (j < p.first_blocks || j >= n - p.last_blocks) key = kForced;
    p.keys[(int64_t(blockIdx.y)) * p.row_blocks + j] = key;
}

// The largest keys of a token's blocks for one KV head, in the order of the blocks; equal ones from
// the first.  The smallest key taken is found 8 bits at a time.
constexpr int kPickThreads = 256;
__global__ __launch_bounds__(kPickThreads) void pick_kernel(const SelectParams p) {
    __shared__ int s_hist[256];
    __shared__ int s_part[2][kPickThreads / 64];
    __shared__ uint64_t s_prefix;
    __shared__ int s_left;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int t = p.first_token + int(blockIdx.x) / p.h_kv, g = int(blockIdx.x) % p.h_kv;
    const Token tok = token_of(p, t);
    if (tok.row < 0) return;
    int32_t* out = p.blocks + (int64_t(t) * p.h_kv + g) * p.top;
    const int n = tok.last < 0 ? 0 : tok.last / p.block_tokens + 1;
    if (n <= p.top) {
        for (int i = tid; i < p.top; i += kPickThreads) out[i] = i < n ? i : -1;
        return;
    }
    const uint64_t* keys = p.keys + int64_t(blockIdx.x) * p.row_blocks;
    uint64_t prefix = 0;
    int left = p.top;  // of the keys that begin with the prefix
    for (int shift = 56; shift >= 0; shift -= 8) {
        s_hist[tid] = 0;
        __syncthreads();
        for (int j = tid; j < n; j += kPickThreads) {
            const uint64_t k = keys[j];
            if (shift == 56 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&s_hist[(k >> shift) & 255], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int rest = left, v = 255;
            while (rest > s_hist[v]) rest -= s_hist[v--];
            s_prefix = prefix | uint64_t(v) << shift;
            s_left = rest;
        }
        __syncthreads();
        prefix = s_prefix;
        left = s_left;
    }
    // above the border all, at the border the first `left`
    int taken = 0, equal = 0;
    for (int j0 = 0; j0 < n; j0 += kPickThreads) {
        const int j = j0 + tid;
        const uint64_t k = j < n ? keys[j] : 0;
        const bool is = j < n && k == prefix;
        const uint64_t eq = __ballot(is);
        __syncthreads();
        if (lane == 0) s_part[0][wave] = __builtin_popcountll(eq);
        __syncthreads();
        int before = equal + __builtin_popcountll(eq & ((1ull << lane) - 1));
        for (int w = 0; w < kPickThreads / 64; ++w) {
            before += w < wave ? s_part[0][w] : 0;
            equal += s_part[0][w];
        }
        const bool take = (j < n && k > prefix) || (is && before < left);
        const uint64_t tk = __ballot(take);
        if (lane == 0) s_part[1][wave] = __builtin_popcountll(tk);
        __syncthreads();
        int at = taken + __builtin_popcountll(tk & ((1ull << lane) - 1));
        for (int w = 0; w < kPickThreads / 64; ++w) {
            at += w < wave ? s_part[1][w] : 0;
            taken += s_part[1][w];
        }
        if (take) out[at] = j;
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
        const int32_t tokens = std::min(all.slab, all.n_tokens - t);
        const dim3 grid(unsigned((p.row_blocks + 255) / 256), unsigned(tokens * p.h_kv));
        hipLaunchKernelGGL(scores_kernel, grid, dim3(256), size_t(p.group) * p.chunks * 16 * 8, stream, p);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(pick_kernel, dim3(unsigned(tokens * p.h_kv)), dim3(kPickThreads), 0, stream, p);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace atf
