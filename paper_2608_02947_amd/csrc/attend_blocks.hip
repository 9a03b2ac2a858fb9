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
// and at every token: chunks without a kept pair are not read; keys lose the pairs kept nowhere, so
// that a number that is none does not count there; where a window ends inside the tile they are
// masked token by token.
#include "atf_internal.hpp"

namespace atf {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kTile = 32;

__device__ __forceinline__ f32x4_t mfma16(u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                   __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ u32x4_t load16(uint64_t at) {
    return *(const __attribute__((address_space(1))) u32x4_t*)(at);
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// halves of a register pair of bf16 numbers that bits 2t, 2t + 1 keep
__device__ __forceinline__ uint32_t pair_mask(uint32_t bits, int t) {
    return ((bits >> (2 * t)) & 1u ? 0x0000FFFFu : 0u) | ((bits >> (2 * t + 1)) & 1u ? 0xFFFF0000u : 0u);
}
__device__ __forceinline__ u32x4_t keep_pairs(u32x4_t x, uint32_t bits) {
    return u32x4_t{x[0] & pair_mask(bits, 0), x[1] & pair_mask(bits, 1), x[2] & pair_mask(bits, 2),
                   x[3] & pair_mask(bits, 3)};
}

template <int D, int NT, int NW>
__global__ __launch_bounds__(NW * 64, 2) void attend_blocks_kernel(const AttendParams p) {
    constexpr int kChunks = D / 16;
    constexpr int kHalf = D / 2;
    constexpr int kM = D / 32;   // products of a score: 2 chunks each
    constexpr int kDB = D / 16;  // 16-dim blocks of the output
    constexpr int kOps = kM * NT;
    constexpr int kOStride = D + 4;
    __shared__ float red_m[NW][16 * NT];
    __shared__ float red_l[NW][16 * NT];
    __shared__ int s_w[kHalf];
    __shared__ __attribute__((aligned(16))) float s_o[NW * 16 * kOStride];

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15;
    const int g4 = lane >> 4;
    const int cols = p.h_kv * p.subgroups;
    const int t = int(blockIdx.x) / cols;
    const int col = int(blockIdx.x) % cols;
    const int g = col / p.subgroups, sub = col % p.subgroups;
    const int hq0 = g * p.group + sub * p.heads_per_block;
    const int NH = min(p.heads_per_block, p.group - sub * p.heads_per_block);

    const int row = __builtin_amdgcn_readfirstlane(p.token_rows[t]);
    if (row < 0 || row >= p.batch) return;  // padding: nothing of it is written
    const int q_pos = __builtin_amdgcn_readfirstlane(min(p.positions[t], 0x7FFFFFFD));
    // the last key (below 0: none)
    const int last = min(min(max(__builtin_amdgcn_readfirstlane(p.n_k_rows[row]), 0), p.max_n_k) - 1, q_pos);

    const int my_w = lane < kHalf ? p.W[lane] : -1;
    if (tid < kHalf) s_w[tid] = my_w;
    // queries: operand (tile n, m)
    u32x4_t qf[kOps];
#pragma unroll
    for (int o = 0; o < kOps; ++o) {
        const int h = 16 * (o / kM) + r16, m = o % kM;
        qf[o] = u32x4_t{0u, 0u, 0u, 0u};
        if (h < NH)
            qf[o] = *reinterpret_cast<const u32x4_t*>(p.q + (int64_t(t) * p.h_q + hq0 + h) * D + (g4 & 1) * kHalf +
                                                      8 * (2 * m + (g4 >> 1)));
    }
    __syncthreads();

    f32x4_t oacc[NT][kDB];
    float m_run[NT], l_run[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int i = 0; i < kDB; ++i) oacc[n][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        m_run[n] = -INFINITY;
        l_run[n] = 0.f;
    }
    const float sc = p.scale_log2;
    const int tk = 16 * (r16 >> 3) + 4 * ((r16 >> 2) & 1) + (r16 & 3);  // this lane's token of s = 0

    // tiles of the list: every NW-th is this wave's; a lane looks one up, 64 at a time
    const int per = p.block_tokens / kTile, tiles = p.top * per;
    const int32_t* list = p.blocks + (int64_t(t) * p.h_kv + g) * p.top;
    for (int i0 = wave; i0 < tiles; i0 += 64 * NW) {
        const int i = i0 + NW * lane;
        int my_page = 0, my_at = 0, my_tb = -1;
        if (i < tiles) {
            const int j = list[i / per];
            if (j >= 0 && last >= 0 && j <= last / p.block_tokens) {
                const int tb = j * p.block_tokens + (i % per) * kTile;
                if (tb <= last) {
                    my_tb = tb;
                    my_page = min(max(p.block_table[int64_t(row) * p.max_pages + tb / p.page_tokens], 0), p.num_pages - 1);
                    my_at = tb % p.page_tokens;
                }
            }
        }
        uint64_t todo = __ballot(my_tb >= 0);
        while (todo) {
            const int l = __builtin_ctzll(todo);
            todo &= todo - 1;
            const int page = __builtin_amdgcn_readlane(my_page, l), at = __builtin_amdgcn_readlane(my_at, l);
            const int tb = __builtin_amdgcn_readlane(my_tb, l);
            const int left = last - tb;  // the tile's last token that counts, if below 31
            const uint64_t full = __ballot(my_w >= q_pos - tb);
            const uint64_t keep = __ballot(my_w >= q_pos - tb - min(left, kTile - 1));
            const int64_t ph = int64_t(page) * p.h_kv + g;
            const uint64_t kb = reinterpret_cast<uint64_t>(p.k_pages) + (ph * kChunks * p.page_tokens + at) * 32;
            const uint64_t vb = reinterpret_cast<uint64_t>(p.v_pages) + (ph * p.page_tokens + at) * (2 * D);
            u32x4_t kf[2][kM], vf[kDB];
#pragma unroll
            for (int m = 0; m < kM; ++m) {
                const int c = 2 * m + (g4 >> 1);
                const bool kept = ((keep >> (8 * c)) & 0xFFull) != 0;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    kf[s][m] = u32x4_t{0u, 0u, 0u, 0u};
                    if (kept)
                        kf[s][m] = load16(kb + (int64_t(c) * p.page_tokens + min(tk + 8 * s, left)) * 32 + 16 * (g4 & 1));
                }
            }
#pragma unroll
            for (int i = 0; i < kDB; ++i) {
                vf[i] = u32x4_t{0u, 0u, 0u, 0u};
                if (16 * (g4 >> 1) <= left) vf[i] = load16(vb + (g4 >> 1) * (32 * D) + (16 * i + r16) * 32 + 16 * (g4 & 1));
            }
            if (keep & ~full) {
#pragma unroll
                for (int m = 0; m < kM; ++m)
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const int z = q_pos - tb - (tk + 8 * s);
                        uint32_t bits = 0;
#pragma unroll
                        for (int e = 0; e < 8; ++e) bits |= s_w[8 * (2 * m + (g4 >> 1)) + e] >= z ? 1u << e : 0u;
                        kf[s][m] = keep_pairs(kf[s][m], bits);
                    }
            } else {
#pragma unroll
                for (int m = 0; m < kM; ++m) {
                    const uint32_t bits = uint32_t(keep >> (8 * (2 * m + (g4 >> 1)))) & 0xFFu;
#pragma unroll
                    for (int s = 0; s < 2; ++s) kf[s][m] = keep_pairs(kf[s][m], bits);
                }
            }
            f32x4_t sacc[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    sacc[n][s] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int m = 0; m < kM; ++m) {
                        const uint32_t bits = uint32_t(keep >> (8 * (2 * m + (g4 >> 1)))) & 0xFFu;
                        sacc[n][s] = mfma16(kf[s][m], keep_pairs(qf[kM * n + m], bits), sacc[n][s]);
                    }
                }
            // tokens past the row's keys: no probability, and no value that is not a number
            if (left < kTile - 1) {
                const int bound = left - 16 * (g4 >> 1) - 4 * (g4 & 1);
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const bool out = 8 * s + v > bound;
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            if (out) sacc[n][s][v] = -INFINITY;
                        // element 4 s + v of the lane's 8 values
                        if (out) {
#pragma unroll
                            for (int i = 0; i < kDB; ++i) vf[i][2 * s + v / 2] &= v & 1 ? 0x0000FFFFu : 0xFFFF0000u;
                        }
                    }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float mx = -INFINITY;
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int v = 0; v < 4; ++v) mx = fmaxf(mx, sacc[n][s][v]);
                mx = fmaxf(mx, __shfl_xor(mx, 16));
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                const float m_new = fmaxf(m_run[n], mx * sc);
                const float m_use = m_new == -INFINITY ? 0.f : m_new;
                const float alpha = exp2_fast(m_run[n] - m_use);
                m_run[n] = m_new;
                l_run[n] *= alpha;
#pragma unroll
                for (int i = 0; i < kDB; ++i) oacc[n][i] *= alpha;
                // P as two bf16 numbers, what fits and what is left over: one would round every
                // probability to 2^-9, and the output's own rounding is that size
                u32x4_t ph_, pl_;
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        uint32_t h[2];
                        bf16x2_t rest;
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const float e = exp2_fast(__builtin_fmaf(sacc[n][s][2 * k + x], sc, -m_use));
                            l_run[n] += e;
                            h[x] = __float_as_uint(e) & 0xFFFF0000u;
                            rest[x] = (__bf16)(e - __uint_as_float(h[x]));
                        }
                        ph_[2 * s + k] = h[0] >> 16 | h[1];
                        pl_[2 * s + k] = __builtin_bit_cast(uint32_t, rest);
                    }
#pragma unroll
                for (int i = 0; i < kDB; ++i) {
                    oacc[n][i] = mfma16(vf[i], ph_, oacc[n][i]);
                    oacc[n][i] = mfma16(vf[i], pl_, oacc[n][i]);
                }
            }
        }
    }

    // ---- combine the waves' states, in wave order
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
        if (r16 < heads) {
#pragma unroll
            for (int i = 0; i < kDB; ++i)
                *reinterpret_cast<f32x4_t*>(&s_o[(16 * wave + r16) * kOStride + 16 * i + 4 * g4]) = oacc[n][i] * f;
        }
        __syncthreads();
        for (int e = tid; e < heads * (D / 4); e += NW * 64) {
            const int r = e / (D / 4), x = 4 * (e % (D / 4)), h = 16 * n + r;
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < NW; ++w) M = fmaxf(M, red_m[w][h]);
            f32x4_t o = {0.f, 0.f, 0.f, 0.f};
            float L = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                o += *reinterpret_cast<const f32x4_t*>(&s_o[(16 * w + r) * kOStride + x]);
                if (red_m[w][h] != -INFINITY) L += red_l[w][h] * exp2_fast(red_m[w][h] - M);
            }
            const bool empty = L == 0.f;  // no key: O = 0, LSE = -inf
            bf16x2_t lo, hi;
            lo[0] = (__bf16)(empty ? 0.f : o[0] / L);
            lo[1] = (__bf16)(empty ? 0.f : o[1] / L);
            hi[0] = (__bf16)(empty ? 0.f : o[2] / L);
            hi[1] = (__bf16)(empty ? 0.f : o[3] / L);
            const int64_t at = int64_t(t) * p.h_q + hq0 + h;
            *reinterpret_cast<uint2*>(p.o + at * D + x) =
                make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
            if (x == 0) p.lse[at] = empty ? -INFINITY : M * 0.69314718055994531f + logf(L);
        }
    }
}

template <int D>
hipError_t launch_d(const AttendParams& p, hipStream_t stream) {
    const int64_t blocks = int64_t(p.n_tokens) * p.h_kv * p.subgroups;
    if (blocks * 256 > 0xFFFFFFFF) return hipErrorInvalidConfiguration;
    const dim3 grid(static_cast<unsigned>(blocks));
    if (p.heads_per_block > 16)
        hipLaunchKernelGGL((attend_blocks_kernel<D, 2, 4>), grid, dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL((attend_blocks_kernel<D, 1, 4>), grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_blocks(const AttendParams& p, int head_dim, hipStream_t stream) {
    (void)hipGetLastError();
    return head_dim == 64 ? launch_d<64>(p, stream) : launch_d<128>(p, stream);
}

}  // namespace atf
