// Appends with the heads' norms: queries and keys as the projections produce them are normed
// per head, turned to their positions and written, the queries to q_out, the keys with their
// values into the caches, bf16 or 8-bit (q8.hpp), contiguous or paged, in one pass.
//
//   x' = x * rsqrt(mean(x^2) + eps) * w     over one head's d numbers, in fp32
//   rotate-half RoPE of x' at the token's position, rounded once, to bf16 or to e4m3
//
// A lane holds 8 dims of a vector, 8 or 16 lanes a vector, a wave 8 or 4 consecutive tokens of
// one head.  The sum of squares and the row's largest magnitude cross the lanes by DPP; the
// other half of the pairs comes from the lane of the same chunk in the other half.  Angles
// belong to tokens, not heads: a wave forms cos and sin (and their products with the norm's
// weights) once and goes through its heads with them.
#include "atf_internal.hpp"
#include "q8.hpp"

#include <algorithm>

namespace atf {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
    return uint32_t(__builtin_amdgcn_mov_dpp(int(x), kCtrl, 0xF, 0xF, true));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kQuadReverse = 0x1B;  // within 4 lanes
constexpr int kRor8 = 0x128, kMirror16 = 0x140, kMirror8 = 0x141;

// The sum, or the largest, over the kLanes (8 or 16) lanes of a vector, in each of them.
template <int kLanes>
__device__ __forceinline__ float sum_lanes(float x) {
    x += __uint_as_float(dpp<kXor1>(__float_as_uint(x)));
    x += __uint_as_float(dpp<kXor2>(__float_as_uint(x)));
    x += __uint_as_float(dpp<kMirror8>(__float_as_uint(x)));  // equal within 4 lanes by now
    if constexpr (kLanes == 16) x += __uint_as_float(dpp<kMirror16>(__float_as_uint(x)));
    return x;
}
template <int kLanes>
__device__ __forceinline__ uint32_t max_lanes(uint32_t x) {
    x = max(x, dpp<kXor1>(x));
    x = max(x, dpp<kXor2>(x));
    x = max(x, dpp<kMirror8>(x));
    if constexpr (kLanes == 16) x = max(x, dpp<kMirror16>(x));
    return x;
}
// the register of the lane of the other half: l ^ 8 of 16, l ^ 4 of 8
template <int kLanes>
__device__ __forceinline__ uint32_t other_lane(uint32_t x) {
    if constexpr (kLanes == 16) return dpp<kRor8>(x);
    return dpp<kQuadReverse>(dpp<kMirror8>(x));
}

// cos and sin of the angle of pair rho (0.64 fixed point, revolutions) at position pos.  The
// nearest quarter turn is taken off the 32-bit fraction in integers; what is left, at most
// pi/4, goes through the Taylor series to x^9 and x^10 (truncation below 2^-28), so both are
// within about an ulp: 8-bit keys round on from here, and the hardware's own sine is 2^-20 off.
__device__ __forceinline__ void cos_sin(uint32_t pos, uint32_t rho_hi, uint32_t rho_lo, float& cs, float& sn) {
    const uint32_t f = pos * rho_hi + __umulhi(pos, rho_lo);
    const uint32_t quarter = (f + 0x20000000u) >> 30;
    const float x = float(int32_t(f - (quarter << 30))) * 1.4629180792671596e-9f;  // 2 pi / 2^32
    const float y = x * x;
    float s = __builtin_fmaf(y, 2.7557319e-6f, -1.9841270e-4f);
    s = __builtin_fmaf(y, s, 8.3333333e-3f);
    s = __builtin_fmaf(y, s, -1.6666667e-1f);
    s = __builtin_fmaf(x * y, s, x);
    float c = __builtin_fmaf(y, -2.7557319e-7f, 2.4801587e-5f);
    c = __builtin_fmaf(y, c, -1.3888889e-3f);
    c = __builtin_fmaf(y, c, 4.1666667e-2f);
    c = __builtin_fmaf(y, c, -0.5f);
    c = __builtin_fmaf(y, c, 1.f);
    const bool swap = quarter & 1;
    const float a = swap ? s : c, b = swap ? c : s;
    cs = (quarter + 1) & 2 ? -a : a;
    sn = quarter & 2 ? -b : b;
}

__device__ __forceinline__ float bf_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf_hi(uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); }

__device__ __forceinline__ u32x4_t to_bf16(const float* y) {
    u32x4_t r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bf16x2_t two;
        two[0] = (__bf16)y[2 * i];
        two[1] = (__bf16)y[2 * i + 1];
        r[i] = __builtin_bit_cast(uint32_t, two);
    }
    return r;
}

// The largest finite magnitude of 8 numbers, as bits (0 if there is none).
__device__ __forceinline__ uint32_t finite_max(const float* y) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t a = __float_as_uint(y[e]) & 0x7FFFFFFFu;
        m = max(m, a < q8::kInfBits ? a : 0u);
    }
    return m;
}

template <int D, bool kQ8>
__global__ __launch_bounds__(256) void append_normed_kernel(const AppendNormedParams p) {
    constexpr int kLanes = D / 8;          // lanes of a vector
    constexpr int kTokens = 64 / kLanes;   // tokens of a wave
    constexpr int kChunks = D / 16;
    const int lane = threadIdx.x & 63;
    const int l = lane % kLanes;
    const int c = l % kChunks, hf = l / kChunks;  // pair-chunk, half of the pairs
    const int heads = p.h_q + 2 * p.h_kv;
    const int64_t rows = int64_t(p.batch) * p.n_new;
    const int parts = (heads + p.heads_per_wave - 1) / p.heads_per_wave;
    const int64_t unit = int64_t(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (unit >= (rows + kTokens - 1) / kTokens * parts) return;
    const int64_t row = unit / parts * kTokens + lane / kLanes;
    const int h0 = int(unit % parts) * p.heads_per_wave, h1 = min(h0 + p.heads_per_wave, heads);

    // the token: its row of the batch, its position, its place in the caches
    const bool given = row < rows;
    const int64_t r = given ? row : rows - 1;
    const int b = int(r / p.n_new), t = int(r % p.n_new);
    const int first = p.pos_rows != nullptr ? p.pos_rows[b] : p.pos0;
    const bool active = given && first >= 0 && int64_t(first) + t < 0x7FFFFFFF;
    const int pos = active ? first + t : 0;
    bool stored = active;
    int64_t entry = b, cap = p.cache_tokens;
    int tok = pos;
    if (p.block_table != nullptr) {
        const int at = pos / p.page_tokens;
        stored = stored && at < p.max_pages;
        const int page = stored ? p.block_table[int64_t(b) * p.max_pages + at] : -1;
        stored = stored && page >= 0 && page < p.num_pages;
        entry = stored ? page : 0;
        cap = p.page_tokens;
        tok = pos % p.page_tokens;
    } else {
        stored = stored && pos < p.cache_tokens;
    }

    float cs[8], sn[8];  // sn with the half's sign: x'_own = own * cs + other * sn
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        cos_sin(uint32_t(pos), p.rope_rho_hi[8 * c + e], p.rope_rho_lo[8 * c + e], cs[e], sn[e]);
        if (hf == 0) sn[e] = -sn[e];
    }

    // heads h from .. to of one kind: normed by `weight` (if any), turned, handed to `put`
    const auto turned = [&](const uint16_t* src, int n_heads, const float* weight, int from, int to,
                            auto put) __attribute__((always_inline)) {
        if (from >= to) return;
        float wc[8], ws[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            wc[e] = weight != nullptr ? weight[8 * l + e] * cs[e] : cs[e];
            ws[e] = weight != nullptr ? weight[8 * (l ^ kChunks) + e] * sn[e] : sn[e];
        }
        for (int h = from; h < to; ++h) {
            const u32x4_t x = *reinterpret_cast<const u32x4_t*>(src + (r * n_heads + h) * D + 8 * l);
            float y[8], ss = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t o = other_lane<kLanes>(x[i]);
                const float a0 = bf_lo(x[i]), a1 = bf_hi(x[i]);
                ss = __builtin_fmaf(a0, a0, ss);
                ss = __builtin_fmaf(a1, a1, ss);
                y[2 * i] = __builtin_fmaf(a0, wc[2 * i], bf_lo(o) * ws[2 * i]);
                y[2 * i + 1] = __builtin_fmaf(a1, wc[2 * i + 1], bf_hi(o) * ws[2 * i + 1]);
            }
            if (weight != nullptr) {
                const float rs = rsqrtf(__builtin_fmaf(sum_lanes<kLanes>(ss), 1.f / D, p.eps));
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] *= rs;
            }
            put(h, y);
        }
    };

    turned(p.q, p.h_q, p.q_weight, h0, min(h1, p.h_q), [&](int h, const float* y) __attribute__((always_inline)) {
        if (active) *reinterpret_cast<u32x4_t*>(p.q_out + (r * p.h_q + h) * D + 8 * l) = to_bf16(y);
    });
    turned(p.k_src, p.h_kv, p.k_weight, max(h0 - p.h_q, 0), min(h1 - p.h_q, p.h_kv),
           [&](int g, const float* y) __attribute__((always_inline)) {
               const int64_t eg = entry * p.h_kv + g;
               const int64_t at = ((eg * kChunks + c) * cap + tok) * 16 + 8 * hf;
               if constexpr (kQ8) {
                   const uint32_t byte = q8::scale_byte(max_lanes<kLanes>(finite_max(y)));
                   const float inv = q8::inverse_power(byte);
                   float z[8];
#pragma unroll
                   for (int e = 0; e < 8; ++e) z[e] = q8::scaled(y[e], inv);
                   if (stored) {
                       *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.k_dst) + at) =
                           make_uint2(q8::pack4(z[0], z[1], z[2], z[3]), q8::pack4(z[4], z[5], z[6], z[7]));
                       if (l == 0) p.k_scale[eg * p.scale_tokens + tok] = uint8_t(byte);
                   }
               } else if (stored) {
                   *reinterpret_cast<u32x4_t*>(static_cast<uint16_t*>(p.k_dst) + at) = to_bf16(y);
               }
           });
    for (int g = max(h0 - p.h_q - p.h_kv, 0); g < h1 - p.h_q - p.h_kv; ++g) {
        const u32x4_t x = *reinterpret_cast<const u32x4_t*>(p.v_src + (r * p.h_kv + g) * D + 8 * l);
        const int64_t eg = entry * p.h_kv + g;
        const int64_t at = ((eg * ((cap + 15) / 16) + tok / 16) * D + 8 * l) * 16;
        if constexpr (kQ8) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = e & 1 ? bf_hi(x[e / 2]) : bf_lo(x[e / 2]);
            const uint32_t byte = q8::scale_byte(max_lanes<kLanes>(finite_max(y)));
            const float inv = q8::inverse_power(byte);
            uint8_t* dst = static_cast<uint8_t*>(p.v_dst) + at + tok % 16;
            uint32_t w[2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                w[i] = q8::pack4(q8::scaled(y[4 * i], inv), q8::scaled(y[4 * i + 1], inv),
                                 q8::scaled(y[4 * i + 2], inv), q8::scaled(y[4 * i + 3], inv));
            if (stored) {
#pragma unroll
                for (int e = 0; e < 8; ++e) dst[16 * e] = uint8_t(w[e / 4] >> (8 * (e % 4)));
                if (l == 0) p.v_scale[eg * p.scale_tokens + tok] = uint8_t(byte);
            }
        } else if (stored) {
            const int s = tok % 16;
            uint16_t* dst = static_cast<uint16_t*>(p.v_dst) + at + 8 * (s / 4 % 2) + 4 * (s / 8) + s % 4;
#pragma unroll
            for (int e = 0; e < 8; ++e) dst[16 * e] = uint16_t(e & 1 ? x[e / 2] >> 16 : x[e / 2]);
        }
    }
}

template <int D>
hipError_t launch_d(AppendNormedParams p, hipStream_t stream) {
    constexpr int kTokens = 64 / (D / 8);
    const int64_t groups = (int64_t(p.batch) * p.n_new + kTokens - 1) / kTokens;
    p.heads_per_wave = 1;
    const int64_t units = groups * (p.h_q + 2 * p.h_kv);
    const int64_t blocks = (units + 3) / 4;
    if (blocks < 1 || blocks > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
    (void)hipGetLastError();
    if (p.k_scale != nullptr)
        hipLaunchKernelGGL((append_normed_kernel<D, true>), dim3(unsigned(blocks)), dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL((append_normed_kernel<D, false>), dim3(unsigned(blocks)), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_append_normed(const AppendNormedParams& p, int head_dim, hipStream_t stream) {
    return head_dim == 64 ? launch_d<64>(p, stream) : launch_d<128>(p, stream);
}

}  // namespace atf
