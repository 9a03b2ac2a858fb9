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
//
// Bound by HBM where the call is long: 32,768 tokens of 28/4 heads of 128 into 8-bit caches move
// 571 MB in 110 us (5.2 TB/s, a device copy reaches 5.4), 16,384 of 24/8 heads into bf16 ones 336 MB
// in 67 us; 3,885 tokens of 16/16 heads of 64 40 MB in 13 us, where vector work (busy 0.63) and a
// launch's start and end count; one token of each of 16 rows takes 3.9 us.  8 dims a lane make
// every access of a vector 16 bytes; with fewer lanes a vector the keys' 16-byte chunks would be
// gathered, with more the row's sum would cross more lanes.
#include "atf_internal.hpp"
#include "q8.hpp"

#include <algorithm>
#include <type_traits>

namespace atf {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
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
// nearest quarter turn is taken off the 64-bit fraction in integers; what is left, at most
// pi/4, is turned to radians in two floats, whose first goes through the Taylor series to x^9 and
// x^10 (truncation below 2^-28) and whose second is added to first order.  The fraction's low word
// (rounded to it, so that the two do not cancel) is part of the second: next to a quarter turn the
// smaller of sine and cosine is little more.  Both are within about 1.2 ulp, 0.3 in the root mean
// square, of those of the angle as it is held, pos times 2^-64 of a turn off (the hardware's own
// sine is 2^-20 off).
__device__ __forceinline__ void cos_sin(uint32_t pos, uint32_t rho_hi, uint32_t rho_lo, float& cs, float& sn) {
    const uint32_t rest = pos * rho_lo;
    const uint32_t f = pos * rho_hi + __umulhi(pos, rho_lo) + (rest >> 31);
    const uint32_t quarter = (f + 0x20000000u) >> 30;
    const int32_t r = int32_t(f - (quarter << 30));
    const float rh = float(r);
    const float rl = __builtin_fmaf(float(int32_t(rest)), 2.3283064365386963e-10f, float(r - int32_t(rh)));  // 2^-32
    constexpr float kUnit = 1.4629180792671596e-9f, kUnitLow = float(1.4629180792671596e-9 - double(kUnit));  // 2 pi / 2^32
    const float x = rh * kUnit;
    const float low = __builtin_fmaf(rh, kUnit, -x) + __builtin_fmaf(rh, kUnitLow, rl * kUnit);
    const float y = x * x;
    float s = __builtin_fmaf(y, 2.7557319e-6f, -1.9841270e-4f);
    s = __builtin_fmaf(y, s, 8.3333333e-3f);
    s = __builtin_fmaf(y, s, -1.6666667e-1f);
    s = __builtin_fmaf(x * y, s, low) + x;
    float c = __builtin_fmaf(y, -2.7557319e-7f, 2.4801587e-5f);
    c = __builtin_fmaf(y, c, -1.3888889e-3f);
    c = __builtin_fmaf(y, c, 4.1666667e-2f);
    c = __builtin_fmaf(y, c, -0.5f);
    c = __builtin_fmaf(y, c, -x * low) + 1.f;
    const bool swap = quarter & 1;
    const float a = swap ? s : c, b = swap ? c : s;
    cs = (quarter + 1) & 2 ? -a : a;
    sn = quarter & 2 ? -b : b;
}

// The same in 64 bits, from 64 bits of the fraction: Taylor series to x^13 and x^14 (truncation below
// 2^-41).
__device__ __forceinline__ void cos_sin64(uint32_t pos, uint32_t rho_hi, uint32_t rho_lo, double& cs, double& sn) {
    const uint64_t f = uint64_t(pos) * (uint64_t(rho_hi) << 32 | rho_lo);
    const uint32_t quarter = uint32_t((f + (uint64_t(1) << 61)) >> 62);
    const double x = double(int64_t(f - (uint64_t(quarter) << 62))) * 3.4061215800304553e-19;  // 2 pi / 2^64
    const double y = x * x;
    double s = __builtin_fma(y, 1.0 / 6227020800.0, -1.0 / 39916800.0);
    s = __builtin_fma(y, s, 1.0 / 362880.0);
    s = __builtin_fma(y, s, -1.0 / 5040.0);
    s = __builtin_fma(y, s, 1.0 / 120.0);
    s = __builtin_fma(y, s, -1.0 / 6.0);
    s = __builtin_fma(x * y, s, x);
    double c = __builtin_fma(y, -1.0 / 87178291200.0, 1.0 / 479001600.0);
    c = __builtin_fma(y, c, -1.0 / 3628800.0);
    c = __builtin_fma(y, c, 1.0 / 40320.0);
    c = __builtin_fma(y, c, -1.0 / 720.0);
    c = __builtin_fma(y, c, 1.0 / 24.0);
    c = __builtin_fma(y, c, -0.5);
    c = __builtin_fma(y, c, 1.0);
    const bool swap = quarter & 1;
    const double a = swap ? s : c, b = swap ? c : s;
    cs = (quarter + 1) & 2 ? -a : a;
    sn = quarter & 2 ? -b : b;
}

// x as fp32, and where it is none, the odd one of its two neighbours: what rounds it on rounds as if
// from x itself.
__device__ __forceinline__ float to_odd(double x) {
    const float f = float(x);
    const double rest = x - double(f);
    uint32_t bits = __float_as_uint(f);
    if (fabsf(f) < INFINITY && rest != 0. && (bits & 1u) == 0u) bits += (rest > 0.) == (x > 0.) ? 1u : ~0u;
    return __uint_as_float(bits);
}

template <int kCtrl>
__device__ __forceinline__ double dpp64(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, uint64_t(dpp<kCtrl>(uint32_t(u >> 32))) << 32 | dpp<kCtrl>(uint32_t(u)));
}
template <int kLanes>
__device__ __forceinline__ double other_lane64(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, uint64_t(other_lane<kLanes>(uint32_t(u >> 32))) << 32 | other_lane<kLanes>(uint32_t(u)));
}
template <int kLanes>
__device__ __forceinline__ double sum_lanes64(double x) {
    x += dpp64<kXor1>(x);
    x += dpp64<kXor2>(x);
    x += dpp64<kMirror8>(x);
    if constexpr (kLanes == 16) x += dpp64<kMirror16>(x);
    return x;
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

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// The largest magnitude of n numbers, as bits: of all of them (above the finite ones' bits if one
// is not finite), or of the finite ones (0 if there is none).
template <int n, bool kFinite>
__device__ __forceinline__ uint32_t largest(const float* y) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < n; ++e) {
        const uint32_t a = magnitude(y[e]);
        m = max(m, kFinite && a >= q8::kInfBits ? 0u : a);
    }
    return m;
}

// Calls f with whether every lane's numbers, whose largest magnitude is m, are plain ones.
template <typename F>
__device__ __forceinline__ void by_kind(uint32_t m, F f) {
    if (__any(m > q8::kPlainBits))
        f(std::false_type{});
    else
        f(std::true_type{});
}

template <bool kStream, typename T>
__device__ __forceinline__ T load_from(const void* from) {
    const T* f = static_cast<const T*>(from);
    return kStream ? __builtin_nontemporal_load(f) : *f;
}
template <bool kStream>
__device__ __forceinline__ void store16(void* to, u32x4_t x) {
    if constexpr (kStream)
        __builtin_nontemporal_store(x, static_cast<u32x4_t*>(to));
    else
        *static_cast<u32x4_t*>(to) = x;
}

// A token of the call: its row of the batch, its position, its place in the caches.
struct Token {
    int64_t entry;  // row of the contiguous caches, or page
    int cap, tok;   // the entry's tokens, and the token in it
    int pos;
    bool active, stored;
};

__device__ __forceinline__ Token locate(const AppendNormedParams& p, int b, int t, bool given) {
    const int first = p.pos_rows != nullptr ? p.pos_rows[b] : p.pos0;
    Token k;
    k.active = given && first >= 0 && int64_t(first) + t < 0x7FFFFFFF;
    k.pos = k.active ? first + t : 0;
    if (p.block_table != nullptr) {
        const int at = k.pos / p.page_tokens;
        k.stored = k.active && at < p.max_pages;
        const int page = k.stored ? p.block_table[int64_t(b) * p.max_pages + at] : -1;
        k.stored = k.stored && page >= 0 && page < p.num_pages;
        k.entry = k.stored ? page : 0;
        k.cap = p.page_tokens;
        k.tok = k.pos - at * p.page_tokens;
    } else {
        k.stored = k.active && k.pos < p.cache_tokens;
        k.entry = b;
        k.cap = p.cache_tokens;
        k.tok = k.pos;
    }
    return k;
}

// The tokens of row b that its caches have room for: [0, n), and those of them at its ends that
// do not fill a 16-token block of the V cache: [0, head) and [tail, n).
struct Ends {
    int first, n, head, tail;
};
__device__ __forceinline__ Ends ends_of(const AppendNormedParams& p, int b) {
    Ends e;
    e.first = p.pos_rows != nullptr ? p.pos_rows[b] : p.pos0;
    const int64_t room = p.block_table != nullptr ? int64_t(p.max_pages) * p.page_tokens : p.cache_tokens;
    e.n = e.first < 0 ? 0 : int(max(int64_t(0), min(int64_t(p.n_new), room - e.first)));
    e.head = min(e.n, (16 - (e.first & 15)) & 15);
    e.tail = max(e.head, e.n - ((e.first + e.n) & 15));
    return e;
}

// The values of whole 16-token blocks: D / 2 lanes take a block, 2 dims of its 16 tokens each, so
// that a block is turned to dim-major in the lane's registers and stored 16 bytes at a time.
template <int D, bool kQ8, bool kStream>
__device__ __forceinline__ void value_blocks(const AppendNormedParams& p, uint32_t wave) {
    constexpr int kLanes = D / 2;
    const int lane = threadIdx.x & 63;
    const int x = lane % kLanes;  // dims 2x, 2x + 1
    const uint32_t nblk = (uint32_t(p.n_new) + 14u) / 16u + 1u;
    const uint32_t units = uint32_t(p.batch) * nblk * uint32_t(p.h_kv);
    const uint32_t unit = wave * (64 / kLanes) + lane / kLanes, u = min(unit, units - 1);
    const int g = int(u % uint32_t(p.h_kv));
    const uint32_t rest = u / uint32_t(p.h_kv);
    const int b = int(rest / nblk), k = int(rest % nblk);
    const Ends e = ends_of(p, b);
    const int t0 = 16 * k - (e.first & 15);  // the block's first token in the call
    const Token at = locate(p, b, max(t0, 0), unit < units && t0 >= e.head && t0 + 16 <= e.tail);
    if (!__any(at.stored)) return;
    const int64_t row = int64_t(p.h_kv) * D;
    const uint16_t* src = p.v_src + ((int64_t(b) * p.n_new + (at.stored ? t0 : 0)) * p.h_kv + g) * D + 2 * x;
    uint32_t v[16];
#pragma unroll
    for (int t = 0; t < 16; ++t) v[t] = load_from<kStream, uint32_t>(src + (at.stored ? t * row : 0));
    const int64_t eg = at.entry * p.h_kv + g;
    const int64_t block = (eg * ((int64_t(at.cap) + 15) / 16) + at.tok / 16) * D + 2 * x;  // row of dim 2x
    u32x4_t out[2][kQ8 ? 1 : 2];
    if constexpr (kQ8) {
        uint32_t all = 0;
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            const float y[2] = {bf_lo(v[t]), bf_hi(v[t])};
            all = max(all, largest<2, false>(y));
        }
        u32x4_t bytes;
        by_kind(all, [&](auto plain) __attribute__((always_inline)) {
            constexpr bool kPlain = decltype(plain)::value;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t w[2];  // two tokens of two dims each
                bytes[i] = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float y[2] = {bf_lo(v[4 * i + j]), bf_hi(v[4 * i + j])};
                    uint32_t m = max_lanes<16>(largest<2, !kPlain>(y));
                    const auto m16 = __builtin_amdgcn_permlane16_swap(m, m, false, false);
                    m = max(m16[0], m16[1]);
                    if constexpr (kLanes == 64) {
                        const auto m32 = __builtin_amdgcn_permlane32_swap(m, m, false, false);
                        m = max(m32[0], m32[1]);
                    }
                    const uint32_t byte = q8::scale_byte(m);
                    const float inv = q8::inverse_power(byte);
                    const float z0 = q8::scaled<kPlain>(y[0], inv), z1 = q8::scaled<kPlain>(y[1], inv);
                    w[j / 2] = j % 2 ? q8::pack2<1>(z0, z1, w[j / 2]) : q8::pack2<0>(z0, z1, 0u);
                    bytes[i] |= byte << (8 * j);
                }
                out[0][0][i] = __builtin_amdgcn_perm(w[1], w[0], 0x06040200u);
                out[1][0][i] = __builtin_amdgcn_perm(w[1], w[0], 0x07050301u);
            }
        });
        if (at.stored) {
            uint8_t* dst = static_cast<uint8_t*>(p.v_dst) + block * 16;
            *reinterpret_cast<u32x4_t*>(dst) = out[0][0];
            *reinterpret_cast<u32x4_t*>(dst + 16) = out[1][0];
            if (x == 0) *reinterpret_cast<u32x4_t*>(p.v_scale + eg * p.scale_tokens + at.tok) = bytes;
        }
    } else {
        // slot 8h + 4a + b of a dim's row holds token 8a + 4h + b
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int t = 8 * (i / 2 % 2) + 4 * (i / 4) + 2 * (i % 2);
            out[0][i / 4][i % 4] = __builtin_amdgcn_perm(v[t + 1], v[t], 0x05040100u);
            out[1][i / 4][i % 4] = __builtin_amdgcn_perm(v[t + 1], v[t], 0x07060302u);
        }
        if (at.stored) {
            uint16_t* dst = static_cast<uint16_t*>(p.v_dst) + block * 16;
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<u32x4_t*>(dst + 8 * j) = out[j / 2][j % 2];
        }
    }
}

// kStream: the vectors of the call are read and the queries written past the caches, which they
// would only sweep.
template <int D, bool kQ8, bool kStream>
__global__ __launch_bounds__(256) void append_normed_kernel(const AppendNormedParams p) {
    constexpr int kLanes = D / 8;          // lanes of a vector
    constexpr int kTokens = 64 / kLanes;   // tokens of a wave
    constexpr int kChunks = D / 16;
    constexpr int kAhead = 8;              // heads loaded before the first is used
    const int lane = threadIdx.x & 63;
    uint32_t wave = blockIdx.x * 4u + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // (the blocks of values first: their waves take longest, and would end the call alone)
    if (blockIdx.x * 4u < p.block_waves) {
        value_blocks<D, kQ8, kStream>(p, wave);
        return;
    }
    wave -= p.block_waves;
    // this wave's tokens and its heads, all of one kind: values by themselves, keys, queries
    const bool alone = wave < p.value_waves;
    if (!alone) wave -= p.value_waves;
    // (in a long call a token's queries and keys side by side, which HBM reads 2 to 5 % faster, else
    // the keys first, which take longest)
    int kind = 2;
    uint32_t parts = p.kv_parts, part;
    if (kStream && !alone) {
        parts += p.q_parts;
        part = wave % parts;
        kind = part < p.q_parts ? 0 : 1;
        if (kind == 1) part -= p.q_parts;
    } else {
        if (!alone) kind = wave < p.key_waves ? 1 : 0;
        if (kind == 0) {
            wave -= p.key_waves;
            parts = p.q_parts;
            if (parts == 0) return;  // a wave past the last one's work, of a call without queries
        }
        part = wave % parts;
    }
    const int n_heads = kind == 0 ? p.h_q : p.h_kv, hpw = kind == 0 ? p.q_heads_per_wave : p.kv_heads_per_wave;
    const int from = int(part) * hpw, to = min(from + hpw, n_heads);
    const uint32_t rows = uint32_t(p.batch) * (alone && p.value_ends ? 32u : uint32_t(p.n_new));
    const uint32_t row = wave / parts * uint32_t(kTokens) + uint32_t(lane / kLanes);
    if (wave / parts * uint32_t(kTokens) >= rows) return;
    uint32_t b, t;
    bool given = row < rows;
    if (alone && p.value_ends) {
        // 32 places a row of the batch: the tokens before its first whole block, and after the last
        b = min(row / 32u, uint32_t(p.batch) - 1u);
        const uint32_t j = row % 32u;
        const Ends e = ends_of(p, int(b));
        t = j < 16u ? j : uint32_t(e.tail) + j - 16u;
        given = given && (j < 16u ? int(t) < e.head : int(t) < e.n);
        if (!given) t = 0;
    } else {
        b = min(row, rows - 1) / uint32_t(p.n_new);
        t = min(row, rows - 1) - b * uint32_t(p.n_new);
    }
    const uint32_t r = b * uint32_t(p.n_new) + t;
    const int l = lane % kLanes;
    const int c = l % kChunks, hf = l / kChunks;  // pair-chunk, half of the pairs
    const uint16_t* src = (kind == 0 ? p.q : kind == 1 ? p.k_src : p.v_src) + int64_t(r) * n_heads * D + 8 * l;
    u32x4_t x[kAhead];
    const auto load = [&](int h) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            x[i] = load_from<kStream, u32x4_t>(src + int64_t(min(h + i, to - 1)) * D);
    };
    load(from);

    const Token at = locate(p, int(b), int(t), given);
    const int64_t eg0 = at.entry * p.h_kv;
    float wc[8], ws[8];  // ws with the half's sign: x'_own = own * wc + other * ws
    const float* weight = kind == 0 ? p.q_weight : p.k_weight;
    if (kind != 2) {
        // the two lanes of a chunk share its 8 angles: half of them each, then both have all
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float cs, sn;
            cos_sin(uint32_t(at.pos), p.rope_rho_hi[8 * c + 4 * hf + e], p.rope_rho_lo[8 * c + 4 * hf + e], cs, sn);
            const float co = __uint_as_float(other_lane<kLanes>(__float_as_uint(cs)));
            const float so = __uint_as_float(other_lane<kLanes>(__float_as_uint(sn)));
            wc[e] = hf ? co : cs;
            wc[4 + e] = hf ? cs : co;
            ws[e] = hf ? so : -sn;
            ws[4 + e] = hf ? sn : -so;
        }
        if (weight != nullptr) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                wc[e] *= weight[8 * l + e];
                ws[e] *= weight[8 * (l ^ kChunks) + e];
            }
        }
    }
    const auto turned = [&](u32x4_t v, float* y) __attribute__((always_inline)) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t o = other_lane<kLanes>(v[i]);
            const float a0 = bf_lo(v[i]), a1 = bf_hi(v[i]);
            ss = __builtin_fmaf(a0, a0, ss);
            ss = __builtin_fmaf(a1, a1, ss);
            y[2 * i] = __builtin_fmaf(a0, wc[2 * i], bf_lo(o) * ws[2 * i]);
            y[2 * i + 1] = __builtin_fmaf(a1, wc[2 * i + 1], bf_hi(o) * ws[2 * i + 1]);
        }
        if (weight != nullptr) {
            // (one Newton step on the hardware's root, which is an ulp off)
            const float mean = __builtin_fmaf(sum_lanes<kLanes>(ss), 1.f / D, p.eps);
            float rs = rsqrtf(mean);
            const float off = __builtin_fmaf(-mean * rs, rs, 1.f);
            if (fabsf(off) < 0.5f) rs = __builtin_fmaf(0.5f * rs, off, rs);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] *= rs;
        }
    };
    // Numbers of a key so near to the middle of two e4m3 numbers (their lower 20 bits near half a
    // step), or whose largest is so near to 448 powers, that fp32's own error may decide: within kNear
    // ulps (that error is 0.4 ulps in the root mean square, with norm 0.75).  One head of a wave in 500
    // has one; it is formed again in 64 bits once the wave is through.  Of 537 million random numbers
    // 350 to 440 round to the other side (plain fp32: 780 to 960), at 0.04 to 0.09 of plain fp32's
    // error: none of those next to a border that are no small difference (plain fp32: 35 to 41), but
    // small ones, below 2^-6 of the power, whose steps are others, and what is left of a larger
    // difference.  The heads met again cost the calls where a wave's time counts: 64 rows of one token
    // 5.0 -> 5.6 us, 3,885 tokens of 16/16 heads of 64 12.7 -> 12.9, 32,768 of 28/4 110.8 -> 111.3.
    // Without norm and angle fp32 is exact.
    constexpr uint32_t kNear = 2;
    [[maybe_unused]] bool exact = weight == nullptr;
    if constexpr (kQ8) {
#pragma unroll
        for (int e = 0; e < 8; ++e) exact = exact && (kind == 2 || ws[e] == 0.f);
    }
    [[maybe_unused]] const auto doubtful = [&](const float* y, uint32_t m) __attribute__((always_inline)) {
        uint32_t near = (m << 9) + ((kNear << 9) - 0xC0000000u);  // (up to 16 times as far above it)
#pragma unroll
        for (int e = 0; e < 8; ++e) near = min(near, (__float_as_uint(y[e]) << 12) + ((kNear << 12) - 0x80000000u));
        return __any(near < (kNear << 13) && !exact) != 0;
    };
    [[maybe_unused]] const auto refined = [&](u32x4_t v, float* y) __attribute__((always_inline)) {
        double rs = 1.;
        if (weight != nullptr) {
            double ss = 0.;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const double a0 = bf_lo(v[i]), a1 = bf_hi(v[i]);
                ss = __builtin_fma(a0, a0, ss);
                ss = __builtin_fma(a1, a1, ss);
            }
            rs = 1. / __builtin_sqrt(sum_lanes64<kLanes>(ss) / D + double(p.eps));
        }
        // as above, 4 angles a lane: elements i and 4 + i a turn of the loop, which is short code (it is
        // met cold) and moves what is used or made to where the next turn has it
        u32x4_t rh, rl;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            rh[i] = p.rope_rho_hi[8 * c + 4 * hf + i];
            rl[i] = p.rope_rho_lo[8 * c + 4 * hf + i];
        }
#pragma clang loop unroll(disable)
        for (int i = 0; i < 4; ++i) {
            float w[4] = {1.f, 1.f, 1.f, 1.f};
            if (weight != nullptr) {
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = weight[8 * (k & 1 ? l ^ kChunks : l) + 4 * (k / 2) + i];
            }
            double cs, sn;
            cos_sin64(uint32_t(at.pos), rh[0], rl[0], cs, sn);
            const double co = other_lane64<kLanes>(cs), so = other_lane64<kLanes>(sn);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const double a = double(bf_lo(v[2 * k])) * w[2 * k];
                const double o = double(bf_lo(other_lane<kLanes>(v[2 * k]))) * w[2 * k + 1];
                const double x = __builtin_fma(a, k == hf ? cs : co, (hf ? o : -o) * (k == hf ? sn : so)) * rs;
#pragma unroll
                for (int e = 0; e < 3; ++e) y[4 * k + e] = y[4 * k + e + 1];
                y[4 * k + 3] = to_odd(x);
                v[2 * k] = i & 1 ? v[2 * k + 1] : v[2 * k] >> 16;
            }
#pragma unroll
            for (int e = 0; e < 3; ++e) {
                rh[e] = rh[e + 1];
                rl[e] = rl[e + 1];
            }
        }
    };
    // a row's 8 numbers of this lane as e4m3, and the row's power; m is its largest magnitude
    [[maybe_unused]] const auto quantised = [&](const float* y, uint32_t m, uint32_t& byte) __attribute__((always_inline)) {
        uint2 w;
        by_kind(m, [&](auto plain) __attribute__((always_inline)) {
            constexpr bool kPlain = decltype(plain)::value;
            byte = q8::scale_byte(kPlain ? m : max_lanes<kLanes>(largest<8, true>(y)));
            const float inv = q8::inverse_power(byte);
            float z[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = q8::scaled<kPlain>(y[e], inv);
            w = make_uint2(q8::pack4(z[0], z[1], z[2], z[3]), q8::pack4(z[4], z[5], z[6], z[7]));
        });
        return w;
    };
    const auto query = [&](int h, u32x4_t v) __attribute__((always_inline)) {
        float y[8];
        turned(v, y);
        if (at.active) store16<kStream>(p.q_out + (int64_t(r) * p.h_q + h) * D + 8 * l, to_bf16(y));
    };
    [[maybe_unused]] const auto store_q8 = [&](int g, const float* y, uint32_t m) __attribute__((always_inline)) {
        const int64_t to_k = (((eg0 + g) * kChunks + c) * at.cap + at.tok) * 16 + 8 * hf;
        uint32_t byte;
        const uint2 w = quantised(y, m, byte);
        if (at.stored) {
            *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.k_dst) + to_k) = w;
            if (l == 0) p.k_scale[(eg0 + g) * p.scale_tokens + at.tok] = uint8_t(byte);
        }
    };
    [[maybe_unused]] uint64_t again = 0;  // the heads, counted from the wave's first, that are formed in 64 bits
    const auto key = [&](int g, u32x4_t v) __attribute__((always_inline)) {
        float y[8];
        turned(v, y);
        if constexpr (kQ8) {
            const uint32_t m = max_lanes<kLanes>(largest<8, false>(y));
            if (doubtful(y, m))
                again |= uint64_t(1) << (g - from);
            else
                store_q8(g, y, m);
        } else if (at.stored) {
            const int64_t to_k = (((eg0 + g) * kChunks + c) * at.cap + at.tok) * 16 + 8 * hf;
            *reinterpret_cast<u32x4_t*>(static_cast<uint16_t*>(p.k_dst) + to_k) = to_bf16(y);
        }
    };
    // a value by itself: its dims are 16 numbers apart
    const auto value = [&](int g, u32x4_t v) __attribute__((always_inline)) {
        const int64_t to_v = (((eg0 + g) * ((int64_t(at.cap) + 15) / 16) + at.tok / 16) * D + 8 * l) * 16;
        if constexpr (kQ8) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = e & 1 ? bf_hi(v[e / 2]) : bf_lo(v[e / 2]);
            uint8_t* dst = static_cast<uint8_t*>(p.v_dst) + to_v + at.tok % 16;
            uint32_t byte;
            const uint2 x2 = quantised(y, max_lanes<kLanes>(largest<8, false>(y)), byte);
            const uint32_t w[2] = {x2.x, x2.y};
            if (at.stored) {
#pragma unroll
                for (int e = 0; e < 8; ++e) dst[16 * e] = uint8_t(w[e / 4] >> (8 * (e % 4)));
                if (l == 0) p.v_scale[(eg0 + g) * p.scale_tokens + at.tok] = uint8_t(byte);
            }
        } else if (at.stored) {
            const int s = at.tok % 16;
            uint16_t* dst = static_cast<uint16_t*>(p.v_dst) + to_v + 8 * (s / 4 % 2) + 4 * (s / 8) + s % 4;
#pragma unroll
            for (int e = 0; e < 8; ++e) dst[16 * e] = uint16_t(e & 1 ? v[e / 2] >> 16 : v[e / 2]);
        }
    };
    const auto heads = [&](auto one) __attribute__((always_inline)) {
        for (int h = from; h < to; h += kAhead) {
            if (h != from) load(h);
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (h + i < to) one(h + i, x[i]);
        }
    };
    if (kind == 0)
        heads(query);
    else if (kind == 1)
        heads(key);
    else
        heads(value);
    if constexpr (kQ8) {
        for (; again != 0; again &= again - 1) {
            const int g = from + __builtin_ctzll(again);
            float y[8];
            refined(*reinterpret_cast<const u32x4_t*>(src + int64_t(g) * D), y);
            store_q8(g, y, max_lanes<kLanes>(largest<8, false>(y)));
        }
    }
}

template <int D>
hipError_t launch_d(AppendNormedParams p, hipStream_t stream) {
    constexpr int kTokens = 64 / (D / 8);
    const int64_t groups = (int64_t(p.batch) * p.n_new + kTokens - 1) / kTokens;
    // one head a wave until the chip is about full of waves (4 run on a SIMD), then as many as keep it
    // full, so that a token's angles serve them all, in equal parts.  As many as would leave 3400 waves
    // if all of a token's heads could be shared out evenly; queries and keys are by themselves, so that
    // there are more (16,384 for 32,768 tokens of 28/4 heads of 128, 3,888 for 3,885 of 16/16 of 64).
    // Against enough to leave 4096: 1,000 tokens of 28/4 heads of 128 into 8-bit caches 11.5 -> 8.2 us,
    // 4,000 of 14/2 heads of 64 11.6 -> 8.4, 3,885 of 16/16 13.5 -> 12.7; 900 of 40/2 11.3 -> 12.0;
    // 16,384 and more the same
    const int64_t target = 3400;
    const int64_t heads = p.h_q + p.h_kv;
    const int64_t most = std::max<int64_t>(1, (groups * heads + target - 1) / target);
    const auto part = [&](int32_t h, int64_t most, int32_t& per_wave, uint32_t& parts) {
        parts = uint32_t((h + most - 1) / most);
        per_wave = h > 0 ? int32_t((h + parts - 1) / parts) : 1;
    };
    part(p.h_q, most, p.q_heads_per_wave, p.q_parts);
    part(p.h_kv, std::min<int64_t>(most, 64), p.kv_heads_per_wave, p.kv_parts);  // (of the keys at most 64: a wave counts them in bits)
    const int64_t row_waves = groups * (int64_t(p.q_parts) + p.kv_parts);
    // values: token by token in a short call, else whole 16-token blocks (in whole workgroups) and
    // the tokens at the rows' ends by themselves
    const bool blocks = p.n_new >= 16;
    const int64_t units = int64_t(p.batch) * ((int64_t(p.n_new) + 14) / 16 + 1) * p.h_kv;
    const int64_t block_waves = blocks ? ((units + 128 / D - 1) / (128 / D) + 3) / 4 * 4 : 0;
    const bool aligned = p.pos_rows == nullptr && p.pos0 % 16 == 0 && p.n_new % 16 == 0;
    p.value_ends = blocks;
    const int64_t alone = blocks ? (aligned ? 0 : (int64_t(p.batch) * 32 + kTokens - 1) / kTokens) : groups;
    const int64_t waves = block_waves + alone * p.kv_parts + row_waves;
    // (a grid has less than 2^32 threads)
    if (waves < 1 || waves > (int64_t(1) << 26) - 4 || units > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
    p.block_waves = uint32_t(block_waves);
    p.value_waves = uint32_t(alone * p.kv_parts);
    p.key_waves = uint32_t(groups * p.kv_parts);
    const dim3 grid(unsigned((waves + 3) / 4));
    // queries that the L2s (8 of 4 MB) cannot hold for their reader
    const bool past = int64_t(p.batch) * p.n_new * p.h_q * D * 2 > (32 << 20);
    const auto launch = [&](auto kernel) {
        (void)hipGetLastError();
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, p);
        return hipGetLastError();
    };
    if (p.k_scale != nullptr)
        return past ? launch(append_normed_kernel<D, true, true>) : launch(append_normed_kernel<D, true, false>);
    return past ? launch(append_normed_kernel<D, false, true>) : launch(append_normed_kernel<D, false, false>);
}

}  // namespace

hipError_t launch_append_normed(const AppendNormedParams& p, int head_dim, hipStream_t stream) {
    return head_dim == 64 ? launch_d<64>(p, stream) : launch_d<128>(p, stream);
}

}  // namespace atf
