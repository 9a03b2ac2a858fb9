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

// The largest finite magnitude of n numbers, as bits (0 if there is none).
template <int n>
__device__ __forceinline__ uint32_t finite_max(const float* y) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < n; ++e) {
        const uint32_t a = __float_as_uint(y[e]) & 0x7FFFFFFFu;
        m = max(m, a < q8::kInfBits ? a : 0u);
    }
    return m;
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

// The values of whole 16-token blocks (and of the parts at a row's ends): D / 4 lanes take a
// block, 4 dims of its 16 tokens each, so that a block is turned to dim-major in the lane's
// registers and stored 16 bytes at a time.
template <int D, bool kQ8, bool kStream>
__device__ __forceinline__ void value_blocks(const AppendNormedParams& p, uint32_t wave) {
    constexpr int kLanes = D / 4;
    const int lane = threadIdx.x & 63;
    const int x = lane % kLanes;  // dims 4x .. 4x + 3
    const uint32_t nblk = (uint32_t(p.n_new) + 14u) / 16u + 1u;
    const uint32_t units = uint32_t(p.batch) * nblk * uint32_t(p.h_kv);
    const uint32_t unit = wave * (64 / kLanes) + lane / kLanes, u = min(unit, units - 1);
    const int g = int(u % uint32_t(p.h_kv));
    const uint32_t rest = u / uint32_t(p.h_kv);
    const int b = int(rest / nblk), k = int(rest % nblk);
    const int first = p.pos_rows != nullptr ? p.pos_rows[b] : p.pos0;
    // the block's first token in the call, and those of its tokens that are in the call
    const int t0 = 16 * k - (first & 15);
    int lo = max(0, -t0), hi = min(16, p.n_new - t0);
    const Token at = locate(p, b, max(t0, 0), unit < units && hi > lo);
    if (!at.stored) hi = lo;
    hi = min(hi, at.cap - (at.tok & ~15));  // (a contiguous cache may end inside the block)
    if (__all(hi <= lo)) return;
    const int64_t row = int64_t(p.h_kv) * D;
    const uint16_t* src = p.v_src + ((int64_t(b) * p.n_new + t0) * p.h_kv + g) * D + 4 * x;
    const bool whole = lo == 0 && hi == 16;
    uint2 v[16];
    if (__all(whole)) {
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            const u32x2_t y = load_from<kStream, u32x2_t>(src + t * row);
            v[t] = make_uint2(y[0], y[1]);
        }
    } else {
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            v[t] = make_uint2(0u, 0u);
            if (t >= lo && t < hi) v[t] = *reinterpret_cast<const uint2*>(src + t * row);
        }
    }
    const int64_t eg = at.entry * p.h_kv + g;
    const int64_t block = (eg * ((at.cap + 15) / 16) + at.tok / 16) * D + 4 * x;  // row of dim 4x
    if constexpr (kQ8) {
        uint32_t byte[16], w[16];
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            const float y[4] = {bf_lo(v[t].x), bf_hi(v[t].x), bf_lo(v[t].y), bf_hi(v[t].y)};
            uint32_t m = max_lanes<16>(finite_max<4>(y));
            if constexpr (kLanes == 32) {
                const auto both = __builtin_amdgcn_permlane16_swap(m, m, false, false);
                m = max(both[0], both[1]);
            }
            byte[t] = q8::scale_byte(m);
            const float inv = q8::inverse_power(byte[t]);
            w[t] = q8::pack4(q8::scaled(y[0], inv), q8::scaled(y[1], inv), q8::scaled(y[2], inv), q8::scaled(y[3], inv));
        }
        uint8_t* dst = static_cast<uint8_t*>(p.v_dst) + block * 16;
        uint8_t* scale = p.v_scale + eg * p.scale_tokens + (at.tok & ~15);
        if (whole) {
            u32x4_t out[4], bytes;  // out[dim][4 tokens]
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t* q = &w[4 * i];
                const uint32_t ab = __builtin_amdgcn_perm(q[1], q[0], 0x05010400u), cd = __builtin_amdgcn_perm(q[3], q[2], 0x05010400u);
                const uint32_t AB = __builtin_amdgcn_perm(q[1], q[0], 0x07030602u), CD = __builtin_amdgcn_perm(q[3], q[2], 0x07030602u);
                out[0][i] = __builtin_amdgcn_perm(cd, ab, 0x05040100u);
                out[1][i] = __builtin_amdgcn_perm(cd, ab, 0x07060302u);
                out[2][i] = __builtin_amdgcn_perm(CD, AB, 0x05040100u);
                out[3][i] = __builtin_amdgcn_perm(CD, AB, 0x07060302u);
                bytes[i] = byte[4 * i] | byte[4 * i + 1] << 8 | byte[4 * i + 2] << 16 | byte[4 * i + 3] << 24;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<u32x4_t*>(dst + 16 * j) = out[j];
            if (x == 0) *reinterpret_cast<u32x4_t*>(scale) = bytes;
        } else {
#pragma unroll
            for (int t = 0; t < 16; ++t)
                if (t >= lo && t < hi) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) dst[16 * j + t] = uint8_t(w[t] >> (8 * j));
                    if (x == 0) scale[t] = uint8_t(byte[t]);
                }
        }
    } else {
        // slot 8h + 4a + b of a dim's row holds token 8a + 4h + b
        uint16_t* dst = static_cast<uint16_t*>(p.v_dst) + block * 16;
        if (whole) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                u32x4_t out[2];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int t = 8 * (i / 2 % 2) + 4 * (i / 4) + 2 * (i % 2);
                    out[i / 4][i % 4] = __builtin_amdgcn_perm(j / 2 ? v[t + 1].y : v[t + 1].x, j / 2 ? v[t].y : v[t].x,
                                                              j % 2 ? 0x07060302u : 0x05040100u);
                }
                *reinterpret_cast<u32x4_t*>(dst + 16 * j) = out[0];
                *reinterpret_cast<u32x4_t*>(dst + 16 * j + 8) = out[1];
            }
        } else {
#pragma unroll
            for (int t = 0; t < 16; ++t)
                if (t >= lo && t < hi) {
                    uint16_t* to = dst + 8 * (t / 4 % 2) + 4 * (t / 8) + t % 4;
                    to[0] = uint16_t(v[t].x);
                    to[16] = uint16_t(v[t].x >> 16);
                    to[32] = uint16_t(v[t].y);
                    to[48] = uint16_t(v[t].y >> 16);
                }
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
    if (wave >= p.row_waves) return;
    // this wave's tokens and its heads, all of one kind: queries, keys, values
    const int hpw = p.heads_per_wave;
    const uint32_t q_parts = uint32_t(p.h_q + hpw - 1) / uint32_t(hpw), k_parts = uint32_t(p.h_kv + hpw - 1) / uint32_t(hpw);
    const uint32_t parts = q_parts + k_parts + (p.value_rows ? k_parts : 0u);
    uint32_t part = wave % parts;
    const int kind = part < q_parts ? 0 : part < q_parts + k_parts ? 1 : 2;
    part -= kind == 0 ? 0u : kind == 1 ? q_parts : q_parts + k_parts;
    const int n_heads = kind == 0 ? p.h_q : p.h_kv;
    const int from = int(part) * hpw, to = min(from + hpw, n_heads);
    const uint32_t rows = uint32_t(p.batch) * uint32_t(p.n_new);
    const uint32_t row = wave / parts * uint32_t(kTokens) + uint32_t(lane / kLanes);
    const uint32_t r = min(row, rows - 1);
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

    const uint32_t b = r / uint32_t(p.n_new);
    const Token at = locate(p, int(b), int(r - b * uint32_t(p.n_new)), row < rows);
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
            const float rs = rsqrtf(__builtin_fmaf(sum_lanes<kLanes>(ss), 1.f / D, p.eps));
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] *= rs;
        }
    };
    const auto query = [&](int h, u32x4_t v) __attribute__((always_inline)) {
        float y[8];
        turned(v, y);
        if (at.active) store16<kStream>(p.q_out + (int64_t(r) * p.h_q + h) * D + 8 * l, to_bf16(y));
    };
    const auto key = [&](int g, u32x4_t v) __attribute__((always_inline)) {
        float y[8];
        turned(v, y);
        const int64_t to_k = (((eg0 + g) * kChunks + c) * at.cap + at.tok) * 16 + 8 * hf;
        if constexpr (kQ8) {
            const uint32_t byte = q8::scale_byte(max_lanes<kLanes>(finite_max<8>(y)));
            const float inv = q8::inverse_power(byte);
            float z[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = q8::scaled(y[e], inv);
            if (at.stored) {
                *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.k_dst) + to_k) =
                    make_uint2(q8::pack4(z[0], z[1], z[2], z[3]), q8::pack4(z[4], z[5], z[6], z[7]));
                if (l == 0) p.k_scale[(eg0 + g) * p.scale_tokens + at.tok] = uint8_t(byte);
            }
        } else if (at.stored) {
            *reinterpret_cast<u32x4_t*>(static_cast<uint16_t*>(p.k_dst) + to_k) = to_bf16(y);
        }
    };
    // a value by itself: its dims are 16 numbers apart
    const auto value = [&](int g, u32x4_t v) __attribute__((always_inline)) {
        const int64_t to_v = (((eg0 + g) * ((at.cap + 15) / 16) + at.tok / 16) * D + 8 * l) * 16;
        if constexpr (kQ8) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = e & 1 ? bf_hi(v[e / 2]) : bf_lo(v[e / 2]);
            const uint32_t byte = q8::scale_byte(max_lanes<kLanes>(finite_max<8>(y)));
            const float inv = q8::inverse_power(byte);
            uint8_t* dst = static_cast<uint8_t*>(p.v_dst) + to_v + at.tok % 16;
            uint32_t w[2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                w[i] = q8::pack4(q8::scaled(y[4 * i], inv), q8::scaled(y[4 * i + 1], inv),
                                 q8::scaled(y[4 * i + 2], inv), q8::scaled(y[4 * i + 3], inv));
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
}

template <int D>
hipError_t launch_d(AppendNormedParams p, hipStream_t stream) {
    constexpr int kTokens = 64 / (D / 8);
    const int64_t groups = (int64_t(p.batch) * p.n_new + kTokens - 1) / kTokens;
    // one head a wave until the chip is full of waves, then as many as keep it full, so that a
    // token's angles serve them all
    const int64_t target = 4096;
    p.value_rows = p.n_new < 8;
    const int64_t heads = p.h_q + p.h_kv;
    p.heads_per_wave = int32_t(std::min(heads, std::max<int64_t>(1, groups * heads / target)));
    const auto parts = [&](int64_t h) { return (h + p.heads_per_wave - 1) / p.heads_per_wave; };
    const int64_t row_waves = groups * (parts(p.h_q) + (p.value_rows ? 2 : 1) * parts(p.h_kv));
    const int64_t units = int64_t(p.batch) * ((int64_t(p.n_new) + 14) / 16 + 1) * p.h_kv;
    // whole workgroups of blocks
    const int64_t block_waves = p.value_rows ? 0 : ((units + 256 / D - 1) / (256 / D) + 3) / 4 * 4;
    const int64_t waves = row_waves + block_waves;
    if (waves < 1 || waves > 0x7FFFFFFF || units > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
    p.row_waves = uint32_t(row_waves);
    p.block_waves = uint32_t(block_waves);
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
