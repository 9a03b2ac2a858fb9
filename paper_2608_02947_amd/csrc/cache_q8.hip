// Reading an 8-bit cache back into bf16 caches: every number times its row's power, exactly (an
// e4m3 number has 4 significant bits), in the layouts the prefill and the bf16 decode read.
// Moves 3 bytes a number; bound by HBM: 131,072 tokens of 4 heads of 128 404 MB in 72 us (5.6 TB/s;
// a device copy reaches 5.4).
#include "atf_internal.hpp"
#include "q8.hpp"

#include <algorithm>

namespace atf {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t two_bf16(float a, float b) {
    bf16x2_t two;
    two[0] = (__bf16)a;
    two[1] = (__bf16)b;
    return __builtin_bit_cast(uint32_t, two);
}

// Grid y: (batch row, KV head).  x: first the keys, one thread per token of a chunk, chunk by
// chunk (few streams at a time: a thread that took four chunks of its token moved 131,072 x 4
// heads in 87 us for 71), then the values, one thread per (16-token block, dim).
template <int D>
__global__ __launch_bounds__(256) void read_q8_kernel(const ReadQ8Params p) {
    constexpr int kChunks = D / 16;
    const int g = blockIdx.y % p.h_kv, b = blockIdx.y / p.h_kv;
    // the entry of the source that holds position t: (row of KV head g, first position, capacity)
    const auto entry = [&](int t, int64_t& eg, int& base, int64_t& cap) __attribute__((always_inline)) {
        eg = int64_t(b) * p.h_kv + g;
        base = 0;
        cap = p.src_tokens;
        if (p.block_table != nullptr) {
            const int at = t / p.page_tokens;
            const int page = min(max(p.block_table[int64_t(b) * p.max_pages + at], 0), p.num_pages - 1);
            eg = int64_t(page) * p.h_kv + g;
            base = at * p.page_tokens;
            cap = p.page_tokens;
        }
    };
    const int64_t bh = int64_t(b) * p.h_kv + g;
    int64_t eg, cap;
    int base;
    if (blockIdx.x < p.key_blocks * kChunks) {
        const uint32_t c = blockIdx.x / p.key_blocks, i = (blockIdx.x - c * p.key_blocks) * 256u + threadIdx.x;
        if (i >= uint32_t(p.n_k)) return;
        const int t = p.pos0 + int(i);
        entry(t, eg, base, cap);
        const float f = q8::power(p.k_scale[eg * p.scale_tokens + t - base]);
        const u32x4_t x = *reinterpret_cast<const u32x4_t*>(p.k_src + ((eg * kChunks + c) * cap + t - base) * 16);
        uint16_t* dst = p.k_dst + ((bh * kChunks + c) * p.dst_tokens + t) * 16;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u32x4_t y;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x2_t v = j & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(x[2 * h + j / 2], true)
                                        : __builtin_amdgcn_cvt_pk_f32_fp8(x[2 * h + j / 2], false);
                y[j] = two_bf16(v[0] * f, v[1] * f);
            }
            *reinterpret_cast<u32x4_t*>(dst + 8 * h) = y;
        }
    } else {
        const uint64_t i = uint64_t(blockIdx.x - p.key_blocks * kChunks) * 256u + threadIdx.x;
        const int blk = p.pos0 / 16 + int(i / D), x = int(i % D);
        if (blk > (p.pos0 + p.n_k - 1) / 16) return;
        entry(16 * blk, eg, base, cap);
        const int sb = blk - base / 16;
        const u32x4_t v = *reinterpret_cast<const u32x4_t*>(p.v_src + ((eg * ((cap + 15) / 16) + sb) * D + x) * 16);
        const u32x4_t f = *reinterpret_cast<const u32x4_t*>(p.v_scale + eg * p.scale_tokens + 16 * sb);
        uint32_t out[8];  // slots 2j, 2j + 1: tokens 8 (j / 2 % 2) + 4 (j / 4) + 2 (j % 2) ..
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int t = 8 * (j / 2 % 2) + 4 * (j / 4) + 2 * (j % 2);
            const f32x2_t two = t & 2 ? __builtin_amdgcn_cvt_pk_f32_fp8(v[t / 4], true)
                                      : __builtin_amdgcn_cvt_pk_f32_fp8(v[t / 4], false);
            const uint32_t s = f[t / 4] >> (8 * (t % 4));
            out[j] = two_bf16(two[0] * q8::power(s & 255u), two[1] * q8::power(s >> 8 & 255u));
        }
        uint16_t* dst = p.v_dst + ((bh * ((int64_t(p.dst_tokens) + 15) / 16) + blk) * D + x) * 16;
        const int lo = p.pos0 - 16 * blk, hi = p.pos0 + p.n_k - 16 * blk;
        if (lo <= 0 && hi >= 16) {
            *reinterpret_cast<u32x4_t*>(dst) = u32x4_t{out[0], out[1], out[2], out[3]};
            *reinterpret_cast<u32x4_t*>(dst + 8) = u32x4_t{out[4], out[5], out[6], out[7]};
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int t = 8 * (j / 2 % 2) + 4 * (j / 4) + 2 * (j % 2) + k;
                    if (t >= lo && t < hi) dst[2 * j + k] = uint16_t(k ? out[j] >> 16 : out[j]);
                }
        }
    }
}

template <int D>
hipError_t launch_read_d(ReadQ8Params p, hipStream_t stream) {
    const int64_t rows = int64_t(p.batch) * p.h_kv, end = int64_t(p.pos0) + p.n_k;
    if (rows < 1 || rows > 65535 || p.n_k < 1) return hipErrorInvalidConfiguration;
    (void)hipGetLastError();
    // (2^27 tokens and more in several launches: a grid has less than 2^32 threads a side)
    constexpr int64_t kMost = int64_t(1) << 27;
    for (int64_t from = p.pos0; from < end; from += kMost) {
        p.pos0 = int32_t(from);
        p.n_k = int32_t(std::min(kMost, end - from));
        p.key_blocks = uint32_t((p.n_k + 255) / 256);
        const int64_t nblk = (from + p.n_k - 1) / 16 + 1 - from / 16;
        const int64_t blocks = int64_t(p.key_blocks) * (D / 16) + (nblk * D + 255) / 256;
        hipLaunchKernelGGL(read_q8_kernel<D>, dim3(unsigned(blocks), unsigned(rows)), dim3(256), 0, stream, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_read_q8(const ReadQ8Params& p, int head_dim, hipStream_t stream) {
    return head_dim == 64 ? launch_read_d<64>(p, stream) : launch_read_d<128>(p, stream);
}

}  // namespace atf
