// Pages and slots of a batch from its rows' lengths, and tokens appended through their slots, gfx950.
//
// Plan (plan_kernel, one workgroup).  Rows b = 0 .. B - 1 hold n_b tokens and get m_b.  With
// p(x) = ceil(x / page_tokens):
//   a row that ends (m_b < 0) gives back its p(n_b) pages: they go on top of the stack of free ones,
//     rows and pages in order; f is the stack's height then
//   a row that grows needs p(n_b + m_b) - p(n_b) pages; with E_b the sum of the needs up to and with
//     row b it gets them if E_b <= f: page i of it is entry f - 1 - (E_b - need_b) - i
//   token i of it is at position n_b + i: slot = page of the position * page_tokens + the rest
// So it takes two sums over the rows: of the pages given back, then, row by row, of the needs and of
// the tokens.  1,024 rows at a time, a thread each; the pages of a row move by pieces of 256, a
// wave each, in turn.  Tokens are found from their number by a search in the rows' first tokens:
// in the same workgroup if they are few, else by slots_kernel, which finds a row's first position,
// or -1 if the row got nothing, where the plan left it: at the row's first token.
//
// Bound by latency: a launch, and a few loads that wait for one another.
#include "atf_internal.hpp"
#include "rope.hpp"

#include <algorithm>

namespace atf {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;
constexpr int kPiece = 256;        // pages that a wave moves at once
constexpr int kSlotThreads = 256;
constexpr int kSlotRows = 2048;    // rows whose first tokens slots_kernel holds in LDS

__device__ __forceinline__ int64_t scan_wave(int64_t x, int lane) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    return x;
}

// Each thread's sum of the threads up to it, and the sum of all.  `part` is free again after the
// next barrier.
__device__ __forceinline__ int64_t scan_block(int64_t x, int64_t* part, int64_t* all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    x = scan_wave(x, lane);
    if (lane == 63) part[wave] = x;
    __syncthreads();
    int64_t before = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < kPlanWaves; ++w) {
        const int64_t y = part[w];
        before += w < wave ? y : 0;
        sum += y;
    }
    *all = sum;
    return x + before;
}

struct PlanRow {
    int n, grow;     // tokens it holds, tokens it is to get
    int have, need;  // pages of the former, pages that the latter take
    bool ends, fits;
};
__device__ __forceinline__ PlanRow plan_row(const PlanParams& p, int b) {
    PlanRow r = {0, 0, 0, 0, false, false};
    if (b >= p.batch) return r;
    const int64_t cap = int64_t(p.max_pages) * p.page_tokens;
    const int m = p.n_new_rows[b];
    r.n = int(min(int64_t(max(p.n_k_rows[b], 0)), cap));
    r.ends = m < 0;
    r.grow = max(m, 0);
    r.have = int((uint32_t(r.n) + p.page_tokens - 1) / uint32_t(p.page_tokens));
    r.fits = int64_t(r.n) + r.grow <= cap;
    if (r.fits) r.need = int((uint32_t(r.n) + r.grow + p.page_tokens - 1) / uint32_t(p.page_tokens)) - r.have;
    return r;
}

// The row of token t: the last one whose first token is not past it and that has tokens
// (starts[0 .. n], ascending, starts[0] <= t < starts[n]).
template <typename T>
__device__ __forceinline__ int row_of_token(const T* starts, int n, int t) {
    int lo = 0, hi = n;  // starts[lo] <= t < starts[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= t)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

__device__ __forceinline__ void write_token(const PlanParams& p, int t, int row, int pos) {
    int64_t slot = -1;
    if (pos >= 0) {
        const int page = p.block_table[int64_t(row) * p.max_pages + pos / p.page_tokens];
        if (page >= 0) slot = int64_t(page) * p.page_tokens + pos % p.page_tokens;
    }
    p.slots[t] = slot;
    p.token_rows[t] = pos >= 0 ? row : -1;
    p.positions[t] = pos;
}

// kTokens: the tokens too (rows fit one pass then)
template <bool kTokens>
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(const PlanParams p) {
    __shared__ int64_t s_part[3][kPlanWaves];
    __shared__ int s_start[kTokens ? kPlanThreads + 1 : 1];
    __shared__ int s_first[kTokens ? kPlanThreads : 1];
    // rows whose pages move by pieces: pages, the first entry of the row, of the stack
    __shared__ int s_rows;
    __shared__ int s_count[kPlanThreads], s_entry[kPlanThreads], s_stack[kPlanThreads];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int max_tokens = p.max_tokens;

    // a row's pages to (given) or from the stack; few at once by the row's own thread
    const auto move = [&](int rows0, int b, int count, int entry, int64_t stack, bool given) {
        int slot = -1;
        if (count > 0 && count <= 2) {
            int32_t* at = p.block_table + int64_t(b) * p.max_pages + entry;
            for (int i = 0; i < count; ++i) {
                if (given) {
                    if (stack + i < p.free_capacity) p.free_pages[stack + i] = at[i];
                } else {
                    at[i] = p.free_pages[stack - i];
                }
            }
        } else if (count > 2) {
            slot = tid;
        }
        s_count[tid] = slot >= 0 ? count : 0;
        s_entry[tid] = entry;
        s_stack[tid] = int(stack);
        if (tid == 0) s_rows = 0;
        __syncthreads();
        if (slot >= 0) atomicMax(&s_rows, tid + 1);
        __syncthreads();
        const int rows = s_rows;
        for (int r = 0, turn = wave; r < rows; ++r) {
            const int n = s_count[r];
            if (n == 0) continue;
            int32_t* at = p.block_table + int64_t(rows0 + r) * p.max_pages + s_entry[r];
            const int64_t from = s_stack[r];
            for (; turn * kPiece < n; turn += kPlanWaves) {
#pragma unroll
                for (int k = 0; k < kPiece / 64; ++k) {
                    const int i = turn * kPiece + 64 * k + lane;
                    if (i >= n) continue;
                    if (given) {
                        if (from + i < p.free_capacity) p.free_pages[from + i] = at[i];
                    } else {
                        at[i] = p.free_pages[from - i];
                    }
                }
            }
            turn -= (n + kPiece - 1) / kPiece;  // the next row's pieces go on with the next wave
        }
        __syncthreads();
    };

    // pages given back
    const int64_t f0 = min(max(*p.free_count, 0), p.free_capacity);
    int64_t given = 0;
    for (int r0 = 0; r0 < p.batch; r0 += kPlanThreads) {
        const PlanRow r = plan_row(p, r0 + tid);
        int64_t all;
        const int64_t mine = r.ends ? r.have : 0;
        const int64_t end = scan_block(mine, s_part[0], &all);
        if (all == 0) {
            __syncthreads();
            continue;
        }
        move(r0, r0 + tid, int(mine), 0, min(f0 + given + end - mine, int64_t(p.free_capacity)), true);
        given += all;
    }
    const int64_t f = min(f0 + given, int64_t(p.free_capacity));

    // pages taken
    int64_t needed = 0, tokens = 0, taken = 0, refused = 0;
    for (int r0 = 0; r0 < p.batch; r0 += kPlanThreads) {
        const int b = r0 + tid;
        const PlanRow r = plan_row(p, b);
        int64_t all_need, all_grow, all_taken;
        const int64_t need_end = needed + scan_block(r.need, s_part[0], &all_need);
        const int64_t end = tokens + scan_block(r.grow, s_part[1], &all_grow);
        const bool ok = r.grow > 0 && r.fits && need_end <= f && end <= max_tokens;
        const int64_t start = end - r.grow;
        // (one sum for both: the pages of 1,024 rows are fewer than 2^40)
        scan_block((int64_t(r.grow > 0 && !ok) << 40) + (ok ? r.need : 0), s_part[2], &all_taken);
        const int64_t all_refused = all_taken >> 40;
        all_taken &= (int64_t(1) << 40) - 1;
        const int first = ok ? r.n : -1;
        if (b < p.batch) {
            p.row_starts[b + 1] = int(min(end, int64_t(max_tokens)));
            p.n_k_out[b] = r.ends ? 0 : ok ? r.n + r.grow : r.n;
            if (!kTokens && r.grow > 0 && start < max_tokens) p.positions[start] = first;
        }
        if (kTokens) {
            s_start[tid + 1] = int(min(end, int64_t(max_tokens)));
            s_first[tid] = first;
        }
        move(r0, b, ok ? r.need : 0, r.have, f - 1 - (need_end - r.need), false);
        needed += all_need;
        tokens += all_grow;
        taken += all_taken;
        refused += all_refused;
    }
    if (tid == 0) {
        p.row_starts[0] = 0;
        p.counts[0] = int(f - taken);
        p.counts[1] = int(min(tokens, int64_t(max_tokens)));
        p.counts[2] = int(refused);
        if (kTokens) s_start[0] = 0;
    }
    if constexpr (kTokens) {
        __syncthreads();
        const int n = int(min(tokens, int64_t(max_tokens)));
        for (int t = tid; t < max_tokens; t += kPlanThreads) {
            int row = -1, pos = -1;
            if (t < n) {
                row = row_of_token(s_start, p.batch, t);
                pos = s_first[row] < 0 ? -1 : s_first[row] + t - s_start[row];
            }
            write_token(p, t, row, pos);
        }
    }
}

__global__ __launch_bounds__(kSlotThreads) void slots_kernel(const PlanParams p) {
    __shared__ int s_start[kSlotRows + 1];
    const bool held = p.batch <= kSlotRows;
    if (held) {
        for (int i = threadIdx.x; i <= p.batch; i += kSlotThreads) s_start[i] = p.row_starts[i];
        __syncthreads();
    }
    const int n = p.row_starts[p.batch];
    for (int64_t at = int64_t(blockIdx.x) * kSlotThreads + threadIdx.x; at < p.max_tokens;
         at += int64_t(gridDim.x) * kSlotThreads) {
        const int t = int(at);
        int row = -1, pos = -1;
        if (t < n) {
            row = held ? row_of_token(s_start, p.batch, t) : row_of_token(p.row_starts, p.batch, t);
            const int start = held ? s_start[row] : p.row_starts[row];
            const int first = p.positions[start];  // (the row's first token writes it again, as it is)
            pos = first < 0 ? -1 : first + t - start;
        }
        write_token(p, t, row, pos);
    }
}

// Appends through slots.  A run is tokens, one behind the other in the call, whose slots follow each
// other inside a 16-token block of a page: a wave writes one head of a run.  Token t leads a run if
// its slot starts a block or does not follow the slot of t - 1.  kWindow tokens a wave: 1 where
// tokens are few (most waves of a prompt have no leader then), else 16, where prompts have one or two.
//   keys: lanes along a token's row, 16 bytes each of both halves of a chunk, 32 bytes stored
//   values: a lane takes 2 dims; a whole block's 16 tokens by two 16-byte stores a dim, others by
//     2 bytes a token
template <int D, bool kTurn, int kWindow>
__global__ __launch_bounds__(256) void append_slots_kernel(const AppendSlotsParams p) {
    constexpr int kChunks = D / 16;
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const int lane = threadIdx.x & 63;
    const int64_t windows = (int64_t(p.n_tokens) + kWindow - 1) / kWindow;
    const int64_t unit = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    const int g = int(unit % p.h_kv);
    const int64_t win = unit / p.h_kv;
    if (win >= windows) return;
    const int t0 = int(win) * kWindow;
    // slots of the tokens t0 - 1 .. t0 + kWindow + 14
    int64_t slot = -1;
    {
        const int64_t t = int64_t(t0) - 1 + lane;
        if (lane <= kWindow + 15 && t >= 0 && t < p.n_tokens) slot = p.slots[t];
        if (slot < 0 || slot >= p.pool_tokens) slot = -1;
    }
    const int64_t before = __shfl_up(slot, 1);
    const uint64_t valid = __ballot(slot >= 0);
    const uint64_t leads = __ballot(lane > 0 && slot >= 0 && (slot % 16 == 0 || slot != before + 1));
    uint64_t todo = leads & (((uint64_t(1) << kWindow) - 1) << 1);
    while (todo) {
        const int l = __builtin_ctzll(todo);
        todo &= todo - 1;
        // the run: up to the next leader, the next token that is not stored, or 16
        const uint64_t stops = (leads | ~valid) >> (l + 1);
        const int n = min(16, __builtin_ctzll(stops) + 1);  // (lanes past the window's end stop it)
        const int t = t0 - 1 + l;
        const int64_t first = __shfl(slot, l);
        const int64_t page = first / p.page_tokens;
        const int at = int(first % p.page_tokens);
        const int64_t ph = page * p.h_kv + g;
        uint16_t* kd = p.k_pages + (ph * kChunks * p.page_tokens + at) * 16;
        uint16_t* vd = p.v_pages + (ph * (p.page_tokens / 16) + at / 16) * int64_t(D) * 16;
        const int64_t row = int64_t(p.h_kv) * D, src0 = (int64_t(t) * p.h_kv + g) * D;
        // keys: record i = (token i / chunks, chunk i % chunks)
        for (int i = lane; i < n * kChunks; i += 64) {
            const int x = i / kChunks, c = i % kChunks;
            const uint16_t* src = p.k_new + src0 + x * row + 8 * c;
            u32x4 lo = *reinterpret_cast<const u32x4*>(src), hi = *reinterpret_cast<const u32x4*>(src + D / 2);
            if constexpr (kTurn) {
                const uint32_t pos = uint32_t(p.positions[t + x]);
                float cs8[8], sn8[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float u = rope::revolutions(pos, make_uint2(p.rope_rho_hi[8 * c + e], p.rope_rho_lo[8 * c + e]));
                    cs8[e] = __builtin_amdgcn_cosf(u);
                    sn8[e] = __builtin_amdgcn_sinf(u);
                }
                const u32x4 a = lo, b = hi;
                lo = rope::rotate_cs(a, b, 0, cs8, sn8);
                hi = rope::rotate_cs(b, a, 1, cs8, sn8);
            }
            u32x4* dst = reinterpret_cast<u32x4*>(kd + (int64_t(c) * p.page_tokens + x) * 16);
            dst[0] = lo;
            dst[1] = hi;
        }
        // values: slot 8h + 4a + b of a dim's 16 holds token 8a + 4h + b
        if (2 * lane < D) {
            const int b0 = at % 16;
            for (int x = 0; x < n; ++x) {
                const uint32_t two = *reinterpret_cast<const uint32_t*>(p.v_new + src0 + x * row + 2 * lane);
                const int k = b0 + x, s = 8 * ((k >> 2) & 1) + 4 * (k >> 3) + (k & 3);
                vd[(2 * lane) * 16 + s] = uint16_t(two);
                vd[(2 * lane + 1) * 16 + s] = uint16_t(two >> 16);
            }
        }
    }
}

template <int D, bool kTurn>
hipError_t launch_append_slots_d(const AppendSlotsParams& p, hipStream_t stream) {
    const bool few = int64_t(p.n_tokens) * p.h_kv <= 8192;
    const int64_t windows = few ? p.n_tokens : (int64_t(p.n_tokens) + 15) / 16;
    const int64_t blocks = (windows * p.h_kv + 3) / 4;
    if (blocks * 256 > 0xFFFFFFFF) return hipErrorInvalidConfiguration;
    const dim3 grid(static_cast<unsigned>(blocks));
    if (few)
        hipLaunchKernelGGL((append_slots_kernel<D, kTurn, 1>), grid, dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL((append_slots_kernel<D, kTurn, 16>), grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_plan_pages(const PlanParams& p, hipStream_t stream) {
    (void)hipGetLastError();
    if (p.batch <= kPlanThreads && p.max_tokens <= 8192) {
        hipLaunchKernelGGL(plan_kernel<true>, dim3(1), dim3(kPlanThreads), 0, stream, p);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(plan_kernel<false>, dim3(1), dim3(kPlanThreads), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.max_tokens == 0) return e;
    const unsigned blocks = unsigned(std::min<int64_t>(2048, (int64_t(p.max_tokens) + kSlotThreads - 1) / kSlotThreads));
    hipLaunchKernelGGL(slots_kernel, dim3(blocks), dim3(kSlotThreads), 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_append_slots(const AppendSlotsParams& p, bool turn, int head_dim, hipStream_t stream) {
    (void)hipGetLastError();
    if (head_dim == 64) return turn ? launch_append_slots_d<64, true>(p, stream) : launch_append_slots_d<64, false>(p, stream);
    return turn ? launch_append_slots_d<128, true>(p, stream) : launch_append_slots_d<128, false>(p, stream);
}

}  // namespace atf
