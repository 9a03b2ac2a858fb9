// Pages and slots of a batch from its rows' lengths, and tokens appended through their slots, gfx950.
//
// Plan (plan_kernel, one workgroup).  Rows b = 0 .. B - 1 hold n_b tokens and get m_b.  With
// p(x) = ceil(x / page_tokens):
//   a row that ends (m_b < 0) gives back its p(n_b) pages: they go on top of the stack of free ones,
//     rows and pages in order; f is the stack's height then
//   a row that grows needs p(n_b + m_b) - p(n_b) pages; with E_b the sum of the needs up to and with
//     row b it gets them if E_b <= f: page i of it is entry f - 1 - (E_b - need_b) - i
//   token i of it is at position n_b + i: slot = page of the position * page_tokens + the rest
// So it takes sums over the rows, of the pages given back, of the needs and of the tokens: a pass for
// 1,024 rows, a thread each.  Up to 2 pages or tokens of a row are its thread's work, more go by
// pieces of 256, a wave each in turn.  Where tokens are many slots_kernel writes them: it finds a
// token's row by a search in the rows' first tokens, and the row's first position, or -1 if the row got
// nothing, where the plan left it: at the row's first token.
//
// Bound by latency: a launch, and loads that wait for one another (200 rows of a step with 5,900 tokens 10.2
// us in a captured graph, 24 prompts with 274,000 tokens 11.2).
#include "atf_internal.hpp"
#include "rope.hpp"
#include "scan.hpp"

#include <algorithm>

namespace atf {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;
constexpr int kPiece = 256;        // pages that a wave moves at once
constexpr int kSlotThreads = 256;
constexpr int kSlotRows = 2048;    // rows whose first tokens slots_kernel holds in LDS

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

// Rows of one pass whose pages or tokens move by pieces, and what each row needs for that.
struct PlanPass {
    int count[3];                 // rows listed: pages given back, pages taken, tokens written
    int rows[3][kPlanThreads];
    int n[kPlanThreads], grow[kPlanThreads], start[kPlanThreads], have[kPlanThreads], need[kPlanThreads];
    int64_t stack[kPlanThreads];  // the stack's entry of the row's first page
};
constexpr int kGive = 0, kTake = 1, kWrite = 2;

// body(row of the pass, first) for each piece of the listed rows, a wave each in turn
template <typename Size, typename Body>
__device__ __forceinline__ void by_pieces(const PlanPass& s, int list, Size size, Body body) {
    int turn = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rows = s.count[list];
    for (int k = 0; k < rows; ++k) {
        const int r = __builtin_amdgcn_readfirstlane(s.rows[list][k]);
        const int pieces = (__builtin_amdgcn_readfirstlane(size(r)) + kPiece - 1) / kPiece;
        for (; turn < pieces; turn += kPlanWaves) body(r, turn * kPiece);
        turn -= pieces;  // the next row's go on with the next wave
    }
}

// Int holds the sums of all rows' pages and tokens; kOne: the rows are one pass (their numbers stay
// in registers), and kTokens: their tokens are written here.
template <typename Int, bool kOne, bool kTokens>
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(const PlanParams p) {
    __shared__ Int s_part[2][3][kPlanWaves];
    __shared__ PlanPass s;
    __shared__ int s_refused;
    __shared__ int64_t s_taken;
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t f0 = min(max(*p.free_count, 0), p.free_capacity);
    if (tid < 3) s.count[tid] = 0;
    if (tid == 0) s_refused = 0, s_taken = 0;

    const auto table = [&](int b) { return p.block_table + int64_t(b) * p.max_pages; };
    const auto give = [&](int r0, const PlanRow& r, int64_t stack) {
        // (past the capacity: nothing)
        stack = min(stack, int64_t(p.free_capacity));
        if (r.ends && r.have <= 2) {
            for (int i = 0; i < r.have; ++i)
                if (stack + i < p.free_capacity) p.free_pages[stack + i] = table(r0 + tid)[i];
        } else if (r.ends) {
            s.rows[kGive][atomicAdd(&s.count[kGive], 1)] = tid;
            s.have[tid] = r.have;
            s.stack[tid] = stack;
        }
    };
    const auto give_pieces = [&](int r0) {
        by_pieces(s, kGive, [&](int r) { return s.have[r]; }, [&](int r, int first) {
            const int32_t* from = table(r0 + r);
            int32_t page[kPiece / 64];
#pragma unroll
            for (int k = 0; k < kPiece / 64; ++k) page[k] = from[min(first + 64 * k + lane, s.have[r] - 1)];
#pragma unroll
            for (int k = 0; k < kPiece / 64; ++k) {
                const int i = first + 64 * k + lane;
                if (i < s.have[r] && s.stack[r] + i < p.free_capacity) p.free_pages[s.stack[r] + i] = page[k];
            }
        });
    };
    // (rest: the token's place in its page)
    const auto write = [&](int t, int b, int pos, int page, int rest) {
        const bool is = pos >= 0;
        p.slots[t] = is && page >= 0 ? int64_t(page) * p.page_tokens + rest : -1;
        p.token_rows[t] = is ? b : -1;
        p.positions[t] = pos;
    };

    PlanRow r = plan_row(p, tid);
    Int all[3], x[3] = {Int(r.ends ? r.have : 0), Int(r.need), Int(min(r.grow, p.max_tokens + 1))};
    int64_t f;
    if constexpr (kOne) {
        const Int back = x[0];
        scan::block<kPlanWaves>(x, all, s_part[0]);
        f = min(f0 + all[0], int64_t(p.free_capacity));
        if (all[0] > 0) {
            give(0, r, f0 + x[0] - back);
            __syncthreads();
            give_pieces(0);
            __syncthreads();
        }
    } else {
        int64_t given = 0;
        for (int r0 = 0; r0 < p.batch; r0 += kPlanThreads) {
            r = plan_row(p, r0 + tid);
            Int y[1] = {Int(r.ends ? r.have : 0)}, sum[1];
            const Int back = y[0];
            scan::block<kPlanWaves>(y, sum, s_part[0]);
            give(r0, r, f0 + given + y[0] - back);
            __syncthreads();
            give_pieces(r0);
            __syncthreads();
            if (tid == 0) s.count[kGive] = 0;
            given += sum[0];
            __syncthreads();
        }
        f = min(f0 + given, int64_t(p.free_capacity));
    }

    int64_t needed = 0, tokens = 0;
    for (int r0 = 0; r0 < (kOne ? 1 : p.batch); r0 += kPlanThreads) {
        const int b = r0 + tid;
        if constexpr (!kOne) {
            r = plan_row(p, b);
            x[0] = 0;
            x[1] = Int(r.need);
            x[2] = Int(min(r.grow, p.max_tokens + 1));
            scan::block<kPlanWaves>(x, all, s_part[1]);
        }
        const int64_t need_end = needed + x[1], end = tokens + x[2];
        const bool ok = r.grow > 0 && r.fits && need_end <= f && end <= p.max_tokens;
        const int start = int(min(end - min(r.grow, p.max_tokens + 1), int64_t(p.max_tokens)));
        const int64_t stack = f - 1 - (need_end - r.need);
        if (b < p.batch) {
            p.row_starts[b + 1] = int(min(end, int64_t(p.max_tokens)));
            p.n_k_out[b] = r.ends ? 0 : ok ? r.n + r.grow : r.n;
            if (!kTokens && r.grow > 0 && start < p.max_tokens) p.positions[start] = ok ? r.n : -1;
        }
        // the rows that get pages come before all others that want some
        if (ok && r.need > 0) atomicMax(reinterpret_cast<unsigned long long*>(&s_taken), (unsigned long long)(need_end));
        const uint64_t no = __ballot(r.grow > 0 && !ok);
        if (lane == 0 && no != 0) atomicAdd(&s_refused, __builtin_popcountll(no));
        const int count = kTokens ? min(r.grow, p.max_tokens - start) : 0;
        bool info = false;
        if (ok && r.need <= 2) {
            for (int i = 0; i < r.need; ++i) table(b)[r.have + i] = p.free_pages[stack - i];
        } else if (ok) {
            s.rows[kTake][atomicAdd(&s.count[kTake], 1)] = tid;
            info = true;
        }
        if (kTokens && count > 2) {
            s.rows[kWrite][atomicAdd(&s.count[kWrite], 1)] = tid;
            info = true;
        } else if (kTokens) {
            for (int i = 0; i < count; ++i) {
                const int pos = ok ? r.n + i : -1, at = max(pos, 0) / p.page_tokens;
                write(start + i, b, pos, !ok ? -1 : at < r.have ? table(b)[at] : p.free_pages[stack - (at - r.have)],
                      pos - at * p.page_tokens);
            }
        }
        if (info) {
            s.n[tid] = ok ? r.n : -1;
            s.grow[tid] = count;
            s.start[tid] = start;
            s.have[tid] = r.have;
            s.need[tid] = ok ? r.need : 0;
            s.stack[tid] = stack;
        }
        __syncthreads();
        by_pieces(s, kTake, [&](int q) { return s.need[q]; }, [&](int q, int first) {
            int32_t page[kPiece / 64];
            int32_t* to = table(r0 + q) + s.have[q];
#pragma unroll
            for (int k = 0; k < kPiece / 64; ++k) page[k] = p.free_pages[s.stack[q] - min(first + 64 * k + lane, s.need[q] - 1)];
#pragma unroll
            for (int k = 0; k < kPiece / 64; ++k)
                if (first + 64 * k + lane < s.need[q]) to[first + 64 * k + lane] = page[k];
        });
        if constexpr (kTokens)
            by_pieces(s, kWrite, [&](int q) { return s.grow[q]; }, [&](int q, int first) {
                const int n = s.n[q], have = s.have[q];
                int32_t page[kPiece / 64];
                int rest[kPiece / 64];
#pragma unroll
                for (int k = 0; k < kPiece / 64; ++k) {
                    const uint32_t pos = uint32_t(max(n, 0) + min(first + 64 * k + lane, s.grow[q] - 1));
                    const int at = int(pos / uint32_t(p.page_tokens));
                    rest[k] = int(pos) - at * p.page_tokens;
                    page[k] = -1;
                    if (n >= 0) page[k] = at < have ? table(r0 + q)[at] : p.free_pages[s.stack[q] - (at - have)];
                }
#pragma unroll
                for (int k = 0; k < kPiece / 64; ++k) {
                    const int i = first + 64 * k + lane;
                    if (i < s.grow[q]) write(s.start[q] + i, r0 + q, n < 0 ? -1 : n + i, page[k], rest[k]);
                }
            });
        needed += all[1];
        tokens = min(tokens + all[2], int64_t(p.max_tokens) + 1);
        if constexpr (!kOne) {
            __syncthreads();
            if (tid == 0) s.count[kTake] = 0;
            __syncthreads();
        }
    }
    const int packed = int(min(tokens, int64_t(p.max_tokens)));
    if (tid == 0) {
        p.row_starts[0] = 0;
        p.counts[0] = int(f - s_taken);
        p.counts[1] = packed;
        p.counts[2] = s_refused;
    }
    if constexpr (kTokens)
        for (int t = packed + tid; t < p.max_tokens; t += kPlanThreads) write(t, -1, -1, -1, 0);
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
// its slot starts a block or does not follow the slot of t - 1.  A wave looks for the leaders of
// kWindow tokens: 1 where tokens are few (most waves of a prompt have no leader then), else 16, where
// prompts have one or two.
//   keys: a lane takes one chunk of one token, 16 bytes of each half, and stores 32 bytes
//   values: a whole block's as rotate.hip's appends take them: 2 dims x the 8 tokens of one half of the
//     slots (slot 8h + e holds token 8(e/4) + 4h + e%4) a lane, two 16-byte stores; of others 2 dims a
//     lane, 8 tokens loaded before the first is stored, 2 bytes a store
// Bound by HBM where tokens are many: 11,991 of 8 heads of 128, keys turned (98 MB), 24.0 us, 4.1 TB/s of
// the 5.4 that a large copy reaches, which takes 18.2 for the bytes; the rest is start and end.  Loads
// past the caches take 24.3 us, stores past them 36.8, lanes in the order of the tokens 25.4.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <int D, bool kTurn, int kWindow>
__global__ __launch_bounds__(256) void append_slots_kernel(const AppendSlotsParams p) {
    constexpr int kChunks = D / 16;
    constexpr int kSteps = D / 64;
    const int lane = threadIdx.x & 63;
    const uint32_t unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const int g = int(unit % uint32_t(p.h_kv));
    const int64_t t0 = int64_t(unit / uint32_t(p.h_kv)) * kWindow;
    if (t0 >= p.n_tokens) return;
    // slots of the tokens t0 - 1 .. t0 + kWindow + 14
    int64_t slot = -1;
    if (lane <= kWindow + 15 && t0 - 1 + lane >= 0 && t0 - 1 + lane < p.n_tokens) slot = p.slots[t0 - 1 + lane];
    if (slot >= p.pool_tokens) slot = -1;
    const int64_t before = __shfl_up(slot, 1);
    const uint64_t valid = __ballot(slot >= 0);
    const uint64_t leads = __ballot(lane > 0 && slot >= 0 && (slot % 16 == 0 || slot != before + 1));
    uint64_t todo = leads & (((uint64_t(1) << kWindow) - 1) << 1);
    const int64_t row = int64_t(p.h_kv) * D;
    while (todo) {
        const int l = __builtin_ctzll(todo);
        todo &= todo - 1;
        // the run: up to the next leader or the next token that is not stored
        const uint64_t stops = (leads | ~valid) >> (l + 1);
        const int n = min(16, __builtin_ctzll(stops) + 1);  // (lanes past the window's end stop it)
        const int64_t t = t0 - 1 + l;
        // its 16-token block of the pool (the pool has fewer than 2^31 of them)
        const uint32_t blk = uint32_t(__builtin_amdgcn_readlane(int(slot >> 4), l));
        const int at = __builtin_amdgcn_readlane(int(slot), l) & 15;
        const uint32_t per = uint32_t(p.page_tokens) / 16, page = blk / per, in = blk - page * per;
        const int64_t ph = int64_t(page) * p.h_kv + g;
        uint16_t* kd = p.k_pages + (ph * kChunks * p.page_tokens + in * 16) * 16;
        uint16_t* vd = p.v_pages + (ph * per + in) * int64_t(D) * 16;
        const uint16_t* ks = p.k_new + (t * p.h_kv + g) * D;
        const uint16_t* vs = p.v_new + (t * p.h_kv + g) * D;

        const auto key = [&](int x, int c, u32x4 lo, u32x4 hi) __attribute__((always_inline)) {
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
            u32x4* dst = reinterpret_cast<u32x4*>(kd + (int64_t(c) * p.page_tokens + at + x) * 16);
            dst[0] = lo;
            dst[1] = hi;
        };
        if (n == 16) {
            u32x4 kx[kSteps], ky[kSteps];
            uint32_t vx[kSteps][8];
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
                const int x = (lane + 64 * j) / kChunks, c = lane % kChunks;
                kx[j] = *reinterpret_cast<const u32x4*>(ks + x * row + 8 * c);
                ky[j] = *reinterpret_cast<const u32x4*>(ks + x * row + 8 * c + D / 2);
            }
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
                const int i = lane + 64 * j, two = i % (D / 2), h = i / (D / 2);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    vx[j][e] = *reinterpret_cast<const uint32_t*>(vs + (8 * (e / 4) + 4 * h + e % 4) * row + 2 * two);
            }
#pragma unroll
            for (int j = 0; j < kSteps; ++j) key((lane + 64 * j) / kChunks, lane % kChunks, kx[j], ky[j]);
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
                const int i = lane + 64 * j, two = i % (D / 2), h = i / (D / 2);
                u32x4 a, b;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    a[e] = (vx[j][2 * e] & 0xFFFFu) | vx[j][2 * e + 1] << 16;
                    b[e] = vx[j][2 * e] >> 16 | (vx[j][2 * e + 1] & 0xFFFF0000u);
                }
                *reinterpret_cast<u32x4*>(vd + (2 * two) * 16 + 8 * h) = a;
                *reinterpret_cast<u32x4*>(vd + (2 * two + 1) * 16 + 8 * h) = b;
            }
        } else {
            for (int i = lane; i < n * kChunks; i += 64) {
                const uint16_t* src = ks + (i / kChunks) * row + 8 * (i % kChunks);
                key(i / kChunks, i % kChunks, *reinterpret_cast<const u32x4*>(src), *reinterpret_cast<const u32x4*>(src + D / 2));
            }
            if (2 * lane < D)
                for (int x0 = 0; x0 < n; x0 += 8) {
                    uint32_t vx[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) vx[e] = *reinterpret_cast<const uint32_t*>(vs + min(x0 + e, n - 1) * row + 2 * lane);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (x0 + e >= n) continue;
                        const int x = at + x0 + e, to = 8 * ((x >> 2) & 1) + 4 * (x >> 3) + (x & 3);
                        vd[(2 * lane) * 16 + to] = uint16_t(vx[e]);
                        vd[(2 * lane + 1) * 16 + to] = uint16_t(vx[e] >> 16);
                    }
                }
        }
    }
}

template <int D, bool kTurn>
hipError_t launch_append_slots_d(const AppendSlotsParams& p, hipStream_t stream) {
    // A step's tokens lie apart, and a wave of 16 takes their runs one behind the other; of a prompt's, most waves of
    // one lead no run.  Which it is only the device knows (us, waves of 1 and of 16; 8 heads of 128: 512 tokens of a
    // step 8.1 and 21.0, 1,024 12.2 and 22.3, 2,048 24.8 and 32.4, of a prompt 9.4 and 6.8, 15.4 and 7.2, 26.7 and
    // 8.7; 16 heads of 64: 512 of a step 8.5 and 19.4, 1,024 12.9 and 21.4, of a prompt 7.6 and 4.9, 9.1 and 5.3)
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
    // sums of the pages and of the tokens (at most max_tokens + 1 a row) in 32 bits
    const bool one = p.batch <= kPlanThreads && int64_t(p.batch) * p.max_pages <= INT32_MAX &&
                     p.batch * (int64_t(p.max_tokens) + 1) <= INT32_MAX;
    // (200 rows with 5,900 tokens 11.6 us in one launch, 11.3 in two)
    if (one && p.max_tokens <= 2048) {
        hipLaunchKernelGGL((plan_kernel<int32_t, true, true>), dim3(1), dim3(kPlanThreads), 0, stream, p);
        return hipGetLastError();
    }
    if (one)
        hipLaunchKernelGGL((plan_kernel<int32_t, true, false>), dim3(1), dim3(kPlanThreads), 0, stream, p);
    else
        hipLaunchKernelGGL((plan_kernel<int64_t, false, false>), dim3(1), dim3(kPlanThreads), 0, stream, p);
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
