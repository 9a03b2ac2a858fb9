// Internal declarations shared by the host side of libatf.so and its kernels.
// Not part of the public ABI (include/atf.h is).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace atf {

constexpr int kMaxPairs = 64;     // d/2 for d = 128
constexpr int kChunkPairs = 8;    // pairs per QK K-step and per decode K-cache chunk
constexpr int kMaxChunks = kMaxPairs / kChunkPairs;

// Window table in the form every kernel consumes: per pair the integer threshold
// W_r (keep the pair's term at distance z iff z <= W_r), and per chunk of
// kChunkPairs consecutive pairs the smallest and largest threshold.
struct WindowTable {
    int32_t W[kMaxPairs];
    int32_t chunk_min[kMaxChunks];
    int32_t chunk_max[kMaxChunks];
};

struct PrefillParams {
    const uint16_t* q;   // [B][n_q][h_q][d]
    const uint16_t* k;   // [B][h_kv][d/16][cache_tokens][16] (pair-chunk-major)
    const uint16_t* v;   // [B][h_kv][ceil(cache_tokens/16)][d][16] (see atf_pack_vcache)
    uint16_t* o;         // [B][n_q][h_q][d]
    float* lse;          // [B][h_q][n_q]
    int32_t batch, n_q, n_k, q_pos0, h_q, h_kv, group;
    int32_t cache_tokens;  // tokens each cache entry is allocated for (>= n_k)
    int32_t pos_per_tile;  // query positions per workgroup (rows = positions x group)
    int32_t n_qtiles;
    int32_t mono;        // thresholds non-decreasing in r
    float scale_log2;    // softmax scale * log2(e)
    WindowTable win;
};

// Prefill with RoPE at read time: q and the K cache hold unrotated vectors, rotated
// in the kernel as DecodeParams describes. A type of its own, so that the kernels
// of pre-rotated caches keep their argument block.
struct PrefillRotParams : PrefillParams {
    uint32_t rope_rho_hi[kMaxPairs];
    uint32_t rope_rho_lo[kMaxPairs];
};

struct DecodeParams {
    const uint16_t* q;       // [B][h_q][d]
    const uint16_t* kpcm;    // [B][h_kv][d/16][cache_tokens][16]
    const uint16_t* vpk;     // [B][h_kv][ceil(cache_tokens/16)][d][16] (see atf_pack_vcache)
    uint16_t* o;             // [B][h_q][d]
    float* lse;              // [B][h_q]
    float* ws_m;             // [B][h_q][splits]   running max (log2 domain)
    float* ws_l;             // [B][h_q][splits]   normaliser
    float* ws_o;             // [B][h_q][splits][d] unnormalised output
    int32_t batch, n_k, q_pos, h_q, h_kv, group;
    int32_t cache_tokens;     // tokens each cache entry is allocated for (>= n_k)
    int32_t heads_per_block;  // query heads handled by one workgroup (divides group, <= 32)
    int32_t n_valid;          // keys 0 .. n_valid - 1 are causal
    const int32_t* n_k_rows;  // ragged batch: device [B] keys of each row (clamped to
                              // [0, n_k]), or nullptr: every row has n_k keys
    const int32_t* q_pos_rows;  // ragged batch: device [B] query position of each row
                                // (clamped to [0, 2^31 - 2]), or nullptr: q_pos
    const int32_t* block_table;  // paged caches: device [B][max_pages] page of each row's
                                 // page_tokens-token span (clamped to [0, num_pages)),
                                 // or nullptr: contiguous caches
    int32_t max_pages, num_pages, page_tokens;
    int32_t* ws_plan;         // ragged batch: [B + 1] index of each row's first work item
                              // (written by the split kernel for the merge), else unused
    int32_t splits;           // uniform batch: splits per row; ragged batch: work items the
                              // batch's keys are spread over (a row adds at most one more)
    int32_t split_tokens;     // uniform batch: tokens per split (multiple of the workgroup's
                              // token step); ragged batch: unused (derived on the device)
    float scale_log2;
    WindowTable win;
    // RoPE at read time: q and the K cache hold unrotated vectors; pair r of a vector
    // at position pos is rotated by pos * theta_r, with rho_r = theta_r / (2 pi) mod 1
    // as a 0.64 fixed-point fraction (hi and lo words)
    int32_t rotate;
    int32_t cols16;           // decode_split16_kernel, not decode_split_kernel
    int32_t direct;           // one split per row, which writes the output itself (no merge)
    uint32_t rope_rho_hi[kMaxPairs];
    uint32_t rope_rho_lo[kMaxPairs];
};

// Append of n_new tokens at cache positions pos0 .. (rotate.hip): a NULL k_src or v_src
// leaves that cache alone (the packs).
struct AppendParams {
    const uint16_t* k_src;       // [B][n_new][h_kv][d]
    const uint16_t* v_src;
    uint16_t* k_dst;             // [B][h_kv][d/16][cache_tokens][16], or pages
                                 // [num_pages][h_kv][d/16][page_tokens][16]
    uint16_t* v_dst;             // [B][h_kv][ceil(cache_tokens/16)][d][16], or pages
                                 // [num_pages][h_kv][page_tokens/16][d][16]
    const int32_t* block_table;  // [B][max_pages], or nullptr: contiguous caches
    int32_t batch, n_new, h_kv, pos0;
    int32_t cache_tokens;        // capacity of the contiguous caches
    int32_t zero_tail;           // V: write zeros to the slots of the last block past the source
    int32_t max_pages, num_pages, page_tokens;
};

// With the keys turned on the way in.  A type of its own: 512 bytes more of arguments take 0.3
// us of a launch.
struct AppendRotParams : AppendParams {
    uint32_t rope_rho_hi[kMaxPairs];
    uint32_t rope_rho_lo[kMaxPairs];
};

// Decode over 8-bit caches (decode_q8.hip).  A type of its own, without what its kernel does not
// read (the arguments' way to the chip is part of a short call): fields as DecodeParams.
struct DecodeQ8States {
    uint16_t* o;
    float* lse;
    float* ws_m;
    float* ws_l;
    float* ws_o;
    int32_t* ws_plan;         // ragged batch split over work items, else nullptr: a row has `splits`
    int32_t batch, h_q, splits;
};
struct DecodeQ8Params : DecodeQ8States {
    const uint16_t* q;
    const uint8_t* k;         // e4m3 [B][h_kv][d/16][cache_tokens][16], or pages
    const uint8_t* v;         // e4m3 [B][h_kv][ceil(cache_tokens/16)][d][16], tokens in order
    const uint8_t* k_scale;   // [B][h_kv][scale_tokens], or pages [num_pages][h_kv][page_tokens]
    const uint8_t* v_scale;
    const int32_t* n_k_rows;
    const int32_t* q_pos_rows;
    const int32_t* block_table;
    int32_t n_k, q_pos, n_valid, h_kv, group;
    int32_t cache_tokens;
    uint32_t scale_tokens;    // cache_tokens rounded up to 16 (2^31 at most), or page_tokens
    int32_t max_pages, num_pages, page_tokens;
    int32_t heads_per_block;  // at most 32; need not divide the group: the last of the
    int32_t subgroups;        // `subgroups` workgroups of a KV head takes what is left
    int32_t split_tokens;
    int32_t direct;
    int32_t waves;            // of a workgroup: 4 or 8
    float scale_log2;
    int32_t W[kMaxPairs];
};

// Append with the heads' norms and the rotation (append_normed.hip), of bf16 caches or, with
// k_scale set, 8-bit ones.
struct AppendNormedParams {
    const uint16_t* q;           // [B][n_new][h_q][d], or nullptr (h_q is 0 then)
    const uint16_t* k_src;       // [B][n_new][h_kv][d]
    const uint16_t* v_src;
    uint16_t* q_out;             // like q
    void* k_dst;                 // caches or page pools
    void* v_dst;
    uint8_t* k_scale;            // 8-bit caches: [B][h_kv][scale_tokens] or pages, else nullptr
    uint8_t* v_scale;
    const float* q_weight;       // [d], or nullptr: not normed
    const float* k_weight;
    float eps;
    const int32_t* pos_rows;     // device [B] first position of each row (negative: idle), or
                                 // nullptr: pos0
    const int32_t* block_table;  // [B][max_pages], or nullptr: contiguous caches
    int32_t batch, n_new, h_q, h_kv, pos0;
    int32_t cache_tokens;        // capacity of the contiguous caches
    uint32_t scale_tokens;       // cache_tokens rounded up to 16 (2^31 at most), or page_tokens
    int32_t max_pages, num_pages, page_tokens;
    // set by the launcher: heads of a wave, and waves of a token's heads; waves of whole value
    // blocks, which come first; waves of values by themselves, and whether those are only the
    // tokens at the rows' ends; waves of keys
    int32_t q_heads_per_wave, kv_heads_per_wave;
    uint32_t q_parts, kv_parts;
    int32_t value_ends;
    uint32_t block_waves, value_waves, key_waves;
    uint32_t rope_rho_hi[kMaxPairs];
    uint32_t rope_rho_lo[kMaxPairs];
};

// 8-bit caches (or pages) read back into contiguous bf16 caches (cache_q8.hip): positions
// pos0 .. pos0 + n_k - 1 of every row.
struct ReadQ8Params {
    const uint8_t* k_src;
    const uint8_t* k_scale;
    const uint8_t* v_src;
    const uint8_t* v_scale;
    uint16_t* k_dst;             // [B][h_kv][d/16][dst_tokens][16]
    uint16_t* v_dst;             // [B][h_kv][ceil(dst_tokens/16)][d][16]
    const int32_t* block_table;  // [B][max_pages], or nullptr: contiguous source
    int32_t batch, n_k, pos0, h_kv;
    int32_t src_tokens, dst_tokens;
    uint32_t scale_tokens;
    int32_t max_pages, num_pages, page_tokens;
    uint32_t key_blocks;         // set by the launcher
};

// One pass of RoPE over a pair-chunk-major K cache (rotate.hip): key t of every (batch,
// kv head) turned to position t, tokens 0 .. n_k - 1.
struct RotateParams {
    const uint16_t* src;   // [B][h_kv][d/16][cache_tokens][16]
    uint16_t* dst;         // same layout; only the tokens named are written
    int32_t batch, n_k, h_kv, cache_tokens;
    uint32_t rope_rho_hi[kMaxPairs];
    uint32_t rope_rho_lo[kMaxPairs];
};

// Pages handed out and slots found from the rows' lengths (pages.hip).
struct PlanParams {
    int32_t* block_table;        // [B][max_pages]
    int32_t* free_pages;         // [free_capacity], the first *free_count of them free
    const int32_t* free_count;
    const int32_t* n_k_rows;     // [B] tokens each row holds
    const int32_t* n_new_rows;   // [B] tokens it gets; negative: the row ends
    int32_t* n_k_out;            // [B], may be n_k_rows
    int32_t* row_starts;         // [B + 1]
    int64_t* slots;              // [max_tokens], as the two below
    int32_t* token_rows;
    int32_t* positions;
    int32_t* counts;             // [3], may begin at free_count
    int32_t batch, max_pages, page_tokens, free_capacity, max_tokens;
};

// Tokens appended through their slots (pages.hip).
struct AppendSlotsParams {
    const uint16_t* k_new;       // [n_tokens][h_kv][d]
    const uint16_t* v_new;
    uint16_t* k_pages;           // [num_pages][h_kv][d/16][page_tokens][16]
    uint16_t* v_pages;           // [num_pages][h_kv][page_tokens/16][d][16]
    const int64_t* slots;        // [n_tokens]; outside [0, pool_tokens): not stored
    const int32_t* positions;    // [n_tokens], keys turned; else nullptr
    int64_t pool_tokens;         // num_pages * page_tokens
    int32_t n_tokens, h_kv, page_tokens;
    uint32_t rope_rho_hi[kMaxPairs];
    uint32_t rope_rho_lo[kMaxPairs];
};

// Bounds of the keys of the blocks that hold the rows' newest tokens (blocks.hip).
struct BoundsParams {
    const uint16_t* k_pages;
    uint16_t* bounds;            // [num_pages][h_kv][page_tokens/block_tokens][d/16][2][16]
    const int32_t* block_table;
    const int32_t* n_k_rows;
    const int32_t* n_new_rows;
    int32_t batch, max_pages, num_pages, page_tokens, block_tokens, h_kv;
    int32_t max_new;
    uint32_t row_blocks;         // most blocks of a row that max_new tokens lie in
};

// The blocks that query tokens take (blocks.hip).
struct SelectParams {
    const uint16_t* q;           // [n_tokens][h_q][d]
    const uint16_t* bounds;      // as BoundsParams
    int32_t* blocks;             // [n_tokens][h_kv][top]
    const int32_t* block_table;
    const int32_t* token_rows;   // [n_tokens]; outside [0, batch): nothing is written
    const int32_t* positions;    // [n_tokens]
    const int32_t* n_k_rows;     // [batch], clamped to [0, max_n_k]
    // workspace: scores as integers of their order [slab][h_kv][key_stride], the same in 64 bits
    // where fp32 does not do, and the largest sum of magnitudes that each wave met
    int32_t* keys;
    uint64_t* exact_keys;
    float* sizes;                // [slab][h_kv][ranges]
    int32_t batch, max_pages, num_pages, page_blocks, block_tokens;
    int32_t n_tokens, max_n_k, row_blocks, top, first_blocks, last_blocks;
    int32_t h_q, h_kv, group, chunks;
    int32_t key_stride;          // row_blocks rounded up to 16
    int32_t pack;                // tokens whose heads share the columns of a product
    int32_t ranges;              // waves of a (token, KV head): each takes every ranges-th tile
    int32_t slab, first_token, tokens;  // tokens of a launch at most; set by the launcher: the
                                 // first of this one, and their number
    int32_t W[kMaxPairs];
};

// Attention over listed blocks (attend_blocks.hip).
struct AttendParams {
    const uint16_t* q;           // [n_tokens][h_q][d]
    const uint16_t* k_pages;
    const uint16_t* v_pages;
    uint16_t* o;                 // like q
    float* lse;                  // [n_tokens][h_q]
    const int32_t* block_table;
    const int32_t* token_rows;
    const int32_t* positions;
    const int32_t* n_k_rows;     // clamped to [0, max_n_k]
    const int32_t* blocks;       // [n_tokens][h_kv][top]
    int32_t batch, max_pages, num_pages, page_tokens, block_tokens;
    int32_t n_tokens, max_n_k, top, h_q, h_kv, group;
    int32_t heads_per_block, subgroups;  // as DecodeQ8Params
    int32_t waves;               // of a workgroup: 1, 2, 4 or 8
    int32_t splits, split_tiles; // workgroups of a list, 32-token tiles of each
    float* ws_m;                 // [n_tokens][h_q][splits], split lists, as the two below
    float* ws_l;
    float* ws_o;                 // [n_tokens][h_q][splits][d]
    float scale_log2;
    int32_t W[kMaxPairs];
};

// Most (token, query head)s of a selection or of the attention over it, and blocks of a list.
constexpr int64_t kMaxTokenHeads = int64_t(1) << 23;
constexpr int32_t kMaxTopBlocks = 4096;
// Workspace that a selection takes for the scores of the tokens of one launch, at most (more where
// a single token needs it).
constexpr int64_t kSelectSlabBytes = int64_t(256) << 20;

// Kernel launchers (one in each .hip file, two in prefill.hip and rotate.hip).  Return the HIP error
// of the launch.
hipError_t launch_prefill(const PrefillParams& p, int head_dim, hipStream_t stream);
hipError_t launch_prefill_rotating(const PrefillRotParams& p, int head_dim, hipStream_t stream);
// The kernel a prefill takes: 4 or 8 waves per row block of prefill_short_kernel, 0 for
// prefill_kernel, -1 if it is refused (the tests ask).
int32_t prefill_waves(int32_t batch, int32_t n_q, int32_t n_k, int32_t q_pos0, int32_t h_kv, int32_t group,
                      int32_t cache_tokens, const int32_t* thresholds, int32_t head_dim, bool rotate);
hipError_t launch_decode(const DecodeParams& p, int head_dim, hipStream_t stream);
hipError_t launch_decode_q8(const DecodeQ8Params& p, int head_dim, hipStream_t stream);
hipError_t launch_append_normed(const AppendNormedParams& p, int head_dim, hipStream_t stream);
hipError_t launch_read_q8(const ReadQ8Params& p, int head_dim, hipStream_t stream);
hipError_t launch_append(const AppendRotParams& p, bool turn, int head_dim, hipStream_t stream);
hipError_t launch_plan_pages(const PlanParams& p, hipStream_t stream);
hipError_t launch_append_slots(const AppendSlotsParams& p, bool turn, int head_dim, hipStream_t stream);
hipError_t launch_block_bounds(const BoundsParams& p, int head_dim, hipStream_t stream);
hipError_t launch_select_blocks(const SelectParams& p, hipStream_t stream);
// Waves of a workgroup and workgroups of a list for `groups` (token, KV head, head subgroup)s of lists of
// `tiles` 32-token tiles; the second: where a workspace holds the states of `room` splits.
struct AttendPlan {
    int32_t waves, splits, split_tiles;
};
AttendPlan attend_plan(int64_t groups, int64_t tiles);
AttendPlan attend_plan(int64_t groups, int64_t tiles, int64_t room);
hipError_t launch_attend_blocks(const AttendParams& p, int head_dim, hipStream_t stream);
hipError_t launch_rotate_kcache(const RotateParams& p, int head_dim, hipStream_t stream);

// Most splits per (batch, kv head) of a uniform batch, and most work items per column of
// `cols` = kv heads x head subgroups of a ragged one: what the workspace has room for.
int32_t decode_splits(int32_t batch, int32_t h_kv, int64_t n_k);
int32_t decode_ragged_items(int32_t cols);
// The kernel and the numbers a call uses; n_valid bounds a ragged batch's rows.
bool decode_cols16(int32_t batch, int32_t h_q, int32_t h_kv, int32_t head_dim, int64_t n_valid,
                   int64_t cache_tokens, int32_t heads_per_block, bool ragged);
int32_t decode_plan_splits(int32_t batch, int32_t h_q, int32_t h_kv, int64_t n_k, int64_t n_valid,
                           int32_t heads_per_block, bool cols16, bool rotate);
int32_t decode_plan_items(int32_t cols, bool cols16);
// Whether a batch runs without splits (with cols16 only).
bool decode_direct(int32_t batch, int32_t h_q, int32_t h_kv, int32_t head_dim, int64_t n_valid,
                   int32_t heads_per_block, bool rotate, bool ragged);
// The token of a wave's next block, `step` past t0 in [0, t_end), or t_end if that is none (the end may be
// 2^31 - 1: no sum is formed past it).
__host__ __device__ int32_t decode_next(int32_t t0, int32_t t_end, int32_t step);
// The same questions of the decode over 8-bit caches.
int32_t decode_q8_waves(int32_t tiles, int64_t groups, int64_t n_valid, bool ragged, bool direct);
int32_t decode_q8_slots(int32_t head_dim, int32_t tiles, int32_t waves);
bool decode_q8_direct(int64_t groups, int32_t head_dim, int32_t tiles, int64_t n_valid, bool ragged);
int64_t decode_q8_splits(int64_t groups, int64_t slots, int64_t room);
// The first token of a wave's 64-token blocks in a workgroup's tokens [t_begin, t_end), t_end if it has
// none (the end may be 2^31 - 1: no sum is formed past it).
__host__ __device__ int32_t decode_q8_first(int32_t t_begin, int32_t t_end, int32_t wave);
// Caches from this many tokens are out of the 32-bit lane offsets of decode_split16_kernel
// (they reach over one chunk's stream) and take decode_split_kernel.
constexpr int64_t kDecode16MaxTokens = (int64_t(1) << 27) - 64;
// Tokens handled per decode workgroup iteration (the split granularity).
constexpr int32_t kDecodeTokenStep = 128;
// The same of the 8-bit caches' decode: 64 tokens a wave, of four waves or of half of eight.
constexpr int32_t kDecodeQ8TokenStep = 256;
// Largest split count the merge kernel accepts.
constexpr int32_t kDecodeMaxSplits = 4096;
// Query heads one decode workgroup handles at most (columns of its MFMA tiles).
constexpr int32_t kDecodeMaxHeads = 32;
// Size of the library's own decode scratch array (decode.hip), the workspace of
// atf_decode_noalloc; equal to ATF_DECODE_NOALLOC_SCRATCH_BYTES of atf.h.
constexpr size_t kNoAllocScratchBytes = size_t(16) << 20;
// Device address of that array on the current device, resolved once per device
// (hipGetSymbolAddress) and kept for the life of the process.
hipError_t noalloc_scratch(void** out);

}  // namespace atf
