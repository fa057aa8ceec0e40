// Internal declarations of the paged cache's operators (fd_kv.cu: entry points; fd_kv_rows.cu: rotary positions, append, eviction;
// fd_kv_attend.cu: attention and its column sums; fd_kv_decode.cu: attention of few rows).
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "fd_internal.h"

struct fd_kv {
    fd_kv_desc d{};
    int box_rows = 0, few_rows = 0;  // rows of a page that one TMA box takes: gcd(page_size, 128); with few rows gcd(page_size, 16 or 32)
    int device = 0, sm_count = 148;
    CUtensorMap map_k, map_v;        // (coordinate, row of the page, head, page)
    CUtensorMap few_k, few_v;
};

#include <atomic>

namespace fd {
namespace kv {

// Lets a kernel have `bytes` of dynamic shared memory on the current device; asks the runtime once per kernel and device (0.5 us a call).
template <auto KERNEL>
cudaError_t allow_smem(size_t bytes) {
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// Bits of a cache's first status word; the second holds the code of a wait that ran out.
constexpr unsigned kBadPage = 1, kBadLength = 2;

// A batch as the kernels see it.
struct Batch {
    const int* table; int64_t table_stride;
    const int* kv_len; const int* q_start;
    int batch, max_pages, total_q, max_len, page_size, num_pages;
    int page_shift;                  // log2(page_size), or -1: moving rows spends most of its instructions on divisions otherwise
    unsigned int* status;
    // Page of a slot and the slot's row in it.
    __device__ __forceinline__ int page_of(int slot) const { return page_shift >= 0 ? slot >> page_shift : slot / page_size; }
    __device__ __forceinline__ int row_of(int slot) const { return page_shift >= 0 ? slot & (page_size - 1) : slot % page_size; }
};

// Sequence b's tokens in the cache, never more than its row of the page table holds.
__device__ __forceinline__ int kv_length(const Batch& B, int b, bool report) {
    const int n = B.kv_len[b];
    const int64_t room = (int64_t)B.max_pages * B.page_size;
    const int cap = room < B.max_len ? (int)room : B.max_len;
    if (n >= 0 && n <= cap) return n;
    if (report) atomicOr(B.status, kBadLength);
    return n < 0 ? 0 : cap;
}
__device__ __forceinline__ int q_begin(const Batch& B, int b) { return min(max(B.q_start[b], 0), B.total_q); }

struct Heads {
    void* p; int64_t token_stride, head_stride; int heads;
};
inline Heads heads_of(const fd_heads& h) { return Heads{h.p_dev, h.token_stride, h.head_stride, h.heads}; }

struct RowsArgs {                    // rotary positions, and an append when `append`
    Heads x, y;                      // turned: x -> y (y may be x); heads 0: none
    Heads k, v;                      // new rows of the cache (append)
    void* k_pool; void* v_pool;
    int64_t k_page, k_token, k_head, v_page, v_token, v_head;
    const int* positions; const double* freqs;
    Batch batch;
    int tokens, head_dim, rot, layout, append;
    float scale;                     // negative angles: sine times -1
    float sign;
};
cudaError_t launch_rows(const RowsArgs& a, int dtype, int sm_count, cudaStream_t stream);

struct EvictArgs {
    Batch batch;
    const float* w_in; float* w_out; int64_t w_stride;
    const int* new_table; int64_t new_table_stride; int new_max_pages;
    int keep, first, recent, heads, head_dim;
    int* kept; int* new_len;
    void* k_pool; void* v_pool;
    int64_t k_page, k_token, k_head, v_page, v_token, v_head;
};
cudaError_t launch_evict(const EvictArgs& a, cudaStream_t stream);

struct AttendArgs {
    Batch batch;
    Heads q, out;
    int q_heads, heads, group, head_dim, dtype;
    int tile_tokens;                 // tokens of a 128-row tile: 128 / group; its rows are (token, query head of the group)
    int causal, window;              // window 0: none
    float scale_log2;                // scale * log2(e)
    float* lse;
    const float* w_in; float* w_out; int64_t w_stride;
    int row_tiles;                   // many rows: tiles of 128 rows a CTA
    int splits, split_tiles;         // many rows: the cache in `splits` parts of split_tiles tiles of 128 tokens
    int sm_count;
    int ctas, few_rows;              // few rows: CTAs that share the batch's caches; rows a sequence has at most; first CTA and number of the parts of each
    int2* parts;                     // (sequence, head)
    float* part_o; float* part_lse;  // [split][token][query head]([head_dim]); few rows: [slot][kFewRows]([head_dim])
    float* scores; int64_t score_stride;     // few rows and weights: scale_log2 q.k of every row and slot, [sequence][head][few_rows][score_stride]
    float* folds;                    // few rows, caches that fill an accumulator more than once: sums of every warp
    int box_rows;
    const void* v_pool; int64_t v_page, v_token, v_head;
};
// At most this many rows (new tokens x query heads of a group) of a sequence go through the kernel for few rows.
constexpr int kFewRows = 16;
constexpr int kFewWarps = 4;             // warps of a CTA of that kernel; each goes through a quarter of what the CTA has of a cache
constexpr int kMaxSplits = 1024;         // parts of a cache
// Longest stretch of tokens that one accumulator of matrix products sums.  The tensor core truncates: of values of one sign, 1e-7 of the sum is lost with every 16
// tokens (262144 tokens: 1.7e-3, nearly four half steps of fp16; mma.sync the same); parts are joined with rounding, so the loss ends at 2.1e-4.
constexpr int kPartTokens = 32768;

// How the work of a call is cut, and what its workspace holds.
struct Plan {
    bool few;
    int row_tiles, splits, split_tiles, ctas;
    int64_t score_stride;
    size_t parts, part_o, part_lse, scores, folds;  // in floats, in this order, each a multiple of 4
    size_t bytes() const { return (parts + part_o + part_lse + scores + folds) * sizeof(float); }
};
Plan plan_attend(const fd_kv* kv, const fd_kv_batch* b, int q_heads, bool weights);
cudaError_t launch_attend(const AttendArgs& a, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t stream);
cudaError_t launch_weigh(const AttendArgs& a, const CUtensorMap& mq, const CUtensorMap& mk, cudaStream_t stream);
cudaError_t launch_few(const AttendArgs& a, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t stream);

}  // namespace kv
}  // namespace fd
