// What follows the attention kernels: the parts of a cache joined, the weights of few rows.
#include "fd_kv_dev.h"

namespace fd {
namespace kv {
namespace {

// Joins the parts of the cache: out = sum_s 2^(lse_s - lse) o_s.  Few parts: a warp a row; many: the eight warps of a block share the parts of one
// row (147 parts of 56 rows: a warp a row took 70 us, one wait for memory after the other).  The parts' factors are made in parallel first.
// The first `weigh` blocks turn the scores that k_few left into weights: w_j += sum over the rows that see token j of 2^(score - lse), four tokens a thread.
constexpr int kWeighTokens = 1024;

__device__ __forceinline__ void weigh_block(const AttendArgs& a, int block) {
    __shared__ float s_lse[kFewRows];
    __shared__ int s_lo[kFewRows], s_hi[kFewRows];
    const int per = (a.batch.max_len + kWeighTokens - 1) / kWeighTokens;
    const int h = (block / per) % a.heads, b = block / (per * a.heads), key0 = (block % per) * kWeighTokens + threadIdx.x;
    Work w;
    w.b = b; w.begin = q_begin(a.batch, b); w.count = max(0, q_begin(a.batch, b + 1) - w.begin); w.t0 = 0;
    w.n = kv_length(a.batch, b, false);
    if (key0 - (int)threadIdx.x >= w.n) return;
    const int rows = w.count <= kFewRows / a.group ? w.count * a.group : 0;
    if ((int)threadIdx.x < rows) {
        const int r = threadIdx.x, token = r / a.group;
        const int64_t at = (int64_t)(w.begin + token) * a.q_heads + h * a.group + r % a.group, all = (int64_t)a.batch.total_q * a.q_heads;
        float lse;
        if (a.splits > 1) {
            float top = -INFINITY, sum = 0.f;
#pragma unroll 8
            for (int s = 0; s < a.splits; ++s) top = max_nan(top, a.part_lse[s * all + at]);
#pragma unroll 8
            for (int s = 0; s < a.splits; ++s) sum += ex2f(a.part_lse[s * all + at] - top);
            lse = top == -INFINITY ? -INFINITY : top + log2f(sum);
        } else {
            const float x = a.lse[at];
            lse = x == -INFINITY ? x : (float)((double)x * 1.44269504088896340736);
        }
        s_lse[r] = lse;
        s_lo[r] = see_lo(a, w, token);
        s_hi[r] = see_hi(a, w, token);
    }
    __syncthreads();
    float sum[kWeighTokens / 256];
    const float* s = a.scores + ((int64_t)b * a.heads + h) * kFewRows * a.score_stride + key0;
#pragma unroll
    for (int k = 0; k < kWeighTokens / 256; ++k) sum[k] = 0.f;
    for (int r = 0; r < rows; ++r) {
        const float lse = s_lse[r];
        const int lo = s_lo[r], hi = s_hi[r];
#pragma unroll
        for (int k = 0; k < kWeighTokens / 256; ++k) {
            const int key = key0 + 256 * k;
            if (key >= lo && key < hi) sum[k] += ex2f(s[r * a.score_stride + 256 * k] - lse);
        }
    }
#pragma unroll
    for (int k = 0; k < kWeighTokens / 256; ++k) {
        const int key = key0 + 256 * k;
        if (key >= w.n) continue;
        const int64_t at = ((int64_t)b * a.heads + h) * a.w_stride + key;
        a.w_out[at] = (a.w_in ? a.w_in[at] : 0.f) + sum[k];
    }
}

template <class T, int D, int W>
__global__ void __launch_bounds__(256) k_join(const AttendArgs a, const int weigh) {
    constexpr int E = D / 32;
    __shared__ float s_f[W == 1 ? 8 * 32 : kMaxSplits];
    __shared__ float s_o[W == 1 ? 1 : 8 * D], s_top[8], s_sum[8];
    grid_wait();
    if ((int)blockIdx.x < weigh) { weigh_block(a, blockIdx.x); return; }
    const int block = blockIdx.x - weigh;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, me = W == 1 ? lane : (int)threadIdx.x;
    const int64_t row = W == 1 ? (int64_t)block * 8 + warp : block;
    const int64_t rows = (int64_t)q_begin(a.batch, a.batch.batch) * a.q_heads, all = (int64_t)a.batch.total_q * a.q_heads;
    if (row >= rows) return;
    float* f = W == 1 ? s_f + 32 * warp : s_f;
    float top = -INFINITY;
    for (int s = me; s < a.splits; s += 32 * W) top = max_nan(top, f[s] = a.part_lse[s * all + row]);
    for (int o = 16; o; o >>= 1) top = max_nan(top, __shfl_xor_sync(~0u, top, o));
    if (W > 1) {
        if (lane == 0) s_top[warp] = top;
        __syncthreads();
        for (int k = 0; k < 8; ++k) top = max_nan(top, s_top[k]);
    }
    float sum = 0.f;
    if (top != -INFINITY)
        for (int s = me; s < a.splits; s += 32 * W) sum += f[s] = ex2f(f[s] - top);           // (a part without rows in sight: 0)
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    if (W > 1) {
        if (lane == 0) s_sum[warp] = sum;
        __syncthreads();
        sum = 0.f;
        for (int k = 0; k < 8; ++k) sum += s_sum[k];
    } else __syncwarp();
    float o[E];
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] = 0.f;
    if (top != -INFINITY) {
        const float* p = a.part_o + row * D + lane * E;
#pragma unroll 4
        for (int s = W == 1 ? 0 : warp; s < a.splits; s += W) {
            const float w = f[s];
            if (w == 0.f) continue;                                // (its o may not have been written)
            const float* q = p + s * all * D;
            if (E == 4) {
                const float4 v = *(const float4*)q;
                o[0] = fmaf(w, v.x, o[0]); o[1] = fmaf(w, v.y, o[1]); o[E - 2] = fmaf(w, v.z, o[E - 2]); o[E - 1] = fmaf(w, v.w, o[E - 1]);
            } else {
                const float2 v = *(const float2*)q;
                o[0] = fmaf(w, v.x, o[0]); o[1] = fmaf(w, v.y, o[1]);
            }
        }
    }
    if (W > 1) {
#pragma unroll
        for (int i = 0; i < E; ++i) s_o[warp * D + lane * E + i] = o[i];
        __syncthreads();
        if (warp) return;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            o[i] = 0.f;
            for (int k = 0; k < 8; ++k) o[i] += s_o[k * D + lane * E + i];
        }
    }
    const float inv = top == -INFINITY ? 0.f : 1.0f / sum;
    const int64_t token = row / a.q_heads;
    const int head = (int)(row - token * a.q_heads);
    uint32_t* dst = (uint32_t*)((T*)a.out.p + token * a.out.token_stride + head * a.out.head_stride + lane * E);
#pragma unroll
    for (int i = 0; i < E / 2; ++i) dst[i] = Elem<T>::pack(o[2 * i] * inv, o[2 * i + 1] * inv);
    if (a.lse && lane == 0) a.lse[row] = top == -INFINITY ? -INFINITY : (float)((double)(top + log2f(sum)) * 0.69314718055994530942);
}

template <class T, int D>
cudaError_t join_t(const AttendArgs& a, cudaStream_t stream) {
    const int64_t rows = a.splits > 1 ? (int64_t)a.batch.total_q * a.q_heads : 0;
    const int64_t weigh = a.scores && a.w_out ? (int64_t)ceil_div(a.batch.max_len, kWeighTokens) * a.heads * a.batch.batch : 0;
    if (rows + weigh == 0) return cudaSuccess;
    ++g_launches;
    if (a.splits > 16) return launch_behind(stream, dim3((unsigned)(rows + weigh)), dim3(256), 0, k_join<T, D, 8>, a, (int)weigh);
    return launch_behind(stream, dim3((unsigned)(ceil_div(rows, 8) + weigh)), dim3(256), 0, k_join<T, D, 1>, a, (int)weigh);
}

}  // namespace

cudaError_t launch_join(const AttendArgs& a, cudaStream_t stream) { return FD_KV_PICK(join_t, a, stream); }

}  // namespace kv
}  // namespace fd
