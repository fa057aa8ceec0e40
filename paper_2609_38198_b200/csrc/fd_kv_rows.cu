// Rotary positions, appends to a paged cache and evictions from it: kernels that move rows and do little else.
#include "fd_kv.h"

namespace fd {
namespace kv {
namespace {

// ------------------------------------------------------------------------------------------------ rotary positions, append
// A block takes a few tokens.  First cosine and sine of every (token, frequency) go to shared memory, once for all heads: the angle is position * frequency in
// turns, reduced to half a turn in fp64 (a position of 2^31 is off by 1e-7 turns at most), and only the remainder is fp32.  Then
// the threads run over (token, head, unit): a unit is two vectors of 16 bytes, the two halves of VEC pairs (HALF) or VEC neighbouring pairs,
// both read before either is written, so y may be x.  Bytes bound it: each row is read once and written once.
constexpr int kRowThreads = 256;
constexpr double kTurn = 0.15915494309189533577;      // 1 / (2 pi)

template <class T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f(float v) { return v; }
template <> __device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f(float v) { return v; }
template <> __device__ __forceinline__ __half from_f(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }

template <class T, int VEC> struct alignas(VEC * sizeof(T)) Vec { T v[VEC]; };

template <class T, int VEC, bool HALF>
__global__ void __launch_bounds__(kRowThreads) k_rows(const RowsArgs a, const int block_tokens) {
    extern __shared__ float2 turn[];                         // [block_tokens][rot / 2]
    __shared__ int64_t place[16][2];                         // pool offset of a token's key and value row of head 0, -1: nowhere
    using V = Vec<T, VEC>;
    const int t0 = blockIdx.x * block_tokens, nt = min(block_tokens, a.tokens - t0);
    const int half = a.rot / 2;
    for (int i = threadIdx.x; i < nt * half; i += kRowThreads) {
        const int t = i / half, f = i - t * half;
        const double turns = (double)a.positions[t0 + t] * a.freqs[f] * kTurn;
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        turn[i] = make_float2(c * a.scale, s * a.scale * a.sign);
    }
    if (a.append && threadIdx.x < nt) {
        const Batch& B = a.batch;
        const int t = t0 + threadIdx.x;
        int lo = 0, hi = B.batch;                            // last sequence that begins at or before t
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (q_begin(B, mid) <= t) lo = mid; else hi = mid;
        }
        const int begin = q_begin(B, lo), end = q_begin(B, lo + 1);
        place[threadIdx.x][0] = -1;
        if (t >= begin && t < end) {
            const int n = kv_length(B, lo, true), slot = n - (end - begin) + (t - begin);
            const int page = slot < 0 ? -1 : B.table[lo * B.table_stride + slot / B.page_size];
            if (slot < 0) atomicOr(B.status, kBadLength);
            else if (page < 0 || page >= B.num_pages) atomicOr(B.status, kBadPage);
            else {
                place[threadIdx.x][0] = page * a.k_page + (slot % B.page_size) * a.k_token;
                place[threadIdx.x][1] = page * a.v_page + (slot % B.page_size) * a.v_token;
            }
        }
    }
    __syncthreads();
    const int unit_count = a.head_dim / (2 * VEC), turned = a.rot / (2 * VEC);
    const int heads = a.x.heads + (a.append ? a.k.heads + a.v.heads : 0);
    const int items = nt * heads * unit_count;
    for (int i = threadIdx.x + blockIdx.y * kRowThreads; i < items; i += kRowThreads * gridDim.y) {
        const int hu = i / unit_count, u = i - hu * unit_count;
        const int t = hu / heads;
        int h = hu - t * heads;
        const T* src;
        T* dst;
        bool rot = u < turned;
        if (h < a.x.heads) {
            src = (const T*)a.x.p + (t0 + t) * a.x.token_stride + h * a.x.head_stride;
            dst = (T*)a.y.p + (t0 + t) * a.y.token_stride + h * a.y.head_stride;
        } else {
            h -= a.x.heads;
            if (place[t][0] < 0) continue;
            if (h < a.k.heads) {
                src = (const T*)a.k.p + (t0 + t) * a.k.token_stride + h * a.k.head_stride;
                dst = (T*)a.k_pool + place[t][0] + h * a.k_head;
            } else {
                h -= a.k.heads;
                src = (const T*)a.v.p + (t0 + t) * a.v.token_stride + h * a.v.head_stride;
                dst = (T*)a.v_pool + place[t][1] + h * a.v_head;
                rot = false;
            }
        }
        const int o0 = HALF && u < turned ? u * VEC : 2 * u * VEC, o1 = HALF && u < turned ? o0 + half : o0 + VEC;
        V p = *(const V*)(src + o0), q = *(const V*)(src + o1);
        if (rot) {
            const float2* cs = turn + t * half + u * VEC;
            if (HALF) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float x = to_f(p.v[j]), y = to_f(q.v[j]);
                    const float2 w = cs[j];
                    p.v[j] = from_f<T>(x * w.x - y * w.y);
                    q.v[j] = from_f<T>(y * w.x + x * w.y);
                }
            } else if (VEC == 1) {
                const float x = to_f(p.v[0]), y = to_f(q.v[0]);
                const float2 w = cs[0];
                p.v[0] = from_f<T>(x * w.x - y * w.y);
                q.v[0] = from_f<T>(y * w.x + x * w.y);
            } else {
#pragma unroll
                for (int j = 0; j < VEC; j += 2) {
                    const float x = to_f(p.v[j]), y = to_f(p.v[j + (VEC > 1)]);
                    const float2 w = cs[j / 2];
                    p.v[j] = from_f<T>(x * w.x - y * w.y);
                    p.v[j + (VEC > 1)] = from_f<T>(y * w.x + x * w.y);
                }
#pragma unroll
                for (int j = 0; j < VEC; j += 2) {
                    const float x = to_f(q.v[j]), y = to_f(q.v[j + (VEC > 1)]);
                    const float2 w = cs[VEC / 2 + j / 2];
                    q.v[j] = from_f<T>(x * w.x - y * w.y);
                    q.v[j + (VEC > 1)] = from_f<T>(y * w.x + x * w.y);
                }
            }
        }
        *(V*)(dst + o0) = p;
        *(V*)(dst + o1) = q;
    }
}

bool aligned(const Heads& h, int64_t vec, size_t size) {
    return h.heads == 0 || ((reinterpret_cast<uintptr_t>(h.p) % (vec * size)) == 0 && h.token_stride % vec == 0 && h.head_stride % vec == 0);
}

template <class T, int VEC>
cudaError_t launch_rows_t(const RowsArgs& a, int sm_count, cudaStream_t stream) {
    const int heads = a.x.heads + (a.append ? a.k.heads + a.v.heads : 0);
    const int per_token = heads * (a.head_dim / (2 * VEC));
    // four tokens a block once that still fills the GPU; few tokens: blocks share a token's heads
    int block_tokens = (a.tokens >= 4 * 4 * sm_count) ? 4 : 1;
    int shares = 1;
    while (block_tokens == 1 && shares < 8 && (int64_t)a.tokens * shares < 2 * sm_count && per_token > kRowThreads * shares) shares *= 2;
    const dim3 grid((unsigned)ceil_div(a.tokens, block_tokens), (unsigned)shares);
    const size_t smem = (size_t)block_tokens * (a.rot / 2) * sizeof(float2);
    if (a.layout == FD_ROTARY_HALF) k_rows<T, VEC, true><<<grid, kRowThreads, smem, stream>>>(a, block_tokens);
    else k_rows<T, VEC, false><<<grid, kRowThreads, smem, stream>>>(a, block_tokens);
    ++g_launches;
    return cudaGetLastError();
}
template <class T>
cudaError_t launch_rows_any(const RowsArgs& a, int sm_count, cudaStream_t stream) {
    constexpr int VEC = 16 / sizeof(T);
    // vectors of 16 bytes where every row allows them; single elements otherwise (odd head sizes, strides and pointers)
    const bool wide = a.head_dim % (2 * VEC) == 0 && a.rot % (2 * VEC) == 0 && aligned(a.x, VEC, sizeof(T)) && aligned(a.y, VEC, sizeof(T)) &&
                      (!a.append || (aligned(a.k, VEC, sizeof(T)) && aligned(a.v, VEC, sizeof(T))));
    return wide ? launch_rows_t<T, VEC>(a, sm_count, stream) : launch_rows_t<T, 1>(a, sm_count, stream);
}

// ------------------------------------------------------------------------------------------------ eviction
// k_select: one block per (sequence, head).  The weights of the middle tokens are mapped to unsigned keys of the same order; four passes of 8
// bits find the key of rank m from the top, and a last pass in slot order writes down the kept slots (all keys above it, the
// first of those equal to it).  Slots and weights are read before the positions they move to are written: a kept slot moves down only,
// never beyond the slots read so far, so the weights may be compacted in place.
constexpr int kSelThreads = 1024;

__device__ __forceinline__ unsigned weight_key(float w) {
    if (w != w) return 0u;                                   // NaN: below every number
    const unsigned u = __float_as_uint(w + 0.0f);            // (-0 counts as 0)
    return (u >> 31) ? ~u : (u | 0x80000000u);
}

__global__ void __launch_bounds__(kSelThreads) k_select(const EvictArgs a) {
    __shared__ unsigned hist[256];
    __shared__ unsigned s_prefix, s_left;
    __shared__ int warp_sum[2][32], base[2];
    grid_go();
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int n = kv_length(a.batch, b, true);
    const int64_t row = (int64_t)b * a.heads + h;
    const float* w = a.w_in + row * a.w_stride;
    float* wo = a.w_out + row * a.w_stride;
    int* kept = a.kept + row * a.keep;
    const bool all = n <= a.keep;
    const int lo = min(a.first, n), hi = max(lo, n - a.recent);
    unsigned prefix = 0, left = all ? 0 : (unsigned)(a.keep - a.first - a.recent);      // (first + recent <= keep < n)
    if (!all) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
            for (int i = lo + tid; i < hi; i += kSelThreads) {
                const unsigned k = weight_key(w[i]);
                if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1u);
            }
            __syncthreads();
            if (tid < 32) {                                  // bins from the top: lane l holds bins 255 - 8 l ... 248 - 8 l
                unsigned c[8], sum = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) { c[j] = hist[255 - 8 * lane - j]; sum += c[j]; }
                unsigned before = sum;
                for (int o = 1; o < 32; o <<= 1) { const unsigned v = __shfl_up_sync(~0u, before, o); if (lane >= o) before += v; }
                before -= sum;
                // the bin in which the `left` largest end (left 0: none is taken, any bin that holds nothing above it)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (before <= left && left < before + c[j]) { s_prefix = prefix | ((unsigned)(255 - 8 * lane - j) << shift); s_left = left - before; }
                    before += c[j];
                }
            }
            __syncthreads();
            prefix = s_prefix; left = s_left;
            __syncthreads();
        }
    }
    // keys above `prefix` are kept, and the first `left` of those equal to it
    if (tid < 2) base[tid] = 0;
    __syncthreads();
    for (int i0 = 0; i0 < n; i0 += kSelThreads) {
        const int i = i0 + tid;
        float v = 0.f;
        bool keep = false, equal = false;
        if (i < n) {
            v = w[i];
            if (all || i < lo || i >= hi) keep = true;
            else {
                const unsigned k = weight_key(v);
                keep = k > prefix; equal = k == prefix;
            }
        }
        const unsigned be = __ballot_sync(~0u, equal);
        if (lane == 0) warp_sum[0][warp] = __popc(be);
        __syncthreads();
        int before = base[0];
        for (int j = 0; j < warp; ++j) before += warp_sum[0][j];
        if (equal && (unsigned)(before + __popc(be & ((1u << lane) - 1))) < left) keep = true;
        const unsigned bk = __ballot_sync(~0u, keep);
        if (lane == 0) warp_sum[1][warp] = __popc(bk);
        __syncthreads();
        int at = base[1];
        for (int j = 0; j < warp; ++j) at += warp_sum[1][j];
        at += __popc(bk & ((1u << lane) - 1));
        if (keep) { kept[at] = i; wo[at] = v; }
        __syncthreads();
        if (tid == kSelThreads - 1) {
            base[1] = at + (keep ? 1 : 0);
            base[0] = before + __popc(be);
        }
        __syncthreads();
    }
    const int total = all ? n : a.keep;
    for (int i = total + tid; i < a.keep; i += kSelThreads) kept[i] = -1;
    for (int i = total + tid; i < n; i += kSelThreads) wo[i] = 0.f;
}

// k_move: one block per (sequence, head, 64-byte slice of the key or the value rows): slices of a row move independently, so in place they are in nobody's
// way.  A wave of rows is read, the block waits, and the wave is written: row r comes from slot kept[r] >= r, so later waves read nothing that was written.
constexpr int kMoveThreads = 256, kMoveDepth = 8;

__global__ void __launch_bounds__(kMoveThreads) k_move(const EvictArgs a) {
    grid_wait();
    const int h = blockIdx.y, b = blockIdx.z, slices = a.head_dim / 32;
    const bool val = (int)blockIdx.x >= slices;
    const int slice = blockIdx.x - (val ? slices : 0);
    const Batch& B = a.batch;
    const int count = min(kv_length(B, b, false), a.keep);
    const int64_t page_s = val ? a.v_page : a.k_page, token_s = val ? a.v_token : a.k_token, head_s = val ? a.v_head : a.k_head;
    uint16_t* pool = (uint16_t*)(val ? a.v_pool : a.k_pool) + h * head_s + slice * 32 + (threadIdx.x & 3) * 8;
    const int* kept = a.kept + ((int64_t)b * a.heads + h) * a.keep;
    const int* from = B.table + b * B.table_stride;
    const int* to = a.new_table + b * a.new_table_stride;
    const int room = (int)min((int64_t)a.new_max_pages * B.page_size, (int64_t)count);
    if (room < count && threadIdx.x == 0) atomicOr(B.status, kBadLength);
    for (int r0 = 0; r0 < room; r0 += kMoveDepth * (kMoveThreads / 4)) {
        uint4 v[kMoveDepth];
        int64_t at[kMoveDepth];
#pragma unroll
        for (int u = 0; u < kMoveDepth; ++u) {
            const int r = r0 + u * (kMoveThreads / 4) + (threadIdx.x >> 2);
            at[u] = -1;
            if (r < room) {
                const int s = kept[r];
                const int pf = from[s / B.page_size], pt = to[r / B.page_size];
                if (pf < 0 || pf >= B.num_pages || pt < 0 || pt >= B.num_pages) atomicOr(B.status, kBadPage);
                else if (pf != pt || s % B.page_size != r % B.page_size) {
                    v[u] = *(const uint4*)(pool + pf * page_s + (s % B.page_size) * token_s);
                    at[u] = pt * page_s + (r % B.page_size) * token_s;
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kMoveDepth; ++u)
            if (at[u] >= 0) *(uint4*)(pool + at[u]) = v[u];
    }
    if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) a.new_len[b] = count;
}

}  // namespace

cudaError_t launch_rows(const RowsArgs& a, int dtype, int sm_count, cudaStream_t stream) {
    switch (dtype) {
        case FD_BF16: return launch_rows_any<__nv_bfloat16>(a, sm_count, stream);
        case FD_FP16: return launch_rows_any<__half>(a, sm_count, stream);
        default: return launch_rows_any<float>(a, sm_count, stream);
    }
}

cudaError_t launch_evict(const EvictArgs& a, cudaStream_t stream) {
    k_select<<<dim3(a.heads, a.batch.batch), kSelThreads, 0, stream>>>(a);
    ++g_launches;
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    ++g_launches;
    return launch_behind(stream, dim3(2 * a.head_dim / 32, a.heads, a.batch.batch), dim3(kMoveThreads), 0, k_move, a);
}

}  // namespace kv
}  // namespace fd
