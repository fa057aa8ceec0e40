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

// A row that is read once (8192 tokens of 32 heads: 28.3 -> 27.2 us; the results are left to the cache, for what reads them next.  Appends lose 2 us of 44 by it).
template <class V> __device__ __forceinline__ V load_once(const void* p) {
    if constexpr (sizeof(V) == 16) {
        const uint4 x = __ldcs((const uint4*)p);
        return *(const V*)&x;
    } else return *(const V*)p;
}

template <class T, int VEC, bool HALF, bool APPEND>
__global__ void __launch_bounds__(kRowThreads, APPEND ? 8 : 6) k_rows(const RowsArgs a, const int block_tokens) {
    extern __shared__ float2 turn[];                         // [block_tokens][rot / 2]
    __shared__ int64_t place[16][2];                         // pool offset of a token's key and value row of head 0, -1: nowhere
    using V = Vec<T, VEC>;
    grid_wait();
    grid_go();
    // (an append may be padded, and its first tokens may belong to no sequence)
    const int live = APPEND ? q_begin(a.batch, a.batch.batch) : a.tokens;
    const int b0 = blockIdx.x * block_tokens, t0 = APPEND ? max(b0, q_begin(a.batch, 0)) : b0, nt = max(0, min(block_tokens - (t0 - b0), live - t0));
    const int half = a.rot / 2;
    for (int i = threadIdx.x; i < nt * half; i += kRowThreads) {
        const int t = i / half, f = i - t * half;
        const double turns = (double)a.positions[t0 + t] * a.freqs[f] * kTurn;
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        turn[i] = make_float2(c * a.scale, s * a.scale * a.sign);
    }
    if (APPEND && (int)threadIdx.x < nt) {
        const Batch& B = a.batch;
        const int t = t0 + threadIdx.x;
        int lo = 0, hi = B.batch;                            // last sequence that begins at or before t
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (q_begin(B, mid) <= t) lo = mid; else hi = mid;
        }
        const int begin = q_begin(B, lo), end = q_begin(B, lo + 1);
        place[threadIdx.x][0] = place[threadIdx.x][1] = -1;
        if (t >= begin && t < end) {
            // (of a length that kv_length had to cut nothing is written: the slots at the bound hold older tokens)
            const int n = kv_length(B, lo, true), slot = n == B.kv_len[lo] ? n - (end - begin) + (t - begin) : -1;
            const int page = slot < 0 ? -1 : B.table[lo * B.table_stride + B.page_of(slot)];
            if (slot < 0) atomicOr(B.status, kBadLength);
            else if (page < 0 || page >= B.num_pages) atomicOr(B.status, kBadPage);
            else {
                place[threadIdx.x][0] = page * a.k_page + B.row_of(slot) * a.k_token;
                place[threadIdx.x][1] = page * a.v_page + B.row_of(slot) * a.v_token;
            }
        }
    }
    __syncthreads();
    const int unit_count = a.head_dim / (2 * VEC), turned = a.rot / (2 * VEC);
    const int heads = a.x.heads + (APPEND ? a.k.heads + a.v.heads : 0);
    // this thread's units: (token, head, unit) numbers `me`, me + all, ...; they advance without divisions
    const int all = kRowThreads * gridDim.y, me = threadIdx.x + blockIdx.y * kRowThreads;
    int u = me % unit_count, h = me / unit_count, t = h / heads;
    h -= t * heads;
    const int du = all % unit_count, dh = (all / unit_count) % heads, dt = all / unit_count / heads;
    for (; t < nt; u += du, h += dh, t += dt) {
        if (u >= unit_count) { u -= unit_count; ++h; }
        if (h >= heads) { h -= heads; ++t; }
        if (t >= nt) break;
        const T* src;
        T* dst;
        bool rot = u < turned;
        if (!APPEND || h < a.x.heads) {
            src = (const T*)a.x.p + (t0 + t) * a.x.token_stride + h * a.x.head_stride;
            dst = (T*)a.y.p + (t0 + t) * a.y.token_stride + h * a.y.head_stride;
        } else {
            int k = h - a.x.heads;
            if (place[t][0] < 0) continue;
            if (k < a.k.heads) {
                src = (const T*)a.k.p + (t0 + t) * a.k.token_stride + k * a.k.head_stride;
                dst = (T*)a.k_pool + place[t][0] + k * a.k_head;
            } else {
                k -= a.k.heads;
                src = (const T*)a.v.p + (t0 + t) * a.v.token_stride + k * a.v.head_stride;
                dst = (T*)a.v_pool + place[t][1] + k * a.v_head;
                rot = false;
            }
        }
        const int o0 = HALF && u < turned ? u * VEC : 2 * u * VEC, o1 = HALF && u < turned ? o0 + half : o0 + VEC;
        V p = APPEND ? *(const V*)(src + o0) : load_once<V>(src + o0), q = APPEND ? *(const V*)(src + o1) : load_once<V>(src + o1);
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
    // Four tokens a block, in appends eight (6 prompts of 700 to 2048 tokens: 45.3 -> 43.5 us; without an append they cost 1.4 us of 28), once that still fills the GPU.
    // Few tokens: blocks share a token's heads.
    const int most = a.append ? 8 : 4;
    int block_tokens = a.tokens >= 4 * most * sm_count ? most : 1;
    int shares = 1;
    while (block_tokens == 1 && shares < 8 && (int64_t)a.tokens * shares < 2 * sm_count && per_token > kRowThreads * shares) shares *= 2;
    const dim3 grid((unsigned)ceil_div(a.tokens, block_tokens), (unsigned)shares);
    const size_t smem = (size_t)block_tokens * (a.rot / 2) * sizeof(float2);
    ++g_launches;
    return launch_behind(stream, grid, dim3(kRowThreads), smem, a.layout == FD_ROTARY_HALF ? (a.append ? k_rows<T, VEC, true, true> : k_rows<T, VEC, true, false>)
                                                                                           : (a.append ? k_rows<T, VEC, false, true> : k_rows<T, VEC, false, false>), a, block_tokens);
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
// k_select: one block per (sequence, head).  The weights of the middle tokens are mapped to unsigned keys of the same order, kept in shared memory (beyond
// kSelKeys tokens they are read again each time).  The m-th largest key is found 11, 11 and 10 bits at a time by a histogram and a scan of
// it from the top.  (Two bits at a time, by counting the keys at or above three candidates, needs 16 rounds of a barrier each: 600 keys took 12.5 us, now 9.)  Then each
// warp counts, and after a scan over the warps writes down, the kept slots of its stretch in order: all keys above the found one, the first of those
// equal to it.
constexpr int kSelKeys = 40960;

__device__ __forceinline__ unsigned weight_key(float w) {
    if (w != w) return 0u;                                   // NaN: below every number
    const unsigned u = __float_as_uint(w + 0.0f);            // (-0 counts as 0)
    return (u >> 31) ? ~u : (u | 0x80000000u);
}

// 512 threads up to 4096 tokens (1100 tokens: 9.8 us a call against 10.9 with 1024), 1024 beyond (8192 tokens: 45.9 us against 50.2).
template <int kSelThreads>
__global__ void __launch_bounds__(kSelThreads) k_select(const EvictArgs a) {
    constexpr int kSelWarps = kSelThreads / 32, kSelBins = 2048 / kSelThreads;
    extern __shared__ unsigned s_key[];
    __shared__ unsigned hist[2048];
    __shared__ unsigned warp_total[kSelWarps], s_bin, s_left;
    __shared__ unsigned warp_above[kSelWarps], warp_equal[kSelWarps];
    grid_wait();
    grid_go();
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int n = kv_length(a.batch, b, true);
    const int64_t row = (int64_t)b * a.heads + h;
    int* kept = a.kept + row * a.keep;
    const bool whole = n == a.batch.kv_len[b];               // (a length that kv_length had to cut: nothing is kept, moved or counted, so that nothing is lost)
    if (n <= a.keep || !whole) {
        for (int i = tid; i < a.keep; i += kSelThreads) kept[i] = whole && i < n ? i : -1;
        return;
    }
    const int lo = a.first, hi = n - a.recent, len = hi - lo;            // (first + recent <= keep < n)
    const unsigned left = (unsigned)(a.keep - a.first - a.recent);       // < len
    const float* w = a.w_in + row * a.w_stride + lo;
    const bool held = len <= kSelKeys;
    if (held) for (int i = tid; i < len; i += kSelThreads) s_key[i] = weight_key(w[i]);
    __syncthreads();
    auto key = [&](int i) { return held ? s_key[i] : weight_key(w[i]); };
    unsigned found = 0, want = left;
    if (left == 0) found = 0xffffffffu;                                  // (above every key)
    for (int pass = 0; pass < 3 && left > 0; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const unsigned mask = pass == 2 ? 1023u : 2047u;
        for (int i = tid; i < 2048; i += kSelThreads) hist[i] = 0;
        __syncthreads();
#pragma unroll 4
        for (int i = tid; i < len; i += kSelThreads) {
            const unsigned k = key(i);
            if (pass == 0 || (k >> (pass == 1 ? 21 : 10)) == (found >> (pass == 1 ? 21 : 10))) atomicAdd(&hist[(k >> shift) & mask], 1u);
        }
        __syncthreads();
        // bins from the top, a few a thread: the one in which the want-th largest lies
        unsigned c[kSelBins], sum = 0;
#pragma unroll
        for (int j = 0; j < kSelBins; ++j) sum += c[j] = hist[2047 - kSelBins * tid - j];
        unsigned upto = sum;
        for (int o = 1; o < 32; o <<= 1) { const unsigned v = __shfl_up_sync(~0u, upto, o); if (lane >= o) upto += v; }
        if (lane == 31) warp_total[warp] = upto;
        __syncthreads();
        for (int j = 0; j < warp; ++j) upto += warp_total[j];
        unsigned before = upto - sum;
#pragma unroll
        for (int j = 0; j < kSelBins; ++j) {
            if (before < want && want <= before + c[j]) { s_bin = 2047 - kSelBins * tid - j; s_left = want - before; }
            before += c[j];
        }
        __syncthreads();
        found |= s_bin << shift;
        want = s_left;
    }
    const int stretch = (len + kSelThreads - 1) / kSelThreads * 32, i0 = warp * stretch, i1 = min(len, i0 + stretch);
    unsigned above = 0, equal = 0;
#pragma unroll 4
    for (int i = i0; i < i1; i += 32) {
        const unsigned k = i + lane < i1 ? key(i + lane) : 0u;
        above += __popc(__ballot_sync(~0u, i + lane < i1 && k > found));
        equal += __popc(__ballot_sync(~0u, i + lane < i1 && k == found));
    }
    if (lane == 0) { warp_above[warp] = above; warp_equal[warp] = equal; }
    __syncthreads();
    unsigned all_above = 0, above_before = 0, equal_before = 0;
    for (int j = 0; j < kSelWarps; ++j) {
        all_above += warp_above[j];
        if (j < warp) { above_before += warp_above[j]; equal_before += warp_equal[j]; }
    }
    const unsigned take = left - all_above;                              // of the equal ones
#pragma unroll 4
    for (int i = i0; i < i1; i += 32) {
        const bool in = i + lane < i1;
        const unsigned k = in ? key(i + lane) : 0u, below = (1u << lane) - 1;
        const unsigned ba = __ballot_sync(~0u, in && k > found), be = __ballot_sync(~0u, in && k == found);
        const unsigned at_above = above_before + __popc(ba & below), at_equal = equal_before + __popc(be & below);
        if (in && (k > found || (k == found && at_equal < take))) kept[lo + at_above + min(at_equal, take)] = lo + i + lane;
        above_before += __popc(ba);
        equal_before += __popc(be);
    }
    for (int i = tid; i < lo; i += kSelThreads) kept[i] = i;
    for (int i = tid; i < a.recent; i += kSelThreads) kept[a.keep - a.recent + i] = hi + i;
}

// k_move: moves the kept rows, a few blocks for the key and the value rows of each (sequence, head).  To other pages: every block takes a range of rows, whole rows at a
// time.  In place: every block takes a slice of 64 bytes of all rows, since slices move independently; a wave of rows is read, the block waits,
// and the wave is written.  Row r comes from slot kept[r] >= r, so later waves read nothing that was written.  Three waves are under way at
// once in both: the slots of the next but one, the pages of the next, the rows of this.  One more block a head moves the weights, in waves as well.
constexpr int kMoveThreads = 256, kMoveDepth = 2;

template <int LANES, bool IN_PLACE>
__device__ __forceinline__ void move_rows(const EvictArgs& a, uint16_t* pool, int64_t page_s, int64_t token_s, const int* kept, const int* from, const int* to, int r0, int room) {
    constexpr int kRows = kMoveThreads / LANES, kWave = kMoveDepth * kRows;
    const Batch& B = a.batch;
    const int mine = (int)threadIdx.x / LANES;
    pool += threadIdx.x % LANES * 8;
    int slot[2][kMoveDepth], pf[kMoveDepth], pt[kMoveDepth];
    auto slots = [&](int r0, int (&s)[kMoveDepth]) {
#pragma unroll
        for (int u = 0; u < kMoveDepth; ++u) {
            const int r = r0 + u * kRows + mine;
            s[u] = r < room ? kept[r] : -1;
        }
    };
    auto pages = [&](int r0, const int (&s)[kMoveDepth]) {
#pragma unroll
        for (int u = 0; u < kMoveDepth; ++u) {
            const int r = r0 + u * kRows + mine;
            pf[u] = s[u] >= 0 ? from[B.page_of(s[u])] : 0;
            pt[u] = s[u] >= 0 ? to[B.page_of(r)] : 0;
        }
    };
    slots(r0, slot[0]);
    slots(r0 + kWave, slot[1]);
    pages(r0, slot[0]);
    for (; r0 < room; r0 += kWave) {
        int64_t dst[kMoveDepth];
        uint4 v[kMoveDepth];
        bool bad = false;
#pragma unroll
        for (int u = 0; u < kMoveDepth; ++u) {
            const int r = r0 + u * kRows + mine, s = slot[0][u];
            const int64_t src = pf[u] * page_s + B.row_of(s) * token_s;
            dst[u] = pt[u] * page_s + B.row_of(r) * token_s;
            const bool off = pf[u] < 0 || pf[u] >= B.num_pages || pt[u] < 0 || pt[u] >= B.num_pages;
            bad |= off;
            if (s < 0 || off || src == dst[u]) dst[u] = -1;
            if (dst[u] >= 0) v[u] = *(const uint4*)(pool + src);
            slot[0][u] = slot[1][u];
        }
        slots(r0 + 2 * kWave, slot[1]);
        pages(r0 + kWave, slot[0]);
        if (bad) atomicOr(B.status, kBadPage);
        if (IN_PLACE) __syncthreads();
#pragma unroll
        for (int u = 0; u < kMoveDepth; ++u)
            if (dst[u] >= 0) *(uint4*)(pool + dst[u]) = v[u];
    }
}

template <int D>
__global__ void __launch_bounds__(kMoveThreads) k_move(const EvictArgs a, const int shares, const bool write_len) {
    const int h = blockIdx.y, b = blockIdx.z;
    grid_wait();
    grid_go();
    const Batch& B = a.batch;
    const int* kept = a.kept + ((int64_t)b * a.heads + h) * a.keep;
    if ((int)blockIdx.x == 2 * shares) {
        const int n = kv_length(B, b, false), raw = B.kv_len[b], count = min(n, a.keep);
        if (write_len && h == 0 && threadIdx.x == 0) a.new_len[b] = n == raw ? count : raw;
        if (n != raw) return;
        const float* w = a.w_in + ((int64_t)b * a.heads + h) * a.w_stride;
        float* out = a.w_out + ((int64_t)b * a.heads + h) * a.w_stride;
        constexpr int kDeep = 4;
        for (int r0 = 0; r0 < n; r0 += kDeep * kMoveThreads) {
            float v[kDeep];
#pragma unroll
            for (int u = 0; u < kDeep; ++u) {
                const int r = r0 + u * kMoveThreads + threadIdx.x;
                v[u] = r < count ? w[kept[r]] : 0.f;
            }
            __syncthreads();
#pragma unroll
            for (int u = 0; u < kDeep; ++u) {
                const int r = r0 + u * kMoveThreads + threadIdx.x;
                if (r < n) out[r] = v[u];
            }
        }
        return;
    }
    const bool val = (int)blockIdx.x >= shares;
    const int share = blockIdx.x - (val ? shares : 0);
    const int64_t page_s = val ? a.v_page : a.k_page, token_s = val ? a.v_token : a.k_token;
    uint16_t* pool = (uint16_t*)(val ? a.v_pool : a.k_pool) + h * (val ? a.v_head : a.k_head);
    const int* from = B.table + b * B.table_stride;
    const int* to = a.new_table + b * a.new_table_stride;
    // (kept holds -1 behind the last row, so no length is waited for; the tables are the same or have no page in common, so their first pages tell)
    if (from[0] == to[0]) {
        if (share < D / 32) move_rows<4, true>(a, pool + share * 32, page_s, token_s, kept, from, to, 0, a.keep);
    } else {
        const int per = (a.keep + shares - 1) / shares;
        move_rows<D / 8, false>(a, pool, page_s, token_s, kept, from, to, share * per, min(a.keep, (share + 1) * per));
    }
}

// New lengths written over the old ones: only once every block that reads the old ones is done.
__global__ void k_new_len(const EvictArgs a) {
    grid_wait();
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b >= a.batch.batch) return;
    const int n = kv_length(a.batch, b, false);
    if (n == a.batch.kv_len[b]) a.new_len[b] = min(n, a.keep);
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
    const size_t smem = sizeof(unsigned) * (size_t)(a.batch.max_len < kSelKeys ? a.batch.max_len : kSelKeys);
    // (512 threads need no leave for their shared memory, but a call without it lost 4 us between the two kernels: 1100 tokens 13.9 us against 10.2)
    const bool many = a.batch.max_len > 4096;
    cudaError_t e = many ? allow_smem<k_select<1024>>(kSelKeys * sizeof(unsigned)) : allow_smem<k_select<512>>(kSelKeys * sizeof(unsigned));
    if (e != cudaSuccess) return e;
    ++g_launches;
    e = launch_behind(stream, dim3(a.heads, a.batch.batch), dim3(many ? 1024 : 512), smem, many ? k_select<1024> : k_select<512>, a);
    if (e != cudaSuccess) return e;
    const bool over = a.new_len == a.batch.kv_len;
    // blocks for about 16 KB in flight on every SM twice over, of 64 rows or more; in place as many as a row has slices of 64 bytes do work
    int shares = a.head_dim / 32;
    while (shares < 32 && 2 * (int64_t)shares * a.heads * a.batch.batch < 1200 && a.keep / (2 * shares) >= 64) shares *= 2;
    const dim3 grid(2 * shares + 1, a.heads, a.batch.batch);
    ++g_launches;
    e = launch_behind(stream, grid, dim3(kMoveThreads), 0, a.head_dim == 128 ? k_move<128> : k_move<64>, a, shares, !over);
    if (e != cudaSuccess || !over) return e;
    ++g_launches;
    return launch_behind(stream, dim3((unsigned)ceil_div(a.batch.batch, 256)), dim3(256), 0, k_new_len, a);
}

}  // namespace kv
}  // namespace fd
