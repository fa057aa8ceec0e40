// Attention of few rows a sequence (single tokens, a few drafted ones) over a paged cache: kernels bound by the cache's bytes.
//
// k_few.  A sequence has at most 16 rows (new token, query head of the group) per cached head, so a tile of tcgen05 would be 7/8 padding and, worse, every 128
// tokens would wait for the chain product -> TMEM -> softmax -> TMEM -> product.  Here each warp goes its own way: it takes every fourth chunk of 16
// tokens of the CTA's part (32 where a row has 64 coordinates), keeps several chunks of keys and values in flight by TMA in a ring of its own (no barrier between warps),
// multiplies with mma.sync m16n8k16 out of ldmatrix fragments and holds scores, weights and the 16 x D result in registers.  Two CTAs of four warps an SM
// keep 192 KB in flight.  The warps' results are joined in shared memory at the end, the parts of a cache by k_join.
// With weights wanted, each row's scaled scores go to the workspace (4 bytes a row and token, beside 4 D bytes of keys and values), and k_join
// turns them into weights once the norm is known: the keys are not read again.
#include <algorithm>

#include "fd_kv_dev.h"

namespace fd {
namespace kv {
namespace {

constexpr int kWarpsFew = 4;

template <int D>
struct GeoFew {
    static constexpr int kKeys = D == 128 ? 16 : 32;             // tokens of a chunk: 8 KB of keys and values
    static constexpr int kStages = 3;
    static constexpr int kHalf = kKeys * 128;                    // 64 coordinates of a chunk
    static constexpr int kTile = (D / 64) * kHalf;               // keys or values of a chunk
    static constexpr int kSmem = 1024 + kWarpsFew * kStages * 2 * kTile + 256 + kWarpsFew * 16 * 8;
    static_assert(kWarpsFew * 16 * D * 4 <= kWarpsFew * kStages * 2 * kTile, "the warps' results fit in the ring");
};

template <class T> __device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma16816<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool TRANS>
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
    if (TRANS)
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
    else
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

// Takes elements that are not finite out of a fragment of values, and the rows of tokens behind the sequence; true if there were any of the former.
template <class T>
__device__ __forceinline__ bool clean(uint32_t& v, int valid) {                // valid: of this register's two tokens, those that exist
    constexpr uint32_t E = Elem<T>::kExponent;
    if (valid < 2) v &= valid == 1 ? 0xffffu : 0u;
    bool hit = false;
    if ((v & E) == E) { v &= 0xffff0000u; hit = true; }
    if ((v & (E << 16)) == (E << 16)) { v &= 0xffffu; hit = true; }
    return hit;
}

template <class T, int D>
__global__ void __launch_bounds__(kWarpsFew * 32, 2)
k_few(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const AttendArgs a) {
    using G = GeoFew<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* base = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint64_t* bars = (uint64_t*)(base + kWarpsFew * G::kStages * 2 * G::kTile);
    int* flags = (int*)(bars + kWarpsFew * G::kStages);              // abort, odd
    float* s_m = (float*)(flags + 2);                                // [warp][16] maxima, then [warp][16] sums
    float* s_l = s_m + kWarpsFew * 16;
    volatile int* abort_flag = flags;
    unsigned int* status = a.batch.status + 1;
    grid_go();

    const int warp = warp_index(), lane = threadIdx.x & 31;
    const int split = blockIdx.x % a.splits, h = (blockIdx.x / a.splits) % a.heads, b = blockIdx.x / (a.splits * a.heads);
    Work w;
    w.b = b; w.begin = q_begin(a.batch, b); w.count = max(0, q_begin(a.batch, b + 1) - w.begin); w.t0 = 0;
    if (w.count == 0) return;
    if (w.count > kFewRows / a.group) {                              // more than max_new promised
        if (threadIdx.x == 0) atomicOr(a.batch.status, kBadLength);
        return;
    }
    w.n = kv_length(a.batch, b, threadIdx.x == 0);
    w = uniform(w);
    constexpr int KEYS = G::kKeys, NT = KEYS / 8;
    const int rows = w.count * a.group, part = a.split_tiles * 64;
    const int k0 = max(see_lo(a, w, 0), split * part), k1 = a.splits > 1 ? min(see_hi(a, w, w.count - 1), (split + 1) * part) : see_hi(a, w, w.count - 1);
    const int full0 = see_lo(a, w, w.count - 1), full1 = see_hi(a, w, 0);          // every row sees [full0, full1)
    const int c0 = k0 / KEYS, chunks = max(0, (k1 + KEYS - 1) / KEYS - c0);
    const int mine = chunks > warp ? (chunks - warp + kWarpsFew - 1) / kWarpsFew : 0;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kWarpsFew * G::kStages; ++i) mbar_init(&bars[i], 1);
        flags[0] = flags[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();

    uint8_t* ring = base + warp * G::kStages * 2 * G::kTile;
    uint64_t* full = bars + warp * G::kStages;
    const int boxes = KEYS / a.box_rows;                             // 1, 2 or 4 a chunk
    int page = 0;                                                    // of box 32 k + lane of this warp's boxes, all chunks in a row
    auto issue = [&](int i) {
        const int e = i * boxes;
        if ((e & 31) == 0) {
            const int ii = (e + lane) / boxes, key = (c0 + warp + kWarpsFew * ii) * KEYS + ((e + lane) % boxes) * a.box_rows;
            page = 0;
            if (ii < mine && key < w.n) {
                page = a.batch.table[b * a.batch.table_stride + key / a.batch.page_size];
                if (page < 0 || page >= a.batch.num_pages) { page = a.batch.num_pages; atomicOr(a.batch.status, kBadPage); }   // (outside: TMA fills with zeros)
            }
        }
        const int at = __shfl_sync(~0u, page, (e + lane) & 31), st = i % G::kStages;
        const int key0 = (c0 + warp + kWarpsFew * i) * KEYS, key = key0 + lane * a.box_rows;
        const int live = min(boxes, (w.n - key0 + a.box_rows - 1) / a.box_rows);
        uint8_t* k = ring + st * 2 * G::kTile;
        if (lane == 0) mbar_expect_tx(&full[st], (uint32_t)(live * a.box_rows * D * 4));
        __syncwarp();
        if (lane < live) {
#pragma unroll
            for (int x = 0; x < D / 64; ++x) {
                tma_load_4d(k + x * G::kHalf + lane * a.box_rows * 128, &map_k, x * 64, key % a.batch.page_size, h, at, &full[st]);
                tma_load_4d(k + G::kTile + x * G::kHalf + lane * a.box_rows * 128, &map_v, x * 64, key % a.batch.page_size, h, at, &full[st]);
            }
        }
        __syncwarp();
    };
    for (int i = 0; i < G::kStages && i < mine; ++i) issue(i);

    // fragments: this thread's rows are g and g + 8, its columns 2 t, 2 t + 1 of every 8
    const int g = lane >> 2, t = lane & 3;
    uint32_t qf[D / 16][4];
    int lo[2], hi[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int row = g + 8 * r, token = row / a.group;
        const bool on = row < rows;
        lo[r] = on ? see_lo(a, w, token) : 0;
        hi[r] = on ? see_hi(a, w, token) : 0;
        const T* q = (const T*)a.q.p + (w.begin + token) * a.q.token_stride + (h * a.group + row % a.group) * a.q.head_stride + 2 * t;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            qf[k][r] = on ? *(const uint32_t*)(q + 16 * k) : 0u;
            qf[k][2 + r] = on ? *(const uint32_t*)(q + 16 * k + 8) : 0u;
        }
    }
    float* score_row[2];
#pragma unroll
    for (int r = 0; r < 2; ++r)
        score_row[r] = a.scores && a.w_out && g + 8 * r < rows ? a.scores + (((int64_t)b * a.heads + h) * kFewRows + g + 8 * r) * a.score_stride + 2 * t : nullptr;

    float o[D / 8][4];
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][e] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    const float c = a.scale_log2;
    bool odd = false, ok = true;
    // ldmatrix: matrix i = lane / 8, its row lane % 8; keys: matrices (token half i / 2, coordinate half i % 2); values, transposed: (token half i % 2, coordinate group i / 2)
    const int mi = lane >> 3, mr = lane & 7;
    const uint32_t krow = (uint32_t)(((mi >> 1) * 8 + mr) * 128), vrow = (uint32_t)(((mi & 1) * 8 + mr) * 128);

    int i = 0;
    for (; i < mine; ++i) {
        const int st = i % G::kStages, key = (c0 + warp + kWarpsFew * i) * KEYS;
        ok = __all_sync(~0u, mbar_wait(&full[st], (i / G::kStages) & 1, abort_flag, status, 41));
        if (!ok) break;
        const uint32_t ks = smem_u32(ring + st * 2 * G::kTile), vs = ks + G::kTile;
        float s[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
                uint32_t f[4];
                ldmatrix4<false>(f, ks + (k / 4) * G::kHalf + n * 1024 + krow + ((uint32_t)(((k % 4) * 2 + (mi & 1)) ^ mr) << 4));
                mma16816<T>(s[n], qf[k], f[0], f[1]);
                mma16816<T>(s[n + 1], qf[k], f[2], f[3]);
            }
        const bool whole = key >= full0 && key + KEYS <= full1;
        if (!whole) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = key + 8 * n + 2 * t + (e & 1);
                    if (j < lo[e >> 1] || j >= hi[e >> 1]) s[n][e] = -INFINITY;
                }
        }
#pragma unroll
        for (int r = 0; r < 2; ++r)
            if (score_row[r]) {
#pragma unroll
                for (int n = 0; n < NT; ++n) *(float2*)(score_row[r] + key + 8 * n) = make_float2(s[n][2 * r] * c, s[n][2 * r + 1] * c);
            }
        float top[2];
        bool raise = false;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            top[r] = m[r];
#pragma unroll
            for (int n = 0; n < NT; ++n) top[r] = max_nan(top[r], s[n][2 * r], s[n][2 * r + 1]);
            raise |= !((top[r] - m[r]) * c <= kLazy) && top[r] != m[r];
        }
        if (__any_sync(~0u, raise)) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                top[r] = max_nan(top[r], __shfl_xor_sync(~0u, top[r], 1));
                top[r] = max_nan(top[r], __shfl_xor_sync(~0u, top[r], 2));
                const float f = top[r] == m[r] ? 1.0f : ex2f((m[r] - top[r]) * c);
                m[r] = top[r];
                l[r] *= f;
#pragma unroll
                for (int n = 0; n < D / 8; ++n) { o[n][2 * r] *= f; o[n][2 * r + 1] *= f; }
            }
        }
        uint32_t p[NT / 2][4];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const float mc = m[r] == -INFINITY ? 0.f : m[r] * c;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float e0 = ex2f(fmaf(s[n][2 * r], c, -mc)), e1 = ex2f(fmaf(s[n][2 * r + 1], c, -mc));
                l[r] += e0 + e1;
                p[n / 2][2 * (n % 2) + r] = Elem<T>::pack(e0, e1);
            }
        }
#pragma unroll
        for (int x = 0; x < KEYS / 16; ++x) {
            const int left0 = min(max(w.n - (key + 16 * x + 2 * t), 0), 2), left1 = min(max(w.n - (key + 16 * x + 8 + 2 * t), 0), 2);
#pragma unroll
            for (int n = 0; n < D / 16; ++n) {
                uint32_t f[4];
                ldmatrix4<true>(f, vs + (n / 4) * G::kHalf + x * 2048 + vrow + ((uint32_t)(((n % 4) * 2 + (mi >> 1)) ^ mr) << 4));
                if (!whole) odd |= clean<T>(f[0], left0) | clean<T>(f[1], left1) | clean<T>(f[2], left0) | clean<T>(f[3], left1);
                mma16816<T>(o[2 * n], p[x], f[0], f[1]);
                mma16816<T>(o[2 * n + 1], p[x], f[2], f[3]);
            }
        }
        __syncwarp();
        if (i + G::kStages < mine) issue(i + G::kStages);
    }
    if (!ok && lane == 0) {                      // aborted: copies in flight land before the CTA exits (bounded)
        for (int k = i; k < min(i + G::kStages, mine); ++k) {
            const long long t0 = clock64();
            while (!mbar_try_wait(&full[k % G::kStages], (k / G::kStages) & 1) && clock64() - t0 < 20000000ll) {}
        }
    }
    if (odd) flags[1] = 1;
    // the warps' results, over the ring
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(~0u, l[r], 1);
        l[r] += __shfl_xor_sync(~0u, l[r], 2);
        if (t == 0) { s_m[warp * 16 + g + 8 * r] = m[r]; s_l[warp * 16 + g + 8 * r] = l[r]; }
    }
    __syncthreads();
    float* s_o = (float*)base;                   // [warp][16][D]
#pragma unroll
    for (int r = 0; r < 2; ++r)
        if (g + 8 * r < rows)
#pragma unroll
            for (int n = 0; n < D / 8; ++n)
                *(float2*)(s_o + (warp * 16 + g + 8 * r) * D + 8 * n + 2 * t) = make_float2(o[n][2 * r], o[n][2 * r + 1]);
    __syncthreads();
    if (*abort_flag) return;
    const bool any_odd = *(volatile int*)&flags[1];
    for (int x = threadIdx.x; x < rows * (D / 4); x += kWarpsFew * 32) {
        const int row = x / (D / 4), d = (x % (D / 4)) * 4;
        float top = -INFINITY;
#pragma unroll
        for (int k = 0; k < kWarpsFew; ++k) top = max_nan(top, s_m[k * 16 + row]);
        float v[4] = {0.f, 0.f, 0.f, 0.f}, sum = 0.f;
        if (top != -INFINITY) {
#pragma unroll
            for (int k = 0; k < kWarpsFew; ++k) {
                const float mk = s_m[k * 16 + row];
                if (mk == -INFINITY) continue;
                const float f = mk == top ? 1.0f : ex2f((mk - top) * c);
                const float4 y = *(const float4*)(s_o + (k * 16 + row) * D + d);
                sum = fmaf(f, s_l[k * 16 + row], sum);
                v[0] = fmaf(f, y.x, v[0]); v[1] = fmaf(f, y.y, v[1]); v[2] = fmaf(f, y.z, v[2]); v[3] = fmaf(f, y.w, v[3]);
            }
            const float inv = 1.0f / sum;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] *= inv;
        }
        const int token = row / a.group, head = h * a.group + row % a.group;
        const int64_t at = w.begin + token;
        if (any_odd) {
            // what is not finite among tokens that some row does not see, for the rows that see it
            for (int key = max(see_lo(a, w, token), k0); key < min(see_hi(a, w, token), k1); ++key) {
                const int chunk = key / KEYS * KEYS;
                if (chunk >= full0 && chunk + KEYS <= full1) continue;
                const int page = a.batch.table[b * a.batch.table_stride + key / a.batch.page_size];
                if (page < 0 || page >= a.batch.num_pages) continue;
                const int64_t from = page * a.v_page + (key % a.batch.page_size) * a.v_token + h * a.v_head + d;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float y = Elem<T>::at(a.v_pool, from + e);
                    if (!isfinite(y)) v[e] += y;
                }
            }
        }
        const float lse2 = top == -INFINITY ? -INFINITY : top * c + log2f(sum);
        if (a.splits > 1) {
            const int64_t to = split * (int64_t)a.batch.total_q * a.q_heads + at * a.q_heads + head;
            if (d == 0) a.part_lse[to] = lse2;
            if (top != -INFINITY) *(float4*)(a.part_o + to * D + d) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
            *(uint2*)((T*)a.out.p + at * a.out.token_stride + head * a.out.head_stride + d) = make_uint2(Elem<T>::pack(v[0], v[1]), Elem<T>::pack(v[2], v[3]));
            if (d == 0 && a.lse) a.lse[at * a.q_heads + head] = lse2 == -INFINITY ? -INFINITY : (float)((double)lse2 * 0.69314718055994530942);
        }
    }
}

template <class T, int D>
cudaError_t few_t(const AttendArgs& a, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t stream) {
    cudaError_t e = cudaFuncSetAttribute(k_few<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, GeoFew<D>::kSmem);
    if (e != cudaSuccess) return e;
    k_few<T, D><<<(unsigned)((int64_t)a.batch.batch * a.heads * a.splits), kWarpsFew * 32, GeoFew<D>::kSmem, stream>>>(mk, mv, a);
    ++g_launches;
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    return a.splits > 1 || a.w_out ? launch_join(a, stream) : cudaSuccess;
}

}  // namespace

cudaError_t launch_few(const AttendArgs& a, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t stream) { return FD_KV_PICK(few_t, a, mk, mv, stream); }

}  // namespace kv
}  // namespace fd
