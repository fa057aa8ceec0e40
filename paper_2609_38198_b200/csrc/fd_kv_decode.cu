// Attention of few rows a sequence (single tokens, a few drafted ones) over a paged cache: kernels bound by the cache's bytes.
//
// k_few.  A sequence has at most 16 rows (new token, query head of the group) per cached head, so a tile of tcgen05 would be 7/8 padding and, worse, every 128
// tokens would wait for the chain product -> TMEM -> softmax -> TMEM -> product.  Here each warp goes its own way: it takes every fourth chunk of 16
// tokens of the CTA's part (32 where a row has 64 coordinates), keeps several chunks of keys and values in flight by TMA in a ring of its own (no barrier between warps),
// multiplies with mma.sync m16n8k16 out of ldmatrix fragments and holds scores, weights and the 16 x D result in registers.  Two CTAs of four warps an SM
// keep 192 KB in flight.  The caches of a batch are laid end to end in units of 64 tokens, and every CTA takes an equal stretch of them whatever the
// lengths (which only the device knows): with a fixed number of parts a cache, two contexts of 131072 and 78000 tokens took 58 us, now 50.  Bytes bound it:
// 64 sequences of 1400 to 4096 tokens 127 us a call, 5.7 TB/s.  A CTA's warps are joined in shared memory at the end of each cache it touches; a cache
// that several CTAs share is joined by k_few_join.
// With weights wanted, each row's scaled scores go to the workspace (4 bytes a row and token, beside 4 D bytes of keys and values), and k_few_join
// turns them into weights once the norm is known: the keys are not read again.
#include <algorithm>

#include "fd_kv_dev.h"

namespace fd {
namespace kv {
namespace {

constexpr int kWarpsFew = kFewWarps;
// (see Elem; raising the maximum costs little beside the cache's bytes)
template <class T> constexpr float kLazy = 8.f;
template <> constexpr float kLazy<__half> = 3.f;
template <class T> constexpr float kShift = Elem<T>::kTop - kLazy<T>;

template <int D>
struct GeoFew {
    static constexpr int kKeys = D == 128 ? 16 : 32;             // tokens of a chunk: 8 KB of keys and values
    static constexpr int kStages = 3;
    static constexpr int kHalf = kKeys * 128;                    // 64 coordinates of a chunk
    static constexpr int kTile = (D / 64) * kHalf;               // keys or values of a chunk
    static constexpr int kSmem = 1024 + kWarpsFew * kStages * 2 * kTile + 256 + kWarpsFew * 16 * 8;     // barriers, flags, maxima and sums
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

constexpr int kUnit = 64;                // tokens of a unit of work

// What the call does with sequence b, and the units of one of its heads (0: no new tokens, or more than max_new promised).
__device__ __forceinline__ Work few_work(const AttendArgs& a, int b, bool report) {
    Work w;
    w.b = b; w.begin = q_begin(a.batch, b); w.count = max(0, q_begin(a.batch, b + 1) - w.begin); w.t0 = 0;
    w.n = kv_length(a.batch, b, report);
    if (w.count > a.few_rows / a.group) {
        if (report) atomicOr(a.batch.status, kBadLength);
        w.count = 0;
    }
    return w;
}
__device__ __forceinline__ int few_first(const AttendArgs& a, const Work& w) { return see_lo(a, w, 0) / kUnit; }
__device__ __forceinline__ int few_units(const AttendArgs& a, const Work& w) {
    return w.count == 0 ? 0 : max(1, (see_hi(a, w, w.count - 1) + kUnit - 1) / kUnit - few_first(a, w));
}
// CTA c of `ctas` takes units [c U / ctas, (c + 1) U / ctas); the CTA that has unit u.  (No more CTAs than units: each has one, so those that share a cache follow
// each other.)
__device__ __forceinline__ int few_ctas(const AttendArgs& a, int64_t total) { return (int)min((int64_t)a.ctas, total); }
__device__ __forceinline__ int cta_of(int64_t u, int64_t total, int ctas) { return (int)(((u + 1) * ctas - 1) / total); }

template <class T, int D>
__global__ void __launch_bounds__(kWarpsFew * 32, 2)
k_few(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const AttendArgs a) {
    using G = GeoFew<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* base = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint64_t* bars = (uint64_t*)(base + kWarpsFew * G::kStages * 2 * G::kTile);
    int64_t* s_scan = (int64_t*)(bars + kWarpsFew * G::kStages);     // [warp] sums; [4] units before the first sequence
    int* flags = (int*)(s_scan + 5);                                 // abort, the latest cache with elements that are not finite, first sequence
    float* s_m = (float*)(flags + 4);                                // [warp][16] maxima, then [warp][16] sums
    float* s_l = s_m + kWarpsFew * 16;
    volatile int* abort_flag = flags;
    unsigned int* status = a.batch.status + 1;
    grid_wait();
    grid_go();

    const int warp = warp_index(), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kWarpsFew * G::kStages; ++i) mbar_init(&bars[i], 1);
        flags[0] = flags[1] = 0;
        flags[2] = -1;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // units of all sequences: every thread counts a stretch of them
    const int stretch = (a.batch.batch + kWarpsFew * 32 - 1) / (kWarpsFew * 32), b0 = min(a.batch.batch, (int)threadIdx.x * stretch), b1 = min(a.batch.batch, b0 + stretch);
    int64_t mine_units = 0;
    for (int b = b0; b < b1; ++b) mine_units += (int64_t)a.heads * few_units(a, few_work(a, b, blockIdx.x == 0));
    int64_t upto = mine_units;
    for (int o = 1; o < 32; o <<= 1) { const int64_t v = __shfl_up_sync(~0u, upto, o); if (lane >= o) upto += v; }
    if (lane == 31) s_scan[warp] = upto;
    __syncthreads();
    int64_t total = 0;
    for (int k = 0; k < kWarpsFew; ++k) { if (k < warp) upto += s_scan[k]; total += s_scan[k]; }
    const int ctas = few_ctas(a, total);
    const bool busy = (int)blockIdx.x < ctas;
    const int64_t u0 = busy ? blockIdx.x * total / ctas : 0, u1 = busy ? (blockIdx.x + 1) * total / ctas : 0;
    int64_t before = upto - mine_units;
    if (busy && u0 >= before && u0 < upto)
        for (int b = b0; b < b1; ++b) {
            const int64_t units = (int64_t)a.heads * few_units(a, few_work(a, b, false));
            if (u0 >= before && u0 < before + units) { flags[2] = b; s_scan[4] = before; }
            before += units;
        }
    __syncthreads();
    if (u0 >= u1) return;

    uint8_t* ring = base + warp * G::kStages * 2 * G::kTile;
    uint64_t* full = bars + warp * G::kStages;
    constexpr int KEYS = G::kKeys, NT = KEYS / 8;
    const int g = lane >> 2, t = lane & 3;
    const float c = a.scale_log2;
    // ldmatrix: matrix i = lane / 8, its row lane % 8; keys: matrices (token half i / 2, coordinate half i % 2); values, transposed: (token half i % 2, coordinate group i / 2)
    const int mi = lane >> 3, mr = lane & 7;
    const uint32_t krow = (uint32_t)(((mi >> 1) * 8 + mr) * 128), vrow = (uint32_t)(((mi & 1) * 8 + mr) * 128);
    const int boxes = KEYS / a.box_rows;                             // 1, 2 or 4 a chunk
    int done = 0, segment = 1;                                       // chunks this warp has been through; caches, the CTA
    bool ok = true;

    Work w = uniform(few_work(a, uniform(flags[2]), false));
    int64_t at_b = s_scan[4];                                        // first unit of sequence w.b
    for (int64_t u = u0; u < u1 && ok;) {
        const int units = uniform(few_units(a, w));
        if (units == 0 || u >= at_b + (int64_t)a.heads * units) {        // the next sequence
            at_b += (int64_t)a.heads * units;
            w = uniform(few_work(a, w.b + 1, false));
            continue;
        }
        const int h = uniform((int)((u - at_b) / units)), first = uniform((int)((u - at_b) % units)), last = uniform((int)min((int64_t)units, first + (u1 - u)));
        const int64_t seg = at_b + (int64_t)h * units;                   // this cache's units [seg, seg + units)
        const int b = w.b, rows = w.count * a.group;
        const int k0 = max(see_lo(a, w, 0), (few_first(a, w) + first) * kUnit), k1 = min(see_hi(a, w, w.count - 1), (few_first(a, w) + last) * kUnit);
        const int full0 = see_lo(a, w, w.count - 1), full1 = see_hi(a, w, 0);          // every row sees [full0, full1)
        const int c0 = k0 / KEYS, chunks = max(0, (k1 + KEYS - 1) / KEYS - c0);
        const int mine = chunks > warp ? (chunks - warp + kWarpsFew - 1) / kWarpsFew : 0;
        int page = 0;                                                    // of box 32 k + lane of this warp's boxes, all chunks in a row
        auto issue = [&](int i) {
            const int e = i * boxes;
            if ((e & 31) == 0) {
                const int ii = (e + lane) / boxes, key = (c0 + warp + kWarpsFew * ii) * KEYS + ((e + lane) % boxes) * a.box_rows;
                page = 0;
                if (ii < mine && key < w.n) {
                    page = a.batch.table[b * a.batch.table_stride + a.batch.page_of(key)];
                    if (page < 0 || page >= a.batch.num_pages) { page = a.batch.num_pages; atomicOr(a.batch.status, kBadPage); }   // (outside: TMA fills with zeros)
                }
            }
            const int at = __shfl_sync(~0u, page, (e + lane) & 31), st = (done + i) % G::kStages;
            const int key0 = (c0 + warp + kWarpsFew * i) * KEYS, key = key0 + lane * a.box_rows;
            const int live = min(boxes, (w.n - key0 + a.box_rows - 1) / a.box_rows);
            uint8_t* k = ring + st * 2 * G::kTile;
            if (lane == 0) mbar_expect_tx(&full[st], (uint32_t)(live * a.box_rows * D * 4));
            __syncwarp();
            if (lane < live) {
#pragma unroll
                for (int x = 0; x < D / 64; ++x) {
                    tma_load_4d(k + x * G::kHalf + lane * a.box_rows * 128, &map_k, x * 64, a.batch.row_of(key), h, at, &full[st]);
                    tma_load_4d(k + G::kTile + x * G::kHalf + lane * a.box_rows * 128, &map_v, x * 64, a.batch.row_of(key), h, at, &full[st]);
                }
            }
            __syncwarp();
        };
        for (int i = 0; i < G::kStages && i < mine; ++i) issue(i);

        // fragments: this thread's rows are g and g + 8, its columns 2 t, 2 t + 1 of every 8
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
            score_row[r] = a.scores && a.w_out && g + 8 * r < rows ? a.scores + (((int64_t)b * a.heads + h) * a.few_rows + g + 8 * r) * a.score_stride + 2 * t : nullptr;

        float o[D / 8][4];
#pragma unroll
        for (int n = 0; n < D / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][e] = 0.f;
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
        bool odd = false;

        // Accumulators that a warp has filled with kPartTokens tokens (mma.sync truncates as tcgen05 does) are added to fp32 sums in the workspace, with rounding and at
        // the maximum of the moment; each thread has its own.  first: nothing is there yet; last: the sums come back into the registers.
        auto fold = [&](bool first, bool last) {
            float4* f = (float4*)a.folds + ((int64_t)(blockIdx.x * kWarpsFew + warp) * (D / 8 + 1)) * 32 + lane;
            if (!first) {
                const float4 z = f[D / 8 * 32];
                const float fa[2] = {rescale(z.x, m[0], c, kShift<T>), rescale(z.y, m[1], c, kShift<T>)};
                l[0] = fmaf(fa[0], z.z, l[0]);
                l[1] = fmaf(fa[1], z.w, l[1]);
#pragma unroll
                for (int n = 0; n < D / 8; ++n) {
                    const float4 y = f[n * 32];
                    o[n][0] = fmaf(fa[0], y.x, o[n][0]); o[n][1] = fmaf(fa[0], y.y, o[n][1]);
                    o[n][2] = fmaf(fa[1], y.z, o[n][2]); o[n][3] = fmaf(fa[1], y.w, o[n][3]);
                }
            }
            if (last) return;
            f[D / 8 * 32] = make_float4(m[0], m[1], l[0], l[1]);
            l[0] = l[1] = 0.f;
#pragma unroll
            for (int n = 0; n < D / 8; ++n) {
                f[n * 32] = make_float4(o[n][0], o[n][1], o[n][2], o[n][3]);
                o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
            }
        };
        constexpr int kFold = kPartTokens / KEYS;

        int i = 0;
        for (; i < mine; ++i) {
            const int st = (done + i) % G::kStages, key = (c0 + warp + kWarpsFew * i) * KEYS;
            ok = __all_sync(~0u, mbar_wait(&full[st], ((done + i) / G::kStages) & 1, abort_flag, status, 41));
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
                raise |= !((top[r] - m[r]) * c <= kLazy<T>) && top[r] != m[r];
            }
            if (__any_sync(~0u, raise)) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    top[r] = max_nan(top[r], __shfl_xor_sync(~0u, top[r], 1));
                    top[r] = max_nan(top[r], __shfl_xor_sync(~0u, top[r], 2));
                    const float f = rescale(m[r], top[r], c, kShift<T>);
                    m[r] = top[r];
                    l[r] *= f;
#pragma unroll
                    for (int n = 0; n < D / 8; ++n) { o[n][2 * r] *= f; o[n][2 * r + 1] *= f; }
                }
            }
            uint32_t p[NT / 2][4];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float mc = held(m[r], c, kShift<T>);
                float sum = 0.f;                     // (of the chunk first: beside one large weight every addition loses up to half a step of it)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float e0 = ex2f(fmaf(s[n][2 * r], c, -mc)), e1 = ex2f(fmaf(s[n][2 * r + 1], c, -mc));
                    sum += e0 + e1;
                    p[n / 2][2 * (n % 2) + r] = Elem<T>::pack(e0, e1);
                }
                l[r] += sum;
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
            if ((i + 1) % kFold == 0 && i + 1 < mine && a.folds) fold(i + 1 == kFold, false);
        }
        if (ok && mine > kFold && a.folds) fold(false, true);
        if (!ok && lane == 0) {                      // aborted: copies in flight land before the CTA exits (bounded)
            for (int k = i; k < min(i + G::kStages, mine); ++k) {
                const long long t0 = clock64();
                while (!mbar_try_wait(&full[(done + k) % G::kStages], ((done + k) / G::kStages) & 1) && clock64() - t0 < 20000000ll) {}
            }
        }
        done += mine;
        if (odd) flags[1] = segment;
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
        const int cta0 = cta_of(seg, total, ctas), cta1 = cta_of(seg + units - 1, total, ctas);
        const int64_t slot = 2 * blockIdx.x + ((int)blockIdx.x == cta0 ? 1 : 0);       // a CTA shares its first cache and its last one
        if ((int)blockIdx.x == cta0 && threadIdx.x == 0) a.parts[(int64_t)b * a.heads + h] = make_int2(cta0, cta1 - cta0 + 1);
        const bool any_odd = *(volatile int*)&flags[1] == segment;
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
                    const float f = rescale(mk, top, c, kShift<T>);
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
                    const int page = a.batch.table[b * a.batch.table_stride + a.batch.page_of(key)];
                    if (page < 0 || page >= a.batch.num_pages) continue;
                    const int64_t from = page * a.v_page + a.batch.row_of(key) * a.v_token + h * a.v_head + d;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float y = Elem<T>::at(a.v_pool, from + e);
                        if (!isfinite(y)) v[e] += y;
                    }
                }
            }
            const float lse2 = top == -INFINITY ? -INFINITY : held(top, c, kShift<T>) + log2f(sum);
            if (cta0 != cta1) {
                // (zeros, where the row sees nothing of the part: the join multiplies every part's result by a factor, which is 0 there)
                if (d == 0) a.part_lse[slot * kFewRows + row] = lse2;
                *(float4*)(a.part_o + (slot * kFewRows + row) * D + d) = make_float4(v[0], v[1], v[2], v[3]);
            } else {
                *(uint2*)((T*)a.out.p + at * a.out.token_stride + head * a.out.head_stride + d) = make_uint2(Elem<T>::pack(v[0], v[1]), Elem<T>::pack(v[2], v[3]));
                if (d == 0 && a.lse) a.lse[at * a.q_heads + head] = lse2 == -INFINITY ? -INFINITY : (float)((double)lse2 * 0.69314718055994530942);
            }
        }
        u += last - first;
        ++segment;
        fence_async();                               // the ring goes back to TMA
        __syncthreads();
    }
}

// Joins the parts of the caches that several CTAs of k_few share: out = sum_p 2^(lse_p - lse) o_p, and turns the scores that k_few left into weights, w_j +=
// sum over the rows that see token j of 2^(score - lse).  The first `weigh` blocks, the same number to
// each (sequence, head), take 512 tokens at a time, four a thread (max_len may lie far above the lengths: no more blocks than keep the GPU busy); the others a
// row each, its parts shared by the warps.
constexpr int kJoinWarps = 4, kJoinThreads = 32 * kJoinWarps, kWeighTokens = 4 * kJoinThreads;

// The parts of a cache: the first CTA that has one and their number (written down by that CTA), and the slot of the p-th.
struct Parts {
    int cta0, count;
    __device__ __forceinline__ int64_t slot(int p) const { return p == 0 ? 2 * (int64_t)cta0 + 1 : 2 * ((int64_t)cta0 + p); }
};
__device__ __forceinline__ Parts few_parts(const AttendArgs& a, int b, int h) {
    // (held to what there is: a CTA that gave up in a bounded wait has written nothing)
    const int2 p = a.parts[(int64_t)b * a.heads + h];
    const int c0 = min(max(p.x, 0), a.ctas - 1);
    return Parts{c0, min(max(p.y, 1), a.ctas - c0)};
}

template <class T, int D>
__global__ void __launch_bounds__(kJoinThreads) k_few_join(const AttendArgs a, const int weigh) {
    __shared__ float s_lse[kFewRows];
    __shared__ int s_lo[kFewRows], s_hi[kFewRows];
    __shared__ float s_o[kJoinWarps][D];
    grid_wait();
    grid_go();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if ((int)blockIdx.x < weigh) {
        const int per = weigh / (a.heads * a.batch.batch), h = (blockIdx.x / per) % a.heads, first = (blockIdx.x % per) * kWeighTokens;
        const Work w = few_work(a, blockIdx.x / (per * a.heads), false);
        if (first >= w.n) return;
        const int rows = w.count * a.group;
        if (rows > 0) {
            const Parts parts = few_parts(a, w.b, h);
            for (int r = warp; r < rows; r += kJoinWarps) {      // a warp a row
                const int token = r / a.group;
                const int64_t at = (int64_t)(w.begin + token) * a.q_heads + h * a.group + r % a.group;
                float lse;
                if (parts.count > 1) {
                    float top = -INFINITY, sum = 0.f;
                    for (int p = lane; p < parts.count; p += 32) top = max_nan(top, a.part_lse[parts.slot(p) * kFewRows + r]);
                    for (int o = 16; o; o >>= 1) top = max_nan(top, __shfl_xor_sync(~0u, top, o));
                    for (int p = lane; p < parts.count; p += 32) sum += ex2f(a.part_lse[parts.slot(p) * kFewRows + r] - top);
                    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
                    lse = top == -INFINITY ? -INFINITY : top + log2f(sum);
                } else {
                    const float x = a.lse[at];
                    lse = x == -INFINITY ? x : (float)((double)x * 1.44269504088896340736);
                }
                if (lane == 0) { s_lse[r] = lse; s_lo[r] = see_lo(a, w, token); s_hi[r] = see_hi(a, w, token); }
            }
        }
        __syncthreads();
        for (int64_t key0 = first; key0 < w.n; key0 += (int64_t)per * kWeighTokens) {
            float sum[4];
            const int key1 = (int)key0 + threadIdx.x;
            const float* s = a.scores + ((int64_t)w.b * a.heads + h) * a.few_rows * a.score_stride + key1;
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[k] = 0.f;
            for (int r = 0; r < rows; ++r) {
                const float lse = s_lse[r];
                const int lo = s_lo[r], hi = s_hi[r];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int key = key1 + kJoinThreads * k;
                    if (key >= lo && key < hi) sum[k] += ex2f(s[r * a.score_stride + kJoinThreads * k] - lse);
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int key = key1 + kJoinThreads * k;
                if (key >= w.n) continue;
                const int64_t at = ((int64_t)w.b * a.heads + h) * a.w_stride + key;
                a.w_out[at] = (a.w_in ? a.w_in[at] : 0.f) + sum[k];
            }
        }
        return;
    }
    const int block = blockIdx.x - weigh, r = block % a.few_rows, h = block / a.few_rows % a.heads;
    const int b = block / (a.few_rows * a.heads), begin = q_begin(a.batch, b), count = max(0, q_begin(a.batch, b + 1) - begin);
    const Parts parts = few_parts(a, b, h);                      // (anything, where nothing is new)
    if (r >= count * a.group || count > a.few_rows / a.group || parts.count == 1) return;        // one part: written by its CTA
    constexpr int E = D / 32;
    float o[E], top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] = 0.f;
    for (int p = lane; p < parts.count; p += 32) top = max_nan(top, a.part_lse[parts.slot(p) * kFewRows + r]);
    for (int x = 16; x; x >>= 1) top = max_nan(top, __shfl_xor_sync(~0u, top, x));
    for (int p0 = 0; p0 < parts.count && top != -INFINITY; p0 += 32) {
        const float f = p0 + lane < parts.count ? ex2f(a.part_lse[parts.slot(p0 + lane) * kFewRows + r] - top) : 0.f;
        sum += f;
        const int n = min(32, parts.count - p0);
#pragma unroll 8
        for (int p = warp; p < n; p += kJoinWarps) {
            const float x = __shfl_sync(~0u, f, p);
            const float* q = a.part_o + (parts.slot(p0 + p) * kFewRows + r) * D + lane * E;
            if (E == 4) {
                const float4 v = *(const float4*)q;
                o[0] = fmaf(x, v.x, o[0]); o[1] = fmaf(x, v.y, o[1]); o[E - 2] = fmaf(x, v.z, o[E - 2]); o[E - 1] = fmaf(x, v.w, o[E - 1]);
            } else {
                const float2 v = *(const float2*)q;
                o[0] = fmaf(x, v.x, o[0]); o[1] = fmaf(x, v.y, o[1]);
            }
        }
    }
    for (int x = 16; x; x >>= 1) sum += __shfl_xor_sync(~0u, sum, x);
#pragma unroll
    for (int i = 0; i < E; ++i) s_o[warp][lane * E + i] = o[i];
    __syncthreads();
    if (warp) return;
#pragma unroll
    for (int k = 1; k < kJoinWarps; ++k)
#pragma unroll
        for (int i = 0; i < E; ++i) o[i] += s_o[k][lane * E + i];
    const int token = r / a.group, head = h * a.group + r % a.group;
    const int64_t at = begin + token;
    const float inv = top == -INFINITY ? 0.f : 1.0f / sum;
    uint32_t* dst = (uint32_t*)((T*)a.out.p + at * a.out.token_stride + head * a.out.head_stride + lane * E);
#pragma unroll
    for (int i = 0; i < E / 2; ++i) dst[i] = Elem<T>::pack(o[2 * i] * inv, o[2 * i + 1] * inv);
    if (a.lse && lane == 0) a.lse[at * a.q_heads + head] = top == -INFINITY ? -INFINITY : (float)((double)(top + log2f(sum)) * 0.69314718055994530942);
}

template <class T, int D>
cudaError_t few_t(const AttendArgs& a, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t stream) {
    cudaError_t e = allow_smem<k_few<T, D>>(GeoFew<D>::kSmem);
    if (e != cudaSuccess) return e;
    ++g_launches;
    if ((e = launch_behind(stream, dim3((unsigned)a.ctas), dim3(kWarpsFew * 32), GeoFew<D>::kSmem, k_few<T, D>, mk, mv, a)) != cudaSuccess) return e;
    const int64_t caches = (int64_t)a.batch.batch * a.heads, join = a.ctas > 1 ? caches * a.few_rows : 0;
    const int64_t per = a.w_out ? std::min<int64_t>(ceil_div(a.batch.max_len, kWeighTokens), std::max<int64_t>(1, ceil_div(16 * (int64_t)a.sm_count, caches))) : 0, weigh = per * caches;
    if (weigh + join > INT32_MAX) return cudaErrorInvalidConfiguration;
    if (weigh + join == 0) return cudaSuccess;
    ++g_launches;
    return launch_behind(stream, dim3((unsigned)(weigh + join)), dim3(kJoinThreads), 0, k_few_join<T, D>, a, (int)weigh);
}

}  // namespace

cudaError_t launch_few(const AttendArgs& a, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t stream) { return FD_KV_PICK(few_t, a, mk, mv, stream); }

}  // namespace kv
}  // namespace fd
