// Attention of new tokens over a paged cache, and its column sums, on tcgen05 / TMEM.
//
// k_attend.  One CTA takes two tiles of 128 rows (one, where no sequence has more: then two CTAs share an SM); a row is a (new token, query head of the group), so that all rows of a tile read the same cached
// head.  Per tile of 128 cached tokens:
//   S = Q K^T         (Q in shared memory, K by TMA page by page) into 128 fp32 columns of TMEM;
//   m, P = 2^(c S - c m)   one thread a row: the maximum over the tile, then exponentials, rounded to the element type and written back over S.
//                     The maximum in use is raised only when a row exceeds it by 2^8 (fp16: 2^5, see Elem): weights above 1 lose nothing in floating
//                     point, and the accumulator is read back and rescaled in the first tiles only;
//   O += P V          (P in TMEM, V row-major in shared memory as an MN-major operand) into D fp32 columns.
// While one tile's rows are exponentiated the tensor core works on the other's.  Rounding P to 16 bits changes a weight by half an ulp at
// most (fp16: or 2^-35 of the largest), independently per weight, which the operand of a tensor product costs; the norm sums the unrounded weights in fp32.
//
// Bounds: the tensor core (2 x 1024 clocks for two row tiles of 128 coordinates) and the MUFU (2 x 1024) could be busy all the time; what a pass takes is the chain
// of one row tile -- scores ready, 600 clocks to read them and find the maximum, 1430 for 128 exponentials of one warp, 950 until the product and the next
// scores are through -- about 3500 clocks while both row tiles take turns.  8192 new tokens over 16384: 1.60 ms, 1.03 PFLOP/s; without any exponentials 1.36
// ms (the power limit is near: a library product sustains 1.40 PFLOP/s).  Tried without gain: half a row a thread (16 warps, the maxima
// exchanged: the same 3880 clocks under the profiler), an eighth of the exponentials as polynomials on the FMA pipe (1.57), a quarter (1.70), weights handed over
// in one piece (1.64; in four pieces of 32 tokens the product starts on the first).
//
// Warps 0-3 / 4-7: softmax of row tile 0 / 1; 8: TMA; 9: MMA; 10, 11: values of tiles that some row sees only in part.  What a row does not see gets P = 0
// exactly, but 0 x inf = NaN: in those tiles rows behind the sequence are zeroed in shared memory, and so are elements that are not finite; the latter
// are added again at the end, row by row, to the rows that see them (never on finite data).
// Every wait is bounded; on expiry the CTA raises a status word, lets its copies and products end, frees TMEM and exits.
#include <algorithm>

#include "fd_kv_dev.h"

namespace fd {
namespace kv {
namespace {

using namespace tc;

__device__ __forceinline__ void tma_load_3d(void* smem_dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(smem_u32(smem_dst)), "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
          "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
// As mbar_wait, for hand-offs inside a tile: polls without backing off.
__device__ __forceinline__ bool mbar_wait_near(uint64_t* bar, uint32_t parity, volatile int* abort_flag, unsigned int* status, int code) {
    if (mbar_try_wait(bar, parity)) return true;
    const long long t0 = clock64();
    int spins = 0;
    while (!mbar_try_wait(bar, parity))
        if ((++spins & 255) == 0) {
            if (*abort_flag) return false;
            if (clock64() - t0 > kWaitCycles) {
                *abort_flag = 1;
                atomicCAS(status, 0u, (unsigned)(0x100 | code));
                return false;
            }
        }
    return true;
}
// Waits, bounded, for what a CTA that gives up has in flight.
__device__ __forceinline__ void land(uint64_t* bar, uint32_t parity) {
    const long long t0 = clock64();
    while (!mbar_try_wait(bar, parity) && clock64() - t0 < 20000000ll) {}
}
// (see Elem; 2 x 2048 fp16 tokens with weights: 605 us with 2^8, 608 with 2^6, 618 with 2^5, 631 with 2^4)
template <class T> constexpr float kLazy = 8.f;
template <> constexpr float kLazy<__half> = 5.f;
template <class T> constexpr float kShift = Elem<T>::kTop - kLazy<T>;
// Instruction descriptor, fp32 accumulation, M = 128; `mn`: the B operand is MN-major.
template <class T> constexpr uint32_t idesc_kv(int n, bool mn) {
    return (1u << 4) | (Elem<T>::kFormat << 7) | (Elem<T>::kFormat << 10) | ((mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}

template <int D>
struct Geo {
    static constexpr int kChunks = D / 64;                     // 128-byte columns of an operand tile
    static constexpr int kChunkBytes = 128 * 128;              // 128 rows of one
    static constexpr int kTile = kChunks * kChunkBytes;
};
// A CTA's row tiles: two, or one where no sequence has more rows and the cache's bytes count; then two CTAs an SM fill each other's waits (5 new tokens of 8 sequences of
// 6000 to 16384, 64 query heads on 8: 157 -> 116 us; 2 tokens of 24 sequences of 1400 to 4096, 64 coordinates: 59 -> 35 us).
template <int D, int TILES>
struct GeoAt {
    static constexpr int kSlots = TILES == 2 ? (D == 128 ? 5 : 8) : (D == 128 ? 2 : 4);        // ring of key and value tiles
    static constexpr int kSmem = 1024 + (TILES + kSlots) * Geo<D>::kTile + 512;
    static constexpr int kSoftWarps = 4 * TILES, kThreads = 32 * (kSoftWarps + 4), kCols = 256 * TILES;
    // Key and value tiles take turns in the ring; the j-th value tile is use number value_use(j) of its slot by values.
    static __device__ __forceinline__ int value_use(int j) { return j / (kSlots % 2 ? kSlots : kSlots / 2); }
};

template <int SLOTS>
struct Bars {
    uint64_t q_full, full[SLOTS], empty[SLOTS], clean[SLOTS];
    uint64_t s_full[2], p_full[2][4], pv_done[2], drained;
    uint32_t tmem_base;
    int abort_flag, odd;                                        // odd: elements that are not finite were taken out of a tile
};

// The slot-th group of `per` tokens of the batch, or b = -1.
__device__ __forceinline__ Work find_work(const Batch& B, int slot, int per) {
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int b0 = 0; b0 < B.batch; b0 += 32) {
        const int b = b0 + lane;
        int begin = 0, count = 0;
        if (b < B.batch) { begin = q_begin(B, b); count = max(0, q_begin(B, b + 1) - begin); }
        const int tiles = (count + per - 1) / per;
        int upto = tiles;
        for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(~0u, upto, o); if (lane >= o) upto += v; }
        const unsigned hit = __ballot_sync(~0u, slot < before + upto);
        if (hit) {
            const int l = __ffs(hit) - 1;
            Work w;
            w.b = b0 + l;
            w.begin = __shfl_sync(~0u, begin, l);
            w.count = __shfl_sync(~0u, count, l);
            w.t0 = (slot - before - __shfl_sync(~0u, upto - tiles, l)) * per;
            w.n = kv_length(B, w.b, lane == 0);
            return w;
        }
        before += __shfl_sync(~0u, upto, 31);
    }
    return Work{-1, 0, 0, 0, 0};
}
// Bits [lo, hi) of a 32-column group that begins at column c.
__device__ __forceinline__ uint32_t col_mask(int lo, int hi, int c) {
    const int l = min(max(lo - c, 0), 32), h = min(max(hi - c, 0), 32);
    const uint32_t up = h >= 32 ? 0xffffffffu : (1u << h) - 1, down = l >= 32 ? 0xffffffffu : (1u << l) - 1;
    return up & ~down;
}

// Loads 128 tokens of the cache from `tile` on into a ring slot; rows behind the sequence stay as they are.  One warp, converged.
template <int D>
__device__ __forceinline__ void load_tile(uint8_t* dst, const CUtensorMap* map, const AttendArgs& a, const Work& w, int tile, int h, uint64_t* bar) {
    const int lane = threadIdx.x & 31, boxes = 128 / a.box_rows;
    const int key = tile * 128 + lane * a.box_rows;
    const bool mine = lane < boxes && key < w.n;
    int page = 0;
    if (mine) {
        page = a.batch.table[w.b * a.batch.table_stride + a.batch.page_of(key)];
        if (page < 0 || page >= a.batch.num_pages) { page = a.batch.num_pages; atomicOr(a.batch.status, kBadPage); }   // (outside: TMA fills with zeros)
    }
    const int total = __popc(__ballot_sync(~0u, mine));
    if (lane == 0) mbar_expect_tx(bar, total * a.box_rows * D * 2);
    __syncwarp();
    if (mine)
#pragma unroll
        for (int c = 0; c < Geo<D>::kChunks; ++c)
            tma_load_4d(dst + c * Geo<D>::kChunkBytes + lane * a.box_rows * 128, map, c * 64, a.batch.row_of(key), h, page, bar);
    __syncwarp();
}

template <class T, int D, int TILES>
__global__ void __launch_bounds__(GeoAt<D, TILES>::kThreads, TILES == 2 ? 1 : 2)
k_attend(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
         const AttendArgs a) {
    using G = Geo<D>;
    using A = GeoAt<D, TILES>;
    constexpr int kSoftWarps = A::kSoftWarps;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* base = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* q_base = base;
    uint8_t* ring = base + TILES * G::kTile;
    Bars<A::kSlots>* bars = (Bars<A::kSlots>*)(ring + A::kSlots * G::kTile);
    volatile int* abort_flag = &bars->abort_flag;
    unsigned int* status = a.batch.status + 1;

    grid_wait();
    grid_go();
    // work items: split fastest, then head, then token group, the last groups (which see most) first
    const int split = blockIdx.x % a.splits, h = (blockIdx.x / a.splits) % a.heads;
    const int groups = gridDim.x / (a.splits * a.heads), slot = groups - 1 - blockIdx.x / (a.splits * a.heads);
    const int per = TILES * a.tile_tokens;
    const Work w = uniform(find_work(a.batch, slot, per));
    if (w.b < 0) return;
    const int t_last = min(w.count, w.t0 + per) - 1;
    const int tiles = (t_last - w.t0) / a.tile_tokens + 1;               // row tiles with work
    int j0 = see_lo(a, w, w.t0) / 128, j1 = (see_hi(a, w, t_last) + 127) / 128;
    if (a.splits > 1) { j0 = max(j0, split * a.split_tiles); j1 = min(j1, (split + 1) * a.split_tiles); }
    const int num = max(0, j1 - j0);
    // tiles [full0, full1) are seen whole by every row
    const int full0 = (see_lo(a, w, t_last) + 127) / 128, full1 = see_hi(a, w, w.t0) / 128;

    const int warp = warp_index(), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        mbar_init(&bars->q_full, 1); mbar_init(&bars->drained, 1);
        for (int s = 0; s < A::kSlots; ++s) { mbar_init(&bars->full[s], 1); mbar_init(&bars->empty[s], 1); mbar_init(&bars->clean[s], 2); }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&bars->s_full[t], 1); mbar_init(&bars->pv_done[t], 1);
            for (int k = 0; k < 4; ++k) mbar_init(&bars->p_full[t][k], 4);
        }
        bars->abort_flag = 0; bars->odd = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kSoftWarps) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem_base)), "r"(A::kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;

    int issued = 0;                                                      // tiles of the ring that this warp has asked for
    if (warp >= kSoftWarps) {
        if (warp == kSoftWarps && num > 0) {
            // ---------------------------------------------------------------- TMA
            const int rows = a.tile_tokens * a.group;
            if (lane == 0) {
                mbar_expect_tx(&bars->q_full, tiles * rows * D * 2);
                for (int t = 0; t < tiles; ++t)
                    for (int c = 0; c < G::kChunks; ++c)
                        tma_load_3d(q_base + t * G::kTile + c * G::kChunkBytes, &map_q, c * 64, h * a.group, w.begin + w.t0 + t * a.tile_tokens, &bars->q_full);
            }
            __syncwarp();
            bool ok = true;
            int it = 0;
            for (; it < 2 * num; ++it) {
                const int s = it % A::kSlots;
                ok = mbar_wait(&bars->empty[s], ((it / A::kSlots) & 1) ^ 1, abort_flag, status, 1);
                ok = __all_sync(~0u, ok);
                if (!ok) break;
                load_tile<D>(ring + s * G::kTile, (it & 1) ? &map_v : &map_k, a, w, j0 + it / 2, h, &bars->full[s]);
            }
            issued = it;
        } else if (warp == kSoftWarps + 1 && num > 0) {
            // ---------------------------------------------------------------- MMA (one thread)
            if (elect_one()) {
                constexpr uint32_t id_s = idesc_kv<T>(128, false), id_o = idesc_kv<T>(D, true);
                const uint64_t qd = smem_desc(smem_u32(q_base), 1024, 2);
                const uint64_t kd = smem_desc(smem_u32(ring), 1024, 2);
                // values: rows of 64 coordinates are the MN direction (next 64: one chunk on), 8 tokens to the next 1024 bytes
                const uint64_t vd = kd | ((uint64_t)(G::kChunkBytes >> 4) << 16);
                const uint32_t q_lo = (uint32_t)qd, k_lo = (uint32_t)kd, v_lo = (uint32_t)vd, hi = (uint32_t)(kd >> 32);
                auto scores = [&](int t, int slot_k) {
                    const uint32_t s_addr = tmem + 128u * t, qt = q_lo + (uint32_t)(t * G::kTile >> 4), kt = k_lo + (uint32_t)(slot_k * G::kTile >> 4);
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t o = (uint32_t)((k / 4) * (G::kChunkBytes >> 4) + (k % 4) * 2);
                        if (k == 0) mma_ss2<0>(s_addr, qt + o, hi, kt + o, hi, id_s);
                        else mma_ss2<1>(s_addr, qt + o, hi, kt + o, hi, id_s);
                    }
                    tc_commit(&bars->s_full[t]);
                };
                bool ok = mbar_wait(&bars->q_full, 0, abort_flag, status, 2) && mbar_wait(&bars->full[0], 0, abort_flag, status, 3);
                if (ok) {
                    tc_fence_after();
                    for (int t = 0; t < tiles; ++t) scores(t, 0);
                    tc_commit(&bars->empty[0]);
                }
                for (int j = 0; j < num && ok; ++j) {
                    const int iv = 2 * j + 1, sv = iv % A::kSlots, ik = 2 * j + 2, sk = ik % A::kSlots;
                    ok = mbar_wait(&bars->full[sv], (iv / A::kSlots) & 1, abort_flag, status, 4) &&
                         mbar_wait(&bars->clean[sv], A::value_use(j) & 1, abort_flag, status, 5);
                    for (int t = 0; t < tiles && ok; ++t) {
                        const uint32_t o_addr = tmem + 128u * TILES + (uint32_t)D * t, p_addr = tmem + 128u * t, vt = v_lo + (uint32_t)(sv * G::kTile >> 4);
#pragma unroll
                        for (int part = 0; part < 4; ++part) {                  // 32 tokens each
                            ok = mbar_wait_near(&bars->p_full[t][part], j & 1, abort_flag, status, 6);
                            if (!ok) break;
                            tc_fence_after();
#pragma unroll
                            for (int k = 2 * part; k < 2 * part + 2; ++k) {
                                if (k == 0 && j == 0) mma_ts2<0>(o_addr, p_addr, vt, hi, id_o);
                                else mma_ts2<1>(o_addr, p_addr + 32 * part + 8 * (k & 1), vt + (uint32_t)(k * 2048 >> 4), hi, id_o);
                            }
                        }
                        if (!ok) break;
                        tc_commit(&bars->pv_done[t]);
                        if (j + 1 < num) {
                            if (t == 0) {
                                ok = mbar_wait(&bars->full[sk], (ik / A::kSlots) & 1, abort_flag, status, 7);
                                if (!ok) break;
                                tc_fence_after();
                            }
                            scores(t, sk);
                        }
                    }
                    if (!ok) break;
                    tc_commit(&bars->empty[sv]);
                    if (j + 1 < num) tc_commit(&bars->empty[sk]);
                }
            }
        } else if (num > 0) {
            // ---------------------------------------------------------------- values that some row does not see
            bool ok = true;
            for (int j = 0; j < num; ++j) {
                const int iv = 2 * j + 1, sv = iv % A::kSlots, tile = j0 + j;
                ok = __all_sync(~0u, mbar_wait(&bars->full[sv], (iv / A::kSlots) & 1, abort_flag, status, 8));
                if (!ok) break;
                if (tile < full0 || tile >= full1) {
                    uint8_t* v = ring + sv * G::kTile;
                    bool odd = false;
                    for (int i = threadIdx.x - 32 * (kSoftWarps + 2); i < G::kTile / 16; i += 64) {       // 16 bytes of row (i / 8) % 128; the swizzle stays within the row
                        uint4* p = (uint4*)(v + 16 * i);
                        if (tile * 128 + (i / 8) % 128 >= w.n) { *p = make_uint4(0, 0, 0, 0); continue; }
                        uint4 x = *p;
                        uint32_t* e = &x.x;
                        bool hit = false;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            constexpr uint32_t E = Elem<T>::kExponent;
                            if ((e[k] & E) == E) { e[k] &= 0xffff0000u; hit = true; }
                            if ((e[k] & (E << 16)) == (E << 16)) { e[k] &= 0xffffu; hit = true; }
                        }
                        if (hit) { *p = x; odd = true; }
                    }
                    if (odd) bars->odd = 1;
                    fence_async();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars->clean[sv]);
            }
        }
    } else {
        // -------------------------------------------------------------------- softmax (thread = row)
        const int t = warp >> 2, q = warp & 3, r = q * 32 + lane;
        const uint32_t lane_addr = (uint32_t)(q * 32) << 16;
        const uint32_t s_addr = tmem + lane_addr + 128u * t, o_addr = tmem + lane_addr + 128u * TILES + (uint32_t)D * t;
        const int token = w.t0 + t * a.tile_tokens + r / a.group, head = h * a.group + r % a.group;
        const bool valid = r < a.tile_tokens * a.group && token < w.count;
        const bool warp_on = __any_sync(~0u, valid);                     // warps without rows only keep the hand-offs going
        const int lo = see_lo(a, w, token), hi = valid ? see_hi(a, w, token) : 0;
        const float c = a.scale_log2;
        float m = -INFINITY, l = 0.f;
        bool ok = true;
        if (t < tiles) {
            for (int j = 0; j < num; ++j) {
                const int tile = j0 + j;
                ok = __all_sync(~0u, mbar_wait_near(&bars->s_full[t], j & 1, abort_flag, status, 9));
                if (!ok) break;
                if (!warp_on) {
                    if (lane < 4) mbar_arrive(&bars->p_full[t][lane]);
                    continue;
                }
                tc_fence_after();
                // One row tile: two CTAs share the registers, so the scores are read twice, 32 tokens at a time; two row tiles: once (read twice they take 2.5 % longer).
                constexpr bool kHold = TILES == 2;
                uint32_t s[kHold ? 4 : 2][32];
                float mx[4];
                const bool whole = tile >= full0 && tile < full1;
                auto hide = [&](int k, uint32_t (&x)[32]) {              // what the row does not see
                    if (whole) return;
                    const uint32_t see = col_mask(lo, hi, tile * 128 + 32 * k);
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (!((see >> i) & 1)) x[i] = 0xff800000u;
                };
                tmem_ld32(s_addr, s[0]);
                if (kHold) {
                    tmem_ld32(s_addr + 32, s[1]);
                    tmem_wait_ld();
                    tmem_ld32(s_addr + 64, s[kHold ? 2 : 0]);
                    tmem_ld32(s_addr + 96, s[kHold ? 3 : 0]);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint32_t (&x)[32] = s[kHold ? k : k % 2];
                    if (kHold && k == 2) tmem_wait_ld();
                    if (!kHold) {
                        tmem_wait_ld();
                        if (k < 3) tmem_ld32(s_addr + 32 * (k + 1), s[(k + 1) % 2]);
                    }
                    hide(k, x);
                    float y[2];
#pragma unroll
                    for (int z = 0; z < 2; ++z) {
                        y[z] = max_nan(__uint_as_float(x[16 * z]), __uint_as_float(x[16 * z + 1]));
#pragma unroll
                        for (int i = 2; i < 16; i += 2) y[z] = max_nan(y[z], __uint_as_float(x[16 * z + i]), __uint_as_float(x[16 * z + i + 1]));
                    }
                    mx[k] = max_nan(y[0], y[1]);
                }
                const float top = max_nan(max_nan(mx[0], mx[1], mx[2]), mx[3], m);
                const bool raise = !((top - m) * c <= kLazy<T>) && top != m;        // (first tile: from -inf; a NaN goes through)
                if (__any_sync(~0u, raise)) {
                    const float alpha = raise ? rescale(m, top, c, kShift<T>) : 1.0f;
                    if (raise) m = top;
                    l *= alpha;
                    if (j > 0) {
                        if (!__all_sync(~0u, mbar_wait_near(&bars->pv_done[t], (j - 1) & 1, abort_flag, status, 10))) { ok = false; break; }
                        tc_fence_after();
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            uint32_t o[16];
                            tmem_ld16(o_addr + 16 * k, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                            tmem_st16(o_addr + 16 * k, o);
                        }
                        tmem_wait_st();
                    }
                }
                const float mc = held(m, c, kShift<T>);
                const uint64_t cc = pair2(c, c), mm = pair2(-mc, -mc);
                uint64_t sum[2] = {0, 0};
                if (!kHold) tmem_ld32(s_addr, s[0]);
                // 32 tokens at a time: the store of one part completes while the next part's exponentials are taken, then the product may have it
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint32_t (&sk)[32] = s[kHold ? k : k % 2];
                    if (!kHold) {
                        tmem_wait_ld();
                        if (k < 3) tmem_ld32(s_addr + 32 * (k + 1), s[(k + 1) % 2]);
                        hide(k, sk);
                    }
                    uint32_t p[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const uint64_t x = fma2(pair2(__uint_as_float(sk[2 * i]), __uint_as_float(sk[2 * i + 1])), cc, mm);
                        const uint64_t e = ex2_mufu(x);
                        sum[i & 1] = add2(sum[i & 1], e);
                        const float2 v = split2(e);
                        p[i] = Elem<T>::pack(v.x, v.y);
                    }
                    if (k > 0) {
                        tmem_wait_st();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&bars->p_full[t][k - 1]);
                    }
                    tmem_st16(s_addr + 32 * k, p);
                }
                const float2 part = split2(add2(sum[0], sum[1]));
                l += part.x + part.y;
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars->p_full[t][3]);
            }
            if (ok && num > 0) ok = __all_sync(~0u, mbar_wait(&bars->pv_done[t], (num - 1) & 1, abort_flag, status, 11));
        }
        if (ok && t < tiles && warp_on) {
            tc_fence_after();
            const bool empty = m == -INFINITY;
            // (the tensor core adds with truncation: see kPartTokens)
            const float inv = empty ? 0.f : 1.0f / l;
            const int64_t row = w.begin + token;
            const bool odd = num > 0 && *(volatile int*)&bars->odd;
            if (valid) {
                if (a.splits > 1) a.part_lse[(split * (int64_t)a.batch.total_q + row) * a.q_heads + head] = empty ? -INFINITY : held(m, c, kShift<T>) + log2f(l);
                else if (a.lse) a.lse[row * a.q_heads + head] = empty ? -INFINITY : (float)((double)(held(m, c, kShift<T>) + log2f(l)) * 0.69314718055994530942);
            }
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const int d0 = 16 * k;
                uint32_t u[16];
                float o[16];
                if (num > 0) { tmem_ld16(o_addr + d0, u); tmem_wait_ld(); }
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = empty ? 0.f : __uint_as_float(u[i]) * inv;
                if (odd && valid) {
                    // what is not finite in tiles that this CTA's rows see in part, for the rows that see it
                    for (int key = max(lo, j0 * 128); key < min(hi, j1 * 128); ++key) {
                        if (key / 128 >= full0 && key / 128 < full1) { key = full1 * 128 - 1; continue; }
                        const int page = a.batch.table[w.b * a.batch.table_stride + a.batch.page_of(key)];
                        if (page < 0 || page >= a.batch.num_pages) continue;
                        const int64_t at = page * a.v_page + a.batch.row_of(key) * a.v_token + h * a.v_head + d0;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float v = Elem<T>::at(a.v_pool, at + i);
                            if (!isfinite(v)) o[i] += v;
                        }
                    }
                }
                if (valid) {
                    if (a.splits > 1) {
                        float4* dst = (float4*)(a.part_o + ((split * (int64_t)a.batch.total_q + row) * a.q_heads + head) * D + d0);
#pragma unroll
                        for (int i = 0; i < 4; ++i) dst[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                    } else {
                        uint4* dst = (uint4*)((T*)a.out.p + row * a.out.token_stride + head * a.out.head_stride + d0);
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            dst[i] = make_uint4(Elem<T>::pack(o[8 * i], o[8 * i + 1]), Elem<T>::pack(o[8 * i + 2], o[8 * i + 3]),
                                                Elem<T>::pack(o[8 * i + 4], o[8 * i + 5]), Elem<T>::pack(o[8 * i + 6], o[8 * i + 7]));
                    }
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {                                                   // whoever gave up: copies and products in flight end before the CTA does
        if (warp == kSoftWarps && num > 0 && lane == 0) {
            for (int k = max(0, issued - A::kSlots); k < issued; ++k) land(&bars->full[k % A::kSlots], (k / A::kSlots) & 1);
            land(&bars->q_full, 0);
        }
        if (warp == kSoftWarps + 1 && elect_one()) { tc_commit(&bars->drained); land(&bars->drained, 0); }
        __syncthreads();
    }
    if (warp == kSoftWarps) {
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(A::kCols) : "memory");
    }
}

// Joins the parts of the cache: out = sum_s 2^(lse_s - lse) o_s.  Few parts: a warp a row; many: the eight warps of a block share the parts of one
// row (147 parts of 56 rows: a warp a row took 70 us, one wait for memory after the other).  The parts' factors are made in parallel first.
template <class T, int D, int W>
__global__ void __launch_bounds__(256) k_join(const AttendArgs a) {
    constexpr int E = D / 32;
    __shared__ float s_f[W == 1 ? 8 * 32 : kMaxSplits];
    __shared__ float s_o[W == 1 ? 1 : 8 * D], s_top[8], s_sum[8];
    grid_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, me = W == 1 ? lane : (int)threadIdx.x;
    const int64_t row = W == 1 ? (int64_t)blockIdx.x * 8 + warp : blockIdx.x;
    const int64_t rows = (int64_t)q_begin(a.batch, a.batch.batch) * a.q_heads, all = (int64_t)a.batch.total_q * a.q_heads;
    if (row >= rows || row < (int64_t)q_begin(a.batch, 0) * a.q_heads) return;             // (of no sequence)
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

// k_weigh: what every cached token received, w_j += sum over rows of 2^(c s - lse).  One CTA takes a tile of 128 cached tokens as the M side (S^T = K Q^T: a thread
// owns a token, so the sum over rows is a sum over its columns and needs no exchange) and goes through the rows that see them, 128 at a
// time; two warpgroups share the columns.  The exponentials bound it.  Two CTAs an SM fill each other's waits and even out the lengths: with
// one CTA of two tiles 2 x 2048 new tokens over 8192 and 4900 took 365 us.
constexpr int kWeighWarps = 8, kThreadsWe = 32 * (kWeighWarps + 3), kWeighCols = 256;
template <int D>
struct GeoWeigh {
    static constexpr int kSlots = D == 128 ? 2 : 4;               // ring of row tiles
    static constexpr int kSmem = 1024 + (1 + kSlots) * Geo<D>::kTile + 4 * 128 * 4 + 128 * 4 + 512;
};
template <int D>
struct WeighBars {
    uint64_t k_full, full[GeoWeigh<D>::kSlots], empty[GeoWeigh<D>::kSlots], s_full[2], s_empty[2], l_full[4], drained;
    uint32_t tmem_base;
    int abort_flag;
};

template <class T, int D>
__global__ void __launch_bounds__(kThreadsWe, 2)
k_weigh(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const AttendArgs a) {
    using G = Geo<D>;
    constexpr int kSlots = GeoWeigh<D>::kSlots;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* base = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* k_base = base;
    uint8_t* ring = base + G::kTile;
    float* l_ring = (float*)(ring + kSlots * G::kTile);                       // [4][128]: -lse of a row tile, -inf for rows that are none
    float* s_acc = l_ring + 4 * 128;                                          // [token]: sums of the second column halves
    WeighBars<D>* bars = (WeighBars<D>*)(s_acc + 128);
    volatile int* abort_flag = &bars->abort_flag;
    unsigned int* status = a.batch.status + 1;

    grid_wait();
    grid_go();
    const int h = blockIdx.y, b = blockIdx.z, key0 = blockIdx.x * 128;
    Work w;
    w.b = b; w.begin = q_begin(a.batch, b); w.count = max(0, q_begin(a.batch, b + 1) - w.begin); w.n = kv_length(a.batch, b, false); w.t0 = 0;
    w = uniform(w);
    if (key0 >= w.n) return;
    const int key_last = min(w.n, key0 + 128) - 1, off = w.n - w.count;
    // tokens that see one of these slots: [ta, tb)
    const int ta = a.causal ? max(0, key0 - off) : 0, tb = a.window ? (int)min((int64_t)w.count, max((int64_t)0, (int64_t)key_last - off + a.window)) : w.count;
    const int q0 = ta / a.tile_tokens, num = tb > ta ? (tb - 1) / a.tile_tokens + 1 - q0 : 0;
    const int rows = a.tile_tokens * a.group;

    const int warp = warp_index(), lane = threadIdx.x & 31;
    const int key = key0 + (warp & 3) * 32 + lane;                            // of the first 8 warps
    float acc = 0.f;
    if (threadIdx.x == 0) {
        mbar_init(&bars->k_full, 1); mbar_init(&bars->drained, 1);
        for (int s = 0; s < kSlots; ++s) { mbar_init(&bars->full[s], 1); mbar_init(&bars->empty[s], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&bars->s_full[i], 1); mbar_init(&bars->s_empty[i], kWeighWarps); }
        for (int i = 0; i < 4; ++i) mbar_init(&bars->l_full[i], 1);
        bars->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kWeighWarps) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem_base)), "r"(kWeighCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;

    int issued = 0;                                                           // row tiles that this thread has asked for
    if (warp == kWeighWarps && num > 0) {
        // -------------------------------------------------------------------- TMA
        load_tile<D>(k_base, &map_k, a, w, blockIdx.x, h, &bars->k_full);
        if (lane == 0) {
            bool ok = true;
            int it = 0;
            for (; it < num && ok; ++it) {
                const int s = it % kSlots;
                ok = mbar_wait(&bars->empty[s], ((it / kSlots) & 1) ^ 1, abort_flag, status, 21);
                if (!ok) break;
                mbar_expect_tx(&bars->full[s], rows * D * 2);
                for (int c = 0; c < G::kChunks; ++c)
                    tma_load_3d(ring + s * G::kTile + c * G::kChunkBytes, &map_q, c * 64, h * a.group, w.begin + (q0 + it) * a.tile_tokens, &bars->full[s]);
            }
            issued = it;
        }
    } else if (warp == kWeighWarps + 1 && num > 0) {
        // -------------------------------------------------------------------- MMA (one thread)
        if (elect_one()) {
            constexpr uint32_t id = idesc_kv<T>(128, false);
            const uint64_t kd = smem_desc(smem_u32(k_base), 1024, 2), qd = smem_desc(smem_u32(ring), 1024, 2);
            const uint32_t k_lo = (uint32_t)kd, q_lo = (uint32_t)qd, hi = (uint32_t)(kd >> 32);
            bool ok = mbar_wait(&bars->k_full, 0, abort_flag, status, 22);
            for (int i = 0; i < num && ok; ++i) {
                const int s = i % kSlots, buf = i & 1;
                ok = mbar_wait_near(&bars->full[s], (i / kSlots) & 1, abort_flag, status, 23) &&
                     mbar_wait_near(&bars->s_empty[buf], ((i >> 1) & 1) ^ 1, abort_flag, status, 24);
                if (!ok) break;
                tc_fence_after();
                const uint32_t s_addr = tmem + 128u * buf, qt = q_lo + (uint32_t)(s * G::kTile >> 4);
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint32_t o = (uint32_t)((k / 4) * (G::kChunkBytes >> 4) + (k % 4) * 2);
                    if (k == 0) mma_ss2<0>(s_addr, k_lo + o, hi, qt + o, hi, id);
                    else mma_ss2<1>(s_addr, k_lo + o, hi, qt + o, hi, id);
                }
                tc_commit(&bars->s_full[buf]);
                tc_commit(&bars->empty[s]);
            }
        }
    } else if (warp == kWeighWarps + 2 && num > 0) {
        // -------------------------------------------------------------------- -lse of each row tile, in powers of two
        // (This warp has to keep up with a tile of exponentials: places are worked out once, and the next tile's values are under way while this tile's wait.)
        constexpr float kHi = 1.44269502f, kLo = 1.92596303e-8f;               // log2(e)
        int token[4], at[4];
        float next[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int r = lane + 32 * k;
            token[k] = r < rows ? q0 * a.tile_tokens + r / a.group : 1 << 30;
            at[k] = r / a.group * a.q_heads + r % a.group;
        }
        const float* lse = a.lse + (int64_t)(w.begin + q0 * a.tile_tokens) * a.q_heads + h * a.group;
        auto fetch = [&](int i) {
            const float* l = lse + (int64_t)i * a.tile_tokens * a.q_heads;
#pragma unroll
            for (int k = 0; k < 4; ++k) next[k] = token[k] < w.count - i * a.tile_tokens ? l[at[k]] : -INFINITY;
        };
        fetch(0);
        bool ok = true;
        for (int i = 0; i < num; ++i) {
            float v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = next[k] == -INFINITY ? -INFINITY : -fmaf(next[k], kHi, next[k] * kLo);
            fetch(i + 1);                                                       // (behind the last: no row is valid, nothing is read)
            // Slot i % 4 may be written once tile i - 4 has been read.  Score buffers are handed back before the values of their slot are read, so tile i - 4 is surely done
            // when the buffer of tile i - 2 comes back, the latest that can have happened by now.
            if (i >= 2) ok = __all_sync(~0u, mbar_wait_near(&bars->s_empty[i & 1], ((i >> 1) & 1) ^ 1, abort_flag, status, 25));
            if (!ok) break;
#pragma unroll
            for (int k = 0; k < 4; ++k) l_ring[(i & 3) * 128 + lane + 32 * k] = v[k];
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->l_full[i & 3]);
        }
    } else if (warp < kWeighWarps) {
        // -------------------------------------------------------------------- a thread owns a token and half of the rows
        const int half = warp >> 2;
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        const uint64_t cc = pair2(a.scale_log2, a.scale_log2);
        bool ok = true;
        for (int i = 0; i < num; ++i) {
            const int buf = i & 1, tok0 = (q0 + i) * a.tile_tokens;
            ok = __all_sync(~0u, mbar_wait_near(&bars->l_full[i & 3], (i >> 2) & 1, abort_flag, status, 26) &&
                                 mbar_wait_near(&bars->s_full[buf], (i >> 1) & 1, abort_flag, status, 27));
            if (!ok) break;
            tc_fence_after();
            const uint32_t addr = tmem + lane_addr + 128u * buf + 64u * half;
            const float* lr = l_ring + (i & 3) * 128 + 64 * half;
            // columns of rows that see this token: [cl, ch)
            const int valid = min(rows, (w.count - tok0) * a.group);
            int cl = 0, ch = valid;
            if (a.causal) cl = max(0, key - off - tok0) * a.group;
            if (a.window) ch = (int)min((int64_t)valid, max((int64_t)0, (int64_t)key - off + a.window - tok0) * a.group);
            const bool whole = __all_sync(~0u, cl == 0 && ch >= 128);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                uint32_t s[32];
                tmem_ld32(addr + 32 * k, s);
                tmem_wait_ld();
                if (k == 1) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars->s_empty[buf]);
                }
                if (whole) {
                    uint64_t sum[2] = {0, 0};
#pragma unroll
                    for (int x = 0; x < 32; x += 4) {
                        const float4 lv = *(const float4*)(lr + 32 * k + x);
                        sum[0] = add2(sum[0], ex2_mufu(fma2(pair2(__uint_as_float(s[x]), __uint_as_float(s[x + 1])), cc, pair2(lv.x, lv.y))));
                        sum[1] = add2(sum[1], ex2_mufu(fma2(pair2(__uint_as_float(s[x + 2]), __uint_as_float(s[x + 3])), cc, pair2(lv.z, lv.w))));
                    }
                    const float2 p = split2(add2(sum[0], sum[1]));
                    acc += p.x + p.y;
                } else if (64 * half + 32 * k < valid) {
                    const uint32_t see = col_mask(cl, ch, 64 * half + 32 * k);
                    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int x = 0; x < 32; ++x) {
                        const float p = ex2f(fmaf(__uint_as_float(s[x]), a.scale_log2, lr[32 * k + x]));
                        sum[x & 3] += (see >> x) & 1 ? p : 0.f;
                    }
                    acc += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                }
            }
        }
        if (half) s_acc[(warp & 3) * 32 + lane] = acc;
    }
    tc_fence_before();
    __syncthreads();
    if (warp < 4 && key < w.n && !*abort_flag) {
        const int64_t at = ((int64_t)b * a.heads + h) * a.w_stride + key;
        a.w_out[at] = (a.w_in ? a.w_in[at] : 0.f) + (acc + s_acc[key - key0]);
    }
    if (*abort_flag) {                                                        // as in k_attend
        if (warp == kWeighWarps && num > 0 && lane == 0) {
            for (int k = max(0, issued - kSlots); k < issued; ++k) land(&bars->full[k % kSlots], (k / kSlots) & 1);
            land(&bars->k_full, 0);
        }
        if (warp == kWeighWarps + 1 && elect_one()) { tc_commit(&bars->drained); land(&bars->drained, 0); }
        __syncthreads();
    }
    if (warp == kWeighWarps) {
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kWeighCols) : "memory");
    }
}

template <class T, int D, int TILES>
cudaError_t launch_tiles(const AttendArgs& a, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t stream) {
    using A = GeoAt<D, TILES>;
    const cudaError_t e = allow_smem<k_attend<T, D, TILES>>(A::kSmem);
    if (e != cudaSuccess) return e;
    const int64_t groups = a.batch.total_q / (TILES * a.tile_tokens) + std::min(a.batch.batch, a.batch.total_q);
    if (groups * a.heads > INT32_MAX / a.splits) return cudaErrorInvalidConfiguration;
    ++g_launches;
    return launch_behind(stream, dim3((unsigned)(groups * a.heads * a.splits)), dim3(A::kThreads), A::kSmem, k_attend<T, D, TILES>, mq, mk, mv, a);
}
template <class T, int D>
cudaError_t attend_t(const AttendArgs& a, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t stream) {
    const int64_t rows = (int64_t)a.batch.total_q * a.q_heads;
    if (rows > INT32_MAX) return cudaErrorInvalidConfiguration;
    const cudaError_t e = a.row_tiles == 1 ? launch_tiles<T, D, 1>(a, mq, mk, mv, stream) : launch_tiles<T, D, 2>(a, mq, mk, mv, stream);
    if (e != cudaSuccess || a.splits == 1) return e;
    ++g_launches;
    if (a.splits > 16) return launch_behind(stream, dim3((unsigned)rows), dim3(256), 0, k_join<T, D, 8>, a);
    return launch_behind(stream, dim3((unsigned)ceil_div(rows, 8)), dim3(256), 0, k_join<T, D, 1>, a);
}
template <class T, int D>
cudaError_t weigh_t(const AttendArgs& a, const CUtensorMap& mq, const CUtensorMap& mk, cudaStream_t stream) {
    cudaError_t e = allow_smem<k_weigh<T, D>>(GeoWeigh<D>::kSmem);
    if (e != cudaSuccess) return e;
    ++g_launches;
    return launch_behind(stream, dim3((unsigned)ceil_div(a.batch.max_len, 128), a.heads, a.batch.batch), dim3(kThreadsWe), GeoWeigh<D>::kSmem, k_weigh<T, D>, mq, mk, a);
}

}  // namespace

cudaError_t launch_attend(const AttendArgs& a, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t stream) {
    return FD_KV_PICK(attend_t, a, mq, mk, mv, stream);
}
cudaError_t launch_weigh(const AttendArgs& a, const CUtensorMap& mq, const CUtensorMap& mk, cudaStream_t stream) {
    return FD_KV_PICK(weigh_t, a, mq, mk, stream);
}

}  // namespace kv
}  // namespace fd
