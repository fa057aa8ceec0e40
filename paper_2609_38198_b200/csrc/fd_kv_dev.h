// Device code that the attention kernels over paged keys and values share.
#pragma once

#include "fd_kv.h"
#include "fd_tc_common.h"

namespace fd {
namespace kv {

using namespace tc;

__device__ __forceinline__ void tma_load_4d(void* smem_dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(smem_u32(smem_dst)), "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ float max_nan(float a, float b) {       // a NaN is passed on
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

__device__ __forceinline__ float max_nan(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ uint64_t ex2_mufu(uint64_t x) {
    const float2 c = split2(x);
    return pair2(ex2f(c.x), ex2f(c.y));
}

// An element type.  A softmax weight is held as 2^(score - m + kShift), where m is the running maximum in use, raised when a score exceeds it by kLazy powers of two;
// kTop = kLazy + kShift bounds the exponent.  bf16 has fp32's range: no shift, and m is hardly ever raised.  fp16's normal numbers end at 2^-14 and its steps
// at 2^-24, so its weights fill the range from above: one keeps its 11 bits down to 2^-(14 + kShift) of the largest and is off by at most 2^-(25 + kShift) of it
// below.  (Without the shift, of 32767 tokens 18 below one other 69 % of the sum was lost: their weights became 0 while the norm counted them.)
template <class T> struct Elem;
template <> struct Elem<__nv_bfloat16> {
    static constexpr float kTop = 8.f;
    static constexpr uint32_t kFormat = 1, kExponent = 0x7f80u;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static __device__ __forceinline__ float at(const void* p, int64_t i) { return __bfloat162float(((const __nv_bfloat16*)p)[i]); }
};
template <> struct Elem<__half> {
    static constexpr float kTop = 15.f;
    static constexpr uint32_t kFormat = 0, kExponent = 0x7c00u;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack_f16x2(lo, hi); }
    static __device__ __forceinline__ float at(const void* p, int64_t i) { return __half2float(((const __half*)p)[i]); }
};

// What is taken off a score times c for the running maximum m: rounded up, so that no weight exceeds 2^kTop however large the scores, and the same number wherever sums made
// with one maximum are brought to another or to a logarithm (m * c alone is off by half a step of scores that may be millions).
__device__ __forceinline__ float held(float m, float c, float shift) { return m == -INFINITY ? 0.f : __fmaf_ru(m, c, -shift); }
// Factor from sums made with maximum m to maximum top >= m.
__device__ __forceinline__ float rescale(float m, float top, float c, float shift) {
    return m == top ? 1.0f : m == -INFINITY ? 0.f : ex2f(held(m, c, shift) - held(top, c, shift));
}

// Which rows a CTA works on: sequence, its first token, what it may see.
struct Work {
    int b, begin, count, n;           // sequence, its first row in q, its new tokens, its tokens in the cache
    int t0;                           // first token of the first tile
};
// The same value in a register that the compiler knows to be the same for the whole warp: loops and addresses made of it stay in uniform registers, without which
// every MMA that a thread issues costs about 45 clocks (tc::elect_one).
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ Work uniform(const Work& w) { return Work{uniform(w.b), uniform(w.begin), uniform(w.count), uniform(w.n), uniform(w.t0)}; }
// Slots that token t of a sequence sees: [lo, hi).
__device__ __forceinline__ int see_hi(const AttendArgs& a, const Work& w, int t) { return a.causal ? min(w.n, max(0, w.n - w.count + t + 1)) : w.n; }
__device__ __forceinline__ int see_lo(const AttendArgs& a, const Work& w, int t) { return a.window ? max(0, w.n - w.count + t + 1 - a.window) : 0; }

// Calls fn<element type, head_dim> for the arguments `a`.
#define FD_KV_PICK(fn, ...)                                                                                     \
    (a.dtype == FD_BF16 ? (a.head_dim == 128 ? fn<__nv_bfloat16, 128>(__VA_ARGS__) : fn<__nv_bfloat16, 64>(__VA_ARGS__)) \
                        : (a.head_dim == 128 ? fn<__half, 128>(__VA_ARGS__) : fn<__half, 64>(__VA_ARGS__)))

}  // namespace kv
}  // namespace fd
