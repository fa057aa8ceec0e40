// Entry points of the paged cache's operators and of rotary positions: argument checks, tensor maps, launches (fd.h: "kept keys and values").
#include <float.h>
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <algorithm>
#include <new>

#include "fd_kv.h"

namespace fd {
namespace kv {
namespace {

struct Err {
    char* buf; size_t len;
    Err(char* b, size_t n) : buf(b), len(n) { if (buf && len) buf[0] = 0; }
    fd_status operator()(fd_status st, const char* fmt, ...) const {
        if (buf && len) {
            va_list ap;
            va_start(ap, fmt);
            vsnprintf(buf, len, fmt, ap);
            va_end(ap);
        }
        return st;
    }
    fd_status cuda(cudaError_t e, const char* what) const { return (*this)(FD_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e)); }
};

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encoder() {
    static const EncodeFn fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess) p = nullptr;
        return reinterpret_cast<EncodeFn>(p);
    }();
    return fn;
}
// Tensor map of 16-bit elements, 128-byte swizzled boxes of 64 elements; strides in elements.
bool make_map(CUtensorMap* m, void* base, int dtype, int rank, const uint64_t* dims, const int64_t* strides, const uint32_t* box) {
    const EncodeFn fn = encoder();
    if (!fn) return false;
    cuuint64_t d[4], s[3];
    cuuint32_t b[4], one[4] = {1, 1, 1, 1};
    for (int i = 0; i < rank; ++i) { d[i] = dims[i]; b[i] = box[i]; }
    for (int i = 0; i + 1 < rank; ++i) s[i] = (cuuint64_t)strides[i] * 2;
    return fn(m, dtype == FD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)rank, base, d, s, b, one,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              d[0] > 64 ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : CU_TENSOR_MAP_L2_PROMOTION_L2_128B,      // (a row of a head, not of its neighbour)
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int64_t kMaxStride = (int64_t)1 << 38;      // (a tensor map's strides end at 2^40 bytes)

bool misaligned(const void* p, size_t size) { return reinterpret_cast<uintptr_t>(p) % size != 0; }

// A tensor of heads that is read or written in vectors of 16 bytes, or by TMA.
fd_status check_wide(const Err& err, const fd_heads& h, int head_dim, const char* what) {
    if (!h.p_dev || h.heads < 1) return err(FD_ERR_INVALID, "%s: no tensor", what);
    if (h.token_stride < 0 || h.head_stride < 0 || h.token_stride > kMaxStride || h.head_stride > kMaxStride || (h.heads > 1 && h.head_stride < head_dim))
        return err(FD_ERR_INVALID, "%s: bad strides", what);
    if ((reinterpret_cast<uintptr_t>(h.p_dev) & 15) || (h.token_stride & 7) || (h.head_stride & 7))
        return err(FD_ERR_INVALID, "%s: pointer and strides must be multiples of 16 bytes", what);
    return FD_OK;
}
fd_status check_rows(const Err& err, const fd_heads& h, int head_dim, int size, const char* what) {
    if (!h.p_dev || h.heads < 1) return err(FD_ERR_INVALID, "%s: no tensor", what);
    if (h.token_stride < 0 || h.head_stride < 0 || h.token_stride > kMaxStride || h.head_stride > kMaxStride || (h.heads > 1 && h.head_stride < head_dim))
        return err(FD_ERR_INVALID, "%s: bad strides", what);
    if (misaligned(h.p_dev, size)) return err(FD_ERR_INVALID, "%s: misaligned pointer", what);
    return FD_OK;
}
fd_status check_rotary(const Err& err, int head_dim, int rot, int layout, double scale, const void* positions, const void* freqs) {
    if (head_dim < 2 || head_dim > 1024 || (head_dim & 1)) return err(FD_ERR_UNSUPPORTED, "head_dim = %d: an even number up to 1024 is covered", head_dim);
    if (rot < 2 || rot > head_dim || (rot & 1)) return err(FD_ERR_INVALID, "rot_dim = %d: an even number in [2, head_dim]", rot);
    if (layout != FD_ROTARY_HALF && layout != FD_ROTARY_INTERLEAVED) return err(FD_ERR_INVALID, "unknown layout %d", layout);
    if (!(fabs(scale) <= 3e38)) return err(FD_ERR_INVALID, "scale is not finite");
    if (!positions || !freqs) return err(FD_ERR_INVALID, "positions and freqs must be non-null");
    if (misaligned(positions, 4) || misaligned(freqs, 8)) return err(FD_ERR_INVALID, "positions or freqs: misaligned pointer");
    return FD_OK;
}
fd_status check_bounds(const Err& err, const fd_kv_batch* b) {
    if (b->total_q < 0 || b->max_new < 0 || b->max_new > b->total_q || (b->max_new == 0 && b->total_q > 0) || b->max_len < 0) return err(FD_ERR_INVALID, "bad bounds: total_q %d, max_new %d, max_len %d", b->total_q, b->max_new, b->max_len);
    if (b->max_len > (1 << 30) || b->total_q > (1 << 30)) return err(FD_ERR_UNSUPPORTED, "lengths up to 2^30 tokens are covered");
    return FD_OK;
}
fd_status check_batch(const Err& err, const fd_kv* kv, const fd_kv_batch* b, bool queries) {
    if (!kv || !b) return err(FD_ERR_INVALID, "cache and batch must be non-null");
    if (b->batch < 0 || b->batch > 65535) return err(FD_ERR_INVALID, "batch = %d: 0 to 65535", b->batch);
    if (b->batch == 0) return FD_OK;
    if (!b->table_dev || !b->kv_len_dev || (queries && !b->q_start_dev)) return err(FD_ERR_INVALID, "page table, lengths and starts must be non-null");
    if (misaligned(b->table_dev, 4) || misaligned(b->kv_len_dev, 4) || (queries && misaligned(b->q_start_dev, 4))) return err(FD_ERR_INVALID, "page table, lengths or starts: misaligned pointer");
    if (b->max_pages < 1 || b->table_stride < 0) return err(FD_ERR_INVALID, "bad page table: %d pages a row, stride %lld", b->max_pages, (long long)b->table_stride);
    FD_TRY(check_bounds(err, b));
    return FD_OK;
}
Batch batch_of(const fd_kv* kv, const fd_kv_batch* b) {
    const int p = kv->d.page_size;
    return Batch{b->table_dev, b->table_stride, b->kv_len_dev, b->q_start_dev, b->batch, b->max_pages, b->total_q, b->max_len, p, kv->d.num_pages,
                 (p & (p - 1)) ? -1 : __builtin_ctz(p), kv->d.status_dev};
}
fd_status check_device(const Err& err, const fd_kv* kv) {
    int dev = -1;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return err.cuda(e, "cudaGetDevice");
    if (dev != kv->device) return err(FD_ERR_INVALID, "the cache belongs to device %d, device %d is current", kv->device, dev);
    return FD_OK;
}
bool overlap(const fd_heads& a, const fd_heads& b, int tokens, int head_dim, int size) {
    auto range = [&](const fd_heads& h, uintptr_t* lo, uintptr_t* hi) {
        *lo = reinterpret_cast<uintptr_t>(h.p_dev);
        *hi = *lo + (uintptr_t)((tokens - 1) * h.token_stride + (h.heads - 1) * h.head_stride + head_dim) * size;
    };
    uintptr_t al, ah, bl, bh;
    range(a, &al, &ah); range(b, &bl, &bh);
    return al < bh && bl < ah;
}
// Whether no two rows of a result overlap: rows that lie dt tokens and dh heads apart begin dt * token_stride + dh * head_stride apart, which has to be head_dim or
// more in either direction.
bool rows_apart(const fd_heads& h, int tokens, int head_dim) {
    const int64_t ts = h.token_stride, hs = h.head_stride;
    if (tokens <= 1) return true;                                // (a head stride below head_dim is refused for every tensor)
    if (ts < head_dim) return false;
    if (ts >= (h.heads - 1) * hs + head_dim || h.heads == 1) return true;
    for (int64_t dh = 1; dh < h.heads; ++dh) {                   // the two multiples of ts next to dh * hs
        const int64_t dt = dh * hs / ts, rest = dh * hs % ts;
        if ((rest < head_dim && dt < tokens) || (ts - rest < head_dim && dt + 1 < tokens)) return false;
    }
    return true;
}
// Whether two arrays of `rows` rows of `len` elements of 4 bytes, `stride` elements apart in both, overlap without being the same.
bool partly_over(const void* a, const void* b, int64_t rows, int64_t stride, int64_t len) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b), d = x < y ? y - x : x - y, l = 4 * (uintptr_t)len, s = 4 * (uintptr_t)stride;
    if (d == 0 || len <= 0 || d >= (uintptr_t)(rows - 1) * s + l) return false;
    return d % s < l || s - d % s < l;                           // (rows of the one may lie between those of the other)
}
bool same(const fd_heads& a, const fd_heads& b) { return a.p_dev == b.p_dev && a.token_stride == b.token_stride && a.head_stride == b.head_stride && a.heads == b.heads; }

}  // namespace

// Few rows a sequence: as many CTAs as the GPU holds at once (two an SM), each with 64 tokens of a cache or more, share the caches evenly.  Else: the cache in parts of
// at least two tiles of 128, as many as fill the GPU once if every sequence were as long as the longest, none longer than kPartTokens (beyond kMaxSplits of them: as long as that
// many parts are).
Plan plan_attend(const fd_kv* kv, const fd_kv_batch* b, int q_heads, bool weights) {
    Plan p{};
    const int64_t heads = kv->d.heads, group = q_heads / heads, sms = kv->sm_count, live = std::min(b->batch, b->total_q);
    const size_t rows = (size_t)b->total_q * q_heads, dim = kv->d.head_dim;
    p.splits = 1;
    p.few = (int64_t)b->max_new * group <= kFewRows;
    if (p.few) {
        p.ctas = (int)std::min<int64_t>(2 * sms, live * heads * std::max<int64_t>(1, ceil_div(b->max_len, 64)));
        p.parts = (size_t)round_up(2 * (int64_t)b->batch * heads, 4);
        p.part_o = (size_t)2 * p.ctas * kFewRows * dim;
        p.part_lse = (size_t)2 * p.ctas * kFewRows;
        // (a warp's tokens of a cache: a quarter of it, and the rest of a chunk)
        if (b->max_len >= kFewWarps * kPartTokens) p.folds = (size_t)p.ctas * kFewWarps * (dim / 8 + 1) * 32 * 4;
        if (weights) {
            p.score_stride = round_up(b->max_len, 64);
            p.scores = (size_t)b->batch * heads * b->max_new * group * p.score_stride;
        }
        return p;
    }
    p.row_tiles = b->max_new <= 128 / group ? 1 : 2;
    const int64_t tiles = std::max<int64_t>(1, ceil_div(b->max_len, 128));
    const int64_t ctas = p.row_tiles == 1 ? live * heads : (b->total_q / (2 * (128 / group)) + live) * heads, room = p.row_tiles == 1 ? 2 * sms : sms;
    const int64_t s = std::min<int64_t>(std::max<int64_t>({1, std::min(room / ctas, tiles / 2), ceil_div(b->max_len, kPartTokens)}), kMaxSplits);
    p.split_tiles = (int)ceil_div(tiles, s);
    p.splits = (int)ceil_div(tiles, p.split_tiles);
    if (p.splits > 1) { p.part_o = p.splits * rows * dim; p.part_lse = (p.splits * rows + 3) / 4 * 4; }
    return p;
}

}  // namespace kv
}  // namespace fd

using namespace fd;
using namespace fd::kv;

extern "C" {

fd_status fd_rotary_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double original_len, double lo, double hi, double* freqs_host) {
    if (!freqs_host || rot_dim < 2 || (rot_dim & 1) || rot_dim > 1024 || !(base > 0) || !(base < 1e300)) return FD_ERR_INVALID;
    if (scaling < FD_ROTARY_PLAIN || scaling > FD_ROTARY_RAMP) return FD_ERR_INVALID;
    if (scaling != FD_ROTARY_PLAIN && (!(factor > 0) || !(factor < 1e300))) return FD_ERR_INVALID;
    if (scaling == FD_ROTARY_BASE && rot_dim == 2) return FD_ERR_INVALID;
    if (scaling == FD_ROTARY_RAMP && (!(original_len > 0) || !(original_len < 1e300) || !(lo >= 0) || !(hi > lo) || !(hi < 1e300))) return FD_ERR_INVALID;
    const double b = scaling == FD_ROTARY_BASE ? base * pow(factor, rot_dim / (rot_dim - 2.0)) : base;
    for (int i = 0; i < rot_dim / 2; ++i) {
        const double f = pow(b, -2.0 * i / rot_dim);
        double out = f;
        if (scaling == FD_ROTARY_LINEAR) out = f / factor;
        if (scaling == FD_ROTARY_RAMP) {
            double part = (original_len * f / 6.28318530717958647693 - lo) / (hi - lo);
            part = part < 0 ? 0 : part > 1 ? 1 : part;
            out = f / factor * (1 - part) + f * part;
        }
        freqs_host[i] = out;
    }
    return FD_OK;
}

fd_status fd_rotary(const fd_heads* x, const fd_heads* out, int32_t dtype, int32_t tokens, int32_t head_dim, const int32_t* positions_dev,
                    const double* freqs_dev, int32_t rot_dim, int32_t layout, double scale, int32_t inverse, void* cuda_stream, char* errbuf, size_t errbuf_len) {
    const Err err(errbuf, errbuf_len);
    if (!x || !out) return err(FD_ERR_INVALID, "x and out must be non-null");
    if (dtype < FD_BF16 || dtype > FD_FP32) return err(FD_ERR_INVALID, "unknown element type %d", dtype);
    if (tokens < 0) return err(FD_ERR_INVALID, "tokens = %d", tokens);
    if (tokens == 0 || x->heads == 0) return FD_OK;
    FD_TRY(check_rotary(err, head_dim, rot_dim, layout, scale, positions_dev, freqs_dev));
    const int size = dtype == FD_FP32 ? 4 : 2;
    FD_TRY(check_rows(err, *x, head_dim, size, "x"));
    FD_TRY(check_rows(err, *out, head_dim, size, "out"));
    if (x->heads != out->heads || x->heads > 65536) return err(FD_ERR_INVALID, "x has %d heads, out %d", x->heads, out->heads);
    if (!rows_apart(*out, tokens, head_dim)) return err(FD_ERR_INVALID, "out: rows overlap");
    if (!same(*x, *out) && overlap(*x, *out, tokens, head_dim, size)) return err(FD_ERR_INVALID, "out overlaps x without being x");
    int dev = 0, sms = 148;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return err.cuda(e, "device");
    RowsArgs a{};
    a.x = heads_of(*x); a.y = heads_of(*out);
    a.positions = positions_dev; a.freqs = freqs_dev;
    a.tokens = tokens; a.head_dim = head_dim; a.rot = rot_dim; a.layout = layout;
    a.scale = (float)scale; a.sign = inverse ? -1.f : 1.f;
    e = launch_rows(a, dtype, sms, static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? FD_OK : err.cuda(e, "k_rows");
}

fd_status fd_kv_create(fd_kv** out, const fd_kv_desc* d, char* errbuf, size_t errbuf_len) {
    const Err err(errbuf, errbuf_len);
    if (!out) return err(FD_ERR_INVALID, "out must be non-null");
    *out = nullptr;
    if (!d || !d->k_dev || !d->v_dev || !d->status_dev) return err(FD_ERR_INVALID, "pools and status words must be non-null");
    if (d->dtype != FD_BF16 && d->dtype != FD_FP16) return err(FD_ERR_UNSUPPORTED, "element type %d: FD_BF16 and FD_FP16 are covered", d->dtype);
    if (d->head_dim != 64 && d->head_dim != 128) return err(FD_ERR_UNSUPPORTED, "head_dim = %d: 64 and 128 are covered", d->head_dim);
    if (d->page_size < 8 || d->page_size % 8 || d->page_size > (1 << 20)) return err(FD_ERR_UNSUPPORTED, "page_size = %d: multiples of 8 are covered", d->page_size);
    if (d->num_pages < 1 || d->heads < 1 || d->heads > 65535) return err(FD_ERR_INVALID, "bad pool: %d pages, %d heads", d->num_pages, d->heads);
    if ((reinterpret_cast<uintptr_t>(d->k_dev) & 15) || (reinterpret_cast<uintptr_t>(d->v_dev) & 15)) return err(FD_ERR_INVALID, "pools must be 16-byte aligned");
    if (reinterpret_cast<uintptr_t>(d->status_dev) & 3) return err(FD_ERR_INVALID, "status words are misaligned");
    for (const int64_t s : {d->k_page_stride, d->k_token_stride, d->k_head_stride, d->v_page_stride, d->v_token_stride, d->v_head_stride})
        if (s < d->head_dim || (s & 7) || s > kMaxStride) return err(FD_ERR_INVALID, "stride %lld: a multiple of 8 elements, head_dim or more", (long long)s);
    fd_kv* kv = new (std::nothrow) fd_kv();
    if (!kv) return err(FD_ERR_INVALID, "out of host memory");
    kv->d = *d;
    int g = d->page_size, m = 128;
    while (m) { const int r = g % m; g = m; m = r; }
    kv->box_rows = g;
    cudaError_t e = cudaGetDevice(&kv->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&kv->sm_count, cudaDevAttrMultiProcessorCount, kv->device);
    if (e != cudaSuccess) { delete kv; return err.cuda(e, "device"); }
    const uint64_t dims[4] = {(uint64_t)d->head_dim, (uint64_t)d->page_size, (uint64_t)d->heads, (uint64_t)d->num_pages};
    const uint32_t box[4] = {64, (uint32_t)kv->box_rows, 1, 1};
    const int chunk = d->head_dim == 128 ? 16 : 32;
    const uint32_t few[4] = {64, (uint32_t)(kv->few_rows = g < chunk ? g : chunk), 1, 1};
    const int64_t ks[3] = {d->k_token_stride, d->k_head_stride, d->k_page_stride}, vs[3] = {d->v_token_stride, d->v_head_stride, d->v_page_stride};
    if (!make_map(&kv->map_k, d->k_dev, d->dtype, 4, dims, ks, box) || !make_map(&kv->map_v, d->v_dev, d->dtype, 4, dims, vs, box) ||
        !make_map(&kv->few_k, d->k_dev, d->dtype, 4, dims, ks, few) || !make_map(&kv->few_v, d->v_dev, d->dtype, 4, dims, vs, few)) {
        delete kv;
        return err(FD_ERR_CUDA, "cuTensorMapEncodeTiled refused the pools");
    }
    *out = kv;
    return FD_OK;
}

void fd_kv_destroy(fd_kv* kv) { delete kv; }

fd_status fd_kv_synchronize(fd_kv* kv, void* cuda_stream) {
    if (!kv) return FD_ERR_INVALID;
    const Err err(nullptr, 0);
    FD_TRY(check_device(err, kv));
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    unsigned int words[2] = {0, 0};
    if (cudaMemcpyAsync(words, kv->d.status_dev, sizeof words, cudaMemcpyDeviceToHost, s) != cudaSuccess) return FD_ERR_CUDA;
    if (cudaStreamSynchronize(s) != cudaSuccess) return FD_ERR_CUDA;
    if (!words[0] && !words[1]) return FD_OK;
    if (cudaMemsetAsync(kv->d.status_dev, 0, sizeof words, s) != cudaSuccess) return FD_ERR_CUDA;
    return words[1] ? FD_ERR_TIMEOUT : FD_ERR_INVALID;
}

fd_status fd_kv_append(const fd_kv* kv, const fd_kv_batch* b, const fd_kv_append_args* x, void* cuda_stream, char* errbuf, size_t errbuf_len) {
    const Err err(errbuf, errbuf_len);
    FD_TRY(check_batch(err, kv, b, true));
    if (!x) return err(FD_ERR_INVALID, "arguments must be non-null");
    if (b->batch == 0 || b->total_q == 0) return FD_OK;
    const fd_kv_desc& d = kv->d;
    FD_TRY(check_rows(err, x->k, d.head_dim, 2, "k"));
    FD_TRY(check_rows(err, x->v, d.head_dim, 2, "v"));
    if (x->k.heads != d.heads || x->v.heads != d.heads) return err(FD_ERR_INVALID, "k has %d heads, v %d, the cache %d", x->k.heads, x->v.heads, d.heads);
    const bool turn = x->positions_dev != nullptr, q = x->q.p_dev != nullptr;
    if (turn) FD_TRY(check_rotary(err, d.head_dim, x->rot_dim, x->layout, x->scale, x->positions_dev, x->freqs_dev));
    if (q) {
        if (!turn) return err(FD_ERR_INVALID, "q without positions");
        FD_TRY(check_rows(err, x->q, d.head_dim, 2, "q"));
        FD_TRY(check_rows(err, x->q_out, d.head_dim, 2, "q_out"));
        if (x->q.heads != x->q_out.heads || x->q.heads > 65536) return err(FD_ERR_INVALID, "q has %d heads, q_out %d", x->q.heads, x->q_out.heads);
        if (!same(x->q, x->q_out) && overlap(x->q, x->q_out, b->total_q, d.head_dim, 2)) return err(FD_ERR_INVALID, "q_out overlaps q without being q");
        if (!rows_apart(x->q_out, b->total_q, d.head_dim)) return err(FD_ERR_INVALID, "q_out: rows overlap");
    }
    FD_TRY(check_device(err, kv));
    RowsArgs a{};
    if (q) { a.x = heads_of(x->q); a.y = heads_of(x->q_out); }
    a.k = heads_of(x->k); a.v = heads_of(x->v);
    a.k_pool = d.k_dev; a.v_pool = d.v_dev;
    a.k_page = d.k_page_stride; a.k_token = d.k_token_stride; a.k_head = d.k_head_stride;
    a.v_page = d.v_page_stride; a.v_token = d.v_token_stride; a.v_head = d.v_head_stride;
    a.positions = x->positions_dev; a.freqs = x->freqs_dev;
    a.batch = batch_of(kv, b);
    a.tokens = b->total_q; a.head_dim = d.head_dim; a.rot = turn ? x->rot_dim : 0; a.layout = turn ? x->layout : FD_ROTARY_HALF; a.append = 1;
    a.scale = (float)x->scale; a.sign = 1.f;
    const cudaError_t e = launch_rows(a, d.dtype, kv->sm_count, static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? FD_OK : err.cuda(e, "k_rows");
}

size_t fd_kv_attend_bytes(const fd_kv* kv, const fd_kv_batch* b, int32_t q_heads, int32_t weights) {
    if (!kv || !b || q_heads < 1 || q_heads % kv->d.heads || q_heads / kv->d.heads > 128 || b->batch < 1 || b->batch > 65535 || b->total_q < 1) return 0;
    if (check_bounds(Err(nullptr, 0), b) != FD_OK) return 0;
    return plan_attend(kv, b, q_heads, weights != 0).bytes();
}

fd_status fd_kv_attend(const fd_kv* kv, const fd_kv_batch* b, const fd_kv_attend_args* x, void* workspace_dev, size_t workspace_bytes, void* cuda_stream,
                       char* errbuf, size_t errbuf_len) {
    const Err err(errbuf, errbuf_len);
    FD_TRY(check_batch(err, kv, b, true));
    if (!x) return err(FD_ERR_INVALID, "arguments must be non-null");
    if (b->batch == 0) return FD_OK;
    const fd_kv_desc& d = kv->d;
    if (misaligned(x->lse_dev, 4) || misaligned(x->weights_in_dev, 4) || misaligned(x->weights_out_dev, 4)) return err(FD_ERR_INVALID, "lse or weights: misaligned pointer");
    if (x->weights_out_dev) {
        if (!x->lse_dev && b->total_q > 0) return err(FD_ERR_INVALID, "weights need lse");
        if (x->weights_stride < b->max_len) return err(FD_ERR_INVALID, "weights: stride %lld is below max_len = %d", (long long)x->weights_stride, b->max_len);
        if (x->weights_in_dev && partly_over(x->weights_in_dev, x->weights_out_dev, (int64_t)b->batch * d.heads, x->weights_stride, b->max_len))
            return err(FD_ERR_INVALID, "weights_out overlaps weights_in without being it");
    } else if (x->weights_in_dev) return err(FD_ERR_INVALID, "weights_in without weights_out");
    if (b->total_q > 0) {
        FD_TRY(check_wide(err, x->q, d.head_dim, "q"));
        FD_TRY(check_wide(err, x->out, d.head_dim, "out"));
        if (x->q.heads != x->out.heads || x->q.heads % d.heads) return err(FD_ERR_INVALID, "q has %d heads, out %d, the cache %d", x->q.heads, x->out.heads, d.heads);
        if (x->q.heads / d.heads > 128) return err(FD_ERR_UNSUPPORTED, "%d query heads a cached head: up to 128 are covered", x->q.heads / d.heads);
        if (overlap(x->q, x->out, b->total_q, d.head_dim, 2)) return err(FD_ERR_INVALID, "out overlaps q");
        if (b->total_q > 1 && x->q.token_stride < d.head_dim) return err(FD_ERR_INVALID, "q: rows of two tokens overlap");
        if (!rows_apart(x->out, b->total_q, d.head_dim)) return err(FD_ERR_INVALID, "out: rows overlap");
    }
    if (!(x->scale > 0) || !(x->scale < 1e30)) return err(FD_ERR_INVALID, "scale must be positive");
    // (a hidden score is -inf, and -inf times a scale that rounds to 0 is NaN)
    if (!((float)(x->scale * kLog2e) >= FLT_MIN)) return err(FD_ERR_UNSUPPORTED, "scale = %g: below what fp32 holds as a normal number", x->scale);
    if (x->window < 0 || (x->window > 0 && !x->causal)) return err(FD_ERR_INVALID, "a window is positive and causal (0: none)");
    FD_TRY(check_device(err, kv));
    if (b->total_q == 0 && !x->weights_out_dev) return FD_OK;
    AttendArgs a{};
    a.batch = batch_of(kv, b);
    a.out = heads_of(x->out);
    a.heads = d.heads; a.head_dim = d.head_dim; a.dtype = d.dtype;
    a.q_heads = b->total_q > 0 ? x->q.heads : d.heads; a.group = a.q_heads / d.heads; a.tile_tokens = 128 / a.group;
    a.causal = x->causal ? 1 : 0; a.window = std::min(x->window, 1 << 30);       // (no length is above 2^30)
    a.scale_log2 = (float)(x->scale * kLog2e);
    a.lse = x->lse_dev;
    a.w_in = x->weights_in_dev; a.w_out = x->weights_out_dev; a.w_stride = x->weights_stride;
    a.box_rows = kv->box_rows; a.sm_count = kv->sm_count;
    a.v_pool = d.v_dev; a.v_page = d.v_page_stride; a.v_token = d.v_token_stride; a.v_head = d.v_head_stride;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    CUtensorMap mq;
    bool few = false;
    if (b->total_q > 0) {
        const Plan p = plan_attend(kv, b, a.q_heads, a.w_out != nullptr);
        const size_t need = p.bytes();
        if (need && (!workspace_dev || workspace_bytes < need)) return err(FD_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
        if (need && (reinterpret_cast<uintptr_t>(workspace_dev) & 15)) return err(FD_ERR_INVALID, "workspace must be 16-byte aligned");
        few = p.few;
        a.row_tiles = p.row_tiles; a.splits = p.splits; a.split_tiles = p.split_tiles; a.ctas = p.ctas; a.few_rows = few ? b->max_new * a.group : 0;
        a.parts = static_cast<int2*>(workspace_dev);
        a.part_o = static_cast<float*>(workspace_dev) + p.parts;
        a.part_lse = a.part_o + p.part_o;
        a.scores = p.scores ? a.part_lse + p.part_lse : nullptr; a.score_stride = p.score_stride;
        a.folds = p.folds ? a.part_lse + p.part_lse + p.scores : nullptr;
        a.q = heads_of(x->q);
        cudaError_t e;
        if (few) {
            a.box_rows = kv->few_rows;
            e = launch_few(a, kv->few_k, kv->few_v, stream);
        } else {
            const uint64_t dims[3] = {(uint64_t)d.head_dim, (uint64_t)a.q_heads, (uint64_t)b->total_q};
            const uint32_t box[3] = {64, (uint32_t)a.group, (uint32_t)a.tile_tokens};
            // (a stride that no step uses may be anything the map accepts)
            const int64_t strides[2] = {a.q_heads > 1 ? x->q.head_stride : d.head_dim, b->total_q > 1 ? x->q.token_stride : d.head_dim};
            if (!make_map(&mq, x->q.p_dev, d.dtype, 3, dims, strides, box)) return err(FD_ERR_CUDA, "cuTensorMapEncodeTiled refused q");
            e = launch_attend(a, mq, kv->map_k, kv->map_v, stream);
        }
        if (e != cudaSuccess) return err.cuda(e, "attention");
    } else {
        mq = kv->map_k;                            // no rows: the weights are copied, nothing is loaded through it
    }
    if (a.w_out && b->max_len > 0 && !few) {
        const cudaError_t e = launch_weigh(a, mq, kv->map_k, stream);
        if (e != cudaSuccess) return err.cuda(e, "k_weigh");
    }
    return FD_OK;
}

fd_status fd_kv_evict(const fd_kv* kv, const fd_kv_batch* b, const fd_kv_evict_args* x, void* cuda_stream, char* errbuf, size_t errbuf_len) {
    const Err err(errbuf, errbuf_len);
    FD_TRY(check_batch(err, kv, b, false));
    if (!x) return err(FD_ERR_INVALID, "arguments must be non-null");
    if (b->batch == 0) return FD_OK;
    const fd_kv_desc& d = kv->d;
    if (!x->weights_in_dev || !x->weights_out_dev || !x->kept_dev || !x->new_len_dev || !x->new_table_dev) return err(FD_ERR_INVALID, "weights, kept, new_len and new_table must be non-null");
    for (const void* p : {(const void*)x->weights_in_dev, (const void*)x->weights_out_dev, (const void*)x->kept_dev, (const void*)x->new_len_dev, (const void*)x->new_table_dev})
        if (misaligned(p, 4)) return err(FD_ERR_INVALID, "weights, kept, new_len or new_table: misaligned pointer");
    if (x->keep < 1 || x->first < 0 || x->recent < 0 || (int64_t)x->first + x->recent > x->keep) return err(FD_ERR_INVALID, "keep = %d, first = %d, recent = %d", x->keep, x->first, x->recent);
    if (x->keep > (1 << 30)) return err(FD_ERR_UNSUPPORTED, "keep = %d: lengths up to 2^30 tokens are covered", x->keep);
    if (x->weights_stride < b->max_len) return err(FD_ERR_INVALID, "weights: stride %lld is below max_len = %d", (long long)x->weights_stride, b->max_len);
    if (partly_over(x->weights_in_dev, x->weights_out_dev, (int64_t)b->batch * d.heads, x->weights_stride, b->max_len))
        return err(FD_ERR_INVALID, "weights_out overlaps weights_in without being it");
    if (partly_over(x->new_len_dev, b->kv_len_dev, 1, b->batch, b->batch)) return err(FD_ERR_INVALID, "new_len overlaps kv_len without being it");
    // (written to: no two sequences may have a page in common, which rows that overlap would)
    if (x->new_max_pages < 1 || x->new_table_stride < x->new_max_pages) return err(FD_ERR_INVALID, "bad new page table: %d pages a row, stride %lld", x->new_max_pages, (long long)x->new_table_stride);
    if (x->new_max_pages < ceil_div(x->keep < b->max_len ? x->keep : b->max_len, d.page_size)) return err(FD_ERR_INVALID, "new page table: %d pages a row hold fewer tokens than are kept", x->new_max_pages);
    FD_TRY(check_device(err, kv));
    EvictArgs a{};
    a.batch = batch_of(kv, b);
    a.w_in = x->weights_in_dev; a.w_out = x->weights_out_dev; a.w_stride = x->weights_stride;
    a.new_table = x->new_table_dev; a.new_table_stride = x->new_table_stride; a.new_max_pages = x->new_max_pages;
    a.keep = x->keep; a.first = x->first; a.recent = x->recent; a.heads = d.heads; a.head_dim = d.head_dim;
    a.kept = x->kept_dev; a.new_len = x->new_len_dev;
    a.k_pool = d.k_dev; a.v_pool = d.v_dev;
    a.k_page = d.k_page_stride; a.k_token = d.k_token_stride; a.k_head = d.k_head_stride;
    a.v_page = d.v_page_stride; a.v_token = d.v_token_stride; a.v_head = d.v_head_stride;
    const cudaError_t e = launch_evict(a, static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? FD_OK : err.cuda(e, "eviction");
}

}  // extern "C"
