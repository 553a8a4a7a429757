// The paged cache of keys and values, and attention of one new row of each of many running sequences over it.
#include "attention.h"

#include <math.h>

namespace fx {

typedef __attribute__((ext_vector_type(2))) float f32v2;

struct CacheArgs {
    unsigned char *k, *v;
    uint8_t *k_exp, *v_exp;
    const int32_t *table, *start;       // start: of the rows written or read, or the lengths of a step
    int64_t ld_table;
    int32_t cols, pages, page_rows, kv_heads, dim, pitch;
};

// Row of the cache (over pages, heads, positions) that a position has, or -1
__host__ __device__ __forceinline__ int64_t cache_row(const CacheArgs& c, int64_t seq, int64_t pos, int head) {
    if (pos < 0) return -1;
    const int64_t col = pos / c.page_rows;
    if (col >= c.cols) return -1;
    const int32_t page = c.table[seq * c.ld_table + col];
    if (page < 0 || page >= c.pages) return -1;
    return ((int64_t)page * c.kv_heads + head) * c.page_rows + pos % c.page_rows;
}

// e4m3 code of x, which is at most 448 in size or NaN
__device__ __forceinline__ uint32_t to_e4m3(float a, float b) { return __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xFFFF; }

// the least e + 127 in 0 .. 255 with top <= 448 2^e = 1.75 2^(e + 8)
__host__ __device__ __forceinline__ int exponent_of(float top) {
    uint32_t u;
    memcpy(&u, &top, 4);
    if (u < 0x00800000u) return 0;                      // below 2^-126 all is left to e = -127
    const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFF) > 0x600000u ? 1 : 0);
    return e < 0 ? 0 : e;
}

template <int DT, bool E4M3>
__global__ void k_cache_write(CacheArgs c, const int32_t* first, int32_t n_seqs, int64_t rows, HeadsView k, HeadsView v) {
    typedef typename AttnType<DT>::T T;
    const int lane = threadIdx.x & 63;
    for (int64_t i = blockIdx.x * (int64_t)(blockDim.x / 64) + threadIdx.x / 64; i < rows * c.kv_heads; i += (int64_t)gridDim.x * (blockDim.x / 64)) {
        const int64_t r = i / c.kv_heads;
        const int head = (int)(i % c.kv_heads);
        int64_t seq = r, in = 0;
        if (first) {
            int lo = 0, hi = n_seqs;            // the last sequence that begins at r or before, and has rows
            while (hi - lo > 1) { const int mid = (lo + hi) / 2; if (first[mid] <= r) lo = mid; else hi = mid; }
            seq = lo;
            in = r - first[lo];
        }
        const int64_t at = cache_row(c, seq, (int64_t)c.start[seq] + in, head);
        if (at < 0) continue;
        for (int which = 0; which < 2; ++which) {
            const HeadsView& s = which ? v : k;
            const T* src = (const T*)(s.p + r * s.ld + head * s.hs);
            unsigned char* dst = (which ? c.v : c.k) + at * c.pitch * (E4M3 ? 1 : AttnType<DT>::ES);
            float x[4], top = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int d = lane * 4 + e;
                x[e] = d < c.dim ? (float)src[d] : 0.f;
                if (isfinite(x[e])) top = fmaxf(top, fabsf(x[e]));
            }
            if (E4M3) {
                for (int o = 1; o < 64; o *= 2) top = fmaxf(top, __shfl_xor(top, o, 64));
                const int ex = exponent_of(top);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = isfinite(x[e]) ? ldexpf(x[e], 127 - ex) : NAN;
                if (lane * 4 < c.pitch) ((uint32_t*)dst)[lane] = to_e4m3(x[0], x[1]) | to_e4m3(x[2], x[3]) << 16;
                if (lane == 0) (which ? c.v_exp : c.k_exp)[at] = (uint8_t)ex;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (lane * 4 + e < c.pitch) ((T*)dst)[lane * 4 + e] = lane * 4 + e < c.dim ? src[lane * 4 + e] : T(0.f);
            }
        }
    }
}

template <int DT, bool E4M3>
__global__ void k_cache_read(CacheArgs c, const int32_t* first, int32_t n_seqs, int64_t rows, HeadsView k, HeadsView v) {
    typedef typename AttnType<DT>::T T;
    const int lane = threadIdx.x & 63;
    for (int64_t i = blockIdx.x * (int64_t)(blockDim.x / 64) + threadIdx.x / 64; i < rows * c.kv_heads; i += (int64_t)gridDim.x * (blockDim.x / 64)) {
        const int64_t r = i / c.kv_heads;
        const int head = (int)(i % c.kv_heads);
        int lo = 0, hi = n_seqs;
        while (hi - lo > 1) { const int mid = (lo + hi) / 2; if (first[mid] <= r) lo = mid; else hi = mid; }
        const int64_t at = cache_row(c, lo, (int64_t)c.start[lo] + r - first[lo], head);
        for (int which = 0; which < 2; ++which) {
            const HeadsView& s = which ? v : k;
            T* dst = (T*)(s.p + r * s.ld + head * s.hs);
            const unsigned char* src = (which ? c.v : c.k) + at * c.pitch * (E4M3 ? 1 : AttnType<DT>::ES);
            for (int d = lane; d < c.dim; d += 64) {
                T x = T(0.f);
                if (at >= 0) {
                    if (E4M3) x = (T)ldexpf(__builtin_amdgcn_cvt_pk_f32_fp8((int)src[d], false)[0], (int)(which ? c.v_exp : c.k_exp)[at] - 127);
                    else x = ((const T*)src)[d];
                }
                dst[d] = x;
            }
        }
    }
}

// One wave a row and query head
template <int DT, bool E4M3>
__global__ void k_attention_step(CacheArgs c, int64_t rows, int64_t most, int heads, float scale, HeadsView q, HeadsView out, float* lse) {
    typedef typename AttnType<DT>::T T;
    const int lane = threadIdx.x & 63, group = heads / c.kv_heads;
    const int64_t i = blockIdx.x;
    const int64_t b = i / heads;
    const int head = (int)(i % heads), kv = head / group;
    const T* qr = (const T*)(q.p + b * q.ld + head * q.hs);
    const int64_t n = c.start[b] < most ? c.start[b] : most;
    float m = -INFINITY, sum = 0.f, acc[4] = {};
    for (int64_t p0 = 0; p0 < n; p0 += 64) {
        const int64_t pos = p0 + lane, at = pos < n ? cache_row(c, b, pos, kv) : -1;
        float s = -INFINITY;
        if (at >= 0) {
            float d = 0.f;
            const unsigned char* src = c.k + at * c.pitch * (E4M3 ? 1 : AttnType<DT>::ES);
            for (int e = 0; e < c.dim; ++e) d = fmaf((float)qr[e], E4M3 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)src[e], false)[0] : (float)((const T*)src)[e], d);
            if (E4M3) d = ldexpf(d, (int)c.k_exp[at] - 127);
            s = d * scale;
        }
        float top = s;
        for (int o = 1; o < 64; o *= 2) top = fmaxf(top, __shfl_xor(top, o, 64));
        const float m2 = fmaxf(m, top), mu = m2 == -INFINITY ? 0.f : m2, f = m == -INFINITY ? 0.f : expf(m - mu);
        m = m2;
        const float p = at >= 0 ? expf(s - mu) : 0.f;
        float part = p;
        for (int o = 1; o < 64; o *= 2) part += __shfl_xor(part, o, 64);
        sum = sum * f + part;
        for (int e = 0; e < 4; ++e) acc[e] *= f;
        for (int j = 0; j < 64; ++j) {
            const int64_t a2 = __shfl(at, j, 64);
            const float pj = __shfl(p, j, 64);
            if (a2 < 0) continue;
            const unsigned char* src = c.v + a2 * c.pitch * (E4M3 ? 1 : AttnType<DT>::ES);
            for (int e = 0; e < 4; ++e) {
                const int d = lane + 64 * e;
                if (d >= c.dim) continue;
                float x = E4M3 ? ldexpf(__builtin_amdgcn_cvt_pk_f32_fp8((int)src[d], false)[0], (int)c.v_exp[a2] - 127) : (float)((const T*)src)[d];
                acc[e] = fmaf(pj, x, acc[e]);
            }
        }
    }
    T* o = (T*)(out.p + b * out.ld + head * out.hs);
    for (int e = 0; e < 4; ++e)
        if (lane + 64 * e < c.dim) o[lane + 64 * e] = (T)(sum == 0.f ? 0.f : acc[e] / sum);
    if (lse && lane == 0) lse[b * heads + head] = sum == 0.f ? -INFINITY : m + logf(sum);
}

// ------------------------------------------------------------------ host
static fx_status check_cache(const char* who, const fx_cache* c, fx_dtype dt, CacheArgs* a) {
    if (!c || (dt != FX_F32 && dt != FX_F16 && dt != FX_BF16) || c->kv_heads < 1 || c->dim < 1 || c->pages < 0 || c->page_rows < 1 || c->table_cols < 0 ||
        c->ld_table < c->table_cols) {
        set_error("%s: null cache, unknown dtype, or a size that is not positive", who);
        return FX_EINVAL;
    }
    if (c->store != FX_F32 && c->store != FX_F16 && c->store != FX_BF16 && c->store != FX_E4M3) { set_error("%s: unknown type of the cache", who); return FX_EINVAL; }
    if (c->store != FX_E4M3 && c->store != (int32_t)dt) { set_error("%s: rows of one type and a cache of another", who); return FX_EUNSUPPORTED; }
    if (c->dim > kMostDim) { set_error("%s: more than %d dimensions", who, kMostDim); return FX_ERANGE; }
    if (c->kv_heads > 65535) { set_error("%s: more than 65535 heads", who); return FX_ERANGE; }
    if (c->pages > 0 && (!c->d_k || !c->d_v || (uintptr_t)c->d_k % 16 || (uintptr_t)c->d_v % 16 || c->d_k == c->d_v)) {
        set_error("%s: d_k or d_v is null or not aligned to 16 bytes, or they are the same", who);
        return FX_EINVAL;
    }
    if (c->pages > 0 && (c->store == FX_E4M3 ? !c->d_k_exp || !c->d_v_exp || c->d_k_exp == c->d_v_exp : c->d_k_exp || c->d_v_exp)) {
        set_error("%s: exponents belong to a cache of 8 bits, one array for keys and one for values", who);
        return FX_EINVAL;
    }
    if ((c->table_cols > 0 && !c->d_table) || (uintptr_t)c->d_table % 4) { set_error("%s: d_table is null or not aligned to its elements", who); return FX_EINVAL; }
    *a = CacheArgs{(unsigned char*)c->d_k, (unsigned char*)c->d_v, c->d_k_exp, c->d_v_exp, c->d_table, nullptr, c->ld_table, c->table_cols, c->pages, c->page_rows,
                   c->kv_heads, c->dim, (c->dim + 15) / 16 * 16};
    return FX_OK;
}

}  // namespace fx

using namespace fx;

extern "C" fx_status fx_cache_write(const fx_cache* c, const fx_sequences* q, int64_t rows, const int32_t* d_start, fx_dtype dt, const void* d_k, int64_t ld_k,
                                    int64_t hs_k, const void* d_v, int64_t ld_v, int64_t hs_v, void* stream) {
    const char* who = "fx_cache_write";
    CacheArgs a;
    FX_TRY(check_cache(who, c, dt, &a));
    if (rows < 0 || (q && rows != q->rows)) { set_error("%s: %lld rows do not fit the sequences", who, (long long)rows); return FX_EINVAL; }
    const HeadsTensor t[] = {{"d_k", d_k, ld_k, hs_k, rows, c->kv_heads, false, true, nullptr}, {"d_v", d_v, ld_v, hs_v, rows, c->kv_heads, false, true, nullptr}};
    for (const HeadsTensor& x : t) FX_TRY(check_heads(who, x, c->dim, dtype_size(dt)));
    if (rows > 0 && (!d_start || (uintptr_t)d_start % 4)) { set_error("%s: d_start is null or not aligned to its elements", who); return FX_EINVAL; }
    if (rows > 0x7FFFFFFFll) { set_error("%s: more than 2^31-1 rows", who); return FX_ERANGE; }
    if (rows == 0 || a.pages == 0) return FX_OK;
    a.start = d_start;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps(kProfCache, st);
    const int es = dtype_size(dt);
    const HeadsView k{(unsigned char*)d_k, ld_k * es, hs_k * es}, v{(unsigned char*)d_v, ld_v * es, hs_v * es};
    const unsigned blocks = (unsigned)std::min<int64_t>((rows * c->kv_heads + 3) / 4, 1 << 16);
    const int32_t* first = q ? q->d_first : nullptr;
    const int32_t n = q ? q->B : 0;
#define FX_RUN(DT, E) k_cache_write<DT, E><<<blocks, 256, 0, st>>>(a, first, n, rows, k, v)
#define FX_RUN_TYPES() do { const bool e = c->store == FX_E4M3; \
        if (dt == FX_F32) { if (e) FX_RUN(FX_F32, true); else FX_RUN(FX_F32, false); } \
        else if (dt == FX_F16) { if (e) FX_RUN(FX_F16, true); else FX_RUN(FX_F16, false); } \
        else { if (e) FX_RUN(FX_BF16, true); else FX_RUN(FX_BF16, false); } } while (0)
    FX_RUN_TYPES();
#undef FX_RUN
    FX_HIP_TRY(hipGetLastError());
    return FX_OK;
}

extern "C" fx_status fx_cache_read(const fx_cache* c, const fx_sequences* q, const int32_t* d_start, fx_dtype dt, void* d_k, int64_t ld_k, int64_t hs_k,
                                   void* d_v, int64_t ld_v, int64_t hs_v, void* stream) {
    const char* who = "fx_cache_read";
    CacheArgs a;
    FX_TRY(check_cache(who, c, dt, &a));
    if (!q) { set_error("%s: null sequences", who); return FX_EINVAL; }
    const int64_t rows = q->rows;
    const HeadsTensor t[] = {{"d_k", d_k, ld_k, hs_k, rows, c->kv_heads, true, true, nullptr}, {"d_v", d_v, ld_v, hs_v, rows, c->kv_heads, true, true, nullptr}};
    for (const HeadsTensor& x : t) FX_TRY(check_heads(who, x, c->dim, dtype_size(dt)));
    if (rows > 0 && d_k == d_v) { set_error("%s: d_k and d_v are the same", who); return FX_EINVAL; }
    if (rows > 0 && (!d_start || (uintptr_t)d_start % 4)) { set_error("%s: d_start is null or not aligned to its elements", who); return FX_EINVAL; }
    if (rows == 0) return FX_OK;
    a.start = d_start;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps(kProfCache, st);
    const int es = dtype_size(dt);
    const HeadsView k{(unsigned char*)d_k, ld_k * es, hs_k * es}, v{(unsigned char*)d_v, ld_v * es, hs_v * es};
    const unsigned blocks = (unsigned)std::min<int64_t>((rows * c->kv_heads + 3) / 4, 1 << 16);
    const int32_t* first = q->d_first;
    const int32_t n = q->B;
#define FX_RUN(DT, E) k_cache_read<DT, E><<<blocks, 256, 0, st>>>(a, first, n, rows, k, v)
    FX_RUN_TYPES();
#undef FX_RUN
    FX_HIP_TRY(hipGetLastError());
    return FX_OK;
}

extern "C" fx_status fx_attention_step(const fx_cache* c, int64_t rows, const int32_t* d_len, int64_t most, fx_dtype dt, int32_t heads, float scale, const void* d_q,
                                       int64_t ld_q, int64_t hs_q, void* d_out, int64_t ld_out, int64_t hs_out, float* d_lse, void* stream) {
    const char* who = "fx_attention_step";
    CacheArgs a;
    FX_TRY(check_cache(who, c, dt, &a));
    if (rows < 0 || most < 0 || heads < 1 || heads % c->kv_heads || !std::isfinite(scale)) {
        set_error("%s: negative sizes, heads that are no multiple of the key heads, or a scale that is not finite", who);
        return FX_EINVAL;
    }
    if (heads > 65535) { set_error("%s: more than 65535 heads", who); return FX_ERANGE; }
    const HeadsTensor t[] = {{"d_q", d_q, ld_q, hs_q, rows, heads, false, true, nullptr}, {"d_out", d_out, ld_out, hs_out, rows, heads, true, true, nullptr}};
    for (const HeadsTensor& x : t) FX_TRY(check_heads(who, x, c->dim, dtype_size(dt)));
    if (rows > 0 && (!d_len || (uintptr_t)d_len % 4 || (uintptr_t)d_lse % 4)) { set_error("%s: d_len is null, or it or d_lse is not aligned to its elements", who); return FX_EINVAL; }
    if (rows > 0 && d_q == d_out) { set_error("%s: d_out is where d_q is", who); return FX_EINVAL; }
    if (rows * heads > 0x7FFFFFFFll / 64 || rows > 0x7FFFFFFFll) { set_error("%s: too many rows", who); return FX_ERANGE; }
    if (rows == 0) return FX_OK;
    a.start = d_len;
    const int64_t all = (int64_t)a.cols * a.page_rows;
    most = most == 0 ? all : std::min(most, all);
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps(kProfAttnStep, st);
    const int es = dtype_size(dt);
    const HeadsView q{(unsigned char*)d_q, ld_q * es, hs_q * es}, out{(unsigned char*)d_out, ld_out * es, hs_out * es};
#define FX_RUN(DT, E) k_attention_step<DT, E><<<(unsigned)(rows * heads), 64, 0, st>>>(a, rows, most, heads, scale, q, out, d_lse)
    FX_RUN_TYPES();
#undef FX_RUN
    FX_HIP_TRY(hipGetLastError());
    return FX_OK;
}
