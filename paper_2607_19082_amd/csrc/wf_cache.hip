// The 4-bit key/value cache: its plan, and the kernels that quantise tokens
// into its pages and read them back.  Layout and format: wf_cache.h.
#include <cmath>
#include <new>

#include "wf_cache.h"

namespace wf {

constexpr int kKvThreads = 256;

// ---- kernels ----------------------------------------------------------------

// The head's record that holds token `pos`, or null with the reason in the
// error word.
template <int DP>
__device__ __forceinline__ uint8_t* kv_record(const KvCache& c, const int* table, int table_pages, int b, int head, int pos) {
    const int at = pos >> c.page_shift;
    if (pos < 0 || at >= table_pages) {
        atomicOr(c.err, kErrKvRange);
        return nullptr;
    }
    const int page = table[(size_t)b * table_pages + at];
    if (page < 0 || page >= c.pages) {
        atomicOr(c.err, kErrKvPage);
        return nullptr;
    }
    return c.pool + (size_t)page * c.page_bytes() + (size_t)head * c.head_bytes() +
           (size_t)((pos & ((1 << c.page_shift) - 1)) / kKvTile) * KvLayout<DP>::kRecord;
}

template <class T>
__device__ __forceinline__ void load8(const T* p, int m, float (&x)[8]) {
    if (m >= 8) {
        T t[8];
        __builtin_memcpy(t, p, sizeof t);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)t[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < m ? (float)p[e] : 0.0f;
    }
}

template <class T>
__device__ __forceinline__ void store8(T* p, int m, const float (&x)[8]) {
    if (m >= 8) {
        T t[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = (T)x[e];
        __builtin_memcpy(p, t, sizeof t);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < m) p[e] = (T)x[e];
    }
}

// One lane quantises eight channels; four lanes share a block.
template <int DP, class T>
__global__ __launch_bounds__(kKvThreads) void k_kv_write(KvCache c, KvRows k, KvRows v, KvTokens a) {
    using L = KvLayout<DP>;
    constexpr int W = DP / 8;
    const long long id = (long long)blockIdx.x * kKvThreads + threadIdx.x;
    const int w = id % W;
    const long long r = id / W;
    const int head = r % c.heads;
    const long long bi = r / c.heads;
    const int i = bi % a.n, b = bi / a.n;
    const bool value = blockIdx.y;
    uint8_t* base = nullptr;
    int pos = 0;
    float x[8] = {};
    if (b < a.B && i < (a.counts ? a.counts[b] : a.n)) {
        pos = a.first[b] + i;
        base = kv_record<DP>(c, a.table, a.table_pages, b, head, pos);
        const KvRows& s = value ? v : k;
        load8((const T*)s.p + b * s.sb + i * s.sr + head * s.sh + w * 8, c.dim - w * 8, x);
    }
    // the bits of |x| order as the values do; a NaN's lie above infinity's
    unsigned top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __builtin_bit_cast(unsigned, x[e]) & 0x7fffffffu);
    top = max(top, (unsigned)__shfl_xor((int)top, 1));
    top = max(top, (unsigned)__shfl_xor((int)top, 2));
    if (!base) return;
    // the smallest power with 6 * 2^e >= top: 6 is 1.5 * 2^2, so e is top's
    // exponent less 2, and one more where its mantissa is above 1.5
    const bool nan = top >= 0x7f800000u;
    int e = (int)((top + 0x3fffffu) >> 23) - 129;
    e = nan || e < -kKvMaxPower ? -kKvMaxPower : (e > kKvMaxPower ? kKvMaxPower : e);
    const float inv = __builtin_bit_cast(float, (unsigned)(127 - e) << 23);   // exact: a power of two
    unsigned code = 0;
    if (!nan) {
        // round to nearest even, saturating at 6
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[0] * inv, x[1] * inv, 1.0f, 0);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[2] * inv, x[3] * inv, 1.0f, 1);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[4] * inv, x[5] * inv, 1.0f, 2);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[6] * inv, x[7] * inv, 1.0f, 3);
    }
    const int t = pos & (kKvTile - 1);
    const uint8_t power = nan ? kKvNan : e + 127;
    if (!value) {
        *(unsigned*)(base + L::key_word(t, w)) = code;
        if (w % 4 == 0) base[L::key_power(t, w / 4)] = power;
    } else {
        uint8_t* at = base + L::value_word(t, w);
        if constexpr (L::kRows == 4) {
            *(uint16_t*)at = (uint16_t)code;
            *(uint16_t*)(at + 16) = (uint16_t)(code >> 16);
        } else {
            *(unsigned*)at = code;
        }
        if (w % 4 == 0) base[L::value_power(t, w / 4)] = power;
    }
}

// One lane reads eight channels back.  Tokens past a sequence's count, and
// those that the table does not reach, are zeros.
template <int DP, class T>
__global__ __launch_bounds__(kKvThreads) void k_kv_read(KvCache c, KvRows k, KvRows v, KvTokens a) {
    using L = KvLayout<DP>;
    typedef float f2 __attribute__((ext_vector_type(2)));
    constexpr int W = DP / 8;
    const long long id = (long long)blockIdx.x * kKvThreads + threadIdx.x;
    const int w = id % W;
    const long long r = id / W;
    const int head = r % c.heads;
    const long long bi = r / c.heads;
    const int i = bi % a.n, b = bi / a.n;
    const bool value = blockIdx.y;
    if (b >= a.B || w * 8 >= c.dim) return;
    const KvRows& s = value ? v : k;
    T* out = (T*)s.p + b * s.sb + i * s.sr + head * s.sh + w * 8;
    float x[8] = {};
    if (i < (a.counts ? a.counts[b] : a.n)) {
        const int pos = a.first[b] + i, t = pos & (kKvTile - 1);
        const uint8_t* base = kv_record<DP>(c, a.table, a.table_pages, b, head, pos);
        if (base) {
            unsigned code, power;
            if (!value) {
                code = *(const unsigned*)(base + L::key_word(t, w));
                power = base[L::key_power(t, w / 4)];
            } else {
                const uint8_t* at = base + L::value_word(t, w);
                if constexpr (L::kRows == 4) code = *(const uint16_t*)at | (unsigned)*(const uint16_t*)(at + 16) << 16;
                else code = *(const unsigned*)at;
                power = base[L::value_power(t, w / 4)];
            }
            const float scale = __builtin_bit_cast(float, power << 23);   // 255: the conversion gives NaN
#define WF_PAIR(j)                                                                    \
    {                                                                                 \
        const f2 y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, j);        \
        x[2 * j] = y[0];                                                              \
        x[2 * j + 1] = y[1];                                                          \
    }
            WF_PAIR(0) WF_PAIR(1) WF_PAIR(2) WF_PAIR(3)
#undef WF_PAIR
        }
    }
    store8(out, c.dim - w * 8, x);
}

template <int DP, class T>
static void launch_kv(bool write, const KvCache& c, const KvRows& k, const KvRows& v, const KvTokens& a, hipStream_t st) {
    const long long lanes = (long long)a.B * a.n * c.heads * (DP / 8);
    const dim3 grid((unsigned)((lanes + kKvThreads - 1) / kKvThreads), 2);
    if (write) hipLaunchKernelGGL((k_kv_write<DP, T>), grid, dim3(kKvThreads), 0, st, c, k, v, a);
    else hipLaunchKernelGGL((k_kv_read<DP, T>), grid, dim3(kKvThreads), 0, st, c, k, v, a);
}

template <class T>
static void launch_kv_dp(bool write, const KvCache& c, const KvRows& k, const KvRows& v, const KvTokens& a, hipStream_t st) {
    if (c.dp == 64) launch_kv<64, T>(write, c, k, v, a, st);
    else if (c.dp == 128) launch_kv<128, T>(write, c, k, v, a, st);
    else launch_kv<256, T>(write, c, k, v, a, st);
}

void launch_kv_write(const KvCache& c, int precision, const KvRows& k, const KvRows& v, const KvTokens& a, hipStream_t st) {
    if (precision == WF_BF16) launch_kv_dp<__bf16>(true, c, k, v, a, st);
    else launch_kv_dp<float>(true, c, k, v, a, st);
}

void launch_kv_read(const KvCache& c, int precision, const KvRows& k, const KvRows& v, const KvTokens& a, hipStream_t st) {
    if (precision == WF_BF16) launch_kv_dp<__bf16>(false, c, k, v, a, st);
    else launch_kv_dp<float>(false, c, k, v, a, st);
}

// ---- plan and entry points ------------------------------------------------------

struct Cache {
    KvCache c{};
    float* work = nullptr;           // partial results of split attention calls
};

static int kv_fail(hipError_t e, const char* what) { return fail(WF_E_HIP, std::string(what) + ": " + hipGetErrorString(e)); }

static void free_cache(Cache* c) {
    if (!c) return;
    if (c->c.pool) (void)hipFree(c->c.pool);
    if (c->c.err) (void)hipFree(c->c.err);
    if (c->work) (void)hipFree(c->work);
    delete c;
}

// Rows of a call: the strides are in elements and the channels contiguous.
static int kv_rows(const wf_rows* r, int precision, const char* name, KvRows* out) {
    if (!r || !r->data) return fail(WF_E_INVALID, std::string(name) + " is NULL");
    if ((uintptr_t)r->data % (precision == WF_BF16 ? 2 : 4)) return fail(WF_E_INVALID, std::string(name) + " is not aligned to its element");
    *out = {r->data, r->stride[0], r->stride[1], r->stride[2]};
    return WF_OK;
}

static int kv_tokens(const Cache* c, int precision, int B, int n, const int32_t* table, int table_pages, const int32_t* first,
                     const int32_t* counts, KvTokens* out) {
    if (!c) return fail(WF_E_INVALID, "cache is NULL");
    if (precision != WF_FP32 && precision != WF_BF16) return fail(WF_E_INVALID, "unknown precision");
    if (B < 0 || n < 0 || table_pages < 0) return fail(WF_E_INVALID, "B, n and table_pages must not be negative");
    if (B && n && (!table || !first)) return fail(WF_E_INVALID, "table or first is NULL");
    if ((long long)B * n * c->c.heads * (c->c.dp / 8) / kKvThreads >= 0x7fffffffLL)
        return fail(WF_E_UNSUPPORTED, "more than 2^39 channels in one call");
    *out = {table, first, counts, table_pages, B, n};
    return WF_OK;
}

static int kv_launched(const char* what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? WF_OK : kv_fail(e, what);
}

}  // namespace wf

using namespace wf;

extern "C" {

int wf_cache_plan(const wf_cache_desc* d, wf_cache_t* out) {
    if (!out) return fail(WF_E_INVALID, "out is NULL");
    *out = nullptr;
    if (!d) return fail(WF_E_INVALID, "desc is NULL");
    if (d->heads < 1 || d->pages < 1) return fail(WF_E_INVALID, "heads and pages must be positive");
    if (d->heads > 4096) return fail(WF_E_UNSUPPORTED, "more than 4096 heads");
    if (d->dim < 8 || d->dim > 256 || d->dim % 8) return fail(WF_E_UNSUPPORTED, "dim must be a multiple of 8 in [8, 256]");
    if (d->page < 32 || d->page > 1024 || (d->page & (d->page - 1)))
        return fail(WF_E_UNSUPPORTED, "page must be a power of two in [32, 1024]");
    Cache* c = new (std::nothrow) Cache();
    if (!c) return fail(WF_E_NOMEM, "host allocation");
    KvCache& k = c->c;
    k.heads = d->heads; k.dim = d->dim; k.pages = d->pages;
    k.dp = d->dim <= 64 ? 64 : (d->dim <= 128 ? 128 : 256);
    while ((1 << k.page_shift) < d->page) ++k.page_shift;
    const size_t bytes = k.page_bytes() * k.pages;
    hipError_t e = hipMalloc((void**)&k.pool, bytes);
    if (e == hipSuccess) e = hipMalloc((void**)&k.err, sizeof(int));
    if (e == hipSuccess) e = hipMalloc((void**)&c->work, (size_t)kAttendWorkRows * (k.dp + 2) * sizeof(float));
    if (e != hipSuccess) {
        free_cache(c);
        return fail(WF_E_NOMEM, std::string("cache: ") + hipGetErrorString(e));
    }
    // a page that is never written reads as zeros
    e = hipMemset(k.pool, 0, bytes);
    if (e == hipSuccess) e = hipMemset(k.err, 0, sizeof(int));
    if (e == hipSuccess) e = hipDeviceSynchronize();
    if (e != hipSuccess) {
        free_cache(c);
        return kv_fail(e, "cache fill");
    }
    *out = reinterpret_cast<wf_cache_t>(c);
    return WF_OK;
}

void wf_cache_destroy(wf_cache_t cache) { free_cache(reinterpret_cast<Cache*>(cache)); }

int wf_cache_write(wf_cache_t cache, int32_t precision, const wf_rows* k, const wf_rows* v, int32_t B, int32_t n,
                   const int32_t* table, int32_t table_pages, const int32_t* first, const int32_t* counts, hipStream_t stream) {
    const Cache* c = reinterpret_cast<Cache*>(cache);
    KvTokens a;
    KvRows kr, vr;
    int rc = kv_tokens(c, precision, B, n, table, table_pages, first, counts, &a);
    if (rc != WF_OK || !B || !n) return rc;
    if ((rc = kv_rows(k, precision, "k", &kr)) != WF_OK || (rc = kv_rows(v, precision, "v", &vr)) != WF_OK) return rc;
    launch_kv_write(c->c, precision, kr, vr, a, stream);
    return kv_launched("wf_cache_write");
}

int wf_cache_read(wf_cache_t cache, int32_t precision, const wf_rows* k, const wf_rows* v, int32_t B, int32_t n,
                  const int32_t* table, int32_t table_pages, const int32_t* first, const int32_t* counts, hipStream_t stream) {
    const Cache* c = reinterpret_cast<Cache*>(cache);
    KvTokens a;
    KvRows kr, vr;
    int rc = kv_tokens(c, precision, B, n, table, table_pages, first, counts, &a);
    if (rc != WF_OK || !B || !n) return rc;
    if ((rc = kv_rows(k, precision, "k", &kr)) != WF_OK || (rc = kv_rows(v, precision, "v", &vr)) != WF_OK) return rc;
    launch_kv_read(c->c, precision, kr, vr, a, stream);
    return kv_launched("wf_cache_read");
}

int wf_cache_attend(wf_cache_t cache, int32_t precision, const wf_rows* q, const wf_rows* out, int32_t B, int32_t n,
                    int32_t q_heads, const int32_t* table, int32_t table_pages, const int32_t* visible,
                    const uint8_t* mask, const int64_t* mask_stride, int32_t max_visible, float scale, hipStream_t stream) {
    const Cache* c = reinterpret_cast<Cache*>(cache);
    if (!c) return fail(WF_E_INVALID, "cache is NULL");
    if (precision != WF_FP32 && precision != WF_BF16) return fail(WF_E_INVALID, "unknown precision");
    if (B < 0 || n < 0 || table_pages < 0) return fail(WF_E_INVALID, "B, n and table_pages must not be negative");
    if (q_heads < 1 || q_heads % c->c.heads) return fail(WF_E_INVALID, "q_heads must be a positive multiple of the cache's heads");
    if (!(scale > 0.0f) || !std::isfinite(scale)) return fail(WF_E_INVALID, "scale must be positive and finite");
    if (max_visible < 0 || max_visible > (long long)table_pages << c->c.page_shift)
        return fail(WF_E_INVALID, "max_visible must lie in [0, table_pages * page]");
    if (mask && !mask_stride) return fail(WF_E_INVALID, "mask_stride is NULL");
    if (!B || !n) return WF_OK;
    if (!visible || (max_visible && !table)) return fail(WF_E_INVALID, "visible or table is NULL");
    AttendArgs a{};
    int rc;
    if ((rc = kv_rows(q, precision, "q", &a.q)) != WF_OK || (rc = kv_rows(out, precision, "out", &a.o)) != WF_OK) return rc;
    if ((long long)n * (q_heads / c->c.heads) >= 1 << 30 || (long long)B * n * q_heads >= 1LL << 31)
        return fail(WF_E_UNSUPPORTED, "more than 2^31 query rows in one call");
    a.c = c->c;
    a.table = table; a.visible = visible; a.mask = mask;
    if (mask) { a.mb = mask_stride[0]; a.mr = mask_stride[1]; }
    a.table_pages = table_pages; a.B = B; a.n = n; a.group = q_heads / c->c.heads;
    a.max_visible = max_visible;
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    attend_plan(a, precision);
    a.part_o = c->work;
    a.part_ml = c->work + (size_t)kAttendWorkRows * c->c.dp;
    launch_attend(a, precision, stream);
    return kv_launched("wf_cache_attend");
}

int wf_cache_sync(wf_cache_t cache, hipStream_t stream) {
    Cache* c = reinterpret_cast<Cache*>(cache);
    if (!c) return fail(WF_E_INVALID, "cache is NULL");
    int err = 0;
    hipError_t e = hipStreamSynchronize(stream);
    if (e == hipSuccess) e = hipMemcpy(&err, c->c.err, sizeof err, hipMemcpyDeviceToHost);
    if (e == hipSuccess && err) e = hipMemset(c->c.err, 0, sizeof err);
    if (e != hipSuccess) return kv_fail(e, "wf_cache_sync");
    if (err & kErrKvPage) return fail(WF_E_INVALID, "a page table entry lies outside the pool");
    if (err & kErrKvRange) return fail(WF_E_CAPACITY, "a token lies past its page table, or a row sees more than max_visible tokens");
    return WF_OK;
}

}  // extern "C"
