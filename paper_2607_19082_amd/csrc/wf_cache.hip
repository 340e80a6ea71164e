// The 4-bit key/value cache: its plan, and the kernels that quantise tokens
// into its pages and read them back.  Layout and format: wf_cache.h.
#include <atomic>
#include <cmath>
#include <new>

#include "wf_cache.h"

namespace wf {

typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef float f2 __attribute__((ext_vector_type(2)));

constexpr int kKvThreads = 256;

// ---- kernels ----------------------------------------------------------------

// What a workgroup writes or reads: one record of one head, the tokens of it
// that the call takes.  Records are the cache's, not the call's, so that a wave
// takes tokens whose bytes lie together whatever the call's first token is.
struct KvWork {
    uint8_t* record;                 // null: not to be touched, `reason` says why
    int b, head, reason;
    long long i0;                    // the call's token at the record's start, which may be before its first
    int count;
};

template <int DP>
__device__ __forceinline__ KvWork kv_work(const KvCache& c, const KvTokens& a) {
    const int block = blockIdx.x, above = a.heads_(block), b = a.records_(above);
    const int head = block - above * c.heads, rec = above - b * a.records;
    const int first = a.first[b], count = a.counts ? min(a.counts[b], a.n) : a.n;
    const long long at = (long long)(first >> 5) + rec;            // the record's place in the sequence
    KvWork w{nullptr, b, head, 0, at * kKvTile - first, count};
    const int per_page = c.page_shift - 5;
    if (at < 0 || at >> per_page >= a.table_pages) {
        w.reason = kErrKvRange;
        return w;
    }
    const int page = a.table[(size_t)b * a.table_pages + (at >> per_page)];
    if (page < 0 || page >= c.pages) {
        w.reason = kErrKvPage;
        return w;
    }
    w.record = c.pool + (size_t)page * c.page_bytes() + (size_t)head * c.head_bytes() +
               (size_t)(at & ((1 << per_page) - 1)) * KvLayout<DP>::kRecord;
    return w;
}

// Eight channels of which m exist.
template <class T>
__device__ __forceinline__ void load8(const T* p, int m, float (&x)[8]) {
    if (m >= 8) {
        T t[8];
        __builtin_memcpy(t, p, sizeof t);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)t[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.0f;
    }
}

// The power byte of a block whose largest magnitude has the bits `top`, and
// the factor 2^-e.  The smallest power with 6 * 2^e >= top: 6 is 1.5 * 2^2, so
// e is top's exponent less 2, and one more where its mantissa is above 1.5.
__device__ __forceinline__ unsigned kv_power(unsigned top, float& inv) {
    const bool nan = top >= 0x7f800000u;
    int e = (int)((top + 0x3fffffu) >> 23) - 129;
    e = top == 0 ? 0 : (e < -kKvMaxPower ? -kKvMaxPower : (e > kKvMaxPower ? kKvMaxPower : e));
    inv = nan ? 0.0f : __builtin_bit_cast(float, (unsigned)(127 - e) << 23);   // exact: a power of two
    return nan ? kKvNan : e + 127;
}

// Eight channels as 4-bit codes, rounded to the nearest (a tie to the even
// code) and cut off at 6; a block that is not finite holds zeros.
__device__ __forceinline__ unsigned kv_code(const float (&x)[8], float inv) {
    unsigned code = 0;
    if (inv == 0.0f) return code;
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[0] * inv, x[1] * inv, 1.0f, 0);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[2] * inv, x[3] * inv, 1.0f, 1);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[4] * inv, x[5] * inv, 1.0f, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[6] * inv, x[7] * inv, 1.0f, 3);
}

// Lanes take eight channels of a token each, the token's first, then the next
// token: four lanes share a block, and find its largest magnitude in two
// exchanges.  Bound by memory: two prompts of 8191 tokens, 8 heads of 128 in
// bf16, take 17 us for 67 MB read and 18 written, 5.0 TB/s; a token 3.6 us, the
// chain of its loads.
template <int DP, class T>
__global__ __launch_bounds__(kKvThreads) void k_kv_write(KvCache c, KvRows k, KvRows v, KvTokens a) {
    using L = KvLayout<DP>;
    constexpr int W = DP / 8, N = kKvTile * W / kKvThreads;        // words of a token; a lane's tokens
    const KvWork o = kv_work<DP>(c, a);
    const int w = threadIdx.x % W;
    float x[2][N][8];
    bool on[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int t = (j * kKvThreads + threadIdx.x) / W;
        const long long i = o.i0 + t;
        on[j] = i >= 0 && i < o.count;
        if (on[j] && o.record) {
            load8((const T*)k.p + o.b * k.sb + i * k.sr + o.head * k.sh + w * 8, c.dim - w * 8, x[0][j]);
            load8((const T*)v.p + o.b * v.sb + i * v.sr + o.head * v.sh + w * 8, c.dim - w * 8, x[1][j]);
        } else {
            if (on[j]) atomicOr(c.err, o.reason);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[0][j][e] = x[1][j][e] = 0.0f;
        }
    }
    if (!o.record) return;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int t = (j * kKvThreads + threadIdx.x) / W;
        unsigned code[2], power[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            // the bits of |x| order as the values do; a NaN's lie above infinity's
            int top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __builtin_bit_cast(int, x[s][j][e]) & 0x7fffffff);
            top = lanes4(top, [](int a, int b) { return max(a, b); });
            float inv;
            power[s] = kv_power((unsigned)top, inv);
            code[s] = kv_code(x[s][j], inv);
        }
        uint8_t* at = o.record + L::value_at(t, w * 8);
        if constexpr (L::kRows == 4) {
            // a word is half of two lanes' runs: where the token beside this
            // one is written too, the pair of lanes swaps halves
            const unsigned other = (unsigned)__shfl_xor((int)code[1], W);
            const bool both = __shfl_xor((int)on[j], W);
            if (on[j]) {
                if (both) {
                    if (t % 2 == 0) *(unsigned*)at = (code[1] & 0xffff) | other << 16;
                    else *(unsigned*)(at + 14) = other >> 16 | (code[1] & 0xffff0000u);
                } else {
                    *(uint16_t*)at = (uint16_t)code[1];
                    *(uint16_t*)(at + 16) = (uint16_t)(code[1] >> 16);
                }
            }
        } else if (on[j]) {
            *(unsigned*)at = code[1];
        }
        if (on[j]) {
            *(unsigned*)(o.record + L::key_at(t, w * 8)) = code[0];
            if (w % 4 == 0) {
                o.record[L::key_power(t, w / 4)] = (uint8_t)power[0];
                o.record[L::value_power(t, w / 4)] = (uint8_t)power[1];
            }
        }
    }
}

// The same tokens read back, 16 bytes of a token a lane.  Those past a
// sequence's count, and those that the table does not reach, are zeros.
// STREAM, for aligned rows: stores that pass the caches by.  Written through
// them, 8 heads of 128 in bf16 take 9.7 us for 4096 tokens and 37.6 for 32768;
// past them 5.6 and 27.1, more than what a kernel that reads the result next
// then loses (1.2 and 4.4 us).
template <int DP, class T, bool STREAM>
__global__ __launch_bounds__(kKvThreads) void k_kv_read(KvCache c, KvRows k, KvRows v, KvTokens a) {
    using L = KvLayout<DP>;
    constexpr int C = 16 / sizeof(T), W = DP / C, N = kKvTile * W / kKvThreads;   // channels of a lane; lanes of a token
    const KvWork o = kv_work<DP>(c, a);
    const int d = threadIdx.x % W * C;
    unsigned code[2][N], power[2][N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int t = (j * kKvThreads + threadIdx.x) / W;
        const long long i = o.i0 + t;
        code[0][j] = code[1][j] = power[0][j] = power[1][j] = 0;
        if (i < 0 || i >= o.count) continue;
        if (!o.record) {
            atomicOr(c.err, o.reason);
            continue;
        }
        const uint8_t *kp = o.record + L::key_at(t, d), *vp = o.record + L::value_at(t, d);
        if constexpr (C == 4) {
            code[0][j] = *(const uint16_t*)kp;
            code[1][j] = *(const uint16_t*)vp;
        } else {
            code[0][j] = *(const unsigned*)kp;
            if constexpr (L::kRows == 4) code[1][j] = *(const uint16_t*)vp | (unsigned)*(const uint16_t*)(vp + 16) << 16;
            else code[1][j] = *(const unsigned*)vp;
        }
        power[0][j] = o.record[L::key_power(t, d / kKvBlock)];
        power[1][j] = o.record[L::value_power(t, d / kKvBlock)];
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int t = (j * kKvThreads + threadIdx.x) / W;
        const long long i = o.i0 + t;
        if (i < 0 || i >= a.n || d >= c.dim) continue;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const KvRows& r = s ? v : k;
            const float scale = __builtin_bit_cast(float, power[s][j] << 23);   // 255: the conversion gives NaN
            T x[C];
            auto two = [&](int e, const f2& y) {
                x[e] = (T)y[0];
                x[e + 1] = (T)y[1];
            };
            two(0, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[s][j], scale, 0));
            two(2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[s][j], scale, 1));
            if constexpr (C == 8) {
                two(4, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[s][j], scale, 2));
                two(6, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[s][j], scale, 3));
            }
            T* out = (T*)r.p + o.b * r.sb + i * r.sr + o.head * r.sh + d;
            if constexpr (STREAM) {
                u4 u;
                __builtin_memcpy(&u, x, 16);
                __builtin_nontemporal_store(u, (u4*)out);
            } else {
                __builtin_memcpy(out, x, 16);
            }
        }
    }
}

template <int DP, class T>
static void launch_kv(bool write, const KvCache& c, const KvRows& k, const KvRows& v, const KvTokens& a, hipStream_t st) {
    const dim3 grid((unsigned)((long long)a.B * a.records * c.heads));
    auto aligned = [](const KvRows& r) {
        return ((uintptr_t)r.p | (uintptr_t)((r.sb | r.sr | r.sh) * sizeof(T))) % 16 == 0;
    };
    if (write) hipLaunchKernelGGL((k_kv_write<DP, T>), grid, dim3(kKvThreads), 0, st, c, k, v, a);
    else if (aligned(k) && aligned(v)) hipLaunchKernelGGL((k_kv_read<DP, T, true>), grid, dim3(kKvThreads), 0, st, c, k, v, a);
    else hipLaunchKernelGGL((k_kv_read<DP, T, false>), grid, dim3(kKvThreads), 0, st, c, k, v, a);
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

// Takes the error word: what kernels on other streams record meanwhile is
// either taken or stays for the next time.
__global__ void k_kv_take_errors(int* err, int* out) { *out = atomicExch(err, 0); }

// ---- plan and entry points ------------------------------------------------------

constexpr unsigned kKvHead = 256, kKvTaken = kKvHead / sizeof(int) - 1;   // (that many syncs may be under way together)

struct Cache {
    KvCache c{};
    int device = 0;                  // its memory's, on which its kernels run
    // one allocation: the error word and kKvTaken words that syncs take it to, the
    // pool, the workspace
    void* memory = nullptr;
    std::atomic<unsigned> syncs{0};
    float* work = nullptr;           // partial results of split attention calls
};

static void free_cache(Cache* c) {
    if (!c) return;
    if (c->memory) (void)hipFree(c->memory);
    delete c;
}

static int kv_tokens(const Cache* c, int precision, int B, int n, const int32_t* table, int table_pages, const int32_t* first,
                     const int32_t* counts, KvTokens* out) {
    if (!c) return fail(WF_E_INVALID, "cache is NULL");
    if (precision != WF_FP32 && precision != WF_BF16) return fail(WF_E_INVALID, "unknown precision");
    if (B < 0 || n < 0 || table_pages < 0) return fail(WF_E_INVALID, "B, n and table_pages must not be negative");
    if (B && n && (!table || !first)) return fail(WF_E_INVALID, "table or first is NULL");
    // records that n tokens may reach into, wherever the first one lies
    const long long records = ((long long)n + 2 * (kKvTile - 1)) / kKvTile;
    if (B * records * c->c.heads * kKvThreads >= 1LL << 32) return fail(WF_E_UNSUPPORTED, "2^24 or more records in one call");
    *out = {table, first, counts, table_pages, B, n, (int)records, {}, {}};
    out->heads_.by(c->c.heads);
    out->records_.by((unsigned)records);
    return WF_OK;
}

// What the attention calls have in common: their checks, and the arguments but
// for the split.
static int kv_attend(const Cache* c, int precision, const wf_rows* q, const wf_rows* out, int B, int n, int q_heads, const int32_t* table,
                     int table_pages, const int32_t* visible, int max_visible, float scale, AttendArgs* to) {
    AttendArgs& a = *to;
    if (!c) return fail(WF_E_INVALID, "cache is NULL");
    if (precision != WF_FP32 && precision != WF_BF16) return fail(WF_E_INVALID, "unknown precision");
    if (B < 0 || n < 0 || table_pages < 0) return fail(WF_E_INVALID, "B, n and table_pages must not be negative");
    if (q_heads < 1 || q_heads % c->c.heads) return fail(WF_E_INVALID, "q_heads must be a positive multiple of the cache's heads");
    if (!(scale > 0.0f) || !std::isfinite(scale)) return fail(WF_E_INVALID, "scale must be positive and finite");
    if (max_visible < 0 || max_visible > (long long)table_pages << c->c.page_shift)
        return fail(WF_E_INVALID, "max_visible must lie in [0, table_pages * page]");
    // the kernel counts tokens in 32 bits, up to the end of the last one's tile and the next
    if (max_visible > INT32_MAX - 2 * kKvTile) return fail(WF_E_UNSUPPORTED, "max_visible is beyond 2^31 - 65");
    if (!B || !n) return WF_OK;
    if (!visible || (max_visible && !table)) return fail(WF_E_INVALID, "visible or table is NULL");
    int rc;
    if ((rc = kv_rows(q, precision, "q", &a.q)) != WF_OK || (rc = kv_rows(out, precision, "out", &a.o)) != WF_OK) return rc;
    if ((long long)n * (q_heads / c->c.heads) >= 1 << 30 || (long long)B * n * q_heads >= 1LL << 31)
        return fail(WF_E_UNSUPPORTED, "more than 2^31 query rows in one call");
    a.c = c->c;
    a.table = table; a.visible = visible;
    a.table_pages = table_pages; a.B = B; a.n = n; a.group = q_heads / c->c.heads;
    a.max_visible = max_visible;
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.part_o = c->work;
    a.part_ml = c->work + attend_work_rows(c->c.dp) * c->c.dp;
    return WF_OK;
}

}  // namespace wf

using namespace wf;

extern "C" {

// (a message that cannot be built is the one thing that throws in these)

int wf_cache_plan(const wf_cache_desc* d, wf_cache_t* out) try {
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
    // (a record is a multiple of 64 bytes)
    const size_t head = kKvHead, pool = (k.page_bytes() * k.pages + 255) / 256 * 256;
    const size_t work = attend_work_rows(k.dp) * (k.dp + 2) * sizeof(float);
    hipError_t e = hipGetDevice(&c->device);
    if (e != hipSuccess) {
        free_cache(c);
        return kv_fail(e, "hipGetDevice");
    }
    e = hipMalloc(&c->memory, head + pool + work);
    if (e != hipSuccess) {
        (void)hipGetLastError();     // reported here, not by the next launch
        c->memory = nullptr;
        free_cache(c);
        return fail(WF_E_NOMEM, std::string("cache: ") + hipGetErrorString(e));
    }
    k.err = static_cast<int*>(c->memory);
    k.pool = static_cast<uint8_t*>(c->memory) + head;
    c->work = reinterpret_cast<float*>(k.pool + pool);
    // no error, and a page that is never written reads as zeros
    e = hipMemset(c->memory, 0, head + pool);
    if (e == hipSuccess) e = hipDeviceSynchronize();
    if (e != hipSuccess) {
        free_cache(c);
        return kv_fail(e, "cache fill");
    }
    *out = reinterpret_cast<wf_cache_t>(c);
    return WF_OK;
} catch (...) {
    return WF_E_NOMEM;
}

void wf_cache_destroy(wf_cache_t cache) { free_cache(reinterpret_cast<Cache*>(cache)); }

int wf_cache_write(wf_cache_t cache, int32_t precision, const wf_rows* k, const wf_rows* v, int32_t B, int32_t n,
                   const int32_t* table, int32_t table_pages, const int32_t* first, const int32_t* counts, hipStream_t stream) try {
    const Cache* c = reinterpret_cast<Cache*>(cache);
    KvTokens a;
    KvRows kr, vr;
    int rc = kv_tokens(c, precision, B, n, table, table_pages, first, counts, &a);
    if (rc != WF_OK || !B || !n) return rc;
    if ((rc = kv_rows(k, precision, "k", &kr)) != WF_OK || (rc = kv_rows(v, precision, "v", &vr)) != WF_OK) return rc;
    const OnDevice on(c->device);
    if (on.error() != hipSuccess) return kv_fail(on.error(), "the cache's device");
    launch_kv_write(c->c, precision, kr, vr, a, stream);
    return kv_launched("wf_cache_write");
} catch (...) {
    return WF_E_NOMEM;
}

int wf_cache_read(wf_cache_t cache, int32_t precision, const wf_rows* k, const wf_rows* v, int32_t B, int32_t n,
                  const int32_t* table, int32_t table_pages, const int32_t* first, const int32_t* counts, hipStream_t stream) try {
    const Cache* c = reinterpret_cast<Cache*>(cache);
    KvTokens a;
    KvRows kr, vr;
    int rc = kv_tokens(c, precision, B, n, table, table_pages, first, counts, &a);
    if (rc != WF_OK || !B || !n) return rc;
    if ((rc = kv_rows(k, precision, "k", &kr)) != WF_OK || (rc = kv_rows(v, precision, "v", &vr)) != WF_OK) return rc;
    const OnDevice on(c->device);
    if (on.error() != hipSuccess) return kv_fail(on.error(), "the cache's device");
    launch_kv_read(c->c, precision, kr, vr, a, stream);
    return kv_launched("wf_cache_read");
} catch (...) {
    return WF_E_NOMEM;
}

int wf_cache_attend(wf_cache_t cache, int32_t precision, const wf_rows* q, const wf_rows* out, int32_t B, int32_t n,
                    int32_t q_heads, const int32_t* table, int32_t table_pages, const int32_t* visible,
                    const uint8_t* mask, const int64_t* mask_stride, int32_t max_visible, float scale, hipStream_t stream) try {
    const Cache* c = reinterpret_cast<Cache*>(cache);
    if (mask && !mask_stride) return fail(WF_E_INVALID, "mask_stride is NULL");
    AttendArgs a{};
    int rc = kv_attend(c, precision, q, out, B, n, q_heads, table, table_pages, visible, max_visible, scale, &a);
    if (rc != WF_OK || !B || !n) return rc;
    a.mask = mask;
    if (mask) { a.mb = mask_stride[0]; a.mr = mask_stride[1]; }
    if (attend_plan(a, precision) >= 1LL << 32) return fail(WF_E_UNSUPPORTED, "2^32 or more threads in one call");
    const OnDevice on(c->device);
    if (on.error() != hipSuccess) return kv_fail(on.error(), "the cache's device");
    launch_attend(a, precision, stream);
    return kv_launched("wf_cache_attend");
} catch (...) {
    return WF_E_NOMEM;
}

int wf_cache_attend_window(wf_cache_t cache, int32_t precision, const wf_rows* q, const wf_rows* out, int32_t B, int32_t n,
                           int32_t q_heads, const int32_t* table, int32_t table_pages, const int32_t* visible, int32_t window,
                           int32_t sinks, int32_t max_visible, float scale, hipStream_t stream) try {
    const Cache* c = reinterpret_cast<Cache*>(cache);
    if (window < 1 || sinks < 0) return fail(WF_E_INVALID, "window must be positive and sinks not negative");
    AttendRunsArgs a{};
    int rc = kv_attend(c, precision, q, out, B, n, q_heads, table, table_pages, visible, max_visible, scale, &a);
    if (rc != WF_OK || !B || !n) return rc;
    a.window = window;
    a.sinks = sinks < max_visible ? sinks : max_visible;
    // (where every row sees all that is visible, the window has no part in it)
    const bool all = (long long)window + sinks >= max_visible;
    if ((all ? attend_plan(a, precision) : attend_window_plan(a, precision)) >= 1LL << 32)
        return fail(WF_E_UNSUPPORTED, "2^32 or more threads in one call");
    const OnDevice on(c->device);
    if (on.error() != hipSuccess) return kv_fail(on.error(), "the cache's device");
    if (all) launch_attend(a, precision, stream);
    else launch_attend_window(a, precision, stream);
    return kv_launched("wf_cache_attend_window");
} catch (...) {
    return WF_E_NOMEM;
}

int wf_cache_attend_shared(wf_cache_t cache, int32_t precision, const wf_rows* q, const wf_rows* out, int32_t B, int32_t n,
                           int32_t q_heads, const int32_t* prefix_table, int32_t prefix_pages, const int32_t* prefix_visible,
                           int32_t max_prefix, const int32_t* table, int32_t table_pages, const int32_t* visible,
                           int32_t max_visible, float scale, hipStream_t stream) try {
    const Cache* c = reinterpret_cast<Cache*>(cache);
    AttendRunsArgs a{};
    int rc = kv_attend(c, precision, q, out, B, n, q_heads, table, table_pages, visible, max_visible, scale, &a);
    if (rc != WF_OK) return rc;
    if (prefix_pages < 0) return fail(WF_E_INVALID, "prefix_pages must not be negative");
    if (max_prefix < 0 || max_prefix > (long long)prefix_pages << c->c.page_shift)
        return fail(WF_E_INVALID, "max_prefix must lie in [0, prefix_pages * page]");
    // tiles of both runs are counted together, in tokens
    if ((long long)max_prefix + max_visible > INT32_MAX - 4 * kKvTile)
        return fail(WF_E_UNSUPPORTED, "max_prefix and max_visible are together beyond 2^31 - 129");
    if (!B || !n) return WF_OK;
    if (!prefix_visible || (max_prefix && !prefix_table)) return fail(WF_E_INVALID, "prefix_visible or prefix_table is NULL");
    a.first_table = prefix_table; a.first_visible = prefix_visible;
    a.first_pages = prefix_pages; a.max_first = max_prefix;
    AttendStack stack;
    if (attend_shared_plan(a, precision, &stack) >= 1LL << 32) return fail(WF_E_UNSUPPORTED, "2^32 or more threads in one call");
    const OnDevice on(c->device);
    if (on.error() != hipSuccess) return kv_fail(on.error(), "the cache's device");
    launch_attend_shared(a, precision, stack, stream);
    return kv_launched("wf_cache_attend_shared");
} catch (...) {
    return WF_E_NOMEM;
}

int wf_cache_sync(wf_cache_t cache, hipStream_t stream) try {
    Cache* c = reinterpret_cast<Cache*>(cache);
    if (!c) return fail(WF_E_INVALID, "cache is NULL");
    const OnDevice on(c->device);
    if (on.error() != hipSuccess) return kv_fail(on.error(), "the cache's device");
    int err = 0, *taken = c->c.err + 1 + c->syncs++ % kKvTaken;
    hipError_t e = hipStreamSynchronize(stream);
    if (e == hipSuccess) {
        hipLaunchKernelGGL(k_kv_take_errors, dim3(1), dim3(1), 0, stream, c->c.err, taken);
        e = hipGetLastError();
    }
    if (e == hipSuccess) e = hipMemcpyAsync(&err, taken, sizeof err, hipMemcpyDeviceToHost, stream);
    if (e == hipSuccess) e = hipStreamSynchronize(stream);
    if (e != hipSuccess) return kv_fail(e, "wf_cache_sync");
    if (err & kErrKvPage) return fail(WF_E_INVALID, "a page table entry lies outside the pool");
    if (err & kErrKvRange) return fail(WF_E_CAPACITY, "a token lies past its page table, or a row sees more than max_visible tokens");
    return WF_OK;
} catch (...) {
    return WF_E_NOMEM;
}

}  // extern "C"
