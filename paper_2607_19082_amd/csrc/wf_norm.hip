// Norms of queries and keys for each head, with the position rotation in the
// same pass:
//   y_c = x_c / sqrt(mean_c x_c^2 + eps) * gain_c
//   (y_a, y_b) -> (y_a cos t - y_b sin t, y_a sin t + y_b cos t)
// for the pairs of the rotated channels, t = position * frequency of the pair.
//
// A unit of work is eight channels, four pairs: a lane holds a unit of one head
// at a time, LPH lanes a head, and goes on to the token's next heads with its
// sines and cosines and gains in registers.  The sum of squares is a sum of
// doubles over the lanes of a head: squares of any finite channels neither
// overflow nor vanish there, and its square root is split into a power of two
// and a float, so that rows of any finite size come out right.
//
// Angles are fixed-point turns: position times frequency, modulo one turn, is
// the low 64 bits of a product of integers, exact but for the frequency's own
// rounding to 2^-64 of a turn.  A position of 2^31 is as exact as one of 1.
//
// Bound by memory where there are many tokens (MI355X): 2 x 8191 tokens of 32
// query and 8 key heads of 128 in bf16, 321 MB both ways with the second
// sequence shorter, 75 us, 4.3 TB/s where a large copy reaches 4.6; vector
// instructions take 53% of the time beside it.  Heads in turn share a lane's
// sines, which would otherwise cost more than the rest.  A token 3.9 us, a
// launch and its chain of loads.
#include <cmath>
#include <new>

#include "wf_cache.h"

namespace wf {

constexpr int kNormThreads = 256;
constexpr int kNormPairs = 128;      // of a head, at most
// Outputs of more bytes than the second-level caches hold are stored past them:
// 2 x 8191 tokens of 40 heads of 128 in bf16 (321 MB both ways) 76 us, through
// them 81; shorter ones stay where the next kernel finds them.
constexpr long long kNormStream = 32 << 20;

struct NormArgs {
    KvRows x[2], y[2];               // queries, keys: in, out
    const float* gain[2];            // [dim] or null
    const int *positions, *counts;   // counts: null, or [B]
    int tokens, n, axes;
    int q_heads, heads;              // heads: of both
    int dim, units, turned;          // units of a head, and those that are rotated
    int log_heads;                   // log2 of the heads of one token that a wave takes at once
    int chunks, per_chunk;           // waves that share a token's heads; heads of one
    KvDiv n_, chunks_, axis_;        // axis_: units of an axis
    double eps, each;                // each: 1 / dim
    // of an axis's pairs, 2^-64 turns a position: with the arguments, so that a
    // plan needs no memory of the device, and a captured call no plan
    uint64_t turns[kNormPairs];
};

// Sine and cosine of u / 2^32 turns.  To the nearest quarter turn, the rest |x|
// <= pi / 4 by the series of both, whose first terms left out are 2e-9 and 1e-10:
// off by less than 2^-23.
__device__ __forceinline__ void turn_of(unsigned u, float& sine, float& cosine) {
    const unsigned q = (u + 0x20000000u) >> 30;
    const float x = (float)(int)(u - (q << 30)) * 1.4629180792671596e-9f;       // 2 pi / 2^32
    const float z = x * x;
    const float s = x + x * z * (-1.0f / 6 + z * (1.0f / 120 + z * (-1.0f / 5040 + z * (1.0f / 362880))));
    const float c = 1.0f + z * (-0.5f + z * (1.0f / 24 + z * (-1.0f / 720 + z * (1.0f / 40320 + z * (-1.0f / 3628800)))));
    sine = q & 1 ? c : s;
    cosine = q & 1 ? s : c;
    if (q & 2) sine = -sine;
    if ((q + 1) & 2) cosine = -cosine;
}

// A sum over the LPH lanes of a head, the same bits in each.
template <int CTRL>
__device__ __forceinline__ double lane_move(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const unsigned lo = lane_move<CTRL>((int)(unsigned)u), hi = lane_move<CTRL>((int)(unsigned)(u >> 32));
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int LPH>
__device__ __forceinline__ double head_sum(double x) {
    x += lane_move<0xb1>(x);             // quad_perm 1 0 3 2
    x += lane_move<0x4e>(x);             // quad_perm 2 3 0 1
    x += lane_move<0x141>(x);            // the other quad of eight
    if constexpr (LPH >= 16) x += lane_move<0x128>(x);      // the other eight of a row
    if constexpr (LPH >= 32) {           // the other row of two
        const uint64_t u = __builtin_bit_cast(uint64_t, x);
        const unsigned w[2] = {(unsigned)u, (unsigned)(u >> 32)};
        const auto lo = __builtin_amdgcn_permlane16_swap(w[0], w[0], false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap(w[1], w[1], false, false);
        x = __builtin_bit_cast(double, (uint64_t)hi[0] << 32 | lo[0]) + __builtin_bit_cast(double, (uint64_t)hi[1] << 32 | lo[1]);
    }
    return x;
}

template <int N, bool STREAM, class T>
__device__ __forceinline__ void store(T* p, const T* x) {
    typedef unsigned Words __attribute__((ext_vector_type(N * sizeof(T) / 4), aligned(sizeof(T))));
    Words w;
    __builtin_memcpy(&w, x, sizeof w);
    if constexpr (STREAM) __builtin_nontemporal_store(w, (Words*)p);
    else *(Words*)p = w;
}

// The four pairs of a unit: NEIGHBOURS pairs channels 2 j and 2 j + 1, and the
// unit's eight lie together; else the pair's second channel is half of the
// axis's channels on.  STREAM: stores past the caches.
template <class T, int LPH, bool NEIGHBOURS, bool STREAM>
__global__ __launch_bounds__(kNormThreads) void k_head_norm(NormArgs a) {
    constexpr int kHeads = 64 / LPH;     // of a wave at once, of one token or several
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned id = blockIdx.x * (kNormThreads / 64) + wave;
    const unsigned group = a.chunks_(id), chunk = id - group * a.chunks;
    const int step = 1 << a.log_heads, slot = lane / LPH, unit = lane % LPH;
    const unsigned token = group * (kHeads >> a.log_heads) + (slot >> a.log_heads);
    const unsigned t = token < (unsigned)a.tokens ? token : 0;
    const int b = a.n_(t), i = t - b * a.n;
    const bool on = token < (unsigned)a.tokens && unit < a.units && (!a.counts || i < a.counts[b]);
    if (!__any(on)) return;

    const bool turned = unit < a.turned;
    const int axis_units = a.turned / a.axes, axis = turned ? a.axis_(unit) : 0, u = unit - axis * axis_units;
    int at[2] = {8 * min(unit, a.units - 1), 0};
    if (!NEIGHBOURS && turned) at[0] = axis * 8 * axis_units + 4 * u;
    at[1] = at[0] + (!NEIGHBOURS && turned ? 4 * axis_units : 4);

    const T *q = (const T*)a.x[0].p + b * a.x[0].sb + i * a.x[0].sr, *k = (const T*)a.x[1].p + b * a.x[1].sb + i * a.x[1].sr;
    auto load = [&](int h, T (&x)[8]) {
        h = min(h, a.heads - 1);
        const T* p = h < a.q_heads ? q + h * a.x[0].sh : k + (h - a.q_heads) * a.x[1].sh;
        if constexpr (NEIGHBOURS) {
            __builtin_memcpy(x, p + at[0], sizeof x);
        } else {
            __builtin_memcpy(x, p + at[0], sizeof x / 2);
            __builtin_memcpy(x + 4, p + at[1], sizeof x / 2);
        }
    };
    const int first = chunk * a.per_chunk, last = min(first + a.per_chunk, a.heads);
    int h = first + (slot & (step - 1));
    T x[8];
    load(h, x);

    float gain[2][8], sine[4], cosine[4];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) gain[s][e] = a.gain[s] ? a.gain[s][at[e / 4] + e % 4] : 1.0f;
    if (turned) {
        const int64_t p = a.positions[(size_t)t * a.axes + axis];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint64_t turns = (uint64_t)p * a.turns[4 * u + j];
            turn_of((unsigned)((turns + 0x80000000u) >> 32), sine[j], cosine[j]);
        }
    }

    for (int h0 = first; h0 < last; h0 += step, h += step) {
        T next[8];
        load(h0 + step < last ? h + step : h, next);
        double sum = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = __builtin_fma((double)(float)x[e], (double)(float)x[e], sum);
        sum = head_sum<LPH>(unit < a.units ? sum : 0.0);
        // 1 / sqrt(m) = 2^-half / sqrt(rest), rest in [1/2, 2): one step after
        // the instruction's own estimate
        const double m = __builtin_fma(sum, a.each, a.eps);
        const int half = __builtin_amdgcn_frexp_exp(m) >> 1;
        const float rest = (float)__builtin_amdgcn_ldexp(m, -2 * half);
        float r = __builtin_amdgcn_rsqf(rest);
        r = __builtin_isinf(rest) ? 0.0f : r * __builtin_fmaf(-0.5f * rest * r, r, 1.5f);
        const bool key = h >= a.q_heads;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = __builtin_amdgcn_ldexpf((float)x[e], -half) * (r * (key ? gain[1][e] : gain[0][e]));
        if (turned) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float &p = y[NEIGHBOURS ? 2 * j : j], &s = y[NEIGHBOURS ? 2 * j + 1 : 4 + j];
                const float was = p;
                p = __builtin_fmaf(was, cosine[j], -s * sine[j]);
                s = __builtin_fmaf(was, sine[j], s * cosine[j]);
            }
        }
        if (on && h < last) {
            T out[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) out[e] = (T)y[e];
            T* p = key ? (T*)a.y[1].p + b * a.y[1].sb + i * a.y[1].sr + (h - a.q_heads) * a.y[1].sh
                       : (T*)a.y[0].p + b * a.y[0].sb + i * a.y[0].sr + h * a.y[0].sh;
            if constexpr (NEIGHBOURS) {
                store<8, STREAM>(p + at[0], out);
            } else {
                store<4, STREAM>(p + at[0], out);
                store<4, STREAM>(p + at[1], out + 4);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = next[e];
    }
}

// ---- host -----------------------------------------------------------------------

// Waves that fill the chip: fewer heads each make more sines and shorter runs.  us
// at 2048 / 4096 / 8192 / 16384: a 4K grid's 10 fp32 heads of 64 39.7 / 40.0 /
// 45.8 / 49.6, the prompts above 80.9 / 81.3 / 81.0 / 86.3 (through the caches).
constexpr int kNormFill = 4096;

struct HeadNorm {
    int device = 0;
    int dim = 0, rotated = 0, axes = 1, pairs = 0;
    float eps = 0.0f;
    uint64_t turns[kNormPairs] = {};
};

// How the heads of a token are dealt to lanes and waves.  Returns the waves.
static long long norm_plan(NormArgs& a, int lph) {
    const int most = 64 / lph;
    // few tokens: a head's lanes as wide as they come, one pass each; many: so
    // many heads of a token at once that the last pass is full
    a.log_heads = 0;
    while (2 << a.log_heads <= most && 2 << a.log_heads <= a.heads) ++a.log_heads;
    auto passes = [&](int log) { return (a.heads + (1 << log) - 1) >> log; };
    auto groups = [&](int log) { const int at_once = most >> log; return ((long long)a.tokens + at_once - 1) / at_once; };
    if (groups(a.log_heads) * passes(a.log_heads) > kNormFill)
        for (int log = a.log_heads; log >= 0; --log)
            if ((long long)(passes(log) << log) < (long long)(passes(a.log_heads) << a.log_heads)) a.log_heads = log;
    const long long g = groups(a.log_heads);
    const int p = passes(a.log_heads);
    long long chunks = (kNormFill + g - 1) / g;
    chunks = chunks < p ? chunks : p;
    const int per = (int)((p + chunks - 1) / chunks);
    a.per_chunk = per << a.log_heads;
    a.chunks = (p + per - 1) / per;
    a.chunks_.by(a.chunks);
    return g * a.chunks;
}

template <class T, int LPH, bool NEIGHBOURS>
static void launch_norm(const NormArgs& a, long long waves, hipStream_t st) {
    const dim3 grid((unsigned)((waves + kNormThreads / 64 - 1) / (kNormThreads / 64)));
    const bool stream = (long long)a.tokens * a.heads * a.dim * (long long)sizeof(T) > kNormStream;
    if (stream) hipLaunchKernelGGL((k_head_norm<T, LPH, NEIGHBOURS, true>), grid, dim3(kNormThreads), 0, st, a);
    else hipLaunchKernelGGL((k_head_norm<T, LPH, NEIGHBOURS, false>), grid, dim3(kNormThreads), 0, st, a);
}

template <class T, int LPH>
static void launch_norm_pairs(const NormArgs& a, bool neighbours, long long waves, hipStream_t st) {
    if (neighbours) launch_norm<T, LPH, true>(a, waves, st);
    else launch_norm<T, LPH, false>(a, waves, st);
}

template <class T>
static void launch_norm_dim(const NormArgs& a, bool neighbours, int lph, long long waves, hipStream_t st) {
    if (lph == 8) launch_norm_pairs<T, 8>(a, neighbours, waves, st);
    else if (lph == 16) launch_norm_pairs<T, 16>(a, neighbours, waves, st);
    else launch_norm_pairs<T, 32>(a, neighbours, waves, st);
}

}  // namespace wf

using namespace wf;

extern "C" {

int wf_head_norm_plan(const wf_head_norm_desc* d, wf_head_norm_t* out) try {
    if (!out) return fail(WF_E_INVALID, "out is NULL");
    *out = nullptr;
    if (!d) return fail(WF_E_INVALID, "desc is NULL");
    if (d->dim < 8 || d->dim > 256 || d->dim % 8) return fail(WF_E_UNSUPPORTED, "dim must be a multiple of 8 in [8, 256]");
    if (d->axes != 1 && d->axes != 2) return fail(WF_E_INVALID, "axes must be 1 or 2");
    if (d->pairs != WF_PAIRS_HALVES && d->pairs != WF_PAIRS_NEIGHBOURS) return fail(WF_E_INVALID, "unknown pairs");
    if (d->rotated < 0 || d->rotated > d->dim) return fail(WF_E_INVALID, "rotated must lie in [0, dim]");
    if (d->rotated % (8 * d->axes)) return fail(WF_E_UNSUPPORTED, "rotated must be a multiple of 8 for each axis");
    if (!(d->eps >= 0x1p-126f) || !std::isfinite(d->eps)) return fail(WF_E_INVALID, "eps must be positive, finite and not subnormal");
    const int each = d->rotated / (2 * d->axes);
    if (each && !d->frequencies) return fail(WF_E_INVALID, "frequencies is NULL");
    uint64_t turns[kNormPairs] = {};
    for (int j = 0; j < each; ++j) {
        // radians to 2^-64 turns, modulo one turn
        constexpr long double kTurn = 0.159154943091895335768883763372514362L;     // 1 / (2 pi)
        const double f = d->frequencies[j];
        if (!(std::fabs(f) <= 6.2831853071795865)) return fail(WF_E_INVALID, "frequencies must be finite and at most a turn a position");
        long double x = (long double)f * kTurn;
        x = rintl(ldexpl(x - floorl(x), 64));
        turns[j] = x < 0x1p64L ? (uint64_t)x : 0;
    }
    HeadNorm* p = new (std::nothrow) HeadNorm();
    if (!p) return fail(WF_E_NOMEM, "host allocation");
    p->dim = d->dim; p->rotated = d->rotated; p->axes = d->axes; p->pairs = d->pairs; p->eps = d->eps;
    for (int j = 0; j < each; ++j) p->turns[j] = turns[j];
    const hipError_t e = hipGetDevice(&p->device);
    if (e != hipSuccess) {
        delete p;
        return kv_fail(e, "hipGetDevice");
    }
    *out = reinterpret_cast<wf_head_norm_t>(p);
    return WF_OK;
} catch (...) {
    return WF_E_NOMEM;
}

void wf_head_norm_destroy(wf_head_norm_t plan) { delete reinterpret_cast<HeadNorm*>(plan); }

int wf_head_norm(wf_head_norm_t plan, int32_t precision, const wf_rows* q, const wf_rows* q_out, int32_t q_heads, const float* q_gain,
                 const wf_rows* k, const wf_rows* k_out, int32_t k_heads, const float* k_gain, int32_t B, int32_t n,
                 const int32_t* positions, const int32_t* counts, hipStream_t stream) try {
    const HeadNorm* p = reinterpret_cast<HeadNorm*>(plan);
    if (!p) return fail(WF_E_INVALID, "plan is NULL");
    if (precision != WF_FP32 && precision != WF_BF16) return fail(WF_E_INVALID, "unknown precision");
    if (B < 0 || n < 0) return fail(WF_E_INVALID, "B and n must not be negative");
    if (q_heads < 1 || k_heads < 0) return fail(WF_E_INVALID, "q_heads must be positive and k_heads not negative");
    if (q_heads > 65536 || k_heads > 65536) return fail(WF_E_UNSUPPORTED, "more than 65536 heads");
    if (!B || !n) return WF_OK;
    if ((long long)B * n >= 1LL << 31) return fail(WF_E_UNSUPPORTED, "2^31 or more tokens in one call");
    if (p->rotated && !positions) return fail(WF_E_INVALID, "positions is NULL");
    NormArgs a{};
    int rc;
    if ((rc = kv_rows(q, precision, "q", &a.x[0])) != WF_OK || (rc = kv_rows(q_out, precision, "q_out", &a.y[0])) != WF_OK) return rc;
    if (k_heads && ((rc = kv_rows(k, precision, "k", &a.x[1])) != WF_OK || (rc = kv_rows(k_out, precision, "k_out", &a.y[1])) != WF_OK)) return rc;
    a.gain[0] = q_gain; a.gain[1] = k_heads ? k_gain : nullptr;
    a.positions = positions; a.counts = counts;
    __builtin_memcpy(a.turns, p->turns, sizeof a.turns);
    a.tokens = B * n; a.n = n; a.axes = p->axes;
    a.q_heads = q_heads; a.heads = q_heads + k_heads;
    a.dim = p->dim; a.units = p->dim / 8; a.turned = p->rotated / 8;
    a.eps = p->eps; a.each = 1.0 / p->dim;
    a.n_.by((unsigned)n);
    a.axis_.by(a.turned ? (unsigned)(a.turned / a.axes) : 1u);
    const int lph = p->dim <= 64 ? 8 : (p->dim <= 128 ? 16 : 32);
    const long long waves = norm_plan(a, lph);
    if (waves >= 1LL << 26) return fail(WF_E_UNSUPPORTED, "2^32 or more threads in one call");
    const OnDevice on(p->device);
    if (on.error() != hipSuccess) return kv_fail(on.error(), "the plan's device");
    if (precision == WF_BF16) launch_norm_dim<__bf16>(a, p->pairs == WF_PAIRS_NEIGHBOURS, lph, waves, stream);
    else launch_norm_dim<float>(a, p->pairs == WF_PAIRS_NEIGHBOURS, lph, waves, stream);
    return kv_launched("wf_head_norm");
} catch (...) {
    return WF_E_NOMEM;
}

}  // extern "C"
