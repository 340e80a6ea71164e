// Attention over the 4-bit key/value cache:
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = exp(scale q_i . k_j - m_i)
// over the tokens j that row i sees (j < visible_i, and its mask), zeros where
// it sees none.  One pass over the cache with a running maximum m and sum.
//
// Rows are (query, head of the group) pairs that share a key head, 16 to an
// MFMA column tile.  A wave takes tiles of 32 tokens: S = K Q^T (rows are
// tokens, columns queries) in two 16 x 16 products, and O^T += V^T P^T (rows
// are channels).  The operand row r of the first products is the token
// 8 (r / 4) + r % 4 (+ 4 for the second), so that lane 16 g + c ends up with
// the scores of query c and tokens 8 g .. 8 g + 7, which is the operand that
// the second product takes: probabilities stay in their registers.  Keys and
// values go from memory to registers and become bf16 there, exactly, with the
// power of their block (one conversion for two values).
//
// Operands: keys and values are exact in bf16.  bf16 queries are too; fp32
// queries are three bf16 parts (24 bits).  Probabilities are two bf16 parts
// (16 bits) for bf16 calls, so that the output's own rounding is the only one
// that shows, and three (24 bits) for fp32 calls.  bf16 has fp32's range, so a
// probability keeps these bits however far it lies below the row's largest:
// where the tokens that weigh most hold zeros in a channel, the small ones are
// all that the channel has.  (Half precision takes 22 bits in two parts, but
// ends at 2^-24.)  Scores, maxima, sums and outputs are held in fp32; a row's
// sum is that of its rounded probabilities.
//
// The waves of a workgroup share the tokens and join at the end; with few rows
// the tokens are also split over workgroups, and a second kernel joins their
// results.
//
// What bounds it (8 heads of 128, bf16, MI355X): a token each of 32 sequences
// of 8192 tokens, 4 query heads a key head, takes 56 us for 286 MB, 5.1 TB/s
// where a kernel that only reads reaches 5.7.  A tile costs a wave ~170 vector
// instructions, 96 of them conversions and the exchange of values between
// tokens, and 26 products; the two hardly overlap, so with many rows (1024
// queries, 32 heads, 16384 tokens: 350 us, 0.76 PFLOP/s) their sum is the time.
// In fp32 a tile of 128 channels has 51 products, and one tile of rows a
// workgroup (the same 1024 queries 643 us, 0.41 PFLOP/s).
// A short call (a token over 1001: 8 us) is 4 us of launch, loads that wait for
// each other and the join of the waves, and 1 for each tile of a wave.
#include <cmath>
#include <type_traits>

#include "wf_cache.h"

namespace wf {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef float f8 __attribute__((ext_vector_type(8)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef unsigned u2 __attribute__((ext_vector_type(2)));
// read-only for the whole launch, at addresses that a wave shares: scalar loads
typedef const int __attribute__((address_space(4))) * SharedInts;

constexpr int kAtMaxSplits = 256;
constexpr int kAtJoin = 256;        // threads of the kernel that joins the splits
// Waves of a workgroup.  (16 instead of 8: 8.4 against 7.4 us for a token over
// 1001, 14.6 against 13.8 for 45 fp32 rows over 32300, since the larger workgroup
// starts later.)
template <int DP, class T, int NT>
constexpr int kAtWaves = NT == 1 && DP * sizeof(T) < 1024 ? 8 : 4;
// a row's maximum is raised only when a score passes it by this much (in
// powers of two): its probabilities then stay below 2^8
constexpr float kAtSlack = 8.0f;
// Probabilities are held times 2^7, so that the third part (2^-24 of the
// first) is a normal number down to 2^-109 of the row's largest; the sums that
// divide them are too.
constexpr float kAtLift = 7.0f;
// Rows whose maximum lies beyond this (in powers of two) round the product of
// score and scale before they subtract the maximum.  Below, one multiply-add
// takes the exact product, which passes its rounded value, the maximum, by half
// a unit in the last place: 1/4 here, but 32 and more from 2^29 on.
constexpr float kAtFar = 4194304.0f;

// bf16 parts of queries and of probabilities
template <class T>
struct AtParts;
template <>
struct AtParts<__bf16> {
    static constexpr int kQ = 1, kP = 2;
};
template <>
struct AtParts<float> {
    static constexpr int kQ = 3, kP = 3;
};

__device__ __forceinline__ f4 mfma(b8 a, b8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Eight values as N bf16 parts, the largest first.  What a part leaves is one
// dot product: r - 1 * part + 0 * its neighbour, exact.  The pairs (-1, 0) and
// (0, -1) come from registers: as an instruction's own constant, -1 stands for
// the other pair.
template <int N>
__device__ __forceinline__ void parts(const float (&x)[8], b8 (&p)[N]) {
    unsigned first, second;
    asm("s_mov_b32 %0, 0xbf80" : "=s"(first));
    asm("s_mov_b32 %0, 0xbf800000" : "=s"(second));
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        f2 r = {x[e], x[e + 1]};
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const b2 h = __builtin_convertvector(r, b2);
            p[n][e] = h[0];
            p[n][e + 1] = h[1];
            if (n + 1 < N) {
                r[0] = __builtin_amdgcn_fdot2_f32_bf16(h, __builtin_bit_cast(b2, first), r[0], false);
                r[1] = __builtin_amdgcn_fdot2_f32_bf16(h, __builtin_bit_cast(b2, second), r[1], false);
            }
        }
    }
}

// Two 4-bit values of byte J of w, times the power.
template <int J>
__device__ __forceinline__ unsigned pair_of(unsigned w, float power) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, power, J));
}

// A tile of 32 tokens of one head as a lane holds it.
template <int DP>
struct AtKeys {
    unsigned w[DP / 16], power;
};
template <int DP>
struct AtValues {
    unsigned w[DP / 16], power[2];
};

template <int DP>
__device__ __forceinline__ void load_keys(AtKeys<DP>& k, const uint8_t* record, int lane) {
    using L = KvLayout<DP>;
#pragma unroll
    for (int n = 0; n < L::kLane; n += 16)
        __builtin_memcpy(k.w + n / 4, __builtin_assume_aligned(record + L::piece(0, n) + lane * 16u, 16), 16);
    const uint8_t* powers = record + 32 * DP + (unsigned)(L::key_lane_powers(lane) - 32 * DP);
    if constexpr (L::kPowers == 2) {
        uint16_t p;
        __builtin_memcpy(&p, __builtin_assume_aligned(powers, 2), 2);
        k.power = p;
    } else {
        __builtin_memcpy(&k.power, __builtin_assume_aligned(powers, 4), 4);
    }
}

template <int DP>
__device__ __forceinline__ void load_values(AtValues<DP>& v, const uint8_t* record, int lane) {
    using L = KvLayout<DP>;
    const unsigned powers = L::value_powers((lane & 15) * L::kRows / kKvBlock) - L::value_powers(0) + 8 * (lane >> 4);
    __builtin_memcpy(v.power, __builtin_assume_aligned(record + L::value_powers(0) + powers, 8), 8);
#pragma unroll
    for (int n = 0; n < L::kLane; n += 16)
        __builtin_memcpy(v.w + n / 4, __builtin_assume_aligned(record + 16 * DP + L::piece(0, n) + lane * 16u, 16), 16);
}

// Byte N of a word as the exponent of a scale.  The bits beside it are the
// word's others: a conversion reads the exponent alone.
template <int N>
__device__ __forceinline__ float power_at(unsigned w) {
    return __builtin_bit_cast(float, N == 0 ? w << 23 : (N == 1 ? w << 15 : (N == 2 ? w << 7 : w >> 1)));
}

__device__ __forceinline__ bool power_is_nan(float p) { return (~__builtin_bit_cast(unsigned, p) & 0x7f800000u) == 0; }

// The operand of half A of the keys, channels from 8 KK of each quarter.
template <int DP, int A, int KK>
__device__ __forceinline__ b8 key_frag(const AtKeys<DP>& t) {
    constexpr int kPerLane = KvLayout<DP>::kPowers / 2;    // powers of a half in a lane
    const unsigned w = t.w[A * (DP / 32) + KK];
    const float power = power_at<A * kPerLane + KK * kPerLane / (DP / 32)>(t.power);
    u4 r = {pair_of<0>(w, power), pair_of<1>(w, power), pair_of<2>(w, power), pair_of<3>(w, power)};
    return __builtin_bit_cast(b8, r);
}

template <int DP, int NT, int NQ, int A, int KK = 0>
__device__ __forceinline__ void add_scores(const AtKeys<DP>& x, const b8 (&q)[NT][DP / 32][NQ], f4 (&s)[NT][2]) {
    if constexpr (KK < DP / 32) {
        const b8 f = key_frag<DP, A, KK>(x);
#pragma unroll
        for (int n = NQ - 1; n >= 0; --n)
#pragma unroll
            for (int t = 0; t < NT; ++t) s[t][A] = mfma(f, q[t][KK][n], s[t][A]);
        add_scores<DP, NT, NQ, A, KK + 1>(x, q, s);
    }
}

// Tiles 2 B and 2 B + 1 of the values as operands: rows are channels kRows i +
// 2 B (+ 1), k the lane's eight tokens.
template <int DP, int B>
__device__ __forceinline__ void value_frags(const unsigned (&v)[DP / 16], const float (&power)[8], b8 (&f)[2]) {
    u4 lo, hi;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        unsigned x, y;
        if constexpr (DP == 64) {                 // a word holds two tokens
            x = pair_of<B>(v[p], power[2 * p]);
            y = pair_of<B + 2>(v[p], power[2 * p + 1]);
        } else if constexpr (DP == 128) {
            x = pair_of<B>(v[2 * p], power[2 * p]);
            y = pair_of<B>(v[2 * p + 1], power[2 * p + 1]);
        } else {                                  // two words a token
            x = pair_of<B % 4>(v[4 * p + B / 4], power[2 * p]);
            y = pair_of<B % 4>(v[4 * p + 2 + B / 4], power[2 * p + 1]);
        }
        lo[p] = __builtin_amdgcn_perm(y, x, 0x05040100);
        hi[p] = __builtin_amdgcn_perm(y, x, 0x07060302);
    }
    f[0] = __builtin_bit_cast(b8, lo);
    f[1] = __builtin_bit_cast(b8, hi);
}

template <int DP, int NT, int NP, int B = 0>
__device__ __forceinline__ void add_values(const unsigned (&v)[DP / 16], const float (&power)[8], const b8 (&p)[NT][NP],
                                           f4 (&o)[NT][DP / 16]) {
    if constexpr (B < DP / 32) {
        b8 f[2];
        value_frags<DP, B>(v, power, f);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int m = NP - 1; m >= 0; --m)
#pragma unroll
                for (int t = 0; t < NT; ++t) o[t][2 * B + s] = mfma(f[s], p[t][m], o[t][2 * B + s]);
        add_values<DP, NT, NP, B + 1>(v, power, p, o);
    }
}

// Eight bits as ones and zeros.
__device__ __forceinline__ b8 bits(unsigned x) {
    b8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (__bf16)(float)(x >> e & 1);
    return r;
}

// The tile's probabilities into their sums and, times its values, the outputs.
template <int DP, int NT, int N>
__device__ __forceinline__ void add_products(const unsigned (&v)[DP / 16], const float (&power)[8], const float (&w)[NT][8], f4 (&l)[NT],
                                             f4 (&o)[NT][DP / 16]) {
    b8 p[NT][N], ones;
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = 1.0f;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        parts<N>(w[t], p[t]);
#pragma unroll
        for (int n = N - 1; n >= 0; --n) l[t] = mfma(ones, p[t][n], l[t]);
    }
    add_values<DP, NT, N>(v, power, p, o);
}

// x y - z with the product rounded by itself
__device__ __forceinline__ float product_less(float x, float y, float z) {
#pragma clang fp contract(off)
    return x * y - z;
}

// Weight of a partial result with maximum m (less the lift) and sum l; 0 where
// it saw no token.  Where the tokens it saw are all at -infinity, l is 1 and o
// 0: nothing beside a finite maximum, and 0 / 0 where the row has none.
__device__ __forceinline__ float at_weight(float m, float l, float most) {
    const float w = __builtin_amdgcn_exp2f(m - most);
    return m == -INFINITY && l == 0.0f ? 0.0f : (m == most ? 1.0f : w);
}

// What a row's joined sum divides it by.
__device__ __forceinline__ float at_scale(float most, float sum) {
    return sum == 0.0f ? 0.0f : (most == -INFINITY ? __builtin_nanf("") : 1.0f / sum);
}

// Eight channels of a row, into the output.
template <class T>
__device__ __forceinline__ void write_row(const AttendArgs& a, int b, int head, int row, int d, const f8& v) {
    const int i = a.group_(row), h = (head - i) * a.group + row;
    T out[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = (T)v[e];
    __builtin_memcpy((T*)a.o.p + b * a.o.sb + i * a.o.sr + h * a.o.sh + d, out, sizeof out);
}

// Waves of a SIMD that the registers are shared out for (none spills).
template <int DP, class T, int NT>
constexpr int kAtWavesOfSimd = NT == 1 && DP * sizeof(T) <= 256 ? 4 : (NT * DP * sizeof(T) <= 256 ? 3 : (NT * DP * sizeof(T) <= 512 ? 2 : 1));

constexpr int kAtBatch = 256;       // sequences that are taken by length, at most

// The sequence that holds a place among all, from the longest down and, past
// the first `ahead` places, from the shortest up: workgroups of the two halves
// share a compute unit, and each then has about the same to do.  64 sequences
// of 0 to 8192 tokens, 8 heads of 128: 60 us, in the order given 66 (of 8192
// tokens each 108 and 105).
__device__ __forceinline__ int by_length(const AttendArgs& a, int place, int ahead) {
    __shared__ int length[kAtBatch], found;
    const int u = threadIdx.x;
    int mine = 0;
    if (u < a.B) {
        for (int i = 0; i < a.n; ++i) mine = max(mine, a.visible[(size_t)u * a.n + i]);
        length[u] = mine;
    }
    __syncthreads();
    if (u < a.B) {
        int rank = 0;
        for (int v = 0; v < a.B; ++v) rank += length[v] > mine || (length[v] == mine && v < u);
        if (rank == (place < ahead ? place : a.B - 1 - (place - ahead))) found = u;
    }
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(found);
}

// One workgroup: 16 NT rows of a sequence's key head, and a share of its
// tokens.
template <int DP, class T, int NT, bool MASK>
__global__ __launch_bounds__((64 * kAtWaves<DP, T, NT>), (kAtWavesOfSimd<DP, T, NT>)) void k_attend(AttendArgs a) {
    constexpr int NW = kAtWaves<DP, T, NT>, NQ = AtParts<T>::kQ, NP = AtParts<T>::kP, NK = DP / 32, ND = DP / 16;
    using L = KvLayout<DP>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
    const int rows = a.n * a.group, nrt = (rows + 16 * NT - 1) / (16 * NT);
    const int group = a.splits_(blockIdx.x), split = blockIdx.x - group * a.splits;
    const int bh = a.tiles_(group), place = group - bh * nrt;
    const int rt = nrt - 1 - place;                    // under a causal order the last rows see most: first
    int b = a.heads_(bh);
    const int head = bh - b * a.c.heads;
    if constexpr (NT == 1)
        if (a.ahead) b = by_length(a, b, a.ahead);

    const SharedInts table = (SharedInts)(a.table + (size_t)b * a.table_pages);
    const int in_page = a.c.page_shift - 5;
    const uint8_t* pool = a.c.pool + (size_t)head * a.c.head_bytes();
    const size_t page_bytes = a.c.page_bytes();

    // What the rows see, their queries, and the page that the wave begins with
    // if a row sees all it may: in flight together, since each waits as long as
    // a short call's whole arithmetic takes.
    const int expect = (a.splits_((a.max_visible + kKvTile - 1) / kKvTile + a.splits - 1) * split + wave) >> in_page;
    const int expected = a.max_visible ? table[min(expect, a.table_pages - 1)] : 0;
    int see[NT], most = 0, least = a.max_visible;
    T raw[NT][NK][8];
    const uint8_t* mask[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = rt * 16 * NT + t * 16 + col;
        const bool on = row < rows;                    // a column past the last row repeats the first
        const int i = on ? a.group_(row) : 0, h = (head - i) * a.group + (on ? row : 0);
        see[t] = a.visible[(size_t)b * a.n + i];
        mask[t] = MASK ? a.mask + b * a.mb + i * a.mr : nullptr;
        const T* p = (const T*)a.q.p + b * a.q.sb + i * a.q.sr + h * a.q.sh;
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) __builtin_memcpy(raw[t][kk], p + min(DP / 4 * g + 8 * kk, a.c.dim - 8), sizeof raw[t][kk]);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const bool on = rt * 16 * NT + t * 16 + col < rows;
        if (on && see[t] > a.max_visible) atomicOr(a.c.err, kErrKvRange);
        see[t] = on ? max(0, min(see[t], a.max_visible)) : 0;
        most = max(most, see[t]);
        if (on) least = min(least, see[t]);
    }
    most = __builtin_amdgcn_readfirstlane(lanes16(most, [](int x, int y) { return max(x, y); }));
    least = __builtin_amdgcn_readfirstlane(lanes16(least, [](int x, int y) { return min(x, y); }));

    // the tiles of this split, dealt to the waves in turn
    const int tiles = (most + kKvTile - 1) / kKvTile;
    const int share = a.splits_(tiles + a.splits - 1);
    const int t0 = split * share, t1 = min(tiles, t0 + share);

    b8 q[NT][NK][NQ];
    auto make_queries = [&] {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) {
                const bool in = DP / 4 * g + 8 * kk < a.c.dim;
                if constexpr (NQ == 1) {
                    u4 w;
                    __builtin_memcpy(&w, raw[t][kk], sizeof w);
                    q[t][kk][0] = __builtin_bit_cast(b8, in ? w : u4{0, 0, 0, 0});
                } else {
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = in ? (float)raw[t][kk][e] : 0.0f;
                    parts<NQ>(x, q[t][kk]);
                }
            }
    };

    f4 o[NT][ND], l[NT], bad[NT];
    // the row's maximum so far, and the score that raises it (none: 0 and
    // -infinity)
    float sub[NT], raise[NT];
    bool far[NT];                          // of any row of the wave
    unsigned seen[NT];                     // not 0: the row sees a token of the lane's
    bool all;                              // every row sees a whole tile

    // One pass over the wave's tiles; false where it has to be made again with
    // care: where a value that is not a number reached an output (it may stand
    // at a token that only other rows see, and 0 times it is not 0).  The
    // careful pass takes blocks that are not finite as zeros, and is the same
    // otherwise; a count of those that each row sees says which channels they
    // spoil.
    auto pass = [&](auto careful) {
        constexpr bool kCareful = decltype(careful)::value;
        all = false;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int r = 0; r < ND; ++r) o[t][r] = f4{0, 0, 0, 0};
            l[t] = bad[t] = f4{0, 0, 0, 0};
            raise[t] = -INFINITY;
            sub[t] = 0.0f;
            far[t] = false;
            seen[t] = 0;
        }
        const int tile0 = t0 + wave;
        if (tile0 < t1) {
            AtKeys<DP> keys;
            AtValues<DP> values;
            u2 allow[NT];                  // the mask's bytes of the lane's tokens
            auto page_of = [&](int tile) { return table[min(tile, t1 - 1) >> in_page]; };
            auto record_of = [&](int tile, int page) {
                return pool + (size_t)page * page_bytes + (size_t)(min(tile, t1 - 1) & ((1 << in_page) - 1)) * L::kRecord;
            };
            auto load_mask = [&](int tile) {
                const int at = min(tile, t1 - 1) * kKvTile + 8 * g;
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    if (at + 8 <= a.max_visible) {
                        __builtin_memcpy(&allow[t], mask[t] + at, 8);
                    } else {
                        uint64_t x = 0;
                        for (int e = 0; at + e < a.max_visible; ++e) x |= (uint64_t)mask[t][at + e] << 8 * e;
                        allow[t] = __builtin_bit_cast(u2, x);
                    }
                }
            };
            // a page outside the pool: its tokens are left out (another page's
            // are loaded in their place)
            auto inside = [&](int page) { return page >= 0 && page < a.c.pages; };
            const int page = tile0 >> in_page == expect ? expected : page_of(tile0);
            bool there = inside(page), missing = !there;
            const uint8_t* record = record_of(tile0, there ? page : 0);
            load_keys(keys, record, lane);
            if constexpr (MASK) load_mask(tile0);
            int next = page_of(tile0 + NW);
            if constexpr (!kCareful) make_queries();
            // The next tile's keys are loaded as soon as this one's are used
            // up, its values then, and the page of the one after it.  Past
            // the end it is the last tile again, so that the loads in flight
            // are the same on every path.
            for (int tile = tile0; tile < t1; tile += NW) {
                load_values(values, record, lane);
                // the loads go out before the wait for the keys
                __builtin_amdgcn_sched_barrier(0);
                const bool next_there = inside(next);
                record = record_of(tile + NW, next_there ? next : 0);
                next = page_of(tile + 2 * NW);
                f4 s[NT][2];
#pragma unroll
                for (int t = 0; t < NT; ++t) s[t][0] = s[t][1] = f4{0, 0, 0, 0};
                add_scores<DP, NT, NQ, 0>(keys, q, s);
                add_scores<DP, NT, NQ, 1>(keys, q, s);
                load_keys(keys, record, lane);
                const int at = tile * kKvTile + 8 * g;         // the lane's first token
                const bool edge = MASK || !there || (tile + 1) * kKvTile > least;   // some row may not see all of it
                unsigned sees[NT];                     // the lane's tokens that its row sees
#pragma unroll
                for (int t = 0; t < NT; ++t) sees[t] = 0xff;
                if (edge) {
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const int left = there ? see[t] - at : 0;
                        sees[t] = 0;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            bool on = e < left;
                            if constexpr (MASK) on = on && (allow[t][e / 4] >> 8 * (e % 4) & 0xff);
                            sees[t] |= (unsigned)on << e;
                            s[t][e / 4][e % 4] = on ? s[t][e / 4][e % 4] : -INFINITY;
                        }
                        seen[t] |= sees[t];
                    }
                }
                if constexpr (MASK) load_mask(tile + NW);
                all |= !edge;
                if (edge) {
                    // past the last token that any row sees, a page holds anything
                    const int n = max(0, min(8, there ? most - at : 0));
                    const uint64_t in = n == 8 ? ~0ull : (1ull << 8 * n) - 1;
                    values.power[0] = (values.power[0] & (unsigned)in) | (0x7f7f7f7fu & ~(unsigned)in);
                    values.power[1] = (values.power[1] & (unsigned)(in >> 32)) | (0x7f7f7f7fu & ~(unsigned)(in >> 32));
                }
                float power[8] = {power_at<0>(values.power[0]), power_at<1>(values.power[0]), power_at<2>(values.power[0]), power_at<3>(values.power[0]),
                                  power_at<0>(values.power[1]), power_at<1>(values.power[1]), power_at<2>(values.power[1]), power_at<3>(values.power[1])};
                if constexpr (kCareful) {
                    unsigned spoilt = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (power_is_nan(power[e])) {
                            spoilt |= 1u << e;
                            power[e] = 1.0f;
                        }
#pragma unroll
                    for (int t = 0; t < NT; ++t) bad[t] = mfma(bits(spoilt), bits(sees[t]), bad[t]);
                }
                float w[NT][8];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    // NaN where a score is: the row's maximum then stays as it is,
                    // and its outputs become NaN through the exponent
                    float top = s[t][0][0];
#pragma unroll
                    for (int e = 1; e < 8; ++e) top = __builtin_elementwise_maximum(top, s[t][e / 4][e % 4]);
                    top *= a.scale_log2;
                    if (__any(top > raise[t])) {
                        // only the rows that pass their own: what another row
                        // sees does not change this one's bits
                        top = lane_rows(top, [](float x, float y) { return fmaxf(x, y); });
                        const bool none = raise[t] == -INFINITY, up = top > raise[t];
                        const float to = up ? top - kAtLift : sub[t], by = none ? 0.0f : exp2f(sub[t] - to);
                        sub[t] = to;
                        raise[t] = up ? top + kAtSlack : raise[t];
                        far[t] = __any(fabsf(to) >= kAtFar);
#pragma unroll
                        for (int r = 0; r < ND; ++r) o[t][r] *= by;
                        l[t] *= by;
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[t][e] = __builtin_fmaf(s[t][e / 4][e % 4], a.scale_log2, -sub[t]);
                    if (far[t])
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (fabsf(sub[t]) >= kAtFar) w[t][e] = product_less(s[t][e / 4][e % 4], a.scale_log2, sub[t]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[t][e] = __builtin_amdgcn_exp2f(w[t][e]);
                }
                add_products<DP, NT, NP>(values.w, power, w, l, o);
                there = next_there;
                missing |= !there;
            }
            if (missing && lane == 0) atomicOr(a.c.err, kErrKvPage);
        }
        if constexpr (kCareful) {
            return true;
        } else {
            bool nan = false;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < ND; ++r)
#pragma unroll
                    for (int e = 0; e < 4; ++e) nan |= o[t][r][e] != o[t][r][e];
            return !__any(nan);
        }
    };
    if (!pass(std::false_type())) pass(std::true_type());
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (bad[t][e] > 0.0f)
#pragma unroll
                for (int r = 0; r < ND; ++r) o[t][r][e] = __builtin_nanf("");

    // join the waves, one tile of 16 rows after the other
    constexpr int kPitch = DP + 4, W = DP / 8, kThreads = 64 * NW;
    __shared__ __attribute__((aligned(16))) float lds[NW * 16 * kPitch];
    __shared__ float sm[NW][16], sl[NW][16], top[16];
    const int row0 = rt * 16 * NT, here = min(16 * NT, rows - row0);
    const size_t part = (((size_t)(b * a.c.heads + head) * nrt + place) * a.splits + split) * 16 * NT;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        if (t) __syncthreads();
        const float some = lane_rows(all || seen[t] ? 1.0f : 0.0f, [](float x, float y) { return fmaxf(x, y); });
        if (lane < 16) {
            const bool none = raise[t] == -INFINITY;
            sm[wave][lane] = none ? -INFINITY : sub[t];
            sl[wave][lane] = none ? l[t][0] + some : l[t][0];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int r = 0; r < ND; r += 4)
                *(f4*)&lds[(wave * 16 + col) * kPitch + ND * (4 * g + e) + r] =
                    f4{o[t][r][e], o[t][r + 1][e], o[t][r + 2][e], o[t][r + 3][e]};
        __syncthreads();
        if (threadIdx.x < 16) {
            // each wave's weight, with the sum's inverse in it where the row
            // is complete
            const int c = threadIdx.x;
            float most = sm[0][c], sum = 0.0f, by[NW];
#pragma unroll
            for (int w = 1; w < NW; ++w) most = fmaxf(most, sm[w][c]);
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                by[w] = at_weight(sm[w][c], sl[w][c], most);
                sum += by[w] * sl[w][c];
            }
            const float scale = a.splits > 1 ? 1.0f : at_scale(most, sum);
#pragma unroll
            for (int w = 0; w < NW; ++w) sm[w][c] = by[w] * scale;
            top[c] = most;
            sl[0][c] = sum;
        }
        __syncthreads();
        for (int x = threadIdx.x; x < min(16, here - t * 16) * W; x += kThreads) {
            const int c = x / W, d = x % W * 8;
            f8 v = {};
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                f8 y;
                __builtin_memcpy(&y, __builtin_assume_aligned(&lds[(w * 16 + c) * kPitch + d], 16), sizeof y);
                v += sm[w][c] * y;
            }
            if (a.splits == 1) {
                if (d < a.c.dim) write_row<T>(a, b, head, row0 + t * 16 + c, d, v);
            } else {
                const size_t at = part + t * 16 + c;
                __builtin_memcpy(__builtin_assume_aligned(a.part_o + at * DP + d, 16), &v, sizeof v);
                if (d == 0) {
                    const f2 z = {top[c], sl[0][c]};
                    __builtin_memcpy(__builtin_assume_aligned(a.part_ml + at * 2, 8), &z, sizeof z);
                }
            }
        }
    }
}

// Joins the splits of one row: eight channels a lane, the splits dealt to
// groups of lanes.  The first wave turns the splits' maxima and sums into
// weights while the partial results are on their way.  Bound by its chain of
// launch, load and two exchanges: 3.9 us for 225 rows in 17 splits, 4.7 for 32
// rows in 32.
template <int DP, class T, int NT>
__global__ __launch_bounds__(kAtJoin) void k_attend_join(AttendArgs a) {
    constexpr int W = DP / 8, G = kAtJoin / W, K = kAtMaxSplits / 64, Y = 4;
    __shared__ float weight[kAtMaxSplits];
    __shared__ __attribute__((aligned(16))) float so[kAtJoin / 64][DP];
    constexpr int tile_rows = 16 * NT;
    const unsigned rows = a.n * a.group, row = blockIdx.x, bh = blockIdx.y;
    const int g = threadIdx.x / W, d = threadIdx.x % W * 8, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned nrt = (rows + tile_rows - 1) / tile_rows;
    const size_t first = ((size_t)bh * nrt + (nrt - 1 - row / tile_rows)) * a.splits * tile_rows + row % tile_rows;
    const float* po = a.part_o + first * DP + d;
    f2 z[K];
    if (wave == 0)
#pragma unroll
        for (int k = 0; k < K; ++k)
            __builtin_memcpy(&z[k], __builtin_assume_aligned(a.part_ml + (first + (size_t)min(k * 64 + lane, a.splits - 1) * tile_rows) * 2, 8), 8);
    f8 y[Y];
#pragma unroll
    for (int j = 0; j < Y; ++j)
        __builtin_memcpy(&y[j], __builtin_assume_aligned(po + (size_t)min(g + j * G, a.splits - 1) * tile_rows * DP, 16), 32);
    __builtin_amdgcn_sched_barrier(0);
    if (wave == 0) {
        float most = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) most = fmaxf(most, z[k][0]);
        most = lanes64(most, [](float x, float y) { return fmaxf(x, y); });
#pragma unroll
        for (int k = 0; k < K; ++k) {
            z[k][0] = k * 64 + lane < a.splits ? at_weight(z[k][0], z[k][1], most) : 0.0f;
            sum += z[k][0] * z[k][1];
        }
        sum = lanes64(sum, [](float x, float y) { return x + y; });
        const float scale = at_scale(most, sum);
#pragma unroll
        for (int k = 0; k < K; ++k) weight[k * 64 + lane] = z[k][0] * scale;
    }
    __syncthreads();
    f8 v = {};
    for (int s = g; s < a.splits; s += Y * G) {
        float by[Y];
#pragma unroll
        for (int j = 0; j < Y; ++j) by[j] = weight[min(s + j * G, kAtMaxSplits - 1)];
#pragma unroll
        for (int j = 0; j < Y; ++j)
            if (s + j * G < a.splits) v += by[j] * y[j];
        if (s + Y * G < a.splits)
#pragma unroll
            for (int j = 0; j < Y; ++j)
                __builtin_memcpy(&y[j], __builtin_assume_aligned(po + (size_t)min(s + (Y + j) * G, a.splits - 1) * tile_rows * DP, 16), 32);
    }
    // the groups of a wave, then the waves
#pragma unroll
    for (int x = W; x < 64; x <<= 1)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += __shfl_xor(v[e], x);
    if (lane < W) __builtin_memcpy(__builtin_assume_aligned(&so[wave][d], 16), &v, 32);
    __syncthreads();
    if (threadIdx.x >= W || d >= a.c.dim) return;
#pragma unroll
    for (int w = 1; w < kAtJoin / 64; ++w) {
        f8 z;
        __builtin_memcpy(&z, __builtin_assume_aligned(&so[w][d], 16), 32);
        v += z;
    }
    const int b = a.heads_(bh);
    write_row<T>(a, b, bh - b * a.c.heads, row, d, v);
}

// ---- host -----------------------------------------------------------------------

// Column tiles of a workgroup: two, which share a tile's conversions, where they
// fit the registers and there are enough rows to fill the chip all the same.
// us with one / two, 8 heads, 8192 tokens: of 128 in bf16, 256 tiles of rows 34
// / 39, 512 64 / 57, 1024 129 / 97, 2048 227 / 190; of 64 in bf16, 512 42 / 45,
// 768 61 / 67, 1024 76 / 67; of 64 in fp32, 512 54 / 54, 768 80 / 91, 1024 103 /
// 94.  Hence tiles times channels.
template <int DP, class T>
constexpr bool kAtTwoTiles = DP * sizeof(T) <= 256;
constexpr long long kAtManyRows = 1 << 16;

static int row_tiles(const AttendArgs& a, int precision) {
    const int rows = a.n * a.group;
    const long long tiles = (long long)a.B * a.c.heads * ((rows + 15) / 16);
    return rows > 16 && tiles * a.c.dp >= kAtManyRows && a.c.dp * (precision == WF_BF16 ? 2 : 4) <= 256 ? 2 : 1;
}

long long attend_plan(AttendArgs& a, int precision) {
    const int bytes = a.c.dp * (precision == WF_BF16 ? 2 : 4), nt = row_tiles(a, precision), rows = a.n * a.group;
    const int waves = nt == 1 && bytes < 1024 ? 8 : 4;
    const long long groups = (long long)a.B * a.c.heads * ((rows + 16 * nt - 1) / (16 * nt));
    // A tile takes a wave about 1 us and the join 3, so up to four tiles a wave
    // are not split; more are, down to one tile each.  us with no split, four
    // tiles each, two and one: a token over 1001 (8 heads of 128, bf16) 7.3, 7.4,
    // 8.3, 7.4, over 2047 11.0, 10.2, 8.5, 7.8, over 8192 33, 10.6, 9.1, 8.7; 45
    // fp32 rows over 1024 7.2, 7.2, 8.5, 7.8, over 4096 16.9, 10.7, 9.0, 8.5.
    const long long tiles = ((long long)a.max_visible + kKvTile - 1) / kKvTile;
    const long long by_len = tiles <= 4 * waves ? 1 : (tiles + waves - 1) / waves;
    long long s = kAtTarget / groups;
    // Long calls (8192 tokens) that would leave many compute units idle take two
    // workgroups each where that fills a fifth more: us without and with, 8 key
    // heads of 128 in bf16, 17 tokens 42 / 37, 11 27 / 26, 18 over 0 to 8192 37 /
    // 29, 136 tiles of rows 33 / 30; at 4096 tokens 24 / 23, 18 / 18, at 2048
    // 13.5 / 16.  A few workgroups more than compute units would take as long as
    // two each, and are split into four: 33 tokens over 4096 44 / 39, 8192 81 /
    // 67, 16384 156 / 123, 40 over 8192 84 / 74, 44 87 / 82; 320 tiles of rows
    // over 4096 32 / 35, 8192 59 / 51, 16384 111 / 88; of 64 channels in fp32 29 /
    // 33, 52 / 46, 99 / 75; 36 tokens over 0 to 8192 46 / 48, 0 to 16384 83 / 80.
    if (tiles >= 256) {
        const long long twice = 2 * kAtTarget / groups;
        if (s && 5 * twice > 12 * s) s = twice;
        if (!s && groups <= kAtTarget * 5 / 4) s = 4;
    }
    s = s < by_len ? s : by_len;
    s = s < kAtMaxSplits ? s : kAtMaxSplits;
    a.splits = s < 2 ? 1 : (int)s;
    a.splits_.by(a.splits);
    a.tiles_.by((unsigned)((rows + 16 * nt - 1) / (16 * nt)));
    a.heads_.by(a.c.heads);
    a.group_.by(a.group);
    // A token each of sequences that may be of unequal lengths, and two
    // workgroups on most compute units.  With more of them the units take the
    // next as they finish: in the order given and longest first, 128 sequences
    // of 0 to 8192 tokens 129 / 119 us, but of 8192 each 199 / 207, and 256 of 0
    // to 8192 226 / 228, of 8192 each 395 / 406.
    const bool two = groups > kAtTarget && groups <= 2 * kAtTarget && bytes <= 256 && a.splits == 1;
    a.ahead = nt == 1 && rows <= 16 && a.B > 1 && a.B <= kAtBatch && two ? (int)(kAtTarget / a.c.heads) : 0;
    return groups * a.splits * waves * 64;
}

template <int DP, class T, int NT>
static void join(const AttendArgs& a, hipStream_t st) {
    hipLaunchKernelGGL((k_attend_join<DP, T, NT>), dim3(a.n * a.group, a.B * a.c.heads), dim3(kAtJoin), 0, st, a);
}

template <int DP, class T, int NT>
static void launch_nt(const AttendArgs& a, hipStream_t st) {
    const int rows = a.n * a.group;
    const long long groups = (long long)a.B * a.c.heads * ((rows + 16 * NT - 1) / (16 * NT));
    constexpr int kThreads = 64 * kAtWaves<DP, T, NT>;
    const dim3 grid((unsigned)(groups * a.splits));
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, a); };
    if (a.mask) launch(k_attend<DP, T, NT, true>);
    else launch(k_attend<DP, T, NT, false>);
    if (a.splits > 1) join<DP, T, NT>(a, st);
}

template <int DP, class T>
static void launch_dp(const AttendArgs& a, int nt, hipStream_t st) {
    if constexpr (kAtTwoTiles<DP, T>)
        if (nt == 2) return launch_nt<DP, T, 2>(a, st);
    launch_nt<DP, T, 1>(a, st);
}

template <class T>
static void launch_precision(const AttendArgs& a, int nt, hipStream_t st) {
    if (a.c.dp == 64) launch_dp<64, T>(a, nt, st);
    else if (a.c.dp == 128) launch_dp<128, T>(a, nt, st);
    else launch_dp<256, T>(a, nt, st);
}

void launch_attend(const AttendArgs& a, int precision, hipStream_t st) {
    const int nt = row_tiles(a, precision);
    if (precision == WF_BF16) launch_precision<__bf16>(a, nt, st);
    else launch_precision<float>(a, nt, st);
}

}  // namespace wf
