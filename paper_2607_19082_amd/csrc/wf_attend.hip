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
//
// The other forms take the same tiles from other lists.  With a window a tile of
// rows goes over its rows' first tokens and then over the tiles that one of them
// sees a token of: 64 tokens with windows of 1024 in 0 to 8192 15 us (4.1 TB/s), 1024 rows
// with windows of 4096 100 (0.69 PFLOP/s).  Behind a shared prefix each row goes
// over that and its own tokens (8 x 128 rows behind 16384 352 us, 0.78 PFLOP/s),
// or, where sequences have few rows, those of all sequences fill the tiles over
// the prefix together: 64 tokens behind 8192, with 100 of their own each, 32 / 8
// heads, 24 us, where 64 times the prefix takes 68.
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

// Forms of the kernel.  Rows see a prefix of their sequence (kAtMask: what a mask
// leaves of it); two runs of tokens, the first of its own table (kAtRuns); or the
// rows of all sequences a first run together, as workgroups before those of each
// sequence's own tokens, and a kernel of its own joins both (kAtStack).
enum AtMode { kAtPlain, kAtMask, kAtRuns, kAtStack };
template <int MODE>
using AtArgs = std::conditional_t<MODE == kAtPlain || MODE == kAtMask, AttendArgs, AttendRunsArgs>;

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

// A team of TEAM waves (a workgroup's, as a rule): 16 NT rows of a sequence's key
// head, and a share of its tokens.
template <int DP, class T, int NT, int MODE, int TEAM = kAtWaves<DP, T, NT>>
__global__ __launch_bounds__((64 * kAtWaves<DP, T, NT>), (kAtWavesOfSimd<DP, T, NT>)) void k_attend(AtArgs<MODE> a) {
    constexpr bool MASK = MODE == kAtMask, RUNS = MODE == kAtRuns, STACK = MODE == kAtStack;
    // A wave at its values' products goes ahead of the SIMD's others.  us without
    // and with, 32 / 8 heads of 128: 8 x 128 causal rows behind 16384 in bf16 360 /
    // 357, 4 x 128 behind 8192 in fp32 180 / 173, 64 tokens behind 8192 with 777 of
    // their own each in bf16 34.5 / 34.2, in fp32 46.5 / 44.8; of 64 channels in
    // fp32, two tiles of rows, 58.2 / 60.6.
    constexpr bool kAhead = (RUNS || STACK) && !(NT == 2 && sizeof(T) == 4);
    constexpr int NW = kAtWaves<DP, T, NT>, NQ = AtParts<T>::kQ, NP = AtParts<T>::kP, NK = DP / 32, ND = DP / 16;
    constexpr int TEAMS = NW / TEAM;
    static_assert(TEAMS == 1 || RUNS, "teams are of calls by runs");
    using L = KvLayout<DP>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
    const int team = TEAMS == 1 ? 0 : wave / TEAM, member = TEAMS == 1 ? wave : wave % TEAM;
    // what the workgroup takes: a sequence's own tokens, or all sequences' rows
    // over the prefix as if they were one's
    int block = blockIdx.x, n = a.n, splits = a.splits, max_visible = a.max_visible, table_pages = a.table_pages;
    const int *visible = a.visible, *of_table = a.table;
    KvDiv splits_ = a.splits_, tiles_ = a.tiles_;
    bool stacked = false;
    if constexpr (STACK) {
        stacked = block < a.stack_blocks;
        if (stacked) {
            n = a.B * a.n;
            splits = a.stack_splits; splits_ = a.stack_splits_; tiles_ = a.stack_tiles_;
            max_visible = a.max_first; table_pages = a.first_pages;
            visible = a.first_visible; of_table = a.first_table;
        } else {
            block -= a.stack_blocks;
        }
    }
    const int rows = n * a.group, nrt = (rows + 16 * NT - 1) / (16 * NT);
    bool idle = false;                                 // a team past the last
    if constexpr (TEAMS > 1) {
        block = a.units_of_die ? block / kXcds * TEAMS + team : block * TEAMS + team;      // of the die, or of all
        idle = block >= (a.units_of_die ? a.units_of_die * a.unit_workgroups : a.B * a.c.heads * nrt);
        block = idle ? 0 : block;
        if (a.units_of_die) block = block * kXcds + blockIdx.x % kXcds;
    }
    int group = splits_(block), split = block - group * splits;
    const int bh = tiles_(group);
    int place = group - bh * nrt, b = a.heads_(bh), head = bh - b * a.c.heads;
    if constexpr (RUNS || STACK)
        if (a.units_of_die && (RUNS || stacked)) {
            const int t = block / kXcds, u = a.unit_(t), unit = block % kXcds * a.units_of_die + u, l = t - u * a.unit_workgroups;
            if constexpr (STACK) {
                split = l;
                head = tiles_(unit);
                place = unit - head * nrt;
                b = 0;
            } else {
                place = splits_(l);
                split = l - place * splits;
                head = a.batch_(unit);
                b = unit - head * a.B;
            }
        }
    const int rt = nrt - 1 - place;                    // under a causal order the last rows see most: first
    if constexpr (NT == 1 && (MODE == kAtPlain || MODE == kAtMask))
        if (a.ahead) b = by_length(a, b, a.ahead);

    const SharedInts table = (SharedInts)(of_table + (size_t)b * table_pages);
    const int in_page = a.c.page_shift - 5;
    const uint8_t* pool = a.c.pool + (size_t)head * a.c.head_bytes();
    const size_t page_bytes = a.c.page_bytes();

    // What the rows see, their queries, and the page that the wave begins with
    // if a row sees all it may: in flight together, since each waits as long as
    // a short call's whole arithmetic takes.
    const int expect = RUNS ? -1 : (int)(splits_((max_visible + kKvTile - 1) / kKvTile + splits - 1) * split + member) >> in_page;
    const int expected = !RUNS && max_visible ? table[min(expect, table_pages - 1)] : 0;
    int see[NT], most = 0, least = max_visible;
    int see_first[NT];                                 // kAtRuns: tokens of the first run,
    unsigned from[NT];                                 // and the first token of the second
    T raw[NT][NK][8];
    const uint8_t* mask[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = rt * 16 * NT + t * 16 + col;
        const bool on = row < rows && !idle;           // a column past the last row repeats the first
        const int i = on ? a.group_(row) : 0, h = (head - i) * a.group + (on ? row : 0);
        see[t] = visible[(size_t)b * n + i];
        if constexpr (RUNS) see_first[t] = a.window ? 0 : a.first_visible[(size_t)b * n + i];
        mask[t] = nullptr;
        if constexpr (MASK) mask[t] = a.mask + b * a.mb + i * a.mr;
        const T* p = (const T*)a.q.p + h * a.q.sh;
        if constexpr (STACK) {
            const int of = stacked ? (int)a.n_(i) : b;
            p += of * a.q.sb + (stacked ? i - of * a.n : i) * a.q.sr;
        } else {
            p += b * a.q.sb + i * a.q.sr;
        }
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) __builtin_memcpy(raw[t][kk], p + min(DP / 4 * g + 8 * kk, a.c.dim - 8), sizeof raw[t][kk]);
    }
    __builtin_amdgcn_sched_barrier(0);
    // kAtRuns: the least and most tokens of the first run, and the least and
    // most of the second's first tokens, that a row sees
    int least_first = 0, most_first = 0, low = 0, high = 0;
    if constexpr (RUNS) {
        least_first = a.window ? a.sinks : a.max_first;
        low = max_visible;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const bool on = rt * 16 * NT + t * 16 + col < rows && !idle;
        if (on && see[t] > max_visible) atomicOr(a.c.err, kErrKvRange);
        if constexpr (STACK)                           // no workgroups look at the rows' own tokens
            if (!a.splits && on && a.visible[a.group_(rt * 16 * NT + t * 16 + col)] > 0) atomicOr(a.c.err, kErrKvRange);
        see[t] = on ? max(0, min(see[t], max_visible)) : 0;
        most = max(most, see[t]);
        if (on) least = min(least, see[t]);
        if constexpr (RUNS) {
            from[t] = 0;
            if (a.window) {
                // the first tokens are a run of their own where the window does
                // not reach them
                const int start = see[t] - a.window;
                if (start > a.sinks) {
                    from[t] = start;
                    see_first[t] = a.sinks;
                }
            } else {
                if (on && see_first[t] > a.max_first) atomicOr(a.c.err, kErrKvRange);
                see_first[t] = on ? max(0, min(see_first[t], a.max_first)) : 0;
            }
            most_first = max(most_first, see_first[t]);
            if (on) least_first = min(least_first, see_first[t]);
            if (see[t]) low = min(low, (int)from[t]);
            high = max(high, (int)from[t]);
        }
    }
    most = __builtin_amdgcn_readfirstlane(lanes16(most, [](int x, int y) { return max(x, y); }));
    least = __builtin_amdgcn_readfirstlane(lanes16(least, [](int x, int y) { return min(x, y); }));

    // the tiles of this split, dealt to the waves in turn
    int tiles = (most + kKvTile - 1) / kKvTile;
    int first_tiles = 0, skip = 0;                     // tile first_tiles + x is the second run's tile skip + x
    SharedInts first_table = table;
    if constexpr (RUNS) {
        if (!a.window) first_table = (SharedInts)a.first_table;
        most_first = __builtin_amdgcn_readfirstlane(lanes16(most_first, [](int x, int y) { return max(x, y); }));
        least_first = __builtin_amdgcn_readfirstlane(lanes16(least_first, [](int x, int y) { return min(x, y); }));
        low = __builtin_amdgcn_readfirstlane(lanes16(low, [](int x, int y) { return min(x, y); }));
        high = __builtin_amdgcn_readfirstlane(lanes16(high, [](int x, int y) { return max(x, y); }));
        first_tiles = (most_first + kKvTile - 1) / kKvTile;
        skip = min(low / kKvTile, tiles);
        tiles += first_tiles - skip;
    }
    const int share = splits_(tiles + splits - 1);
    const int t0 = split * share, t1 = min(tiles, t0 + share);
    // Where the rows' counts lie apart, tiles between their windows are no row's,
    // and are left out: a tile may be where one row's tokens end before it and
    // another's begin past it (not so within a window of the first that any row
    // sees, but a row that sees its sequence from the start may see few).  us with
    // and without, windows of 64: rows at 100 and 8000 tokens 8.5 / 43, at 100 and
    // 128000 8.8 / 616; 16 rows anywhere in 128000 20 / 571.
    bool gaps = false;
    if constexpr (RUNS) gaps = a.window && high - least >= kKvTile && (low == 0 || high - low > a.window);

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
    // spoil.  It is also the one that leaves out what no row sees, so that the
    // other's loop has no part in that: with gaps, the first pass ends after a tile.
    auto pass = [&](auto careful) {
        constexpr bool kCareful = decltype(careful)::value, kSkips = RUNS && kCareful;
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
        // where a tile lies in its run
        auto place_of = [&](int tile) { return RUNS && tile >= first_tiles ? tile - first_tiles + skip : tile; };
        // the wave's first tile from this one on that a row sees a token of
        auto seen_from = [&](int tile) {
            if constexpr (RUNS)
                while (gaps && tile >= first_tiles && tile < t1) {
                    const int at = place_of(tile) * kKvTile;
                    int to = INT32_MAX;    // the first token from there on that a row sees
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        if (see[t] > at) to = min(to, max((int)from[t], at));
                    to = __builtin_amdgcn_readfirstlane(lanes16(to, [](int x, int y) { return min(x, y); }));
                    const int ahead = (to - at) / kKvTile;
                    if (!ahead) break;
                    tile += (ahead + TEAM - 1) / TEAM * TEAM;
                }
            return tile;
        };
        const int tile0 = seen_from(t0 + member), end = gaps && !kCareful ? min(t1, tile0 + 1) : t1;
        if (tile0 < t1) {
            AtKeys<DP> keys;
            AtValues<DP> values;
            u2 allow[NT];                  // the mask's bytes of the lane's tokens
            // past the end the last tile again, or the first where the last may be no row's
            auto of_list = [&](int tile) { return kSkips && tile >= t1 ? tile0 : min(tile, end - 1); };
            auto further = [&](int tile) { return kSkips ? seen_from(tile) : tile; };
            auto page_of = [&](int tile) {
                const int u = of_list(tile);
                return RUNS && u < first_tiles ? first_table[place_of(u) >> in_page] : table[place_of(u) >> in_page];
            };
            auto record_of = [&](int tile, int page) {
                return pool + (size_t)page * page_bytes + (size_t)(place_of(of_list(tile)) & ((1 << in_page) - 1)) * L::kRecord;
            };
            auto load_mask = [&](int tile) {
                const int at = of_list(tile) * kKvTile + 8 * g;
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
            // the wave's next tile and the one after it, where they may be further on
            int second = further(tile0 + TEAM), third = further(second + TEAM), next = page_of(second);
            if constexpr (!kCareful) make_queries();
            // The next tile's keys are loaded as soon as this one's are used
            // up, its values then, and the page of the one after it.  Past
            // the end it is another again, so that the loads in flight are the
            // same on every path.
            for (int tile = tile0; tile < end; tile = kSkips ? second : tile + TEAM, second = third, third = further(second + TEAM)) {
                load_values(values, record, lane);
                // the loads go out before the wait for the keys
                __builtin_amdgcn_sched_barrier(0);
                const bool next_there = inside(next);
                record = record_of(kSkips ? second : tile + TEAM, next_there ? next : 0);
                next = page_of(kSkips ? third : tile + 2 * TEAM);
                f4 s[NT][2];
#pragma unroll
                for (int t = 0; t < NT; ++t) s[t][0] = s[t][1] = f4{0, 0, 0, 0};
                add_scores<DP, NT, NQ, 0>(keys, q, s);
                add_scores<DP, NT, NQ, 1>(keys, q, s);
                load_keys(keys, record, lane);
                const bool in_first = RUNS && tile < first_tiles;
                const int spot = place_of(tile), at = spot * kKvTile + 8 * g;       // the lane's first token
                bool edge = MASK || !there;                    // some row may not see all of it
                if constexpr (RUNS) edge |= in_first ? (spot + 1) * kKvTile > least_first : (spot + 1) * kKvTile > least || spot * kKvTile < high;
                else edge |= (tile + 1) * kKvTile > least;
                unsigned sees[NT];                     // the lane's tokens that its row sees
#pragma unroll
                for (int t = 0; t < NT; ++t) sees[t] = 0xff;
                if (edge) {
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const int left = there ? (in_first ? see_first[t] : see[t]) - at : 0;
                        const int before = RUNS && !in_first ? (int)from[t] - at : 0;
                        sees[t] = 0;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            bool on = e < left;
                            if constexpr (RUNS) on = on && e >= before;
                            if constexpr (MASK) on = on && (allow[t][e / 4] >> 8 * (e % 4) & 0xff);
                            sees[t] |= (unsigned)on << e;
                            s[t][e / 4][e % 4] = on ? s[t][e / 4][e % 4] : -INFINITY;
                        }
                        seen[t] |= sees[t];
                    }
                }
                if constexpr (MASK) load_mask(tile + TEAM);
                all |= !edge;
                if (edge) {
                    // past the last token that any row sees, a page holds anything
                    const int n = max(0, min(8, there ? (in_first ? most_first : most) - at : 0));
                    uint64_t in = n == 8 ? ~0ull : (1ull << 8 * n) - 1;
                    if constexpr (RUNS) {              // and before the first
                        const int m = max(0, min(8, in_first ? 0 : low - at));
                        in &= m == 8 ? 0ull : ~0ull << 8 * m;
                    }
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
                if constexpr (kAhead) __builtin_amdgcn_s_setprio(1);
                add_products<DP, NT, NP>(values.w, power, w, l, o);
                if constexpr (kAhead) __builtin_amdgcn_s_setprio(0);
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
            return !gaps && !__any(nan);
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
    constexpr int kPitch = DP + 4, W = DP / 8;
    __shared__ __attribute__((aligned(16))) float lds[NW * 16 * kPitch];
    __shared__ float sm[NW][16], sl[NW][16], top[TEAMS][16];
    const int row0 = rt * 16 * NT, here = idle ? 0 : min(16 * NT, rows - row0), wave0 = team * TEAM;
    size_t part = (((size_t)(b * a.c.heads + head) * nrt + place) * splits + split) * 16 * NT;
    if constexpr (STACK)
        if (!stacked) part = a.own_part + (((size_t)(b * a.c.heads + head) * nrt + place) * splits + split) * a.own_rows;
    const bool whole = !STACK && splits == 1;          // nothing is left to join
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
        if (member == 0 && lane < 16) {
            // each wave's weight, with the sum's inverse in it where the row
            // is complete
            const int c = lane;
            float most = sm[wave0][c], sum = 0.0f, by[TEAM];
#pragma unroll
            for (int w = 1; w < TEAM; ++w) most = fmaxf(most, sm[wave0 + w][c]);
#pragma unroll
            for (int w = 0; w < TEAM; ++w) {
                by[w] = at_weight(sm[wave0 + w][c], sl[wave0 + w][c], most);
                sum += by[w] * sl[wave0 + w][c];
            }
            const float scale = whole ? at_scale(most, sum) : 1.0f;
#pragma unroll
            for (int w = 0; w < TEAM; ++w) sm[wave0 + w][c] = by[w] * scale;
            top[team][c] = most;
            sl[wave0][c] = sum;
        }
        __syncthreads();
        for (int x = member * 64 + lane; x < min(16, here - t * 16) * W; x += 64 * TEAM) {
            const int c = x / W, d = x % W * 8;
            f8 v = {};
#pragma unroll
            for (int w = 0; w < TEAM; ++w) {
                f8 y;
                __builtin_memcpy(&y, __builtin_assume_aligned(&lds[((wave0 + w) * 16 + c) * kPitch + d], 16), sizeof y);
                v += sm[wave0 + w][c] * y;
            }
            if (whole) {
                if (d < a.c.dim) write_row<T>(a, b, head, row0 + t * 16 + c, d, v);
            } else {
                const size_t at = part + t * 16 + c;
                __builtin_memcpy(__builtin_assume_aligned(a.part_o + at * DP + d, 16), &v, sizeof v);
                if (d == 0) {
                    const f2 z = {top[team][c], sl[wave0][c]};
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

// The same for the other forms' calls: a wave a row, whose lanes take the splits'
// maxima and sums, and then eight channels each of every few splits; nothing
// waits for another wave.  64 tokens of 32 heads behind a prefix in two splits:
// 3.4 us, where a workgroup a row takes 4.7.
template <int DP, class T, int NT, int MODE>
__global__ __launch_bounds__(kAtJoin) void k_attend_join_rows(AtArgs<MODE> a) {
    constexpr int W = DP / 8, G = 64 / W, K = kAtMaxSplits / 64, Y = 4, tile_rows = 16 * NT;
    const int lane = threadIdx.x & 63, g = lane / W, d = lane % W * 8;
    const unsigned rows = a.n * a.group, bh = blockIdx.y;
    const unsigned row = __builtin_amdgcn_readfirstlane(blockIdx.x * (kAtJoin / 64) + (threadIdx.x >> 6));
    if (row >= rows) return;
    const unsigned nrt = (rows + tile_rows - 1) / tile_rows, place = nrt - 1 - row / tile_rows;
    const int b = a.heads_(bh);
    size_t first = ((size_t)bh * nrt + place) * a.splits * tile_rows + row % tile_rows, stacked = 0;
    int splits = a.splits, stack_splits = 0, pitch = tile_rows;
    if constexpr (MODE == kAtStack) {
        const unsigned all = a.B * rows, at = b * rows + row, tiles = (all + tile_rows - 1) / tile_rows;
        stacked = ((size_t)(bh - b * a.c.heads) * tiles + (tiles - 1 - at / tile_rows)) * a.stack_splits * tile_rows + at % tile_rows;
        pitch = a.own_rows;
        first = a.own_part + ((size_t)bh * nrt + place) * a.splits * pitch + row % tile_rows;
        stack_splits = a.stack_splits;
        splits += stack_splits;
    }
    // the row of a split's partial result
    auto part = [&](int s) {
        s = min(s, splits - 1);
        return s < stack_splits ? stacked + (size_t)s * tile_rows : first + (size_t)(s - stack_splits) * pitch;
    };
    f2 z[K];
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (k * 64 < splits) __builtin_memcpy(&z[k], __builtin_assume_aligned(a.part_ml + part(k * 64 + lane) * 2, 8), 8);
    f8 y[Y];
#pragma unroll
    for (int j = 0; j < Y; ++j) __builtin_memcpy(&y[j], __builtin_assume_aligned(a.part_o + part(g + j * G) * DP + d, 16), 32);
    __builtin_amdgcn_sched_barrier(0);
    float most = -INFINITY, sum = 0.0f, weight[K] = {};
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (k * 64 < splits) most = fmaxf(most, z[k][0]);
    most = lanes64(most, [](float x, float y) { return fmaxf(x, y); });
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (k * 64 + lane < splits) {
            weight[k] = at_weight(z[k][0], z[k][1], most);
            sum += weight[k] * z[k][1];
        }
    sum = lanes64(sum, [](float x, float y) { return x + y; });
    const float scale = at_scale(most, sum);
    f8 v = {};
    for (int s = 0; s < splits; s += Y * G) {
        f8 x[Y];
#pragma unroll
        for (int j = 0; j < Y; ++j) {
            x[j] = y[j];
            if (s + Y * G < splits) __builtin_memcpy(&y[j], __builtin_assume_aligned(a.part_o + part(s + (Y + j) * G + g) * DP + d, 16), 32);
        }
        // (64 is a multiple of the splits of a step)
        float of = weight[0];
#pragma unroll
        for (int k = 1; k < K; ++k) of = s >= k * 64 ? weight[k] : of;
#pragma unroll
        for (int j = 0; j < Y; ++j) {
            const int split = s + j * G + g;
            const float by = __shfl(of, split % 64) * scale;
            if (split < splits) v += by * x[j];
        }
    }
    // the groups of the wave
#pragma unroll
    for (int x = W; x < 64; x <<= 1)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += __shfl_xor(v[e], x);
    if (lane < W && d < a.c.dim) write_row<T>(a, b, bh - b * a.c.heads, row, d, v);
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

// How the tiles of a workgroup's rows are split: not where they are so few a
// wave.  Returns the threads of the launch.
static long long split_plan(AttendArgs& a, int precision, long long tiles, int few) {
    const int bytes = a.c.dp * (precision == WF_BF16 ? 2 : 4), nt = row_tiles(a, precision), rows = a.n * a.group;
    const int waves = nt == 1 && bytes < 1024 ? 8 : 4;
    const long long groups = (long long)a.B * a.c.heads * ((rows + 16 * nt - 1) / (16 * nt));
    // A tile takes a wave about 1 us and the join 3, so up to four tiles a wave
    // are not split; more are, down to one tile each.  us with no split, four
    // tiles each, two and one: a token over 1001 (8 heads of 128, bf16) 7.3, 7.4,
    // 8.3, 7.4, over 2047 11.0, 10.2, 8.5, 7.8, over 8192 33, 10.6, 9.1, 8.7; 45
    // fp32 rows over 1024 7.2, 7.2, 8.5, 7.8, over 4096 16.9, 10.7, 9.0, 8.5.
    const long long by_len = tiles <= few * waves ? 1 : (tiles + waves - 1) / waves;
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
    return groups * a.splits * waves * 64;
}

static long long tiles_of(long long tokens) { return (tokens + kKvTile - 1) / kKvTile; }

long long attend_plan(AttendArgs& a, int precision) {
    const int bytes = a.c.dp * (precision == WF_BF16 ? 2 : 4), nt = row_tiles(a, precision), rows = a.n * a.group;
    const long long groups = (long long)a.B * a.c.heads * ((rows + 16 * nt - 1) / (16 * nt));
    const long long threads = split_plan(a, precision, tiles_of(a.max_visible), 4);
    // A token each of sequences that may be of unequal lengths, and two
    // workgroups on most compute units.  With more of them the units take the
    // next as they finish: in the order given and longest first, 128 sequences
    // of 0 to 8192 tokens 129 / 119 us, but of 8192 each 199 / 207, and 256 of 0
    // to 8192 226 / 228, of 8192 each 395 / 406.
    const bool two = groups > kAtTarget && groups <= 2 * kAtTarget && bytes <= 256 && a.splits == 1;
    a.ahead = nt == 1 && rows <= 16 && a.B > 1 && a.B <= kAtBatch && two ? (int)(kAtTarget / a.c.heads) : 0;
    return threads;
}

// The other forms' calls are split from a tile a wave later: a second launch is 3
// us of the host, which a call waits for that no graph holds.  us with and
// without a split, a call after another and (from a graph): a token, 38 tiles,
// 10.6 / 9.6 (8.0 / 9.4), 45 fp32 rows, 33 tiles 10.8 / 8.1 (8.3 / 8.1), 38 tiles
// 10.5 / 8.9 (8.3 / 9.0); 46 tiles 10.5 / 10.4 (8.0 / 10.3).
constexpr int kAtFew = 5;

// A window's rows read its tokens, those that the other rows of their tile are
// ahead by under a causal order, and the first tokens.
static long long window_tiles(const AttendRunsArgs& a, int precision) {
    const int rows = 16 * row_tiles(a, precision), apart = (rows + a.group - 1) / a.group, ahead = (apart < a.n ? apart : a.n) - 1;
    const long long all = tiles_of(a.max_visible), some = tiles_of(a.sinks) + tiles_of((long long)a.window + ahead) + 1;
    return some < all ? some : all;
}

long long attend_window_plan(AttendRunsArgs& a, int precision) { return split_plan(a, precision, window_tiles(a, precision), kAtFew); }

// Workgroups that read the same tokens, on one die: its cache then holds them.
// Units, all row tiles of a sequence and head (over a shared prefix each row
// tile), are dealt to the dies in the order of heads where they come out even.
// us with and without: 64 tokens of 32 / 8 heads of 128 behind 8192, 100 of their
// own each, 24.1 / 25.0, 16 such tokens 12.6 / 13.1; without own tokens 64 of 64
// channels 19.6 / 20.2, 256 of 128 65.0 / 66.2; 8 x 128 causal rows behind 16384
// 357 / 372.
static void deal(AttendRunsArgs& a, long long units, long long workgroups) {
    a.units_of_die = 0;
    if (units % kXcds) return;
    a.units_of_die = (int)(units / kXcds);
    a.unit_workgroups = (int)workgroups;
    a.unit_.by((unsigned)workgroups);
    a.batch_.by((unsigned)a.B);
}

// Time of a launch in tiles of 16 rows: workgroups on a compute unit in turn, each
// with a start and an end as long as kAtEnds tiles take, a tile of 32 rows as long
// as 1.64 of 16; the join as long as kAtEnds too, and its launch kAtLaunch where
// the host is what a call waits for.  (1.02 us for eight waves' tiles
// of 16 rows, 0.91 for four waves' of 32; 64 tokens of 32 / 8 heads of 128 behind
// 8192 in one to eight splits: 37.9, 25.8, 29.4, 29.6, -, 31.0, -, 31.1 us, with 32
// rows 60.7, 35.5, 28.1, 24.4, -, 27.3, -, 28.4; 16 tokens in 2, 4, 8 and 16 splits
// 21.9, 15.0, 12.3, 15.3.)
constexpr double kAtEnds = 24.0, kAtLaunch = 12.0;
static double cost_of(long long groups, long long tiles, long long splits, int nt) {
    const double turns = (double)((groups * splits + kAtTarget - 1) / kAtTarget);
    return (nt == 2 ? 1.64 : 1.0) * turns * ((tiles + splits - 1) / splits + kAtEnds);
}

// The rows of all sequences over the prefix and each one's over its own tokens in
// one launch, with a join: its time in tiles, or less than 0 where the partial
// results do not fit the workspace.
static double stack_plan(AttendRunsArgs& a, int precision, int nt) {
    const int waves = nt == 1 && a.c.dp * (precision == WF_BF16 ? 2 : 4) < 1024 ? 8 : 4;
    const long long rows = (long long)a.n * a.group, tile = 16 * nt, all = (a.B * rows + tile - 1) / tile, each = (rows + tile - 1) / tile;
    const long long shared = a.c.heads * all, own = a.max_visible ? a.B * a.c.heads * each : 0;
    const long long shared_tiles = tiles_of(a.max_first), own_tiles = tiles_of(a.max_visible), own_rows = rows < tile ? rows : tile;
    const long long room = (long long)attend_work_rows(a.c.dp);
    double best = -1.0;
    // the most splits that the compute units hold in one, two .. turns, of four tiles or more
    for (int turns = 1; turns <= 4; ++turns) {
        long long s = kAtTarget * turns / shared, most = shared_tiles / 4;
        most = most < kAtMaxSplits / 2 ? most : kAtMaxSplits / 2;
        s = s < most ? s : most;
        s = s < 1 ? 1 : s;
        // own tokens in parts as long as the prefix's, but no more of them than workgroups for two turns
        const long long share = (shared_tiles + s - 1) / s > 4 * waves ? (shared_tiles + s - 1) / s : 4 * waves;
        long long o = own ? (own_tiles + share - 1) / share : 0, fill = own ? 2 * kAtTarget / own : 0;
        fill = fill < kAtMaxSplits / 2 ? fill : kAtMaxSplits / 2;
        o = o < fill ? o : fill;
        o = own && o < 1 ? 1 : o;
        // (so that a part of a batch that fits does)
        while (shared * s * tile + own * o * own_rows > room && (o > 1 || s > 1)) (o > 1 ? o : s) /= 2;
        if (shared * s * tile + own * o * own_rows > room) continue;
        const double part = own ? (nt == 2 ? 1.64 : 1.0) * own * o / kAtTarget * ((own_tiles + o - 1) / o + kAtEnds) : 0.0;
        const double cost = cost_of(shared, shared_tiles, s, nt) + part + kAtEnds + kAtLaunch;
        if (best >= 0.0 && cost >= best) continue;
        best = cost;
        a.stack_splits = (int)s; a.splits = (int)o;
    }
    if (best < 0.0) return best;
    a.stack_splits_.by(a.stack_splits); a.splits_.by(a.splits ? a.splits : 1u);
    a.stack_tiles_.by((unsigned)all); a.tiles_.by((unsigned)each);
    a.heads_.by(a.c.heads); a.group_.by(a.group); a.n_.by(a.n);
    a.stack_blocks = (int)(shared * a.stack_splits);
    a.own_part = shared * a.stack_splits * tile;
    a.own_rows = (int)own_rows;
    deal(a, shared, a.stack_splits);
    return best;
}

long long attend_shared_plan(AttendRunsArgs& a, int precision, AttendStack* stack) {
    const long long first = tiles_of(a.max_first), own = tiles_of(a.max_visible);
    const long long threads = split_plan(a, precision, first + own, kAtFew);
    const int nt = row_tiles(a, precision), rows = a.n * a.group;
    *stack = {0, 1};
    if (a.B < 2 || !first || (long long)a.B * rows >= 1 << 24) return threads;
    double best = cost_of((long long)a.B * a.c.heads * ((rows + 16 * nt - 1) / (16 * nt)), first + own, a.splits, nt) + (a.splits > 1 ? kAtEnds + kAtLaunch : 0.0);
    for (int tiles = 1; tiles <= (a.c.dp * (precision == WF_BF16 ? 2 : 4) <= 256 ? 2 : 1); ++tiles) {
        // as many sequences as the workspace takes, in as many launches as that makes
        AttendRunsArgs x = a;
        for (int launches = 1; launches <= 64 && launches < a.B; launches *= 2) {
            x.B = (a.B + launches - 1) / launches;
            const double cost = launches * stack_plan(x, precision, tiles);
            if (cost < 0.0) continue;
            if (cost < best) {
                best = cost;
                *stack = {x.B, tiles};
            }
            break;
        }
    }
    return stack->sequences ? 0 : threads;
}

// Calls by runs whose teams are smaller than a workgroup, and not split.
template <int DP, class T, int NT, int TEAM>
static void launch_teams(const AttendRunsArgs& a, long long groups, hipStream_t st) {
    constexpr int kTeams = kAtWaves<DP, T, NT> / TEAM;
    const long long blocks = a.units_of_die ? kXcds * (((long long)a.units_of_die * a.unit_workgroups + kTeams - 1) / kTeams) : (groups + kTeams - 1) / kTeams;
    hipLaunchKernelGGL((k_attend<DP, T, NT, kAtRuns, TEAM>), dim3((unsigned)blocks), dim3(64 * kAtWaves<DP, T, NT>), 0, st, a);
}

// The kernel of a form and, where its calls are split, the join.
template <int DP, class T, int NT, int MODE>
static void launch_form(const AtArgs<MODE>& a, hipStream_t st) {
    const int rows = a.n * a.group;
    long long groups = (long long)a.B * a.c.heads * ((rows + 16 * NT - 1) / (16 * NT)) * a.splits;
    if constexpr (MODE == kAtRuns) {
        if (a.team == 1) return launch_teams<DP, T, NT, 1>(a, groups, st);
        if (a.team == 2) return launch_teams<DP, T, NT, 2>(a, groups, st);
    }
    if constexpr (MODE == kAtStack) groups += a.stack_blocks;
    hipLaunchKernelGGL((k_attend<DP, T, NT, MODE>), dim3((unsigned)groups), dim3(64 * kAtWaves<DP, T, NT>), 0, st, a);
    if constexpr (MODE == kAtPlain || MODE == kAtMask) {
        if (a.splits > 1) hipLaunchKernelGGL((k_attend_join<DP, T, NT>), dim3(rows, a.B * a.c.heads), dim3(kAtJoin), 0, st, a);
    } else if (MODE == kAtStack || a.splits > 1) {
        const int per = kAtJoin / 64;
        hipLaunchKernelGGL((k_attend_join_rows<DP, T, NT, MODE>), dim3((rows + per - 1) / per, a.B * a.c.heads), dim3(kAtJoin), 0, st, a);
    }
}

template <int DP, class T, int MODE>
static void launch_nt(const AtArgs<MODE>& a, int nt, hipStream_t st) {
    if constexpr (kAtTwoTiles<DP, T>)
        if (nt == 2) return launch_form<DP, T, 2, MODE>(a, st);
    launch_form<DP, T, 1, MODE>(a, st);
}

template <class T, int MODE>
static void launch_dp(const AtArgs<MODE>& a, int nt, hipStream_t st) {
    if (a.c.dp == 64) launch_nt<64, T, MODE>(a, nt, st);
    else if (a.c.dp == 128) launch_nt<128, T, MODE>(a, nt, st);
    else launch_nt<256, T, MODE>(a, nt, st);
}

template <int MODE>
static void launch(const AtArgs<MODE>& a, int precision, int nt, hipStream_t st) {
    if (precision == WF_BF16) launch_dp<__bf16, MODE>(a, nt, st);
    else launch_dp<float, MODE>(a, nt, st);
}

void launch_attend(const AttendArgs& a, int precision, hipStream_t st) {
    const int nt = row_tiles(a, precision);
    if (a.mask) launch<kAtMask>(a, precision, nt, st);
    else launch<kAtPlain>(a, precision, nt, st);
}

// Waves that share a tile of rows: a workgroup's, or two or one where there are
// rows enough to fill the chip so, since a team's start and end cost each of its
// waves as long as three tiles take.  By an estimate in tiles of the chip's work,
// or of one wave where that is longer (a tile takes 0.63 of the time where the
// SIMD has no other wave), and of the end, when not all of it is busy.  us with a
// workgroup's waves, two and one: 2 x 8191 rows with windows of 1024 and 16 first
// (32 / 8 heads of 128, bf16) 498 / 427 / 394, 1024 such rows 38.7 / 33.7 / 39.2,
// 19 x 278 rows of 6 / 3 fp32 heads with windows of 5 38.0 / 15.3 / 11.1, 2 x 600
// rows of 8 / 2 heads of 256 with windows of 128 21.8 / 13.3 / 18.7, 2 x 900 fp32
// rows of 10 / 5 heads of 64 with windows of 2000 47.2 / 55.4 / 65.6, 8 x 128 rows
// behind 1000 tokens 38.7 / 33.6 / 39.8, 4 x 992 of 21 / 3 heads behind 6859 and 590
// own 454 / 476 / 500.
static int team_of(const AttendRunsArgs& a, int precision, int nt, long long tiles) {
    const int bytes = nt * a.c.dp * (precision == WF_BF16 ? 2 : 4), waves = nt == 1 && bytes < 1024 ? 8 : 4, rows = a.n * a.group;
    if (a.splits > 1) return waves;
    // (as k_attend's registers allow)
    const double slots = 4.0 * kAtTarget * (bytes <= 256 ? (nt == 1 ? 4 : 3) : (bytes <= 512 ? 2 : 1));
    const double groups = (double)a.B * a.c.heads * ((rows + 16 * nt - 1) / (16 * nt));
    int best = waves;
    double least = 0.0;
    for (int team : {waves, 2, 1}) {
        const double one = 3.0 + (double)((tiles + team - 1) / team), all = groups * team * one / slots;
        const double cost = (all > 0.63 * one ? all : 0.63 * one) + 0.25 * one;
        if (team != waves && cost > 0.98 * least) continue;
        least = cost;
        best = team;
    }
    return best;
}

static void launch_runs(const AttendRunsArgs& a, int precision, long long tiles, hipStream_t st) {
    const int nt = row_tiles(a, precision), rows = a.n * a.group;
    AttendRunsArgs x = a;
    x.team = team_of(a, precision, nt, tiles);
    // Sequences may be of unequal lengths, so a die gets all of a head's or none:
    // with fewer heads than dies one long sequence would have a die to itself.  us
    // dealt and not, 8 sequences of 512 rows, 8 query heads a key head, windows of
    // 4000: one of 8192 tokens and seven empty, 1 head 97 / 37, 2 heads 100 / 44, 4
    // heads 117 / 82; all of 8192 106 / 107, 195 / 195, 376 / 378.  (Over a prefix
    // tiles differ as their rows do, but a tile has splits for a die's compute units
    // at least: 64 tokens of one head of which 8 see 65536 26.0 / 25.4, 8192 11.7 / 11.4.)
    if (a.c.heads % kXcds == 0) deal(x, (long long)a.B * a.c.heads, (long long)((rows + 16 * nt - 1) / (16 * nt)) * a.splits);
    launch<kAtRuns>(x, precision, nt, st);
}

void launch_attend_window(const AttendRunsArgs& a, int precision, hipStream_t st) { launch_runs(a, precision, window_tiles(a, precision), st); }

void launch_attend_shared(const AttendRunsArgs& a, int precision, const AttendStack& stack, hipStream_t st) {
    if (!stack.sequences) return launch_runs(a, precision, tiles_of(a.max_first) + tiles_of(a.max_visible), st);
    // launches in turn, since they share the workspace
    const long long item = precision == WF_BF16 ? 2 : 4;
    for (int b = 0; b < a.B; b += stack.sequences) {
        AttendRunsArgs x = a;
        x.B = stack.sequences < a.B - b ? stack.sequences : a.B - b;
        x.q.p = (char*)a.q.p + b * a.q.sb * item;
        x.o.p = (char*)a.o.p + b * a.o.sb * item;
        x.table += (size_t)b * a.table_pages;
        x.visible += (size_t)b * a.n;
        x.first_visible += (size_t)b * a.n;
        stack_plan(x, precision, stack.row_tiles);
        launch<kAtStack>(x, precision, stack.row_tiles, st);
    }
}

}  // namespace wf
