// The 4-bit key/value cache: layout of its pages, shared by the kernels that
// write, read and attend to it.
//
// A block of 32 consecutive channels of one token's head holds 4-bit values
// {0, 1/2, 1, 3/2, 2, 3, 4, 6} with a sign and one byte e + 127 for the power
// 2^e that they are multiplied by (255: the block reads as NaN).  gfx950
// converts two of these values with their power in one instruction, so the
// matrix operands come from the cache's words without a table.
//
// A page holds `page` tokens of every head, head by head; a head's part is a
// row of records of 32 tokens, so that a wave streams one head's tokens as one
// run.  A record is laid out as the attention's lanes take it: lane l = 16 g +
// i reads 16 bytes at 16 l of every kilobyte (piece), so each load of a wave
// is one run, and both matrix operands come out of the loaded words without an
// exchange between lanes.  With DP the head size rounded up to 64, 128 or 256:
//   key values    16 DP bytes.  The key operand's row i of its half a is token
//                 8 (i / 4) + 4 a + i % 4, and lane (g, i) holds its quarter
//                 [DP/4 g, DP/4 (g + 1)) of the head: DP/8 bytes for a = 0,
//                 then for a = 1
//   value values  16 DP bytes.  Lane (g, i) holds channels [DP/16 i, DP/16 (i +
//                 1)) of tokens 8 g .. 8 g + 7, DP/32 bytes a token: rows of
//                 the value operand are channels and its k axis is tokens, so
//                 the product with the probabilities needs no transposition
//   key powers    DP bytes: the lane's (where two lanes' quarters share a block,
//                 the pair's), for a = 0 and then 1
//   value powers  [DP/32][32] bytes: a lane's eight tokens in one run
// Channel d of a byte is in its low half for even d.  A token's bytes are its
// own: tokens can be written in any order.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "wf_call.h"

namespace wf {

constexpr int kKvBlock = 32;         // channels that share a power
constexpr int kKvTile = 32;          // tokens of a tile
constexpr int kKvNan = 255;          // power byte of a block that holds no finite value
constexpr int kKvMaxPower = 125;     // powers lie in 2^-125 .. 2^125: every value is a normal number
// device error word: a token or row past the page table, a table entry outside the pool
constexpr int kErrKvRange = 1, kErrKvPage = 2;

// Workgroups that a call is split into: one for each compute unit.  us for 192
// / 256 / 320 / 512: one token over 131072 34 / 33 / 40 / 33; 45 fp32 rows over
// 32300 16 / 14 / 18 / 15; 56 fp32 rows of 256 channels over 20011 27 / 23 / 35
// / 30 (the last ones wait for a place, and the join has more to read).
constexpr int kAtTarget = 256;
// Rows of partial results that a cache's workspace holds: what attend_plan's
// calls can take.  At most 2 kAtTarget workgroups share calls of up to kAtTarget
// of them, and four each a quarter more; they have 32 rows for 128 channels in
// bf16, else 16 (64 channels have 32 from 512 workgroups on, which no call that
// is split has).
inline size_t attend_work_rows(int dp) { return (size_t)4 * (kAtTarget * 5 / 4) * (dp == 128 ? 32 : 16); }

// n / d for n < 2^31 by a product: with 2^l the power from d up, mul =
// floor(2^(31 + l) / d) + 1 is off by less than 2^(31 + l) / (d n).  (The
// compiler's own division is some 25 dependent instructions, and a short
// call's kernels begin with four.)
struct KvDiv {
    unsigned mul;
    int shift;
    void by(unsigned d) {
        for (shift = 31; d > 1ull << (shift - 31);) ++shift;
        mul = (unsigned)((1ull << shift) / d + 1);
    }
    __device__ unsigned operator()(unsigned n) const { return (unsigned)((unsigned long long)n * mul >> shift); }
};

struct KvCache {                     // what the kernels need of a cache
    uint8_t* pool;
    int* err;
    int heads, dim, pages;
    int page_shift;                  // log2 of a page's tokens
    int dp;                          // channels held of a head: 64, 128 or 256
    __host__ __device__ size_t head_bytes() const { return ((size_t)dp * 17 / 16) << page_shift; }
    __host__ __device__ size_t page_bytes() const { return head_bytes() * heads; }
};

// Reductions over lanes in registers (all 64 lanes active), where the exchange
// by __shfl_xor waits for the LDS unit.  lanes16: over a row of 16, lanes64: over
// the four rows too, lanes4: over four.
template <int CTRL>
__device__ __forceinline__ float lane_move(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ __forceinline__ int lane_move(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, true); }

template <class T, class F>
__device__ __forceinline__ T lanes4(T x, F f) {
    x = f(x, lane_move<0xb1>(x));        // quad_perm 1 0 3 2
    return f(x, lane_move<0x4e>(x));     // quad_perm 2 3 0 1
}
template <class T, class F>
__device__ __forceinline__ T lanes16(T x, F f) {
    x = lanes4(x, f);
    x = f(x, lane_move<0x124>(x));       // the quad before
    return f(x, lane_move<0x128>(x));    // and the two before these
}
// over the four rows: f of both halves of a swap of x with itself
template <class F>
__device__ __forceinline__ float lane_rows(float x, F f) {
    auto two = [&](const auto& r) {
        const unsigned a = r[0], b = r[1];
        return f(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
    };
    unsigned u = __builtin_bit_cast(unsigned, x);
    u = __builtin_bit_cast(unsigned, two(__builtin_amdgcn_permlane16_swap(u, u, false, false)));
    return two(__builtin_amdgcn_permlane32_swap(u, u, false, false));
}
template <class F>
__device__ __forceinline__ float lanes64(float x, F f) { return lane_rows(lanes16(x, f), f); }

// Offsets in a record.
template <int DP>
struct KvLayout {
    static constexpr int kBlocks = DP / kKvBlock;
    static constexpr int kUnit = DP / 32;       // bytes of a token in one lane's values
    static constexpr int kRows = DP / 16;       // channels of a token in one lane's values
    static constexpr int kQuarter = DP / 8;     // bytes of a key in one lane
    static constexpr int kLane = DP / 4;        // bytes of a record's keys (or values) in one lane
    static constexpr int kPowers = DP == 256 ? 4 : 2;   // key powers of a lane, both halves
    static constexpr int kRecord = 34 * DP;
    // byte n of a lane's keys or values
    __device__ static constexpr int piece(int lane, int n) { return n / 16 * 1024 + lane * 16 + n % 16; }
    __device__ static constexpr int key_lane_powers(int lane) {
        return 32 * DP + (DP == 64 ? (lane / 32 * 16 + lane % 16) : lane) * kPowers;
    }
    __device__ static constexpr int value_powers(int block) { return 33 * DP + block * kKvTile; }
    // byte of channels d, d + 1 of token t; of a value, a lane's run ends after
    // kRows channels and the next lane's follows 16 bytes on (kUnit 2)
    __device__ static int key_at(int t, int d) {
        const int i = t / 8 * 4 + t % 4, n = d / 2;
        return piece(n / kQuarter * 16 + i, t / 4 % 2 * kQuarter + n % kQuarter);
    }
    __device__ static int key_power(int t, int block) {
        const int i = t / 8 * 4 + t % 4, a = t / 4 % 2;
        if (DP < 256) return 32 * DP + (block * 16 + i) * 2 + a;
        return 32 * DP + ((block / 2 * 16 + i) * 2 + a) * 2 + block % 2;
    }
    __device__ static int value_at(int t, int d) {
        return 16 * DP + piece(t / 8 * 16 + d / kRows, t % 8 * kUnit + d % kRows / 2);
    }
    __device__ static int value_power(int t, int block) { return value_powers(block) + t; }
};

struct KvTokens {                    // the tokens a write or read takes
    const int *table, *first, *counts;
    int table_pages, B, n;
    int records;                     // of a sequence and head that n tokens may reach into
    KvDiv heads_, records_;
};

struct AttendArgs {
    KvCache c;
    KvRows q, o;
    const int *table, *visible;
    const uint8_t* mask;
    long long mb, mr;                // mask strides: sequence, row
    int table_pages, B, n, group;    // group: query heads of a key head
    int max_visible, splits;
    int ahead;                       // > 0: sequences by length, this many from the longest down
    float scale_log2;                // scale * log2(e)
    KvDiv splits_, tiles_, heads_, group_;   // tiles_: of rows
    float *part_o, *part_ml;         // partial results: channels, and (maximum, sum)
};

// What the kernels of the other forms need beside: a first run of tokens before
// the sequence's own.
struct AttendRunsArgs : AttendArgs {
    // a prefix that lies in the cache once
    const int *first_table, *first_visible;
    int first_pages, max_first;
    int team;                        // waves that share a tile of rows
    int window, sinks;               // window > 0: the first run is the sequence's first tokens
    // rows of all sequences together over the prefix, as workgroups before the others
    int stack_blocks, stack_splits;
    KvDiv stack_splits_, stack_tiles_, n_;
    long long own_part;              // the first row of the others' partial results,
    int own_rows;                    // and how many a tile has
    // > 0: a unit of work's place goes by its die, units in the order of heads:
    // this many of each die's
    int units_of_die, unit_workgroups;
    KvDiv unit_, batch_;
};

void launch_kv_write(const KvCache&, int precision, const KvRows& k, const KvRows& v, const KvTokens&, hipStream_t);
void launch_kv_read(const KvCache&, int precision, const KvRows& k, const KvRows& v, const KvTokens&, hipStream_t);
// The splits of a call.  Returns the threads of its launch.
long long attend_plan(AttendArgs&, int precision);
void launch_attend(const AttendArgs&, int precision, hipStream_t);
long long attend_window_plan(AttendRunsArgs&, int precision);
void launch_attend_window(const AttendRunsArgs&, int precision, hipStream_t);
// How the rows of a batch over its prefix are taken: those of so many sequences
// together (0: each sequence's for itself, in one launch), in so many tiles of 16.
struct AttendStack { int sequences, row_tiles; };
long long attend_shared_plan(AttendRunsArgs&, int precision, AttendStack*);
void launch_attend_shared(const AttendRunsArgs&, int precision, const AttendStack&, hipStream_t);

}  // namespace wf
