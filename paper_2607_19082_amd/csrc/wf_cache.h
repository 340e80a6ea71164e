// The 4-bit key/value cache: layout of its pages, shared by the kernels that
// write, read and attend to it.
//
// A block of 32 consecutive channels of one token's head holds 4-bit values
// {0, 1/2, 1, 3/2, 2, 3, 4, 6} with a sign and one byte e + 127 for the power
// 2^e that they are multiplied by (255: the block reads as NaN).  gfx950
// converts two of these values with their power in one instruction, so the
// matrix operands come from the cache's words without a table.
//
// A page holds `page` tokens of every head, head by head, so that a wave
// streams one head's keys and values as long runs.  Of one head, with DP the
// head size rounded up to 64, 128 or 256 and P the page's tokens:
//   key values    [P][DP/2] bytes, channel d in the low (even d) or high half
//                 of byte d/2: an MFMA operand row is a key, and each of its
//                 four k-groups of lanes reads a quarter of the head in one run
//   key powers    [P][DP/32]
//   value values  [P/32][4][16][8][DP/32] bytes: of a group of 32 tokens,
//                 eight tokens of DP/16 channels together for each lane of the
//                 operand whose rows are channels and whose k axis is tokens
//                 (lane 16 g + i: tokens 8 g .. 8 g + 7, channels from
//                 DP/16 i), so that the product with the probabilities needs no
//                 transposition
//   value powers  [P/32][DP/32][32]: a lane's eight tokens in one run
// A token's bytes are its own: tokens can be written in any order.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "wf_internal.h"

namespace wf {

constexpr int kKvBlock = 32;         // channels that share a power
constexpr int kKvTile = 32;          // tokens of a tile
constexpr int kKvNan = 255;          // power byte of a block that holds no finite value
constexpr int kKvMaxPower = 125;     // powers lie in 2^-125 .. 2^125: every value is a normal number
// device error word: a token or row past the page table, a table entry outside the pool
constexpr int kErrKvRange = 1, kErrKvPage = 2;

// rows of partial results that a cache's workspace holds (see attend_plan)
constexpr long long kAttendWorkRows = 1 << 16;

struct KvCache {                     // what the kernels need of a cache
    uint8_t* pool;
    int* err;
    int heads, dim, pages;
    int page_shift;                  // log2 of a page's tokens
    int dp;                          // channels held of a head: 64, 128 or 256
    __host__ __device__ size_t head_bytes() const { return ((size_t)dp * 17 / 16) << page_shift; }
    __host__ __device__ size_t page_bytes() const { return head_bytes() * heads; }
};

// Offsets in one head's part of a page.
template <int DP>
struct KvLayout {
    static constexpr int kBlocks = DP / kKvBlock;
    static constexpr int kUnit = DP / 32;       // bytes of a token in one lane's value run
    static constexpr int kRows = DP / 16;       // channels of a token in one lane's value run
    __device__ static size_t k_codes(int t) { return (size_t)t * (DP / 2); }
    __device__ static size_t k_powers(int shift, int t) { return ((size_t)(DP / 2) << shift) + (size_t)t * kBlocks; }
    __device__ static size_t v_base(int shift) { return (size_t)(DP / 2 + kBlocks) << shift; }
    // the run of a lane (group g of eight tokens, channels from kRows * i) in the tile of token t
    __device__ static size_t v_codes(int shift, int tile, int g, int i) {
        return v_base(shift) + (((size_t)tile * 4 + g) * 16 + i) * 8 * kUnit;
    }
    __device__ static size_t v_powers(int shift, int tile, int block) {
        return v_base(shift) + ((size_t)(DP / 2) << shift) + ((size_t)tile * kBlocks + block) * kKvTile;
    }
};

struct KvRows {                      // [b][row][head][dim], the channels contiguous
    void* p;
    long long sb, sr, sh;            // strides in elements
};

struct KvTokens {                    // the tokens a write or read takes
    const int *table, *first, *counts;
    int table_pages, B, n;
};

struct AttendArgs {
    KvCache c;
    KvRows q, o;
    const int *table, *visible;
    const uint8_t* mask;
    long long mb, mr;                // mask strides: sequence, row
    int table_pages, B, n, group;    // group: query heads of a key head
    int max_visible, splits;
    float scale_log2;                // scale * log2(e)
    float *part_o, *part_ml;
};

void launch_kv_write(const KvCache&, int precision, const KvRows& k, const KvRows& v, const KvTokens&, hipStream_t);
void launch_kv_read(const KvCache&, int precision, const KvRows& k, const KvRows& v, const KvTokens&, hipStream_t);
// Splits of a call and the rows of partial results that it leaves in the
// workspace (0: the kernel writes the output itself).
long long attend_plan(AttendArgs&, int precision);
void launch_attend(const AttendArgs&, int precision, hipStream_t);

}  // namespace wf
