// A trained block (ccdc_block): its configuration, the batch it is bound to, and what its calls share.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstdint>
#include <mutex>
#include <vector>

#include "ccdc.h"

namespace ccdc {

// What a row of the batch belongs to: the numbers that its dropout masks are made from.
struct RowOf {
    int32_t id, token, file;          // the file's number, the token's place in it, the file's place in the batch
};

// Consecutive rows of one file, of which one workgroup sums what is learned.
struct Chunk {
    int32_t file, first, rows;
};
// The same for every batch: the order of a file's sums is its own.  The sums of a chunk, written and read once more, are 4 % of what 32
// rows of bf16 values move; chunks of 16 took 0.99 of the time (14336 x 2048 bf16).
constexpr int kChunkRows = 32;

// f(first row, rows) for the chunks of a file.  (The row after the last may be 2^31.)
template <class F>
void each_chunk(int32_t rows, F f)
{
    for (int64_t t = 0; t < rows; t += kChunkRows) f((int32_t)t, (int32_t)(rows - t < kChunkRows ? rows - t : kChunkRows));
}

constexpr int64_t kJoinWidth = 16384;         // widest rows that one workgroup holds in registers

// Elements of y in all ranges of k together where its product is cut into some: those of 256 tiles.
constexpr int64_t kPartElements = (int64_t)256 * 128 * 128;

// Ranges of k that y's product is cut into where its tiles leave most of the chip without work: as many as fill it, of 512 k at
// least.  Not in training: how many there are goes by the batch's rows, and with them the bits that a file's gradient is made from.
inline int forward_parts(int64_t width, int64_t hidden_ld, int64_t rows)
{
    const int64_t tiles = (width + 127) / 128 * ((rows + 127) / 128);
    return tiles > 128 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(256 / tiles, hidden_ld / 512));
}

constexpr int64_t padded(int64_t n) { return (n + 7) / 8 * 8; }

}  // namespace ccdc

struct ccdc_block_s {
    ccdc_block_config c{};
    int elem = 4;                     // bytes of an element
    int planes = 1;                   // 16-bit numbers that an operand of a product is held in

    bool bound = false;
    int64_t M = 0;                    // tokens of the batch
    int N = 0;
    int64_t hidden_ld = 0, width_ld = 0;          // row strides of the block's own matrices: whole packs of 16 bytes
    std::vector<int32_t> first;       // [N + 1] rows the files begin at
    std::vector<ccdc::RowOf> row_of;  // [M]
    std::vector<ccdc::Chunk> chunks;
    std::vector<int32_t> chunk_first; // [N + 1]

    // bytes from the workspace's beginning: hidden values; gradients of a and u; x, dy, W_in and W_out where products do
    // not take them as they are; sums of the chunks (over all of these)
    size_t at_h = 0, at_dau = 0, at_x = 0, at_dy = 0, at_in = 0, at_out = 0, at_parts = 0, workspace_bytes = 0;
    size_t saved_h = 0, saved_p = 0, saved_q = 0, saved_bytes = 0;

    bool uploaded = false;
    int device = -1;
    int32_t *d_first = nullptr, *d_chunk_first = nullptr;
    ccdc::RowOf *d_row_of = nullptr;
    ccdc::Chunk *d_chunks = nullptr;
    void *d_tables = nullptr, *d_workspace = nullptr;       // d_first .. d_chunks are parts of the first

    // as a plan's (plan.hpp)
    mutable std::mutex ws_mutex;
    mutable void *ws_event = nullptr;
    mutable void *ws_stream = nullptr;
    mutable bool ws_used = false;
};

namespace ccdc {

// The threshold of 16-bit random numbers below which dropout takes a value out: to nearest, ties to even.
inline uint32_t dropout_threshold(double p) { return (uint32_t)std::rint(p * 65536.0); }

int bind_block(ccdc_block_t *b, int files, const int64_t *tokens, const int32_t *ids);

}  // namespace ccdc
