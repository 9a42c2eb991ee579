// The host side of a trained block (csrc/block.cpp, csrc/block.hpp: no GPU code in them) under AddressSanitizer + UBSan, a
// check a command.  Test infrastructure only.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "block.hpp"

// thresholds P ...: what dropout with these probabilities takes out of 65536
static int thresholds(int count, char **p)
{
    for (int i = 0; i < count; i++) std::printf("%u\n", ccdc::dropout_threshold(std::strtod(p[i], nullptr)));
    return 0;
}

// chunks ROWS: the chunks of a file of so many rows, counted, and looked at: without a gap, none empty or too long
static int chunks(long long rows)
{
    long long next = 0, count = 0;
    bool fine = true;
    ccdc::each_chunk((int32_t)rows, [&](int32_t first, int32_t of) {
        fine = fine && first == next && of > 0 && of <= ccdc::kChunkRows;
        next += of;
        count++;
    });
    std::printf("%lld\n", fine && next == rows ? count : -1);
    return 0;
}

#define WANT(condition)                                                                                              \
    do {                                                                                                             \
        if (!(condition)) {                                                                                          \
            std::fprintf(stderr, "%s: mode %d, width %lld, hidden %lld, batch %zu\n", #condition, mode, (long long)width, \
                         (long long)hidden, which);                                                                  \
            return 1;                                                                                                \
        }                                                                                                            \
    } while (0)

// Regions of a buffer that are in use together: on 16 bytes, one after the other, each as large as what is indexed there.
struct Region {
    size_t at;
    int64_t bytes;
};
static bool apart(const std::vector<Region> &all, size_t end)
{
    for (size_t i = 0; i < all.size(); i++)
        if (all[i].at % 16 || all[i].at + (size_t)all[i].bytes > (i + 1 < all.size() ? all[i + 1].at : end)) return false;
    return true;
}

// batches: configurations and batches through the host side of a block; its tables, and what the calls index of what is saved and of the
// workspace, reckoned from the interface's formulas.
static int batches()
{
    const std::vector<std::vector<int64_t>> tokens = {{0}, {1}, {0, 0, 0}, {3, 0, 40}, {32, 33, 31, 0}, {64}, {65}, {300, 1, 0, 129}, {0, 0, 7}, {5000}};
    const int64_t widths[] = {1, 7, 8, 9, 64, 130, 515, 1000, 4096, 16384, 16385, 20000}, hiddens[] = {1, 8, 133, 520, 1024, 4097, 11264};
    long count = 0;
    for (int mode : {CCDC_F32_SUM, CCDC_F32_SUM_XOR, CCDC_BF16_SUM_XOR, CCDC_F16_SUM_XOR})
        for (int64_t width : widths)
            for (int64_t hidden : hiddens) {
                size_t which = 0;
                const ccdc_block_config c = {width, hidden, mode, CCDC_ACT_GELU, CCDC_NORM_RMS, 3, 1e-6f, 1.0f, 0.0f, 0.5f};
                ccdc_block_t *b = nullptr;
                WANT(ccdc_block(&c, &b) == CCDC_OK);
                const bool narrow = mode == CCDC_BF16_SUM_XOR || mode == CCDC_F16_SUM_XOR;
                const int64_t elem = narrow ? 2 : 4, operand = narrow ? 2 : 6, d = (width + 7) / 8 * 8, F = (hidden + 7) / 8 * 8;
                for (; which < tokens.size(); which++) {
                    const auto &of = tokens[which];
                    std::vector<int32_t> ids;
                    for (size_t n = 0; n < of.size(); n++) ids.push_back((int32_t)(7 * n + 2));
                    const bool numbered = which % 2;
                    WANT(ccdc::bind_block(b, (int)of.size(), of.data(), numbered ? ids.data() : nullptr) == CCDC_OK);
                    int64_t M = 0, row = 0, chunk = 0;
                    for (int64_t t : of) M += t;
                    WANT(b->M == M && b->N == (int)of.size() && (int64_t)b->row_of.size() == M);
                    WANT(b->first.size() == of.size() + 1 && b->chunk_first.size() == of.size() + 1 && b->first[0] == 0 && b->chunk_first[0] == 0);
                    for (size_t n = 0; n < of.size(); n++) {
                        for (int64_t t = 0; t < of[n]; t++, row++)
                            WANT(b->row_of[row].file == (int)n && b->row_of[row].token == t && b->row_of[row].id == (numbered ? ids[n] : (int)n));
                        for (int64_t t = 0; t < of[n]; t += b->chunks[chunk].rows, chunk++)
                            WANT(b->chunks[chunk].file == (int)n && b->chunks[chunk].first == row - of[n] + t && b->chunks[chunk].rows > 0 &&
                                 b->chunks[chunk].rows <= ccdc::kChunkRows);
                        WANT(b->first[n + 1] == row && b->chunk_first[n + 1] == chunk);
                    }
                    WANT(row == M && chunk == (int64_t)b->chunks.size());
                    WANT(b->width_ld == d && b->hidden_ld == F);
                    WANT(apart({{b->saved_h, M * F * operand}, {b->saved_p, M * F * 4}, {b->saved_q, M * F * 4}}, b->saved_bytes));
                    // h, in the products' form or (few rows) in elements; the gradients of a and u; x, dy, W_in and W_out as sides of
                    // products; y in ranges of k
                    int64_t ranges = 0;
                    for (int64_t rows = 1; rows <= M; rows++) {
                        const int64_t parts = ccdc::forward_parts(width, F, rows);
                        WANT(parts >= 1);
                        if (parts == 1) continue;
                        const int64_t steps = (F + 63) / 64, each = (steps + parts - 1) / parts * 64, made = (F + each - 1) / each;
                        WANT(made <= parts);
                        ranges = std::max(ranges, made * rows * d * 4);
                    }
                    WANT(apart({{b->at_h, M * F * std::max(operand, elem)}, {b->at_dau, M * 2 * F * operand}, {b->at_x, M * d * operand},
                                {b->at_dy, M * d * operand}, {b->at_in, 2 * hidden * d * operand}, {b->at_out, width * F * operand},
                                {b->at_parts, ranges}}, b->workspace_bytes));
                    if (width <= ccdc::kJoinWidth) WANT((size_t)(chunk * 2 * d * 4) <= b->workspace_bytes);
                    count++;
                }
                delete b;
            }
    std::printf("clean: %ld\n", count);
    return 0;
}

int main(int argc, char **argv)
{
    if (argc > 1 && !std::strcmp(argv[1], "thresholds")) return thresholds(argc - 2, argv + 2);
    if (argc > 2 && !std::strcmp(argv[1], "chunks")) return chunks(std::atoll(argv[2]));
    if (argc > 1 && !std::strcmp(argv[1], "batches")) return batches();
    std::fprintf(stderr, "which check?\n");
    return 2;
}
