// The host side of a trained block (csrc/block.cpp, csrc/block.hpp: no GPU code in them) under AddressSanitizer + UBSan, a
// check a command.  Test infrastructure only.
#include <cstdio>
#include <cstdlib>
#include <cstring>

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

int main(int argc, char **argv)
{
    if (argc > 1 && !std::strcmp(argv[1], "thresholds")) return thresholds(argc - 2, argv + 2);
    if (argc > 2 && !std::strcmp(argv[1], "chunks")) return chunks(std::atoll(argv[2]));
    std::fprintf(stderr, "which check?\n");
    return 2;
}
