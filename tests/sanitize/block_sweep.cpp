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

int main(int argc, char **argv)
{
    if (argc > 1 && !std::strcmp(argv[1], "thresholds")) return thresholds(argc - 2, argv + 2);
    std::fprintf(stderr, "which check?\n");
    return 2;
}
