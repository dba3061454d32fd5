// Host test driver of the lists of moves (g++, sanitizers on): prints what tests/test_decoding_arguments_host.py compares.
#include <cstdio>

#include "../../paper_2502_00535_amd/csrc/nms_decoding_logic.h"

int main()
{
    int count, moves_max, begin, most;
    while (std::scanf("%d %d %d %d", &count, &moves_max, &begin, &most) == 4) std::printf("%d\n", nms_moves_in_stretch(count, moves_max, begin, most));
    return 0;
}
