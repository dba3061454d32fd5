// Host test driver of nms_decoding_logic.h (g++, sanitizers on): prints what tests/test_decoding_host.py compares.
#include <cinttypes>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "../../paper_2502_00535_amd/csrc/nms_decoding_logic.h"

int main(int argc, char **argv)
{
    if (argc < 2) return 2;
    if (!std::strcmp(argv[1], "keys")) {          // bit patterns on stdin -> keys
        uint32_t u;
        while (std::scanf("%" SCNx32, &u) == 1) {
            float f;
            std::memcpy(&f, &u, sizeof f);
            if (nms_cache_key(f) != nms_cache_key_bits(u)) return 3;
            std::printf("%" PRIu32 "\n", nms_cache_key_bits(u));
        }
        return 0;
    }
    if (!std::strcmp(argv[1], "moves")) {         // n_max budget -> moves, scratch bytes of three frames
        int n, b;
        while (std::scanf("%d %d", &n, &b) == 2) std::printf("%d %zu\n", nms_moves_max(n, b), nms_cache_scratch(n, 3, b));
        return 0;
    }
    if (!std::strcmp(argv[1], "route")) {         // n_max frames rows many -> split, vectors, with weights, part, parts, bytes, offsets of the split's scratch
        int n, f, rows, many;
        while (std::scanf("%d %d %d %d", &n, &f, &rows, &many) == 4) {
            const NmsSplitLayout l = nms_split_layout(n, f);
            std::printf("%d %d %d %d %d %zu %zu %zu %zu %zu\n", nms_cache_split(n, f, many), nms_cache_vecs(n, f), nms_cache_add_with_keep(n, f, many, rows), l.part, l.parts, l.keys,
                        l.bins, l.cuts, l.stays, l.bytes);
        }
        return 0;
    }
    if (!std::strcmp(argv[1], "verify")) {        // vocabulary sequences -> segments, one launch, scratch
        int v, s;
        while (std::scanf("%d %d", &v, &s) == 2)
            std::printf("%d %d %zu %zu\n", nms_verify_segments(v), nms_verify_in_one_launch(v, s), nms_verify_sums_bytes(v, s), nms_verify_scratch(v, s));
        return 0;
    }
    if (!std::strcmp(argv[1], "piece")) {         // address row sequence head slot -> bytes to a lane
        unsigned long long at;
        nms_cache_tensor t = {};
        while (std::scanf("%llu %lld %lld %lld %lld", &at, &t.row_bytes, &t.sequence_stride, &t.head_stride, &t.slot_stride) == 5) {
            t.rows = reinterpret_cast<void *>((uintptr_t)at);
            std::printf("%d\n", nms_cache_piece(t));
        }
        return 0;
    }
    if (!std::strcmp(argv[1], "offset")) {        // strides, sequence, head, slot, page_slots (0: no pages), pages, then a table of 2 x 4
        nms_cache_tensor t = {};
        int sequence, head, slot, page_slots, pages;
        while (std::scanf("%lld %lld %lld %d %d %d %d %d", &t.sequence_stride, &t.head_stride, &t.slot_stride, &sequence, &head, &slot, &page_slots,
                          &pages) == 8) {
            int32_t *table = static_cast<int32_t *>(std::malloc(8 * sizeof(int32_t)));
            for (int i = 0; i < 8; ++i)
                if (std::scanf("%" SCNd32, table + i) != 1) return 4;
            const nms_cache_pages p = {page_slots > 0 ? table : nullptr, 4, page_slots, pages, 0};
            std::printf("%lld\n", nms_cache_row_offset(t, p, sequence, head, slot));
            std::free(table);
        }
        return 0;
    }
    return 2;
}
