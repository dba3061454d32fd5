// Host-checkable logic of the decoding step's choices (verification of drafted tokens, eviction from a cache): keys,
// sizes, workspace layout and addresses.  Compiled by hipcc for the library and by a plain host compiler for the tests.
#ifndef NMS_DECODING_LOGIC_H
#define NMS_DECODING_LOGIC_H

#include <stddef.h>
#include <stdint.h>
#include <string.h>

#include "../../include/nms.h"
#include "nms_pair.h"  // NMS_HD

// ---- keys of the cache's order ----------------------------------------------------------------
// A larger key stays longer; slots with equal keys stay in ascending order.  Sums that are not a number get the lowest key,
// and both zeros the same one.  Protected rows lie above +infinity.
#define NMS_CACHE_KEY_PROTECTED 0xffffffffu
NMS_HD uint32_t nms_cache_key_bits(uint32_t u)
{
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;
    if (u == 0x80000000u) u = 0u;
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
NMS_HD uint32_t nms_cache_key(float sum)
{
    uint32_t u;
    memcpy(&u, &sum, sizeof u);
    return nms_cache_key_bits(u);
}

// ---- sizes --------------------------------------------------------------------------------------
NMS_HD int nms_moves_max(int n_max, int budget)
{
    const int behind = n_max > budget ? n_max - budget : 0;
    return budget < behind ? budget : behind;
}
// Moves begin .. begin + most - 1 of a list: how many of them it has.  `count` is what the list says, any number where it comes from elsewhere.
NMS_HD int nms_moves_in_stretch(int count, int moves_max, int begin, int most)
{
    const int all = count < 0 ? 0 : count < moves_max ? count : moves_max;
    return all <= begin ? 0 : all - begin < most ? all - begin : most;
}
static inline size_t nms_decoding_align256(size_t v) { return (v + 255) & ~(size_t)255; }
// ---- eviction: the route ------------------------------------------------------------------------
// A frame is one workgroup with the keys of all its slots in registers, or (split) is shared by several workgroups in three launches: frames that
// registers do not hold, and long ones of small batches where many rows move.  Keep vector alone, us, one workgroup / split: 8 x 16,384 slots 11.7 / 15.9;
// 8 x 32,768 17.1 / 17.3; 32 x 32,768 17.3 / 21.9; 64 x 32,768 17.9 / 24.3.  Whole path with 64 query rows: 8 x 20,000 50.6 / 41.5; 16 x 32,768 59.5 / 53.0;
// 32 x 32,768 86.2 / 84.1; 64 x 32,768 151 / 154; 32 x 16,384 49.2 / 57.5.
#define NMS_CACHE_WAVES 16   // most wavefronts to a workgroup
#define NMS_CACHE_FEW 64     // moves that need no list in memory: their rows move in the same launch
static inline bool nms_cache_split(int n_max, int frames, bool many_moves) { return n_max > 32768 || (n_max > 16384 && frames <= 32 && many_moves); }
// Vectors of four slots to a lane: one while sixteen wavefronts reach and the batch's wavefronts are on the chip at once, two or more otherwise.  A step
// of one token, us, one vector / two (bf16 weights): 8 heads x 2001 slots 9.1 / 10.7; 8 x 3501 10.3 / 10.6; 512 x 2001 11.6 / 12.5; 1024 x 1501
// (6144 wavefronts) 13.2 / 13.7; 512 x 3501 (7168) 20.0 / 14.5; 1024 x 2501 28.1 / 18.2; 2048 x 1501 27.3 / 20.0.
static inline int nms_cache_vecs(int n_max, int frames)
{
    if (n_max <= 1024 || (n_max <= 3584 && (long long)frames * ((n_max + 255) / 256) <= 6144)) return 1;
    int vecs = 2;
    while (n_max > NMS_CACHE_WAVES * 256 * vecs) vecs *= 2;
    return vecs;
}
// The weights are added by the launch that finds the rows that stay where there are few query rows, by one of its own otherwise.  Whole call, us, with it /
// on their own (bf16): 4 query rows, 8 x 4001 11.5 / 12.6, 512 x 2001 12.2 / 20.3; 16, 8 x 4001 16.9 / 13.2, 256 x 4001 23.4 / 23.9, 1024 x 1001 18.5 / 23.5;
// 32, 8 x 4001 24.1 / 14.1, 256 x 4001 36.8 / 30.6, 1024 x 1001 27.8 / 29.7.
// Between 8193 and 16,384 slots with 4 / 8 rows: f32, 8 x 12,000 16.2 / 13.2 and 20.4 / 13.4, 256 x 12,000 27.6 / 36.1 and 37.8 / 37.4; bf16, 8 x 12,000
// 15.0 / 13.2 and 18.8 / 13.3, 256 x 12,000 21.4 / 38.7 and 28.2 / 39.5.  So the rule loses up to a third of a call where few long frames leave
// compute units idle, and gains up to nine twentieths where they do not; f32 there spills 11 vector registers (the other instantiations none).
static inline bool nms_cache_add_with_keep(int n_max, int frames, bool many_moves, long long rows)
{
    return !nms_cache_split(n_max, frames, many_moves) && nms_cache_vecs(n_max, frames) <= 4 && (rows <= 8 || (rows <= 16 && frames >= 1024));
}

// Scratch: the list of moves (of the whole path), and what the three launches hand on.
static inline size_t nms_cache_list_bytes(int n_max, int frames, int budget)
{
    return nms_decoding_align256((size_t)frames * ((size_t)nms_moves_max(n_max, budget) + 1) * 2 * sizeof(int32_t));
}
struct NmsSplitLayout {
    int part, parts;                       // slots to a part, most parts to a frame
    size_t keys, bins, cuts, stays, bytes; // offsets, and all of it
};
static inline NmsSplitLayout nms_split_layout(int n_max, int frames)
{
    NmsSplitLayout l;
    // The largest part, or a smaller one where that leaves compute units idle and the cut's workgroup does not have the counts of more than 64 parts to add
    // up.  Keep vector alone, us, 1024 / 2048 / 4096 slots: 1 x 100,003 27.9 / 24.2 / -; 8 x 100,003 33.2 / - / 27.3; 8 x 20,000 18.2 / 21.0 / -.
    l.part = 4096;
    while (l.part > 1024 && (long long)frames * (n_max / l.part) < 128 && n_max / (l.part / 2) <= 64) l.part /= 2;
    l.parts = (n_max + l.part - 1) / l.part + 1;
    l.keys = 0;
    l.bins = l.keys + nms_decoding_align256((size_t)frames * n_max * sizeof(uint32_t));
    l.cuts = l.bins + nms_decoding_align256((size_t)frames * l.parts * 2048 * sizeof(uint16_t));
    l.stays = l.cuts + nms_decoding_align256((size_t)frames * sizeof(uint64_t));
    l.bytes = l.stays + nms_decoding_align256((size_t)frames * l.parts * sizeof(uint32_t));
    return l;
}
static inline size_t nms_cache_scratch(int n_max, int frames, int budget)
{
    return nms_cache_list_bytes(n_max, frames, budget) + (nms_cache_split(n_max, frames, true) ? nms_split_layout(n_max, frames).bytes : 0);
}

// ---- verification: the cut of a row, and the route -------------------------------------------
#define NMS_VERIFY_SEGMENT 2048
NMS_HD int nms_verify_segments(int vocabulary) { return (vocabulary + NMS_VERIFY_SEGMENT - 1) / NMS_VERIFY_SEGMENT; }
// One launch with a workgroup per sequence where the row is short for sixteen wavefronts or the sequences fill the compute units, else the
// segments' sums over the whole chip and a second launch.  Whole call, us, one launch / two (target and draft in f32; bf16): 1 x 8000 6.9 / 8.7, 6.6 / 8.6;
// 1 x 40,000 9.5 / 9.9, 8.8 / 9.2; 1 x 50,000 11.3 / 9.5, 11.0 / 9.1; 64 x 50,000 12.0 / 11.5, 11.5 / 10.2; 128 x 50,000 14.1 / 15.9, 11.9 / 12.3;
// 128 x 100,000 20.0 / 22.1, 17.1 / 17.4; 256 x 131,000 40.3 / 43.3, 25.1 / 28.0.
static inline bool nms_verify_in_one_launch(int vocabulary, int sequences)
{
    return nms_verify_segments(vocabulary) <= 20 || sequences >= 128;
}
// Scratch of the route of two launches: the segments' sums, then what was accepted.
static inline size_t nms_verify_sums_bytes(int vocabulary, int sequences)
{
    return nms_decoding_align256((size_t)sequences * (size_t)nms_verify_segments(vocabulary) * sizeof(double));
}
static inline size_t nms_verify_scratch(int vocabulary, int sequences)
{
    if (nms_verify_in_one_launch(vocabulary, sequences)) return 0;
    return nms_verify_sums_bytes(vocabulary, sequences) + nms_decoding_align256((size_t)sequences * 2 * sizeof(int32_t));
}

// ---- buffers ------------------------------------------------------------------------------------
struct NmsBuffer {
    const void *at;   // nullptr: not given
    size_t bytes;
};
static inline bool nms_overlap(const NmsBuffer &a, const NmsBuffer &b)
{
    const uintptr_t i = (uintptr_t)a.at, j = (uintptr_t)b.at;
    return i != 0 && j != 0 && (i < j ? j - i < a.bytes : i - j < b.bytes) && a.bytes > 0 && b.bytes > 0;
}

// ---- addresses ----------------------------------------------------------------------------------
// Byte offset of row (sequence, head, slot), or -1 when its page is none of the tensor's.
NMS_HD long long nms_cache_row_offset(const nms_cache_tensor &t, const nms_cache_pages &pages, int sequence, int head, int slot)
{
    long long block = sequence;
    if (pages.table != nullptr) {
        block = pages.table[(long long)sequence * pages.table_stride + slot / pages.page_slots];
        slot %= pages.page_slots;
        if (block < 0 || block >= pages.pages) return -1;
    }
    return block * t.sequence_stride + head * t.head_stride + slot * t.slot_stride;
}

// Bytes that one lane moves at once: the widest power of two up to 16 that divides every address of the tensor's rows.
static inline int nms_cache_piece(const nms_cache_tensor &t)
{
    const unsigned long long all = (unsigned long long)(uintptr_t)t.rows | (unsigned long long)t.row_bytes | (unsigned long long)t.sequence_stride |
                                   (unsigned long long)t.head_stride | (unsigned long long)t.slot_stride | 16ull;
    return (int)(all & (~all + 1));
}

#endif
