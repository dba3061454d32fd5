// Part of decoding_kernels.hip (included there, inside its anonymous namespace): rows of a cache into their new slots.
#pragma once

// ----------------------------------------------------------------------------- moves

// Rows that stay move into the slots of rows that go, and only those: the fewest bytes that leave the rows together in front, and no row is read that
// another one overwrites.  Bound by the rows' bytes, read and written: 32 heads x 1792 rows of 256 bytes in two tensors (59 MB) 12.9 us, 4.6 TB/s;
// 96 x some 880 of 160 bytes (56 MB) 13.9.  A lane moves up to 16 bytes, whatever divides the tensor's addresses; 32 rows to a workgroup, as many workgroups
// as the sizes allow moves (those beyond a frame's own number end at once).

struct MoveTensor {
    nms_cache_tensor t;
    int piece;     // bytes that a lane moves at once (nms_cache_piece)
    int pieces;    // of a row
};
struct MoveArgs {
    const int32_t *moves;
    float *sums;          // of long frames: they and the positions move with the rows, and the places that they leave are set to 0
    int32_t *positions;
    int n_max, heads, budget, moves_max, n_tensors;
    nms_cache_pages pages;
    MoveTensor tensors[NMS_CACHE_MAX_TENSORS];
};

template <typename P>
__device__ __forceinline__ void move_piece(char *to, const char *from, int j)
{
    reinterpret_cast<P *>(to)[j] = reinterpret_cast<const P *>(from)[j];
}

// Rows r = 0 .. rows - 1 of a frame by `threads` threads; move(r) names (to, from).  A row's source lies at or beyond slot `budget` and its target
// below, so no row is both and all moves are independent.
template <typename Move>
__device__ __forceinline__ void move_rows(const MoveArgs &a, int frame, int rows, int threads, Move &&move)
{
    const int sequence = frame / a.heads, head = frame % a.heads;
    for (int which = 0; which < a.n_tensors; ++which) {
        const MoveTensor &m = a.tensors[which];
        for (int w = threadIdx.x; w < rows * m.pieces; w += threads) {
            const int r = w / m.pieces, j = w - r * m.pieces;
            const int2 pair = move(r);
            if (pair.x < 0 || pair.x >= a.budget || pair.y < a.budget || pair.y >= a.n_max) continue;
            const long long t = nms_cache_row_offset(m.t, a.pages, sequence, head, pair.x);
            const long long s = nms_cache_row_offset(m.t, a.pages, sequence, head, pair.y);
            if (t < 0 || s < 0) continue;
            char *rows_at = static_cast<char *>(m.t.rows);
            if (m.piece == 16) move_piece<uint4>(rows_at + t, rows_at + s, j);
            else if (m.piece == 8) move_piece<uint2>(rows_at + t, rows_at + s, j);
            else if (m.piece == 4) move_piece<uint32_t>(rows_at + t, rows_at + s, j);
            else if (m.piece == 2) move_piece<uint16_t>(rows_at + t, rows_at + s, j);
            else move_piece<uint8_t>(rows_at + t, rows_at + s, j);
        }
    }
}

constexpr int kMoveRows = 32;
__global__ void __launch_bounds__(256) cache_move_kernel(MoveArgs a)
{
    const int frame = blockIdx.y;
    const int2 *list = reinterpret_cast<const int2 *>(a.moves) + (long long)frame * (a.moves_max + 1);
    const int begin = blockIdx.x * kMoveRows, rows = nms_moves_in_stretch(list[0].x, a.moves_max, begin, kMoveRows);
    if (rows == 0) return;
    if (a.sums != nullptr && threadIdx.x < (unsigned)rows) {
        const int2 pair = list[1 + begin + threadIdx.x];
        const long long base = (long long)frame * a.n_max;
        a.sums[base + pair.x] = a.sums[base + pair.y];
        a.sums[base + pair.y] = 0.0f;
        if (a.positions != nullptr) a.positions[base + pair.x] = a.positions[base + pair.y];
    }
    move_rows(a, frame, rows, 256, [&](int r) { return list[1 + begin + r]; });
}
