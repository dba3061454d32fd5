// Part of decoding_kernels.hip (included there, inside its anonymous namespace): rows of a cache into their new slots.
#pragma once

// ----------------------------------------------------------------------------- moves

struct MoveTensor {
    nms_cache_tensor t;
    int piece;     // bytes that a lane moves at once (nms_cache_piece)
    int pieces;    // of a row
};
struct MoveArgs {
    const int32_t *moves;
    int n_max, heads, budget, moves_max, n_tensors;
    nms_cache_pages pages;
    MoveTensor tensors[NMS_CACHE_MAX_TENSORS];
};

template <typename P>
__device__ __forceinline__ void move_piece(char *to, const char *from, int j)
{
    reinterpret_cast<P *>(to)[j] = reinterpret_cast<const P *>(from)[j];
}

// A row's source lies at or beyond slot k and its target below, so no row is both and all moves are independent.
constexpr int kMoveRows = 32;
__global__ void __launch_bounds__(256) cache_move_kernel(MoveArgs a)
{
    const int frame = blockIdx.y, sequence = frame / a.heads, head = frame % a.heads;
    const int32_t *list = a.moves + (long long)frame * (a.moves_max + 1) * 2;
    const int total = min(list[0], a.moves_max);
    const int begin = blockIdx.x * kMoveRows, rows = min(total - begin, kMoveRows);
    if (rows <= 0) return;
    for (int which = 0; which < a.n_tensors; ++which) {
        const MoveTensor &m = a.tensors[which];
        for (int w = threadIdx.x; w < rows * m.pieces; w += 256) {
            const int r = w / m.pieces, j = w - r * m.pieces;
            const int to = list[2 + 2 * (begin + r)], from = list[3 + 2 * (begin + r)];
            if (to < 0 || to >= a.budget || from < a.budget || from >= a.n_max) continue;
            const long long t = nms_cache_row_offset(m.t, a.pages, sequence, head, to);
            const long long s = nms_cache_row_offset(m.t, a.pages, sequence, head, from);
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
