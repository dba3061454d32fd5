// The choices of a decoding step (gfx950, wave64): how many drafted tokens stand, and which rows of a cache stay.
//
// As for boxes, candidates have scores, the order is total (higher score, then lower index), and the outcome says which of
// them stand.  The kernels live in kernels/verify.h, cache_move.h, cache_keep.h and cache_split.h (included below inside the
// anonymous namespace); the launch logic and the extern "C" entry points follow.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "nms_decoding_logic.h"
#include "nms_launch.h"

namespace {

struct bf16_bits { uint16_t u; };
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(_Float16 v) { return (float)v; }
__device__ __forceinline__ float to_float(bf16_bits v) { return __uint_as_float((unsigned)v.u << 16); }

__device__ __forceinline__ int frame_count(const int32_t *counts, int s, int n_max)
{
    if (counts == nullptr) return n_max;
    const int c = counts[s];
    return c < 0 ? 0 : (c > n_max ? n_max : c);
}

// The wavefront's number in its workgroup, known to be the same in all lanes: branches and addresses that depend on it are scalar.
__device__ __forceinline__ int wave_of_thread() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

#include "kernels/verify.h"
#include "kernels/cache_move.h"
#include "kernels/cache_keep.h"
#include "kernels/cache_split.h"

// ----------------------------------------------------------------------------- host side

inline bool known_type(int type) { return type == NMS_TYPE_F32 || type == NMS_TYPE_F16 || type == NMS_TYPE_BF16; }

inline int workspace_status(const void *workspace, size_t ws_bytes, size_t need)
{
    if (need == 0) return NMS_OK;
    return workspace == nullptr || (uintptr_t)workspace % 256 != 0 || ws_bytes < need ? NMS_ERR_WORKSPACE : NMS_OK;
}

template <typename T, bool kDraft>
int verify_launch(const VerifyArgs &a, int sequences, void *workspace, hipStream_t stream)
{
    const int segments = nms_verify_segments(a.vocabulary);
    const dim3 each(sequences), block(kVerifyThreads);
    begin_launch();
    if (nms_verify_in_one_launch(a.vocabulary, sequences)) {
        verify_kernel<T, kDraft, false><<<each, block, 0, stream>>>(a, segments, VerifyScratch{nullptr, nullptr});
        return launch_status();
    }
    char *room = static_cast<char *>(workspace);
    const VerifyScratch scratch = {reinterpret_cast<double *>(room), reinterpret_cast<int2 *>(room + nms_verify_sums_bytes(a.vocabulary, sequences))};
    const dim3 grid((segments + kVerifySumWaves - 1) / kVerifySumWaves, sequences);
    verify_sums_kernel<T, kDraft><<<grid, dim3(kVerifySumWaves * 64), 0, stream>>>(a, segments, scratch);
    const int st = launch_status();
    if (st != NMS_OK) return st;
    begin_launch();
    verify_kernel<T, kDraft, true><<<each, block, 0, stream>>>(a, segments, scratch);
    return launch_status();
}

template <typename T>
int verify_launch(const VerifyArgs &a, int sequences, void *workspace, hipStream_t stream)
{
    return a.draft != nullptr ? verify_launch<T, true>(a, sequences, workspace, stream) : verify_launch<T, false>(a, sequences, workspace, stream);
}

int cache_sizes_status(int n_max, int heads, int sequences, int budget)
{
    if (n_max < 0 || heads < 0 || sequences < 0 || budget < 0) return NMS_ERR_INVALID_ARG;
    if (n_max > NMS_MAX_SLOTS || (long long)heads * sequences > NMS_MAX_FRAMES) return NMS_ERR_TOO_LARGE;
    return NMS_OK;
}

int weights_status(const nms_cache_weights *w)
{
    if (w == nullptr) return NMS_OK;
    if (!known_type(w->type) || w->group < 0 || w->tokens < 0 || w->columns < 0 || w->row_stride < w->columns) return NMS_ERR_INVALID_ARG;
    if ((long long)w->group * w->tokens > NMS_MAX_QUERY_ROWS) return NMS_ERR_TOO_LARGE;
    if (w->weights == nullptr && w->group > 0 && w->tokens > 0 && w->columns > 0) return NMS_ERR_INVALID_ARG;
    return NMS_OK;
}

// The numbers of a sequence are read by every workgroup of its heads, and some have written what they have to write by then.
bool overwrites(const CacheArgs &a, const nms_cache_weights *w, int heads, int sequences, bool positions_too)
{
    const size_t slots = (size_t)heads * sequences * a.n_max, each = (size_t)sequences * sizeof(int32_t);
    const size_t moves = (size_t)heads * sequences * ((size_t)a.moves_max + 1) * 2 * sizeof(int32_t);
    const NmsBuffer written[] = {{a.sums, slots * sizeof(float)}, {positions_too ? a.positions : nullptr, slots * sizeof(int32_t)}, {a.keep, slots},
                                 {a.kept, each}, {a.moves, moves}};
    const NmsBuffer read[] = {{a.counts, each}, {a.lengths, each}, {w != nullptr ? w->valid_tokens : nullptr, each}};
    for (const NmsBuffer &out : written)
        for (const NmsBuffer &in : read)
            if (nms_overlap(out, in)) return true;
    return false;
}

int tensors_status(const nms_cache_tensor *tensors, int n_tensors, const nms_cache_pages *pages, int n_max)
{
    if (n_tensors < 0 || (n_tensors > 0 && tensors == nullptr)) return NMS_ERR_INVALID_ARG;
    if (n_tensors > NMS_CACHE_MAX_TENSORS) return NMS_ERR_TOO_LARGE;
    for (int i = 0; i < n_tensors; ++i) {
        const nms_cache_tensor &t = tensors[i];
        if (t.rows == nullptr || t.row_bytes < 1 || t.row_bytes > (1 << 20)) return NMS_ERR_INVALID_ARG;
        if (t.sequence_stride < 0 || t.head_stride < 0 || t.slot_stride < 0) return NMS_ERR_INVALID_ARG;  // an offset below 0 stands for a bad page
    }
    if (pages == nullptr) return NMS_OK;
    if (pages->table == nullptr || pages->page_slots < 1 || pages->pages < 0 || pages->reserved != 0) return NMS_ERR_INVALID_ARG;
    return (long long)pages->table_stride * pages->page_slots < n_max ? NMS_ERR_INVALID_ARG : NMS_OK;
}

WeightArgs weight_args(const nms_cache_weights *w)
{
    if (w == nullptr || w->group == 0 || w->tokens == 0 || w->columns == 0) return {};
    return {w->weights, w->row_stride, w->valid_tokens, w->group, w->tokens, w->columns};
}

int add_launch(const CacheArgs &a, const WeightArgs &w, int type, int frames, hipStream_t stream)
{
    const int columns = w.columns < a.n_max ? w.columns : a.n_max;
    const dim3 grid((columns + kAddSlots - 1) / kAddSlots, frames), block(kAddWaves * 64);
    begin_launch();
    if (type == NMS_TYPE_F32) cache_add_kernel<float><<<grid, block, 0, stream>>>(a, w);
    else if (type == NMS_TYPE_F16) cache_add_kernel<_Float16><<<grid, block, 0, stream>>>(a, w);
    else cache_add_kernel<bf16_bits><<<grid, block, 0, stream>>>(a, w);
    return launch_status();
}

template <int kVecs>
int keep_launch(const CacheArgs &a, const WeightArgs &w, int type, const MoveArgs &m, int frames, hipStream_t stream)
{
    const dim3 grid(frames), block((a.n_max + 256 * kVecs - 1) / (256 * kVecs) * 64);
    const size_t lds = (size_t)a.moves_max * (2 * sizeof(uint16_t) + (w.weights != nullptr ? sizeof(float) : 0));
    begin_launch();
    if constexpr (kVecs <= 4) {
        if (w.weights != nullptr) {
            if (type == NMS_TYPE_F32) cache_keep_kernel<kVecs, float><<<grid, block, lds, stream>>>(a, w, m);
            else if (type == NMS_TYPE_F16) cache_keep_kernel<kVecs, _Float16><<<grid, block, lds, stream>>>(a, w, m);
            else cache_keep_kernel<kVecs, bf16_bits><<<grid, block, lds, stream>>>(a, w, m);
            return launch_status();
        }
    }
    cache_keep_kernel<kVecs, void><<<grid, block, lds, stream>>>(a, w, m);
    return launch_status();
}

MoveArgs move_args(const int32_t *moves, int n_max, int heads, int budget, const nms_cache_tensor *tensors, int n_tensors,
                   const nms_cache_pages *pages)
{
    MoveArgs m = {};
    m.moves = moves, m.n_max = n_max, m.heads = heads, m.budget = budget, m.moves_max = nms_moves_max(n_max, budget), m.n_tensors = n_tensors;
    if (pages != nullptr) m.pages = *pages;
    for (int i = 0; i < n_tensors; ++i) {
        m.tensors[i].t = tensors[i];
        m.tensors[i].piece = nms_cache_piece(tensors[i]);
        m.tensors[i].pieces = (int)(tensors[i].row_bytes / m.tensors[i].piece);
    }
    return m;
}

int move_launch(const MoveArgs &m, int frames, hipStream_t stream)
{
    if (m.moves_max == 0 || (m.n_tensors == 0 && m.sums == nullptr)) return NMS_OK;
    begin_launch();
    cache_move_kernel<<<dim3((m.moves_max + kMoveRows - 1) / kMoveRows, frames), dim3(256), 0, stream>>>(m);
    return launch_status();
}

// The keep vector and the moves of frames that several workgroups share.
int split_launch(const CacheArgs &a, void *scratch, int frames, hipStream_t stream)
{
    const NmsSplitLayout at = nms_split_layout(a.n_max, frames);
    char *room = static_cast<char *>(scratch);
    SplitArgs x = {reinterpret_cast<uint32_t *>(room + at.keys), reinterpret_cast<uint16_t *>(room + at.bins),
                   reinterpret_cast<unsigned long long *>(room + at.cuts), reinterpret_cast<uint32_t *>(room + at.stays), at.parts, at.part};
    const dim3 grid(at.parts, frames), block(kSplitThreads);
    begin_launch();
    cache_split_keys_kernel<<<grid, block, 0, stream>>>(a, x);
    int st = launch_status();
    if (st != NMS_OK) return st;
    begin_launch();
    cache_split_cut_kernel<<<dim3(frames), dim3(kCutThreads), 0, stream>>>(a, x);
    st = launch_status();
    if (st != NMS_OK) return st;
    begin_launch();
    cache_split_keep_kernel<<<grid, block, 0, stream>>>(a, x);
    return launch_status();
}

// The keep vector and the moves; rows of `m` move in the same launch where there are few, by one of their own otherwise.
int keep_and_move(const CacheArgs &a, const nms_cache_weights *weights, const MoveArgs &m, void *scratch, int frames, hipStream_t stream)
{
    WeightArgs w = weight_args(weights);
    const int type = weights != nullptr ? weights->type : 0;
    const bool few = a.moves_max <= NMS_CACHE_FEW, many = !few && (a.moves != nullptr || a.move_sums);
    if (w.weights != nullptr && !nms_cache_add_with_keep(a.n_max, frames, many, w.group * (long long)w.tokens)) {
        const int st = add_launch(a, w, type, frames, stream);
        if (st != NMS_OK) return st;
        w = {};
    }
    if (nms_cache_split(a.n_max, frames, many)) {
        const int st = split_launch(a, scratch, frames, stream);
        if (st != NMS_OK) return st;
        MoveArgs with_sums = m;
        if (a.move_sums) with_sums.sums = a.sums, with_sums.positions = a.positions;
        return move_launch(with_sums, frames, stream);
    }
    CacheArgs b = a;
    if (few && a.move_sums) b.moves = nullptr;  // the list stays in LDS
    const MoveArgs none = {}, &now = few ? m : none;
    int st;
    switch (nms_cache_vecs(a.n_max, frames)) {
    case 1: st = keep_launch<1>(b, w, type, now, frames, stream); break;
    case 2: st = keep_launch<2>(b, w, type, now, frames, stream); break;
    case 4: st = keep_launch<4>(b, w, type, now, frames, stream); break;
    default: st = keep_launch<8>(b, w, type, now, frames, stream); break;
    }
    return st != NMS_OK || few ? st : move_launch(m, frames, stream);
}

}  // namespace

extern "C" {

size_t nms_verify_workspace_bytes(int vocabulary, int sequences)
{
    if (vocabulary < 1 || vocabulary > NMS_MAX_VOCABULARY || sequences < 0 || sequences > NMS_MAX_FRAMES) return 0;
    return nms_verify_scratch(vocabulary, sequences);
}

int nms_verify_batched(const void *target, long long target_stride, const void *draft, long long draft_stride, int type,
                       const int32_t *drafts, const int32_t *counts, int drafts_max, int vocabulary, int sequences,
                       const float *uniforms, int32_t *tokens_out, int32_t *accepted_out, void *workspace, size_t ws_bytes,
                       void *stream)
{
    if (!known_type(type) || drafts_max < 0 || vocabulary < 1 || sequences < 0 || target_stride < vocabulary ||
        (draft != nullptr && drafts_max > 0 && draft_stride < vocabulary))
        return NMS_ERR_INVALID_ARG;
    if (drafts_max > NMS_MAX_DRAFTS || vocabulary > NMS_MAX_VOCABULARY || sequences > NMS_MAX_FRAMES) return NMS_ERR_TOO_LARGE;
    if (sequences == 0) return NMS_OK;
    if (target == nullptr || (drafts == nullptr && drafts_max > 0) || uniforms == nullptr || tokens_out == nullptr || accepted_out == nullptr)
        return NMS_ERR_INVALID_ARG;
    const size_t each = (size_t)sequences * sizeof(int32_t);
    const NmsBuffer out[] = {{tokens_out, each * (drafts_max + 1)}, {accepted_out, each}};  // written while other sequences' inputs are read
    for (const NmsBuffer &in : {NmsBuffer{drafts, each * drafts_max}, NmsBuffer{counts, each}, NmsBuffer{uniforms, each * (drafts_max + 1)}})
        if (nms_overlap(out[0], in) || nms_overlap(out[1], in)) return NMS_ERR_INVALID_ARG;
    if (nms_overlap(out[0], out[1])) return NMS_ERR_INVALID_ARG;
    const int st = workspace_status(workspace, ws_bytes, nms_verify_workspace_bytes(vocabulary, sequences));
    if (st != NMS_OK) return st;
    const VerifyArgs a = {target, draft, target_stride, draft_stride, drafts, counts, uniforms, tokens_out, accepted_out, drafts_max, vocabulary};
    hipStream_t on = static_cast<hipStream_t>(stream);
    if (type == NMS_TYPE_F32) return verify_launch<float>(a, sequences, workspace, on);
    if (type == NMS_TYPE_F16) return verify_launch<_Float16>(a, sequences, workspace, on);
    return verify_launch<bf16_bits>(a, sequences, workspace, on);
}

int nms_cache_moves_max(int n_max, int budget)
{
    if (n_max < 0 || n_max > NMS_MAX_SLOTS || budget < 0) return -1;
    return nms_moves_max(n_max, budget);
}

size_t nms_cache_workspace_bytes(int n_max, int heads, int sequences, int budget)
{
    if (cache_sizes_status(n_max, heads, sequences, budget) != NMS_OK) return 0;
    return nms_cache_scratch(n_max, heads * sequences, budget);
}

int nms_cache_keep_batched(float *sums, const int32_t *positions, const int32_t *counts, const int32_t *lengths, int n_max,
                           int heads, int sequences, const nms_cache_weights *weights, int budget, int first, int recent,
                           uint8_t *keep_out, int32_t *kept_out, int32_t *moves_out, void *workspace, size_t ws_bytes, void *stream)
{
    int st = cache_sizes_status(n_max, heads, sequences, budget);
    if (st != NMS_OK) return st;
    if (first < 0 || recent < 0) return NMS_ERR_INVALID_ARG;
    st = weights_status(weights);
    if (st != NMS_OK) return st;
    if (n_max == 0 || heads == 0 || sequences == 0) return NMS_OK;
    const CacheArgs a = {sums, const_cast<int32_t *>(positions), counts, lengths, keep_out, kept_out, moves_out, n_max, heads, budget, first, recent,
                         nms_moves_max(n_max, budget), false};
    if (sums == nullptr || overwrites(a, weights, heads, sequences, false)) return NMS_ERR_INVALID_ARG;
    st = workspace_status(workspace, ws_bytes, nms_cache_workspace_bytes(n_max, heads, sequences, budget));
    if (st != NMS_OK) return st;
    return keep_and_move(a, weights, MoveArgs{}, workspace, heads * sequences, static_cast<hipStream_t>(stream));
}

int nms_cache_move_batched(const int32_t *moves, int n_max, int heads, int sequences, int budget, const nms_cache_tensor *tensors,
                           int n_tensors, const nms_cache_pages *pages, void *stream)
{
    int st = cache_sizes_status(n_max, heads, sequences, budget);
    if (st != NMS_OK) return st;
    st = tensors_status(tensors, n_tensors, pages, n_max);
    if (st != NMS_OK) return st;
    if (n_max == 0 || heads == 0 || sequences == 0 || n_tensors == 0) return NMS_OK;
    if (moves == nullptr) return NMS_ERR_INVALID_ARG;
    return move_launch(move_args(moves, n_max, heads, budget, tensors, n_tensors, pages), heads * sequences, static_cast<hipStream_t>(stream));
}

int nms_cache_evict_batched(float *sums, int32_t *positions, const int32_t *counts, const int32_t *lengths, int n_max,
                            int heads, int sequences, const nms_cache_weights *weights, int budget, int first, int recent,
                            const nms_cache_tensor *tensors, int n_tensors, const nms_cache_pages *pages,
                            uint8_t *keep_out, int32_t *kept_out, void *workspace, size_t ws_bytes, void *stream)
{
    int st = cache_sizes_status(n_max, heads, sequences, budget);
    if (st != NMS_OK) return st;
    if (first < 0 || recent < 0 || (positions == nullptr && recent > 0)) return NMS_ERR_INVALID_ARG;
    st = weights_status(weights);
    if (st != NMS_OK) return st;
    st = tensors_status(tensors, n_tensors, pages, n_max);
    if (st != NMS_OK) return st;
    if (n_max == 0 || heads == 0 || sequences == 0) return NMS_OK;
    CacheArgs a = {sums, positions, counts, lengths, keep_out, kept_out, nullptr, n_max, heads, budget, first, recent, nms_moves_max(n_max, budget), true};
    if (sums == nullptr || overwrites(a, weights, heads, sequences, true)) return NMS_ERR_INVALID_ARG;
    st = workspace_status(workspace, ws_bytes, nms_cache_workspace_bytes(n_max, heads, sequences, budget));
    if (st != NMS_OK) return st;
    const int frames = heads * sequences;
    // the list of moves first, then what finds it
    int32_t *moves = a.moves = static_cast<int32_t *>(workspace);
    void *scratch = static_cast<char *>(workspace) + nms_cache_list_bytes(n_max, frames, budget);
    return keep_and_move(a, weights, move_args(moves, n_max, heads, budget, tensors, n_tensors, pages), scratch, frames, static_cast<hipStream_t>(stream));
}

}  // extern "C"
