// Part of decoding_kernels.hip (included there, inside its anonymous namespace): which rows of a cache stay.
#pragma once

// ----------------------------------------------------------------------------- sums and order of a cache

struct CacheArgs {
    float *sums;
    int32_t *positions;
    const int32_t *counts, *lengths;
    uint8_t *keep;
    int32_t *kept, *moves;
    int n_max, heads, budget, first, recent, moves_max;
    bool move_sums;  // the whole path: sums and positions move with their rows
};

struct WeightArgs {
    const void *weights;
    long long row_stride;
    const int32_t *valid;
    int group, tokens, columns;
};

__device__ __forceinline__ int slots_of(const CacheArgs &a, int sequence)
{
    return frame_count(a.counts, sequence, a.n_max);
}

template <typename T>
__device__ __forceinline__ double as_weight(T v)
{
    const float f = to_float(v);
    return (__float_as_uint(f) & 0x7f800000u) != 0x7f800000u ? (double)f : 0.0;
}

// sums[i] += the weights of slot i: a lane per slot, the query rows one after the other.
template <typename T>
__global__ void __launch_bounds__(256) cache_add_kernel(CacheArgs a, WeightArgs w)
{
    const int frame = blockIdx.y, sequence = frame / a.heads;
    const int i = blockIdx.x * 256 + threadIdx.x;
    const int n = min(slots_of(a, sequence), w.columns);
    if (i >= n) return;
    int tokens = w.valid != nullptr ? w.valid[sequence] : w.tokens;
    tokens = tokens < 0 ? 0 : min(tokens, w.tokens);
    const T *row = static_cast<const T *>(w.weights) + (long long)frame * w.group * w.tokens * w.row_stride + i;
    double sum = (double)a.sums[(long long)frame * a.n_max + i];
    for (int g = 0; g < w.group; ++g)
        for (int t = 0; t < tokens; ++t) sum += as_weight(row[((long long)g * w.tokens + t) * w.row_stride]);
    a.sums[(long long)frame * a.n_max + i] = (float)sum;
}

constexpr int kKeepThreads = 1024;
constexpr int kKeepWaves = kKeepThreads / 64;

// Sum of one number per wavefront over the workgroup, and of the wavefronts before one's own.
__device__ __forceinline__ int2 across_waves(int v, int *room, int wave, int lane)
{
    __syncthreads();
    if (lane == 0) room[wave] = v;
    __syncthreads();
    int2 r = make_int2(0, 0);
    for (int i = 0; i < kKeepWaves; ++i) {
        r.x += room[i];
        r.y += i < wave ? room[i] : 0;
    }
    return r;
}

// One workgroup per frame.  The key that parts the rows that stay from those that go is found bit by bit from the top: the largest T with at
// least k keys >= T.  Keys above T stay, and of those equal to it the lowest slots.  Each wavefront has a stretch of neighbouring slots, so that
// ranks among slots are counts of lanes before one's own.
__global__ void __launch_bounds__(kKeepThreads) cache_keep_kernel(CacheArgs a)
{
    __shared__ int room[kKeepWaves];
    const int frame = blockIdx.x, sequence = frame / a.heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = slots_of(a, sequence), k = min(n, a.budget);
    const long long base = (long long)frame * a.n_max;
    const int length = a.lengths != nullptr ? a.lengths[sequence] : n;
    const int stretch = (n + kKeepThreads - 1) / kKeepThreads * 64;
    const int begin = min(wave * stretch, n), end = min(begin + stretch, n);
    auto key = [&](int i) {
        const int position = a.positions != nullptr ? a.positions[base + i] : i;
        const bool protect = position < a.first || (long long)position >= (long long)length - a.recent;
        return protect ? NMS_CACHE_KEY_PROTECTED : nms_cache_key_bits(__float_as_uint(a.sums[base + i]));
    };
    uint32_t threshold = 0;
    int above = 0;  // keys beyond the threshold
    if (k < n && k > 0) {
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t test = threshold | (1u << bit);
            int c = 0;
            for (int i = begin + lane; i < end; i += 64) c += key(i) >= test;
            for (int d = 32; d >= 1; d >>= 1) c += __shfl_xor(c, d);
            if (across_waves(c, room, wave, lane).x >= k) threshold = test;
        }
        int c = 0;
        for (int i = begin + lane; i < end; i += 64) c += key(i) > threshold;
        for (int d = 32; d >= 1; d >>= 1) c += __shfl_xor(c, d);
        above = across_waves(c, room, wave, lane).x;
    }
    const int ties = k == n ? n : k - above;  // of the keys at the threshold, how many stay (k == n: all of them, whatever their keys)
    const bool none = k == 0;
    auto pass = [&](auto &&visit, int ties_before) {
        int seen = ties_before;
        for (int i0 = begin; i0 < end; i0 += 64) {
            const int i = i0 + lane;
            const uint32_t u = i < end ? key(i) : 0u;
            const bool equal = i < end && (k == n || u == threshold);
            const unsigned long long mask = __ballot(equal);
            const int rank = seen + __popcll(mask & ((1ull << lane) - 1));
            seen += __popcll(mask);
            visit(i, i < end && !none && (equal ? rank < ties : k < n && u > threshold));
        }
        return seen;
    };
    int c = 0;
    for (int i = begin + lane; i < end; i += 64) c += k == n || key(i) == threshold;
    for (int d = 32; d >= 1; d >>= 1) c += __shfl_xor(c, d);
    const int ties_before = across_waves(c, room, wave, lane).y;
    int free_slots = 0, moved = 0;
    pass([&](int i, bool stays) {
        free_slots += __popcll(__ballot(i < end && i < k && !stays));
        moved += __popcll(__ballot(i >= k && stays));
        if (a.keep != nullptr && i < end) a.keep[base + i] = stays;
    }, ties_before);
    if (a.keep != nullptr)
        for (int i = n + threadIdx.x; i < a.n_max; i += kKeepThreads) a.keep[base + i] = 0;
    if (a.kept != nullptr && threadIdx.x == 0 && frame % a.heads == 0) a.kept[sequence] = k;
    if (a.moves == nullptr) return;
    int32_t *list = a.moves + (long long)frame * (a.moves_max + 1) * 2;
    const int2 f = across_waves(free_slots, room, wave, lane), m = across_waves(moved, room, wave, lane);
    if (threadIdx.x == 0) list[0] = m.x, list[1] = 0;
    int to = f.y, from = m.y;
    pass([&](int i, bool stays) {
        const bool is_free = i < end && i < k && !stays, moves = i >= k && stays;
        const unsigned long long mf = __ballot(is_free), mm = __ballot(moves), before = (1ull << lane) - 1;
        if (is_free) list[2 + 2 * (to + __popcll(mf & before))] = i;
        if (moves) list[3 + 2 * (from + __popcll(mm & before))] = i;
        to += __popcll(mf);
        from += __popcll(mm);
    }, ties_before);
    if (!a.move_sums) return;
    __syncthreads();
    for (int r = threadIdx.x; r < m.x; r += kKeepThreads) {
        const int t = list[2 + 2 * r], s = list[3 + 2 * r];
        a.sums[base + t] = a.sums[base + s];
        if (a.positions != nullptr) a.positions[base + t] = a.positions[base + s];
    }
    __syncthreads();
    for (int i = k + threadIdx.x; i < n; i += kKeepThreads) a.sums[base + i] = 0.0f;
}
