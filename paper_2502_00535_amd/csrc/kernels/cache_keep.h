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

__device__ __forceinline__ int valid_of(const WeightArgs &w, int sequence)
{
    if (w.valid == nullptr) return w.tokens;
    const int v = w.valid[sequence];
    return v < 0 ? 0 : min(v, w.tokens);
}

template <typename T>
__device__ __forceinline__ double as_weight(T v)
{
    const float f = to_float(v);
    return (double)(__builtin_amdgcn_classf(f, 0x1f8) ? f : 0.0f);  // a finite number of either sign
}

// Four neighbouring slots of a lane; rows may begin at any element.
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Four { T v[4]; };

template <typename T>
__device__ __forceinline__ Four<T> load_four(const T *row, int i, int end)
{
    if (i + 4 <= end) return *reinterpret_cast<const Four<T> *>(row + i);
    Four<T> r = {};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i + j < end) r.v[j] = row[i + j];
    return r;
}
template <typename T>
__device__ __forceinline__ void store_four(T *row, int i, int end, const Four<T> &r)
{
    if (i + 4 <= end) {
        *reinterpret_cast<Four<T> *>(row + i) = r;
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i + j < end) row[i + j] = r.v[j];
}

// sums[i] += the weights of slot i, by a launch of its own where there are many query rows: a wavefront has 256 neighbouring slots, the four
// wavefronts of a workgroup share out the rows, and their sums in 64 bits meet in LDS in the same order always.  Bound by the weights'
// bytes: eight rows are in flight to a lane.
constexpr int kAddWaves = 4;
template <typename T>
__global__ void __launch_bounds__(kAddWaves * 64) cache_add_kernel(CacheArgs a, WeightArgs w)
{
    __shared__ double room[kAddWaves - 1][4][64];
    const int frame = blockIdx.y, sequence = frame / a.heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = min(slots_of(a, sequence), w.columns), i = blockIdx.x * 256 + lane * 4;
    if ((int)blockIdx.x * 256 >= n) return;
    const int tokens = valid_of(w, sequence), rows = w.group * tokens;
    const T *first = static_cast<const T *>(w.weights) + (long long)frame * w.group * w.tokens * w.row_stride;
    double sum[4] = {0.0, 0.0, 0.0, 0.0};
    constexpr int kRows = 8;
    for (int r0 = wave; r0 < rows; r0 += kAddWaves * kRows) {
        Four<T> x[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int r = min(r0 + u * kAddWaves, rows - 1), g = r / tokens;
            x[u] = load_four(first + ((long long)g * w.tokens + (r - g * tokens)) * w.row_stride, i, n);
        }
#pragma unroll
        for (int u = 0; u < kRows; ++u)
            if (r0 + u * kAddWaves < rows) {
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[j] += as_weight(x[u].v[j]);
            }
    }
    if (wave > 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) room[wave - 1][j][lane] = sum[j];
    }
    __syncthreads();
    if (wave > 0 || i >= n) return;
    float *sums = a.sums + (long long)frame * a.n_max;
    Four<float> s = load_four(sums, i, n);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        for (int v = 0; v < kAddWaves - 1; ++v) sum[j] += room[v][j][lane];
        s.v[j] = (float)((double)s.v[j] + sum[j]);
    }
    store_four(sums, i, n, s);
}

// ---- the rows that stay: one workgroup per frame, all of its slots in registers

// A lane has kVecs times four neighbouring slots, a wavefront 256 * kVecs neighbouring ones, so that the rank of a slot among others is a
// count over the wavefronts before, the vectors before, the lanes before and the lane's own.
constexpr int kKeepMaxWaves = 16;
constexpr int kKeepBinsPerThread = 2;
constexpr int kKeepBins = kKeepMaxWaves * 64 * kKeepBinsPerThread;
constexpr int kFewCandidates = 64;

// Keys of slots that hold a row are at least 1, so that 0 can stand for those that hold none.
__device__ __forceinline__ uint32_t live_key(float sum, bool protect)
{
    return protect ? NMS_CACHE_KEY_PROTECTED : nms_cache_key_bits(__float_as_uint(sum)) + 1u;
}

__device__ __forceinline__ uint32_t wave_max(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
__device__ __forceinline__ uint32_t wave_running_count(uint32_t x)  // inclusive, over the lanes
{
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, true);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, true);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, true);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, true);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);
    return x;
}

struct KeepRoom {
    uint32_t bins[kKeepBins];
    uint32_t wave_a[kKeepMaxWaves], wave_b[kKeepMaxWaves], wave_c[kKeepMaxWaves];
    uint32_t found[3];                        // bin, how many lie beyond it, how many in it
    uint32_t few, few_keys[kFewCandidates], few_slots[kFewCandidates];
};

// Where the order is cut: a row stays if its key is larger, or the same and its slot not beyond the last one.
struct Cut {
    uint32_t key;
    int last;
};

// The cut behind the best k of n rows, 0 < k < n.  Keys are counted in bins between the smallest and the largest, the bin in which the k-th
// lies is cut into bins again, until it has few rows (they are compared one with another) or a single key; then the same by slots.  Counting
// costs an atomic addition in LDS per row and round; sums of attention weights spread over dozens of binary orders, so that one or two rounds do.  Lanes of a
// wavefront that fall into the first one's bin are added as one, or rows with equal sums would queue up there.
template <int kVecs, typename Key>
__device__ Cut find_cut(KeepRoom &room, int k, Key &&key, int base_slot, int wave, int lane)
{
    const int waves = blockDim.x >> 6, bins = blockDim.x * kKeepBinsPerThread;
    uint32_t largest = 0, smallest = 0, rows = 0, guarded = 0;  // smallest: of the complement
#pragma unroll
    for (int e = 0; e < kVecs * 4; ++e) {
        const uint32_t u = key(e);
        const bool row = u != 0u, protect = u == NMS_CACHE_KEY_PROTECTED;
        guarded += __popcll(__ballot(protect));
        rows += __popcll(__ballot(row && !protect));
        largest = max(largest, protect ? 0u : u);
        smallest = max(smallest, row && !protect ? ~u : 0u);
    }
    largest = wave_max(largest);
    smallest = wave_max(smallest);
    if (lane == 0) room.wave_a[wave] = largest, room.wave_b[wave] = smallest, room.wave_c[wave] = rows, room.bins[wave] = guarded;
    __syncthreads();
    rows = guarded = 0;
    for (int i = 0; i < waves; ++i) {
        largest = max(largest, room.wave_a[i]);
        smallest = max(smallest, room.wave_b[i]);
        rows += room.wave_c[i];
        guarded += room.bins[i];
    }
    __syncthreads();
    uint32_t lo = ~smallest, hi = largest, need = (uint32_t)k - guarded, left = rows;
    bool by_slot = false;       // the second stage: among rows of one key (lo == hi == cut.key), by the complement of their slots
    Cut cut = {0u, 0x7fffffff};
    if ((uint32_t)k <= guarded) {  // more protected rows than may stay
        if ((uint32_t)k == guarded) return {NMS_CACHE_KEY_PROTECTED - 1u, -1};
        lo = hi = NMS_CACHE_KEY_PROTECTED, need = (uint32_t)k, left = guarded;
    }
    for (;;) {
        if (left == need) {  // all of them: the cut lies below
            if (by_slot) return {cut.key, (int)~lo};
            return {lo, 0x7fffffff};
        }
        if (!by_slot && lo == hi) {
            by_slot = true;
            cut.key = lo;
            lo = ~(uint32_t)(waves * 256 * kVecs - 1), hi = ~0u;  // complements of the frame's slots
        }
        auto value = [&](int e) { return by_slot ? ~(uint32_t)(base_slot + (e >> 2) * 256 + (e & 3)) : key(e); };
        auto among = [&](int e, uint32_t v) { return v >= lo && v <= hi && (!by_slot || key(e) == cut.key); };
        if (left <= kFewCandidates) {
            if (threadIdx.x == 0) room.few = 0;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kVecs * 4; ++e) {
                const uint32_t v = value(e);
                if (among(e, v)) {
                    const uint32_t at = atomicAdd(&room.few, 1u);
                    if (at < (uint32_t)kFewCandidates) {
                        room.few_keys[at] = key(e);
                        room.few_slots[at] = (uint32_t)(base_slot + (e >> 2) * 256 + (e & 3));
                    }
                }
            }
            __syncthreads();
            const uint32_t mine = lane < (int)left ? room.few_keys[lane] : 0u, slot = lane < (int)left ? room.few_slots[lane] : ~0u;
            uint32_t rank = 0;
            for (int i = 0; i < (int)left; ++i) {
                const uint32_t other = (uint32_t)__builtin_amdgcn_readlane((int)mine, i), at = (uint32_t)__builtin_amdgcn_readlane((int)slot, i);
                rank += other > mine || (other == mine && at < slot);
            }
            const int which = __builtin_ctzll(__ballot(lane < (int)left && rank == need - 1) | (1ull << 63));
            return {(uint32_t)__builtin_amdgcn_readlane((int)mine, which), __builtin_amdgcn_readlane((int)slot, which)};
        }
        const uint32_t range = hi - lo;
        int shift = 0;
        while ((range >> shift) >= (uint32_t)bins) ++shift;
#pragma unroll
        for (int i = 0; i < kKeepBinsPerThread; ++i) room.bins[i * blockDim.x + threadIdx.x] = 0;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kVecs * 4; ++e) {
            const uint32_t v = value(e), bin = (v - lo) >> shift;
            const bool in = among(e, v);
            const unsigned long long who = __ballot(in);
            if (who == 0) continue;
            const int leader = __builtin_ctzll(who);
            const bool same = in && bin == (uint32_t)__builtin_amdgcn_readlane((int)bin, leader);
            const int many = __popcll(__ballot(same));
            if (lane == leader) atomicAdd(&room.bins[bin], (uint32_t)many);
            else if (in && !same) atomicAdd(&room.bins[bin], 1u);
        }
        __syncthreads();
        // thread t has bins 2 t and 2 t + 1; how many rows lie in larger bins
        const uint32_t b0 = room.bins[2 * threadIdx.x], b1 = room.bins[2 * threadIdx.x + 1], own = b0 + b1;
        const uint32_t upto = wave_running_count(own);
        if (lane == 63) room.wave_a[wave] = upto;
        __syncthreads();
        uint32_t below = 0;
        for (int i = 0; i < wave; ++i) below += room.wave_a[i];
        const uint32_t above = left - (below + upto);  // in the bins of threads after this one
        if (above < need && need <= above + own) {
            const bool upper = need <= above + b1;
            room.found[0] = 2 * threadIdx.x + (upper ? 1 : 0);
            room.found[1] = upper ? above : above + b1;
            room.found[2] = upper ? b1 : b0;
        }
        __syncthreads();
        const uint32_t bin = room.found[0];
        need -= room.found[1];
        left = room.found[2];
        lo += bin << shift;
        const uint32_t top = lo + ((1u << shift) - 1u);
        hi = top < lo || top > hi ? hi : top;
    }
}

template <int kVecs, typename W>
__global__ void __launch_bounds__(kKeepMaxWaves * 64) cache_keep_kernel(CacheArgs a, WeightArgs w, MoveArgs m)
{
    __shared__ KeepRoom room;
    extern __shared__ uint16_t targets[];  // free slots in their order, moves_max of them
    const int frame = blockIdx.x, sequence = frame / a.heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int n = slots_of(a, sequence), k = min(n, a.budget);
    const long long base = (long long)frame * a.n_max;
    const int length = a.lengths != nullptr ? a.lengths[sequence] : n;
    const int base_slot = wave * (256 * kVecs) + lane * 4;  // of element e: base_slot + (e >> 2) * 256 + (e & 3)
    float sum[kVecs * 4];
    unsigned long long guard = 0;
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
        const int i = base_slot + v * 256;
        const Four<float> s = load_four(a.sums + base, i, n);
        Four<int32_t> p = {{i, i + 1, i + 2, i + 3}};
        if (a.positions != nullptr) p = load_four(a.positions + base, i, n);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            sum[v * 4 + j] = s.v[j];
            const bool protect = p.v[j] < a.first || (long long)p.v[j] >= (long long)length - a.recent;
            guard |= (unsigned long long)protect << (v * 4 + j);
        }
    }
    if constexpr (!std::is_same<W, void>::value) {
        const int columns = min(n, w.columns), tokens = valid_of(w, sequence);
        const W *row = static_cast<const W *>(w.weights) + (long long)frame * w.group * w.tokens * w.row_stride;
        double total[kVecs * 4];
#pragma unroll
        for (int e = 0; e < kVecs * 4; ++e) total[e] = (double)sum[e];
        for (int g = 0; g < w.group; ++g)
#pragma unroll 2
            for (int t = 0; t < tokens; ++t) {
                const W *at = row + ((long long)g * w.tokens + t) * w.row_stride;
                Four<W> x[kVecs];
#pragma unroll
                for (int v = 0; v < kVecs; ++v) x[v] = load_four(at, base_slot + v * 256, columns);
#pragma unroll
                for (int e = 0; e < kVecs * 4; ++e) total[e] += as_weight(x[e >> 2].v[e & 3]);
            }
#pragma unroll
        for (int e = 0; e < kVecs * 4; ++e) sum[e] = (float)total[e];
    }
    auto slot_of = [&](int e) { return base_slot + (e >> 2) * 256 + (e & 3); };
    auto key = [&](int e) { return slot_of(e) < n ? live_key(sum[e], guard >> e & 1) : 0u; };
    Cut cut = {0u, -1};                                          // all rows stay
    if (k == 0) cut.key = ~0u;                                   // none does
    else if (k < n) cut = find_cut<kVecs>(room, k, key, base_slot, wave, lane);
    unsigned long long stay = 0;
#pragma unroll
    for (int e = 0; e < kVecs * 4; ++e) {
        const uint32_t u = key(e);
        stay |= (unsigned long long)(u > cut.key || (u == cut.key && u != 0u && slot_of(e) <= cut.last)) << e;
    }
    if (a.keep != nullptr) {
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            Four<uint8_t> f;
#pragma unroll
            for (int j = 0; j < 4; ++j) f.v[j] = stay >> (v * 4 + j) & 1;
            store_four(a.keep + base, base_slot + v * 256, a.n_max, f);
        }
    }
    if (a.kept != nullptr && threadIdx.x == 0 && frame % a.heads == 0) a.kept[sequence] = k;
    // moves: slots below k whose row goes are free, rows that stay beyond take them in order
    unsigned long long is_free = 0, moves = 0;
    uint32_t frees = 0, moved = 0;
    if (a.moves_max > 0 && (a.moves != nullptr || a.move_sums)) {
#pragma unroll
        for (int e = 0; e < kVecs * 4; ++e) {
            const int i = slot_of(e);
            const bool s = stay >> e & 1, f = i < k && !s, b = i >= k && s;
            is_free |= (unsigned long long)f << e;
            moves |= (unsigned long long)b << e;
            frees += __popcll(__ballot(f));
            moved += __popcll(__ballot(b));
        }
    }
    if (lane == 0) room.wave_b[wave] = frees, room.wave_c[wave] = moved;
    __syncthreads();
    uint32_t to = 0, from = 0, total = 0;
    for (int i = 0; i < waves; ++i) {
        to += i < wave ? room.wave_b[i] : 0;
        from += i < wave ? room.wave_c[i] : 0;
        total += room.wave_c[i];
    }
    const unsigned long long before = (1ull << lane) - 1;
    // ranks in order of slots: visit(e, rank) for each flagged element
    auto ranked = [&](unsigned long long flags, uint32_t rank0, auto &&visit) {
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            uint32_t rank = rank0, all = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const unsigned long long mask = __ballot(flags >> (v * 4 + j) & 1);
                rank += __popcll(mask & before);
                all += __popcll(mask);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (flags >> (v * 4 + j) & 1) visit(v * 4 + j, rank++);
            rank0 += all;
        }
    };
    if (frees > 0) ranked(is_free, to, [&](int e, uint32_t r) { targets[r] = (uint16_t)slot_of(e); });
    __syncthreads();
    int2 *list = a.moves != nullptr ? reinterpret_cast<int2 *>(a.moves) + (long long)frame * (a.moves_max + 1) : nullptr;
    if (list != nullptr && threadIdx.x == 0) list[0] = make_int2((int)total, 0);
    if (moved > 0)
        ranked(moves, from, [&](int e, uint32_t r) {
            const int t = targets[r], i = slot_of(e);
            if (list != nullptr) list[1 + r] = make_int2(t, i);
            if (r < (uint32_t)kFewCandidates) room.few_slots[r] = (uint32_t)i;
            if (a.move_sums) {
                a.sums[base + t] = sum[e];
                if (a.positions != nullptr) a.positions[base + t] = a.positions[base + i];
            }
        });
    // sums as they are held now: added (with weights), moved, and none behind the rows that stay
    if (a.move_sums || !std::is_same<W, void>::value) {
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            const int i = base_slot + v * 256;
            Four<float> s;
#pragma unroll
            for (int j = 0; j < 4; ++j) s.v[j] = a.move_sums && i + j >= k ? 0.0f : sum[v * 4 + j];
            const bool none_free = !a.move_sums || (is_free >> (v * 4) & 15) == 0;
            if (!std::is_same<W, void>::value || (i + 4 > k && i < n)) {
                if (none_free) store_four(a.sums + base, i, n, s);
                else
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (i + j < n && !(is_free >> (v * 4 + j) & 1)) a.sums[base + i + j] = s.v[j];
            }
        }
    }
    if (m.n_tensors > 0) {  // few rows to move: in the same launch
        __syncthreads();
        move_rows(m, frame, (int)total, (int)blockDim.x, [&](int r) { return make_int2(targets[r], (int)room.few_slots[r]); });
    }
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

// Frames of more slots than a workgroup's registers hold.  The key that parts the rows that stay from those that go is found bit by bit from the top: the largest T with at
// least k keys >= T.  Keys above T stay, and of those equal to it the lowest slots.  Each wavefront has a stretch of neighbouring slots, so that
// ranks among slots are counts of lanes before one's own.
__global__ void __launch_bounds__(kKeepThreads) cache_keep_long_kernel(CacheArgs a)
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
