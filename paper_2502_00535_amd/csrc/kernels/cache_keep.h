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

// ---- the rows that stay: one workgroup per frame, the keys of all its slots in registers

// A lane has kVecs times four neighbouring slots, a wavefront 256 * kVecs neighbouring ones, so that the rank of a slot among others is a
// count over the wavefronts before, the vectors before, the lanes before and the lane's own.
constexpr int kKeepMaxWaves = 16;
constexpr int kKeepBins = kKeepMaxWaves * 64 * 2;  // two to a thread
constexpr int kFew = 64;                           // candidates that are compared one with another; moves that need no list in memory

// Keys of slots that hold a row are at least 1, so that 0 can stand for those that hold none.
__device__ __forceinline__ uint32_t live_key(float sum, bool protect)
{
    return protect ? NMS_CACHE_KEY_PROTECTED : nms_cache_key_bits(__float_as_uint(sum)) + 1u;
}

// Over the 64 lanes of a wavefront, all of them active: the largest number (in every lane), and running counts.
template <typename Op>
__device__ __forceinline__ uint32_t wave_fold(uint32_t x, Op &&op)
{
    x = op(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, true));   // row_shr:1
    x = op(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, true));   // row_shr:2
    x = op(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, true));   // row_shr:4
    x = op(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, true));   // row_shr:8
    x = op(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));  // row_bcast:15 into rows 1, 3
    x = op(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));  // row_bcast:31 into rows 2, 3
    return x;
}
__device__ __forceinline__ uint32_t of_lane(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }
__device__ __forceinline__ uint32_t wave_max(uint32_t x) { return of_lane(wave_fold(x, [](uint32_t p, uint32_t q) { return max(p, q); }), 63); }
__device__ __forceinline__ uint32_t wave_running_count(uint32_t x) { return wave_fold(x, [](uint32_t p, uint32_t q) { return p + q; }); }

struct KeepRoom {
    uint32_t bins[kKeepBins];
    uint32_t wave_a[kKeepMaxWaves], wave_b[kKeepMaxWaves], wave_c[kKeepMaxWaves];
    uint32_t found[3];             // bin, how many lie beyond it, how many in it
    uint32_t few, few_keys[kFew];
    uint16_t from[kFew];
};

// Where the best `need` of the `left` keys between lo and hi end (0 < need <= left): at the least that stays, and how many keys equal to it are
// wanted and there.
struct Cut {
    uint32_t key, wanted, there;
};

// Keys are counted in bins between lo and hi, the bin in which the need-th lies is cut into bins again, until few keys are left (which are compared
// one with another), or one, or all that are left are wanted.  Counting costs an atomic addition in LDS per key and round; sums of attention weights
// spread over dozens of binary orders, so that a round or two do.  Where the lanes of a wavefront crowd into one bin (equal sums: they would queue up
// there) they are added as one.
template <int kVecs>
__device__ __forceinline__ Cut find_cut(KeepRoom &room, const uint32_t (&key)[kVecs * 4], uint32_t lo, uint32_t hi, uint32_t need, uint32_t left,
                                        int wave, int lane)
{
    const int log_bins = 31 - __builtin_clz(blockDim.x * 2);
    for (;;) {
        if (left == need) return {lo, 0u, 0u};    // all that are left: whatever lies at or beyond lo
        if (lo == hi) return {lo, need, left};
        const uint32_t range = hi - lo;
        if (left <= (uint32_t)kFew) {
            if (threadIdx.x == 0) room.few = 0;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kVecs * 4; ++e)
                if (key[e] - lo <= range) room.few_keys[atomicAdd(&room.few, 1u) & (kFew - 1)] = key[e];
            __syncthreads();
            const bool there = lane < (int)left;
            const uint32_t mine = there ? room.few_keys[lane] : 0u;
            uint32_t larger = 0, equal = 0;
            for (int i = 0; i < (int)left; ++i) {
                const uint32_t other = of_lane(mine, i);
                larger += other > mine;
                equal += other == mine;
            }
            const unsigned long long at = __ballot(there && larger < need && need <= larger + equal);
            const int which = __builtin_ctzll(at | (1ull << 63));
            return {of_lane(mine, which), need - of_lane(larger, which), of_lane(equal, which)};
        }
        const int bits = 32 - __builtin_clz(range), shift = bits > log_bins ? bits - log_bins : 0;
        room.bins[threadIdx.x] = 0;
        room.bins[blockDim.x + threadIdx.x] = 0;
        __syncthreads();
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            const uint32_t bin0 = (key[v * 4] - lo) >> shift;
            const unsigned long long in0 = __ballot(key[v * 4] - lo <= range);
            const unsigned long long same0 = in0 != 0 ? __ballot(bin0 == of_lane(bin0, __builtin_ctzll(in0))) & in0 : 0ull;
            if (__popcll(same0) <= 8) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (key[v * 4 + j] - lo <= range) atomicAdd(&room.bins[(key[v * 4 + j] - lo) >> shift], 1u);
            } else {
#pragma unroll 1
                for (int j = 0; j < 4; ++j) {
                    const uint32_t u = (j == 0 ? key[v * 4] : j == 1 ? key[v * 4 + 1] : j == 2 ? key[v * 4 + 2] : key[v * 4 + 3]) - lo, bin = u >> shift;
                    const unsigned long long in = __ballot(u <= range);
                    if (in == 0) continue;
                    const unsigned long long same = __ballot(bin == of_lane(bin, __builtin_ctzll(in))) & in, leader = same & (0ull - same);
                    if (((in & ~same) | leader) >> lane & 1) atomicAdd(&room.bins[bin], (leader >> lane & 1) != 0 ? (uint32_t)__popcll(same) : 1u);
                }
            }
        }
        __syncthreads();
        // thread t has bins 2 t and 2 t + 1; how many keys lie in larger bins
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
        need -= room.found[1];
        left = room.found[2];
        lo += room.found[0] << shift;
        const uint32_t top = lo + ((1u << shift) - 1u);
        hi = top < lo || top > hi ? hi : top;
    }
}

template <int kVecs, typename W>
__global__ void __launch_bounds__(kKeepMaxWaves * 64) cache_keep_kernel(CacheArgs a, WeightArgs w, MoveArgs m)
{
    constexpr int kEach = kVecs * 4;
    constexpr bool kWeights = !std::is_same<W, void>::value;
    __shared__ KeepRoom room;
    extern __shared__ uint16_t targets[];  // free slots in their order, moves_max of them
    const int frame = blockIdx.x, sequence = frame / a.heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int n = slots_of(a, sequence), k = min(n, a.budget);
    const long long base = (long long)frame * a.n_max;
    const long long since = (long long)(a.lengths != nullptr ? a.lengths[sequence] : n) - a.recent;  // places at or beyond it are protected
    const int newest = since < INT32_MIN ? INT32_MIN : (int)since;
    const int base_slot = wave * (256 * kVecs) + lane * 4;
    auto slot_of = [&](int e) { return base_slot + (e >> 2) * 256 + (e & 3); };
    const bool whole = (wave + 1) * (256 * kVecs) <= n;  // of the wavefront: every slot holds a row
    uint32_t key[kEach], largest = 0, smallest = 0, guarded = 0;  // smallest: as its complement; both without the protected rows
    auto take = [&](int v, const Four<float> &s, const Four<int32_t> &p) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool protect = p.v[j] < a.first || p.v[j] >= newest;
            const uint32_t u = live_key(s.v[j], protect);
            const bool there = whole || base_slot + v * 256 + j < n;
            key[v * 4 + j] = there ? u : 0u;
            largest = max(largest, there && !protect ? u : 0u);
            smallest = max(smallest, there && !protect ? ~u : 0u);
            guarded += there && protect;
        }
    };
    auto places = [&](int v) {
        const int i = base_slot + v * 256;
        if (a.positions == nullptr) return Four<int32_t>{{i, i + 1, i + 2, i + 3}};
        return whole ? *reinterpret_cast<const Four<int32_t> *>(a.positions + base + i) : load_four(a.positions + base, i, n);
    };
    auto sums_of = [&](int v) {
        const int i = base_slot + v * 256;
        return whole ? *reinterpret_cast<const Four<float> *>(a.sums + base + i) : load_four(a.sums + base, i, n);
    };
    if constexpr (kWeights) {
        const int columns = min(n, w.columns), tokens = valid_of(w, sequence);
        const W *row = static_cast<const W *>(w.weights) + (long long)frame * w.group * w.tokens * w.row_stride;
        Four<int32_t> p[kVecs];
        Four<float> s[kVecs];
        double total[kEach];
#pragma unroll
        for (int v = 0; v < kVecs; ++v) s[v] = sums_of(v);
#pragma unroll
        for (int v = 0; v < kVecs; ++v) p[v] = places(v);
#pragma unroll
        for (int e = 0; e < kEach; ++e) total[e] = (double)s[e >> 2].v[e & 3];
        const bool all = (wave + 1) * (256 * kVecs) <= columns;
        for (int g = 0; g < w.group; ++g)
            for (int t = 0; t < tokens; ++t) {
                const W *at = row + ((long long)g * w.tokens + t) * w.row_stride;
                Four<W> x[kVecs];
#pragma unroll
                for (int v = 0; v < kVecs; ++v) {
                    const int i = base_slot + v * 256;
                    x[v] = all ? *reinterpret_cast<const Four<W> *>(at + i) : load_four(at, i, columns);
                }
#pragma unroll
                for (int e = 0; e < kEach; ++e) total[e] += as_weight(x[e >> 2].v[e & 3]);
            }
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
#pragma unroll
            for (int j = 0; j < 4; ++j) s[v].v[j] = (float)total[v * 4 + j];
            store_four(a.sums + base, base_slot + v * 256, n, s[v]);
            take(v, s[v], p[v]);
        }
    } else {
        constexpr int kAtOnce = kVecs < 4 ? kVecs : 4;
#pragma unroll
        for (int v0 = 0; v0 < kVecs; v0 += kAtOnce) {
            Four<int32_t> p[kAtOnce];
            Four<float> s[kAtOnce];
#pragma unroll
            for (int v = 0; v < kAtOnce; ++v) s[v] = sums_of(v0 + v);
#pragma unroll
            for (int v = 0; v < kAtOnce; ++v) p[v] = places(v0 + v);
#pragma unroll
            for (int v = 0; v < kAtOnce; ++v) take(v0 + v, s[v], p[v]);
        }
    }
    // which rows stay, a bit to an element
    using Bits = typename std::conditional<(kEach > 32), unsigned long long, uint32_t>::type;
    Bits stay = 0;
    if (k == n) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) stay |= (Bits)(key[e] != 0u) << e;
    } else if (k > 0) {
        largest = wave_max(largest);
        smallest = wave_max(smallest);
        guarded = wave_running_count(guarded);
        if (lane == 63) room.wave_a[wave] = largest, room.wave_b[wave] = smallest, room.wave_c[wave] = guarded;
        __syncthreads();
        guarded = 0;
        for (int i = 0; i < waves; ++i) {
            largest = max(largest, room.wave_a[i]);
            smallest = max(smallest, room.wave_b[i]);
            guarded += room.wave_c[i];
        }
        __syncthreads();
        uint32_t lo = ~smallest, hi = largest, need = (uint32_t)k - guarded, left = (uint32_t)n - guarded;
        if ((uint32_t)k <= guarded) lo = hi = NMS_CACHE_KEY_PROTECTED, need = (uint32_t)k, left = guarded;  // protected rows alone
        Cut cut;
        for (int stage = 0;; ++stage) {
            cut = find_cut<kVecs>(room, key, lo, hi, need, left, wave, lane);
            const bool ties = cut.wanted < cut.there;
#pragma unroll
            for (int e = 0; e < kEach; ++e) stay |= (Bits)(key[e] > cut.key || (key[e] == cut.key && !ties)) << e;
            if (!ties) break;
            // of the rows with that key the lowest slots: once more, with the complements of their slots for keys (no two are the same)
#pragma unroll
            for (int e = 0; e < kEach; ++e) key[e] = key[e] == cut.key ? ~(uint32_t)slot_of(e) : 0u;
            lo = ~(uint32_t)(waves * 256 * kVecs - 1), hi = ~0u, need = cut.wanted, left = cut.there;
        }
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
    if (a.moves == nullptr && !a.move_sums) return;
    // moves: slots below k whose row goes are free, rows that stay beyond take them in order
    Bits is_free = 0, moves = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const bool s = stay >> e & 1, low = slot_of(e) < k;
        is_free |= (Bits)(low && !s) << e;
        moves |= (Bits)(!low && s) << e;
    }
    const uint32_t counts = wave_running_count((uint32_t)__popcll(is_free) << 16 | (uint32_t)__popcll(moves));  // at most 4096 of each in a wavefront
    if (lane == 63) room.wave_b[wave] = counts;
    __syncthreads();
    uint32_t to = 0, from = 0, total = 0;
    for (int i = 0; i < waves; ++i) {
        const uint32_t c = room.wave_b[i];
        to += i < wave ? c >> 16 : 0u;
        from += i < wave ? c & 0xffffu : 0u;
        total += c & 0xffffu;
    }
    // in order of slots: visit(element, its rank) for each of the flagged
    auto ranked = [&](Bits flags, uint32_t rank0, auto &&visit) {
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            const uint32_t own = (uint32_t)(flags >> (v * 4)) & 15u;
            if (__ballot(own != 0) == 0) continue;
            const uint32_t upto = wave_running_count(__popc(own));
            uint32_t rank = rank0 + upto - __popc(own);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (own >> j & 1) visit(v * 4 + j, rank++);
            rank0 += of_lane(upto, 63);
        }
    };
    ranked(is_free, to, [&](int e, uint32_t r) { targets[r] = (uint16_t)slot_of(e); });
    __syncthreads();
    int2 *list = a.moves != nullptr ? reinterpret_cast<int2 *>(a.moves) + (long long)frame * (a.moves_max + 1) : nullptr;
    if (list != nullptr && threadIdx.x == 0) list[0] = make_int2((int)total, 0);
    ranked(moves, from, [&](int e, uint32_t r) {
        const int t = targets[r], i = slot_of(e);
        if (list != nullptr) list[1 + r] = make_int2(t, i);
        if (r < (uint32_t)kFew) room.from[r] = (uint16_t)i;
        if (a.move_sums) {
            a.sums[base + t] = a.sums[base + i];
            if (a.positions != nullptr) a.positions[base + t] = a.positions[base + i];
        }
    });
    if (!a.move_sums) return;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {  // behind the rows that stay: no sums
        const int i = base_slot + v * 256;
        if (i >= k) store_four(a.sums + base, i, n, Four<float>{});
        else if (i + 4 > k) {
#pragma unroll
            for (int j = 1; j < 4; ++j)
                if (i + j >= k && i + j < n) a.sums[base + i + j] = 0.0f;
        }
    }
    if (m.n_tensors > 0) move_rows(m, frame, (int)total, (int)blockDim.x, [&](int r) { return make_int2(targets[r], room.from[r]); });  // few rows: in this launch
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
