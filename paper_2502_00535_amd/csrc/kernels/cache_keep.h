// Part of decoding_kernels.hip (included there, inside its anonymous namespace): which rows of a cache stay.
#pragma once

// ----------------------------------------------------------------------------- sums and order of a cache

// Which k of n rows stay is a cut in a total order (protected, sum, slot): no sort is needed, only the key at which the k-th lies.  Sums become keys of
// 32 bits that order as the definition says; the keys are counted in bins, and the bin of the k-th is looked into until the cut is found.  Everything
// that follows (keep bytes, free slots, moving rows) is a compare with the cut and a count of lanes before one's own.
//
// Bound by: for long frames the bytes of sums and positions, then instructions (1500 per wavefront at 8 vectors to a lane); for short ones the chain of loads, barriers
// (five) and stores.  Kernel time, us: 8 heads x 1025 slots with four query rows and the move of one row 8.2, 512 x 2049 11.3; the keep vector of
// 512 x 1999 7.0 (8 MB), 512 x 32,768 44 (151 MB, 3.4 TB/s; a compute unit loads a frame, then works on it); 32 x 16,384 with 1800 moves each 18.7.

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

// Weights that are not finite add nothing.  Looking at each costs more than adding it (8 cycles of 21 to a wavefront), so they are added as they
// are: a sum in 64 bits of finite floats is finite, and where one comes out that is not the rows are gone over again, with a look at each weight.
template <typename T>
__device__ __forceinline__ T finite_or_none(T v)
{
    return __builtin_amdgcn_classf(to_float(v), 0x1f8) ? v : T{};
}
__device__ __forceinline__ bool is_finite(double v) { return (__double2hiint(v) & 0x7ff00000) != 0x7ff00000; }

// Four neighbouring slots of a lane; rows may begin at any element.
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Four { T v[4]; };

// Elements at or beyond `end` come out as 0.  The last vector is loaded from four elements before the end and shifted, so that a wavefront at the row's
// end has no branch to wait in: for loads that follow each other in a loop, as weights and the parts of long frames do.  Whole call, us, shifted /
// element by element: bf16, 8 heads x 4001 slots with 4 query rows 10.1 / 11.9, 512 x 2001 with 32 29.0 / 38.2 (f32 34.8 / 50.7), the prompt of
// 8 x 100,003 with 128 97.8 / 126.
template <typename T>
__device__ __forceinline__ Four<T> load_four(const T *row, int i, int end)
{
    Four<T> r = {};
    if (end < 4) {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (i + j < end) r.v[j] = row[i + j];
        return r;
    }
    const int at = min(i, end - 4), d = i - at;
    r = *reinterpret_cast<const Four<T> *>(row + at);
    if constexpr (sizeof(T) == 2) {
        unsigned long long x;
        __builtin_memcpy(&x, &r, sizeof x);
        x = d < 4 ? x >> (16 * d) : 0ull;
        __builtin_memcpy(&r, &x, sizeof x);
    } else {
        r.v[0] = d == 0 ? r.v[0] : d == 1 ? r.v[1] : d == 2 ? r.v[2] : d == 3 ? r.v[3] : T{};
        r.v[1] = d == 0 ? r.v[1] : d == 1 ? r.v[2] : d == 2 ? r.v[3] : T{};
        r.v[2] = d == 0 ? r.v[2] : d == 1 ? r.v[3] : T{};
        r.v[3] = d == 0 ? r.v[3] : T{};
    }
    return r;
}
// The same, element by element: for loads that a wavefront makes once, all of them before the first is needed.  Keep vector alone, us, shifted / so:
// 512 x 1999 slots 8.7 / 8.6, 512 x 9001 17.8 / 16.3, 256 x 30,001 26.2 / 22.3, 512 x 32,765 52.7 / 44.5.
template <typename T>
__device__ __forceinline__ Four<T> load_four_once(const T *row, int i, int end)
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
// bytes: eight rows are in flight to a lane (8 heads x 100,003 slots x 128 rows of bf16 47 us, 4.5 TB/s).  Before rows were walked without divisions it
// took 54 to 58, and eight slots to a lane, for 16-byte loads, 64.
constexpr int kAddWaves = 4, kAddSlots = 256;
template <typename T>
__global__ void __launch_bounds__(kAddWaves * 64) cache_add_kernel(CacheArgs a, WeightArgs w)
{
    __shared__ double room[kAddWaves - 1][4][64];
    const int frame = blockIdx.y, sequence = frame / a.heads, lane = threadIdx.x & 63, wave = wave_of_thread();
    const int n = min(slots_of(a, sequence), w.columns), i = blockIdx.x * kAddSlots + lane * 4;
    if ((int)blockIdx.x * kAddSlots >= n) return;
    const bool whole = (int)(blockIdx.x + 1) * kAddSlots <= n;
    const int tokens = valid_of(w, sequence), rows = w.group * tokens;
    const T *first = static_cast<const T *>(w.weights) + (long long)frame * w.group * w.tokens * w.row_stride;
    const long long gap = (long long)(w.tokens - tokens) * w.row_stride;  // between the valid rows of two query heads
    double sum[4];
    constexpr int kRows = 8;
    for (bool look : {false, true}) {
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = 0.0;
        const T *at = first;      // of row r; t: its token
        int t = wave;
        for (; t >= tokens && tokens > 0; t -= tokens) at += w.tokens * w.row_stride;
        at += t * w.row_stride;
        for (int r = wave; r < rows;) {
            Four<T> x[kRows];
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                x[u] = {};
                if (r < rows) x[u] = whole ? *reinterpret_cast<const Four<T> *>(at + i) : load_four(at, i, n);
                r += kAddWaves;
                at += kAddWaves * w.row_stride;
                for (t += kAddWaves; t >= tokens && r < rows; t -= tokens) at += gap;
            }
            if (look) {
#pragma unroll
                for (int u = 0; u < kRows; ++u)
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[u].v[j] = finite_or_none(x[u].v[j]);
            }
#pragma unroll
            for (int u = 0; u < kRows; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[j] += (double)to_float(x[u].v[j]);
        }
        if (__ballot(!(is_finite(sum[0]) && is_finite(sum[1]) && is_finite(sum[2]) && is_finite(sum[3]))) == 0) break;
    }
    if (wave > 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) room[wave - 1][j][lane] = sum[j];
    }
    __syncthreads();
    if (wave > 0) return;
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
constexpr int kKeepMaxWaves = NMS_CACHE_WAVES;
constexpr int kKeepBins = kKeepMaxWaves * 64 * 2;  // two to a thread
constexpr int kFew = 64;                           // candidates that are compared one with another

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

// The first bins are chosen for sums of attention weights: 32 binary orders from 2^-24 to 2^8 (with 2048 bins 64 to an order; the bin of the cut then
// holds some 0.3 % of the rows), whatever lies outside in the first and the last but one; the last is for protected rows.  So keys can be counted while
// others are still on their way.
constexpr uint32_t kBinsBase = 0x80000000u + (103u << 23) + 1u;  // key of 2^-24
constexpr int kBinsLog = 28;                                     // logarithm of how many keys the orders hold
__device__ __forceinline__ uint32_t key_bin(uint32_t key, int shift, uint32_t last)
{
    const uint32_t bin = min((key < kBinsBase ? 0u : key - kBinsBase) >> shift, last - 1u);
    return key == NMS_CACHE_KEY_PROTECTED ? last : bin;
}
__device__ __forceinline__ uint32_t bin_begin(uint32_t bin, int shift, uint32_t last)
{
    return bin == 0u ? 1u : bin == last ? NMS_CACHE_KEY_PROTECTED : kBinsBase + (bin << shift);
}
__device__ __forceinline__ uint32_t bin_end(uint32_t bin, int shift, uint32_t last)
{
    return bin == last ? NMS_CACHE_KEY_PROTECTED : bin_begin(bin + 1u, shift, last) - 1u;
}

struct KeepRoom {
    uint32_t bins[kKeepBins];
    uint32_t wave_a[kKeepMaxWaves], wave_b[kKeepMaxWaves], wave_c[kKeepMaxWaves];
    uint32_t found[3];             // bin, how many lie beyond it, how many in it
    uint32_t few, few_keys[kFew];
};

// Four keys of a lane into the bins: bin(key) names one of them, or kNoBin.  An atomic addition in LDS per key; where the lanes of a wavefront crowd
// into one bin (equal sums: they would queue up there) they are added as one.
constexpr uint32_t kNoBin = ~0u;
template <typename Bin>
__device__ __forceinline__ void count_four(KeepRoom &room, const uint32_t *key, Bin &&bin, int lane)
{
    const uint32_t first = bin(key[0]);
    const unsigned long long in0 = __ballot(first != kNoBin);
    const unsigned long long same0 = in0 != 0 ? __ballot(first == of_lane(first, __builtin_ctzll(in0))) : 0ull;
    if (__popcll(same0) <= 8) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t b = bin(key[j]);
            if (b != kNoBin) atomicAdd(&room.bins[b], 1u);
        }
    } else {
#pragma unroll 1
        for (int j = 0; j < 4; ++j) {
            const uint32_t b = bin(j == 0 ? key[0] : j == 1 ? key[1] : j == 2 ? key[2] : key[3]);
            const unsigned long long in = __ballot(b != kNoBin);
            if (in == 0) continue;
            const unsigned long long same = __ballot(b == of_lane(b, __builtin_ctzll(in))), leader = same & (0ull - same);
            if (((in & ~same) | leader) >> lane & 1) atomicAdd(&room.bins[b], (leader >> lane & 1) != 0 ? (uint32_t)__popcll(same) : 1u);
        }
    }
}

// The bin in which the need-th of the counted keys lies, `left` of them in all; afterwards the need-th of the `left` in that bin is looked for.
__device__ __forceinline__ uint32_t choose_bin(KeepRoom &room, uint32_t &need, uint32_t &left, int wave, int lane)
{
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
    return room.found[0];
}

__device__ __forceinline__ void clear_bins(KeepRoom &room)
{
    room.bins[threadIdx.x] = 0;
    room.bins[blockDim.x + threadIdx.x] = 0;
    __syncthreads();
}

// Where the best `need` of the `left` keys between lo and hi end (0 < need <= left): at the least that stays, and how many keys equal to it are
// wanted and there.  The keys are counted in bins, the bin in which the need-th lies is cut into bins again, until few keys are left (which are
// compared one with another), or one, or all that are left are wanted.
struct Cut {
    uint32_t key, wanted, there;
};
template <int kVecs>
__device__ __forceinline__ Cut find_cut(KeepRoom &room, const uint32_t (&key)[kVecs * 4], uint32_t lo, uint32_t hi, uint32_t need, uint32_t left,
                                        int log_bins, int wave, int lane)
{
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
        clear_bins(room);
#pragma unroll
        for (int v = 0; v < kVecs; ++v)
            count_four(room, key + v * 4, [&](uint32_t u) { return u - lo <= range ? (u - lo) >> shift : kNoBin; }, lane);
        lo += choose_bin(room, need, left, wave, lane) << shift;
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
    extern __shared__ float moved_sums[];  // (with weights) moves_max of them, of
    uint16_t *targets = reinterpret_cast<uint16_t *>(moved_sums + (kWeights ? a.moves_max : 0));  // rows that move into these slots, in order,
    uint16_t *sources = targets + a.moves_max;                                                     // from these
    const int frame = blockIdx.x, sequence = frame / a.heads, lane = threadIdx.x & 63, wave = wave_of_thread(), waves = blockDim.x >> 6;
    const int n = slots_of(a, sequence), k = min(n, a.budget);
    const long long base = (long long)frame * a.n_max;
    const long long since = (long long)(a.lengths != nullptr ? a.lengths[sequence] : n) - a.recent;  // places at or beyond it are protected
    const int newest = since < INT32_MIN ? INT32_MIN : (int)since;
    const int base_slot = wave * (256 * kVecs) + lane * 4;
    auto slot_of = [&](int e) { return base_slot + (e >> 2) * 256 + (e & 3); };
    // All rows stay, or none, or all but one (a decoding step of one token: the smallest key goes); else keys are counted in bins as they come in.
    const bool one_goes = n - k == 1 && k > 0, counted = k > 0 && n - k > 1;
    const int log_bins = 31 - __builtin_clz(blockDim.x * 2), shift = kBinsLog - log_bins;
    auto first_bin = [&](uint32_t u) { return u != 0u ? key_bin(u, shift, (1u << log_bins) - 1u) : kNoBin; };
    if (counted) clear_bins(room);
    uint32_t key[kEach];
    auto take = [&](auto whole, int v, const Four<float> &s, const Four<int32_t> &p) {  // whole: every slot of the wavefront holds a row
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool there = decltype(whole)::value || base_slot + v * 256 + j < n;
            const uint32_t u = live_key(s.v[j], p.v[j] < a.first || p.v[j] >= newest);
            key[v * 4 + j] = there ? u : 0u;
        }
        if (counted) count_four(room, key + v * 4, first_bin, lane);
    };
    auto places = [&](auto whole, int v) {
        const int i = base_slot + v * 256;
        if (a.positions == nullptr) return Four<int32_t>{{i, i + 1, i + 2, i + 3}};
        if (decltype(whole)::value) return *reinterpret_cast<const Four<int32_t> *>(a.positions + base + i);
        return kWeights ? load_four(a.positions + base, i, n) : load_four_once(a.positions + base, i, n);
    };
    auto sums_of = [&](auto whole, int v) {
        const int i = base_slot + v * 256;
        if (decltype(whole)::value) return *reinterpret_cast<const Four<float> *>(a.sums + base + i);
        return kWeights ? load_four(a.sums + base, i, n) : load_four_once(a.sums + base, i, n);
    };
    float sum[kWeights ? kEach : 1];  // with weights: the new sums, in memory only once their places are known
    if constexpr (kWeights) {
        constexpr int kRows = kVecs < 4 ? 4 : 2;  // query rows in flight
        const int columns = min(n, w.columns), tokens = valid_of(w, sequence), rows = w.group * tokens;
        const bool all = (wave + 1) * (256 * kVecs) <= columns;
        const long long gap = (long long)(w.tokens - tokens) * w.row_stride;  // between the valid rows of two query heads
        const W *first = static_cast<const W *>(w.weights) + (long long)frame * w.group * w.tokens * w.row_stride;
        Four<int32_t> p[kVecs];
        Four<float> s[kVecs];
        double total[kEach];
#pragma unroll
        for (int v = 0; v < kVecs; ++v) s[v] = sums_of(std::false_type{}, v);
#pragma unroll
        for (int v = 0; v < kVecs; ++v) p[v] = places(std::false_type{}, v);
        for (bool look : {false, true}) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) total[e] = 0.0;
            const W *at = first;
            for (int r = 0, t = 0; r < rows; r += kRows) {
                Four<W> x[kRows][kVecs];
#pragma unroll
                for (int u = 0; u < kRows; ++u) {
                    if (r + u < rows) {
#pragma unroll
                        for (int v = 0; v < kVecs; ++v) {
                            const int i = base_slot + v * 256;
                            x[u][v] = all ? *reinterpret_cast<const Four<W> *>(at + i) : load_four(at, i, columns);
                        }
                        at += w.row_stride;
                        if (++t == tokens) t = 0, at += gap;
                    } else {
#pragma unroll
                        for (int v = 0; v < kVecs; ++v) x[u][v] = {};
                    }
                }
                if (look) {
#pragma unroll
                    for (int u = 0; u < kRows; ++u)
#pragma unroll
                        for (int e = 0; e < kEach; ++e) x[u][e >> 2].v[e & 3] = finite_or_none(x[u][e >> 2].v[e & 3]);
                }
#pragma unroll
                for (int u = 0; u < kRows; ++u)
#pragma unroll
                    for (int e = 0; e < kEach; ++e) total[e] += (double)to_float(x[u][e >> 2].v[e & 3]);
            }
            bool finite = true;
#pragma unroll
            for (int e = 0; e < kEach; ++e) finite &= is_finite(total[e]);
            if (__ballot(!finite) == 0) break;
        }
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[v * 4 + j] = s[v].v[j] = (float)((double)s[v].v[j] + total[v * 4 + j]);
            take(std::false_type{}, v, s[v], p[v]);
        }
    } else {
        constexpr int kAtOnce = kVecs < 4 ? kVecs : 4;
        auto load = [&](auto whole) {
#pragma unroll
            for (int v0 = 0; v0 < kVecs; v0 += kAtOnce) {
                Four<int32_t> p[kAtOnce];
                Four<float> s[kAtOnce];
#pragma unroll
                for (int v = 0; v < kAtOnce; ++v) s[v] = sums_of(whole, v0 + v);
#pragma unroll
                for (int v = 0; v < kAtOnce; ++v) p[v] = places(whole, v0 + v);
#pragma unroll
                for (int v = 0; v < kAtOnce; ++v) take(whole, v0 + v, s[v], p[v]);
            }
        };
        if ((wave + 1) * (256 * kVecs) <= n) load(std::true_type{});
        else load(std::false_type{});
    }
    // which rows stay, a bit to an element
    static_assert(kEach <= 32, "one word of bits");
    uint32_t stay = 0;
    if (k == n) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) stay |= (uint32_t)(key[e] != 0u) << e;
    } else if (k > 0) {
        uint32_t lo = 0, hi = 0, need = (uint32_t)k, left = (uint32_t)n;
        if (one_goes) {
            uint32_t least = ~0u;
#pragma unroll
            for (int e = 0; e < kEach; ++e) least = min(least, key[e] - 1u);  // of 0, where there is no row: the largest number
            least = wave_max(~least);
            if (lane == 63) room.wave_a[wave] = least;
            __syncthreads();
            for (int i = 0; i < waves; ++i) least = max(least, room.wave_a[i]);
            least = ~least + 1u;
            uint32_t equal = 0;
#pragma unroll
            for (int e = 0; e < kEach; ++e) equal += __popcll(__ballot(key[e] == least));
            if (lane == 0) room.wave_b[wave] = equal;
            __syncthreads();
            equal = 0;
            for (int i = 0; i < waves; ++i) equal += room.wave_b[i];
            lo = hi = equal == 1 ? least + 1u : least;  // no other is the same: whatever lies beyond it stays
            need = equal == 1 ? (uint32_t)k : equal - 1u;
            left = equal == 1 ? (uint32_t)k : equal;
            __syncthreads();
        } else {
            const uint32_t bin = choose_bin(room, need, left, wave, lane), last = (1u << log_bins) - 1u;
            lo = bin_begin(bin, shift, last);
            hi = bin_end(bin, shift, last);
        }
        Cut cut;
        for (;;) {
            cut = find_cut<kVecs>(room, key, lo, hi, need, left, log_bins, wave, lane);
            const bool ties = cut.wanted < cut.there;
#pragma unroll
            for (int e = 0; e < kEach; ++e) stay |= (uint32_t)(key[e] > cut.key || (key[e] == cut.key && !ties)) << e;
            if (!ties) break;
            // of the rows with that key the lowest slots: once more, with the complements of their slots for keys (no two are the same)
#pragma unroll
            for (int e = 0; e < kEach; ++e) key[e] = key[e] == cut.key ? ~(uint32_t)slot_of(e) : 0u;
            lo = ~(uint32_t)(waves * 256 * kVecs - 1), hi = ~0u, need = cut.wanted, left = cut.there;
        }
    }
    // moves: slots below k whose row goes are free, rows that stay beyond take them in order
    uint32_t total = 0;
    if (a.moves_max > 0 && (a.moves != nullptr || a.move_sums)) {
        uint32_t is_free = 0, moves = 0;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const bool s = stay >> e & 1, low = slot_of(e) < k;
            is_free |= (uint32_t)(low && !s) << e;
            moves |= (uint32_t)(!low && s) << e;
        }
        const uint32_t counts = wave_running_count((uint32_t)__popc(is_free) << 16 | (uint32_t)__popc(moves));  // at most 2048 of each in a wavefront
        if (lane == 63) room.wave_b[wave] = counts;
        __syncthreads();
        uint32_t to = 0, from = 0;
        for (int i = 0; i < waves; ++i) {
            const uint32_t c = room.wave_b[i];
            to += i < wave ? c >> 16 : 0u;
            from += i < wave ? c & 0xffffu : 0u;
            total += c & 0xffffu;
        }
        // in order of slots: visit(element, its rank) for each of the flagged
        auto ranked = [&](uint32_t flags, uint32_t rank0, auto &&visit) {
#pragma unroll
            for (int v = 0; v < kVecs; ++v) {
                const uint32_t own = flags >> (v * 4) & 15u;
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
        ranked(moves, from, [&](int e, uint32_t r) {
            sources[r] = (uint16_t)slot_of(e);
            if constexpr (kWeights) moved_sums[r] = sum[e];
        });
        __syncthreads();
        // no two of the stores below have an address in common, so that none of them waits for another
        for (uint32_t r = threadIdx.x; r < total; r += blockDim.x) {
            const int t = targets[r], i = sources[r];
            if (a.moves != nullptr) reinterpret_cast<int2 *>(a.moves)[(long long)frame * (a.moves_max + 1) + 1 + r] = make_int2(t, i);
            if (a.move_sums) {
                float s;
                if constexpr (kWeights) s = moved_sums[r];
                else s = a.sums[base + i];
                if (a.positions != nullptr) a.positions[base + t] = a.positions[base + i];
                a.sums[base + t] = s;
                a.sums[base + i] = 0.0f;
            }
        }
    }
    if (a.moves != nullptr && threadIdx.x == 0) reinterpret_cast<int2 *>(a.moves)[(long long)frame * (a.moves_max + 1)] = make_int2((int)total, 0);
    if (a.kept != nullptr && threadIdx.x == 0 && frame % a.heads == 0) a.kept[sequence] = k;
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
        const int i = base_slot + v * 256;
        const uint32_t flags = stay >> (v * 4) & 15u;
        if (a.keep != nullptr) {
            Four<uint8_t> f;
#pragma unroll
            for (int j = 0; j < 4; ++j) f.v[j] = flags >> j & 1;
            store_four(a.keep + base, i, a.n_max, f);
        }
        // sums: new ones with weights, 0 for rows that go from slots at or beyond k; slots of moves are written above
        if (kWeights && !a.move_sums) {
            Four<float> s;
#pragma unroll
            for (int j = 0; j < 4; ++j) s.v[j] = kWeights ? sum[kWeights ? v * 4 + j : 0] : 0.0f;
            store_four(a.sums + base, i, n, s);
        } else if (a.move_sums && (kWeights || i + 4 > k)) {
            if (kWeights && flags == 15u && i + 4 <= k) {
                Four<float> s;
#pragma unroll
                for (int j = 0; j < 4; ++j) s.v[j] = kWeights ? sum[kWeights ? v * 4 + j : 0] : 0.0f;
                store_four(a.sums + base, i, n, s);
            } else if (flags == 0u && i >= k) {
                store_four(a.sums + base, i, n, Four<float>{});
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool s = flags >> j & 1;
                    if (i + j < n && (i + j >= k ? !s : kWeights && s)) a.sums[base + i + j] = i + j >= k ? 0.0f : sum[kWeights ? v * 4 + j : 0];
                }
            }
        }
    }
    if (m.n_tensors > 0) move_rows(m, frame, (int)total, (int)blockDim.x, [&](int r) { return make_int2(targets[r], sources[r]); });  // few rows: in this launch
}
