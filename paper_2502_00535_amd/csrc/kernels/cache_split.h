// Part of decoding_kernels.hip (included there, inside its anonymous namespace): which rows stay of frames too long for one workgroup.
#pragma once

// ----------------------------------------------------------------------------- long frames, several workgroups each

// Three launches.  The first writes keys and counts them in bins, a workgroup to a part of the slots; the second finds the cut, a workgroup to a
// frame, from the parts' counts and then from the keys of one bin; the third, by parts again, writes keep bytes and moves.  A part lies wholly below
// slot k or wholly at or beyond it, so that its free slots and its moving rows follow from how many of its rows stay.
//
// The bin of the cut holds some 0.3 % of the rows; one that holds more than LDS takes is counted again, finer, from memory.
//
// 8 heads x 100,003 slots, us: keys 7.7, cut 13.4 (a compute unit adds up 25 parts' counts, 100 KB, and looks at 400 KB of keys), keep bytes and moves 7.2.
// Finding the bin and listing its rows by parts, in a launch before the cut, took 18.0 + 8.1 us against 21.1 (parts of 1024 slots, 400 KB of counts).
constexpr int kSplitBins = 2048, kSplitShift = kBinsLog - 11;
constexpr int kSplitThreads = 256;
constexpr int kSplitList = 4096;

struct SplitArgs {
    uint32_t *keys;             // [frames][n_max]
    uint16_t *bins;             // [frames][parts][kSplitBins]
    unsigned long long *cuts;   // [frames]: the least (key, complement of slot) that stays
    uint32_t *stays;            // [frames][parts]
    int parts, part;            // most parts to a frame, slots to a part (1024, 2048 or 4096)
};

// Slots of a part: ceil(k / part) parts cover [0, k), as many as it takes [k, n).
__device__ __forceinline__ int2 split_range(int p, int n, int k, int part)
{
    const int low = (k + part - 1) / part;
    const long long begin = p < low ? (long long)p * part : k + (long long)(p - low) * part;
    const long long end = min(begin + part, (long long)(p < low ? k : n));
    return begin < end ? make_int2((int)begin, (int)end) : make_int2(n, n);
}

__global__ void __launch_bounds__(kSplitThreads) cache_split_keys_kernel(CacheArgs a, SplitArgs x)
{
    __shared__ uint32_t bins[kSplitBins];
    const int frame = blockIdx.y, sequence = frame / a.heads, lane = threadIdx.x & 63;
    const int n = slots_of(a, sequence), k = min(n, a.budget);
    if (k == 0 || k == n) return;
    const int2 range = split_range(blockIdx.x, n, k, x.part);
    const long long base = (long long)frame * a.n_max;
    const long long since = (long long)(a.lengths != nullptr ? a.lengths[sequence] : n) - a.recent;
    const int newest = since < INT32_MIN ? INT32_MIN : (int)since;
    for (int i = threadIdx.x; i < kSplitBins; i += kSplitThreads) bins[i] = 0;
    __syncthreads();
    for (int i0 = range.x; i0 < range.y; i0 += kSplitThreads * 4) {
        const int i = i0 + threadIdx.x * 4;
        const Four<float> s = load_four(a.sums + base, i, range.y);
        Four<int32_t> p = {{i, i + 1, i + 2, i + 3}};
        if (a.positions != nullptr) p = load_four(a.positions + base, i, range.y);
        Four<uint32_t> u;
        uint32_t bin[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u.v[j] = live_key(s.v[j], p.v[j] < a.first || p.v[j] >= newest);
            bin[j] = key_bin(u.v[j], kSplitShift, kSplitBins - 1);
        }
        store_four(x.keys + base, i, range.y, u);
        const unsigned long long in = __ballot(i < range.y);
        if (in == 0) continue;
        const int crowd = __popcll(__ballot(bin[0] == of_lane(bin[0], __builtin_ctzll(in))) & in);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool there = i + j < range.y;
            if (crowd <= 8) {
                if (there) atomicAdd(&bins[bin[j]], 1u);
            } else {  // equal sums would queue up: as one
                const unsigned long long all = __ballot(there);
                if (all == 0) continue;
                const unsigned long long same = __ballot(bin[j] == of_lane(bin[j], __builtin_ctzll(all))) & all, leader = same & (0ull - same);
                if (((all & ~same) | leader) >> lane & 1) atomicAdd(&bins[bin[j]], (leader >> lane & 1) != 0 ? (uint32_t)__popcll(same) : 1u);
            }
        }
    }
    __syncthreads();
    uint32_t *to = reinterpret_cast<uint32_t *>(x.bins + ((long long)frame * x.parts + blockIdx.x) * kSplitBins);
    for (int i = threadIdx.x; i < kSplitBins / 2; i += kSplitThreads) to[i] = bins[2 * i] | bins[2 * i + 1] << 16;  // at most 4096 each
}

constexpr int kCutThreads = 1024;
constexpr int kCutWaves = kCutThreads / 64;
static_assert(kSplitBins == 2 * kCutThreads, "two bins to a thread");

__global__ void __launch_bounds__(kCutThreads) cache_split_cut_kernel(CacheArgs a, SplitArgs x)
{
    __shared__ uint32_t bins[kSplitBins], wave_sums[kCutWaves], found[3], few;
    __shared__ unsigned long long list[kSplitList];
    const int frame = blockIdx.x, sequence = frame / a.heads, lane = threadIdx.x & 63, wave = wave_of_thread();
    const int n = slots_of(a, sequence), k = min(n, a.budget);
    const int parts = (k + x.part - 1) / x.part + (n - k + x.part - 1) / x.part;
    if (k == 0 || k == n) {  // none stays, or all
        if (threadIdx.x == 0) x.cuts[frame] = k == 0 ? ~0ull : 0ull;
        for (int p = threadIdx.x; p < parts; p += kCutThreads) {
            const int2 r = split_range(p, n, k, x.part);
            x.stays[(long long)frame * x.parts + p] = k == 0 ? 0u : (uint32_t)(r.y - r.x);
        }
        return;
    }
    const uint32_t *keys = x.keys + (long long)frame * a.n_max;
    uint32_t b0 = 0, b1 = 0;
    {
        const uint32_t *from = reinterpret_cast<const uint32_t *>(x.bins + (long long)frame * x.parts * kSplitBins) + threadIdx.x;
#pragma unroll 8
        for (int p = 0; p < parts; ++p) {
            const uint32_t c = from[(long long)p * (kSplitBins / 2)];
            b0 += c & 0xffffu;
            b1 += c >> 16;
        }
    }
    // rows as numbers of 64 bits, no two the same: the key, then the complement of the slot
    auto row = [&](uint32_t key, int i) { return (unsigned long long)key << 32 | ~(uint32_t)i; };
    unsigned long long lo = 0, hi = ~0ull;
    uint32_t need = (uint32_t)k, left = (uint32_t)n;
    // thread t has the counts of bins 2 t and 2 t + 1: the one in which the need-th lies
    auto choose = [&]() {
        const uint32_t own = b0 + b1, upto = wave_running_count(own);
        if (lane == 63) wave_sums[wave] = upto;
        __syncthreads();
        uint32_t below = 0;
        for (int i = 0; i < wave; ++i) below += wave_sums[i];
        const uint32_t above = left - (below + upto);
        if (above < need && need <= above + own) {
            const bool upper = need <= above + b1;
            found[0] = 2 * threadIdx.x + (upper ? 1 : 0);
            found[1] = upper ? above : above + b1;
            found[2] = upper ? b1 : b0;
        }
        __syncthreads();
        need -= found[1];
        left = found[2];
        return found[0];
    };
    {
        const uint32_t bin = choose();
        lo = (unsigned long long)bin_begin(bin, kSplitShift, kSplitBins - 1) << 32;
        hi = (unsigned long long)bin_end(bin, kSplitShift, kSplitBins - 1) << 32 | 0xffffffffull;
    }
    const uint32_t first_bin = found[0];
    bool listed = false, recounted = false;  // the rows between lo and hi are in LDS; they were counted again from memory
    uint32_t entries = 0;
    // the rows between lo and hi; in memory their keys are looked at first, in 32 bits, since hardly any passes (one compute unit looks at all of them)
    auto for_rows = [&](auto &&visit) {
        if (listed) {
            for (uint32_t i = threadIdx.x; i < entries; i += kCutThreads)
                if (list[i] - lo <= hi - lo) visit(list[i]);
        } else {
            constexpr int kAtOnce = 8, kStep = kCutThreads * 4;
            const uint32_t least = (uint32_t)(lo >> 32), range = (uint32_t)(hi >> 32) - least;
            auto look = [&](uint32_t key, int i) {
                if (key - least <= range) {
                    const unsigned long long v = row(key, i);
                    if (v - lo <= hi - lo) visit(v);
                }
            };
            int i = threadIdx.x * 4;
            for (; i - (int)threadIdx.x * 4 + kAtOnce * kStep <= n; i += kAtOnce * kStep) {
                Four<uint32_t> u[kAtOnce];
#pragma unroll
                for (int c = 0; c < kAtOnce; ++c) u[c] = *reinterpret_cast<const Four<uint32_t> *>(keys + i + c * kStep);
#pragma unroll
                for (int c = 0; c < kAtOnce; ++c)
#pragma unroll
                    for (int j = 0; j < 4; ++j) look(u[c].v[j], i + c * kStep + j);
            }
            for (; i < n; i += kStep) {
                const Four<uint32_t> u = load_four(keys, i, n);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (i + j < n) look(u.v[j], i + j);
            }
        }
    };
    while (left != need) {
        if (!listed && left <= (uint32_t)kSplitList) {
            if (threadIdx.x == 0) few = 0;
            __syncthreads();
            for_rows([&](unsigned long long v) { list[atomicAdd(&few, 1u) & (kSplitList - 1)] = v; });
            __syncthreads();
            listed = true;
            entries = left;
        }
        const unsigned long long range = hi - lo;  // not 0: the rows differ
        const int bits = 64 - __builtin_clzll(range), shift = bits > 11 ? bits - 11 : 0;
        recounted |= !listed;
        bins[threadIdx.x] = bins[kCutThreads + threadIdx.x] = 0;
        __syncthreads();
        for_rows([&](unsigned long long v) { atomicAdd(&bins[(v - lo) >> shift], 1u); });
        __syncthreads();
        b0 = bins[2 * threadIdx.x], b1 = bins[2 * threadIdx.x + 1];
        const uint32_t bin = choose();
        lo += (unsigned long long)bin << shift;
        const unsigned long long top = lo + ((1ull << shift) - 1);
        hi = top < lo || top > hi ? hi : top;
        if (shift == 0) break;  // one row
    }
    if (threadIdx.x == 0) x.cuts[frame] = lo;
    // how many rows of each part stay: those of larger bins by the part's counts, and those of the cut's bin (all, or by the list)
    uint32_t *stays = x.stays + (long long)frame * x.parts;
    if (!recounted) {
        __syncthreads();
        for (int p = threadIdx.x; p < parts; p += kCutThreads) bins[p] = 0;
        __syncthreads();
        if (listed) {
            const int low = (k + x.part - 1) / x.part;
            for (uint32_t i = threadIdx.x; i < entries; i += kCutThreads) {
                const int slot = (int)~(uint32_t)list[i];
                if (list[i] >= lo) atomicAdd(&bins[slot < k ? slot / x.part : low + (slot - k) / x.part], 1u);
            }
        }
        __syncthreads();
        const uint32_t least = listed ? first_bin + 1 : first_bin;
        for (int p = wave; p < parts; p += kCutWaves) {
            const uint4 *from = reinterpret_cast<const uint4 *>(x.bins + ((long long)frame * x.parts + p) * kSplitBins);
            uint32_t c = 0;
#pragma unroll
            for (int v = 0; v < kSplitBins / 8 / 64; ++v) {
                const uint4 u = from[v * 64 + lane];
                const uint32_t pair[4] = {u.x, u.y, u.z, u.w}, bin = (v * 64 + lane) * 8;
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j) {
                    c += bin + 2 * j >= least ? pair[j] & 0xffffu : 0u;
                    c += bin + 2 * j + 1 >= least ? pair[j] >> 16 : 0u;
                }
            }
            c = of_lane(wave_running_count(c), 63);
            if (lane == 0) stays[p] = c + bins[p];
        }
        return;
    }
    for (int p = wave; p < parts; p += kCutWaves) {
        const int2 r = split_range(p, n, k, x.part);
        uint32_t c = 0;
        for (int i = r.x + lane * 4; i < r.y; i += 256) {
            const Four<uint32_t> u = load_four(keys, i, r.y);
#pragma unroll
            for (int j = 0; j < 4; ++j) c += i + j < r.y && row(u.v[j], i + j) >= lo;
        }
        c = of_lane(wave_running_count(c), 63);
        if (lane == 0) stays[p] = c;
    }
}

__global__ void __launch_bounds__(kSplitThreads) cache_split_keep_kernel(CacheArgs a, SplitArgs x)
{
    constexpr int kWaves = kSplitThreads / 64, kRounds = 4;  // rounds of 1024 slots, 256 to a wavefront
    __shared__ uint32_t room[kWaves], ranks[2];
    const int frame = blockIdx.y, sequence = frame / a.heads, lane = threadIdx.x & 63, wave = wave_of_thread(), part = blockIdx.x;
    const int n = slots_of(a, sequence), k = min(n, a.budget);
    const int low = (k + x.part - 1) / x.part, parts = low + (n - k + x.part - 1) / x.part;
    const long long base = (long long)frame * a.n_max;
    if (a.keep != nullptr)  // slots that hold no row
        for (int i = max(n, part * x.part) + threadIdx.x; i < min(a.n_max, (part + 1) * x.part); i += kSplitThreads) a.keep[base + i] = 0;
    if (part == 0 && threadIdx.x == 0 && a.kept != nullptr && frame % a.heads == 0) a.kept[sequence] = k;
    int2 *list = a.moves != nullptr ? reinterpret_cast<int2 *>(a.moves) + (long long)frame * (a.moves_max + 1) : nullptr;
    if (part >= parts) {
        if (part == 0 && threadIdx.x == 0 && list != nullptr) list[0] = make_int2(0, 0);  // no rows at all
        return;
    }
    // free slots in the parts before, or moving rows in the parts before that lie beyond k; part 0 also names their number
    const uint32_t *stays = x.stays + (long long)frame * x.parts;
    if (wave == 0) {
        uint32_t rank = 0, total = 0;
        for (int p = lane; p < parts; p += 64) {
            const uint32_t s = stays[p];
            if (p < low && p < part && part < low) rank += (uint32_t)min(x.part, k - p * x.part) - s;
            if (p >= low && p < part && part >= low) rank += s;
            total += p >= low ? s : 0u;
        }
        rank = of_lane(wave_running_count(rank), 63);
        total = of_lane(wave_running_count(total), 63);
        if (lane == 0) {
            ranks[0] = rank;
            if (part == 0 && list != nullptr) list[0] = make_int2((int)total, 0);
        }
    }
    const int2 range = split_range(part, n, k, x.part);
    const unsigned long long cut = x.cuts[frame];
    const bool beyond = part >= low;
    const int stretch = x.part / kWaves, begin = range.x + wave * stretch, end = min(begin + stretch, range.y);
    uint32_t flags = 0, count = 0;  // four bits to a round: the rows that move, or the slots that are free
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int i = begin + r * 256 + lane * 4;
        if (begin + r * 256 >= end) break;
        Four<uint32_t> u = {};
        if (k != n && k != 0) u = load_four(x.keys + base, i, end);
        Four<uint8_t> f;
        uint32_t marks = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool there = i + j < end;
            const bool s = there && (k == n || (k != 0 && ((unsigned long long)u.v[j] << 32 | ~(uint32_t)(i + j)) >= cut));
            f.v[j] = s;
            marks |= (uint32_t)(there && s == beyond) << j;
            if (beyond && a.move_sums && there && !s) a.sums[base + i + j] = 0.0f;
        }
        if (a.keep != nullptr) store_four(a.keep + base, i, end, f);
        flags |= marks << (4 * r);
        count += __popc(marks);
    }
    count = wave_running_count(count);
    if (lane == 63) room[wave] = count;
    __syncthreads();
    if (list == nullptr) return;
    uint32_t rank0 = ranks[0];
    for (int i = 0; i < wave; ++i) rank0 += room[i];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const uint32_t own = flags >> (4 * r) & 15u;
        if (__ballot(own != 0) == 0) continue;
        const uint32_t upto = wave_running_count(__popc(own));
        uint32_t rank = rank0 + upto - __popc(own);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (own >> j & 1) {
                const int i = begin + r * 256 + lane * 4 + j;
                if (beyond) list[1 + rank].y = i;
                else list[1 + rank].x = i;
                ++rank;
            }
        rank0 += of_lane(upto, 63);
    }
}
