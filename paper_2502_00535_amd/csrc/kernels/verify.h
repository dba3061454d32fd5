// Part of decoding_kernels.hip (included there, inside its anonymous namespace): verification of drafted tokens.
#pragma once

// ----------------------------------------------------------------------------- verification

// A sequence's drafted tokens stand up to the first that the test u q < p refuses; the next token is drawn from what the target's row has beyond the
// draft's, or from the target's row where none was refused: the least entry whose running sum passes u times the total.  So of all probabilities two
// per drafted token and one row (or two) per sequence are read, once: the row's sum needs every entry, the entry itself one segment of it again.
//
// Numbers are compared and added in 64 bits: products of two floats are exact there, and with V entries in 32 bits the sum would be off by
// up to V 2^-24 of itself, past the borders of most entries.  Conversions and additions in 64 bits take 4.5 and 5.2 cycles to a wavefront, 47 per entry
// with both rows: less than the rows' bytes take on the whole chip (256 x 151,111 floats: 11.6 us of issue, 41 us), more than they take where a
// compute unit has a row alone.
//
// Bound by: the rows' bytes for large batches (232 MB in 41 us of kernel time under the profiler, 47.5 to 49.1 us a call: 4.7 to 4.9 TB/s);
// for small ones by the chain of dependent loads (token, its probabilities, row, entry: 1 x 32,000 floats 9.0 us, 64 x 50,001 f16 4.9 + 5.0 us in two
// launches) and, where the vocabulary is no multiple of a segment, by the row's end, which goes element by element through 20 bytes of scratch
// memory to a lane (up_to_end).  Calls, us: 1 x 30,720 floats 7.7, x 32,000 8.9, x 32,768 7.8; 64 x 49,152 / 50,001 / 51,200 f16 8.1 / 8.9 / 8.2;
// 32 x 151,552 / 151,936 bf16 10.6 / 12.0; where the chip is full it does not show (256 x 151,111 / 151,552 floats 47.3 / 48.2).

template <typename T>
__device__ __forceinline__ float as_probability(T v)
{
    const float f = to_float(v);
    return __builtin_amdgcn_classf(f, 0x180) ? f : 0.0f;  // a finite number above 0 (subnormal or normal) stays as it is
}

struct VerifyArgs {
    const void *target, *draft;
    long long target_stride, draft_stride;
    const int32_t *drafts, *counts;
    const float *uniforms;
    int32_t *tokens, *accepted;
    int drafts_max, vocabulary;
};

// How many drafted tokens of the sequence stand, by one wavefront (every lane gets the answer): 64 tests at a time.  Tokens and random
// numbers are loaded beside the count, not after it, also where it then says that there is no sequence: it is a chain of three (token, its two
// probabilities, the row) as it is.
template <typename T, bool kDraft>
__device__ __forceinline__ int count_accepted(const VerifyArgs &a, int s, int lane, int &count)
{
    const T *target = static_cast<const T *>(a.target) + (long long)s * (a.drafts_max + 1) * a.target_stride;
    const T *draft = kDraft ? static_cast<const T *>(a.draft) + (long long)s * a.drafts_max * a.draft_stride : nullptr;
    count = a.counts != nullptr ? a.counts[s] : a.drafts_max;
    if (a.drafts_max == 0) {
        count = min(count, 0);
        return 0;
    }
    for (int i0 = 0; i0 < a.drafts_max; i0 += 64) {
        const int i = i0 + lane;
        int x = -1;
        double u = 0.0;
        if (i < a.drafts_max) {
            x = a.drafts[(long long)s * a.drafts_max + i];
            u = (double)a.uniforms[(long long)s * (a.drafts_max + 1) + i];
        }
        if (i0 == 0) count = min(count, a.drafts_max);
        if (i0 >= count) break;
        bool refused = false;
        if (i < count) {
            double p = 0.0, q = kDraft ? 0.0 : 1.0;
            if (x >= 0 && x < a.vocabulary) {
                p = (double)as_probability(target[i * a.target_stride + x]);
                if (kDraft) q = (double)as_probability(draft[i * a.draft_stride + x]);
            }
            refused = !(u * q < p);
        }
        const unsigned long long mask = __ballot(refused);
        if (mask != 0) return i0 + __builtin_ctzll(mask);
    }
    return max(count, 0);
}

// The weights that the token is drawn from: w_j = max(p_j - q_j, 0), or p_j.
template <typename T, bool kDraft>
struct Weights {
    const T *p, *q;    // q: the draft's row, nullptr where the target's row counts alone
    int without;       // the entry that counts as 0 (a refused token of a draft without probabilities), or -1
    __device__ __forceinline__ double of(T pj, T qj) const
    {
        double w = (double)as_probability(pj);
        if (kDraft && q != nullptr) {
            w -= (double)as_probability(qj);
            w = __builtin_fmax(w, 0.0);
        }
        return w;
    }
    __device__ __forceinline__ double at(int j) const
    {
        const double w = of(p[j], kDraft && q != nullptr ? q[j] : p[j]);
        return j == without ? 0.0 : w;
    }
};

// Running sum over the 64 lanes of a wavefront (all of them active) with DPP: shifts by 1, 2, 4, 8 inside each row of 16 lanes, then lane 15 of
// each row into the next one (rows 1 and 3), then lane 31 into rows 2 and 3; lanes that get nothing add 0.  Exchanges through LDS in its place
// cost some 100 cycles a step, one after the other.
template <int kControl, int kRows>
__device__ __forceinline__ double from_lane(double v)
{
    const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), kControl, kRows, 0xf, kRows == 0xf);
    const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), kControl, kRows, 0xf, kRows == 0xf);
    return __hiloint2double(hi, lo);
}
__device__ __forceinline__ double wave_running_sum(double v)
{
    v += from_lane<0x111, 0xf>(v);
    v += from_lane<0x112, 0xf>(v);
    v += from_lane<0x114, 0xf>(v);
    v += from_lane<0x118, 0xf>(v);
    v += from_lane<0x142, 0xa>(v);
    v += from_lane<0x143, 0xc>(v);
    return v;
}
__device__ __forceinline__ double of_lane(double v, int lane)  // the lane: the same number in every lane
{
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane), __builtin_amdgcn_readlane(__double2loint(v), lane));
}

// The row is cut into segments; a segment is summed by one wavefront, lane by lane and then across lanes, and the segments' sums are
// added up in their order.  The cut depends on nothing but the vocabulary, so a sequence's sums have the same bits in any batch and
// on either route.  2048 entries are 32 to a lane: with 16-byte loads 8 (f32) or 4 (16 bits) of each row are in flight at once.
constexpr int kVerifySegment = NMS_VERIFY_SEGMENT;
constexpr int kVerifyThreads = 1024;
constexpr int kVerifyMaxSegments = (NMS_MAX_VOCABULARY + kVerifySegment - 1) / kVerifySegment;

template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Piece {  // 16 bytes at the alignment of an element: rows may begin anywhere
    T v[16 / sizeof(T)];
};

// A piece at the row's end: 0 for what lies behind it.  The branches keep the piece in scratch memory, and every piece of the last segment takes this
// way, whole ones too: some 1.2 us of a short call.
template <typename T>
__device__ __forceinline__ Piece<T> up_to_end(const T *row, int at, int vocabulary)
{
    constexpr int kEach = 16 / sizeof(T);
    Piece<T> r = {};
    if (at + kEach <= vocabulary) return *reinterpret_cast<const Piece<T> *>(row + at);
    if (at < vocabulary) {
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (at + j < vocabulary) r.v[j] = row[at + j];
    }
    return r;
}

template <typename T, bool kDraft>
__device__ __forceinline__ double segment_sum(const Weights<T, kDraft> &w, int g, int vocabulary, int lane)
{
    constexpr int kEach = 16 / sizeof(T), kPieces = kVerifySegment / 64 / kEach;
    const int begin = g * kVerifySegment;
    constexpr int kAtOnce = 4;  // pieces of a row in flight, of both rows where there are two
    const bool whole = begin + kVerifySegment <= vocabulary;
    const bool leave_out = !kDraft && w.without >= begin && w.without < begin + kVerifySegment;
    double sum = 0.0;
    auto add = [&](auto two) {
        constexpr bool kTwo = decltype(two)::value;  // two rows
#pragma unroll 1
        for (int i0 = 0; i0 < kPieces; i0 += kAtOnce) {
            Piece<T> p[kAtOnce], q[kAtOnce];
            const int at = begin + (i0 * 64 + lane) * kEach;  // of piece i: at + i * 64 * kEach
            if (whole) {
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) p[i] = *reinterpret_cast<const Piece<T> *>(w.p + at + i * 64 * kEach);
                if constexpr (kTwo) {
#pragma unroll
                    for (int i = 0; i < kAtOnce; ++i) q[i] = *reinterpret_cast<const Piece<T> *>(w.q + at + i * 64 * kEach);
                }
            } else {
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                    p[i] = up_to_end(w.p, at + i * 64 * kEach, vocabulary);
                    if constexpr (kTwo) q[i] = up_to_end(w.q, at + i * 64 * kEach, vocabulary);
                }
            }
            if (leave_out) {
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
                    for (int j = 0; j < kEach; ++j) p[i].v[j] = at + i * 64 * kEach + j == w.without ? T{} : p[i].v[j];
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    if constexpr (kTwo) sum += w.of(p[i].v[j], q[i].v[j]);
                    else sum += (double)as_probability(p[i].v[j]);
                }
                __builtin_amdgcn_sched_barrier(0);  // one piece's numbers in 64 bits at a time, or they spill
            }
        }
    };
    if (kDraft && w.q != nullptr) add(std::true_type{});
    else add(std::false_type{});
    return of_lane(wave_running_sum(sum), 63);
}

// What is drawn of a sequence: where its weights are, and how many tokens came before.
template <typename T, bool kDraft>
struct Drawn {
    Weights<T, kDraft> w;
    int accepted, count;   // count < 0: no sequence at this place
};

template <typename T, bool kDraft>
__device__ __forceinline__ Drawn<T, kDraft> look_up(const VerifyArgs &a, int s, int accepted, int count)
{
    Drawn<T, kDraft> d;
    d.count = count;
    d.accepted = accepted;
    d.w = {nullptr, nullptr, -1};
    if (count < 0) return d;
    d.w.p = static_cast<const T *>(a.target) + ((long long)s * (a.drafts_max + 1) + accepted) * a.target_stride;
    if (accepted < count) {
        if (kDraft) d.w.q = static_cast<const T *>(a.draft) + ((long long)s * a.drafts_max + accepted) * a.draft_stride;
        else d.w.without = a.drafts[(long long)s * a.drafts_max + accepted];
    }
    return d;
}

// The first entry whose running sum lies beyond u times the total, by the whole workgroup, from the segments' sums; -1: all are 0.
// Every wavefront finds the segment by itself (running sums of 64 segments at a time), then takes 128 neighbouring entries of it.
constexpr int kVerifyWaves = kVerifyThreads / 64;
static_assert(kVerifyWaves * 128 == kVerifySegment, "two entries of the segment to a lane");
struct DrawRoom {
    double sums[kVerifyWaves];
    int first[kVerifyWaves], last[kVerifyWaves];
};
template <typename T, bool kDraft>
__device__ __forceinline__ int draw(const Weights<T, kDraft> &w, const double *sums, int segments, int vocabulary, double u, DrawRoom &room,
                                    int lane, int wave)
{
    double total = 0.0;
    for (int g0 = 0; g0 < segments; g0 += 64) {
        const double v = g0 + lane < segments ? sums[g0 + lane] : 0.0;
        total += of_lane(wave_running_sum(v), 63);
    }
    const double mark = u * total;
    double carry = 0.0, before = 0.0;
    int g = -1;
    for (int g0 = 0; g0 < segments; g0 += 64) {
        const double v = g0 + lane < segments ? sums[g0 + lane] : 0.0, upto = wave_running_sum(v);
        const unsigned long long any = __ballot(v > 0.0), beyond = __ballot(v > 0.0 && carry + upto > mark);
        if (any != 0) {  // where rounding leaves no segment beyond the mark: the last one with any weight
            const int at = beyond != 0 ? __builtin_ctzll(beyond) : 63 - __builtin_clzll(any);
            g = g0 + at;
            const double left = of_lane(upto, at > 0 ? at - 1 : 0);
            before = at > 0 ? carry + left : carry;
        }
        if (beyond != 0) break;
        carry += of_lane(upto, 63);
    }
    if (g < 0) return -1;  // the same in every wavefront
    const int at = g * kVerifySegment + wave * 128 + lane * 2;
    const double v0 = at < vocabulary ? w.at(at) : 0.0, v1 = at + 1 < vocabulary ? w.at(at + 1) : 0.0;
    const double upto = wave_running_sum(v0 + v1);
    if (lane == 63) room.sums[wave] = upto;
    __syncthreads();
    for (int i = 0; i < wave; ++i) before += room.sums[i];
    const double c0 = before + (upto - (v0 + v1)) + v0, c1 = before + upto;
    const bool in0 = v0 > 0.0 && c0 > mark, in1 = v1 > 0.0 && c1 > mark;
    const unsigned long long in = __ballot(in0 || in1), any = __ballot(v0 > 0.0 || v1 > 0.0);
    const int first = __builtin_amdgcn_readlane(in0 ? at : at + 1, in != 0 ? __builtin_ctzll(in) : 0);
    const int last = __builtin_amdgcn_readlane(v1 > 0.0 ? at + 1 : at, any != 0 ? 63 - __builtin_clzll(any) : 0);
    if (lane == 0) {
        room.first[wave] = in != 0 ? first : -1;
        room.last[wave] = any != 0 ? last : -1;
    }
    __syncthreads();
    int token = -1;
    for (int i = kVerifyWaves - 1; i >= 0; --i) token = room.last[i] > token ? room.last[i] : token;
    for (int i = kVerifyWaves - 1; i >= 0; --i) token = room.first[i] >= 0 ? room.first[i] : token;
    return token;
}

template <typename T, bool kDraft>
__device__ __forceinline__ void write_tokens(const VerifyArgs &a, int s, const Drawn<T, kDraft> &d, int token, int lane)
{
    int32_t *out = a.tokens + (long long)s * (a.drafts_max + 1);
    for (int i = lane; i <= a.drafts_max; i += 64)
        out[i] = i < d.accepted ? a.drafts[(long long)s * a.drafts_max + i] : (i == d.accepted ? token : -1);
    if (lane == 0) a.accepted[s] = d.accepted;
}

// What the first of two launches leaves for the second.
struct VerifyScratch {
    double *sums;     // [sequences][segments]
    int2 *accepted;   // [sequences]: accepted tokens, drafted tokens
};

// First of two launches: the segments' sums, a wavefront to a segment, by as many workgroups as the row has work for.
constexpr int kVerifySumWaves = 4;
template <typename T, bool kDraft>
__global__ void __launch_bounds__(kVerifySumWaves * 64) verify_sums_kernel(VerifyArgs a, int segments, VerifyScratch to)
{
    const int s = blockIdx.y, lane = threadIdx.x & 63, g = blockIdx.x * kVerifySumWaves + wave_of_thread();
    if (g >= segments) return;
    int count;
    const int accepted = count_accepted<T, kDraft>(a, s, lane, count);
    const Drawn<T, kDraft> d = look_up<T, kDraft>(a, s, accepted, count);
    if (g == 0 && lane == 0) to.accepted[s] = make_int2(accepted, count);
    if (d.count < 0) return;
    const double v = segment_sum<T, kDraft>(d.w, g, a.vocabulary, lane);
    if (lane == 0) to.sums[(long long)s * segments + g] = v;
}

// One workgroup per sequence: the whole path in one launch, or (kGiven) what is left of it once the segments' sums are there.
template <typename T, bool kDraft, bool kGiven>
__global__ void __launch_bounds__(kVerifyThreads) verify_kernel(VerifyArgs a, int segments, VerifyScratch given)
{
    __shared__ double sums[kVerifyMaxSegments];
    __shared__ DrawRoom room;
    const int s = blockIdx.x, lane = threadIdx.x & 63, wave = wave_of_thread();
    int2 found;
    if (kGiven) found = given.accepted[s];
    else found.x = count_accepted<T, kDraft>(a, s, lane, found.y);
    Drawn<T, kDraft> d = look_up<T, kDraft>(a, s, found.x, found.y);
    if (d.count < 0) {
        if (wave == 0) write_tokens<T, kDraft>(a, s, d, -1, lane);
        return;
    }
    const double u = (double)a.uniforms[(long long)s * (a.drafts_max + 1) + a.drafts_max];
    for (int round = 0; round < 2; ++round) {
        if (kGiven && round == 0) {
            for (int g = threadIdx.x; g < segments; g += kVerifyThreads) sums[g] = given.sums[(long long)s * segments + g];
        } else {
            for (int g = wave; g < segments; g += kVerifyThreads / 64) {
                const double v = segment_sum<T, kDraft>(d.w, g, a.vocabulary, lane);
                if (lane == 0) sums[g] = v;
            }
        }
        __syncthreads();
        bool any = false;
        for (int g = lane; g < segments; g += 64) any |= sums[g] > 0.0;
        if (__ballot(any) != 0) break;  // the same in every wavefront
        d.w.q = nullptr, d.w.without = -1;  // nothing is left of the difference: the target's row alone
        __syncthreads();
    }
    const int token = draw<T, kDraft>(d.w, sums, segments, a.vocabulary, u, room, lane, wave);
    if (wave == 0) write_tokens<T, kDraft>(a, s, d, token, lane);
}
