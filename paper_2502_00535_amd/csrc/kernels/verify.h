// Part of decoding_kernels.hip (included there, inside its anonymous namespace): verification of drafted tokens.
#pragma once

// ----------------------------------------------------------------------------- verification

template <typename T>
__device__ __forceinline__ float as_probability(T v)
{
    const unsigned u = __float_as_uint(to_float(v));
    return u - 1u < 0x7f7fffffu ? __uint_as_float(u) : 0.0f;  // a finite number above 0 stays as it is
}

struct VerifyArgs {
    const void *target, *draft;
    long long target_stride, draft_stride;
    const int32_t *drafts, *counts;
    const float *uniforms;
    int32_t *tokens, *accepted;
    int drafts_max, vocabulary;
};

// How many drafted tokens of the sequence stand, by one wavefront (every lane gets the answer): 64 tests at a time.
template <typename T, bool kDraft>
__device__ __forceinline__ int count_accepted(const VerifyArgs &a, int s, int count, int lane)
{
    const T *target = static_cast<const T *>(a.target) + (long long)s * (a.drafts_max + 1) * a.target_stride;
    const T *draft = kDraft ? static_cast<const T *>(a.draft) + (long long)s * a.drafts_max * a.draft_stride : nullptr;
    for (int i0 = 0; i0 < count; i0 += 64) {
        const int i = i0 + lane;
        bool refused = false;
        if (i < count) {
            const int x = a.drafts[(long long)s * a.drafts_max + i];
            const double u = (double)a.uniforms[(long long)s * (a.drafts_max + 1) + i];
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
    return count;
}

// The weights that the token is drawn from.
template <typename T, bool kDraft>
struct Weights {
    const T *p, *q;    // q: the draft's row, nullptr where the target's row counts alone
    int without;       // the entry that counts as 0 (a refused token of a draft without probabilities), or -1
    __device__ __forceinline__ double operator()(int j) const
    {
        double w = (double)as_probability(p[j]);
        if (kDraft && q != nullptr) {
            w -= (double)as_probability(q[j]);
            w = w > 0.0 ? w : 0.0;
        }
        return !kDraft && j == without ? 0.0 : w;
    }
};

// One workgroup per sequence.  Sums in a fixed order: the row is cut into segments of kVerifySegment entries, a segment is summed by one
// wavefront, the segments' sums are added up one after the other, and the entry is looked for in its segment by one wavefront.
constexpr int kVerifySegment = 2048;
constexpr int kVerifyThreads = 1024;
constexpr int kVerifyMaxSegments = (NMS_MAX_VOCABULARY + kVerifySegment - 1) / kVerifySegment;

__device__ __forceinline__ double wave_sum(double v)
{
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

template <typename T, bool kDraft>
__global__ void __launch_bounds__(kVerifyThreads) verify_kernel(VerifyArgs a)
{
    __shared__ double sums[kVerifyMaxSegments];
    const int s = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int count = a.counts != nullptr ? a.counts[s] : a.drafts_max;
    count = count < a.drafts_max ? count : a.drafts_max;
    int32_t *out = a.tokens + (long long)s * (a.drafts_max + 1);
    if (count < 0) {
        for (int i = threadIdx.x; i <= a.drafts_max; i += kVerifyThreads) out[i] = -1;
        if (threadIdx.x == 0) a.accepted[s] = 0;
        return;
    }
    const int accepted = count_accepted<T, kDraft>(a, s, count, lane);
    Weights<T, kDraft> w;
    w.p = static_cast<const T *>(a.target) + ((long long)s * (a.drafts_max + 1) + accepted) * a.target_stride;
    w.q = nullptr;
    w.without = -1;
    if (accepted < count) {
        if (kDraft) w.q = static_cast<const T *>(a.draft) + ((long long)s * a.drafts_max + accepted) * a.draft_stride;
        else w.without = a.drafts[(long long)s * a.drafts_max + accepted];
    }
    const int segments = (a.vocabulary + kVerifySegment - 1) / kVerifySegment;
    double total = 0.0;
    for (int round = 0; round < 2; ++round) {
        for (int g = wave; g < segments; g += kVerifyThreads / 64) {
            double v = 0.0;
            const int end = min((g + 1) * kVerifySegment, a.vocabulary);
            for (int j = g * kVerifySegment + lane; j < end; j += 64) v += w(j);
            v = wave_sum(v);
            if (lane == 0) sums[g] = v;
        }
        __syncthreads();
        total = 0.0;
        for (int g = 0; g < segments; ++g) total += sums[g];
        __syncthreads();
        if (total > 0.0) break;
        w.q = nullptr, w.without = -1;  // nothing is left of the difference: the target's row alone
    }
    for (int i = threadIdx.x; i <= a.drafts_max; i += kVerifyThreads)
        if (i != accepted) out[i] = i < accepted ? a.drafts[(long long)s * a.drafts_max + i] : -1;
    if (wave != 0) return;
    int token = -1;
    if (total > 0.0) {
        const double past = (double)a.uniforms[(long long)s * (a.drafts_max + 1) + a.drafts_max] * total;
        double before = 0.0;
        int g = 0, last = 0;
        for (int i = 0; i < segments; ++i) if (sums[i] > 0.0) last = i;
        for (; g < last && !(before + sums[g] > past); ++g) before += sums[g];
        // lane's own stretch of the segment
        constexpr int kEach = kVerifySegment / 64;
        const int begin = g * kVerifySegment + lane * kEach, end = min(begin + kEach, a.vocabulary);
        double own = 0.0;
        for (int j = begin; j < end; ++j) own += w(j);
        double sum = own;
        for (int d = 1; d < 64; d <<= 1) {
            const double left = __shfl_up(sum, d);
            if (lane >= d) sum += left;
        }
        double c = before + (sum - own);
        int first = -1, final = -1;
        for (int j = begin; j < end; ++j) {
            const double v = w(j);
            if (v > 0.0) {
                c += v;
                final = j;
                if (first < 0 && c > past) first = j;
            }
        }
        unsigned long long mask = __ballot(first >= 0);
        if (mask != 0) token = __shfl(first, __builtin_ctzll(mask));
        else token = __shfl(final, 63 - __builtin_clzll(__ballot(final >= 0)));
    }
    if (lane == 0) {
        out[accepted] = token;
        a.accepted[s] = accepted;
    }
}
