// One token per row, drawn by a given uniform number from what temperature, top-k, top-p and min-p leave (bpe_sample_tokens).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "bpe_numeric.h"

namespace bpe {

constexpr int kSlice = 8192, kSliceThreads = 512, kSliceBits = 48;      // logits of a row per workgroup, bits behind the point of their weights
constexpr int kMostSlices = 512, kBins = 512, kBinsPerOctave = 8;
constexpr int kList = 4096, kFewTokens = 1024;
constexpr int64_t kSlicesAtOnce = 8192;

// What a slice's workgroup leaves for the row's.
struct SlicePart {
    float most;                        // the largest logit
    uint32_t nan;
    int32_t above, top;                // logits above -infinity; the largest one's bin
    uint64_t sum;                      // of the weights
};
struct SliceBins {
    uint64_t mass[kBins];
    uint32_t count[kBins];
};

struct SampleParams {
    const void *logits;
    int64_t stride;
    int32_t row0, n_vocab, bits;       // the launch's first row; bits behind the point of a weight where a row is one piece
    int32_t slices;                    // of a row; 0: it is one piece
    SlicePart *parts;                  // [rows of the launch][slices]
    SliceBins *bins;
    const float *uniform, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int32_t *ids;
    float *logprobs;
};

// Order of the logits as unsigned numbers; -0 and 0 are equal.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __builtin_bit_cast(float, key & 0x80000000u ? key ^ 0x80000000u : ~key); }
constexpr uint32_t kKeyOfMinusInfinity = 0x007fffffu;

// 2^y for y <= 0, in 64 bits: 2^n times a polynomial of ten terms in the rest, |f| <= 1/2, fitted to a relative error of 6e-16 with 1 at 0.  (The constants
// come from scalar registers: left to the compiler, each step copies its constant into the register that it adds to.)
__device__ __forceinline__ double step_of(double s, double f, double constant) {
    double r;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(r) : "v"(s), "v"(f), "s"(constant));
    return r;
}
__device__ __forceinline__ double exp2_of(double y) {
    // (adding 1.5 2^52 leaves the nearest whole number in the low bits: conversions and ldexp take four times as long as additions)
    constexpr double kWhole = 6755399441055744.0;
    y = fmax(y, -1000.0);
    const double t = y + kWhole, f = y - (t - kWhole);
    double s = step_of(step_of(7.070977866508139e-09, f, 1.0205905413765595e-07), f, 1.3215451633221434e-06);
    s = step_of(step_of(s, f, 1.5252672924850737e-05), f, 0.00015403530424776529);
    s = step_of(step_of(s, f, 0.0013333558200794592), f, 0.009618129107618665);
    s = step_of(step_of(s, f, 0.05550410866465167), f, 0.24022650695910075);
    s = step_of(s, f, 0.6931471805599462);
    return __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, fma(s, f, 1.0)) + (__builtin_bit_cast(uint64_t, t) << 52));
}

// A token's weight is exp((x - most) / temperature) in whole multiples of a power of two: sums of them do not depend on their order.
struct Weights {
    float most;
    bool endless;                      // the largest logit is +infinity
    double slope;                      // log2 e / temperature
    double one;                        // adding it puts a weight's bits at the end of the number's
    __device__ __forceinline__ Weights(float most_, double slope_, int bits) : most(most_), endless(most_ == INFINITY), slope(slope_), one(__builtin_ldexp(1.0, 52 - bits)) {}
    __device__ __forceinline__ double exact(float x) const {
        return endless ? (x == INFINITY ? 1.0 : 0.0) : finite(x);
    }
    __device__ __forceinline__ double finite(float x) const { return exp2_of(((double)x - (double)most) * slope); }
    __device__ __forceinline__ uint64_t operator()(float x) const { return __builtin_bit_cast(uint64_t, exact(x) + one) - __builtin_bit_cast(uint64_t, one); }
};

// Bins of logits, the same for all of a row: eight to a factor of two in weight.
struct Bins {
    float scale;
    __device__ __forceinline__ explicit Bins(double slope) : scale((float)fmin(kBinsPerOctave * slope, 1e30)) {}
    // A logit's place among the bins, rounded by itself: fused with a sum behind it, a product just below a whole number would not be what it is where
    // the bins are counted.
    __device__ __forceinline__ float place(float x) const {
#pragma clang fp contract(off)
        return x * scale;
    }
    __device__ __forceinline__ int operator()(float x) const { return (int)__builtin_floorf(fminf(fmaxf(place(x), -1e9f), 1e9f)); }
};

// What a row's request asks for.
struct Request {
    float temperature, top_p, min_p, uniform;
    int top_k;                         // 0: all
    bool greedy, filtered, weighed;    // weighed: the weights of all logits are needed, not of a few largest ones alone
    __device__ __forceinline__ Request(const SampleParams &p, int row) {
        temperature = p.temperature ? p.temperature[row] : 1.0f;
        top_k = p.top_k ? p.top_k[row] : 0;
        if (top_k < 0 || top_k >= p.n_vocab) top_k = 0;
        top_p = p.top_p ? p.top_p[row] : 1.0f;
        min_p = p.min_p ? p.min_p[row] : 0.0f;
        min_p = min_p > 0 ? fminf(min_p, 1.0f) : 0.0f;
        uniform = fminf(fmaxf(p.uniform[row], 0x1p-30f), 1 - 0x1p-24f);
        greedy = !(temperature > 0);
        filtered = top_k > 0 || top_p < 1 || min_p > 0;
        weighed = top_k == 0 || top_k > kFewTokens;
    }
};
constexpr double kLog2e = 1.4426950408889634074;

typedef unsigned long long U64;

// A slice of a row per workgroup, read once and held in registers: its largest logit, the sum of its weights relative to that, and, where
// the row has a filter, counts and sums of the weights by bins of logits.  Bound by instructions: 512 x 100257 f32 55 to 56 us (206 MB, 3.7 TB/s), where 33 vector
// instructions for a logit, most of them the exponential in 64 bits, are 43 at four cycles each.  (In 64 bits, because a token is drawn by where a sum of all
// weights passes a number: the sum has to be good to far less than a weight, and in whole multiples it is the same in any order.)  64 x 100256 bf16 with bins 15.6.
template <class T, bool FILTERS>
__global__ void __launch_bounds__(kSliceThreads, 8) sample_slices_kernel(SampleParams p) {
    constexpr int kChunks = kSlice / 8 / kSliceThreads, kWaves = kSliceThreads / kWave;
    __shared__ SliceBins bins;
    __shared__ float most_of[kWaves];
    __shared__ U64 sum_of[kWaves];
    __shared__ int above_of[kWaves];
    const int tid = threadIdx.x, wv = tid >> 6;
    const int r = blockIdx.x / p.slices, slice = blockIdx.x - r * p.slices, row = p.row0 + r;
    const int begin = slice * kSlice, end = min(p.n_vocab, begin + kSlice);
    const typename T::raw *logits = (const typename T::raw *)p.logits + row * p.stride;
    float v[kChunks][8];
#pragma unroll
    for (int u = 0; u < kChunks; ++u) load8<T>(logits, begin + 8 * (u * kSliceThreads + tid), end, v[u]);
    const Request ask(p, row);
    float most = -INFINITY;
    bool nan = false;
    if (begin + kSlice > end) {
#pragma unroll
        for (int u = 0; u < kChunks; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (begin + 8 * (u * kSliceThreads + tid) + e >= end) v[u][e] = -INFINITY;
    }
#pragma unroll
    for (int u = 0; u < kChunks; ++u)
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            nan |= __builtin_isunordered(v[u][e], v[u][e + 1]);
            most = fmaxf(most, fmaxf(v[u][e], v[u][e + 1]));
        }
    most = max_so_far(most);
    if ((tid & 63) == 63) most_of[wv] = most;
    const bool binned = FILTERS && !ask.greedy;
    if (binned)
        for (int b = tid; b < kBins; b += kSliceThreads) { bins.mass[b] = 0; bins.count[b] = 0; }
    nan = __syncthreads_or(nan);
    most = most_of[0];
#pragma unroll
    for (int s = 1; s < kWaves; ++s) most = fmaxf(most, most_of[s]);
    SlicePart *part = p.parts + (int64_t)r * p.slices + slice;
    if (nan || ask.greedy || most == -INFINITY || most == INFINITY) {
        int endless = 0;
#pragma unroll
        for (int u = 0; u < kChunks; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) endless += v[u][e] == INFINITY;
        endless = wave_sum(endless);
        if ((tid & 63) == 0) above_of[wv] = endless;
        __syncthreads();
        endless = 0;
        for (int s = 0; s < kWaves; ++s) endless += above_of[s];
        if (tid == 0) *part = SlicePart{most, nan, endless, 0, (U64)endless << kSliceBits};      // (nobody reads such a slice's bins)
        return;
    }
    const double slope = kLog2e / (double)ask.temperature;
    const Weights weight(most, slope, kSliceBits);
    const Bins bin(slope);
    const int top = bin(most);
    U64 sum = 0;
    int above = 0;
    // (the weight of -infinity is 0)
    const auto go = [&](auto weighed) {
#pragma unroll
        for (int u = 0; u < kChunks; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = v[u][e];
                U64 w = 0;                                           // (with the bits of `one` in front)
                if constexpr (decltype(weighed)::value) sum += w = __builtin_bit_cast(uint64_t, weight.finite(x) + weight.one);
                if constexpr (FILTERS) {
                    const bool is = x > -INFINITY;
                    above += is;
                    const int b = top - bin(x);
                    if (!is || b >= kBins) continue;
                    if (ask.top_k) atomicAdd(&bins.count[b], 1u);
                    if constexpr (decltype(weighed)::value) atomicAdd((U64 *)&bins.mass[b], w - __builtin_bit_cast(uint64_t, weight.one));
                }
                // (not all logits' intermediate values at once, nor all weights before the first sum)
                if constexpr (decltype(weighed)::value) asm volatile("" : "+v"(sum));
                if (e % 2) __builtin_amdgcn_sched_barrier(0);
            }
    };
    if (!FILTERS || ask.weighed) {
        go(std::true_type());
        sum -= 8 * kChunks * __builtin_bit_cast(uint64_t, weight.one);
    } else {
        go(std::false_type());
    }
    sum = wave_sum(sum);
    above = wave_sum(above);
    if ((tid & 63) == 0) { sum_of[wv] = sum; above_of[wv] = above; }
    __syncthreads();
    if (tid == 0) {
        SlicePart all = {most, 0, 0, top, 0};
        for (int s = 0; s < kWaves; ++s) { all.sum += sum_of[s]; all.above += above_of[s]; }
        *part = all;
    }
    if (!binned) return;
    SliceBins *to = p.bins + (int64_t)r * p.slices + slice;
    if (ask.weighed && tid < (int)sizeof(bins.mass) / 16) ((U4 *)to->mass)[tid] = ((const U4 *)bins.mass)[tid];
    if (ask.top_k && tid < (int)sizeof(bins.count) / 16) ((U4 *)to->count)[tid] = ((const U4 *)bins.count)[tid];
}

constexpr int kSampleThreads = 1024, kSampleWaves = kSampleThreads / kWave;

struct SampleLds {
    U64 part_mass[kSampleWaves];
    uint32_t part_count[kSampleWaves], part_key[kSampleWaves];
    int32_t part_at[kSampleWaves];
    double part_sum[kSampleWaves];
    // which slice, where in it, and the sum of all weights
    int chosen;
    U64 target;
    double total;
    // of the row's slices
    double factor[kMostSlices];
    U64 kept[kMostSlices];
    float most[kMostSlices];
    int top[kMostSlices];
};
struct SampleDigits {
    U64 mass[256], mass_before;
    uint32_t count[256], count_before, digit, there;
};
struct FilterLds {
    SampleDigits digits;
    uint32_t tied[kMostSlices];        // of a slice, logits equal to the bound
    // the bin that holds a border, and what stands in front of it
    int border;
    uint32_t border_before;
    double border_mass;
    // the logits of some bins, from sixteen bytes that hold any of them
    uint32_t in_list, least_key, most_key, in_sifted;
    uint32_t list_key[kList];
    __attribute__((aligned(8))) uint32_t list_at[kList];
    U4 sifted[kList];
    uint32_t sifted_at[kList];
};
struct NoLds {};

// The key of an element of a sequence at which the running sum, from the largest key down, reaches `target` (by mass or by count), and how many of
// that key are needed for it; found eight bits at a time.  `each` calls its argument with every key; of the keys that are equal to
// `bound` so many as `ties` count, lower ones do not.
// (The last bits of a key are no digit where logits have 16 bits: 16 of bf16, 13 of f16 are the same for all of a sign.)
template <class T> constexpr int kLastShift = T::kCode == BPE_F32 ? 0 : T::kCode == BPE_BF16 ? 16 : 8;
template <class T, class Each, class Weight>
__device__ __forceinline__ void find_border(SampleDigits &lds, Each each, const Weight &weight, bool by_mass, U64 target, int shift, uint32_t prefix, uint32_t &bound, uint32_t &ties) {
    const int tid = threadIdx.x, lane = tid & 63;
    uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8), before_count = 0;
    U64 before_mass = 0;
    for (; shift >= kLastShift<T>; shift -= 8) {
        __syncthreads();
        if (tid < 256) { lds.mass[tid] = 0; lds.count[tid] = 0; }
        __syncthreads();
        each([&](uint32_t key) {
            if (key <= bound || (key & mask) != prefix) return;
            atomicAdd(&lds.count[key >> shift & 255], 1u);
            if (by_mass) atomicAdd(&lds.mass[key >> shift & 255], (U64)weight(value_of(key)));
        });
        __syncthreads();
        if (tid < kWave) {
            if (lane == 0 && ties && (bound & mask) == prefix) {
                lds.count[bound >> shift & 255] += ties;
                if (by_mass) lds.mass[bound >> shift & 255] += ties * weight(value_of(bound));
            }
            wave_sync();
            // The last digit from above that holds anything and before which the sum is below the target; the first one if there is none.
            U64 mass[4];
            uint32_t count[4];
            U64 lane_mass = 0;
            uint32_t lane_count = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int d = 255 - 4 * lane - j;
                mass[j] = lane_mass;
                count[j] = lane_count;
                lane_mass += lds.mass[d];
                lane_count += lds.count[d];
            }
            const U64 mass_before = sum_so_far(lane_mass) + before_mass - lane_mass;
            const uint32_t count_before = sum_so_far(lane_count) + before_count - lane_count;
            int first = -1, last = -1;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (lds.count[255 - 4 * lane - j]) {
                    if (first < 0) first = j;
                    if (by_mass ? mass_before + mass[j] < target : count_before + count[j] < target) last = j;
                }
            const U64 any = __ballot(first >= 0), reach = __ballot(last >= 0);
            const int winner = reach ? 63 - __builtin_clzll(reach) : any ? __builtin_ctzll(any) : 0;
            if (lane == winner) {
                const int j = reach ? last : max(first, 0);
                lds.digit = (uint32_t)(255 - 4 * lane - j);
                lds.mass_before = mass_before + mass[j];
                lds.count_before = count_before + count[j];
                lds.there = lds.count[255 - 4 * lane - j];
            }
        }
        __syncthreads();
        prefix |= lds.digit << shift;
        mask |= 255u << shift;
        before_mass = lds.mass_before;
        before_count = lds.count_before;
    }
    if (shift >= 0) prefix |= prefix & 0x80000000u ? 0u : (1u << (shift + 8)) - 1;
    U64 wanted;
    if (by_mass) {
        const U64 one = weight(value_of(prefix));
        wanted = target > before_mass && one ? (target - before_mass + one - 1) / one : 1;
    } else {
        wanted = target > before_count ? target - before_count : 1;
    }
    bound = prefix;
    ties = (uint32_t)min(wanted, (U64)lds.there);
    __syncthreads();
}

// A row per workgroup: without a filter the choice of a slice and of a token in it, 13 us for 512 rows of 100257 (8,192 weights of a row computed again).  With filters a chain of some twenty short
// steps with barriers between them: 1 x 50256 f32, all filters, 26 us (merging bins 3, going over the row's logits for those of one bin 5, twice a border 8,
// min-p and what stays of each slice 3, drawing 3), 64 x 100256 bf16, top-p, 29 for the longest row (5, 9, 3, 3, 5).  What is bound there is the one compute unit that
// a row has: bringing the row and the bins into L2 beforehand gained 1 % at most.  What stays of a row is, in the order of the logits (equal ones by index), the first so many tokens: those above a key
// `bound`, and the first `ties` of that key.
template <class T, bool FILTERS> struct SampleRow {
    const SampleParams &p;
    SampleLds &lds;
    typename std::conditional<FILTERS, FilterLds, NoLds>::type &list;
    const int row, tid, lane, wv, n;
    const typename T::raw *logits;
    const Request ask;
    uint32_t bound = kKeyOfMinusInfinity, ties = 0;
    float most;                        // of the row
    double slope;

    __device__ __forceinline__ SampleRow(const SampleParams &p_, SampleLds &lds_, typename std::conditional<FILTERS, FilterLds, NoLds>::type &list_)
        : p(p_), lds(lds_), list(list_), row(p_.row0 + blockIdx.x), tid(threadIdx.x), lane(threadIdx.x & 63), wv(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)),
          n(p_.n_vocab), logits((const typename T::raw *)p_.logits + row * p_.stride), ask(p_, row) {}

    // Sixteen bytes of logits from token c on, or the row's last sixteen.
    static constexpr int kPer = 16 / (int)sizeof(typename T::raw);
    __device__ __forceinline__ int place_of(int c) const { return min(c, n - kPer); }
    __device__ __forceinline__ U4 some_logits(int c) const { return *(const U4Any *)(logits + place_of(c)); }
    __device__ __forceinline__ void nothing(bool nan) {
        if (tid != 0) return;
        p.ids[row] = -1;
        if (p.logprobs) p.logprobs[row] = nan ? __builtin_nanf("") : -INFINITY;
    }
    __device__ __forceinline__ float log_share(float x, double total) const {
        return (float)((most == INFINITY ? 0.0 : ((double)x - (double)most) / (double)ask.temperature) - log(total));
    }
    __device__ __forceinline__ void best(int at) {
        if (tid != 0) return;
        p.ids[row] = at;
        if (p.logprobs) p.logprobs[row] = 0.0f;
    }
    // The first token of a slice by index whose running sum passes `target`, or the last that weighs anything.  The workgroup holds the slice in
    // registers, eight neighbours per thread, so that threads stand in the order of the tokens.
    __device__ __forceinline__ void draw(int begin, int end, U64 target, uint32_t ties_before, const Weights &weight, double total) {
        float x[8];
        load8<T>(logits, begin + 8 * tid, end, x);
        const int mine = min(max(end - (begin + 8 * tid), 0), 8);
        U64 w[8], sum = 0;
        uint32_t tie_bits = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t key = key_of(x[e]);
            w[e] = e < mine && key > bound ? weight(x[e]) : 0;
            if (e < mine && key == bound) tie_bits |= 1u << e;
            __builtin_amdgcn_sched_barrier(0);
        }
        if (FILTERS && ties > ties_before) {
            const U64 of_tie = weight(value_of(bound));
            const uint32_t here = __popc(tie_bits);
            uint32_t seen = sum_so_far(here);
            if (lane == 63) lds.part_count[wv] = seen;
            __syncthreads();
            seen += ties_before - here;
            for (int s = 0; s < wv; ++s) seen += lds.part_count[s];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (tie_bits >> e & 1 && seen++ < ties) w[e] = of_tie;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += w[e];
        U64 until = sum_so_far(sum);
        if (lane == 63) lds.part_mass[wv] = until;
        __syncthreads();
        U64 all = 0;
#pragma unroll 4
        for (int s = 0; s < kSampleWaves; ++s) {
            if (s == wv) until += all;
            all += lds.part_mass[s];
        }
        target = min(target, all - 1);
        U64 at = until - sum;
        if (at > target || until <= target) return;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            at += w[e];
            if (at > target) {
                p.ids[row] = begin + 8 * tid + e;
                if (p.logprobs) p.logprobs[row] = log_share(to_float<T>(logits[begin + 8 * tid + e]), total);
                return;
            }
        }
    }

    // A row as one piece: every pass reads it again, by one workgroup.  64 x 100256 with top-p 0.9: 220 to 264 us where logits are infinite, or flat (a standard deviation of 0.05), or
    // the temperature is 1e-6; 806 where all are equal (431 with top-k 50 alone): their counts and sums meet at one address in LDS.  64 x 8192 17 us, with all filters 41.
    __device__ __forceinline__ void whole() {
        uint32_t top = 0;
        int top_at = 0;
        bool nan = false;
        for (int v = tid; v < n; v += kSampleThreads) {
            const float x = to_float<T>(logits[v]);
            nan |= x != x;
            const uint32_t key = key_of(x);
            if (key > top) { top = key; top_at = v; }
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) {
            const uint32_t key = (uint32_t)__shfl_xor((int)top, d);
            const int at = __shfl_xor(top_at, d);
            if (key > top || (key == top && at < top_at)) { top = key; top_at = at; }
        }
        if (lane == 0) { lds.part_key[wv] = top; lds.part_at[wv] = top_at; }
        nan = __syncthreads_or(nan);
#pragma unroll 4
        for (int s = 0; s < kSampleWaves; ++s)
            if (lds.part_key[s] > top || (lds.part_key[s] == top && lds.part_at[s] < top_at)) { top = lds.part_key[s]; top_at = lds.part_at[s]; }
        if (nan || top <= kKeyOfMinusInfinity) return nothing(nan);
        if (ask.greedy) return best(top_at);
        most = value_of(top);
        slope = kLog2e / (double)ask.temperature;
        bound = kKeyOfMinusInfinity;
        ties = 0;
        const Weights weight(most, slope, p.bits);
        // First top-k's border, then top-p's, for which all that is left has to be summed up; then, with min-p, the parts of the wavefronts are
        // summed up, the part that the uniform number falls into is cut into parts again, and so on.
        int stage = ask.top_k ? 0 : ask.top_p < 1 ? 1 : 2, from = 0, to = n;
        const double least = ask.min_p;
        double total = 0;
        U64 target = 0, before = 0, of_tie = 0;
        uint32_t ties_before = 0;
        const auto stays = [&](float x) { return stage < 2 || least == 0 || weight.exact(x) >= least; };
        for (;;) {
            const int length = (to - from + kSampleWaves - 1) / kSampleWaves;
            U64 all = 0;
            if (stage > 0) {
                U64 mass = 0;
                uint32_t equal = 0;
                const int begin = (int)min((int64_t)from + (int64_t)wv * length, (int64_t)to), end = (int)min((int64_t)begin + length, (int64_t)to);
                for (int v = begin + lane; v < end; v += kWave) {
                    const float x = to_float<T>(logits[v]);
                    const uint32_t key = key_of(x);
                    if (key > bound && stays(x)) mass += weight(x);
                    equal += key == bound;
                }
                mass = wave_sum(mass);
                equal = wave_sum(equal);
                of_tie = ties && stays(value_of(bound)) ? weight(value_of(bound)) : 0;
                __syncthreads();
                if (lane == 0) { lds.part_mass[wv] = mass; lds.part_count[wv] = equal; }
                __syncthreads();
                all = ties * of_tie;
#pragma unroll 4
                for (int s = 0; s < kSampleWaves; ++s) all += lds.part_mass[s];
            }
            if (stage == 2) {
                if (total == 0) {
                    total = (double)all;
                    target = min((U64)((double)ask.uniform * total), all - 1);
                }
                int s = 0;
#pragma unroll 1
                for (; s < kSampleWaves - 1; ++s) {
                    const U64 here = lds.part_mass[s] + min(lds.part_count[s], ties - min(ties, ties_before)) * of_tie;
                    if (before + here > target) break;
                    before += here;
                    ties_before += lds.part_count[s];
                }
                from = (int)min((int64_t)from + (int64_t)s * length, (int64_t)to);
                to = (int)min((int64_t)from + length, (int64_t)to);
                if (to - from <= kWave) break;
                continue;
            }
            if constexpr (FILTERS) {
                const U64 goal = stage == 0 ? (U64)ask.top_k : ask.top_p > 0 ? (U64)__builtin_ceil((double)ask.top_p * (double)all) : 0;
                find_border<T>(list.digits, [&](auto f) {
                    for (int v = tid; v < n; v += kSampleThreads) f(key_of(to_float<T>(logits[v])));
                }, weight, stage == 1, goal, 24, 0, bound, ties);
            }
            stage = stage == 0 && ask.top_p < 1 ? 1 : 2;
        }
        if (wv != 0) return;
        const int v = from + lane;
        const float x = v < to ? to_float<T>(logits[v]) : -INFINITY;
        const uint32_t key = key_of(x);
        const bool tie = v < to && key == bound;
        const uint32_t place = ties_before + (uint32_t)__popcll(__ballot(tie) & ((1ull << lane) - 1));
        const U64 mine = v < to && key > bound && stays(x) ? weight(x) : tie && place < ties ? of_tie : 0;
        const U64 sum = sum_so_far(mine);
        const U64 passed = __ballot(mine > 0 && before + sum > target);
        if (lane == (passed ? __builtin_ctzll(passed) : 0)) {
            p.ids[row] = v;
            if (p.logprobs) p.logprobs[row] = log_share(x, total * __builtin_ldexp(1.0, -p.bits));
        }
    }

    // Which slice the uniform number falls into, and where there; wavefront 0 goes over them in their order.
    __device__ __forceinline__ void choose_slice(int slices) {
        __syncthreads();
        if (wv == 0) {
            const int per = (slices + kWave - 1) / kWave, from = lane * per, to = min(slices, from + per);
            const auto mass = [&](int s) { return (double)lds.kept[s] * lds.factor[s]; };
            double mine = 0;
            for (int s = from; s < to; ++s) mine += mass(s);
            const double sum = sum_so_far(mine), total = of_last(sum), before = __shfl_up(sum, 1);
            const double target = (double)ask.uniform * total;
            const U64 some = __ballot(mine > 0), past = __ballot(mine > 0 && sum > target);
            const int winner = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some | 1);
            if (lane == winner) {
                double at = lane ? before : 0.0;
                int s = from, last = from;
                double last_at = at;
                for (; s < to; ++s) {
                    const double here = mass(s);
                    if (!(here > 0)) continue;
                    last = s;
                    last_at = at;
                    if (at + here > target) break;
                    at += here;
                }
                lds.chosen = last;
                const double local = (target - last_at) / lds.factor[last];
                lds.target = local > 0 ? (local < 9e18 ? (U64)local : ~0ull >> 1) : 0;
                lds.total = total * __builtin_ldexp(1.0, -kSliceBits);
            }
        }
        __syncthreads();
    }

    // A row in slices.  False where the bins do not tell enough: the row is then taken as one piece.
    static constexpr int kHeld = FILTERS ? 4 : 0;
    __device__ __forceinline__ bool from_slices() {
        // a border will be looked for among all logits: as many as sixteen registers hold are loaded at once, ahead of everything else
        U4 held[kHeld + 1];
#pragma unroll
        for (int u = 0; u < kHeld; ++u) held[u] = some_logits(kPer * (tid + u * kSampleThreads));
        const int slices = p.slices;
        const SlicePart *parts = p.parts + (int64_t)blockIdx.x * slices;
        most = -INFINITY;
        bool nan = false;
        int above = 0;
        for (int s = tid; s < slices; s += kSampleThreads) {
            const SlicePart part = parts[s];
            lds.most[s] = part.most;
            lds.top[s] = part.top;
            lds.kept[s] = part.sum;
            most = part.most;
            nan = part.nan;
            above = part.above;
        }
        above = wave_sum(above);
        most = wave_max(most);
        if (lane == 0) { lds.part_sum[wv] = most; lds.part_count[wv] = above; }
        nan = __syncthreads_or(nan);
        above = 0;
#pragma unroll 4
        for (int s = 0; s < kSampleWaves; ++s) { most = fmaxf(most, (float)lds.part_sum[s]); above += lds.part_count[s]; }
        if (nan || most == -INFINITY) { nothing(nan); return true; }
        if (ask.greedy) {
            int s = 0;
            while (lds.most[s] != most) ++s;
            if (tid == 0) lds.chosen = n;
            __syncthreads();
            for (int v = s * kSlice + tid; v < min(n, (s + 1) * kSlice); v += kSampleThreads)
                if (to_float<T>(logits[v]) == most) atomicMin(&lds.chosen, v);
            __syncthreads();
            best(lds.chosen);
            return true;
        }
        slope = kLog2e / (double)ask.temperature;
        const Bins bin(slope);
        const Weights of_row(most, slope, kSliceBits);
        for (int s = tid; s < slices; s += kSampleThreads) lds.factor[s] = of_row.exact(lds.most[s]);
        if constexpr (FILTERS) {
            if (ask.filtered && !(__builtin_fabsf(most) * bin.scale < 4e6f)) return false;    // (infinite, or where bins are no longer told apart well)
            if (ask.filtered && !filter(slices, above, bin, of_row, held)) return false;
        }
        choose_slice(slices);
        const int s = lds.chosen;
        uint32_t ties_before = 0;
        if constexpr (FILTERS) {
            if (ties)
                for (int other = 0; other < s; ++other) ties_before += list.tied[other];
        }
        draw(s * kSlice, min(n, (s + 1) * kSlice), lds.target, ties_before, Weights(lds.most[s], slope, kSliceBits), lds.total);
        return true;
    }

    // Bound and ties, and what stays of every slice (lds.kept, list.tied).
    __device__ __forceinline__ bool filter(int slices, int above, const Bins &bin, const Weights &of_row, const U4 (&held)[kHeld + 1]) {
        const SliceBins *bins = p.bins + (int64_t)blockIdx.x * slices;
        const int top = bin(most);
        __syncthreads();
        // the row's bins, one per thread of the first half (the second half takes every other slice), and what stands in front of each
        uint32_t count = 0;
        double mass = 0;
        const int own = tid & (kBins - 1);
        for (int s0 = tid / kBins; s0 < slices; s0 += 8) {          // four loads under way at a time
            uint32_t counts[4];
            U64 masses[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int s = min(s0 + 2 * u, slices - 1), b = own - (top - lds.top[s]);
                const bool there = s0 + 2 * u < slices && b >= 0 && lds.most[s] > -INFINITY;
                counts[u] = there && ask.top_k ? bins[s].count[b] : 0;
                masses[u] = there && ask.weighed ? bins[s].mass[b] : 0;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                count += counts[u];
                mass += (double)masses[u] * lds.factor[min(s0 + 2 * u, slices - 1)];
            }
        }
        if (tid >= kBins) {
            list.list_key[own] = count;
            ((double *)list.list_at)[own] = mass;
            count = 0;
            mass = 0;
        }
        __syncthreads();
        if (tid < kBins) {
            count += list.list_key[own];
            mass += ((double *)list.list_at)[own];
        }
        mass *= __builtin_ldexp(1.0, -kSliceBits);
        uint32_t count_before = sum_so_far(count);
        double mass_before = sum_so_far(mass);
        if (lane == 63) { lds.part_count[wv] = count_before; lds.part_sum[wv] = mass_before; }
        count_before -= count;
        {
            const double m = __shfl_up(mass_before, 1);
            mass_before = lane ? m : 0.0;
        }
        __syncthreads();
        double all_mass = 0;
        uint32_t all_count = 0;
#pragma unroll 4
        for (int s = 0; s < kSampleWaves; ++s) {
            if (s == wv) { count_before += all_count; mass_before += all_mass; }
            all_count += lds.part_count[s];
            all_mass += lds.part_sum[s];
        }
        int first = kBins, last = -1;                  // the bins in the list
        const auto collect = [&](int from, int to) {
            first = from;
            last = to;
            __syncthreads();
            if (tid == 0) { list.in_list = 0; list.in_sifted = 0; list.least_key = ~0u; list.most_key = 0; }
            __syncthreads();
            // Bins are the whole parts of bin.place, so comparing that does without rounding down.  First sixteen bytes at a time: those that hold
            // anything within half the width of the middle (multiples of 1/2 below 2^23: the difference may be rounded to half, not past it) are kept; then those one by one.  (Atomics on one address go one after the
            // other: a wavefront reserves its places at once.)
            const float low = (float)(top - to), high = (float)(top - from + 1), middle = 0.5f * (low + high), half = 0.5f * (high - low);
            const auto look = [&](U4 raw, int c) {
                typename T::raw some[kPer];
                __builtin_memcpy(some, &raw, 16);
                float near = INFINITY;
#pragma unroll
                for (int e = 0; e < kPer; ++e) near = fminf(near, __builtin_fabsf(bin.place(to_float<T>(some[e])) - middle));
                const U64 found = __ballot(near <= half);
                if (!found) return;
                uint32_t at = 0;
                if (lane == 0) at = atomicAdd(&list.in_sifted, (uint32_t)__builtin_popcountll(found));
                at = (uint32_t)__builtin_amdgcn_readfirstlane((int)at) + (uint32_t)__popcll(found & ((1ull << lane) - 1));
                if (near <= half && at < (uint32_t)kList) {
                    list.sifted[at] = raw;
                    list.sifted_at[at] = (uint32_t)c;
                }
            };
            const int wave_at = kPer * (tid & ~63);
            constexpr int kStep = kPer * kSampleThreads;
            U4 now[kHeld], next[kHeld];
#pragma unroll
            for (int u = 0; u < kHeld; ++u) now[u] = held[u];
#pragma unroll 1
            for (int at = 0; wave_at + at < n; at += kHeld * kStep) {
#pragma unroll
                for (int u = 0; u < kHeld; ++u) next[u] = some_logits(kPer * tid + at + (kHeld + u) * kStep);
#pragma unroll
                for (int u = 0; u < kHeld; ++u)
                    if (wave_at + at + u * kStep < n) look(now[u], kPer * tid + at + u * kStep);
#pragma unroll
                for (int u = 0; u < kHeld; ++u) now[u] = next[u];
            }
            __syncthreads();
            uint32_t least_key = ~0u, most_key = 0;
            const int sifted = (int)min(list.in_sifted, (uint32_t)kList);
            for (int i0 = tid & ~63; i0 < sifted; i0 += kSampleThreads) {
                const int i = i0 + lane;
                const U4 raw = i < sifted ? list.sifted[i] : U4{0, 0, 0, 0};
                const int first_at = i < sifted ? (int)list.sifted_at[i] : n, token = place_of(first_at);
                typename T::raw some[kPer];
                __builtin_memcpy(some, &raw, 16);
                uint32_t in_bins = 0;
#pragma unroll
                for (int e = 0; e < kPer; ++e) {
                    const float scaled = bin.place(to_float<T>(some[e]));
                    // (the row's last sixteen bytes may hold logits that other ones hold too)
                    in_bins |= (uint32_t)(scaled >= low && scaled < high && token + e >= first_at) << e;
                }
                const uint32_t mine = (uint32_t)__popc(in_bins), until = sum_so_far(mine), all = of_last(until);
                if (!all) continue;
                uint32_t at = 0;
                if (lane == 0) at = atomicAdd(&list.in_list, all);
                at = (uint32_t)__builtin_amdgcn_readfirstlane((int)at) + until - mine;
#pragma unroll
                for (int e = 0; e < kPer; ++e) {
                    if (!(in_bins >> e & 1)) continue;
                    if (at < (uint32_t)kList) {
                        const uint32_t key = key_of(to_float<T>(some[e]));
                        list.list_key[at] = key;
                        list.list_at[at] = (uint32_t)(token + e);
                        least_key = min(least_key, key);
                        most_key = max(most_key, key);
                    }
                    ++at;
                }
            }
            least_key = wave_min(least_key);
            most_key = wave_max(most_key);
            if (lane == 0 && most_key) {
                atomicMin(&list.least_key, least_key);
                atomicMax(&list.most_key, most_key);
            }
            __syncthreads();
            return list.in_list <= (uint32_t)kList && list.in_sifted <= (uint32_t)kList;
        };
        // First top-k's border, then top-p's, then what min-p leaves: each time the bins that hold a border go into the list, unless they are there.
        int border = kBins, in_front_of = 0;
        double total = all_mass, in_front = 0;
        bool with_ties = false;
#pragma unroll 1
        for (int stage = 0; stage < 3; ++stage) {
            int from, to;
            U64 goal = 0;
            double mass_goal = 0;
            bool find = true;
            if (stage == 0) {
                if (!ask.top_k) continue;
                if (ask.top_k < above) {
                    if ((uint32_t)ask.top_k > all_count) return false;
                    if (count_before < (uint32_t)ask.top_k && (uint32_t)ask.top_k <= count_before + count) {
                        list.border = tid;
                        list.border_before = count_before;
                        list.border_mass = mass_before;
                    }
                    __syncthreads();
                    border = list.border;
                    in_front = ask.weighed ? list.border_mass : 0.0;
                    goal = (U64)(ask.top_k - (ask.weighed ? (int)list.border_before : 0));
                } else {
                    // fewer tokens than top-k asks for: all of them
                    if (ask.weighed) continue;
                    if (all_count != (uint32_t)above) return false;
                    border = kBins - 1;
                    find = false;
                }
                from = ask.weighed ? border : 0;
                to = border;
            } else if (stage == 1) {
                if (!(ask.top_p < 1)) continue;
                mass_goal = fmax((double)ask.top_p * total, 5e-324);
                in_front = 0;
                with_ties = ties > 0;
                if (ask.weighed) {
                    __syncthreads();
                    if (tid == 0) list.border = -1;
                    __syncthreads();
                    // (one atomic per wavefront: on one address they go one after the other, and 500 took some 3 us)
                    const U64 in_front_of_goal = __ballot(tid < kBins && mass > 0 && tid <= border && mass_before < mass_goal);
                    if (in_front_of_goal && lane == 0) atomicMax(&list.border, (tid & ~63) + 63 - __builtin_clzll(in_front_of_goal));
                    __syncthreads();
                    const int at = list.border;
                    if (at < 0) return false;
                    if (tid == at) list.border_mass = mass_before;
                    __syncthreads();
                    in_front = list.border_mass;
                    with_ties = with_ties && at == border;
                    border = at;
                }
                from = ask.weighed ? border : 0;
                to = border;
            } else {
                // Bins in front of `from` stay as a whole, bins behind `to` go; what is between is in the list.
                from = ask.weighed ? border : 0;
                to = border;
                if (ask.weighed && ask.min_p > 0) {
                    const double at = (double)top - __builtin_floor(((double)most + log((double)ask.min_p) / (slope / kLog2e)) * (double)bin.scale);
                    const int cut = at < 2.0 * kBins ? (int)at : 2 * kBins;
                    from = max(min(border, cut - 1), 0);
                    to = min(border, cut + 1);
                }
                if (from >= kBins) {                   // nothing goes but what weighs nothing
                    if (ask.min_p > 0) return false;   // (a border that lies below the bins)
                    for (int s = tid; s < slices; s += kSampleThreads) list.tied[s] = 0;
                    return true;
                }
                to = min(to, kBins - 1);
                in_front_of = from;
            }
            if ((first != from || last != to) && !collect(from, to)) return false;
            if (stage == 2) break;
            // weights in the list are relative to its largest, which weighs `unit` multiples in the row
            const Weights weight(value_of(list.most_key), slope, kSliceBits);
            const double unit = of_row.exact(weight.most) * __builtin_ldexp(1.0, -kSliceBits);
            if (find) {
                if (stage == 1) {
                    const double whole_goal = __builtin_ceil((mass_goal - in_front) / unit);
                    goal = whole_goal > 0 ? (whole_goal < 9e18 ? (U64)whole_goal : ~0ull >> 1) : 0;
                }
                const uint32_t differ = list.least_key ^ list.most_key;
                const int shift = max(differ ? (31 - __builtin_clz(differ)) & ~7 : 0, kLastShift<T>);
                uint32_t found_ties = with_ties ? ties : 0;
                find_border<T>(list.digits, [&](auto f) {
                    for (uint32_t i = tid; i < list.in_list; i += kSampleThreads) f(list.list_key[i]);
                }, weight, stage == 1, goal, shift, shift == 24 ? 0u : list.most_key & (~0u << (shift + 8)), bound, found_ties);
                ties = found_ties;
            }
            if (stage == 0 && ask.top_p < 1) {
                U64 sum = 0;
                for (uint32_t i = tid; i < list.in_list; i += kSampleThreads)
                    if (list.list_key[i] > bound) sum += weight(value_of(list.list_key[i]));
                sum = wave_sum(sum);
                __syncthreads();
                if (lane == 0) lds.part_mass[wv] = sum;
                __syncthreads();
                sum = ties * weight(value_of(bound));
#pragma unroll 4
                for (int s = 0; s < kSampleWaves; ++s) sum += lds.part_mass[s];
                total = in_front + (double)sum * unit;
            }
        }
        if (ask.min_p > 0) {
            // The least key in the list that weighs enough (above it all do) is what min-p makes of the bound; if there is none, one that no logit has.
            uint32_t least_key = ~0u;
            for (uint32_t i = tid; i < list.in_list; i += kSampleThreads)
                if (list.list_key[i] >= bound && of_row.exact(value_of(list.list_key[i])) >= (double)ask.min_p) least_key = min(least_key, list.list_key[i]);
            least_key = wave_min(least_key);
            __syncthreads();
            if (lane == 0) lds.part_key[wv] = least_key;
            __syncthreads();
#pragma unroll 4
            for (int s = 0; s < kSampleWaves; ++s) least_key = min(least_key, lds.part_key[s]);
            if (least_key == ~0u) least_key = list.in_list ? list.most_key + 1 : key_of(((float)(top - first) + 0.5f) / bin.scale);
            if (least_key > bound) {
                bound = least_key - 1;
                ties = 0;
            }
        }
        __syncthreads();
        for (int s = tid; s < slices; s += kSampleThreads) { lds.kept[s] = 0; list.tied[s] = 0; }
        __syncthreads();
        for (int s = wv; s < slices && in_front_of > 0; s += kSampleWaves) {
            const int end = in_front_of - (top - lds.top[s]);
            U64 sum = 0;
            if (lds.most[s] > -INFINITY) {
                U64 masses[kBins / kWave];
#pragma unroll
                for (int u = 0; u < kBins / kWave; ++u) masses[u] = lane + u * kWave < end ? bins[s].mass[lane + u * kWave] : 0;
#pragma unroll
                for (int u = 0; u < kBins / kWave; ++u) sum += masses[u];
            }
            sum = wave_sum(sum);
            if (lane == 0) lds.kept[s] = sum;
        }
        __syncthreads();
        for (uint32_t i = tid; i < list.in_list; i += kSampleThreads) {
            const uint32_t key = list.list_key[i];
            const int s = (int)(list.list_at[i] / kSlice);
            if (key == bound) atomicAdd(&list.tied[s], 1u);
            else if (key > bound) atomicAdd(&lds.kept[s], (U64)Weights(lds.most[s], slope, kSliceBits)(value_of(key)));
        }
        __syncthreads();
        if (ties && wv == 0) {
            uint32_t seen = 0;
            for (int s0 = 0; s0 < slices && seen < ties; s0 += kWave) {
                const int s = s0 + lane;
                const uint32_t here = s < slices ? list.tied[s] : 0, until = seen + sum_so_far(here);
                if (here && until - here < ties) lds.kept[s] += min(here, ties - (until - here)) * Weights(lds.most[s], slope, kSliceBits)(value_of(bound));
                seen = of_last(until);
            }
        }
        __syncthreads();
        return true;
    }
};

// PIECES: the row is one piece, always (0), or if its slices do not tell enough (2), or never (1: a row without filters).
template <class T, int PIECES>
__global__ void __launch_bounds__(kSampleThreads, PIECES == 1 ? 8 : 4) sample_rows_kernel(SampleParams p) {
    __shared__ SampleLds lds;
    __shared__ typename std::conditional<PIECES != 1, FilterLds, NoLds>::type list;
    SampleRow<T, PIECES != 1> row(p, lds, list);
    if (PIECES != 0 && (row.from_slices() || PIECES == 1)) return;
    __syncthreads();
    row.whole();
}

}  // namespace bpe

using namespace bpe;

static int sample_sizes_ok(int64_t rows, int64_t n_vocab) {
    if (rows < 0 || rows >= (1ll << 31) || n_vocab < 1 || n_vocab >= (1 << 30)) {
        set_error("bpe_sample_tokens: sizes out of range (rows %lld, n_vocab %lld)", (long long)rows, (long long)n_vocab);
        return 0;
    }
    return 1;
}

// Slices of a row, 0 where it is taken as one piece; and the rows of a launch.
static int64_t sample_slices(int64_t n_vocab) {
    const int64_t slices = (n_vocab + kSlice - 1) / kSlice;
    return slices > 1 && slices <= kMostSlices ? slices : 0;
}
static int64_t sample_rows_at_once(int64_t rows, int64_t slices) { return slices ? std::min(rows, std::max<int64_t>(kSlicesAtOnce / slices, 1)) : std::min(rows, kMaxThreads / kSampleThreads - 1); }
static int64_t sample_need(int64_t rows, int64_t n_vocab) {
    const int64_t slices = sample_slices(n_vocab);
    return sample_rows_at_once(rows, slices) * slices * (int64_t)(sizeof(SlicePart) + sizeof(SliceBins));
}

extern "C" int64_t bpe_sample_tokens_workspace_bytes(int64_t rows, int64_t n_vocab) {
    return sample_sizes_ok(rows, n_vocab) ? sample_need(rows, n_vocab) : BPE_ERR_SIZE;
}

template <class T> static int launch_sample(SampleParams &p, int64_t rows, void *stream) {
    const char *what = "bpe_sample_tokens launch";
    const int64_t at_once = sample_rows_at_once(rows, p.slices);
    const bool filters = p.top_k || p.top_p || p.min_p;
    for (int64_t done = 0; done < rows; done += at_once) {
        const int64_t now = std::min(rows - done, at_once);
        p.row0 = (int32_t)done;
        if (p.slices) {
            const int rc = launch(filters ? sample_slices_kernel<T, true> : sample_slices_kernel<T, false>, dim3((unsigned)(now * p.slices)), kSliceThreads, p, stream, what);
            if (rc != BPE_OK) return rc;
        }
        const int rc = launch(!p.slices ? sample_rows_kernel<T, 0> : filters ? sample_rows_kernel<T, 2> : sample_rows_kernel<T, 1>, dim3((unsigned)now), kSampleThreads, p, stream, what);
        if (rc != BPE_OK) return rc;
    }
    return BPE_OK;
}

extern "C" int bpe_sample_tokens(const void *logits, int64_t logits_stride, int dtype, int64_t rows, int64_t n_vocab, const float *uniform,
                                 const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p, int32_t *ids,
                                 float *logprobs, void *workspace, int64_t workspace_bytes, void *stream) {
    if (!sample_sizes_ok(rows, n_vocab)) return BPE_ERR_SIZE;
    if (!dtype_ok(dtype)) { set_error("bpe_sample_tokens: dtype %d", dtype); return BPE_ERR_OPTION; }
    if (rows == 0) return BPE_OK;
    if (!logits || !uniform || !ids) { set_error("null pointer"); return BPE_ERR_NULL; }
    if (rows > 1 && logits_stride < n_vocab) { set_error("bpe_sample_tokens: a stride is shorter than a row"); return BPE_ERR_SIZE; }
    if (((uintptr_t)logits & (dtype_bytes(dtype) - 1)) ||
        (((uintptr_t)uniform | (uintptr_t)temperature | (uintptr_t)top_k | (uintptr_t)top_p | (uintptr_t)min_p | (uintptr_t)ids | (uintptr_t)logprobs) & 3)) {
        set_error("bpe_sample_tokens: a pointer is not aligned to its type");
        return BPE_ERR_SIZE;
    }
    const int64_t need = sample_need(rows, n_vocab);
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need)) {
        set_error("workspace must be 256-byte aligned and hold %lld bytes (got %lld)", (long long)need, (long long)workspace_bytes);
        return BPE_ERR_WORKSPACE;
    }
    SampleParams p = {};
    p.logits = logits; p.stride = logits_stride; p.n_vocab = (int32_t)n_vocab;
    p.slices = (int32_t)sample_slices(n_vocab);
    p.bins = (SliceBins *)workspace;
    p.parts = (SlicePart *)(p.bins + sample_rows_at_once(rows, p.slices) * p.slices);
    p.bits = 50;
    while (p.bits > 0 && (n_vocab >> (61 - p.bits))) --p.bits;         // all weights together stay below 2^62
    p.uniform = uniform; p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p; p.ids = ids; p.logprobs = logprobs;
    return dtype == BPE_F32 ? launch_sample<F32>(p, rows, stream) : dtype == BPE_BF16 ? launch_sample<Bf16>(p, rows, stream) : launch_sample<F16>(p, rows, stream);
}
