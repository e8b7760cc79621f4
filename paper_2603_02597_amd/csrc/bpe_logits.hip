// Logits under the rules of a request (bpe_adjust_logits) and the best tokens of every row (bpe_top_tokens).
#include <algorithm>

#include "bpe_lookback.h"
#include "bpe_numeric.h"

namespace bpe {

struct AdjustParams {
    const void *logits;
    void *out;
    int64_t logits_stride, out_stride;
    int32_t row0, n_vocab;             // the launch's first row
    int32_t slice, slices;             // tokens of a row per workgroup, a multiple of 32
    bpe_logit_rules rules;
};

// Elements [begin, end) of a list that the rows share, clamped to the list.
__device__ __forceinline__ void row_range(const int32_t *offsets, int64_t n, int row, int &begin, int &end) {
    begin = end = 0;
    if (!offsets) return;
    begin = min(max(offsets[row], 0), (int)n);
    end = min(max(offsets[row + 1], begin), (int)n);
}

// The row's mask, or nullptr; `nothing` if its index is too large.
__device__ __forceinline__ const uint32_t *row_mask(const bpe_logit_rules &r, int row, bool &nothing) {
    nothing = false;
    if (!r.masks) return nullptr;
    const int64_t i = r.mask_index ? r.mask_index[row] : row;
    if (i < 0) return nullptr;
    nothing = i >= r.n_masks;
    return nothing ? nullptr : r.masks + i * r.mask_stride;
}

// A workgroup takes a slice of a row.  With LISTS it first counts the row's history in LDS and marks the biased tokens, then makes one
// pass over the slice, sixteen bytes per lane; the biased tokens, which that pass leaves out, come last.  Every slice of a row
// reads the row's whole history: slices are as long as LDS allows with two workgroups per compute unit.  Every operation is rounded by
// itself (no fused multiply-add), so the result is the formula's to the bit.  Bound by memory for many rows (512 x 100257 f32 with
// lists of 30,000 108 us: 411 MB of logits at 3.8 TB/s, and every list read seven times), by the chain of list, count and pass for few:
// 64 x 100256 bf16 with lists of 8,000 12 us, one row 4 us.
constexpr int kAdjustThreads = 1024, kAdjustSlice = 16384;
constexpr uint32_t kBiased = 0x80000000u;             // in a count
template <class IN, class OUT, bool LISTS>
__global__ void __launch_bounds__(kAdjustThreads) adjust_kernel(AdjustParams p) {
#pragma clang fp contract(off)
    constexpr int kPer = 16 / (int)sizeof(typename IN::raw);
    typedef typename IN::raw InVec __attribute__((ext_vector_type(kPer), aligned(sizeof(typename IN::raw))));
    typedef typename OUT::raw OutVec __attribute__((ext_vector_type(kPer), aligned(sizeof(typename OUT::raw))));
    typedef int32_t Int4Any __attribute__((ext_vector_type(4), aligned(4)));
    typedef uint32_t Counts __attribute__((ext_vector_type(kPer)));
    __shared__ __attribute__((aligned(32))) uint32_t count[LISTS ? kAdjustSlice : 1];
    const bpe_logit_rules &r = p.rules;
    const int row = p.row0 + blockIdx.x / p.slices, first = blockIdx.x % p.slices * p.slice, last = min(first + p.slice, p.n_vocab), tid = threadIdx.x;
    const typename IN::raw *in = (const typename IN::raw *)p.logits + row * p.logits_stride;
    typename OUT::raw *out = (typename OUT::raw *)p.out + row * p.out_stride;
    int bias_begin = 0, bias_end = 0;
    float rep = 1.0f, freq = 0.0f, pres = 0.0f;
    auto punished = [&](float x, uint32_t c) {
        x = x > 0.0f ? x / rep : x * rep;
        x = x - freq * (float)c;
        return x - pres;
    };
    if constexpr (LISTS) {
        for (int i = 4 * tid; i < p.slice; i += 4 * kAdjustThreads) *(U4 *)(count + i) = U4{0, 0, 0, 0};
        rep = r.repetition ? r.repetition[row] : 1.0f;
        freq = r.frequency ? r.frequency[row] : 0.0f;
        pres = r.presence ? r.presence[row] : 0.0f;
        int begin, end;
        row_range(r.history_offsets, r.n_history, row, begin, end);
        row_range(r.bias_offsets, r.n_bias, row, bias_begin, bias_end);
        __syncthreads();
        auto note = [&](int v) {
            if (v >= first && v < last) atomicAdd(&count[v - first], 1u);
        };
        // (places within the row's list are unsigned, so that they pass its end without a wrap however long all the lists are)
        const int32_t *history = r.history + begin;
        const uint32_t length = (uint32_t)(end - begin);
        uint32_t i = 4 * tid;
        for (; i + (12 * kAdjustThreads + 4) <= length; i += 16 * kAdjustThreads) {
            Int4Any v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = *(const Int4Any *)(history + i + q * 4 * kAdjustThreads);
#pragma unroll
            for (int q = 0; q < 4; ++q) { note(v[q][0]); note(v[q][1]); note(v[q][2]); note(v[q][3]); }
        }
        for (; i + 4 <= length; i += 4 * kAdjustThreads) {
            const Int4Any v = *(const Int4Any *)(history + i);
            note(v[0]); note(v[1]); note(v[2]); note(v[3]);
        }
        for (; i < length; ++i) note(history[i]);          // (one thread's: the last one to three)
        for (uint32_t i = tid; i < (uint32_t)(bias_end - bias_begin); i += kAdjustThreads) {
            const int v = r.bias_ids[(int64_t)bias_begin + i];
            if (v >= first && v < last) atomicOr(&count[v - first], kBiased);
        }
        __syncthreads();
    }
    bool nothing;
    const uint32_t *mask = row_mask(r, row, nothing);
    for (int v = first + kPer * tid; v < last; v += kPer * kAdjustThreads) {
        const bool whole = v + kPer <= last;
        InVec t;
        if (whole) {
            t = *(const InVec *)(in + v);
        } else {
#pragma unroll
            for (int e = 0; e < kPer; ++e) t[e] = v + e < last ? in[v + e] : typename IN::raw(0);
        }
        uint32_t allowed = nothing ? 0u : ~0u, biased = 0;
        if (mask) allowed = mask[v >> 5] >> (v & 31);
        float x[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) x[e] = to_float<IN>(t[e]);
        if constexpr (LISTS) {
            const Counts c = *(const Counts *)(count + (v - first));
            uint32_t any = 0;
#pragma unroll
            for (int e = 0; e < kPer; ++e) any |= c[e];
            if (any) {
#pragma unroll
                for (int e = 0; e < kPer; ++e) {
                    if (c[e] & ~kBiased) x[e] = punished(x[e], c[e]);
                    biased |= c[e] >> 31 << e;
                }
            }
        }
        OutVec o;
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[e] = from_float<OUT>(allowed >> e & 1u ? x[e] : -__builtin_inff());
        if (whole && !biased) {
            *(OutVec *)(out + v) = o;
        } else {
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                if (v + e < last && !(biased >> e & 1u)) out[v + e] = o[e];
        }
    }
    if constexpr (LISTS) {
        // The biased tokens, the list from its end: an entry whose token is still marked counts, of several of one token among those
        // at hand the last one.  (A marked token's logit has not been written yet, also in place.)
        for (int back = bias_end; back > bias_begin; back -= kAdjustThreads) {
            __syncthreads();
            const int i = back - 1 - tid;
            int v = -1;
            uint32_t c = 0;
            if (i >= bias_begin) {
                v = r.bias_ids[i];
                v = v >= first && v < last ? v - first : -1;
                if (v >= 0) c = count[v];
                if (!(c & kBiased)) v = -1;
            }
            __syncthreads();
            if (v >= 0) count[v] = 0;
            __syncthreads();
            if (v >= 0) atomicMax(&count[v], (uint32_t)(kAdjustThreads - tid));
            __syncthreads();
            const bool mine = v >= 0 && count[v] == (uint32_t)(kAdjustThreads - tid);
            __syncthreads();
            if (mine) {
                c &= ~kBiased;
                count[v] = c;
                float x = to_float<IN>(in[first + v]);
                if (c) x = punished(x, c);
                x = x + r.bias_values[i];
                const bool keep = mask ? (mask[(first + v) >> 5] >> ((first + v) & 31)) & 1u : !nothing;
                out[first + v] = from_float<OUT>(keep ? x : -__builtin_inff());
            }
        }
    }
}

// ---------------------------------------------------------------------------
// The best tokens of a row, in one pass over it.  A workgroup goes through its part of a row and keeps, in LDS, every logit that
// may still be among the k best: those not below a bound that at least k logits reach.  The bound is cheap: the k-th largest of the
// threads' largest logits so far.  (Of 8,192 random logits it lets 73 through for k = 64, of later ones fewer and fewer.)  What was
// kept is cut down to the k best by histograms over the range of what is left, and put in order by counting.  Logits are compared as
// (value, index from behind) in one 64-bit word, so no two are equal and the order in which lanes append does not matter.  The sum of
// exp(logit - largest so far) goes along in 32 bits, rescaled when the largest grows.
// Bound by memory for many rows of f32 (1024 x 50257, k = 20: 44 us, 4.7 TB/s), by the comparisons and exponentials for 16-bit logits
// (2.6 TB/s), by two launches and their chains of barriers for few: one row of 50256 in parts k = 1 9 us, k = 64 10.8; 64 rows of
// 100256 bf16 k = 64 16 us, k = 256 34.
constexpr int kTopThreads = 256, kTopWaves = kTopThreads / kWave;
constexpr int kTopKeep = 4096;               // words in LDS: four workgroups per compute unit
constexpr int kTopPerThread = 32;            // logits of a thread that are at hand together
constexpr int kTopBins = 1024;
constexpr int kTopRank = 256;                // up to so many words are put in order by counting
constexpr int kMaxTop = 256;
constexpr float kLowest = -3.402823466e38f;       // of the finite floats
constexpr float kLog2E = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// What a part leaves: its largest logit, the sum of exp(logit - largest), a bound that k of its words reach, the number of its words.
struct TopPart { float largest, sum, bound; int32_t words; };

struct TopParams {
    const void *logits;
    int64_t logits_stride;
    int32_t row0, n_vocab, k;                // the launch's first row
    int32_t parts, part_len, part_keep;      // a row is cut into so many parts of part_len logits, each leaves up to part_keep words
    int32_t *ids;
    float *logprobs, *lse;
    uint64_t *kept;                          // [rows][parts][part_keep] words of a part, among them its k best
    struct TopPart *left;                    // [rows][parts]
};

// Floats as unsigned numbers in the same order; both zeros are one value, every NaN the largest.
__device__ __forceinline__ uint32_t order_key(float x) {
    if (x != x) return 0xFFFFFFFFu;
    const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t key) {
    return key == 0xFFFFFFFFu ? __builtin_nanf("") : __builtin_bit_cast(float, key & 0x80000000u ? key ^ 0x80000000u : ~key);
}
__device__ __forceinline__ uint64_t top_word(float x, int v) { return (uint64_t)order_key(x) << 32 | ~(uint32_t)v; }

struct TopShared {
    uint64_t word[kTopKeep];
    uint32_t bin[kTopBins];                  // (also the threads' largest logits)
    uint64_t few[kTopRank];
    float wave_value[kTopWaves];
    float2 wave_sum[kTopWaves];
    uint64_t low, high;
    int n, n_few, above;
};

// A bound that at least k of the `count` words reach and at most kTopRank: a histogram over [low, high], then over the range of the
// bin that the k-th word is in, and so on (each a 1,024th of the one before, so there are at most seven).  No word is above `high`; of
// those from `low` on there are at least k, or else the bound is `low`.
__device__ __forceinline__ uint64_t bound_of_best(TopShared &sh, int count, int k, uint64_t low, uint64_t high) {
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    if (count <= kTopRank) return 0;
    int above = 0;                            // words above `high`: fewer than k
    __syncthreads();                          // the bins may hold the threads' largest logits, which somebody still reads
    for (;;) {
        const int shift = max(0, 54 - __builtin_clzll((high - low) | 1));        // (high - low) >> shift < kTopBins
        for (int i = tid; i < kTopBins; i += kTopThreads) sh.bin[i] = 0;
        __syncthreads();
        for (int i = tid; i < count; i += kTopThreads) {
            const uint64_t w = sh.word[i];
            if (w >= low && w <= high) atomicAdd(&sh.bin[(w - low) >> shift], 1u);
        }
        __syncthreads();
        if (wv == 0) {
            if (lane == 0) sh.n_few = 0;      // (unless a lane finds the k-th word below)
            // a lane takes 16 bins, the highest ones first: words in the bins of the lanes before it, then in its own
            constexpr int kPer = kTopBins / kWave;
            uint32_t in[kPer], mine = 0;
#pragma unroll
            for (int q = 0; q < kPer; ++q) mine += in[q] = sh.bin[kTopBins - 1 - (lane * kPer + q)];
            uint32_t before = wave_scan_inclusive((int)mine) + above - mine;
            if (before < (uint32_t)k && before + mine >= (uint32_t)k) {          // one lane: the k-th word is in one of its bins
                int bin = 0;
                uint32_t there = 0;
                bool found = false;
#pragma unroll
                for (int q = 0; q < kPer; ++q) {
                    if (!found && before + in[q] >= (uint32_t)k) {
                        found = true;
                        bin = kTopBins - 1 - (lane * kPer + q);
                        there = in[q];
                    }
                    if (!found) before += in[q];
                }
                sh.low = low + ((uint64_t)bin << shift);
                const uint64_t width = ((uint64_t)1 << shift) - 1;                // (low + width may pass 64 bits)
                sh.high = high - sh.low < width ? high : sh.low + width;
                sh.above = (int)before;
                sh.n_few = (int)(before + there);
            }
        }
        __syncthreads();
        if (sh.n_few == 0) return low;
        low = sh.low;
        high = sh.high;
        above = sh.above;
        if (sh.n_few <= kTopRank) return low;
        __syncthreads();
    }
}

// The k best of the `count` words, best first, to place(rank, word); returns how many there are.  low, high: see bound_of_best.
template <class Place>
__device__ __forceinline__ int place_best(TopShared &sh, int count, int k, uint64_t low, uint64_t high, Place place) {
    const int tid = threadIdx.x;
    const uint64_t bound = bound_of_best(sh, count, k, low, high);
    __syncthreads();
    if (tid == 0) sh.n_few = 0;
    sh.few[tid] = 0;
    __syncthreads();
    for (int i = tid; i < count; i += kTopThreads) {
        const uint64_t w = sh.word[i];
        if (w >= bound) sh.few[atomicAdd(&sh.n_few, 1)] = w;
    }
    __syncthreads();
    // Several threads to a word count how many of a part of the words are larger.
    const int n = sh.n_few, slots = n <= 32 ? 32 : n <= 64 ? 64 : n <= 128 ? 128 : 256, per = kTopThreads / slots;
    const uint64_t w = sh.few[tid / per];
    typedef uint64_t Words __attribute__((ext_vector_type(2)));
    const Words *others = (const Words *)sh.few + tid % per * (slots / per / 2);
    int rank = 0;
#pragma unroll 8
    for (int o = 0; o < slots / per / 2; ++o) {
        const Words v = others[o];
        rank += (v[0] > w) + (v[1] > w);
    }
    for (int d = 1; d < per; d <<= 1) rank += __shfl_xor(rank, d);
    if (tid % per == 0 && w && rank < k) place(rank, w);
    return min(n, k);
}
static_assert(kTopRank == kTopThreads, "a thread per word");

template <int CTRL> __device__ __forceinline__ float dpp(float v) {
    const int u = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(u, u, CTRL, 0xF, 0xF, false));
}
// The value of the lane whose index differs in bit DISTANCE, or of another one of its group of DISTANCE lanes, which are all alike here.
template <int DISTANCE> __device__ __forceinline__ float other_group(float v) {
    if constexpr (DISTANCE == 1) return dpp<0xB1>(v);         // quad_perm 1 0 3 2
    else if constexpr (DISTANCE == 2) return dpp<0x4E>(v);    // quad_perm 2 3 0 1
    else if constexpr (DISTANCE == 4) return dpp<0x141>(v);   // row_half_mirror
    else if constexpr (DISTANCE == 8) return dpp<0x140>(v);   // row_mirror
    else return __shfl_xor(v, DISTANCE);
}
template <int DISTANCE, class Op> __device__ __forceinline__ float join_groups(float v, Op op) { return op(v, other_group<DISTANCE>(v)); }
template <class Op> __device__ __forceinline__ float wave_join(float v, Op op) {
    v = join_groups<1>(v, op);
    v = join_groups<2>(v, op);
    v = join_groups<4>(v, op);
    v = join_groups<8>(v, op);
    v = join_groups<16>(v, op);
    return join_groups<32>(v, op);
}

// A bound that k of the largest logits of the threads' halves reach: the k-th largest of them (for k <= 128 of the threads' largest),
// cut to the upper 16 bits of its place in the order.  Every wavefront looks at all of them, four or eight per lane, and finds the
// bound bit by bit.  (k = 256 from the threads' largest alone: their smallest is the bound, and 5 to 6 times k words pass.)
template <int PER> __device__ __forceinline__ uint32_t kth_largest(const uint32_t *keys, int k) {
    U4 key[PER];
#pragma unroll
    for (int h = 0; h < PER; ++h) key[h] = ((const U4 *)keys)[h * kWave + (threadIdx.x & 63)];
    uint32_t bound = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t at = bound | 1u << bit;
        int reach = 0;
#pragma unroll
        for (int h = 0; h < PER; ++h)
#pragma unroll
            for (int q = 0; q < 4; ++q) reach += __builtin_popcountll(__ballot(key[h][q] >= at));
        bound = reach >= k ? at : bound;
    }
    return bound;
}
__device__ __forceinline__ float bound_of_threads(TopShared &sh, float largest0, float largest1, int k) {
    static_assert(kTopThreads == 4 * kWave && kTopBins >= 2 * kTopThreads && kMaxTop <= kTopThreads, "");
    uint32_t bound;
    if (k <= kTopThreads / 2) {
        sh.bin[threadIdx.x] = order_key(fmaxf(largest0, largest1));
        __syncthreads();
        bound = kth_largest<1>(sh.bin, k);
    } else {
        sh.bin[threadIdx.x] = order_key(largest0);
        sh.bin[kTopThreads + threadIdx.x] = order_key(largest1);
        __syncthreads();
        bound = kth_largest<2>(sh.bin, k);
    }
    return bound > order_key(-__builtin_inff()) ? key_value(bound) : kLowest;
}

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2E); }
// What exp(x - largest) is taken against: a row of -infinity has no other.
__device__ __forceinline__ float reference_of(float largest) { return largest == -__builtin_inff() ? 0.0f : largest; }

// {largest, sum} of the whole workgroup, in a fixed order.
__device__ __forceinline__ float2 join_sums(TopShared &sh, float largest, float sum) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const float m = wave_join(largest, [](float a, float b) { return fmaxf(a, b); });
    sum = wave_join(sum * exp_of(largest - reference_of(m)), [](float a, float b) { return a + b; });
    if (lane == 0) sh.wave_sum[wv] = make_float2(m, sum);
    __syncthreads();
    float all = -__builtin_inff(), s = 0.0f;
#pragma unroll
    for (int w = 0; w < kTopWaves; ++w) all = fmaxf(all, sh.wave_sum[w].x);
#pragma unroll
    for (int w = 0; w < kTopWaves; ++w) s += sh.wave_sum[w].y * exp_of(sh.wave_sum[w].x - reference_of(all));
    return make_float2(all, s);
}

// log of the sum: NaN if the best logit is one, +infinity if that is; `best`: the word of the best one, 0 if there is none.
__device__ __forceinline__ float log_sum(float2 total, uint64_t best) {
    const float x = best ? key_value((uint32_t)(best >> 32)) : -__builtin_inff();
    if (x != x || x == __builtin_inff() || x == -__builtin_inff()) return x;
    return total.x + __builtin_amdgcn_logf(total.y) * kLn2;
}

// Words from that of a logit on, and up to it; a sum that is NaN leaves open what the largest is.
__device__ __forceinline__ uint64_t words_from(float x) { return (uint64_t)order_key(x) << 32; }
__device__ __forceinline__ uint64_t words_to(float2 total) { return total.y != total.y ? ~0ull : words_from(total.x) | 0xFFFFFFFFu; }

__device__ __forceinline__ void write_row(const TopParams &p, TopShared &sh, int row, int count, uint64_t low, float2 total) {
    const int tid = threadIdx.x;
    const int n = place_best(sh, count, p.k, low, words_to(total), [&](int rank, uint64_t w) {
        sh.word[rank] = w;                                // (every word that is still needed is in sh.few)
    });
    __syncthreads();
    const float lse = log_sum(total, n ? sh.word[0] : 0);
    if (p.lse && tid == 0) p.lse[row] = lse;
    for (int j = tid; j < p.k; j += kTopThreads) {
        const uint64_t w = j < n ? sh.word[j] : 0;
        const float x = key_value((uint32_t)(w >> 32));
        p.ids[(int64_t)row * p.k + j] = j < n ? (int)~(uint32_t)w : -1;
        p.logprobs[(int64_t)row * p.k + j] = j < n ? x - lse : -__builtin_inff();
    }
}

template <class IN>
__global__ void __launch_bounds__(kTopThreads, 4) top_part_kernel(TopParams p) {
    constexpr int kPer = 16 / (int)sizeof(typename IN::raw), kTopVectors = kTopPerThread / kPer, kRound = kTopThreads * kTopPerThread;
    typedef typename IN::raw Vec __attribute__((ext_vector_type(kPer), aligned(sizeof(typename IN::raw))));
    __shared__ __attribute__((aligned(16))) TopShared sh;
    const int tid = threadIdx.x, lane = tid & 63;
    const int row = p.row0 + blockIdx.x / p.parts, part = blockIdx.x % p.parts;
    const int first = part * p.part_len, last = min(first + p.part_len, p.n_vocab);
    const typename IN::raw *in = (const typename IN::raw *)p.logits + row * p.logits_stride;
    if (tid == 0) sh.n = 0;
    float largest = -__builtin_inff(), sum = 0.0f, half[2] = {largest, largest};       // half: of every second vector
    float bound = kLowest;                                // logits below it are out; so is -infinity
    uint64_t bound_word = 0;                              // and words that are not above this one
    int before = 0, n_rounds = 0;
    for (int at = first; at < last; at += kRound, ++n_rounds) {
        float x[kTopVectors][kPer];
#pragma unroll
        for (int q = 0; q < kTopVectors; ++q) {
            const int v = at + (q * kTopThreads + tid) * kPer;
            if (v + kPer <= last) {
                const Vec t = *(const Vec *)(in + v);
#pragma unroll
                for (int e = 0; e < kPer; ++e) x[q][e] = to_float<IN>(t[e]);
            } else {
#pragma unroll
                for (int e = 0; e < kPer; ++e) x[q][e] = -__builtin_inff();
                if (v < last) {                           // one thread of a row at most
#pragma unroll
                    for (int e = 0; e < kPer; ++e)
                        if (v + e < last) x[q][e] = to_float<IN>(in[v + e]);
                }
            }
        }
#pragma unroll
        for (int q = 0; q < kTopVectors; ++q)
#pragma unroll
            for (int e = 0; e < kPer; ++e) half[q & 1] = fmaxf(half[q & 1], x[q][e]);
        const float m = fmaxf(half[0], half[1]);
        const float ref = reference_of(m);
        sum *= exp_of(largest - ref);
#pragma unroll
        for (int q = 0; q < kTopVectors; ++q)
#pragma unroll
            for (int e = 0; e < kPer; ++e) sum += exp_of(x[q][e] - ref);
        largest = m;
        const float bound_before = bound;                 // reached by k of the words that are there
        if ((n_rounds & (n_rounds + 1)) == 0) bound = fmaxf(bound, bound_of_threads(sh, half[0], half[1], p.k));   // rounds 0, 1, 3, 7, ...
        else __syncthreads();
        // A lane's logits that stay, one bit each: few, so they are read again.
        uint32_t stay = 0;
#pragma unroll
        for (int q = 0; q < kTopVectors; ++q)
#pragma unroll
            for (int e = 0; e < kPer; ++e) stay |= x[q][e] < bound ? 0u : 1u << (q * kPer + e);
        auto word_of = [&](int bit) {
            const int v = at + (bit / kPer * kTopThreads + tid) * kPer + bit % kPer;
            return top_word(to_float<IN>(in[v]), v);
        };
        // A wavefront takes room for all of its lanes' at once.  Beyond kTopKeep they are only counted.
        if (__ballot(stay != 0)) {
            const int mine = __builtin_popcount(stay), up_to = wave_scan_inclusive(mine);
            int base = 0;
            if (lane == kWave - 1) base = atomicAdd(&sh.n, up_to);
            int to = up_to - mine + __builtin_amdgcn_readlane(base, kWave - 1);
            for (uint32_t left = stay; left; left &= left - 1, ++to)
                if (to < kTopKeep) sh.word[to] = word_of(__builtin_ctz(left));
        }
        __syncthreads();
        const int n = sh.n;
        if (n <= kTopKeep) { before = n; continue; }
        // More than there is room for: what this round has appended is taken back, the words cut down to the k best, and the
        // round's logits looked at again, one of every thread at a time, with another cut whenever room runs out.
        int count = before;
        auto cut = [&]() {
            const int left = place_best(sh, count, p.k, words_from(bound_before), ~0ull, [&](int rank, uint64_t w) { sh.word[rank] = w; });
            __syncthreads();
            if (left == p.k) bound_word = sh.word[p.k - 1];
            if (tid == 0) sh.n = left;
            __syncthreads();
            count = left;
        };
        cut();
        for (int bit = 0; bit < kTopPerThread; ++bit) {
            if (count > kTopKeep - kTopThreads) cut();
            if (stay >> bit & 1u) {
                const uint64_t w = word_of(bit);
                if (w > bound_word) sh.word[atomicAdd(&sh.n, 1)] = w;
            }
            __syncthreads();
            count = sh.n;
            __syncthreads();
        }
        before = count;
        if (bound_word) bound = fmaxf(bound, key_value((uint32_t)(bound_word >> 32)));
    }
    __syncthreads();
    const float2 total = join_sums(sh, largest, sum);
    if (n_rounds > 1) bound = fmaxf(bound, bound_of_threads(sh, half[0], half[1], p.k));
    if (p.parts == 1) {
        write_row(p, sh, row, before, words_from(bound), total);
        return;
    }
    // The words above the bound go to the workgroup that joins the parts; if they are too many, the k best.
    TopPart &left = p.left[(int64_t)row * p.parts + part];
    uint64_t *out = p.kept + ((int64_t)row * p.parts + part) * p.part_keep;
    const uint64_t low = words_from(bound);
    int n = before;
    if (n_rounds > 1) {                                   // (after one round all words are above the bound)
        if (tid == 0) sh.n_few = 0;
        __syncthreads();
        for (int i = tid; i < before; i += kTopThreads) {
            const uint64_t w = sh.word[i];
            if (w >= low) {
                const int to = atomicAdd(&sh.n_few, 1);
                if (to < p.part_keep) out[to] = w;
            }
        }
        __syncthreads();
        n = sh.n_few;
    } else if (n <= p.part_keep) {
        for (int i = tid; i < n; i += kTopThreads) out[i] = sh.word[i];
    }
    if (n > p.part_keep) {
        __syncthreads();
        n = place_best(sh, before, p.k, low, words_to(total), [&](int rank, uint64_t w) { out[rank] = w; });
    }
    if (tid == 0) left = {total.x, total.y, bound, n};
}

// The best of the parts' best: none is below the highest of the parts' bounds.
__global__ void __launch_bounds__(kTopThreads) top_join_kernel(TopParams p) {
    __shared__ __attribute__((aligned(16))) TopShared sh;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, row = p.row0 + blockIdx.x;
    const TopPart *left = p.left + (int64_t)row * p.parts;
    float bound = kLowest, largest = -__builtin_inff(), sum = 0.0f;
    for (int i = tid; i < p.parts; i += kTopThreads) {
        const TopPart t = left[i];
        const float m = fmaxf(largest, t.largest), ref = reference_of(m);
        sum = sum * exp_of(largest - ref) + t.sum * exp_of(t.largest - ref);
        largest = m;
        bound = fmaxf(bound, t.bound);
    }
    bound = wave_join(bound, [](float a, float b) { return fmaxf(a, b); });
    if (lane == 0) sh.wave_value[wv] = bound;
    if (tid == 0) sh.n = 0;
    const float2 total = join_sums(sh, largest, sum);
#pragma unroll
    for (int w = 0; w < kTopWaves; ++w) bound = fmaxf(bound, sh.wave_value[w]);
    const uint64_t low = words_from(bound);
    const uint64_t *in = p.kept + (int64_t)row * p.parts * p.part_keep;
    // a power of two of threads to every part, eight of its words at a time
    int per = kTopThreads;
    while (per > 1 && per * p.parts > kTopThreads) per /= 2;
    for (int part = tid / per; part < p.parts; part += kTopThreads / per) {
        const int n = left[part].words;
        for (int i = tid % per; i < n; i += 8 * per) {
            uint64_t w[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) w[q] = i + q * per < n ? in[(int64_t)part * p.part_keep + i + q * per] : 0;
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (w[q] >= low && w[q]) sh.word[atomicAdd(&sh.n, 1)] = w[q];
        }
    }
    __syncthreads();
    write_row(p, sh, row, sh.n, low, total);
}

}  // namespace bpe

using namespace bpe;

static bool aligned_to(const void *p, int64_t bytes) { return !((uintptr_t)p & (uintptr_t)(bytes - 1)); }

static int check_rows(const char *what, int64_t rows, int64_t n_vocab, int dtype) {
    if (rows < 0 || rows >= 0x7FFFFFFFll || n_vocab < 1 || n_vocab >= (1 << 30)) {
        set_error("%s: sizes out of range (rows %lld, n_vocab %lld)", what, (long long)rows, (long long)n_vocab);
        return BPE_ERR_SIZE;
    }
    if (!dtype_ok(dtype)) { set_error("%s: dtype %d", what, dtype); return BPE_ERR_OPTION; }
    return BPE_OK;
}

extern "C" int bpe_adjust_logits(const void *logits, int64_t logits_stride, int dtype, int64_t rows, int64_t n_vocab,
                                 const bpe_logit_rules *rules, void *out, int64_t out_stride, int out_dtype, void *stream) {
    const int rc = check_rows("bpe_adjust_logits", rows, n_vocab, dtype);
    if (rc != BPE_OK) return rc;
    if (out_dtype != BPE_F32 && out_dtype != dtype) { set_error("bpe_adjust_logits: out is f32 or of the logits' type (out_dtype %d)", out_dtype); return BPE_ERR_OPTION; }
    if (rows == 0) return BPE_OK;
    if (!logits || !out) { set_error("null pointer"); return BPE_ERR_NULL; }
    if (rows > 1 && (logits_stride < n_vocab || out_stride < n_vocab)) { set_error("bpe_adjust_logits: a stride is shorter than a row"); return BPE_ERR_SIZE; }
    if (!aligned_to(logits, dtype_bytes(dtype)) || !aligned_to(out, dtype_bytes(out_dtype))) {
        set_error("bpe_adjust_logits: a pointer is not aligned to its type");
        return BPE_ERR_SIZE;
    }
    if (logits == out && (dtype != out_dtype || (rows > 1 && logits_stride != out_stride))) {
        set_error("bpe_adjust_logits: in place, types and strides must be equal");
        return BPE_ERR_OPTION;
    }
    AdjustParams p = {};
    if (rules) {
        const bpe_logit_rules &r = *rules;
        if (r.n_history < 0 || r.n_history >= 0x7FFFFFFFll || r.n_bias < 0 || r.n_bias >= 0x7FFFFFFFll || r.n_masks < 0) {
            set_error("bpe_adjust_logits: n_history, n_bias or n_masks out of range");
            return BPE_ERR_SIZE;
        }
        if ((!r.history && r.n_history) || (!r.history != !r.history_offsets && r.n_history)) { set_error("bpe_adjust_logits: history and history_offsets come together"); return BPE_ERR_NULL; }
        if (r.n_bias && (!r.bias_ids || !r.bias_values || !r.bias_offsets)) { set_error("bpe_adjust_logits: bias_ids, bias_values and bias_offsets come together"); return BPE_ERR_NULL; }
        if (!r.masks && r.mask_index) { set_error("bpe_adjust_logits: mask_index without masks"); return BPE_ERR_NULL; }
        if (r.masks && (r.n_masks > 1 && r.mask_stride < (n_vocab + 31) / 32)) { set_error("bpe_adjust_logits: mask_stride is shorter than a row"); return BPE_ERR_SIZE; }
        if (r.masks && !r.mask_index && r.n_masks < rows) { set_error("bpe_adjust_logits: without mask_index there is a mask for every row"); return BPE_ERR_SIZE; }
        p.rules = r;
        if (r.n_history == 0) p.rules.history_offsets = nullptr;
        if (r.n_bias == 0) p.rules.bias_offsets = nullptr;
    }
    p.logits = logits;
    p.out = out;
    p.logits_stride = logits_stride;
    p.out_stride = out_stride;
    p.n_vocab = (int32_t)n_vocab;
    const bool lists = p.rules.n_history > 0 || p.rules.n_bias > 0;
    // As many workgroups as are on the chip at once, if the slices can be as long: 64 rows of 100256 with lists 12.6 us, in twice as
    // many slices 16.5.
    const int64_t per_row = std::max<int64_t>(512 / rows, (n_vocab + kAdjustSlice - 1) / kAdjustSlice);
    p.slice = (int32_t)std::max<int64_t>(((n_vocab + per_row - 1) / per_row + 31) & ~31ll, 2048);
    p.slices = (int32_t)((n_vocab + p.slice - 1) / p.slice);
    void (*kernel)(AdjustParams) = nullptr;
#define ADJUST(IN, OUT) kernel = lists ? adjust_kernel<IN, OUT, true> : adjust_kernel<IN, OUT, false>
    if (dtype == BPE_F32) ADJUST(F32, F32);
    else if (dtype == BPE_BF16 && out_dtype == BPE_F32) ADJUST(Bf16, F32);
    else if (dtype == BPE_BF16) ADJUST(Bf16, Bf16);
    else if (out_dtype == BPE_F32) ADJUST(F16, F32);
    else ADJUST(F16, F16);
#undef ADJUST
    const int64_t at_once = (kMaxThreads - 1) / kAdjustThreads / p.slices;         // (2^30 tokens are 65,536 slices)
    for (int64_t row = 0; row < rows; row += at_once) {
        p.row0 = (int32_t)row;
        const int rc_launch = launch(kernel, dim3((unsigned)(std::min(at_once, rows - row) * p.slices)), kAdjustThreads, p, stream, "bpe_adjust_logits launch");
        if (rc_launch != BPE_OK) return rc_launch;
    }
    return BPE_OK;
}

static int check_top(int64_t rows, int64_t n_vocab, int64_t k) {
    const int rc = check_rows("bpe_top_tokens", rows, n_vocab, BPE_F32);
    if (rc != BPE_OK) return rc;
    if (k < 1 || k > kMaxTop || k > n_vocab) { set_error("bpe_top_tokens: k %lld is outside [1, min(%lld, n_vocab)]", (long long)k, (long long)kMaxTop); return BPE_ERR_SIZE; }
    return BPE_OK;
}

static int64_t align256l(int64_t v) { return (v + 255) & ~255ll; }

// Parts of a row: up to four workgroups per compute unit in all, none of fewer than 8,192 logits, and no more than can leave 2 k words
// each for the one workgroup that joins them.  (f32: 700 rows of 50257 in one part 42 us, in two 53; 300 rows in one 28, in four 32; one
// row in 7 parts 15.3, in 13 16.4.  64 rows of 100256 bf16, k = 256, in 8 parts 34, in 13, which cut down to the k best themselves, 43.)
static int64_t top_parts(int64_t rows, int64_t n_vocab, int64_t k) {
    const int64_t parts = std::min(std::min(1024 / std::max<int64_t>(rows, 1), (n_vocab + 8191) / 8192), (int64_t)kTopKeep / (2 * k));
    return std::max<int64_t>(parts, 1);
}
// Words that a part leaves: what its bound lets through, a little more than k as a rule.
static int64_t part_keep(int64_t parts, int64_t k) { return std::min<int64_t>(std::max<int64_t>(8 * k, 32), kTopKeep / parts); }

extern "C" int64_t bpe_top_tokens_workspace_bytes(int64_t rows, int64_t n_vocab, int64_t k) {
    const int rc = check_top(rows, n_vocab, k);
    if (rc != BPE_OK) return rc;
    const int64_t parts = top_parts(rows, n_vocab, k);
    return parts > 1 ? align256l(8 * rows * parts * part_keep(parts, k)) + (int64_t)sizeof(TopPart) * rows * parts : 0;
}

extern "C" int bpe_top_tokens(const void *logits, int64_t logits_stride, int dtype, int64_t rows, int64_t n_vocab, int64_t k,
                              int32_t *ids, float *logprobs, float *lse, void *workspace, int64_t workspace_bytes, void *stream) {
    if (!dtype_ok(dtype)) { set_error("bpe_top_tokens: dtype %d", dtype); return BPE_ERR_OPTION; }
    const int64_t need = bpe_top_tokens_workspace_bytes(rows, n_vocab, k);
    if (need < 0) return (int)need;
    if (rows == 0) return BPE_OK;
    if (!logits || !ids || !logprobs) { set_error("null pointer"); return BPE_ERR_NULL; }
    if (rows > 1 && logits_stride < n_vocab) { set_error("bpe_top_tokens: the stride is shorter than a row"); return BPE_ERR_SIZE; }
    if (!aligned_to(logits, dtype_bytes(dtype))) { set_error("bpe_top_tokens: logits are not aligned to their type"); return BPE_ERR_SIZE; }
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need)) {
        set_error("workspace must be 256-byte aligned and hold %lld bytes (got %lld)", (long long)need, (long long)workspace_bytes);
        return BPE_ERR_WORKSPACE;
    }
    TopParams p = {};
    p.logits = logits;
    p.logits_stride = logits_stride;
    p.n_vocab = (int32_t)n_vocab;
    p.k = (int32_t)k;
    p.ids = ids;
    p.logprobs = logprobs;
    p.lse = lse;
    const int64_t parts = top_parts(rows, n_vocab, k);
    p.parts = (int32_t)parts;
    p.part_len = (int32_t)(((n_vocab + parts - 1) / parts + 7) & ~7ll);
    p.kept = (uint64_t *)workspace;
    p.part_keep = (int32_t)part_keep(parts, k);
    p.left = (TopPart *)((char *)workspace + align256l(8 * rows * parts * p.part_keep));
    const int64_t at_once = (kMaxThreads - 1) / kTopThreads / parts;
    for (int64_t row = 0; row < rows; row += at_once) {
        const int64_t n = std::min(at_once, rows - row);
        p.row0 = (int32_t)row;
        int rc = launch(dtype == BPE_F32 ? top_part_kernel<F32> : dtype == BPE_BF16 ? top_part_kernel<Bf16> : top_part_kernel<F16>,
                        dim3((unsigned)(n * parts)), kTopThreads, p, stream, "bpe_top_tokens launch");
        if (rc == BPE_OK && parts > 1) rc = launch(top_join_kernel, dim3((unsigned)n), kTopThreads, p, stream, "bpe_top_tokens launch");
        if (rc != BPE_OK) return rc;
    }
    return BPE_OK;
}
