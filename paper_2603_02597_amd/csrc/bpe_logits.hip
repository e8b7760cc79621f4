// Logits under the rules of a request (bpe_adjust_logits) and the best tokens of every row (bpe_top_tokens).
#include <algorithm>

#include "bpe_numeric.h"

namespace bpe {

struct AdjustParams {
    const void *logits;
    void *out;
    int64_t logits_stride, out_stride;
    int32_t rows, n_vocab;
    bpe_logit_rules rules;
};

// Elements [begin, end) of a list that the rows share, clamped to the list.
__device__ __forceinline__ void row_range(const int32_t *offsets, int64_t n, int row, int &begin, int &end) {
    begin = end = 0;
    if (!offsets) return;
    begin = min(max(offsets[row], 0), (int)n);
    end = min(max(offsets[row + 1], begin), (int)n);
}

constexpr int kSlice = 4096;         // tokens of a row per workgroup

// The row's mask, or nullptr; `nothing` if its index is too large.
__device__ __forceinline__ const uint32_t *row_mask(const bpe_logit_rules &r, int row, bool &nothing) {
    nothing = false;
    if (!r.masks) return nullptr;
    const int64_t i = r.mask_index ? r.mask_index[row] : row;
    if (i < 0) return nullptr;
    nothing = i >= r.n_masks;
    return nothing ? nullptr : r.masks + i * r.mask_stride;
}

// A workgroup takes a slice of a row: it counts the row's history and notes its biases in LDS, then makes one pass over the slice.
template <class IN, class OUT>
__global__ void __launch_bounds__(kGroupThreads) adjust_kernel(AdjustParams p) {
#pragma clang fp contract(off)
    __shared__ uint32_t count[kSlice], bias_at[kSlice];
    const bpe_logit_rules &r = p.rules;
    const int first = blockIdx.x * kSlice, last = min(first + kSlice, p.n_vocab), tid = threadIdx.x;
    for (int row = blockIdx.y; row < p.rows; row += gridDim.y) {
        __syncthreads();
        for (int i = tid; i < kSlice; i += kGroupThreads) count[i] = bias_at[i] = 0;
        __syncthreads();
        int begin, end;
        row_range(r.history_offsets, r.n_history, row, begin, end);
        for (int i = begin + tid; i < end; i += kGroupThreads) {
            const int v = r.history[i];
            if (v >= first && v < last) atomicAdd(&count[v - first], 1u);
        }
        row_range(r.bias_offsets, r.n_bias, row, begin, end);
        for (int i = begin + tid; i < end; i += kGroupThreads) {
            const int v = r.bias_ids[i];
            if (v >= first && v < last) atomicMax(&bias_at[v - first], (uint32_t)i + 1u);     // the last entry counts
        }
        __syncthreads();
        const float rep = r.repetition ? r.repetition[row] : 1.0f, freq = r.frequency ? r.frequency[row] : 0.0f,
                    pres = r.presence ? r.presence[row] : 0.0f;
        bool nothing;
        const uint32_t *mask = row_mask(r, row, nothing);
        const typename IN::raw *in = (const typename IN::raw *)p.logits + row * p.logits_stride;
        typename OUT::raw *out = (typename OUT::raw *)p.out + row * p.out_stride;
        for (int v = first + tid; v < last; v += kGroupThreads) {
            float x = to_float<IN>(in[v]);
            if (const uint32_t c = count[v - first]) {
                x = x > 0.0f ? x / rep : x * rep;
                x = x - freq * (float)c;
                x = x - pres;
            }
            if (const uint32_t b = bias_at[v - first]) x = x + r.bias_values[b - 1];
            if (nothing || (mask && !((mask[v >> 5] >> (v & 31)) & 1u))) x = -__builtin_inff();
            out[v] = from_float<OUT>(x);
        }
    }
}

struct TopParams {
    const void *logits;
    int64_t logits_stride;
    int32_t rows, n_vocab, k;
    int32_t *ids;
    float *logprobs, *lse;
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

// A workgroup takes a row and finds its best token, the best of the rest and so on: k passes.
template <class IN>
__global__ void __launch_bounds__(1024) top_kernel(TopParams p) {
    __shared__ uint64_t best_of[16];
    __shared__ float sum_of[16];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    for (int row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const typename IN::raw *in = (const typename IN::raw *)p.logits + row * p.logits_stride;
        uint64_t bound = ~0ull;                    // (key, ~index) of the one found last
        float lse = 0.0f;
        for (int j = 0; j < p.k; ++j) {
            uint64_t best = 0;
            for (int v = tid; v < p.n_vocab; v += 1024) {
                const uint64_t e = (uint64_t)order_key(to_float<IN>(in[v])) << 32 | ~(uint32_t)v;
                if (e < bound && e > best) best = e;
            }
            for (int d = 32; d; d >>= 1) {
                const uint64_t o = __shfl_xor((unsigned long long)best, d);
                best = o > best ? o : best;
            }
            __syncthreads();
            if (lane == 0) best_of[wv] = best;
            __syncthreads();
            for (int w = 0; w < 16; ++w) best = best_of[w] > best ? best_of[w] : best;
            bound = best;
            const float x = key_value((uint32_t)(best >> 32));
            if (j == 0) {
                float sum = 0.0f;
                const float most = x == -__builtin_inff() ? 0.0f : x;
                for (int v = tid; v < p.n_vocab; v += 1024) sum += expf(to_float<IN>(in[v]) - most);
                for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
                if (lane == 0) sum_of[wv] = sum;
                __syncthreads();
                sum = 0.0f;
                for (int w = 0; w < 16; ++w) sum += sum_of[w];
                lse = x == __builtin_inff() ? x : x + logf(sum);
                if (p.lse && tid == 0) p.lse[row] = lse;
            }
            if (tid == 0) {
                const bool none = x == -__builtin_inff();
                p.ids[(int64_t)row * p.k + j] = none ? -1 : (int)~(uint32_t)best;
                p.logprobs[(int64_t)row * p.k + j] = none ? x : x - lse;
            }
        }
    }
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
    p.rows = (int32_t)rows;
    p.n_vocab = (int32_t)n_vocab;
    const dim3 grid((unsigned)((n_vocab + kSlice - 1) / kSlice), (unsigned)std::min<int64_t>(rows, 32768));
    void (*kernel)(AdjustParams) = dtype == BPE_F32 ? adjust_kernel<F32, F32>
                                   : dtype == BPE_BF16 ? (out_dtype == BPE_F32 ? adjust_kernel<Bf16, F32> : adjust_kernel<Bf16, Bf16>)
                                                       : (out_dtype == BPE_F32 ? adjust_kernel<F16, F32> : adjust_kernel<F16, F16>);
    return launch(kernel, grid, kGroupThreads, p, stream, "bpe_adjust_logits launch");
}

constexpr int64_t kMaxTop = 256;

static int check_top(int64_t rows, int64_t n_vocab, int64_t k) {
    const int rc = check_rows("bpe_top_tokens", rows, n_vocab, BPE_F32);
    if (rc != BPE_OK) return rc;
    if (k < 1 || k > kMaxTop || k > n_vocab) { set_error("bpe_top_tokens: k %lld is outside [1, min(%lld, n_vocab)]", (long long)k, (long long)kMaxTop); return BPE_ERR_SIZE; }
    return BPE_OK;
}

extern "C" int64_t bpe_top_tokens_workspace_bytes(int64_t rows, int64_t n_vocab, int64_t k) {
    const int rc = check_top(rows, n_vocab, k);
    return rc != BPE_OK ? rc : 0;
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
    p.rows = (int32_t)rows;
    p.n_vocab = (int32_t)n_vocab;
    p.k = (int32_t)k;
    p.ids = ids;
    p.logprobs = logprobs;
    p.lse = lse;
    return launch(dtype == BPE_F32 ? top_kernel<F32> : dtype == BPE_BF16 ? top_kernel<Bf16> : top_kernel<F16>,
                  dim3((unsigned)std::min<int64_t>(rows, 1 << 20)), 1024, p, stream, "bpe_top_tokens launch");
}
