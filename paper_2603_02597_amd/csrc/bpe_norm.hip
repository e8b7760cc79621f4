// What stands between two blocks of a model: the norm behind a block, its gate, the scaled residual, and the norm in front of the next one.
#include <algorithm>
#include <cmath>

#include "bpe_numeric.h"

namespace bpe {

struct NormParams {
    const void *y, *residual;
    void *total, *out;
    int64_t y_stride, residual_stride, total_stride, out_stride;
    int32_t y_dtype, total_dtype, out_dtype, width, rows;
    int32_t row0;                      // the launch's first row
    bpe_norm_step step;
};

// Eight elements of a row of whatever type.
__device__ __forceinline__ void load8(const void *rows, int64_t row, int c, int width, int dtype, float (&v)[8]) {
    if (dtype == BPE_F32) load8<F32>((const float *)rows + row, c, width, v);
    else if (dtype == BPE_BF16) load8<Bf16>((const uint16_t *)rows + row, c, width, v);
    else load8<F16>((const uint16_t *)rows + row, c, width, v);
}
__device__ __forceinline__ void store8(void *rows, int64_t row, int c, int width, int dtype, const float (&v)[8]) {
    if (dtype == BPE_F32) store8<F32>((float *)rows + row, c, width, v);
    else if (dtype == BPE_BF16) store8<Bf16>((uint16_t *)rows + row, c, width, v);
    else store8<F16>((uint16_t *)rows + row, c, width, v);
}

__device__ __forceinline__ float activate_one(float v, int activation) {
    switch (activation) {
        case BPE_ACT_RELU: return relu(v);
        case BPE_ACT_GELU: return gelu(v);
        case BPE_ACT_GELU_TANH: return gelu_tanh(v);
        case BPE_ACT_SILU: return silu(v);
    }
    return v;
}

// The sum over the THREADS that share a row, in the same order every time: within a wavefront, then over the wavefronts, for which `turn` says which of two places in LDS it is (so that one barrier is enough).
template <int THREADS> __device__ __forceinline__ float row_sum(float v, float (*lds)[16], int turn) {
    v = of_last(sum_so_far(v));
    if constexpr (THREADS > kWave) {
        if ((threadIdx.x & 63) == 0) lds[turn][threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int s = 0; s < THREADS / kWave; ++s) v += lds[turn][s];
    }
    return v;
}

// THREADS share a row and hold CHUNKS times eight columns each, so a row is read once.  Bound by memory: 4001 x 8192, y and gate bf16, the residual in 32
// bits, 96 to 104 us, 460 MB at 4.4 to 4.8 TB/s (a copy: 5.0); rms alone, all bf16, on the same inputs again, 4096 rows of 2048 to 8192 columns 4.9 to 6.4 TB/s, of 16384, where a thread holds two chunks and half as many
// wavefronts fit, 4.7.  64 x 4096: 5.8, a launch and the chain of two norms.
// (An earlier form, four chunks on 256 threads, with sums over lanes through LDS and the residual read behind the first of them: 133 us for 4001 x 8192.)
template <int THREADS, int CHUNKS>
__global__ void __launch_bounds__(THREADS < 256 ? 256 : THREADS, CHUNKS > 1 ? 4 : 8) norm_kernel(NormParams p) {
    __shared__ float lds[2][16];
    const int tid = threadIdx.x % THREADS;
    const int64_t row = p.row0 + (THREADS < 256 ? (int64_t)blockIdx.x * (256 / THREADS) + threadIdx.x / THREADS : blockIdx.x);
    if (row >= p.rows) return;         // (whole wavefronts, and workgroups where they share a row)
    const bpe_norm_step &s = p.step;
    const float over = 1.0f / (float)p.width;
    float v[CHUNKS][8];
#pragma unroll
    for (int u = 0; u < CHUNKS; ++u) load8(p.y, row * p.y_stride, 8 * (tid + u * THREADS), p.width, p.y_dtype, v[u]);
    // (all that comes from memory is on its way before the first sum is waited for)
    float h[CHUNKS][8];
    if (p.residual) {
#pragma unroll
        for (int u = 0; u < CHUNKS; ++u) load8(p.residual, row * p.residual_stride, 8 * (tid + u * THREADS), p.width, p.total_dtype, h[u]);
    }
    int turn = 0;
    // what every element is moved and multiplied by (of the columns that exist: behind a row's end a first norm without a weight leaves what it makes of 0)
    const auto exists = [&](int u, int e) { return 8 * (tid + u * THREADS) + e < p.width; };
    auto statistics = [&](int kind, float eps, float &mean, float &factor) {
        mean = 0;
        if (kind == BPE_NORM_LAYER) {
            float sum = 0;
#pragma unroll
            for (int u = 0; u < CHUNKS; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += exists(u, e) ? v[u][e] : 0.0f;
            mean = row_sum<THREADS>(sum, lds, turn) * over;
            turn ^= 1;
        }
        float squares = 0;
#pragma unroll
        for (int u = 0; u < CHUNKS; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = exists(u, e) ? v[u][e] - mean : 0.0f;
                squares = __builtin_fmaf(d, d, squares);
            }
        factor = 1.0f / __builtin_sqrtf(row_sum<THREADS>(squares, lds, turn) * over + eps);
        turn ^= 1;
    };
    auto normed = [&](int kind, float eps, const void *weight, const void *bias) {
        if (kind == BPE_NORM_NONE) return;
        float mean, factor;
        statistics(kind, eps, mean, factor);
#pragma unroll
        for (int u = 0; u < CHUNKS; ++u) {
            const int c = 8 * (tid + u * THREADS);
            if (c >= p.width) break;
            float w[8], b[8];
            if (weight) load8(weight, 0, c, p.width, s.weight_dtype, w);
            if (bias) load8(bias, 0, c, p.width, s.weight_dtype, b);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[u][e] = (v[u][e] - mean) * factor;
                if (weight) v[u][e] *= w[e];
                if (bias) v[u][e] += b[e];
            }
        }
    };
    normed(s.post, s.post_eps, s.post_weight, s.post_bias);
#pragma unroll
    for (int u = 0; u < CHUNKS; ++u) {
        const int c = 8 * (tid + u * THREADS);
        if (c >= p.width) break;
        if (s.gate) {
            float g[8];
            load8(s.gate, row * s.gate_stride, c, p.width, s.gate_dtype, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[u][e] *= activate_one(g[e], s.gate_activation);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[u][e] *= s.branch_scale;
        if (p.residual) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[u][e] = __builtin_fmaf(s.residual_scale, h[u][e], v[u][e]);
        }
        if (p.total) store8(p.total, row * p.total_stride, c, p.width, p.total_dtype, v[u]);
    }
    if (!p.out) return;
    normed(s.pre, s.pre_eps, s.pre_weight, s.pre_bias);
#pragma unroll
    for (int u = 0; u < CHUNKS; ++u) {
        const int c = 8 * (tid + u * THREADS);
        if (c < p.width) store8(p.out, row * p.out_stride, c, p.width, p.out_dtype, v[u]);
    }
}

}  // namespace bpe

using namespace bpe;

constexpr int64_t kNormWidest = 256 * 64;

extern "C" int bpe_norm(const void *y, int64_t y_stride, int y_dtype, int64_t rows, int64_t width, const bpe_norm_step *step, const void *residual,
                        int64_t residual_stride, void *total, int64_t total_stride, int total_dtype, void *out, int64_t out_stride, int out_dtype,
                        void *stream) {
    if (rows < 0 || rows >= (1ll << 31) || width < 1 || width > kNormWidest) {
        set_error("bpe_norm: sizes out of range (rows %lld, width %lld)", (long long)rows, (long long)width);
        return BPE_ERR_SIZE;
    }
    if (!step) { set_error("null pointer"); return BPE_ERR_NULL; }
    const bpe_norm_step &s = *step;
    if (!dtype_ok(y_dtype) || ((residual || total) && !dtype_ok(total_dtype)) || (out && !dtype_ok(out_dtype)) || (s.gate && !dtype_ok(s.gate_dtype)) ||
        ((s.post_weight || s.post_bias || s.pre_weight || s.pre_bias) && !dtype_ok(s.weight_dtype))) {
        set_error("bpe_norm: a type is not one of float, bf16 and f16");
        return BPE_ERR_OPTION;
    }
    if (s.post < BPE_NORM_NONE || s.post > BPE_NORM_LAYER || s.pre < BPE_NORM_NONE || s.pre > BPE_NORM_LAYER) {
        set_error("bpe_norm: post %d, pre %d", s.post, s.pre);
        return BPE_ERR_OPTION;
    }
    if (s.gate_activation < BPE_ACT_NONE || s.gate_activation > BPE_ACT_SILU) { set_error("bpe_norm: gate_activation %d", s.gate_activation); return BPE_ERR_OPTION; }
    if ((s.post == BPE_NORM_NONE && (s.post_weight || s.post_bias)) || (s.pre == BPE_NORM_NONE && (s.pre_weight || s.pre_bias))) {
        set_error("bpe_norm: weight or bias of a norm that there is none of");
        return BPE_ERR_OPTION;
    }
    if ((s.post != BPE_NORM_NONE && !(s.post_eps >= 0)) || (s.pre != BPE_NORM_NONE && !(s.pre_eps >= 0))) { set_error("bpe_norm: eps is negative"); return BPE_ERR_OPTION; }
    if (rows == 0) return BPE_OK;
    if (!y || (!total && !out)) { set_error("null pointer"); return BPE_ERR_NULL; }
    if (rows > 1 && (y_stride < width || (residual && residual_stride < width) || (total && total_stride < width) || (out && out_stride < width) ||
                     (s.gate && s.gate_stride != 0 && s.gate_stride < width))) {
        set_error("bpe_norm: a stride is shorter than a row");
        return BPE_ERR_SIZE;
    }
    const auto odd = [](const void *at, int dtype) { return at && ((uintptr_t)at & (dtype_bytes(dtype) - 1)); };
    if (odd(y, y_dtype) || odd(residual, total_dtype) || odd(total, total_dtype) || odd(out, out_dtype) || odd(s.gate, s.gate_dtype) || odd(s.post_weight, s.weight_dtype) ||
        odd(s.post_bias, s.weight_dtype) || odd(s.pre_weight, s.weight_dtype) || odd(s.pre_bias, s.weight_dtype)) {
        set_error("bpe_norm: a pointer is not aligned to its type");
        return BPE_ERR_SIZE;
    }
    NormParams p = {};
    p.y = y; p.residual = residual; p.total = total; p.out = out;
    p.y_stride = y_stride; p.residual_stride = residual_stride; p.total_stride = total_stride; p.out_stride = out_stride;
    p.y_dtype = y_dtype; p.total_dtype = total_dtype; p.out_dtype = out_dtype; p.width = (int32_t)width; p.rows = (int32_t)rows;
    p.step = s;
    void (*kernel)(NormParams);
    const int64_t chunks = (width + 7) / 8;
    int threads = 256, per = 1;
    if (chunks <= 64) { kernel = norm_kernel<64, 1>; per = 4; }        // a wavefront per row
    else if (chunks <= 256) kernel = norm_kernel<256, 1>;
    else if (chunks <= 512) { kernel = norm_kernel<512, 1>; threads = 512; }
    else if (chunks <= 1024) { kernel = norm_kernel<1024, 1>; threads = 1024; }
    else { kernel = norm_kernel<1024, 2>; threads = 1024; }
    const int64_t at_once = per * (kMaxThreads / threads - 1);          // rows of a launch
    for (int64_t done = 0; done < rows; done += at_once) {
        p.row0 = (int32_t)done;
        const int rc = launch(kernel, dim3((unsigned)((std::min(rows - done, at_once) + per - 1) / per)), threads, p, stream, "bpe_norm launch");
        if (rc != BPE_OK) return rc;
    }
    return BPE_OK;
}
