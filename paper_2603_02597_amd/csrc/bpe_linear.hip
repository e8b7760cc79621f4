// out = activation(x weight^T + bias) + residual on the matrix cores: the projection of hidden states onto a vocabulary,
// and the small blocks in front of it.
#include <algorithm>

#include "bpe_numeric.h"

namespace bpe {

struct LinearParams {
    const uint16_t *x, *w;
    int64_t x_stride, w_stride;
    int32_t m, n, k;
    const void *bias;
    int32_t bias_dtype, activation;
    const void *residual;
    int64_t residual_stride;
    void *out;
    int64_t out_stride;
    int32_t out_dtype;
};

typedef __bf16 Bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 F16x8 __attribute__((ext_vector_type(8)));

// D = A B + C on 16 x 16 x 32: lane l gives A[l % 16][8 (l / 16) ..+7] and B[8 (l / 16) ..+7][l % 16] and holds
// C[4 (l / 16) ..+3][l % 16].
template <class T> __device__ __forceinline__ F4 mma16(U4 a, U4 b, F4 c);
template <> __device__ __forceinline__ F4 mma16<Bf16>(U4 a, U4 b, F4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Bf16x8, a), __builtin_bit_cast(Bf16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ F4 mma16<F16>(U4 a, U4 b, F4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(F16x8, a), __builtin_bit_cast(F16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ float activate(float v, int activation) {
    switch (activation) {
        case BPE_ACT_RELU: return v > 0.0f ? v : (v != v ? v : 0.0f);
        case BPE_ACT_GELU: return 0.5f * v * (1.0f + erff(v * 0.70710678118654752f));
        case BPE_ACT_GELU_TANH: return 0.5f * v * (1.0f + tanhf(0.79788456080286536f * (v + 0.044715f * v * v * v)));
        case BPE_ACT_SILU: return v / (1.0f + __expf(-v));
        default: return v;
    }
}

// The epilogue of one element.
__device__ __forceinline__ void finish(const LinearParams &p, int i, int j, float v) {
    if (p.bias) v += load_as_float(p.bias, j, p.bias_dtype);
    v = activate(v, p.activation);
    if (p.residual) v += load_as_float(p.residual, i * p.residual_stride + j, p.out_dtype);
    const int64_t at = i * p.out_stride + j;
    if (p.out_dtype == BPE_F32) ((float *)p.out)[at] = v;
    else if (p.out_dtype == BPE_BF16) ((uint16_t *)p.out)[at] = from_float<Bf16>(v);
    else ((uint16_t *)p.out)[at] = from_float<F16>(v);
}

// Eight elements of a row from column t on; zeros behind the row's end and for rows that do not exist.
__device__ __forceinline__ U4 load8(const uint16_t *base, int64_t stride, int row, int rows, int t, int k) {
    H8 v = {0, 0, 0, 0, 0, 0, 0, 0};
    if (row < rows) {
        const uint16_t *at = base + row * stride;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (t + e < k) v[e] = at[t + e];
    }
    return __builtin_bit_cast(U4, v);
}

// A workgroup of four wavefronts makes 64 x 64 of out, a wavefront 32 x 32 (two by two products of 16 x 16), 32 of k at a time through LDS.
template <class T>
__global__ void __launch_bounds__(kGroupThreads) linear_tile_kernel(LinearParams p) {
    __shared__ U4 xs[64][4], ws[64][4];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int j0 = blockIdx.x * 64, i0 = blockIdx.y * 64;
    const int wi = 32 * (wv >> 1), wj = 32 * (wv & 1);
    F4 acc[2][2] = {};
    for (int t = 0; t < p.k; t += 32) {
        __syncthreads();
        xs[tid >> 2][tid & 3] = load8(p.x, p.x_stride, i0 + (tid >> 2), p.m, t + 8 * (tid & 3), p.k);
        ws[tid >> 2][tid & 3] = load8(p.w, p.w_stride, j0 + (tid >> 2), p.n, t + 8 * (tid & 3), p.k);
        __syncthreads();
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b)
                acc[a][b] = mma16<T>(xs[wi + 16 * a + (lane & 15)][lane >> 4], ws[wj + 16 * b + (lane & 15)][lane >> 4], acc[a][b]);
    }
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = i0 + wi + 16 * a + 4 * (lane >> 4) + e, j = j0 + wj + 16 * b + (lane & 15);
                if (i < p.m && j < p.n) finish(p, i, j, acc[a][b][e]);
            }
}

}  // namespace bpe

using namespace bpe;

static int linear_sizes_ok(int64_t m, int64_t n, int64_t k) {
    if (m < 0 || n < 0 || k < 0 || m >= (1 << 30) || n >= (1 << 30) || k >= (1 << 30)) {
        set_error("bpe_linear: sizes out of range (m %lld, n %lld, k %lld)", (long long)m, (long long)n, (long long)k);
        return 0;
    }
    return 1;
}

extern "C" int64_t bpe_linear_workspace_bytes(int64_t m, int64_t n, int64_t k) {
    if (!linear_sizes_ok(m, n, k)) return BPE_ERR_SIZE;
    return 0;
}

extern "C" int bpe_linear(const void *x, int64_t x_stride, const void *weight, int64_t weight_stride, int dtype, int64_t m, int64_t n,
                          int64_t k, const void *bias, int bias_dtype, const void *residual, int64_t residual_stride, int activation,
                          void *out, int64_t out_stride, int out_dtype, void *workspace, int64_t workspace_bytes, void *stream) {
    if (!linear_sizes_ok(m, n, k)) return BPE_ERR_SIZE;
    if (dtype != BPE_BF16 && dtype != BPE_F16) { set_error("bpe_linear: x and weight are bf16 or f16 (dtype %d)", dtype); return BPE_ERR_OPTION; }
    if (out_dtype != BPE_F32 && out_dtype != dtype) { set_error("bpe_linear: out is f32 or of the inputs' type (out_dtype %d)", out_dtype); return BPE_ERR_OPTION; }
    if (bias && !dtype_ok(bias_dtype)) { set_error("bpe_linear: bias_dtype %d", bias_dtype); return BPE_ERR_OPTION; }
    if (activation < BPE_ACT_NONE || activation > BPE_ACT_SILU) { set_error("bpe_linear: activation %d", activation); return BPE_ERR_OPTION; }
    if (m == 0 || n == 0) return BPE_OK;
    if (!out || (k > 0 && (!x || !weight))) { set_error("null pointer"); return BPE_ERR_NULL; }
    if ((m > 1 && (x_stride < k || out_stride < n || (residual && residual_stride < n))) || (n > 1 && weight_stride < k)) {
        set_error("bpe_linear: a stride is shorter than a row");
        return BPE_ERR_SIZE;
    }
    const int64_t need = bpe_linear_workspace_bytes(m, n, k);
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need)) {
        set_error("workspace must be 256-byte aligned and hold %lld bytes (got %lld)", (long long)need, (long long)workspace_bytes);
        return BPE_ERR_WORKSPACE;
    }
    const uintptr_t odd = (uintptr_t)x | (uintptr_t)weight;
    if ((odd & 1) || ((uintptr_t)out & (dtype_bytes(out_dtype) - 1)) || ((uintptr_t)residual & (dtype_bytes(out_dtype) - 1)) ||
        (bias && ((uintptr_t)bias & (dtype_bytes(bias_dtype) - 1)))) {
        set_error("bpe_linear: a pointer is not aligned to its type");
        return BPE_ERR_SIZE;
    }
    LinearParams p = {};
    p.x = (const uint16_t *)x; p.w = (const uint16_t *)weight;
    p.x_stride = x_stride; p.w_stride = weight_stride;
    p.m = (int32_t)m; p.n = (int32_t)n; p.k = (int32_t)k;
    p.bias = bias; p.bias_dtype = bias_dtype; p.activation = activation;
    p.residual = residual; p.residual_stride = residual_stride;
    p.out = out; p.out_stride = out_stride; p.out_dtype = out_dtype;
    const int64_t gx = (n + 63) / 64, gy = (m + 63) / 64;
    if (gy > 65535) { set_error("bpe_linear: m %lld is too large", (long long)m); return BPE_ERR_SIZE; }
    const dim3 grid((unsigned)gx, (unsigned)gy);
    return launch(dtype == BPE_BF16 ? linear_tile_kernel<Bf16> : linear_tile_kernel<F16>, grid, kGroupThreads, p, stream, "bpe_linear launch");
}
