// Matrices to 4 bits (bpe_mx_quantize) and rows of them back (bpe_mx_rows).
#include <algorithm>

#include "bpe_mx.h"

namespace bpe {

struct Mx4Params {
    const void *x;                     // or the rows' result
    void *out;
    int64_t stride;
    const uint8_t *from;
    uint8_t *to;
    int32_t rows, k, dtype;
    int64_t panels, all;               // of a row, of the matrix
    const int32_t *ids;
    int64_t n;
};

// A workgroup makes a panel: a lane takes eight neighbouring columns of a row, so four lanes share a scale.  The largest element's exponent is
// read from its bits; the hardware's conversion divides by the scale, rounds to the nearest (halves to the even code) and stops at 6.
// Codes meet in LDS and leave as whole lines (544 bytes from block to block, 32 of them free, spread the lanes' words over the banks).
// Bound by memory: 50256 x 4096 bf16 108 to 123 us, 412 MB read and 109 written, 4.2 to 4.8 TB/s (a copy: 5.0).  64 x 4096: 3.9, a launch.
constexpr int kBlockPitch = 544;
template <class T>
__global__ void __launch_bounds__(256) mx4_quantize_kernel(Mx4Params p) {
    __shared__ __attribute__((aligned(16))) uint8_t codes[8 * kBlockPitch], scales[256];
    const int tid = threadIdx.x, c = tid & 31, block = c >> 2, quarter = c & 3;
    for (int64_t panel = blockIdx.x; panel < p.all; panel += gridDim.x) {
        const int64_t group = panel / p.panels;
        const int column = (int)(panel - group * p.panels) * kPanelCols + 8 * c;
        float v[4][8];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t row = group * kPanelRows + 8 * u + (tid >> 5);
            load8<T>((const typename T::raw *)p.x + (row < p.rows ? row : 0) * p.stride, column, row < p.rows ? p.k : 0, v[u]);
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int row = 8 * u + (tid >> 5);
            uint32_t most = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) most = max(most, __builtin_bit_cast(uint32_t, v[u][e]) & 0x7fffffffu);
            most = max(most, (uint32_t)__shfl_xor((int)most, 1));
            most = max(most, (uint32_t)__shfl_xor((int)most, 2));
            const uint32_t exponent = most >> 23, byte = exponent == 255 ? 255 : exponent > 2 ? exponent - 2 : 0;
            const float scale = scale_of(byte);
            uint32_t word = 0;
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[u][0], v[u][1], scale, 0);
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[u][2], v[u][3], scale, 1);
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[u][4], v[u][5], scale, 2);
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[u][6], v[u][7], scale, 3);
            *(uint32_t *)(codes + block * kBlockPitch + row * 16 + 4 * quarter) = byte == 255 ? 0u : word;
            if (quarter == 0) scales[(block & 1) * 128 + row * 4 + (block >> 1)] = (uint8_t)byte;
        }
        __syncthreads();
        uint8_t *to = p.to + panel * kPanelBytes;
        *(U4 *)(to + 16 * tid) = *(const U4 *)(codes + (tid >> 5) * kBlockPitch + (tid & 31) * 16);
        if (tid < 16) *(U4 *)(to + kPanelCodes + 16 * tid) = *(const U4 *)(scales + 16 * tid);
    }
}

// All rows, a panel per workgroup: in whole lines through LDS, out as eight columns per lane.  Bound by writing: 50256 x 4096 to f32 155 to 163 us,
// 109 MB read and 824 written, 5.7 to 6.0 TB/s (filling memory: 6.9).
template <class T>
__global__ void __launch_bounds__(256) mx4_values_kernel(Mx4Params p) {
    __shared__ __attribute__((aligned(16))) uint8_t codes[8 * kBlockPitch], scales[256];
    const int tid = threadIdx.x, c = tid & 31, block = c >> 2, quarter = c & 3;
    for (int64_t panel = blockIdx.x; panel < p.all; panel += gridDim.x) {
        const int64_t group = panel / p.panels;
        const int column = (int)(panel - group * p.panels) * kPanelCols + 8 * c;
        const uint8_t *from = p.from + panel * kPanelBytes;
        __syncthreads();
        *(U4 *)(codes + (tid >> 5) * kBlockPitch + (tid & 31) * 16) = *(const U4 *)(from + 16 * tid);
        if (tid < 16) *(U4 *)(scales + 16 * tid) = *(const U4 *)(from + kPanelCodes + 16 * tid);
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int in_panel = 8 * u + (tid >> 5);
            const int64_t row = group * kPanelRows + in_panel;
            float v[8];
            values_of(*(const uint32_t *)(codes + block * kBlockPitch + in_panel * 16 + 4 * quarter), scale_of(scales[(block & 1) * 128 + in_panel * 4 + (block >> 1)]), v);
            if (row < p.rows) store8<T>((typename T::raw *)p.out + row * p.stride, column, p.k, v);
        }
    }
}

// Some rows: eight columns per lane, straight from memory.  A row's sixteen bytes lie 512 apart, so that of a line an eighth is used: 12 MB are read for
// 1.6, but 1500 rows of 2048 take 4.4 us, which is a launch and a chain of two loads.  It shows where many rows come from all over a large matrix: of
// 100256 x 4096 to bf16 1,500 rows take 7 us, 8,192 34, 32,768 126 (268 MB written, 2.1 TB/s).
template <class T>
__global__ void __launch_bounds__(256) mx4_gather_kernel(Mx4Params p) {
    const uint32_t per_row = (uint32_t)(p.k + 7) / 8;
    const int64_t total = p.n * per_row;
    for (int64_t first = (int64_t)blockIdx.x * 256; first < total; first += (int64_t)gridDim.x * 256) {
        const int64_t row0 = first / per_row;
        const uint32_t at = (uint32_t)(first - row0 * per_row) + threadIdx.x;
        const int64_t i = row0 + at / per_row;
        if (i >= p.n) continue;
        const int column = (int)(at % per_row) * 8, id = p.ids[i];
        float v[8] = {};
        if (id >= 0 && id < p.rows) {
            const uint8_t *panel = p.from + ((id >> 5) * p.panels + (column >> 8)) * kPanelBytes;
            const int block = column >> 5 & 7, row = id & 31;
            const uint32_t word = *(const uint32_t *)(panel + block * 512 + row * 16 + (column >> 3 & 3) * 4);
            values_of(word, scale_of(panel[kPanelCodes + (block & 1) * 128 + row * 4 + (block >> 1)]), v);
        }
        store8<T>((typename T::raw *)p.out + i * p.stride, column, p.k, v);
    }
}

static int mx4_sizes_ok(const char *call, int64_t rows, int64_t k) {
    if (rows < 0 || k < 0 || rows >= (1 << 30) || k >= (1 << 30)) {
        set_error("%s: sizes out of range (rows %lld, k %lld)", call, (long long)rows, (long long)k);
        return 0;
    }
    return 1;
}

constexpr int64_t kMostGroups = 1 << 22;        // workgroups of 256 threads of a launch

}  // namespace bpe

using namespace bpe;

extern "C" int64_t bpe_mx_bytes(int64_t rows, int64_t k) { return mx4_sizes_ok("bpe_mx_bytes", rows, k) ? mx4_bytes(rows, k) : BPE_ERR_SIZE; }

extern "C" int bpe_mx_quantize(const void *x, int64_t x_stride, int dtype, int64_t rows, int64_t k, void *mx4, void *stream) {
    if (!mx4_sizes_ok("bpe_mx_quantize", rows, k)) return BPE_ERR_SIZE;
    if (!dtype_ok(dtype)) { set_error("bpe_mx_quantize: dtype %d", dtype); return BPE_ERR_OPTION; }
    if (rows == 0 || k == 0) return BPE_OK;
    if (!x || !mx4) { set_error("null pointer"); return BPE_ERR_NULL; }
    if (rows > 1 && x_stride < k) { set_error("bpe_mx_quantize: a stride is shorter than a row"); return BPE_ERR_SIZE; }
    if (((uintptr_t)x & (dtype_bytes(dtype) - 1)) || ((uintptr_t)mx4 & 15)) { set_error("bpe_mx_quantize: x must be aligned to its type, mx4 to 16 bytes"); return BPE_ERR_SIZE; }
    Mx4Params p = {};
    p.x = x; p.stride = x_stride; p.to = (uint8_t *)mx4; p.rows = (int32_t)rows; p.k = (int32_t)k;
    p.panels = panels_of(k); p.all = mx4_bytes(rows, k) / kPanelBytes;
    auto kernel = dtype == BPE_F32 ? mx4_quantize_kernel<F32> : dtype == BPE_BF16 ? mx4_quantize_kernel<Bf16> : mx4_quantize_kernel<F16>;
    return launch(kernel, dim3((unsigned)std::min(p.all, kMostGroups)), 256, p, stream, "bpe_mx_quantize launch");
}

extern "C" int bpe_mx_rows(const void *mx4, int64_t rows, int64_t k, const int32_t *ids, int64_t n, void *out, int64_t out_stride, int out_dtype,
                            void *stream) {
    if (!mx4_sizes_ok("bpe_mx_rows", rows, k)) return BPE_ERR_SIZE;
    if (!dtype_ok(out_dtype)) { set_error("bpe_mx_rows: out_dtype %d", out_dtype); return BPE_ERR_OPTION; }
    if (n < 0 || n >= (1 << 30) || (!ids && n > rows)) { set_error("bpe_mx_rows: n %lld", (long long)n); return BPE_ERR_SIZE; }
    if (n == 0 || k == 0) return BPE_OK;
    if (!out || (rows > 0 && !mx4)) { set_error("null pointer"); return BPE_ERR_NULL; }
    if (n > 1 && out_stride < k) { set_error("bpe_mx_rows: a stride is shorter than a row"); return BPE_ERR_SIZE; }
    if (((uintptr_t)out & (dtype_bytes(out_dtype) - 1)) || ((uintptr_t)mx4 & 15) || ((uintptr_t)ids & 3)) {
        set_error("bpe_mx_rows: ids and out must be aligned to their types, mx4 to 16 bytes");
        return BPE_ERR_SIZE;
    }
    Mx4Params p = {};
    p.from = (const uint8_t *)mx4; p.out = out; p.stride = out_stride; p.rows = (int32_t)(ids ? rows : n); p.k = (int32_t)k;
    p.panels = panels_of(k); p.all = mx4_bytes(p.rows, k) / kPanelBytes; p.ids = ids; p.n = n;
    if (!ids) {
        auto kernel = out_dtype == BPE_F32 ? mx4_values_kernel<F32> : out_dtype == BPE_BF16 ? mx4_values_kernel<Bf16> : mx4_values_kernel<F16>;
        return launch(kernel, dim3((unsigned)std::min(p.all, kMostGroups)), 256, p, stream, "bpe_mx_rows launch");
    }
    auto kernel = out_dtype == BPE_F32 ? mx4_gather_kernel<F32> : out_dtype == BPE_BF16 ? mx4_gather_kernel<Bf16> : mx4_gather_kernel<F16>;
    return launch(kernel, dim3((unsigned)std::min((n * ((k + 7) / 8) + 255) / 256, kMostGroups)), 256, p, stream, "bpe_mx_rows launch");
}
