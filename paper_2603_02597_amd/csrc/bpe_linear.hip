// out = activation(x weight^T + bias) + residual on the matrix cores: the projection of hidden states onto a vocabulary,
// and the small blocks in front of it.
#include <algorithm>
#include <cmath>
#include <type_traits>

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
    int32_t out_dtype, splits;         // k is cut into so many parts, whose sums meet in `part` if there are several
    float *part;                       // [splits][m][part_stride]
    int32_t part_stride;
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

// The activations without a branch, from the hardware's 2^x and reciprocal (a unit in the last place each).  A factor of 0 meets the largest
// finite value in place of an infinity, so that all give their limits; a NaN stays one through the factor.
constexpr float kMost = 3.402823466e38f, kLog2Of = 1.44269504088896341f;
__device__ __forceinline__ float relu(float v) { return v < 0.0f ? 0.0f : v; }
__device__ __forceinline__ float times_sigmoid(float v, float minus_log2_odds) {
    return fmaxf(v, -kMost) * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(minus_log2_odds));
}
// v (1 + erf(v / sqrt 2)) / 2 = max(v, 0) - |v| q with q = erfc(|v| / sqrt 2) / 2, which is exp(-v^2 / 2) by a function that falls slowly: a
// series of eight terms in t = 1 / (1 + 0.3 |v|), fitted to a relative error of 2.2e-7 (3.3e-9 of |v|) for |v| up to 14, where q leaves
// 32 bits.  No difference of nearly equal numbers, so small results are good too: rms error 2.1e-8 on normal v, 1.6e-9 on -6 .. -2 (0.5 v (1
// + erff(v / sqrt 2)): 2.5e-8, 3.4e-8; 2000 x 20000 x 512 f16 107 us, without an activation 76).
__device__ __forceinline__ float gelu(float v) {
    const float size = __builtin_fabsf(v), t = __builtin_amdgcn_rcpf(1.0f + 0.3f * size);
    const float series = t * (0.11962141f + t * (0.120887813f + t * (0.0989954205f + t * (0.13186087f + t * (-0.0604071882f + t * (0.214153407f +
                         t * (-0.161994644f + t * 0.0368829476f)))))));
    return fmaxf(v, 0.0f) - fminf(size, kMost) * (series * __builtin_amdgcn_exp2f(v * v * (-0.5f * kLog2Of)));
}
// v (1 + tanh u) / 2 = v / (1 + exp(-2 u)), u = sqrt(2 / pi) (v + 0.044715 v^3)
__device__ __forceinline__ float gelu_tanh(float v) {
    constexpr float c = -2.0f * kLog2Of * 0.79788456080286536f;
    return times_sigmoid(v, v * (c + (c * 0.044715f) * (v * v)));
}
__device__ __forceinline__ float silu(float v) { return times_sigmoid(v, v * -kLog2Of); }

template <int ROWS> __device__ __forceinline__ void activate(F4 (&v)[ROWS], int activation) {
#define EACH(FUNCTION) \
    _Pragma("unroll") for (int u = 0; u < ROWS; ++u) { \
        _Pragma("unroll") for (int e = 0; e < 4; ++e) v[u][e] = FUNCTION(v[u][e]); \
        __builtin_amdgcn_sched_barrier(0); /* (not all rows' intermediate values at once) */ \
    }
    switch (activation) {
        case BPE_ACT_RELU: EACH(relu); break;
        case BPE_ACT_GELU: EACH(gelu); break;
        case BPE_ACT_GELU_TANH: EACH(gelu_tanh); break;
        case BPE_ACT_SILU: EACH(silu); break;
    }
#undef EACH
}

typedef float F4Any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t H4Any __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ float out_to_float(const LinearParams &p, uint16_t v) { return p.out_dtype == BPE_BF16 ? to_float<Bf16>(v) : to_float<F16>(v); }
__device__ __forceinline__ uint16_t out_from_float(const LinearParams &p, float v) { return p.out_dtype == BPE_BF16 ? from_float<Bf16>(v) : from_float<F16>(v); }
__device__ __forceinline__ F4 bias_of(const LinearParams &p, int j) {          // of columns j .. j + 3, as far as they exist
    F4 v = {0, 0, 0, 0};
    if (!p.bias) return v;
    if (j + 3 >= p.n) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (j + e < p.n) v[e] = load_as_float(p.bias, j + e, p.bias_dtype);
    } else if (p.bias_dtype == BPE_F32) {
        v = *(const F4Any *)((const float *)p.bias + j);
    } else {
        const H4Any b = *(const H4Any *)((const uint16_t *)p.bias + j);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = p.bias_dtype == BPE_BF16 ? to_float<Bf16>(b[e]) : to_float<F16>(b[e]);
    }
    return v;
}
// What the residual holds for columns j .. j + 3, if all exist, of ROWS rows that are `step` apart: bytes as they are (16-bit ones in
// the first half).  Rows behind the last repeat it.
template <int ROWS> __device__ __forceinline__ void fetch(const LinearParams &p, int i, int step, int j, U4 (&res)[ROWS]) {
    if (!p.residual || j + 3 >= p.n) return;
    typedef uint32_t U2Any __attribute__((ext_vector_type(2), aligned(2)));
    if (p.out_dtype == BPE_F32) {
#pragma unroll
        for (int u = 0; u < ROWS; ++u) res[u] = __builtin_bit_cast(U4, *(const F4Any *)((const float *)p.residual + min(i + u * step, p.m - 1) * p.residual_stride + j));
    } else {
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const U2Any r = *(const U2Any *)((const uint16_t *)p.residual + min(i + u * step, p.m - 1) * p.residual_stride + j);
            res[u] = U4{r[0], r[1], 0, 0};
        }
    }
}
// Bias (of bias_of), activation and residual (of fetch).
template <int ROWS> __device__ __forceinline__ void finish(const LinearParams &p, F4 (&v)[ROWS], F4 bias, const U4 (&res)[ROWS]) {
    if (p.bias) {
#pragma unroll
        for (int u = 0; u < ROWS; ++u) v[u] += bias;
    }
    activate(v, p.activation);
    if (!p.residual) return;
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        if (p.out_dtype == BPE_F32) {
            v[u] += __builtin_bit_cast(F4, res[u]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[u][e] += out_to_float(p, (uint16_t)(res[u][e / 2] >> 16 * (e % 2)));
        }
    }
}
__device__ __forceinline__ H4Any narrow(const LinearParams &p, F4 v) {
    H4Any o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = out_from_float(p, v[e]);
    return o;
}
// The epilogue of these columns, as far as they exist, of these rows, as far as they do.
template <int ROWS>
__device__ __forceinline__ void put(const LinearParams &p, int i, int step, int j, F4 (&v)[ROWS], F4 bias, U4 (&res)[ROWS]) {
    if (p.residual && j + 3 >= p.n) {
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const int64_t from = min(i + u * step, p.m - 1) * p.residual_stride + j;
            res[u] = U4{0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (j + e >= p.n) break;
                if (p.out_dtype == BPE_F32) res[u][e] = ((const uint32_t *)p.residual)[from + e];
                else res[u][e / 2] |= (uint32_t)((const uint16_t *)p.residual)[from + e] << 16 * (e % 2);
            }
        }
    }
    finish(p, v, bias, res);
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        const int64_t row = i + u * step, at = row * p.out_stride + j;
        if (row >= p.m) break;
        if (j + 3 >= p.n) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (j + e >= p.n) break;
                if (p.out_dtype == BPE_F32) ((float *)p.out)[at + e] = v[u][e];
                else ((uint16_t *)p.out)[at + e] = out_from_float(p, v[u][e]);
            }
        } else if (p.out_dtype == BPE_F32) {
            *(F4Any *)((float *)p.out + at) = v[u];
        } else {
            *(H4Any *)((uint16_t *)p.out + at) = narrow(p, v[u]);
        }
    }
}
// The same two for a tile that lies within out as a whole: `row` and the tile's first column `col` are the same in all lanes, which are
// `lane_at` bytes from there, so that addresses cost the vector unit nothing.
template <int ROWS> __device__ __forceinline__ void fetch_whole(const LinearParams &p, int row, int step, int col, uint32_t lane_at, U4 (&res)[ROWS]) {
    if (!p.residual) return;
    typedef uint32_t U2Any __attribute__((ext_vector_type(2), aligned(2)));
    if (p.out_dtype == BPE_F32) {
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const char *from = (const char *)((const float *)p.residual + (row + u * step) * p.residual_stride + col);
            res[u] = __builtin_bit_cast(U4, *(const F4Any *)(from + lane_at));
        }
    } else {
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const char *from = (const char *)((const uint16_t *)p.residual + (row + u * step) * p.residual_stride + col);
            const U2Any r = *(const U2Any *)(from + lane_at);
            res[u] = U4{r[0], r[1], 0, 0};
        }
    }
}
template <int ROWS>
__device__ __forceinline__ void put_whole(const LinearParams &p, int row, int step, int col, uint32_t lane_at, F4 (&v)[ROWS], F4 bias, const U4 (&res)[ROWS]) {
    finish(p, v, bias, res);
    if (p.out_dtype == BPE_F32) {
#pragma unroll
        for (int u = 0; u < ROWS; ++u) *(F4Any *)((char *)((float *)p.out + (row + u * step) * p.out_stride + col) + lane_at) = v[u];
    } else {
#pragma unroll
        for (int u = 0; u < ROWS; ++u) *(H4Any *)((char *)((uint16_t *)p.out + (row + u * step) * p.out_stride + col) + lane_at) = narrow(p, v[u]);
    }
}
__device__ __forceinline__ void put4(const LinearParams &p, int i, int j, F4 v) {
    F4 one[1] = {v};
    U4 res[1];
    fetch(p, i, 1, j, res);
    put(p, i, 1, j, one, bias_of(p, j), res);
}

// Sixteen bytes at any even address: the hardware asks for no more.
typedef uint32_t U4Any __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ U4 load16(const uint16_t *at) { return *(const U4Any *)at; }

// Eight elements without the first `over`, zeros in their place at the end.
__device__ __forceinline__ U4 shift_out(U4 eight, int over) {
    typedef uint64_t Two __attribute__((ext_vector_type(2)));
    const Two v = __builtin_bit_cast(Two, eight);
    const uint32_t shift = 16u * (uint32_t)(over & 3);
    const uint64_t low = over < 4 ? v[0] : v[1], high = over < 4 ? v[1] : 0;
    Two o = {low >> shift | (shift ? high << (64 - shift) : 0), high >> shift};
    if (over >= 8) o = Two{0, 0};
    return __builtin_bit_cast(U4, o);
}
// Eight elements of a row from column t on, zeros behind the row's end: the row's last eight at most, shifted.  No branch for k >= 8.
__device__ __forceinline__ U4 load_tail(const uint16_t *row, int t, int k) {
    if (k < 8) {
        H8 v = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (t + e < k) v[e] = row[t + e];
        return __builtin_bit_cast(U4, v);
    }
    const int over = max(t - (k - 8), 0);                 // elements of the eight that lie behind the end
    return shift_out(load16(row + (t - over)), over);
}

// A few rows of x: the call is as long as reading weight takes, so weight goes from memory straight into the matrix cores'
// registers.  A workgroup takes 16 rows of weight, its four wavefronts a quarter of k each (so a vocabulary of few rows still fills
// the chip); their sums meet in LDS.  A step is 64 columns, whole lines of memory, and four steps are under way at a time.
// weight is the left operand: a lane ends with four neighbouring columns of one row of out; rows behind the last of x repeat it and
// are dropped.  What lies behind the last whole step is loaded before the first one.  Bound by memory: 1 x 50256 x 1024 18 us, 1 x
// 100256 x 4096 142 us, 5.8 TB/s; 1 x 2048 x 2048 7 us, of which 5 are the launch.
constexpr int kRowsAhead = 4;
template <class T>
__global__ void __launch_bounds__(kGroupThreads) linear_rows_kernel(LinearParams p) {
    __shared__ F4 part[kWavesPerGroup][kWave];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int j0 = blockIdx.x * 16, group = 8 * (lane >> 4);
    const int steps = p.k >> 6, from = (int)((int64_t)steps * wv / kWavesPerGroup), to = (int)((int64_t)steps * (wv + 1) / kWavesPerGroup);
    const uint16_t *w = p.w + min(j0 + (lane & 15), p.n - 1) * p.w_stride, *x = p.x + min(lane & 15, p.m - 1) * p.x_stride;
    F4 acc = {0, 0, 0, 0};
    U4 wf[kRowsAhead][2], xf[kRowsAhead][2];
    auto load = [&](int u, int step) {
#pragma unroll
        for (int h = 0; h < 2; ++h) wf[u][h] = load16(w + 64 * (int64_t)step + 32 * h + group);
#pragma unroll
        for (int h = 0; h < 2; ++h) xf[u][h] = load16(x + 64 * (int64_t)step + 32 * h + group);
    };
    auto multiply = [&](int u) {
#pragma unroll
        for (int h = 0; h < 2; ++h) acc = mma16<T>(wf[u][h], xf[u][h], acc);
    };
    // the columns behind the last whole step
    const bool tail = wv == kWavesPerGroup - 1 && (p.k & 63);
    U4 w_tail[2], x_tail[2];
    if (tail) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            w_tail[h] = load_tail(w, (p.k & ~63) + 32 * h + group, p.k);
            x_tail[h] = load_tail(x, (p.k & ~63) + 32 * h + group, p.k);
        }
    }
#pragma unroll
    for (int u = 0; u < kRowsAhead; ++u)
        if (from + u < to) load(u, from + u);
    int step = from;
    for (; step + 2 * kRowsAhead <= to; step += kRowsAhead)
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
            multiply(u);
            load(u, step + kRowsAhead + u);
        }
    for (; step < to; step += kRowsAhead)
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u)
            if (step + u < to) {
                multiply(u);
                if (step + kRowsAhead + u < to) load(u, step + kRowsAhead + u);
            }
    if (tail) {
#pragma unroll
        for (int h = 0; h < 2; ++h) acc = mma16<T>(w_tail[h], x_tail[h], acc);
    }
    part[wv][lane] = acc;
    __syncthreads();
    if (wv != 0) return;
#pragma unroll
    for (int s = 1; s < kWavesPerGroup; ++s) acc += part[s][lane];
    const int i = lane & 15, j = j0 + 4 * (lane >> 4);
    if (i < p.m && j < p.n) put4(p, i, j, acc);
}

// More rows.  A workgroup makes BM x BN of out, WM x WN wavefronts side by side, 64 columns of k at a time through LDS: 128 (BM + BN)
// bytes of rows for 128 BM BN operations.  Large products take the largest tile, whose rows the L2s can bring as fast as the matrix cores
// use them; few rows of x a tile so small that weight comes from memory to all compute units at once, with k cut into parts that
// linear_join_kernel adds up where there are fewer tiles than compute units (plan_linear).
// The loads go straight into LDS, two blocks ahead; products, LDS reads and loads are put in order by hand, so the matrix cores
// see no wait but the one in the middle of a block.  The operands are swapped (weight on the left): a lane ends with neighbouring
// columns of a row.  Bound by memory for few rows: 64 x 100256 x 4096 163 us, 5.2 TB/s.  Bound by the matrix cores for many: 4001 x
// 50256 x 4096 1,301 to 1,395 us by card, 1,266 to 1,181 TFLOP/s, 94 % of a library's plain product there; 4096 x 4096 x 4096 119 us, 87 %.  What is missing is a
// tile's first loads and its result, some 10 us in which the only workgroup of a compute unit leaves the matrix cores alone.
// A last block that is cut off costs about a whole one: 120 x 3664 x 2792 16.2 us, x 2816 14.9.  Rows at odd addresses pass through
// registers: 508 x 2086 x 579 13.1 us, 508 x 2088 x 584 10.2; 64 x 100256 x 4096 231 us, 4001 x 20000 x 2048 383, aligned 163 and 294.
typedef float F16v __attribute__((ext_vector_type(16)));
// D = A B + C on 32 x 32 x 16: lane l gives A[l % 32][8 (l / 32) ..+7] and B[8 (l / 32) ..+7][l % 32] and holds
// C[e % 4 + 8 (e / 4) + 4 (l / 32)][l % 32] in element e.
template <class T> __device__ __forceinline__ F16v mma32(U4 a, U4 b, F16v c);
template <> __device__ __forceinline__ F16v mma32<Bf16>(U4 a, U4 b, F16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(Bf16x8, a), __builtin_bit_cast(Bf16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ F16v mma32<F16>(U4 a, U4 b, F16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(F16x8, a), __builtin_bit_cast(F16x8, b), c, 0, 0, 0);
}

// Sixteen bytes per lane from memory into LDS, at `lds` + 16 * lane, without a register in between.  The compiler does not
// see these loads: wait_and_meet waits for them, and no other load from memory is under way in between.
__device__ __forceinline__ void load_lds(uint32_t lds, const char *base, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory");
}
// All but this wavefront's last LATER loads have arrived and its reads of LDS are done; then the other wavefronts'.
template <int LATER> __device__ __forceinline__ void wait_and_meet() {
    static_assert(LATER < 64, "");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LATER) : "memory");
}

// Which tile of out a workgroup makes.  Workgroups go round the eight chiplets by their index, and each chiplet has an L2 of its
// own: so every chiplet gets a run of neighbouring tiles, eight rows of tiles by as many columns as it takes.
// (In 32 bits: a launch has fewer than 2^24 workgroups, and a division of 64 bits takes a fifth of a microsecond.)
__device__ __forceinline__ bool tile_of(uint32_t tiles_m, uint32_t tiles_n, uint32_t splits, int &tm, int &tn, int &split) {
    const uint32_t tiles = tiles_m * tiles_n, total = tiles * splits, per = (total + 7) / 8;
    uint32_t s = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= per || s >= total) return false;
    split = 0;
    if (splits > 1) {
        split = (int)(s / tiles);
        s -= split * tiles;
    }
    const uint32_t group = s / (8 * tiles_n), rest = s - group * (8 * tiles_n), high = min(8u, tiles_m - 8 * group);
    tn = (int)(high == 8 ? rest / 8 : rest / high);
    tm = (int)(8 * group + rest - tn * high);
    return true;
}
static int64_t tile_grid(int64_t tiles_m, int64_t tiles_n, int splits) { return (tiles_m * tiles_n * splits + 7) / 8 * 8; }

constexpr int lds_of_tile(int bm, int bn, int x_slots) { return 128 * (x_slots * bm + 2 * bn); }
// (as many wavefronts on a SIMD as there are workgroups of four whose LDS a compute unit holds)
template <class T, int BM, int BN, int WM, int WN, int XS, bool DIRECT>
__global__ void __launch_bounds__(WM *WN *kWave, 163840 / lds_of_tile(BM, BN, XS)) linear_block_kernel(LinearParams p) {
    constexpr int NW = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr int kLoadsX = BM / 8 / NW, kLoadsW = BN / 8 / NW, kLoads = kLoadsX + kLoadsW;      // of eight rows of 64 columns
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "");
    constexpr int kX = BM * 128, kW = BN * 128;                        // bytes of a block's rows of x and of weight: XS and two of them
    __shared__ __attribute__((aligned(1024))) char lds[lds_of_tile(BM, BN, XS)];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int tile_m, tile_n, split;
    if (!tile_of((p.m + BM - 1) / BM, (p.n + BN - 1) / BN, p.splits, tile_m, tile_n, split)) return;
    const int i0 = tile_m * BM, j0 = tile_n * BN;
    // Sixteen-byte groups of a row lie in LDS at their index XOR the row's last three bits, so that eight neighbouring rows
    // read at one index meet eight different groups of banks.
    const int row8 = lane >> 3, group = (lane & 7) ^ row8;
    // this part's blocks of 64 columns; the last one of all may be cut off
    const uint32_t all_blocks = (uint32_t)(p.k + 63) >> 6;
    int block0 = 0, blocks = (int)all_blocks;
    if (p.splits > 1) {
        block0 = (int)(all_blocks * (uint32_t)split / (uint32_t)p.splits);
        blocks = (int)(all_blocks * (uint32_t)(split + 1) / (uint32_t)p.splits) - block0;
    }
    const int cut = split == p.splits - 1 ? p.k & 63 : 0;             // the columns of a last block that is cut off, or 0
    // Columns of this lane's group of a cut block that lie behind the row's end, or behind its last whole group where rows are aligned:
    // the group is loaded from so much further in front (eight columns in front of the block at most, and k >= 8) and mended in LDS.
    const int over = max(8 * group + 8 - (DIRECT ? cut & ~7 : cut), 0);
    const char *xb = (const char *)(p.x + i0 * p.x_stride + 64 * (int64_t)block0 - 8), *wb = (const char *)(p.w + j0 * p.w_stride + 64 * (int64_t)block0 - 8);
    uint32_t at[kLoads];               // (from eight columns in front of the block on)
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
        const int row = ((q < kLoadsX ? q : q - kLoadsX) * NW + wv) * 8 + row8;
        at[q] = 2u * (uint32_t)((q < kLoadsX ? min(row, p.m - 1 - i0) * (int)p.x_stride : min(row, p.n - 1 - j0) * (int)p.w_stride) + 8 * group + 8);
    }
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds + wv * 1024;
    U4 held[DIRECT ? 1 : kLoads];      // rows at any alignment pass through registers
    // Load q of block t: of x into the slot at x_slot, or of weight at w_slot.
    auto load_part = [&](int x_slot, int w_slot, int t, int q) {
        const char *base = (q < kLoadsX ? xb : wb) + 128 * (int64_t)t;
        if constexpr (DIRECT) load_lds(lds_base + (q < kLoadsX ? x_slot + q * (NW * 1024) : w_slot + (q - kLoadsX) * (NW * 1024)), base, at[q]);
        else held[q] = load16((const uint16_t *)(base + at[q]));
    };
    auto store_part = [&](int x_slot, int w_slot, int q) {
        if constexpr (!DIRECT)
            *(U4 *)(lds + (q < kLoadsX ? x_slot + q * (NW * 1024) : w_slot + (q - kLoadsX) * (NW * 1024)) + wv * 1024 + 16 * lane) = held[q];
    };
    const int wm = wv / WN, wn = wv % WN;
    const int xrow = (wm * (BM / WM) + (lane & 31)) * 128, wrow = (wn * (BN / WN) + (lane & 31)) * 128;
    const int first = ((lane >> 5) ^ (lane & 7)) * 16;
    F16v acc[TM][TN] = {};
    U4 frag[2][2][TM + TN];            // [half of a block][step of 16 columns][rows of x, rows of weight]
    auto read_part = [&](int x_slot, int w_slot, int half, int q) {
        const int s = q / (TM + TN), f = q % (TM + TN), g = first ^ (32 * (2 * half + s));
        frag[half][s][f] = *(const U4 *)(lds + ((f < TM ? x_slot + xrow : w_slot + wrow) + g) + (f < TM ? f : f - TM) * 4096);
    };
    constexpr int kReads = 2 * (TM + TN), kProducts = 2 * TM * TN;
    // The products of one half of a block, and spread among them: the reads of the other half (of the block in the slots xr, wr), the
    // loads [L0, L1) of block t_load into xl, wl, and the stores [S0, S1) to xs, ws of what passes through registers.
    auto phase = [&](auto which, auto l0, auto l1, auto s0, auto s1, int xr, int wr, int xl, int wl, int t_load, int xs, int ws) {
        constexpr int half = decltype(which)::value, L0 = decltype(l0)::value, L = decltype(l1)::value - L0, S0 = decltype(s0)::value, S = decltype(s1)::value - S0;
#pragma unroll
        for (int q = 0; q < kProducts; ++q) {
#pragma unroll
            for (int r = q * kReads / kProducts; r < (q + 1) * kReads / kProducts; ++r) read_part(xr, wr, half ^ 1, r);
#pragma unroll
            for (int l = L0 + q * L / kProducts; l < L0 + (q + 1) * L / kProducts; ++l) load_part(xl, wl, t_load, l);
#pragma unroll
            for (int l = S0 + q * S / kProducts; l < S0 + (q + 1) * S / kProducts; ++l) store_part(xs, ws, l);
            const int s = q / (TM * TN), a = q / TN % TM, b = q % TN;
            acc[a][b] = mma32<T>(frag[half][s][TM + b], frag[half][s][a], acc[a][b]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto step_back = [&]() {
#pragma unroll
        for (int q = 0; q < kLoads; ++q) at[q] -= 2u * (uint32_t)over;
    };
    // Zeros behind the row's end in a cut block that has arrived.
    auto mend = [&](int x_slot, int w_slot) {
        if (over) {
#pragma unroll
            for (int q = 0; q < kLoads; ++q) {
                U4 *mine = (U4 *)(lds + (q < kLoadsX ? x_slot + q * (NW * 1024) : w_slot + (q - kLoadsX) * (NW * 1024)) + wv * 1024 + 16 * lane);
                if constexpr (DIRECT) {
                    U4 v = {0, 0, 0, 0};
                    if (8 * group < cut) {
                        const int row = ((q < kLoadsX ? q : q - kLoadsX) * NW + wv) * 8 + row8;
                        v = load_tail(q < kLoadsX ? p.x + min(i0 + row, p.m - 1) * p.x_stride : p.w + min(j0 + row, p.n - 1) * p.w_stride, p.k - cut + 8 * group, p.k);
                    }
                    *mine = v;
                } else {
                    *mine = shift_out(*mine, over);
                }
            }
        }
        __syncthreads();
    };
    constexpr std::integral_constant<int, 0> none;
    constexpr std::integral_constant<int, 1> second;
    constexpr std::integral_constant<int, kLoadsX> x_end;
    constexpr std::integral_constant<int, kLoads> all;
    if (blocks > 0) {
        // Slots of block t: x in t % XS, weight in t % 2.  A block's slots are free when the middle of it is reached, where its second
        // half has been read; from there on weight of block t + 2 is loaded, and x too.  With a third slot x of block t + 2 is loaded
        // in the first half of block t already: loads then come evenly, and may take longer.
        constexpr bool kThird = XS == 3;
        int x0 = 0, x1 = kX, x2 = XS == 3 ? 2 * kX : 0, w0 = XS * kX, w1 = w0 + kW;       // of blocks t, t + 1, t + 2
        if (cut && blocks == 1) step_back();
#pragma unroll
        for (int q = 0; q < kLoads; ++q) load_part(x0, w0, 0, q);
#pragma unroll
        for (int q = 0; q < kLoads; ++q) store_part(x0, w0, q);
        wait_and_meet<0>();
        if (cut && blocks == 1) mend(x0, w0);
#pragma unroll
        for (int q = 0; q < kReads; ++q) read_part(x0, w0, 0, q);
        if (cut && blocks == 2) step_back();
#pragma unroll
        for (int q = 0; q < kLoads; ++q) load_part(x1, w1, min(1, blocks - 1), q);
        if constexpr (kThird) {
#pragma unroll
            for (int q = 0; q < kLoadsX; ++q) store_part(x1, w1, q);
        }
        auto step = [&](int t, auto near_end) {
            constexpr bool kNearEnd = decltype(near_end)::value;
            // (behind the last block: that block again, for nobody)
            const int t2 = min(t + 2, blocks - 1);
            if (kNearEnd && t + 3 == blocks) step_back();
            if constexpr (kThird) phase(none, none, x_end, x_end, all, x0, w0, x2, 0, t2, 0, w1);
            else phase(none, none, none, none, all, x0, w0, 0, 0, 0, x1, w1);
            wait_and_meet<kThird && DIRECT ? kLoadsX : 0>();          // block t + 1 is there, and nobody reads block t any more
            if (kNearEnd && t + 2 == blocks) mend(x1, w1);
            if constexpr (kThird) phase(second, x_end, all, none, x_end, x1, w1, 0, w0, t2, x2, 0);
            else phase(second, none, all, none, none, x1, w1, x0, w0, t2, 0, 0);
            const int x = x0, w = w0;
            x0 = x1;
            x1 = kThird ? x2 : x;
            x2 = x;
            w0 = w1;
            w1 = w;
        };
        // (the steps that a cut block asks more of have a loop of their own: 4001 x 50256 x 4096 1,377 us, in one loop 1,409)
        const int calm = cut ? blocks - 3 : blocks;
        int t = 0;
        for (; t < calm; ++t) step(t, std::false_type());
        for (; t < blocks; ++t) step(t, std::true_type());
        wait_and_meet<0>();
    }
    // The result goes through LDS, 32 rows of a wavefront's part at a time, so that a row's columns leave next to each other:
    // the lanes hold one row each, four columns at a time.  (The padding of four columns spreads the rows over the banks.)
    // A batch of rows at a time: their reads and their stores are under way together, and so is the residual of the next batch (but in
    // the smallest tiles, which have few registers and other workgroups beside them).
    constexpr int kCols = 32 * TN, kPitch = kCols + 4, kLanesPerRow = kCols / 4;
    constexpr int kStep = 64 / kLanesPerRow, kBatch = kStep >= 4 ? 4 : 8, kRows = kBatch * kStep;
    const int j = j0 + wn * kCols + 4 * (lane % kLanesPerRow), i = i0 + wm * (BM / WM) + lane / kLanesPerRow;
    const int top = i0 + wm * (BM / WM), left = j0 + wn * kCols;                       // of this wavefront
    const bool whole = i0 + BM <= p.m && j0 + BN <= p.n;
    const uint32_t size = p.out_dtype == BPE_F32 ? 4 : 2, column_at = 4u * (lane % kLanesPerRow);
    const uint32_t out_at = size * ((uint32_t)(lane / kLanesPerRow) * (uint32_t)p.out_stride + column_at);
    const uint32_t res_at = size * ((uint32_t)(lane / kLanesPerRow) * (uint32_t)p.residual_stride + column_at);
    const uint32_t part_at = 4 * ((uint32_t)(lane / kLanesPerRow) * (uint32_t)p.part_stride + column_at);
    constexpr bool kAhead = kStep < 8;
    U4 res[kBatch], next[kAhead ? kBatch : 1];
    F4 bias = {0, 0, 0, 0};
    if (p.splits == 1) {
        bias = bias_of(p, j);
        if (kAhead && whole) fetch_whole(p, top, kStep, left, res_at, next);
        else if (kAhead) fetch(p, i, kStep, j, next);
    }
    static_assert(NW * 32 * kPitch * 4 <= XS * kX + 2 * kW, "the rows of all wavefronts fit the buffers");
    float *stage = (float *)lds + wv * (32 * kPitch);
    const float *mine = stage + lane / kLanesPerRow * kPitch + 4 * (lane % kLanesPerRow);
#pragma unroll 1
    for (int a = 0; a < TM; ++a) {
#pragma unroll
        for (int a_is = 0; a_is < TM; ++a_is) {           // (the registers of acc have no index at run time)
            if (a != a_is) continue;
#pragma unroll
            for (int b = 0; b < TN; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *(F4 *)(stage + (lane & 31) * kPitch + 32 * b + 8 * e + 4 * (lane >> 5)) =
                        F4{acc[a_is][b][4 * e], acc[a_is][b][4 * e + 1], acc[a_is][b][4 * e + 2], acc[a_is][b][4 * e + 3]};
        }
        wave_sync();
#pragma unroll 1
        for (int r = 0; r < 32; r += kRows) {
            F4 v[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) v[u] = *(const F4 *)(mine + (r + u * kStep) * kPitch);
            const int row = i + 32 * a + r;
            if (p.splits == 1 && whole) {
                if constexpr (kAhead) {
#pragma unroll
                    for (int u = 0; u < kBatch; ++u) res[u] = next[u];
                    if (32 * a + r + kRows < BM / WM) fetch_whole(p, top + 32 * a + r + kRows, kStep, left, res_at, next);
                } else {
                    fetch_whole(p, top + 32 * a + r, kStep, left, res_at, res);
                }
                put_whole(p, top + 32 * a + r, kStep, left, out_at, v, bias, res);
                continue;
            }
            if (j >= p.n) continue;
            if (p.splits > 1) {
#pragma unroll
                for (int u = 0; u < kBatch; ++u) {                  // (so few tiles that the lanes' offsets fit 32 bits)
                    char *to = (char *)(p.part + ((int64_t)split * p.m + top + 32 * a + r + u * kStep) * p.part_stride + left);
                    if (whole || row + u * kStep < p.m) *(F4 *)(to + part_at) = v[u];
                }
            } else {
                if constexpr (kAhead) {
#pragma unroll
                    for (int u = 0; u < kBatch; ++u) res[u] = next[u];
                    if (32 * a + r + kRows < BM / WM) fetch(p, row + kRows, kStep, j, next);
                } else {
                    fetch(p, row, kStep, j, res);
                }
                put(p, row, kStep, j, v, bias, res);
            }
        }
        wave_sync();
    }
}

// Rows that lie 2^21 elements apart or more, or have fewer than eight columns: a workgroup of four wavefronts makes 64 x 64 of out, a
// wavefront 32 x 32 (two by two products of 16 x 16), 32 of k at a time through registers into LDS, one step after the other; bound by
// the wait for each step's loads.  200 x 2048 x 2048 with rows
// so far apart 39 us, in tiles 13; 200 x 2048 x 7 6.3 us, of which 5 are the launch.
template <class T>
__global__ void __launch_bounds__(kGroupThreads) linear_tile_kernel(LinearParams p) {
    __shared__ U4 xs[64][4], ws[64][4];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    int tile_m, tile_n, split;
    if (!tile_of((p.m + 63) / 64, (p.n + 63) / 64, 1, tile_m, tile_n, split)) return;
    const int i0 = tile_m * 64, j0 = tile_n * 64;
    const int wi = 32 * (wv >> 1), wj = 32 * (wv & 1);
    const uint16_t *xr = p.x + min(i0 + (tid >> 2), p.m - 1) * p.x_stride, *wr = p.w + min(j0 + (tid >> 2), p.n - 1) * p.w_stride;
    F4 acc[2][2] = {};
    for (int t = 0; t < p.k; t += 32) {
        __syncthreads();
        xs[tid >> 2][tid & 3] = load_tail(xr, t + 8 * (tid & 3), p.k);
        ws[tid >> 2][tid & 3] = load_tail(wr, t + 8 * (tid & 3), p.k);
        __syncthreads();
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b)
                acc[a][b] = mma16<T>(ws[wj + 16 * b + (lane & 15)][lane >> 4], xs[wi + 16 * a + (lane & 15)][lane >> 4], acc[a][b]);
    }
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int i = i0 + wi + 16 * a + (lane & 15), j = j0 + wj + 16 * b + 4 * (lane >> 4);
            if (i < p.m && j < p.n) put4(p, i, j, acc[a][b]);
        }
}

// Adds up the parts of every four neighbours of a row, part by part (so in one order), and finishes them.  Bound by its launch and by
// memory: about 4 us and the parts at 6.7 TB/s.
__global__ void __launch_bounds__(kGroupThreads) linear_join_kernel(LinearParams p) {
    const int64_t groups = p.part_stride / 4, total = groups * p.m, step = (int64_t)gridDim.x * kGroupThreads;
    for (int64_t g = (int64_t)blockIdx.x * kGroupThreads + threadIdx.x; g < total; g += step) {
        const int i = (int)(g / groups), j = 4 * (int)(g % groups);
        F4 v = {0, 0, 0, 0};
#pragma unroll 4
        for (int s = 0; s < p.splits; ++s) v += *(const F4 *)(p.part + ((int64_t)s * p.m + i) * p.part_stride + j);
        put4(p, i, j, v);
    }
}

// Which tiles a product of these sizes takes, and into how many parts k is cut: what an estimate of the time says.  A tile's
// row: its sides, how many of its workgroups a compute unit holds, us for a block of 64 columns when a workgroup waits for
// its loads alone, us for its first loads and its result, and the TFLOP/s of the whole chip when nothing else bounds it.  The
// numbers are fitted to the times of all tiles and parts on 93 sizes (m 5 to 8192, n 256 to 128000, k 64 to 4096) as these were before whole
// tiles left by uniform addresses; as they are now, the choice takes 2.4 % longer there than the best one on average, 19 % at worst.  (They are numbers that choose well;
// not every one is a property of its tile.)
struct LinearTile { int bm, bn, resident; double block_us, tile_us, tflops; };
constexpr LinearTile kLinearTiles[] = {
    {32, 128, 4, 0.43, 3.4, 434}, {32, 256, 2, 0.96, 3.3, 366}, {64, 128, 3, 0.57, 3.8, 500},
    {64, 256, 2, 0.526, 8.0, 576}, {128, 128, 2, 0.69, 5.3, 667}, {256, 256, 1, 1.15, 13.3, 1108}};
constexpr int kLinearTileCount = sizeof(kLinearTiles) / sizeof(kLinearTiles[0]);
struct LinearPlan { int tile, splits; };        // tile -1: linear_rows_kernel

static LinearPlan plan_linear(int64_t m, int64_t n, int64_t k) {
    // Every wavefront of linear_rows_kernel reads all of x: a row or four, or small weights (1 x 2048 x 2048 6.7 us and in tiles
    // 11; 16 x 2048 x 2048 6.4 and 11; 16 x 50256 x 1024 26.9 and 20.9; 4 x 100256 x 4096 138 and 141, 8 rows 175 and 147).
    if (m <= 4 || (m <= 16 && n * k <= (1 << 24))) return {-1, 1};
    LinearPlan best = {0, 1};
    double least = 1e300;
    const double blocks = (double)std::max<int64_t>((k + 63) >> 6, 1);
    for (int t = 0; t < kLinearTileCount; ++t) {
        const LinearTile &l = kLinearTiles[t];
        const double tiles = (double)((m + l.bm - 1) / l.bm) * (double)((n + l.bn - 1) / l.bn);
        for (int splits = 1; splits <= 16; splits *= 2) {
            if (splits > 1 && (tiles * splits > 768 || blocks < 2 * splits)) break;
            const double groups = tiles * splits, per = std::ceil(blocks / splits);
            const double compute = std::ceil(groups / 256) * per * (2.0 * l.bm * l.bn * 64) / (l.tflops * 1e6 / 256);
            const double rounds = groups / (256.0 * l.resident), wait = std::ceil(rounds) * per * l.block_us;
            // weights, x and the result from and to memory, slower from few workgroups; what all tiles load, through the L2s
            const double spread = groups < 384 ? 1.0 + (384 - groups) / 1230 : 1.0;
            const double memory = (2.0 * ((double)n * k + (double)m * k) * spread + 3.1 * (double)m * n) / 4.55e6 + 2.0 * tiles * (l.bm + l.bn) * k / 2.46e7;
            const double join = splits > 1 ? 3.8 + (double)splits * m * n * 8 / 6.7e6 : 0.0;
            const double us = std::max(std::max(compute, wait), memory) + std::max(rounds, 1.0) * l.tile_us + join;
            if (us < least) { least = us; best = {t, splits}; }
        }
    }
    return best;
}
static int64_t part_stride_of(int64_t n) { return (n + 3) & ~3ll; }

template <class T>
static int launch_linear(LinearParams &p, LinearPlan plan, void *workspace, void *stream) {
    const char *what = "bpe_linear launch";
    p.splits = 1;
    const bool direct = p.x_stride % 8 == 0 && p.w_stride % 8 == 0 && !(((uintptr_t)p.x | (uintptr_t)p.w) & 15);
    // (rows at odd addresses cost linear_rows_kernel more than they cost a tile: 1 x 50256 x 1023 46 us and in tiles 27, 4 x 100256 x
    // 4096 448 and 209; 1 x 20000 x 1023 20 and 21)
    if (plan.tile < 0 && !direct && (int64_t)p.n * p.k > (1 << 24)) plan = {0, 1};
    if (plan.tile < 0) {
        constexpr int64_t kAtOnce = 16 * (kMaxThreads / kGroupThreads - 1);           // columns of a launch
        for (int64_t done = 0; done < p.n; done += kAtOnce) {
            LinearParams run = p;
            run.n = (int32_t)std::min(p.n - done, kAtOnce);
            run.w = p.w + done * p.w_stride;
            run.out = (char *)p.out + done * dtype_bytes(p.out_dtype);
            if (p.bias) run.bias = (const char *)p.bias + done * dtype_bytes(p.bias_dtype);
            if (p.residual) run.residual = (const char *)p.residual + done * dtype_bytes(p.out_dtype);
            const int rc = launch(linear_rows_kernel<T>, dim3((unsigned)(((int64_t)run.n + 15) / 16)), kGroupThreads, run, stream, what);
            if (rc != BPE_OK) return rc;
        }
        return BPE_OK;
    }
    // A tile's rows are addressed by 32-bit offsets (of out and the residual the eight that a wavefront writes at a time), and every load is of eight columns: rows that lie further apart or are shorter
    // take the simple kernel.
    const bool far = p.x_stride >= (1 << 21) || p.w_stride >= (1 << 21) || p.out_stride >= (1 << 25) || p.residual_stride >= (1 << 25) || p.k < 8;
    const int64_t bm = far ? 64 : kLinearTiles[plan.tile].bm, bn = far ? 64 : kLinearTiles[plan.tile].bn;
    p.splits = far ? 1 : plan.splits;
    const int64_t grid = tile_grid((p.m + bm - 1) / bm, (p.n + bn - 1) / bn, p.splits);
    if (grid >= kMaxThreads / kGroupThreads) { set_error("bpe_linear: m %d and n %d are too large together", p.m, p.n); return BPE_ERR_SIZE; }
    if (far) return launch(linear_tile_kernel<T>, dim3((unsigned)grid), kGroupThreads, p, stream, what);
    p.part = (float *)workspace;
    p.part_stride = (int32_t)part_stride_of(p.n);
    void (*kernel)(LinearParams) = nullptr;
#define TILE(INDEX, BM, BN, WM, WN, XS) \
    case INDEX: \
        static_assert(kLinearTiles[INDEX].bm == BM && kLinearTiles[INDEX].bn == BN, ""); \
        kernel = direct ? linear_block_kernel<T, BM, BN, WM, WN, XS, true> : linear_block_kernel<T, BM, BN, WM, WN, XS, false>; \
        break
    switch (plan.tile) {
        TILE(0, 32, 128, 1, 4, 2);
        TILE(1, 32, 256, 1, 4, 2);
        TILE(2, 64, 128, 1, 4, 2);
        TILE(3, 64, 256, 1, 4, 2);
        TILE(4, 128, 128, 2, 2, 3);
        TILE(5, 256, 256, 2, 2, 3);
    }
#undef TILE
    const int rc = launch(kernel, dim3((unsigned)grid), kGroupThreads, p, stream, what);
    if (rc != BPE_OK || p.splits == 1) return rc;
    const int64_t groups = p.part_stride / 4 * (int64_t)p.m;
    return launch(linear_join_kernel, dim3((unsigned)std::min<int64_t>((groups + kGroupThreads - 1) / kGroupThreads, 2048)), kGroupThreads, p, stream, what);
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

static int64_t linear_need(const LinearPlan &plan, int64_t m, int64_t n) { return plan.splits > 1 ? 4 * (int64_t)plan.splits * m * part_stride_of(n) : 0; }

extern "C" int64_t bpe_linear_workspace_bytes(int64_t m, int64_t n, int64_t k) {
    if (!linear_sizes_ok(m, n, k)) return BPE_ERR_SIZE;
    return linear_need(plan_linear(m, n, k), m, n);
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
    const LinearPlan plan = plan_linear(m, n, k);
    const int64_t need = linear_need(plan, m, n);
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
    p.x_stride = m > 1 ? x_stride : 0; p.w_stride = n > 1 ? weight_stride : 0;        // (of one row the stride says nothing)
    p.m = (int32_t)m; p.n = (int32_t)n; p.k = (int32_t)k;
    p.bias = bias; p.bias_dtype = bias_dtype; p.activation = activation;
    p.residual = residual; p.residual_stride = residual && m > 1 ? residual_stride : 0;
    p.out = out; p.out_stride = m > 1 ? out_stride : 0; p.out_dtype = out_dtype;
    return dtype == BPE_BF16 ? launch_linear<Bf16>(p, plan, workspace, stream) : launch_linear<F16>(p, plan, workspace, stream);
}
