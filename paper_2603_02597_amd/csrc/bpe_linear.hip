// out = activation(x weight^T + bias) + residual on the matrix cores: the projection of hidden states onto a vocabulary,
// and the small blocks in front of it.
#include <algorithm>
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

// What a call's epilogue is made of; the kernels are compiled for the output's type, the rest are branches that all lanes take together.
template <class OUT>
struct Epilogue {
    const LinearParams &p;
    __device__ __forceinline__ float finish(int i, int j, float v) const {
        if (p.bias) v += load_as_float(p.bias, j, p.bias_dtype);
        v = activate(v, p.activation);
        if (p.residual) v += to_float<OUT>(((const typename OUT::raw *)p.residual)[i * p.residual_stride + j]);
        return v;
    }
    __device__ __forceinline__ void put(int i, int j, float v) const {
        ((typename OUT::raw *)p.out)[i * p.out_stride + j] = from_float<OUT>(finish(i, j, v));
    }
    // Four neighbours of a row; whole = all four exist.
    __device__ __forceinline__ void put4(int i, int j, F4 v) const {
        typedef typename OUT::raw Raw4 __attribute__((ext_vector_type(4), aligned(sizeof(typename OUT::raw))));
        if (j + 3 >= p.n) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (j + e < p.n) put(i, j + e, v[e]);
            return;
        }
        if (p.bias) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += load_as_float(p.bias, j + e, p.bias_dtype);
        }
        if (p.activation != BPE_ACT_NONE) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = activate(v[e], p.activation);
        }
        if (p.residual) {
            const Raw4 r = *(const Raw4 *)((const typename OUT::raw *)p.residual + i * p.residual_stride + j);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += to_float<OUT>(r[e]);
        }
        Raw4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = from_float<OUT>(v[e]);
        *(Raw4 *)((typename OUT::raw *)p.out + i * p.out_stride + j) = o;
    }
};

// Sixteen bytes at any even address: the hardware asks for no more.
typedef uint32_t U4Any __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ U4 load16(const uint16_t *at) { return *(const U4Any *)at; }

// Eight elements of a row from column t on, zeros behind the row's end.
__device__ __forceinline__ U4 load_tail(const uint16_t *row, int t, int k) {
    if (t + 8 <= k) return load16(row + t);
    H8 v = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (t + e < k) v[e] = row[t + e];
    return __builtin_bit_cast(U4, v);
}

// Up to 64 rows of x: the call is as long as reading weight takes, so weight goes from memory straight into the matrix
// cores' registers and every byte of it is asked for once.  A workgroup takes 16 NT rows of weight, its four wavefronts a
// quarter of k each (a long row is 4 streams, and a vocabulary of few rows still fills the chip); their sums meet in LDS.
// weight is the left operand: a lane ends with four neighbouring columns of one row of out.
constexpr int kRowsAhead = 2;        // steps of 32 columns of k whose loads are under way while one is multiplied
template <class T, class OUT, int MT, int NT>
__global__ void __launch_bounds__(kGroupThreads) linear_rows_kernel(LinearParams p) {
    __shared__ F4 part[kWavesPerGroup][MT * NT][kWave];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int j0 = blockIdx.x * (16 * NT);
    const int steps = p.k >> 5, from = (int)((int64_t)steps * wv / kWavesPerGroup), to = (int)((int64_t)steps * (wv + 1) / kWavesPerGroup);
    const uint16_t *w[NT], *x[MT];
#pragma unroll
    for (int b = 0; b < NT; ++b) w[b] = p.w + min(j0 + 16 * b + (lane & 15), p.n - 1) * p.w_stride + 8 * (lane >> 4);
#pragma unroll
    for (int a = 0; a < MT; ++a) x[a] = p.x + min(16 * a + (lane & 15), p.m - 1) * p.x_stride + 8 * (lane >> 4);
    F4 acc[MT][NT] = {};
    U4 wf[kRowsAhead][NT], xf[kRowsAhead][MT];
    auto load = [&](int u, int step) {
#pragma unroll
        for (int b = 0; b < NT; ++b) wf[u][b] = load16(w[b] + 32 * step);
#pragma unroll
        for (int a = 0; a < MT; ++a) xf[u][a] = load16(x[a] + 32 * step);
    };
    auto multiply = [&](int u) {
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int b = 0; b < NT; ++b) acc[a][b] = mma16<T>(wf[u][b], xf[u][a], acc[a][b]);
    };
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
    if (wv == kWavesPerGroup - 1 && (p.k & 31)) {
        const int t = p.k & ~31;
#pragma unroll
        for (int b = 0; b < NT; ++b) wf[0][b] = load_tail(w[b] - 8 * (lane >> 4), t + 8 * (lane >> 4), p.k);
#pragma unroll
        for (int a = 0; a < MT; ++a) xf[0][a] = load_tail(x[a] - 8 * (lane >> 4), t + 8 * (lane >> 4), p.k);
        multiply(0);
    }
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b) part[wv][a * NT + b][lane] = acc[a][b];
    __syncthreads();
    const Epilogue<OUT> epilogue = {p};
    for (int q = wv; q < MT * NT; q += kWavesPerGroup) {
        F4 v = part[0][q][lane];
#pragma unroll
        for (int s = 1; s < kWavesPerGroup; ++s) v += part[s][q][lane];
        const int i = 16 * (q / NT) + (lane & 15), j = j0 + 16 * (q % NT) + 4 * (lane >> 4);
        if (i < p.m && j < p.n) epilogue.put4(i, j, v);
    }
}

// What a wavefront's lanes have written to LDS is there for its other lanes.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// More rows.  A workgroup makes BM x BN of out, WM x WN wavefronts side by side, 64 columns of k at a time through two buffers in LDS.
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
// This wavefront's loads have arrived and its reads of LDS are done; then the other wavefronts'.
__device__ __forceinline__ void wait_and_meet() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Which tile of out a workgroup makes.  Workgroups go round the eight chiplets by their index, and each chiplet has an L2 of its
// own: so every chiplet gets a run of neighbouring tiles, eight rows of tiles by as many columns as it takes.
__device__ __forceinline__ bool tile_of(int64_t tiles_m, int64_t tiles_n, int64_t &tm, int64_t &tn) {
    const int64_t total = tiles_m * tiles_n, per = (total + 7) / 8, s = (int64_t)(blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int64_t)(blockIdx.x >> 3) >= per || s >= total) return false;
    const int64_t group = s / (8 * tiles_n), rest = s % (8 * tiles_n), high = min<int64_t>(8, tiles_m - 8 * group);
    tm = 8 * group + rest % high;
    tn = rest / high;
    return true;
}
static int64_t tile_grid(int64_t tiles_m, int64_t tiles_n) { return (tiles_m * tiles_n + 7) / 8 * 8; }

template <class T, class OUT, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(WM *WN *kWave) linear_block_kernel(LinearParams p) {
    constexpr int NW = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr int kLoadsX = BM / 8 / NW, kLoadsW = BN / 8 / NW, kLoads = kLoadsX + kLoadsW;      // of eight rows of 64 columns
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "");
    constexpr int kBlock = (BM + BN) * 128;
    __shared__ __attribute__((aligned(1024))) char lds[2 * kBlock];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int64_t tile_m, tile_n;
    if (!tile_of((p.m + BM - 1) / BM, (p.n + BN - 1) / BN, tile_m, tile_n)) return;
    const int i0 = (int)tile_m * BM, j0 = (int)tile_n * BN;
    // Sixteen-byte groups of a row lie in LDS at their index XOR the row's last three bits, so that eight neighbouring rows
    // read at one index meet eight different groups of banks.
    const int row8 = lane >> 3, group = (lane & 7) ^ row8;
    const char *xb = (const char *)(p.x + i0 * p.x_stride), *wb = (const char *)(p.w + j0 * p.w_stride);
    uint32_t at[kLoads];
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
        const int row = ((q < kLoadsX ? q : q - kLoadsX) * NW + wv) * 8 + row8;
        at[q] = 2u * (uint32_t)((q < kLoadsX ? min(row, p.m - 1 - i0) * (int)p.x_stride : min(row, p.n - 1 - j0) * (int)p.w_stride) + 8 * group);
    }
    const int blocks = p.k >> 6;
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds + wv * 1024;
    auto load_part = [&](int buf, int t, int q) {
        load_lds(lds_base + buf + q * (NW * 1024), (q < kLoadsX ? xb : wb) + 128 * (int64_t)t, at[q]);
    };
    const int wm = wv / WN, wn = wv % WN;
    const int xrow = (wm * (BM / WM) + (lane & 31)) * 128, wrow = BM * 128 + (wn * (BN / WN) + (lane & 31)) * 128;
    const int first = ((lane >> 5) ^ (lane & 7)) * 16;
    F16v acc[TM][TN] = {};
    U4 frag[2][2][TM + TN];            // [half of a block][step of 16 columns][rows of x, rows of weight]
    auto read_part = [&](int buf, int half, int q) {
        const int s = q / (TM + TN), f = q % (TM + TN), g = first ^ (32 * (2 * half + s));
        frag[half][s][f] = *(const U4 *)(lds + (buf + (f < TM ? xrow : wrow) + g) + (f < TM ? f : f - TM) * 4096);
    };
    constexpr int kReads = 2 * (TM + TN), kProducts = 2 * TM * TN;
    // The products of one half of a block, with the reads of the other half (of the block in `reads`) and, in the second half, the loads
    // of a later block spread among them.
    auto phase = [&](auto which, int reads, int loads, int t_load) {
        constexpr int half = decltype(which)::value;
#pragma unroll
        for (int q = 0; q < kProducts; ++q) {
#pragma unroll
            for (int r = q * kReads / kProducts; r < (q + 1) * kReads / kProducts; ++r) read_part(reads, half ^ 1, r);
            if constexpr (half == 1) {
#pragma unroll
                for (int l = q * kLoads / kProducts; l < (q + 1) * kLoads / kProducts; ++l) load_part(loads, t_load, l);
            }
            const int s = q / (TM * TN), a = q / TN % TM, b = q % TN;
            acc[a][b] = mma32<T>(frag[half][s][TM + b], frag[half][s][a], acc[a][b]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (blocks > 0) {
#pragma unroll
        for (int q = 0; q < kLoads; ++q) load_part(0, 0, q);
        wait_and_meet();
#pragma unroll
        for (int q = 0; q < kReads; ++q) read_part(0, 0, q);
#pragma unroll
        for (int q = 0; q < kLoads; ++q) load_part(kBlock, min(1, blocks - 1), q);
        int mine = 0;
        for (int t = 0; t < blocks; ++t) {
            phase(std::integral_constant<int, 0>(), mine, 0, 0);
            wait_and_meet();             // block t + 1 is there, and nobody reads block t any more
            // (behind the last block but one: that block again, for nobody)
            phase(std::integral_constant<int, 1>(), mine ^ kBlock, mine, min(t + 2, blocks - 1));
            mine ^= kBlock;
        }
        wait_and_meet();
    }
    // The columns behind the last whole block, filled up with zeros.
    if (64 * blocks < p.k) {
#pragma unroll 1
        for (int q = 0; q < kLoads; ++q) {
            const int row = ((q < kLoadsX ? q : q - kLoadsX) * NW + wv) * 8 + row8;
            const uint16_t *from = q < kLoadsX ? p.x + min(i0 + row, p.m - 1) * p.x_stride : p.w + min(j0 + row, p.n - 1) * p.w_stride;
            *(U4 *)(lds + (q * NW + wv) * 1024 + 16 * lane) = load_tail(from, 64 * blocks + 8 * group, p.k);
        }
        __syncthreads();
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int q = 0; q < kReads; ++q) read_part(0, half, q);
#pragma unroll
            for (int q = 0; q < kProducts; ++q) {
                const int s = q / (TM * TN), a = q / TN % TM, b = q % TN;
                acc[a][b] = mma32<T>(frag[half][s][TM + b], frag[half][s][a], acc[a][b]);
            }
        }
        __syncthreads();
    }
    // The result goes through LDS, 32 rows of a wavefront's part at a time, so that a row's columns leave next to each other:
    // the lanes hold one row each, four columns at a time.  (The padding of four columns spreads the rows over the banks.)
    constexpr int kCols = 32 * TN, kPitch = kCols + 4, kLanesPerRow = kCols / 4;
    static_assert(NW * 32 * kPitch * 4 <= 2 * kBlock, "the rows of all wavefronts fit the buffers");
    float *stage = (float *)lds + wv * (32 * kPitch);
    const Epilogue<OUT> epilogue = {p};
#pragma unroll
    for (int a = 0; a < TM; ++a) {
#pragma unroll
        for (int b = 0; b < TN; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *(F4 *)(stage + (lane & 31) * kPitch + 32 * b + 8 * e + 4 * (lane >> 5)) =
                    F4{acc[a][b][4 * e], acc[a][b][4 * e + 1], acc[a][b][4 * e + 2], acc[a][b][4 * e + 3]};
        wave_sync();
        const int j = j0 + wn * kCols + 4 * (lane % kLanesPerRow);
#pragma unroll 1
        for (int r = lane / kLanesPerRow; r < 32; r += 64 / kLanesPerRow) {
            const F4 v = *(const F4 *)(stage + r * kPitch + 4 * (lane % kLanesPerRow));
            const int i = i0 + wm * (BM / WM) + 32 * a + r;
            if (i < p.m && j < p.n) epilogue.put4(i, j, v);
        }
        wave_sync();
    }
}

// Any alignment and any k: a workgroup of four wavefronts makes 64 x 64 of out, a wavefront 32 x 32 (two by two products of 16 x 16),
// 32 of k at a time through registers into LDS.
template <class T, class OUT>
__global__ void __launch_bounds__(kGroupThreads) linear_tile_kernel(LinearParams p) {
    __shared__ U4 xs[64][4], ws[64][4];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    int64_t tile_m, tile_n;
    if (!tile_of((p.m + 63) / 64, (p.n + 63) / 64, tile_m, tile_n)) return;
    const int i0 = (int)tile_m * 64, j0 = (int)tile_n * 64;
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
    const Epilogue<OUT> epilogue = {p};
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int i = i0 + wi + 16 * a + (lane & 15), j = j0 + wj + 16 * b + 4 * (lane >> 4);
            if (i < p.m && j < p.n) epilogue.put4(i, j, acc[a][b]);
        }
}

template <class T, class OUT>
static int launch_linear(LinearParams &p, void *stream) {
    const char *what = "bpe_linear launch";
    if (p.m <= 64) {
        const int mt = (p.m + 15) / 16;
        const int64_t tiles = ((int64_t)p.n + 15) / 16;
        const int nt = mt == 1 ? 1 : tiles >= 2048 ? 4 : tiles >= 1024 ? 2 : 1;
        const dim3 grid((unsigned)((tiles + nt - 1) / nt));
#define ROWS(MT, NT) if (mt == MT && nt == NT) return launch(linear_rows_kernel<T, OUT, MT, NT>, grid, kGroupThreads, p, stream, what)
        ROWS(1, 1);
        ROWS(2, 1); ROWS(2, 2); ROWS(2, 4);
        ROWS(3, 1); ROWS(3, 2); ROWS(3, 4);
        ROWS(4, 1); ROWS(4, 2); ROWS(4, 4);
#undef ROWS
    }
    const bool direct = p.x_stride % 8 == 0 && p.w_stride % 8 == 0 && !(((uintptr_t)p.x | (uintptr_t)p.w) & 15) &&
                        p.x_stride < (1 << 21) && p.w_stride < (1 << 21);
    const int64_t tile = direct ? 256 : 64, grid = tile_grid((p.m + tile - 1) / tile, (p.n + tile - 1) / tile);
    if (grid > 0x7FFFFFFF) { set_error("bpe_linear: m %d and n %d are too large together", p.m, p.n); return BPE_ERR_SIZE; }
    if (direct) return launch(linear_block_kernel<T, OUT, 256, 256, 2, 2>, dim3((unsigned)grid), 256, p, stream, what);
    return launch(linear_tile_kernel<T, OUT>, dim3((unsigned)grid), kGroupThreads, p, stream, what);
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
    if (dtype == BPE_BF16) return out_dtype == BPE_F32 ? launch_linear<Bf16, F32>(p, stream) : launch_linear<Bf16, Bf16>(p, stream);
    return out_dtype == BPE_F32 ? launch_linear<F16, F32>(p, stream) : launch_linear<F16, F16>(p, stream);
}
