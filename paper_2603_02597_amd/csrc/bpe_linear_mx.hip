// out = activation(x weight^T + bias) + residual with weights of 4 bits on the matrix cores; x in 16 bits, or in 4 bits too.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "bpe_mx.h"
#include "bpe_tiles.h"

namespace bpe {

struct LinearMx4Params : TileParams {
    const void *x;                     // 16-bit rows, or panels
    const uint8_t *w;
    int64_t x_stride;
    int32_t k, panels;                 // of a row
};

struct Mx4 { static constexpr int kCode = BPE_MX4; };

// Sixteen bytes of two 4-bit operands, 32 x 32 x 64: lane l gives row l % 32, columns 32 (l / 32) ..+31 and their scale, the byte S of a word; the
// result lies as with mma32.  The scales are taken in by the operation itself.
typedef int I8 __attribute__((ext_vector_type(8)));
template <int S> __device__ __forceinline__ F16v mma_mx4(U4 a, U4 b, F16v c, uint32_t scale_a, uint32_t scale_b) {
    const I8 x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, S, (int)scale_a, S, (int)scale_b);
}

// Two elements of f16 as two bf16 parts each, which hold all 11 bits: no scale of a weight leaves the range of bf16, as it would that of f16.  The first part
// is the element cut off behind 8 bits, so the second has its sign or is 0; of an infinity the first is f16's largest number, cut off, and the second the infinity.
__device__ __forceinline__ void split_f16(uint32_t two, uint32_t &high, uint32_t &low) {
    constexpr float kMostF16 = 65504.0f;
    const float a = to_float<F16>((uint16_t)two), b = to_float<F16>((uint16_t)(two >> 16));
    const uint32_t ha = __builtin_bit_cast(uint32_t, __builtin_amdgcn_fmed3f(a, -kMostF16, kMostF16)) & 0xffff0000u;
    const uint32_t hb = __builtin_bit_cast(uint32_t, __builtin_amdgcn_fmed3f(b, -kMostF16, kMostF16)) & 0xffff0000u;
    const uint32_t la = __builtin_bit_cast(uint32_t, a - __builtin_bit_cast(float, ha)), lb = __builtin_bit_cast(uint32_t, b - __builtin_bit_cast(float, hb));
    high = __builtin_amdgcn_perm(hb, ha, 0x07060302);
    low = __builtin_amdgcn_perm(lb, la, 0x07060302);
}
// Weights for the second parts: the largest number in the place of an infinity (a weight of 2^128 and more), whose product with a part of 0 would be NaN.  The
// product with the first part is the infinity, and this one's has the same sign.  (NaN becomes a number: the first product has it.)
__device__ __forceinline__ U4 finite_of(U4 w) {
    typedef int16_t S8 __attribute__((ext_vector_type(8)));
    const H8 negative = __builtin_elementwise_min(__builtin_bit_cast(H8, w), (H8)0xff7f);
    return __builtin_bit_cast(U4, __builtin_elementwise_min(__builtin_bit_cast(S8, negative), (S8)0x7f7f));
}
constexpr float kMayBeInfinite = 0x1p126f;             // the least scale by which a code is 2^128 and more
// Eight elements of x times as many of weight; of f16 the second parts `low` by finite weights.
template <class T, bool X_LEFT = false> __device__ __forceinline__ F16v mma_by_weight(U4 w, U4 finite, U4 x, U4 low, F16v c) {
    c = X_LEFT ? mma32<Bf16>(x, w, c) : mma32<Bf16>(w, x, c);
    if constexpr (T::kCode == BPE_F16) c = X_LEFT ? mma32<Bf16>(low, finite, c) : mma32<Bf16>(finite, low, c);
    return c;
}
template <class T> __device__ __forceinline__ F16v mma_by_weight(U4 w, U4 x, F16v c) {
    U4 low = {0, 0, 0, 0};
    if constexpr (T::kCode == BPE_F16) {
        U4 high;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            uint32_t h, l;
            split_f16(x[d], h, l);
            high[d] = h;
            low[d] = l;
        }
        x = high;
    }
    return mma_by_weight<T>(w, finite_of(w), x, low, c);
}

// Products whose result leaves by put_wide take column 4 j + b of a wavefront's 128 in lane j of product b.  Of a group of 32 rows in LDS every
// four neighbours are turned by their number, so that the eight that a product reads, every fourth one, meet different banks, and a load
// still takes whole pieces of 64 bytes.  Where lane l of a load finds its sixteen bytes, where lane l of product b reads them, and its scale.
__device__ __forceinline__ uint32_t wide_source(int lane) {
    const int four = (lane & 31) >> 2;
    return (lane >> 5) * 512 + 16 * (4 * four + ((lane - four - (four >> 2)) & 3));
}
__device__ __forceinline__ int wide_place(int lane, int b) {
    const int four = lane & 7;
    return (lane >> 5) * 512 + 16 * (4 * four + ((b + four + (four >> 2)) & 3));
}
__device__ __forceinline__ int wide_scale(int lane, int b) { return (lane >> 5) * 128 + 4 * (4 * (lane & 7) + b); }

// A workgroup makes 32 x 32 of out, its four wavefronts a quarter of k's panels each; operands go from memory into the matrix cores' registers.  For
// what the tiles below cannot address, rows 2^21 elements apart (out and residual: 2^25), and for fewer than eight columns: a wavefront waits for each
// panel's loads.  200 x 2048 x 2048 bf16 with rows so far apart 12 us (in tiles 8), 200 x 2048 x 7 7.
template <class T>
__global__ void __launch_bounds__(kGroupThreads) linear_mx4_rows_kernel(LinearMx4Params p) {
    __shared__ F4 part[kWavesPerGroup][4][kWave];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, h = lane >> 5;
    int tile_m, tile_n, split;
    if (!tile_of((p.m + 31) / 32, (p.n + 31) / 32, 1, tile_m, tile_n, split)) return;
    const int i0 = tile_m * 32, j0 = tile_n * 32;
    F16v acc = {};
    for (int panel = wv; panel < p.panels; panel += kWavesPerGroup) {
        const uint8_t *w = p.w + ((int64_t)tile_n * p.panels + panel) * kPanelBytes;
        const uint32_t ws = *(const uint32_t *)(w + kPanelCodes + 4 * lane);
        if constexpr (T::kCode == BPE_MX4) {
            const uint8_t *x = (const uint8_t *)p.x + ((int64_t)tile_m * p.panels + panel) * kPanelBytes;
            const uint32_t xs = *(const uint32_t *)(x + kPanelCodes + 4 * lane);
#define STEP(S) acc = mma_mx4<S>(*(const U4 *)(w + 1024 * S + 16 * lane), *(const U4 *)(x + 1024 * S + 16 * lane), acc, ws, xs);
            STEP(0) STEP(1) STEP(2) STEP(3)
#undef STEP
        } else {
            const uint16_t *x = (const uint16_t *)p.x + min(i0 + r, p.m - 1) * p.x_stride;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const U4 codes = *(const U4 *)(w + 1024 * s + 16 * lane);
                const float scale = scale_of(ws >> 8 * s & 255);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int column = panel * kPanelCols + 64 * s + 32 * h + 8 * q;
                    acc = mma_by_weight<T>(bf16_of(codes[q], scale), load_tail(x, column, p.k), acc);
                }
            }
        }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) part[wv][q][lane] = F4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    __syncthreads();
    F4 v = part[0][wv][lane];
#pragma unroll
    for (int s = 1; s < kWavesPerGroup; ++s) v += part[s][wv][lane];
    const int i = i0 + r, j = j0 + 8 * wv + 4 * h;
    if (i < p.m && j < p.n) put4(p, i, j, v);
}

// More rows, both operands in 4 bits.  A workgroup makes BM x BN of out, WM x WN wavefronts side by side, half a panel (128 columns of k) of every 32 rows
// at a time through LDS, where it lies as in memory: the matrix cores' reads are 1 KB in one piece.  Loads go straight into LDS, in a ring
// of four such blocks, up to three ahead of the products; products, LDS reads and loads are put in order by hand.  weight is the left
// operand, so a lane ends with neighbouring columns.  (With put_wide it is the right one: 2003 x 50256 x 4096 239 us instead of 273.)
// Bound by the matrix cores and what is between tiles: 2003 x 50256 x 4096 in 256 x 256 239 to 265 us (3.1 to 3.45 PFLOP/s; the matrix cores 53 % busy).  Of that the
// products alone take 142, reads from LDS and barriers 29, loads 30, the first loads and the result of a tile 45, in 7 rounds of 256 workgroups for
// 6.2 rounds' worth of tiles.  8192^3 takes 237 (4.6 PFLOP/s; bf16 1.4).  64 x 100256 x 4096: 40 us, in tiles of 64 x 128.
template <class OUT, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(WM *WN *kWave, 1) linear_mx4_block_kernel(LinearMx4Params p) {
    constexpr int NW = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32, F = TM + TN, GX = BM / 32, GW = BN / 32, G = GX + GW, kRing = 4;
    constexpr int kSlot = G * 2048, kScaleSlot = G * 256, kScales = kRing * kSlot, kLds = kScales + 2 * kScaleSlot;
    constexpr int kCodeLoads = (2 * G + NW - 1) / NW, kScaleLoads = (G + NW - 1) / NW;
    constexpr bool kWide = !std::is_void<OUT>::value;      // (the result by put_wide)
    static_assert(!kWide || (TN == 4 && 2 * GX % NW == 0), "");
    __shared__ __attribute__((aligned(1024))) char lds[kLds];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int tile_m, tile_n, split;
    if (!tile_of((p.m + BM - 1) / BM, (p.n + BN - 1) / BN, p.splits, tile_m, tile_n, split)) return;
    int panel0 = 0, blocks = 2 * p.panels;
    if (p.splits > 1) {
        panel0 = (int)((int64_t)p.panels * split / p.splits);
        blocks = 2 * ((int)((int64_t)p.panels * (split + 1) / p.splits) - panel0);
    }
    // Where a wavefront's loads of the first block begin, of codes (1 KB each) and of scales: groups behind the last are the last one again.
    const char *codes_from[kCodeLoads], *scales_from[kScaleLoads];
    const auto panel_of = [&](int g) {
        const int64_t group = g < GX ? min(tile_m * GX + g, (p.m - 1) / 32) : min(tile_n * GW + g - GX, (p.n - 1) / 32);
        return (g < GX ? (const char *)p.x : (const char *)p.w) + (group * p.panels + panel0) * kPanelBytes;
    };
    const auto unit = [&](int q) { return min(q * NW + wv, 2 * G - 1); };
    const auto group_of = [&](int q) { return min(q * NW + wv, G - 1); };
#pragma unroll
    for (int q = 0; q < kCodeLoads; ++q) codes_from[q] = panel_of(unit(q) >> 1) + (unit(q) & 1) * 1024;
#pragma unroll
    for (int q = 0; q < kScaleLoads; ++q) scales_from[q] = panel_of(group_of(q)) + kPanelCodes;
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    // Loads of block `from` into the place of block t.
    const uint32_t wide_at = wide_source(lane);
    const auto load_codes_at = [&](int from, int t, int q) {
        load_lds(lds_base + (t & 3) * kSlot + unit(q) * 1024, codes_from[q] + ((int64_t)(from >> 1) * kPanelBytes + (from & 1) * 2048),
                 kWide && q * NW >= 2 * GX ? wide_at : 16 * lane);
    };
    const auto load_scales_at = [&](int from, int t, int q) {
        load_lds4(lds_base + kScales + (t >> 1 & 1) * kScaleSlot + group_of(q) * 256, scales_from[q] + (int64_t)(from >> 1) * kPanelBytes, 4 * lane);
    };
    const int wm = wv / WN, wn = wv % WN;
    F16v acc[TM][TN] = {};
    U4 frag[2][2][F];                  // [a block, the next one][step of 64 columns][groups of x, groups of weight]
    uint32_t scale[F], next_scale[F];
    const auto group_at = [&](int f) { return f < TM ? wm * TM + f : GX + wn * TN + f - TM; };
    const int wide_group = GX + wn * TN + ((lane & 31) >> 3);
    const auto read = [&](int t, int into, int q) {
        const int f = q % F;
        const int at = kWide && f >= TM ? wide_group * 2048 + wide_place(lane, f - TM) : group_at(f) * 2048 + 16 * lane;
        frag[into][q / F][f] = *(const U4 *)(lds + (t & 3) * kSlot + 1024 * (q / F) + at);
    };
    const auto read_scale = [&](int t, int f) {
        const int at = kWide && f >= TM ? wide_group * 256 + wide_scale(lane, f - TM) : group_at(f) * 256 + 4 * lane;
        next_scale[f] = *(const uint32_t *)(lds + kScales + (t >> 1 & 1) * kScaleSlot + at);
    };
    constexpr int kReads = 2 * F, kProducts = 2 * TM * TN;
    // The products of block t, the first or second half of its panel, and among them the reads of block t + 1 and the loads of block t + 4 (behind
    // the last block: that one again, for nobody).
    const auto phase = [&](auto which, int t) {
        constexpr int half = decltype(which)::value, R = half ? kReads + F : kReads, L = half ? kCodeLoads : kCodeLoads + kScaleLoads;
        const int to_load = min(t + 4, blocks - 2 + half);
#pragma unroll
        for (int q = 0; q < kProducts; ++q) {
#pragma unroll
            for (int r = q * R / kProducts; r < (q + 1) * R / kProducts; ++r) {
                if (r < kReads) read(t + 1, half ^ 1, r);
                else read_scale(t + 1, r - kReads);
            }
#pragma unroll
            for (int l = q * L / kProducts; l < (q + 1) * L / kProducts; ++l) {
                if (l < kCodeLoads) load_codes_at(to_load, t, l);
                else load_scales_at(to_load, t, l - kCodeLoads);
            }
            const int s = q / (TM * TN), a = q / TN % TM, b = q % TN;
            const int l = kWide ? a : TM + b, r = kWide ? TM + b : a;
            if (s == 0) acc[a][b] = mma_mx4<2 * half>(frag[half][s][l], frag[half][s][r], acc[a][b], scale[l], scale[r]);
            else acc[a][b] = mma_mx4<2 * half + 1>(frag[half][s][l], frag[half][s][r], acc[a][b], scale[l], scale[r]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    constexpr std::integral_constant<int, 0> first;
    constexpr std::integral_constant<int, 1> second;
    // What may still be on its way when block t + 1 has to be there: the loads of the last two phases, one of which had the scales'.
    constexpr int kLater = 2 * kCodeLoads + kScaleLoads;
    if (blocks > 0) {
#pragma unroll
        for (int t = 0; t < kRing; ++t) {
            const int from = t < blocks ? t : blocks - 2 + (t & 1);
#pragma unroll
            for (int q = 0; q < kCodeLoads; ++q) load_codes_at(from, t, q);
            if (t % 2 == 0) {
#pragma unroll
                for (int q = 0; q < kScaleLoads; ++q) load_scales_at(from, t, q);
            }
        }
        wait_and_meet<0>();
#pragma unroll
        for (int q = 0; q < kReads; ++q) read(0, 0, q);
#pragma unroll
        for (int f = 0; f < F; ++f) read_scale(0, f);
        for (int t = 0; t < blocks; t += 2) {
#pragma unroll
            for (int f = 0; f < F; ++f) scale[f] = next_scale[f];
            wait_and_meet<kLater>();
            phase(first, t);
            wait_and_meet<kLater>();
            phase(second, t + 1);
        }
        wait_and_meet<0>();
    }
    if constexpr (kWide) put_wide<OUT>(p, acc, tile_m * BM + wm * (BM / WM), tile_n * BN + wn * 128);
    else put_tile<BM, BN, WM, WN, kLds>(p, acc, lds, tile_m * BM, tile_n * BN, split);
}

// x in 16 bits.  As above, but 64 columns of k at a time: x in rows of 128 bytes whose sixteen-byte groups are permuted by the row (see
// linear_block_kernel), weight in the 1 KB of its 32 rows, made bf16 on the way from LDS into the matrix cores.  Lane l takes columns 32 (l / 32) + 8 q
// ..+7 of the 64 in product q, of x and weight alike, so that each of its sixteen bytes of weight has one scale.  x of block t + 2 is
// loaded in the first half of block t, weight in the second; scales, of four blocks, with the first of them.
// Bound by the matrix cores in 256 x 256 (2003 x 50256 x 4096 708 us, 1165 TFLOP/s, with silu and a residual 766); f16, whose two parts are two
// products, takes twice as long (1,394 to 1,502 by card; bf16 664 to 708).  Rows of x at odd addresses pass through registers, which 256 x 256 has none left for: 1075 in 128 x 128.
constexpr int kXSlots = 3;
template <class T, class OUT, int BM, int BN, int WM, int WN, bool DIRECT>
__global__ void __launch_bounds__(WM *WN *kWave, BM * BN > 32768 ? 1 : 2) linear_x16_block_kernel(LinearMx4Params p) {
    constexpr int NW = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32, GW = BN / 32;
    constexpr int kLoadsX = BM / 8 / NW, kLoadsW = GW / NW;
    static_assert(BM % (8 * NW) == 0 && GW % NW == 0, "");
    constexpr int kX = BM * 128, kW = GW * 1024, kS = GW * 256, kScales = kXSlots * kX + 2 * kW, kLds = kScales + 2 * kS;
    __shared__ __attribute__((aligned(1024))) char lds[kLds];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int tile_m, tile_n, split;
    if (!tile_of((p.m + BM - 1) / BM, (p.n + BN - 1) / BN, p.splits, tile_m, tile_n, split)) return;
    const int i0 = tile_m * BM, j0 = tile_n * BN;
    const int row8 = lane >> 3, group = (lane & 7) ^ row8;
    // this part's panels; blocks of 64 columns, the last one of all may be cut off
    int panel0 = 0, blocks = (p.k + 63) >> 6;
    if (p.splits > 1) {
        panel0 = (int)((int64_t)p.panels * split / p.splits);
        const int end = (int)((int64_t)p.panels * (split + 1) / p.splits);
        blocks = (split == p.splits - 1 ? blocks : 4 * end) - 4 * panel0;
    }
    const int cut = split == p.splits - 1 ? p.k & 63 : 0;
    // (as in linear_block_kernel: what lies behind the row's end is loaded from so much further in front, and mended in LDS)
    const int over = max(8 * group + 8 - (DIRECT ? cut & ~7 : cut), 0);
    const uint16_t *x = (const uint16_t *)p.x;
    const char *xb = (const char *)(x + i0 * p.x_stride + kPanelCols * (int64_t)panel0 - 8);
    uint32_t at[kLoadsX];
#pragma unroll
    for (int q = 0; q < kLoadsX; ++q) at[q] = 2u * (uint32_t)(min((q * NW + wv) * 8 + row8, p.m - 1 - i0) * (int)p.x_stride + 8 * group + 8);
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    const int last_w = (p.n - 1) / 32;
    const auto panel_of = [&](int g, int t) {          // of block t
        return (const char *)p.w + ((int64_t)min(tile_n * GW + g, last_w) * p.panels + panel0 + (t >> 2)) * kPanelBytes;
    };
    U4 held[DIRECT ? 1 : kLoadsX];
    const auto load_x = [&](int slot, int t, int q) {
        const char *base = xb + 128 * (int64_t)t;
        if constexpr (DIRECT) load_lds(lds_base + slot + (q * NW + wv) * 1024, base, at[q]);
        else held[q] = load16((const uint16_t *)(base + at[q]));
    };
    const auto store_x = [&](int slot, int q) {
        if constexpr (!DIRECT) *(U4 *)(lds + slot + (q * NW + wv) * 1024 + 16 * lane) = held[q];
    };
    constexpr bool kWide = !std::is_void<OUT>::value;      // (the result by put_wide)
    static_assert(!kWide || TN == 4, "");
    const uint32_t w_source = kWide ? wide_source(lane) : 16 * lane;
    const auto load_w = [&](int slot, int t, int q) { load_lds(lds_base + slot + (q * NW + wv) * 1024, panel_of(q * NW + wv, t) + 1024 * (t & 3), w_source); };
    const auto load_scales = [&](int t) {
#pragma unroll
        for (int q = 0; q < kLoadsW; ++q) load_lds4(lds_base + kScales + (t >> 2 & 1) * kS + (q * NW + wv) * 256, panel_of(q * NW + wv, t) + kPanelCodes, 4 * lane);
    };
    const int wm = wv / WN, wn = wv % WN;
    const int xrow = (wm * (BM / WM) + (lane & 31)) * 128, first = ((lane >> 5) * 4 ^ (lane & 7)) * 16;
    F16v acc[TM][TN] = {};
    U4 xf[2][2][TM], codes[2][TN];     // x: [half of a block][step][rows]; codes of a whole block, and of the next one
    float scale[2][TN];
    const auto read_x = [&](int slot, int half, int q) { xf[half][q / TM][q % TM] = *(const U4 *)(lds + slot + xrow + (first ^ 16 * (2 * half + q / TM)) + (q % TM) * 4096); };
    const auto read_w = [&](int slot, int t, int into, int q) {
        const int wide_group = wn * TN + ((lane & 31) >> 3), b = q % TN;
        if (q < TN) codes[into][b] = *(const U4 *)(lds + slot + (kWide ? wide_group * 1024 + wide_place(lane, b) : (wn * TN + b) * 1024 + 16 * lane));
        else scale[into][b] = scale_of(*(const uint8_t *)(lds + kScales + (t >> 2 & 1) * kS + (kWide ? wide_group * 256 + wide_scale(lane, b) : (wn * TN + b) * 256 + 4 * lane) + (t & 3)));
    };
    constexpr bool kParts = T::kCode == BPE_F16;
    U4 wf[2][TN], finite[2][TN];       // of a step, and of the next one; for the second parts of f16
    U4 high[2], low[2];                // the parts of a fragment of x in f16, and of the next one
    const auto widen = [&](int from, int step, int into, int b) {
        wf[into][b] = bf16_of(codes[from][b][step], scale[from][b]);
        if constexpr (kParts) finite[into][b] = finite_of(wf[into][b]);
    };
    constexpr int kReadsX = 2 * TM, kProducts = 2 * TM * TN;
    // The products of one half of block t.  Among them: the reads of x of the other half (of the block in slot xr), in the second half codes and scales of the
    // next block, the weights of the next step, and loads.
    const auto phase = [&](auto which, auto lx, auto lw, int xr, int wr, int t, int xl, int wl, int t_load, int xs) {
        constexpr int half = decltype(which)::value, LX = decltype(lx)::value, LW = decltype(lw)::value;
#pragma unroll
        for (int q = 0; q < kProducts; ++q) {
            const int s = q / (TM * TN), in_step = q % (TM * TN), a = in_step / TN, b = in_step % TN;
#pragma unroll
            for (int r = q * kReadsX / kProducts; r < (q + 1) * kReadsX / kProducts; ++r) read_x(xr, half ^ 1, r);
            if constexpr (half == 1) {
                // (in the first of its two steps, so that the second can widen the next block's first step)
                if (s == 0) {
#pragma unroll
                    for (int r = in_step * 2 * TN / (TM * TN); r < (in_step + 1) * 2 * TN / (TM * TN); ++r) read_w(wr, t + 1, 1, r);
                }
            }
#pragma unroll
            for (int l = q * LX / kProducts; l < (q + 1) * LX / kProducts; ++l) load_x(xl, t_load, l);
#pragma unroll
            for (int l = q * LW / kProducts; l < (q + 1) * LW / kProducts; ++l) load_w(wl, t_load, l);
            if constexpr (!DIRECT && half == 1) {
#pragma unroll
                for (int l = q * kLoadsX / kProducts; l < (q + 1) * kLoadsX / kProducts; ++l) store_x(xs, l);
            }
            // (of f16 the parts of the next fragment of x are made meanwhile)
            const int now = (2 * half + s) * TM + a & 1;
            acc[a][b] = mma_by_weight<T, kWide>(wf[s][b], finite[s][b], kParts ? high[now] : xf[half][s][a], low[now], acc[a][b]);
            if constexpr (kParts) {
                const int next_a = a + 1 < TM ? a + 1 : 0, next_s = a + 1 < TM ? s : s + 1;
                const U4 &next = next_s < 2 ? xf[half][next_s & 1][next_a] : xf[half ^ 1][0][next_a];
#pragma unroll
                for (int d = b * 4 / TN; d < (b + 1) * 4 / TN; ++d) {
                    uint32_t h, l;
                    split_f16(next[d], h, l);
                    high[now ^ 1][d] = h;
                    low[now ^ 1][d] = l;
                }
            }
#pragma unroll
            for (int r = in_step * TN / (TM * TN); r < (in_step + 1) * TN / (TM * TN); ++r) {
                if (half == 0 || s == 0) widen(0, 2 * half + s + 1, s ^ 1, r);
                else widen(1, 0, 0, r);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const auto step_back = [&]() {
#pragma unroll
        for (int q = 0; q < kLoadsX; ++q) at[q] -= 2u * (uint32_t)over;
    };
    const auto mend = [&](int slot) {
        if (over) {
#pragma unroll
            for (int q = 0; q < kLoadsX; ++q) {
                U4 *mine = (U4 *)(lds + slot + (q * NW + wv) * 1024 + 16 * lane);
                if constexpr (DIRECT) {
                    U4 v = {0, 0, 0, 0};
                    if (8 * group < cut) v = load_tail(x + min(i0 + (q * NW + wv) * 8 + row8, p.m - 1) * p.x_stride, p.k - cut + 8 * group, p.k);
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
    constexpr std::integral_constant<int, kLoadsX> all_x;
    constexpr std::integral_constant<int, kLoadsW> all_w;
    if (blocks > 0) {
        int x0 = 0, x1 = kX, x2 = 2 * kX, w0 = kXSlots * kX, w1 = w0 + kW;
        if (cut && blocks == 1) step_back();
#pragma unroll
        for (int q = 0; q < kLoadsX; ++q) load_x(x0, 0, q);
#pragma unroll
        for (int q = 0; q < kLoadsX; ++q) store_x(x0, q);
#pragma unroll
        for (int q = 0; q < kLoadsW; ++q) load_w(w0, 0, q);
        load_scales(0);
        wait_and_meet<0>();
        if (cut && blocks == 1) mend(x0);
#pragma unroll
        for (int q = 0; q < kReadsX; ++q) read_x(x0, 0, q);
#pragma unroll
        for (int q = 0; q < 2 * TN; ++q) read_w(w0, 0, 0, q);
#pragma unroll
        for (int q = 0; q < TN; ++q) widen(0, 0, 0, q);
        if constexpr (T::kCode == BPE_F16) {
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                uint32_t h, l;
                split_f16(xf[0][0][0][d], h, l);
                high[0][d] = h;
                low[0][d] = l;
            }
        }
        if (cut && blocks == 2) step_back();
        const int t1 = min(1, blocks - 1);
#pragma unroll
        for (int q = 0; q < kLoadsX; ++q) load_x(x1, t1, q);
#pragma unroll
        for (int q = 0; q < kLoadsX; ++q) store_x(x1, q);
#pragma unroll
        for (int q = 0; q < kLoadsW; ++q) load_w(w1, t1, q);
        const auto step = [&](int t, auto near_end) {
            constexpr bool kNearEnd = decltype(near_end)::value;
            const int t2 = min(t + 2, blocks - 1);             // (behind the last block: that block again, for nobody)
            if (kNearEnd && t + 3 == blocks) step_back();
            phase(none, all_x, none, x0, 0, t, x2, 0, t2, 0);
            wait_and_meet<DIRECT ? kLoadsX : 0>();             // block t + 1 is there, and nobody reads block t any more
            if (kNearEnd && t + 2 == blocks) mend(x1);
            if ((t2 & 3) == 0) load_scales(t2);
            phase(second, none, all_w, x1, w1, t, 0, w0, t2, x2);
            const int xt = x0, wt = w0;
            x0 = x1; x1 = x2; x2 = xt;
            w0 = w1; w1 = wt;
#pragma unroll
            for (int b = 0; b < TN; ++b) { codes[0][b] = codes[1][b]; scale[0][b] = scale[1][b]; }
        };
        const int calm = cut ? blocks - 3 : blocks;
        int t = 0;
        for (; t < calm; ++t) step(t, std::false_type());
        for (; t < blocks; ++t) step(t, std::true_type());
        wait_and_meet<0>();
    }
    if constexpr (kWide) put_wide<OUT>(p, acc, i0 + wm * (BM / WM), j0 + wn * 128);
    else put_tile<BM, BN, WM, WN, kLds>(p, acc, lds, i0, j0, split);
}

// Up to 64 rows of x in 16 bits: the call is as long as reading weight takes, so what counts is how much of it is on its way.  A wavefront takes 32 TN rows of
// weight for itself and brings them straight into its registers, a panel ahead; x goes through LDS, a panel at a time, for all four
// wavefronts of a workgroup.  (x in rows of 512 bytes, whose sixteen-byte groups are permuted by the row, so that sixteen rows read at one
// index meet all banks.)
// 1 x 50256 x 1024 7.4 to 8.6 us (27 MB, 3.2 to 3.7 TB/s with a launch's ramp in it); 32 x 100256 x 4096 41, 64 x 100256 x 4096 57 to 73 (223 MB read, 13 or 26
// written: 42 % of the matrix cores' time, the conversions in their shadow, and 392 workgroups on 256 compute units).  Two panels ahead
// instead of one took as long.
template <class T, int TM, int TN>
__global__ void __launch_bounds__(kGroupThreads, T::kCode == BPE_F16 && TM == 2 ? 1 : 2) linear_x16_stream_kernel(LinearMx4Params p) {
    constexpr bool kParts = T::kCode == BPE_F16;               // (x as its two bf16 parts, one behind the other)
    constexpr int BM = 32 * TM, BN = 128 * TN, kLoadsX = BM / 8, kPart = BM * 512, kSlot = kParts ? 2 * kPart : kPart;
    constexpr int kLds = std::max(2 * kSlot, kWavesPerGroup * 32 * (32 * TN + 4) * 4);
    __shared__ __attribute__((aligned(1024))) char lds[kLds];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 31, h = lane >> 5;
    int tile_m, tile_n, split;
    if (!tile_of((p.m + BM - 1) / BM, (p.n + BN - 1) / BN, p.splits, tile_m, tile_n, split)) return;
    const int i0 = tile_m * BM, j0 = tile_n * BN;
    int panel = 0, end = p.panels;
    if (p.splits > 1) {
        panel = (int)((int64_t)p.panels * split / p.splits);
        end = (int)((int64_t)p.panels * (split + 1) / p.splits);
    }
    const int last_w = (p.n - 1) / 32;
    const char *w[TN];
#pragma unroll
    for (int b = 0; b < TN; ++b) w[b] = (const char *)p.w + (int64_t)min(tile_n * (BN / 32) + wv * TN + b, last_w) * p.panels * kPanelBytes;
    U4 codes[2][TN][4], xr[kLoadsX];
    uint32_t scales[2][TN];
    // (a thread takes sixteen bytes of every eighth row)
    const int x_row = tid >> 5, x_group = tid & 31;
    const uint16_t *x_from = (const uint16_t *)p.x + i0 * p.x_stride + 8 * x_group;
    uint32_t x_at[kLoadsX];
#pragma unroll
    for (int u = 0; u < kLoadsX; ++u) x_at[u] = (uint32_t)(min(x_row + 8 * u, p.m - 1 - i0) * (int)p.x_stride);
    const auto load_x = [&](int panel) {
        const uint16_t *from = x_from + (int64_t)panel * kPanelCols;
        const int over = max(panel * kPanelCols + 8 * x_group + 8 - p.k, 0);       // columns that lie behind the end: loaded from so much further in front
#pragma unroll
        for (int u = 0; u < kLoadsX; ++u) xr[u] = load16(from + x_at[u] - over);
        if ((panel + 1) * (int64_t)kPanelCols > p.k) {
#pragma unroll
            for (int u = 0; u < kLoadsX; ++u) xr[u] = shift_out(xr[u], over);
        }
    };
    const auto store_x = [&](int slot) {
#pragma unroll
        for (int u = 0; u < kLoadsX; ++u) {
            const int row = x_row + 8 * u;
            U4 *to = (U4 *)(lds + slot * kSlot + row * 512 + (x_group ^ (row & 15)) * 16);
            if constexpr (kParts) {
                U4 high, low;
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    uint32_t one, two;
                    split_f16(xr[u][d], one, two);
                    high[d] = one;
                    low[d] = two;
                }
                *to = high;
                to[kPart / 16] = low;
                __builtin_amdgcn_sched_barrier(0);             // (not all parts at once: registers would spill)
            } else {
                *to = xr[u];
            }
        }
    };
    const auto load_w = [&](auto into, int panel) {
        constexpr int I = decltype(into)::value;
#pragma unroll
        for (int b = 0; b < TN; ++b) {
            const char *from = w[b] + (int64_t)panel * kPanelBytes;
#pragma unroll
            for (int s = 0; s < 4; ++s) codes[I][b][s] = *(const U4 *)(from + 1024 * s + 16 * lane);
            scales[I][b] = *(const uint32_t *)(from + kPanelCodes + 4 * lane);
        }
    };
    F16v acc[TM][TN] = {};
    const auto products = [&](auto which, auto infinite) __attribute__((always_inline)) {
        constexpr int I = decltype(which)::value;
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                U4 x[TM], low[TM];
#pragma unroll
                for (int a = 0; a < TM; ++a) {
                    const U4 *from = (const U4 *)(lds + I * kSlot + (32 * a + r) * 512 + ((8 * s + 4 * h + q) ^ (r & 15)) * 16);
                    x[a] = *from;
                    if constexpr (kParts) low[a] = from[kPart / 16];
                }
#pragma unroll
                for (int b = 0; b < TN; ++b) {
                    const U4 wide = bf16_of(codes[I][b][s][q], scale_of(scales[I][b] >> 8 * s & 255));
#pragma unroll
                    for (int a = 0; a < TM; ++a) acc[a][b] = mma_by_weight<T>(wide, decltype(infinite)::value ? finite_of(wide) : wide, x[a], low[a], acc[a][b]);
                }
            }
    };
    constexpr std::integral_constant<int, 0> even;
    constexpr std::integral_constant<int, 1> odd;
    const auto step = [&](auto now, auto next, int panel) {
        // what the other wavefronts have stored is there, and nobody reads the other slot any more (loads stay on their way)
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const int ahead = min(panel + 1, end - 1);             // (behind the last panel: that one again, for nobody)
        load_x(ahead);
        load_w(next, ahead);
        // (weights that are infinities, which hardly any matrix has, have products of their own: finite_of for every weight takes 5 to 12 % longer)
        bool infinite = false;
        if constexpr (kParts) {
            uint32_t most = 0;
#pragma unroll
            for (int b = 0; b < TN; ++b)
#pragma unroll
                for (int s = 0; s < 4; ++s) most = max(most, scales[decltype(now)::value][b] >> 8 * s & 255);
            infinite = __any(scale_of(most) >= kMayBeInfinite);
        }
        if (__builtin_expect(infinite, false)) products(now, std::true_type());
        else products(now, std::false_type());
        store_x(decltype(next)::value);
    };
    if (panel < end) {
        load_x(panel);
        load_w(even, panel);
        store_x(0);
        for (; panel < end; panel += 2) {
            step(even, odd, panel);
            if (panel + 1 < end) step(odd, even, panel + 1);
        }
        __syncthreads();
    }
    put_tile<BM, BN, 1, kWavesPerGroup, kLds>(p, acc, lds, i0, j0, split);
}

// Which tiles a product takes, and into how many parts k is cut: what an estimate of the time says, as for bpe_linear.  A tile's row: its sides, how many
// of its workgroups a compute unit holds, us for a panel when a workgroup waits for its loads alone, us for its first loads and its
// result, and the TFLOP/s of the whole chip when nothing else bounds it.  The numbers are fitted to the times of all tiles and parts on 84
// and 48 sizes (m 1 to 2000, n 2048 to 100256, k 512 to 4096; f16 apart), where the choice takes 1.2 % (0.4 % for 4 bits) longer than the best
// one on average, 16 % at worst.  (They are numbers that choose well; not every one is a property of its tile.)
struct LinearMxTile { int bm, bn, resident; double panel_us, tile_us, tflops; };
constexpr LinearMxTile kX16Tiles[] = {{64, 128, 3, 1.97, 1.45, 851}, {128, 128, 2, 2.43, 3.08, 1050}, {256, 256, 1, 1.46, 7.67, 1470},
                                      // linear_x16_stream_kernel
                                      {32, 128, 4, 0.531, 3.15, 863}, {32, 256, 3, 0.89, 0, 497}, {64, 128, 2, 0.603, 1.38, 730}, {64, 256, 2, 0.181, 4.85, 1170}};
// (f16: two products for each; the tiles that it never takes have no rate)
constexpr LinearMxTile kF16Tiles[] = {{64, 128, 3, 0, 0, 0}, {128, 128, 2, 5.96, 5.28, 450}, {256, 256, 1, 0, 0, 0},
                                      {32, 128, 2, 0.54, 4.28, 495}, {32, 256, 2, 2.28, 3.86, 590}, {64, 128, 1, 0, 0, 0}, {64, 256, 1, 0, 0, 0}};
constexpr LinearMxTile kMx4Tiles[] = {{32, 128, 3, 0.586, 2.41, 1670}, {64, 128, 2, 0.722, 1.86, 2080}, {128, 128, 2, 1.26, 4.13, 3260}, {256, 256, 1, 0.556, 9.43, 4350}};
struct LinearMxPlan { int tile, splits; };

static LinearMxPlan plan_linear_mx(int64_t m, int64_t n, int64_t k, int x_dtype) {
    const bool packed = x_dtype == BPE_MX4, f16 = x_dtype == BPE_F16;
    const LinearMxTile *tiles = packed ? kMx4Tiles : f16 ? kF16Tiles : kX16Tiles;
    const int count = packed ? 4 : 7;
    const double bytes_x = packed ? 0.53 : 2, memory_rate = packed ? 5.77e6 : f16 ? 8.57e6 : 7.58e6, l2_rate = packed ? 4.29e7 : f16 ? 5.55e7 : 6.57e7;
    LinearMxPlan best = {0, 1};
    double least = 1e300;
    const double panels = (double)std::max<int64_t>(panels_of(k), 1);
    for (int t = 0; t < count; ++t) {
        const LinearMxTile &l = tiles[t];
        if (l.tflops == 0) continue;
        const double all = (double)((m + l.bm - 1) / l.bm) * (double)((n + l.bn - 1) / l.bn);
        for (int splits = 1; splits <= 16; splits *= 2) {
            if (splits > 1 && (all * splits > 768 || panels < 2 * splits)) break;
            const double groups = all * splits, per = std::ceil(panels / splits);
            const double compute = std::ceil(groups / 256) * per * (2.0 * l.bm * l.bn * 256) / (l.tflops * 1e6 / 256);
            const double rounds = groups / (256.0 * l.resident), wait = std::ceil(rounds) * per * l.panel_us;
            const double memory = (0.53 * (double)n * k + bytes_x * (double)m * k + 3.1 * (double)m * n) / memory_rate + all * (bytes_x * l.bm + 0.53 * l.bn) * k / l2_rate;
            const double join = splits > 1 ? 3.8 + (double)splits * m * n * 8 / 6.7e6 : 0.0;
            const double us = std::max(std::max(compute, wait), memory) + std::max(rounds, 1.0) * l.tile_us + join;
            if (us < least) { least = us; best = {t, splits}; }
        }
    }
    return best;
}
static int64_t linear_mx_need(const LinearMxPlan &plan, int64_t m, int64_t n) { return plan.splits > 1 ? 4 * (int64_t)plan.splits * m * part_stride_of(n) : 0; }

static int launch_tiles(void (*kernel)(LinearMx4Params), int bm, int bn, LinearMx4Params &p, int splits, void *workspace, void *stream) {
    const char *what = "bpe_linear_mx launch";
    p.splits = splits;
    const int64_t grid = tile_grid(((int64_t)p.m + bm - 1) / bm, ((int64_t)p.n + bn - 1) / bn, splits);
    if (grid >= kMaxThreads / kGroupThreads) { set_error("bpe_linear_mx: m %d and n %d are too large together", p.m, p.n); return BPE_ERR_SIZE; }
    p.part = (float *)workspace;
    p.part_stride = (int32_t)part_stride_of(p.n);
    const int rc = launch(kernel, dim3((unsigned)grid), kGroupThreads, p, stream, what);
    return rc != BPE_OK || splits == 1 ? rc : launch_join(p, stream, what);
}
// (a residual or an activation takes the way through LDS: unrolled over all registers they would be far too much code)
static bool leaves_wide(const LinearMx4Params &p, LinearMxPlan plan) { return plan.splits == 1 && p.activation == BPE_ACT_NONE && !p.residual && p.n % 4 == 0; }
template <class T> static int launch_rows(LinearMx4Params &p, void *stream) { return launch_tiles(linear_mx4_rows_kernel<T>, 32, 32, p, 1, nullptr, stream); }

static int launch_linear_mx4(LinearMx4Params &p, LinearMxPlan plan, void *workspace, void *stream) {
    // (out and the residual are addressed by 32-bit offsets within the rows that a wavefront writes at a time)
    if (p.out_stride >= (1 << 25) || p.residual_stride >= (1 << 25)) return launch_rows<Mx4>(p, stream);
    void (*kernels[])(LinearMx4Params) = {linear_mx4_block_kernel<void, 32, 128, 1, 4>, linear_mx4_block_kernel<void, 64, 128, 1, 4>, linear_mx4_block_kernel<void, 128, 128, 2, 2>,
                                          linear_mx4_block_kernel<void, 256, 256, 2, 2>};
    if (plan.tile == 3 && leaves_wide(p, plan)) {
        kernels[3] = p.out_dtype == BPE_F32 ? linear_mx4_block_kernel<F32, 256, 256, 2, 2> : p.out_dtype == BPE_BF16 ? linear_mx4_block_kernel<Bf16, 256, 256, 2, 2> : linear_mx4_block_kernel<F16, 256, 256, 2, 2>;
    }
    return launch_tiles(kernels[plan.tile], kMx4Tiles[plan.tile].bm, kMx4Tiles[plan.tile].bn, p, plan.splits, workspace, stream);
}

template <class T> static int launch_linear_x16(LinearMx4Params &p, LinearMxPlan plan, void *workspace, void *stream) {
    // (a tile's rows are addressed by 32-bit offsets, and loads are of eight columns)
    if (p.x_stride >= (1 << 21) || p.out_stride >= (1 << 25) || p.residual_stride >= (1 << 25) || p.k < 8) return launch_rows<T>(p, stream);
    const bool direct = p.x_stride % 8 == 0 && !((uintptr_t)p.x & 15);
    // (rows on their way through registers need more of these than there are beside 256 x 256 sums)
    if (plan.tile == 2 && !direct) plan.tile = 1;
    constexpr bool kBf16 = T::kCode == BPE_BF16;
    void (*kernel)(LinearMx4Params) = nullptr;
#define TILE(INDEX, WHERE, BM, BN, KERNEL) \
    case INDEX: \
        static_assert(kX16Tiles[INDEX].bm == BM && kX16Tiles[INDEX].bn == BN && (WHERE || kF16Tiles[INDEX].tflops == 0), ""); \
        if constexpr (WHERE) kernel = KERNEL; \
        break
#define BLOCK(OUT, BM, BN, WM, WN, DIRECT) linear_x16_block_kernel<T, OUT, BM, BN, WM, WN, DIRECT>
#define STREAM(TM, TN) linear_x16_stream_kernel<T, TM, TN>
    switch (plan.tile) {
        TILE(0, kBf16, 64, 128, (direct ? BLOCK(void, 64, 128, 1, 4, true) : BLOCK(void, 64, 128, 1, 4, false)));
        TILE(1, true, 128, 128, (direct ? BLOCK(void, 128, 128, 2, 2, true) : BLOCK(void, 128, 128, 2, 2, false)));
        TILE(2, kBf16, 256, 256, (!leaves_wide(p, plan) ? BLOCK(void, 256, 256, 2, 2, true) : p.out_dtype == BPE_F32 ? BLOCK(F32, 256, 256, 2, 2, true) : BLOCK(T, 256, 256, 2, 2, true)));
        TILE(3, true, 32, 128, (STREAM(1, 1)));
        TILE(4, true, 32, 256, (STREAM(1, 2)));
        TILE(5, kBf16, 64, 128, (STREAM(2, 1)));
        TILE(6, kBf16, 64, 256, (STREAM(2, 2)));
    }
#undef TILE
#undef BLOCK
#undef STREAM
    return launch_tiles(kernel, kX16Tiles[plan.tile].bm, kX16Tiles[plan.tile].bn, p, plan.splits, workspace, stream);
}

}  // namespace bpe

using namespace bpe;

static int linear_mx4_sizes_ok(int64_t m, int64_t n, int64_t k) {
    if (m < 0 || n < 0 || k < 0 || m >= (1 << 30) || n >= (1 << 30) || k >= (1 << 30)) {
        set_error("bpe_linear_mx: sizes out of range (m %lld, n %lld, k %lld)", (long long)m, (long long)n, (long long)k);
        return 0;
    }
    return 1;
}

static int linear_mx4_type_ok(int dtype) {
    if (dtype == BPE_BF16 || dtype == BPE_F16 || dtype == BPE_MX4) return 1;
    set_error("bpe_linear_mx: x is bf16, f16 or mx4 (dtype %d)", dtype);
    return 0;
}

extern "C" int64_t bpe_linear_mx_workspace_bytes(int64_t m, int64_t n, int64_t k, int x_dtype) {
    if (!linear_mx4_sizes_ok(m, n, k)) return BPE_ERR_SIZE;
    if (!linear_mx4_type_ok(x_dtype)) return BPE_ERR_OPTION;
    return linear_mx_need(plan_linear_mx(m, n, k, x_dtype), m, n);
}

extern "C" int bpe_linear_mx(const void *x, int64_t x_stride, int x_dtype, const void *weight, int64_t m, int64_t n, int64_t k, const void *bias,
                              int bias_dtype, const void *residual, int64_t residual_stride, int activation, void *out, int64_t out_stride,
                              int out_dtype, void *workspace, int64_t workspace_bytes, void *stream) {
    if (!linear_mx4_sizes_ok(m, n, k)) return BPE_ERR_SIZE;
    if (!linear_mx4_type_ok(x_dtype)) return BPE_ERR_OPTION;
    if (!dtype_ok(out_dtype) || (out_dtype != BPE_F32 && x_dtype != BPE_MX4 && out_dtype != x_dtype)) {
        set_error("bpe_linear_mx: out is f32 or of x's type, any for x in 4 bits (out_dtype %d)", out_dtype);
        return BPE_ERR_OPTION;
    }
    if (bias && !dtype_ok(bias_dtype)) { set_error("bpe_linear_mx: bias_dtype %d", bias_dtype); return BPE_ERR_OPTION; }
    if (activation < BPE_ACT_NONE || activation > BPE_ACT_SILU) { set_error("bpe_linear_mx: activation %d", activation); return BPE_ERR_OPTION; }
    if (m == 0 || n == 0) return BPE_OK;
    if (!out || (k > 0 && (!x || !weight))) { set_error("null pointer"); return BPE_ERR_NULL; }
    const bool packed = x_dtype == BPE_MX4;
    if (m > 1 && ((!packed && x_stride < k) || out_stride < n || (residual && residual_stride < n))) {
        set_error("bpe_linear_mx: a stride is shorter than a row");
        return BPE_ERR_SIZE;
    }
    if (((uintptr_t)x & (packed ? 15 : 1)) || ((uintptr_t)weight & 15) || ((uintptr_t)out & (dtype_bytes(out_dtype) - 1)) ||
        ((uintptr_t)residual & (dtype_bytes(out_dtype) - 1)) || (bias && ((uintptr_t)bias & (dtype_bytes(bias_dtype) - 1)))) {
        set_error("bpe_linear_mx: a pointer is not aligned to its type (4-bit matrices to 16 bytes)");
        return BPE_ERR_SIZE;
    }
    const LinearMxPlan plan = plan_linear_mx(m, n, k, x_dtype);
    const int64_t need = linear_mx_need(plan, m, n);
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need)) {
        set_error("workspace must be 256-byte aligned and hold %lld bytes (got %lld)", (long long)need, (long long)workspace_bytes);
        return BPE_ERR_WORKSPACE;
    }
    LinearMx4Params p = {};
    p.x = x; p.w = (const uint8_t *)weight;
    p.x_stride = m > 1 ? x_stride : 0;
    p.m = (int32_t)m; p.n = (int32_t)n; p.k = (int32_t)k; p.panels = (int32_t)panels_of(k);
    p.bias = bias; p.bias_dtype = bias_dtype; p.activation = activation;
    p.residual = residual; p.residual_stride = residual && m > 1 ? residual_stride : 0;
    p.out = out; p.out_stride = m > 1 ? out_stride : 0; p.out_dtype = out_dtype; p.splits = 1;
    return packed ? launch_linear_mx4(p, plan, workspace, stream) : x_dtype == BPE_BF16 ? launch_linear_x16<Bf16>(p, plan, workspace, stream) : launch_linear_x16<F16>(p, plan, workspace, stream);
}
