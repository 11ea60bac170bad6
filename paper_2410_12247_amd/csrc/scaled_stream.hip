// Block-scaled products of few rows per expert: one pass over the weights,
// whose stream from memory is what the time goes to.  One token through the Mixtral
// FFN takes 15.6 us for gate and up (59 MB) and 9.8 for down (30 MB), 3.8 and 3.0
// TB/s, some 3 us of each a launch's start; 1 x 4096 x 4096 5.9 us, 2.9 TB/s; 16 tokens
// 14336 x 4096 of eight experts (470 MB) 90 us, 5.2 TB/s.
#include <algorithm>
#include <cmath>

#include "scaled.h"

namespace moe {
namespace {

constexpr int kRawFlags = 0x00020000;     // raw (untyped, unswizzled) buffer
constexpr uint32_t kRange = 0xFFFFFFF0u;  // its size
constexpr uint32_t kOutside = 0xFFFFFFF8u;  // an offset that reads as zero

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int v8i __attribute__((ext_vector_type(8)));

enum { SWIGLU = 0, OUT_F32 = 1, OUT_BF16 = 2 };

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const void *p) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)kRange, kRawFlags);
}
// eight e4m3 values as bf16, exactly
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ float silu_mul(float g, float u) {
    const float e = __builtin_amdgcn_exp2f(g * -1.44269504088896341f);
    return g * __builtin_amdgcn_rcpf(1.0f + e) * u;
}
__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
    const uint16_t ua = __builtin_bit_cast(uint16_t, static_cast<__bf16>(a));
    const uint16_t ub = __builtin_bit_cast(uint16_t, static_cast<__bf16>(b));
    return (uint32_t)ua | ((uint32_t)ub << 16);
}

// The workgroup owns 16 NT weight rows (of each matrix) of one expert over the
// whole of K; its W waves take blocks of 128 k in turn and keep D of them in
// flight, loaded straight into registers in the MFMA's operand layout.  The
// e4m3 values are widened to bf16, where the matrix instruction's products and
// sums are exact to fp32, and the scales applied to a block's fp32 sums: the
// stream leaves the compute units idle most of the time, so this costs nothing
// and the sums are exact to fp32 too.  The waves' sums meet in LDS and are
// added in wave order.
// FROM_H: the token rows are fp32 (the SwiGLU launch's) and quantised here,
// block by block, as they are read.
template <int MODE, bool FROM_H, int NT, int W, int D>
__global__ __launch_bounds__(64 * W) void stream_kernel(ScaledGemm g) {
    constexpr int NM = MODE == SWIGLU ? 2 : 1;  // matrices
    constexpr int NTT = NT * NM;
    __shared__ __attribute__((aligned(16))) floatx4 part[W][NTT][64];
    const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int e = blockIdx.y;
    int row0 = 0, cnt = (int)g.rows_one;
    if (g.offsets) {
        row0 = __builtin_amdgcn_readfirstlane(g.offsets[g.e_first + e]);
        cnt = __builtin_amdgcn_readfirstlane(g.offsets[g.e_first + e + 1]) - row0;
    }
    if (cnt <= 0) return;
    const int K = g.K, SK = scale_pitch(K), nb = scale_blocks(K);
    const int n0 = blockIdx.x * 16 * NT;
    const int64_t we = (int64_t)(g.e_first + e) * g.N + n0;
    const int64_t se = (int64_t)(g.e_first + e) * scale_blocks(g.N) + n0 / kScaleBlock;
    __amdgpu_buffer_rsrc_t wr[NM], sr[NM];
    wr[0] = rsrc(g.w0 + we * K);
    sr[0] = rsrc(g.s0 + se * SK);
    if (NM == 2) {
        wr[NM - 1] = rsrc(g.w1 + we * K);
        sr[NM - 1] = rsrc(g.s1 + se * SK);
    }
    uint32_t woff[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i)
        woff[i] = (uint32_t)(min(i * 16 + col, g.N - 1 - n0) * K + grp * 16);

    for (int m0 = 0; m0 < cnt; m0 += 16) {
        const uint8_t *xb = g.x;
        const uint8_t *sb = g.xs;
        const int64_t first = (int64_t)row0 + m0;
        if (!g.row_map) {
            xb += first * K * (FROM_H ? 4 : 1);
            sb += first * SK;
        }
        const __amdgpu_buffer_rsrc_t xr = rsrc(xb), xsr = rsrc(sb);
        const int r = min(col, cnt - 1 - m0);
        const uint32_t src =
            g.row_map ? (uint32_t)(g.row_map[first + r] / g.slot_div) : (uint32_t)r;
        const uint32_t xoff = (src * (uint32_t)K + grp * 16) * (FROM_H ? 4u : 1u);
        const uint32_t xsoff = src * (uint32_t)SK;
        struct Step {
            u32x4 a[NTT][2];
            u32x4 b[FROM_H ? 8 : 2];
            int sw[NM], sx;
        };
        // Block kb; nothing (zeros) behind K.  A lane takes 16 values of each
        // half, so a request reads 64 bytes of a row in one piece.
        auto load = [&](Step &s, int kb) {
            const uint32_t k = (uint32_t)kb * kScaleBlock;
            const bool in[2] = {kb * kScaleBlock < K, kb * kScaleBlock + 64 < K};
#pragma unroll
            for (int m = 0; m < NM; ++m) {
                s.sw[m] = __builtin_amdgcn_raw_buffer_load_b8(sr[m], kb < nb ? kb : kOutside, 0, 0);
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        s.a[m * NT + i][h] = __builtin_bit_cast(
                            u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                       wr[m], in[h] ? woff[i] + k + h * 64 : kOutside, 0, 0));
            }
            if (!FROM_H)
                s.sx = __builtin_amdgcn_raw_buffer_load_b8(
                    xsr, kb < nb ? xsoff + kb : kOutside, 0, 0);
#pragma unroll
            for (int h = 0; h < (FROM_H ? 8 : 2); ++h) {
                const uint32_t at = FROM_H ? k * 4 + (h >> 2) * 256 + (h & 3) * 16 : k + h * 64;
                s.b[h] = __builtin_bit_cast(
                    u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                               xr, in[FROM_H ? h >> 2 : h] ? xoff + at : kOutside, 0, 0));
            }
        };
        floatx4 acc[NTT];
#pragma unroll
        for (int i = 0; i < NTT; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
        auto compute = [&](const Step &s) {
            bf16x8 b[4];
            int ex;
            if (FROM_H) {
                float m = 0.f;
#pragma unroll
                for (int h = 0; h < 8; ++h)
#pragma unroll
                    for (int q = 0; q < 4; ++q) m = fmaxf(m, fabsf(__uint_as_float(s.b[h][q])));
                m = fmaxf(m, __shfl_xor(m, 16));
                m = fmaxf(m, __shfl_xor(m, 32));
                ex = scale_exponent(m);
                const float inv = scale_inverse(ex);
                auto pack = [&](const u32x4 &v) {
                    return pack_e4m3(__uint_as_float(v[0]), __uint_as_float(v[1]),
                                     __uint_as_float(v[2]), __uint_as_float(v[3]), inv);
                };
#pragma unroll
                for (int h = 0; h < 4; ++h) b[h] = widen(pack(s.b[2 * h]), pack(s.b[2 * h + 1]));
            } else {
                ex = s.sx - 127;
#pragma unroll
                for (int h = 0; h < 4; ++h)
                    b[h] = widen(s.b[h >> 1][2 * (h & 1)], s.b[h >> 1][2 * (h & 1) + 1]);
            }
#pragma unroll
            for (int i = 0; i < NTT; ++i) {
                const int sw = s.sw[i / NT];
                floatx4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int h = 0; h < 4; ++h)
                    p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        widen(s.a[i][h >> 1][2 * (h & 1)], s.a[i][h >> 1][2 * (h & 1) + 1]), b[h],
                        p, 0, 0, 0);
                // (scale byte 255 is NaN)
                const float nan = sw == 255 || ex == 128 ? __builtin_nanf("") : 0.f;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    acc[i][r] += __builtin_amdgcn_ldexpf(p[r] + nan, ex + sw - 127);
            }
        };
        Step s[D];
#pragma unroll
        for (int d = 0; d < D; ++d) load(s[d], wave + W * d);
        for (int kb = wave; kb < nb; kb += W * D) {
#pragma unroll
            for (int d = 0; d < D; ++d) {
                compute(s[d]);
                load(s[d], kb + W * (d + D));
            }
        }
        // The lane holds weight rows 4 (lane / 16) + r of token row lane % 16.
#pragma unroll
        for (int i = 0; i < NTT; ++i) part[wave][i][lane] = acc[i];
        __syncthreads();
        for (int i = wave; i < NT; i += W) {
            floatx4 v = part[0][i][lane], u = NM == 2 ? part[0][NT * (NM - 1) + i][lane] : v;
#pragma unroll
            for (int w = 1; w < W; ++w) {
                v += part[w][i][lane];
                if (NM == 2) u += part[w][NT * (NM - 1) + i][lane];
            }
            const int r = m0 + col, n = n0 + i * 16 + grp * 4;
            if (r >= cnt || n >= g.N) continue;
            const int64_t at = ((int64_t)row0 + r) * g.N + n;
            if (MODE == SWIGLU) {
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] = silu_mul(v[x], u[x]);
            }
            if (MODE == OUT_BF16) {
                uint2 p;
                p.x = pack_bf16x2(v[0], v[1]);
                p.y = pack_bf16x2(v[2], v[3]);
                *reinterpret_cast<uint2 *>((bf16_t *)g.out + at) = p;
            } else {
                *reinterpret_cast<floatx4 *>((float *)g.out + at) = v;
            }
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// Products of a few dozen to some hundred rows, where the tiled launch has too
// few tiles for the chip.  A workgroup owns 32 weight rows x 32 token rows
// over the whole of K; its eight waves take blocks of 128 k in turn, each
// straight from memory into the scaled matrix instruction's operands, two
// blocks in flight per wave, and their sums meet in LDS and are added in wave
// order.  So the chain of a launch is an eighth of K long; every operand row is
// read once per workgroup, from the L2.  Tiles of 64 x 128 -> this, GPU us, rows
// x N x K: 20 x 4096 x 4096 17.7 -> 10.9, 40 x 1024 x 4096 15.4 -> 12.0, 128 x 1152
// x 1024 7.6 -> 5.7, 300 x 512 x 1024 7.2 -> 5.7.
// (Tiles of 64 x 32 and 64 x 64 per workgroup serve more rows at once, but no
// faster than the tiled launch: 700 x 1152 x 1024 10.7 against 8.4.)
// ---------------------------------------------------------------------------
constexpr int MNT = 2, MMT = 2;
constexpr int MW = 8, MD = 2;
template <int MODE>
__global__ __launch_bounds__(64 * MW) void mid_kernel(ScaledGemm g) {
    __shared__ __attribute__((aligned(16))) floatx4 part[MW][MNT * MMT][64];
    const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int e = blockIdx.z;
    int row0 = 0, cnt = (int)g.rows_one;
    if (g.offsets) {
        row0 = __builtin_amdgcn_readfirstlane(g.offsets[g.e_first + e]);
        cnt = __builtin_amdgcn_readfirstlane(g.offsets[g.e_first + e + 1]) - row0;
    }
    const int K = g.K, SK = scale_pitch(K), nb = scale_blocks(K);
    const int n0 = blockIdx.x * 16 * MNT;
    const int64_t we = (int64_t)(g.e_first + e) * g.N + n0;
    const int64_t se = (int64_t)(g.e_first + e) * scale_blocks(g.N) + n0 / kScaleBlock;
    const __amdgpu_buffer_rsrc_t wr = rsrc(g.w0 + we * K), sr = rsrc(g.s0 + se * SK);
    uint32_t woff[MNT];
#pragma unroll
    for (int i = 0; i < MNT; ++i)
        woff[i] = (uint32_t)(min(i * 16 + col, g.N - 1 - n0) * K + grp * 16);
    // (more than once only where tokens name an expert twice: the grid covers one
    // row of every token)
    for (int m0 = blockIdx.y * 16 * MMT; m0 < cnt; m0 += gridDim.y * 16 * MMT) {
        const int64_t first = (int64_t)row0 + m0;
        const __amdgpu_buffer_rsrc_t xr = rsrc(g.x + (g.row_map ? 0 : first * K));
        const __amdgpu_buffer_rsrc_t xsr = rsrc(g.xs + (g.row_map ? 0 : first * SK));
        uint32_t xoff[MMT], xsoff[MMT];
#pragma unroll
        for (int j = 0; j < MMT; ++j) {
            const int r = min(j * 16 + col, cnt - 1 - m0);
            const uint32_t src =
                g.row_map ? (uint32_t)(g.row_map[first + r] / g.slot_div) : (uint32_t)r;
            xoff[j] = src * (uint32_t)K + grp * 16;
            xsoff[j] = src * (uint32_t)SK;
        }
        struct Step {
            u32x4 a[MNT][2], b[MMT][2];
            int sw, sx[MMT];
        };
        auto load = [&](Step &s, int kb) {  // nothing (zeros) behind K
            const uint32_t k = (uint32_t)kb * kScaleBlock;
            const bool in[2] = {kb * kScaleBlock < K, kb * kScaleBlock + 64 < K};
            s.sw = __builtin_amdgcn_raw_buffer_load_b8(sr, kb < nb ? kb : kOutside, 0, 0);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int i = 0; i < MNT; ++i)
                    s.a[i][h] = __builtin_bit_cast(
                        u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                   wr, in[h] ? woff[i] + k + h * 64 : kOutside, 0, 0));
#pragma unroll
                for (int j = 0; j < MMT; ++j)
                    s.b[j][h] = __builtin_bit_cast(
                        u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                   xr, in[h] ? xoff[j] + k + h * 64 : kOutside, 0, 0));
            }
#pragma unroll
            for (int j = 0; j < MMT; ++j)
                s.sx[j] =
                    __builtin_amdgcn_raw_buffer_load_b8(xsr, kb < nb ? xsoff[j] + kb : kOutside, 0, 0);
        };
        auto whole = [](const u32x4 (&v)[2]) {
            return v8i{(int)v[0][0], (int)v[0][1], (int)v[0][2], (int)v[0][3],
                       (int)v[1][0], (int)v[1][1], (int)v[1][2], (int)v[1][3]};
        };
        floatx4 acc[MNT][MMT];
#pragma unroll
        for (int i = 0; i < MNT; ++i)
#pragma unroll
            for (int j = 0; j < MMT; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
        Step s[MD];
#pragma unroll
        for (int d = 0; d < MD; ++d) load(s[d], wave + MW * d);
        for (int kb = wave; kb < nb; kb += MW * MD) {
#pragma unroll
            for (int d = 0; d < MD; ++d) {
#pragma unroll
                for (int i = 0; i < MNT; ++i)
#pragma unroll
                    for (int j = 0; j < MMT; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                            whole(s[d].a[i]), whole(s[d].b[j]), acc[i][j], 0, 0, 0, s[d].sw, 0,
                            s[d].sx[j]);
                load(s[d], kb + MW * (d + MD));
            }
        }
#pragma unroll
        for (int i = 0; i < MNT; ++i)
#pragma unroll
            for (int j = 0; j < MMT; ++j) part[wave][i * MMT + j][lane] = acc[i][j];
        __syncthreads();
        for (int q = wave; q < MNT * MMT; q += MW) {
            floatx4 v = part[0][q][lane];
#pragma unroll
            for (int w = 1; w < MW; ++w) v += part[w][q][lane];
            const int r = m0 + (q % MMT) * 16 + col, n = n0 + q / MMT * 16 + grp * 4;
            if (r >= cnt || n >= g.N) continue;
            const int64_t at = ((int64_t)row0 + r) * g.N + n;
            if (MODE == OUT_BF16) {
                uint2 p;
                p.x = pack_bf16x2(v[0], v[1]);
                p.y = pack_bf16x2(v[2], v[3]);
                *reinterpret_cast<uint2 *>((bf16_t *)g.out + at) = p;
            } else {
                *reinterpret_cast<floatx4 *>((float *)g.out + at) = v;
            }
        }
        __syncthreads();
    }
}

template <int MODE>
hipError_t go_mid(const ScaledGemm &g, int64_t max_rows, hipStream_t s) {
    const dim3 grid((unsigned)((g.N + 16 * MNT - 1) / (16 * MNT)),
                    (unsigned)((max_rows + 16 * MMT - 1) / (16 * MMT)), (unsigned)g.e_count);
    mid_kernel<MODE><<<grid, 64 * MW, 0, s>>>(g);
    return hipGetLastError();
}

template <int MODE, bool FROM_H, int NT, int W, int D>
hipError_t go(const ScaledGemm &g, hipStream_t s) {
    const dim3 grid((unsigned)((g.N + 16 * NT - 1) / (16 * NT)), (unsigned)g.e_count);
    stream_kernel<MODE, FROM_H, NT, W, D><<<grid, 64 * W, 0, s>>>(g);
    return hipGetLastError();
}

template <int MODE, bool FROM_H>
hipError_t go_out(const ScaledGemm &g, const ScaledLoad &load, hipStream_t s) {
    // Few blocks of K: four waves, so that each has several.
    if (FROM_H)
        return scale_blocks(g.K) <= 16 ? go<MODE, true, 2, 4, 2>(g, s)
                                       : go<MODE, true, 2, 8, 2>(g, s);
    // Two weight tiles per wave share the token rows' loads and widening, where
    // that leaves more than half of the compute units a workgroup.
    return g.N / 32 * load.active > device_cu_count() / 2
               ? go<MODE, false, 2, 8, 2>(g, s)
               : go<MODE, false, 1, 8, 2>(g, s);
}

}  // namespace

// The kernel reads an expert's weights once for every 16 of its rows, one workgroup
// after the other's steps, so it is for launches in which no expert can have many,
// however uneven the routing: up to 16 tokens for one product, up to 48 for an FFN,
// whose tiled launches of few tiles (below half a tile per compute unit) leave most
// of the chip idle twice.  Tiled -> this, us, from weights that no cache holds, even
// loads and ones with exponents of 1.2:
//   product 1024 x 2048, 16 experts, top 4: 16 tokens 12.7 -> 10.7 and 12.6 -> 10.9;
//     32 tokens 12.7 -> 11.0 and 12.7 -> 14.0; 48 tokens 12.8 -> 13.5 and 12.9 -> 18.0
//   product 1536 x 5120, 20 of 160 experts, top 6: 16 tokens 26.3 -> 24.2 and 22.3 ->
//     18.4; 61 tokens 31.2 -> 36.5 and 30.0 -> 45.9; 420 tokens 34 -> 65 and 48 -> 222
//   FFN 2048 x 512, 64 experts, top 8: 32 tokens 31.9 -> 15.6 and 31.2 -> 25.5; 48
//     tokens 32.0 -> 16.0 and 31.8 -> 35.4; 60 tokens 32 -> 16 and 32 -> 45
//   FFN 2048 x 768, 20 of 160: 48 tokens 39.9 -> 32.1 and 38.1 -> 38.1; 420 tokens
//     42 -> 57 and 43 -> 254
//   FFN of one token 4096 x 3584 (two experts, 56 tiles) 62 -> 26; of four 61 -> 69
bool scaled_stream_fits(int tiles_n, const ScaledLoad &load) {
    return load.max_rows <= kStreamTokens && load.rows <= kStreamRows * load.active &&
           2 * tiles_n * load.active < device_cu_count();
}
// A product of 32 blocks of K and more, four and more for each wave, goes this way
// up to eight tiles per compute unit: over few rounds the last one is part full.
// Tiled -> this, us: four tokens 14336 x 4096 (5.5 experts, 306 tiles) 71 -> 58, 12
// tokens 3584 x 4096 of eight experts 30.6 -> 29.4, 8 rows x 65536 x 4096 (256) 73 ->
// 60, 16 x 32768 x 8192 (128) 63.5 -> 65.7.  (Not an FFN as a whole: its gate and up
// product has twice the operands in flight, and its down product quantises as it reads.)
// Over more than one round that holds for 32 tokens too: 14336 x 4096 of eight experts
// 118 -> 99, with an exponent of 1.2 119 -> 106; 8192 x 6144 of 16 158 -> 159 and 153 ->
// 162, 17 tokens 160 -> 146 and 158 -> 135; of a round 4096 x 14336 86 -> 96 and 87 ->
// 110.  (Of 160 experts with 20 here, 16384 x 5120, 17 tokens 152 -> 166, 24 with 1.2
// 119 -> 151, 32 256 -> 231.)
bool scaled_stream_product_fits(int n, int k, const ScaledLoad &load) {
    const double tiles = scaled_tiles(false, n) * load.active, cus = device_cu_count();
    const bool wide = scale_blocks(k) >= 32 && tiles <= 8 * cus;
    if (load.max_rows > kStreamRows)
        return load.max_rows <= 2 * kStreamRows && load.rows <= kStreamRows * load.active &&
               wide && tiles > cus;
    return wide || scaled_stream_fits(scaled_tiles(false, n), load);
}

// Where the chip runs the workgroups at once.  The grid covers the most rows an
// expert can have, at no more than eight empty workgroups for each that may run.
bool scaled_mid_fits(int N, const ScaledLoad &load) {
    if (load.rows <= 0) return false;
    const double cus = device_cu_count(), cols = (N + 16 * MNT - 1) / (16 * MNT);
    const double grid = cols * load.experts * ((load.max_rows + 16 * MMT - 1) / (16 * MMT));
    return cols * load.active * std::ceil(load.rows / load.active / (16 * MMT)) <= cus &&
           grid <= 9 * cus;
}
hipError_t launch_mid_scaled(const ScaledGemm &g, int y_type, int64_t max_rows, hipStream_t s) {
    return y_type == MOE_FP32 ? go_mid<OUT_F32>(g, max_rows, s) : go_mid<OUT_BF16>(g, max_rows, s);
}
hipError_t launch_stream_scaled(const ScaledGemm &g, int y_type, bool from_h,
                                const ScaledLoad &load, hipStream_t s) {
    if (y_type == MOE_FP32)
        return from_h ? go_out<OUT_F32, true>(g, load, s) : go_out<OUT_F32, false>(g, load, s);
    return from_h ? go_out<OUT_BF16, true>(g, load, s) : go_out<OUT_BF16, false>(g, load, s);
}
hipError_t launch_stream_swiglu(const ScaledGemm &g, const ScaledLoad &load, hipStream_t s) {
    return go<SWIGLU, false, 2, 8, 2>(g, s);
}

}  // namespace moe
