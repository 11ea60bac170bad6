// Block-scaled 8-bit tensors: what the quantising kernels and the products
// over them share.
//
// A value is an OCP e4m3 number times the power of two of its block.  An
// activation row has one scale byte (E8M0: 2^(byte - 127)) per 128 columns,
// a weight matrix one per 128 x 128 block.  Scale rows are padded to whole
// 4-byte words (scale_pitch), so four blocks' scales load as one word.
#pragma once

#include "common.h"

namespace moe {

constexpr int kScaleBlock = 128;
// Byte offsets into a gathered token matrix and into one tile's rows are 32-bit.
constexpr uint64_t kMaxOffset = uint64_t(1) << 32;

__host__ __device__ constexpr int scale_blocks(int k) { return (k + kScaleBlock - 1) / kScaleBlock; }
__host__ __device__ constexpr int scale_pitch(int k) { return (scale_blocks(k) + 3) / 4 * 4; }

// What a launch of the product kernels covers.  Rows of local expert e (of
// e_count, weights of expert e_first + e) are [offsets[e_first + e],
// offsets[e_first + e + 1]); offsets NULL: one expert of rows_one rows.
// row_map NULL: row r of the product is row r of x, else row
// row_map[r] / slot_div.
struct ScaledGemm {
    const int32_t *offsets;
    int e_first, e_count;
    int64_t rows_one;
    const uint8_t *x, *xs;
    const int32_t *row_map;
    int slot_div;
    const uint8_t *w0, *s0;  // weights and scales (gate of the SwiGLU launch)
    const uint8_t *w1, *s1;  // up
    int N, K;
    void *out;       // y [.][N], or the SwiGLU launch's e4m3 rows
    uint8_t *out_s;  // their scales
};
// What a launch's form is chosen by: the rows expected in all and the experts
// expected to have any, the most rows an expert can have and the experts.
struct ScaledLoad {
    double rows, active;
    int64_t max_rows;
    int experts;
};

// y = x w^T, y_type MOE_FP32 or MOE_BF16.
hipError_t launch_scaled_gemm(const ScaledGemm &g, int y_type, const ScaledLoad &load,
                              hipStream_t s);
// out = Q(silu(x w0^T) * x w1^T).
hipError_t launch_scaled_swiglu(const ScaledGemm &g, const ScaledLoad &load, hipStream_t s);

// The same for few rows per expert (scaled_stream_fits).  The SwiGLU launch
// leaves its rows in fp32 (out [.][N], out_s unused); the product behind it
// takes them so (from_h: x is fp32) and quantises them as it reads them.
// tiles_n: column tiles of the (first) tiled launch (scaled_tiles).
constexpr int64_t kStreamRows = 16;    // expected per expert that has any
constexpr int64_t kStreamTokens = 48;  // the most rows of an expert, in an FFN
bool scaled_stream_fits(int tiles_n, const ScaledLoad &load);
bool scaled_stream_product_fits(int n, int k, const ScaledLoad &load);  // of one product
constexpr int scaled_tiles(bool swiglu, int n) { return (n + (swiglu ? 127 : 255)) / (swiglu ? 128 : 256); }
hipError_t launch_stream_scaled(const ScaledGemm &g, int y_type, bool from_h,
                                const ScaledLoad &load, hipStream_t s);
hipError_t launch_stream_swiglu(const ScaledGemm &g, const ScaledLoad &load, hipStream_t s);

// Products of a few dozen to some hundred rows, where the tiled launch has too
// few tiles (scaled_mid_fits).
bool scaled_mid_fits(int N, const ScaledLoad &load);
hipError_t launch_mid_scaled(const ScaledGemm &g, int y_type, int64_t max_rows, hipStream_t s);

// Rows quantised, with (norm) or without the residual addition and RMS norm.
hipError_t launch_norm_quant(int64_t rows, int cols, const void *x, int x_type,
                             const bf16_t *residual, bool norm, const bf16_t *weight, float eps,
                             bf16_t *total, bf16_t *y, uint8_t *q, uint8_t *scales,
                             hipStream_t s);
hipError_t launch_quant_weights(int experts, int n, int k, const bf16_t *w, uint8_t *q,
                                uint8_t *scales, hipStream_t s);

#ifdef __HIPCC__
namespace {

// Smallest e with amax <= 448 * 2^e (448 = 1.75 * 2^8, the largest e4m3
// value), from the bits of amax: no value of the block is out of range, and
// the scale costs at most one of the format's 17 binades.  0 for an empty
// block.  An infinite amax gives 120: the infinity leaves the conversion as
// NaN and the block's other values vanish beside it.
__device__ __forceinline__ int scale_exponent(float amax) {
    const uint32_t u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return u == 0 ? 0 : max(e, -127);
}
__device__ __forceinline__ uint8_t scale_byte(int e) { return (uint8_t)(e + 127); }
// 2^-e, e in [-127, 121]
__device__ __forceinline__ float scale_inverse(int e) {
    return __uint_as_float((uint32_t)(127 - e) << 23);
}
// Four values times inv, rounded to e4m3 (nearest, ties to even).
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d, float inv) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, v, true);
}

}  // namespace
#endif

}  // namespace moe
