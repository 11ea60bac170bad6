// Rows and weights into block-scaled 8 bits.
//
// norm_quant: s = x + residual, total = bf16(s), v = s rsqrt(mean s^2 + eps) w,
// y = bf16(v) and Q(v) with one scale per 128 columns, in one pass over the row:
// a workgroup holds a row (or a wave holds one, for short rows) in registers, so
// nothing is read twice and Q sees v before its rounding to bf16.  A lane holds
// eight consecutive columns, so a block of 128 is one DPP row of 16 lanes and
// its largest value needs no LDS.
//
// It is bound by memory: 16384 x 5120 (fp32 x, bf16 residual, total and y) moves
// 923 MB in 171 us, 5.4 TB/s; 16384 x 8192 5.7 TB/s; the quantisation alone of
// bf16 rows 16384 x 5120, 254 MB, in 45 us, 5.6 TB/s.  One row of 4096 takes 3.2
// us, a launch's latency and a chain of loads, sum, reciprocal root and stores.
// So the arithmetic between the loads and the two roundings is in 64 bits, under
// the memory's time: in fp32 some 50 of those 84 million values are rounded to
// the neighbour of the definition's, here none (166 us in fp32).  Eight waves a
// row: four with twice the passes take 179 us and 3.7 (one row), sixteen 198.
#include <algorithm>

#include "scaled.h"

namespace moe {
namespace {

constexpr int VEC = 8;

struct NormArgs {
    int64_t rows;
    int cols;
    const void *x;
    const bf16_t *residual, *weight;
    float eps;
    bf16_t *total, *y;
    uint8_t *q, *scales;
    double one_col;  // 1 / cols
};

__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }
__device__ __forceinline__ void load8(const bf16_t *p, float (&v)[VEC]) {
    const u32x4 u = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = bf16_lo(u[i]);
        v[2 * i + 1] = bf16_hi(u[i]);
    }
}
__device__ __forceinline__ void load8(const float *p, float (&v)[VEC]) {
    const floatx4 a = *reinterpret_cast<const floatx4 *>(p);
    const floatx4 b = *reinterpret_cast<const floatx4 *>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = a[i];
        v[4 + i] = b[i];
    }
}
__device__ __forceinline__ void store8(bf16_t *p, const float (&v)[VEC]) {
    u32x4 u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint16_t a = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v[2 * i]));
        const uint16_t b = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v[2 * i + 1]));
        u[i] = (uint32_t)a | ((uint32_t)b << 16);
    }
    *reinterpret_cast<u32x4 *>(p) = u;
}

// the largest of the 16 lanes of a DPP row
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __int_as_float(
        __builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float row_max(float v) {
    v = fmaxf(v, dpp<0x128>(v));  // row_ror:8
    v = fmaxf(v, dpp<0x124>(v));
    v = fmaxf(v, dpp<0x122>(v));
    return fmaxf(v, dpp<0x121>(v));
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    return v;
}
// Eight columns of x + residual, exactly: two fp32 numbers whose sum has 64
// bits' room.
struct Sum8 {
    float x[VEC], r[VEC];
    __device__ __forceinline__ double operator[](int i) const { return (double)x[i] + (double)r[i]; }
    __device__ __forceinline__ void rounded(float (&s)[VEC]) const {
#pragma unroll
        for (int i = 0; i < VEC; ++i) s[i] = x[i] + r[i];
    }
    __device__ __forceinline__ double squares(double v) const {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const double s = (*this)[i];
            v = __builtin_fma(s, s, v);
        }
        return v;
    }
};
__device__ __forceinline__ double inverse_rms(double ss, const NormArgs &a) {
    return rsqrt(__builtin_fma(ss, a.one_col, (double)a.eps));
}
// To fp32 with the last bit set where bits behind it are: what is rounded from
// this to fewer bits (bf16, e4m3) is rounded as if from v itself.
__device__ __forceinline__ float to_odd(double v) {
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    const uint32_t lo = (uint32_t)u;
    const uint32_t cut = (lo & 0xE0000000u) | ((lo & 0x1FFFFFFFu) ? 0x20000000u : 0u);
    return (float)__longlong_as_double((long long)((u & 0xFFFFFFFF00000000ull) | cut));
}
// (x + residual) rstd weight
__device__ __forceinline__ void normalise(const Sum8 &s, double rstd, const bf16_t *weight,
                                          float (&v)[VEC]) {
    float w[VEC];
    if (weight) load8(weight, w);
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = to_odd(weight ? s[i] * rstd * (double)w[i] : s[i] * rstd);
}

// One pass' eight columns of every lane: quantised (all lanes take part; a
// lane past the row's end holds zeros).
__device__ __forceinline__ void quant8(const NormArgs &a, int64_t row, int col,
                                       const float (&v)[VEC]) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < VEC; ++i) m = fmaxf(m, fabsf(v[i]));
    const int e = scale_exponent(row_max(m));
    if (col >= a.cols) return;
    const float inv = scale_inverse(e);
    uint2 p;
    p.x = pack_e4m3(v[0], v[1], v[2], v[3], inv);
    p.y = pack_e4m3(v[4], v[5], v[6], v[7], inv);
    *reinterpret_cast<uint2 *>(a.q + row * a.cols + col) = p;
    if ((threadIdx.x & 15) == 0)
        a.scales[row * scale_pitch(a.cols) + col / kScaleBlock] = scale_byte(e);
}

// WAVES waves share a row of at most 512 WAVES PASSES columns.
template <class X, bool NORM, int WAVES, int PASSES>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void norm_quant_kernel(NormArgs a) {
    constexpr int THREADS = 64 * WAVES;
    const int tid = WAVES == 1 ? (int)(threadIdx.x & 63) : (int)threadIdx.x;
    const int64_t row =
        WAVES == 1 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : (int64_t)blockIdx.x;
    if (row >= a.rows) return;
    const X *x = reinterpret_cast<const X *>(a.x) + row * a.cols;
    Sum8 s[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int col = (p * THREADS + tid) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) s[p].x[i] = 0.f, s[p].r[i] = -0.f;  // x + -0 is x, signs too
        if (col >= a.cols) continue;
        load8(x + col, s[p].x);
        if (NORM && a.residual) load8(a.residual + row * a.cols + col, s[p].r);
    }
    double rstd = 1.;
    if (NORM) {
        double ss = 0.;
#pragma unroll
        for (int p = 0; p < PASSES; ++p) ss = s[p].squares(ss);
        ss = wave_sum(ss);
        if (WAVES > 1) {
            __shared__ double part[WAVES];
            if ((tid & 63) == 0) part[tid >> 6] = ss;
            __syncthreads();
            ss = 0.;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) ss += part[w];
        }
        rstd = inverse_rms(ss, a);
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int col = (p * THREADS + tid) * VEC;
        float v[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = s[p].x[i];
        if (NORM && col < a.cols) {
            if (a.total) {
                s[p].rounded(v);
                store8(a.total + row * a.cols + col, v);
            }
            normalise(s[p], rstd, a.weight ? a.weight + col : nullptr, v);
            if (a.y) store8(a.y + row * a.cols + col, v);
        }
        if (a.q) quant8(a, row, col, v);
    }
}

// Rows longer than the registers hold: read twice.
template <class X, bool NORM>
__global__ __launch_bounds__(1024) void norm_quant_long_kernel(NormArgs a) {
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    const X *x = reinterpret_cast<const X *>(a.x) + row * a.cols;
    auto load = [&](int col, Sum8 &s) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) s.r[i] = -0.f;
        load8(x + col, s.x);
        if (NORM && a.residual) load8(a.residual + row * a.cols + col, s.r);
    };
    double rstd = 1.;
    if (NORM) {
        double ss = 0.;
        for (int col = tid * VEC; col < a.cols; col += 1024 * VEC) {
            Sum8 s;
            load(col, s);
            ss = s.squares(ss);
        }
        ss = wave_sum(ss);
        __shared__ double part[16];
        if ((tid & 63) == 0) part[tid >> 6] = ss;
        __syncthreads();
        ss = 0.;
        for (int w = 0; w < 16; ++w) ss += part[w];
        rstd = inverse_rms(ss, a);
    }
    for (int c0 = 0; c0 < a.cols; c0 += 1024 * VEC) {
        const int col = c0 + tid * VEC;
        float v[VEC] = {};
        if (col < a.cols) {
            Sum8 s;
            load(col, s);
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = s.x[i];
            if (NORM) {
                // (a lane reads its columns of the residual before it writes
                // them: total may be the residual itself)
                if (a.total) {
                    s.rounded(v);
                    store8(a.total + row * a.cols + col, v);
                }
                normalise(s, rstd, a.weight ? a.weight + col : nullptr, v);
                if (a.y) store8(a.y + row * a.cols + col, v);
            }
        }
        if (a.q) quant8(a, row, col, v);
    }
}

// One 128 x 128 block of a weight matrix per workgroup: the block's 64 values
// per thread stay in registers between the maximum and the conversion, so the
// weights are read once.  Bound by memory: 16 x 1344 x 6144 (396 MB moved) 76 us,
// 5.2 TB/s.
__global__ __launch_bounds__(256) void quant_weights_kernel(const bf16_t *__restrict__ w,
                                                            uint8_t *__restrict__ q,
                                                            uint8_t *__restrict__ scales, int n,
                                                            int k) {
    const int kb = blockIdx.x, nb = blockIdx.y;
    const int64_t e = blockIdx.z;
    const int col = kb * kScaleBlock + (threadIdx.x & 15) * VEC;
    const int r0 = nb * kScaleBlock + (threadIdx.x >> 4);
    const bf16_t *we = w + e * n * k;
    float v[8][VEC];
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = r0 + 16 * i;
        if (r < n && col < k) {
            load8(we + (int64_t)r * k + col, v[i]);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[i][j] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) m = fmaxf(m, fabsf(v[i][j]));
    }
    m = row_max(m);
    m = fmaxf(m, __shfl_xor(m, 16));
    m = fmaxf(m, __shfl_xor(m, 32));
    __shared__ float part[4];
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
    const int ex = scale_exponent(m);
    const float inv = scale_inverse(ex);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = r0 + 16 * i;
        if (r >= n || col >= k) continue;
        uint2 p;
        p.x = pack_e4m3(v[i][0], v[i][1], v[i][2], v[i][3], inv);
        p.y = pack_e4m3(v[i][4], v[i][5], v[i][6], v[i][7], inv);
        *reinterpret_cast<uint2 *>(q + (e * n + r) * k + col) = p;
    }
    if (threadIdx.x == 0)
        scales[(e * scale_blocks(n) + nb) * scale_pitch(k) + kb] = scale_byte(ex);
}

// (a launch holds fewer than 2^32 threads)
constexpr int64_t kRowsPerLaunch = 1 << 21;

template <class X, bool NORM>
hipError_t go_norm(NormArgs a, hipStream_t s) {
    for (int64_t left = a.rows; left > 0; left -= kRowsPerLaunch) {
        a.rows = std::min(left, kRowsPerLaunch);
        const dim3 rows((unsigned)a.rows);
        if (a.cols <= 512)
            norm_quant_kernel<X, NORM, 1, 1><<<(unsigned)((a.rows + 3) / 4), 256, 0, s>>>(a);
        else if (a.cols <= 2048)
            norm_quant_kernel<X, NORM, 4, 1><<<rows, 256, 0, s>>>(a);
        else if (a.cols <= 4096)
            norm_quant_kernel<X, NORM, 8, 1><<<rows, 512, 0, s>>>(a);
        else if (a.cols <= 8192)
            norm_quant_kernel<X, NORM, 8, 2><<<rows, 512, 0, s>>>(a);
        else
            norm_quant_long_kernel<X, NORM><<<rows, 1024, 0, s>>>(a);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
        const int64_t n = a.rows * a.cols;
        a.x = reinterpret_cast<const X *>(a.x) + n;
        if (a.residual) a.residual += n;
        if (a.total) a.total += n;
        if (a.y) a.y += n;
        if (a.q) a.q += n, a.scales += a.rows * scale_pitch(a.cols);
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_norm_quant(int64_t rows, int cols, const void *x, int x_type,
                             const bf16_t *residual, bool norm, const bf16_t *weight, float eps,
                             bf16_t *total, bf16_t *y, uint8_t *q, uint8_t *scales,
                             hipStream_t s) {
    const NormArgs a{rows, cols, x, residual, weight, eps, total, y, q, scales,
                     1.0 / cols};
    if (x_type == MOE_FP32)
        return norm ? go_norm<float, true>(a, s) : go_norm<float, false>(a, s);
    return norm ? go_norm<bf16_t, true>(a, s) : go_norm<bf16_t, false>(a, s);
}

hipError_t launch_quant_weights(int experts, int n, int k, const bf16_t *w, uint8_t *q,
                                uint8_t *scales, hipStream_t s) {
    const dim3 grid((unsigned)scale_blocks(k), (unsigned)scale_blocks(n), (unsigned)experts);
    quant_weights_kernel<<<grid, 256, 0, s>>>(w, q, scales, n, k);
    return hipGetLastError();
}

}  // namespace moe
