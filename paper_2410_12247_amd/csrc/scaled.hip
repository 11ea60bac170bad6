// Products over block-scaled 8-bit tensors on the gfx950 matrix cores.
#include <algorithm>

#include "scaled.h"

namespace moe {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr int NXCD = 8;
constexpr int GROUP_N = 8;  // n-tiles per super-column of the tile order

enum { SWIGLU = 0, OUT_F32 = 1, OUT_BF16 = 2 };

__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
    const uint16_t ua = __builtin_bit_cast(uint16_t, static_cast<__bf16>(a));
    const uint16_t ub = __builtin_bit_cast(uint16_t, static_cast<__bf16>(b));
    return (uint32_t)ua | ((uint32_t)ub << 16);
}
// as in the bf16 GEMMs: hardware exp2 and reciprocal (about 1 ulp each; the
// result is rounded to e4m3 next)
__device__ __forceinline__ float silu_mul(float g, float u) {
    const float e = __builtin_amdgcn_exp2f(g * -1.44269504088896341f);
    return g * __builtin_amdgcn_rcpf(1.0f + e) * u;
}

template <int MODE, int BM_>
struct Cfg {
    static constexpr int BM = BM_;
    static constexpr int BN = 256;                          // weight rows of the tile
    static constexpr int BNOUT = MODE == SWIGLU ? 128 : 256;  // output columns
    static constexpr int THREADS = 256;
    static constexpr int WTN = 128, WTM = BM / 2;
    static constexpr int TN = WTN / 32, TM = WTM / 32;
    static constexpr int ES = MODE == OUT_F32 ? 4 : 2;
    static constexpr int OUT_ROW = 128 * ES + 16;  // scratch row of the epilogue
    static constexpr int LDS_BYTES =
        MODE == SWIGLU ? BM * 128 + 2 * BM * 4 : 4 * 32 * OUT_ROW;
};

struct Tile {
    int e;              // expert of the launch
    int64_t r0, n0;     // first product row, first output column
    int m_valid, n_valid;
};

// Walks the tiles of all experts; s_off, s_pre: e_count + 1 ints each in LDS.
template <class C>
struct Walk {
    int *s_off, *s_pre;
    int NT, total;
    __device__ __forceinline__ Walk(const ScaledGemm &g, int *lds) {
        s_off = lds;
        s_pre = lds + kMaxExperts + 1;
        NT = (g.N + C::BNOUT - 1) / C::BNOUT;
        const int tid = threadIdx.x;
        for (int i = tid; i <= g.e_count; i += C::THREADS)
            s_off[i] = g.offsets ? g.offsets[g.e_first + i] : (i == 0 ? 0 : (int)g.rows_one);
        __syncthreads();
        if (tid == 0) {
            int t = 0;
            for (int e = 0; e < g.e_count; ++e) {
                s_pre[e] = t;
                t += (s_off[e + 1] - s_off[e] + C::BM - 1) / C::BM * NT;
            }
            s_pre[g.e_count] = t;
        }
        __syncthreads();
        total = __builtin_amdgcn_readfirstlane(s_pre[g.e_count]);
    }
    __device__ __forceinline__ Tile tile(const ScaledGemm &g, int tau) const {
        auto lds = [](const int &v) { return __builtin_amdgcn_readfirstlane(v); };
        int lo = 0, hi = g.e_count - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (lds(s_pre[mid]) <= tau) lo = mid; else hi = mid - 1;
        }
        const int row0 = lds(s_off[lo]);
        const int cnt = lds(s_off[lo + 1]) - row0;
        const int MT = (cnt + C::BM - 1) / C::BM;
        const int r = tau - lds(s_pre[lo]);
        const int per_sc = GROUP_N * MT;
        const int sc = r / per_sc;
        const int q = r - sc * per_sc;
        const int width = min(GROUP_N, NT - sc * GROUP_N);
        const int mt = q / width, nt = sc * GROUP_N + (q - mt * width);
        Tile t;
        t.e = lo;
        t.r0 = (int64_t)row0 + (int64_t)mt * C::BM;
        t.n0 = (int64_t)nt * C::BNOUT;
        t.m_valid = min(C::BM, cnt - mt * C::BM);
        t.n_valid = min(C::BNOUT, (int)(g.N - t.n0));
        return t;
    }
};

template <int MODE, int BM_>
__global__ __launch_bounds__(256) void scaled_kernel(ScaledGemm g) {
    using C = Cfg<MODE, BM_>;
    __shared__ __attribute__((aligned(16))) char smem[C::LDS_BYTES];
    __shared__ int s_int[2 * (kMaxExperts + 1)];
    const Walk<C> walk(g, s_int);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave & 1, wm = wave >> 1;
    const int K = g.K, SK = scale_pitch(K);

    for (int tau = blockIdx.x; tau < walk.total; tau += gridDim.x) {
        const Tile t = walk.tile(g, tau);
        // operand rows of this lane
        const uint8_t *wrow[C::TN], *xrow[C::TM], *wsc[C::TN], *xsc[C::TM];
        const int64_t we = (int64_t)(g.e_first + t.e) * g.N;
        const int64_t se = (int64_t)(g.e_first + t.e) * scale_blocks(g.N);
#pragma unroll
        for (int i = 0; i < C::TN; ++i) {
            const bool up = MODE == SWIGLU && i >= C::TN / 2;
            const int r = MODE == SWIGLU ? wn * 64 + (i % 2) * 32 : wn * 128 + i * 32;
            const int64_t row = t.n0 + min(r + (lane & 31), t.n_valid - 1);
            wrow[i] = (up ? g.w1 : g.w0) + (we + row) * K;
            wsc[i] = (up ? g.s1 : g.s0) + (se + row / kScaleBlock) * SK;
        }
#pragma unroll
        for (int j = 0; j < C::TM; ++j) {
            const int64_t r = t.r0 + min(wm * C::WTM + j * 32 + (lane & 31), t.m_valid - 1);
            const int64_t src = g.row_map ? g.row_map[r] / g.slot_div : r;
            xrow[j] = g.x + src * K;
            xsc[j] = g.xs + src * SK;
        }
        floatx16 acc[C::TN][C::TM];
#pragma unroll
        for (int i = 0; i < C::TN; ++i)
#pragma unroll
            for (int j = 0; j < C::TM; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
        for (int k = 0; k < K; k += 64) {
            const int at = k + (lane >> 5) * 32;
            v8i a[C::TN], b[C::TM];
            int sa[C::TN], sb[C::TM];
            auto load = [&](const uint8_t *p) {
                const u32x4 lo = *reinterpret_cast<const u32x4 *>(p + at);
                const u32x4 hi = *reinterpret_cast<const u32x4 *>(p + at + 16);
                return v8i{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3],
                           (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
            };
#pragma unroll
            for (int i = 0; i < C::TN; ++i) a[i] = load(wrow[i]), sa[i] = wsc[i][k / kScaleBlock];
#pragma unroll
            for (int j = 0; j < C::TM; ++j) b[j] = load(xrow[j]), sb[j] = xsc[j][k / kScaleBlock];
#pragma unroll
            for (int i = 0; i < C::TN; ++i)
#pragma unroll
                for (int j = 0; j < C::TM; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                        a[i], b[j], acc[i][j], 0, 0, 0, sa[i], 0, sb[j]);
        }
        // The lane holds, of token row wm WTM + 32 j + lane % 32, the weight
        // rows 32 i + 8 (r / 4) + 4 (lane / 32) + r % 4.
        const int half = lane >> 5;
        __syncthreads();
        if constexpr (MODE == SWIGLU) {
            float *smax = reinterpret_cast<float *>(smem + C::BM * 128);  // [2][BM]
#pragma unroll
            for (int j = 0; j < C::TM; ++j) {
                float m = 0.f;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float h = wn * 64 + i * 32 < t.n_valid
                                            ? silu_mul(acc[i][j][r], acc[i + 2][j][r])
                                            : 0.f;
                        acc[i][j][r] = h;
                        m = fmaxf(m, fabsf(h));
                    }
                m = fmaxf(m, __shfl_xor(m, 32));
                if (half == 0) smax[wn * C::BM + wm * C::WTM + j * 32 + lane] = m;
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < C::TM; ++j) {
                const int row = wm * C::WTM + j * 32 + (lane & 31);
                const int e = scale_exponent(fmaxf(smax[row], smax[C::BM + row]));
                const float inv = scale_inverse(e);
                if (wn == 0 && half == 0 && row < t.m_valid)
                    g.out_s[(t.r0 + row) * scale_pitch(g.N) + t.n0 / kScaleBlock] = scale_byte(e);
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int col = wn * 64 + i * 32 + r * 8 + half * 4;
                        // 16-byte chunks swizzled by the row
                        char *p = smem + row * 128 + (((col >> 4) ^ (row & 7)) << 4) + (col & 15);
                        *reinterpret_cast<uint32_t *>(p) =
                            pack_e4m3(acc[i][j][4 * r], acc[i][j][4 * r + 1], acc[i][j][4 * r + 2],
                                      acc[i][j][4 * r + 3], inv);
                    }
            }
            __syncthreads();
            for (int c = threadIdx.x; c < C::BM * 8; c += C::THREADS) {
                const int row = c >> 3, chunk = c & 7;
                if (row < t.m_valid && chunk * 16 < t.n_valid)
                    *reinterpret_cast<u32x4 *>((uint8_t *)g.out + (t.r0 + row) * g.N + t.n0 +
                                               chunk * 16) =
                        *reinterpret_cast<const u32x4 *>(smem + row * 128 +
                                                         ((chunk ^ (row & 7)) << 4));
            }
        } else {
            char *sc = smem + wave * 32 * C::OUT_ROW;
            constexpr int CPR = 128 * C::ES / 16, RPI = 64 / CPR;  // chunks per row, rows per pass
#pragma unroll
            for (int j = 0; j < C::TM; ++j) {
#pragma unroll
                for (int i = 0; i < C::TN; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const floatx16 &v = acc[i][j];
                        char *p = sc + (lane & 31) * C::OUT_ROW +
                                  (i * 32 + r * 8 + half * 4) * C::ES;
                        if (MODE == OUT_F32) {
                            *reinterpret_cast<floatx4 *>(p) =
                                floatx4{v[4 * r], v[4 * r + 1], v[4 * r + 2], v[4 * r + 3]};
                        } else {
                            uint2 u;
                            u.x = pack_bf16x2(v[4 * r], v[4 * r + 1]);
                            u.y = pack_bf16x2(v[4 * r + 2], v[4 * r + 3]);
                            *reinterpret_cast<uint2 *>(p) = u;
                        }
                    }
                __builtin_amdgcn_wave_barrier();
                for (int q = 0; q < 32 / RPI; ++q) {
                    const int rr = q * RPI + lane / CPR, chunk = lane % CPR;
                    const int row = wm * C::WTM + j * 32 + rr;
                    const int col = wn * 128 + chunk * (16 / C::ES);
                    const u32x4 v =
                        *reinterpret_cast<const u32x4 *>(sc + rr * C::OUT_ROW + chunk * 16);
                    if (row < t.m_valid && col < t.n_valid)
                        *reinterpret_cast<u32x4 *>((char *)g.out +
                                                   ((t.r0 + row) * g.N + t.n0 + col) * C::ES) = v;
                }
                __builtin_amdgcn_wave_barrier();
            }
        }
    }
}

template <int MODE>
hipError_t go(const ScaledGemm &g, const ScaledLoad &, hipStream_t s) {
    scaled_kernel<MODE, 128><<<(unsigned)device_cu_count(), 256, 0, s>>>(g);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_scaled_gemm(const ScaledGemm &g, int y_type, const ScaledLoad &load,
                              hipStream_t s) {
    return y_type == MOE_FP32 ? go<OUT_F32>(g, load, s) : go<OUT_BF16>(g, load, s);
}
hipError_t launch_scaled_swiglu(const ScaledGemm &g, const ScaledLoad &load, hipStream_t s) {
    return go<SWIGLU>(g, load, s);
}

}  // namespace moe
