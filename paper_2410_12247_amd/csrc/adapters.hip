// Low-rank adapters of many requests beside a shared projection,
//   y = base + scale (x A^T) B^T,
// and their gradient.  Rows are ordered by adapter, as the dispatch orders
// tokens by expert; a tile is up to 16 or 64 rows of one adapter, found on the
// device from the adapters' offsets.
//
// The sums over K of x A^T ("shrink") go through memory in fp32: rank values a
// row, where the rows themselves have thousands.  The products behind it take
// them cut into bf16 parts (hi + mid + lo hold all 24 bits), so that the matrix
// cores multiply bf16 by bf16 without a rounding.
#include "adapters.h"

namespace moe {
namespace {

constexpr int kWaves = 4;

__device__ __forceinline__ floatx4 mfma(bf16x8 a, bf16x8 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ bf16x8 load8(const bf16_t *p) {
    return *reinterpret_cast<const bf16x8 *>(p);
}

__device__ __forceinline__ int scan64(int v, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// One tile: adapter e's places [first, first + rows), the tile's number among
// the adapter's `tiles`, and the tiles of several-tile adapters before it.
struct Tile {
    int e, rows, index, tiles, several;
    int64_t first;
};

// Tile t of all adapters' tiles of TM rows; e < 0 behind the last.  Every lane
// takes four adapters' counts; a scan over the lanes finds the tile's.
// Offsets outside [0, rows] are cut to it.
template <int TM>
__device__ Tile find_tile(const AdapterRows &o, int t) {
    const int lane = threadIdx.x & 63;
    int at[5], n[4], sum = 0, sev = 0;
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        const int e = min(lane * 4 + i, o.count);
        at[i] = (int)min((int64_t)max(o.offsets[e], 0), o.rows);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        n[i] = (max(at[i + 1] - at[i], 0) + TM - 1) / TM;
        sum += n[i];
        sev += n[i] > 1 ? n[i] : 0;
    }
    const int incl = scan64(sum, lane), sincl = scan64(sev, lane);
    Tile r{-1, 0, 0, 0, 0, 0};
    const uint64_t has = __ballot(incl > t);
    if (!has) return r;
    const int l = __builtin_ctzll(has);
    int left = t - (incl - sum), before = sincl - sev, e = lane * 4, mine = 0;
    int64_t first = at[0];
    int last = at[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (mine == i && left >= n[i] && i < 3) {
            left -= n[i];
            before += n[i] > 1 ? n[i] : 0;
            mine = i + 1;
            e = lane * 4 + i + 1;
            first = at[i + 1];
            last = at[i + 2 > 4 ? 4 : i + 2];
        }
    }
    r.e = __shfl(e, l);
    r.index = __shfl(left, l);
    r.several = __shfl(before, l);
    const int f = __shfl((int)first, l), z = __shfl(last, l);
    r.tiles = (z - f + TM - 1) / TM;
    r.first = f + (int64_t)r.index * TM;
    r.rows = min(TM, (int)(z - r.first));
    return r;
}

__device__ __forceinline__ int row_at(const AdapterRows &o, int64_t place) {
    const int row = o.order[place];
    return (uint32_t)row < (uint64_t)o.rows ? row : -1;
}

// ---- x A^T ---------------------------------------------------------------
// The matrix instruction's M is the rank, its N the rows: a lane ends with four
// consecutive rank values of a row.  Lane group g (16 lanes) takes k = 16 g ..
// 16 g + 15 of every 64, in two 16-byte loads.
template <int RB, int NR>
__global__ __launch_bounds__(64 * kWaves) void shrink_kernel(AdapterRows o, int rank, int K,
                                                             const bf16_t *__restrict__ x,
                                                             const bf16_t *__restrict__ w,
                                                             float *__restrict__ p, int splits) {
    const Tile t = find_tile<16 * RB>(o, blockIdx.x);
    if (t.e < 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
    const int split = blockIdx.y, r0 = blockIdx.z * 16 * NR;
    const bf16_t *xr[RB], *wr[NR];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int row = row_at(o, t.first + min(16 * b + m, t.rows - 1));
        xr[b] = x + (int64_t)max(row, 0) * K + 16 * g;
    }
#pragma unroll
    for (int b = 0; b < NR; ++b)
        wr[b] = w + ((int64_t)t.e * rank + min(r0 + 16 * b + m, rank - 1)) * K + 16 * g;
    floatx4 acc[RB][NR] = {};
    const int steps = K / 64, parts = splits * kWaves, part = split * kWaves + wave;
    const int lo = steps * part / parts, hi = steps * (part + 1) / parts;
#pragma unroll 2
    for (int s = lo; s < hi; ++s) {
        bf16x8 xv[RB][2], wv[NR][2];
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) xv[b][h] = load8(xr[b] + s * 64 + 8 * h);
#pragma unroll
        for (int b = 0; b < NR; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) wv[b][h] = load8(wr[b] + s * 64 + 8 * h);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
                for (int c = 0; c < NR; ++c) acc[b][c] = mfma(wv[c][h], xv[b][h], acc[b][c]);
    }
    // the waves' sums meet in LDS
    __shared__ floatx4 part_sum[kWaves][RB * NR][64];
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int c = 0; c < NR; ++c) part_sum[wave][b * NR + c][lane] = acc[b][c];
    __syncthreads();
    for (int i = wave; i < RB * NR; i += kWaves) {
        floatx4 v = part_sum[0][i][lane];
#pragma unroll
        for (int q = 1; q < kWaves; ++q) v += part_sum[q][i][lane];
        const int row = 16 * (i / NR) + m, r = r0 + 16 * (i % NR) + 4 * g;
        if (row < t.rows && r < rank)
            *reinterpret_cast<floatx4 *>(p + ((int64_t)split * o.rows + t.first + row) * rank + r) =
                v;
    }
}

// ---- + scale u B^T -------------------------------------------------------

// hi + mid (+ lo): the leading 8 bits by cutting, the last part rounded.
template <int S>
__device__ __forceinline__ void cut(float v, uint32_t (&part)[S]) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
        const uint32_t u = __float_as_uint(v);
        if (i + 1 < S) {
            part[i] = u >> 16;
            v = (u & 0x7F800000u) == 0x7F800000u ? 0.f : v - __uint_as_float(u & 0xFFFF0000u);
        } else {
            const bool special = (u & 0x7F800000u) == 0x7F800000u;
            part[i] = (special ? u : u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
        }
    }
}

__device__ __forceinline__ void add_base(float (&v)[16], const bf16_t *b) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const u32x4 u = *reinterpret_cast<const u32x4 *>(b + 8 * h);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[8 * h + 2 * i] += __uint_as_float(u[i] << 16);
            v[8 * h + 2 * i + 1] += __uint_as_float(u[i] & 0xFFFF0000u);
        }
    }
}
__device__ __forceinline__ void add_base(float (&v)[16], const float *b) {
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        const floatx4 u = *reinterpret_cast<const floatx4 *>(b + 4 * h);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[4 * h + i] += u[i];
    }
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __bf16 x = (__bf16)a, y = (__bf16)b;
    return (uint32_t)__builtin_bit_cast(uint16_t, x) |
           ((uint32_t)__builtin_bit_cast(uint16_t, y) << 16);
}
__device__ __forceinline__ void store16(bf16_t *y, const float (&v)[16]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        u32x4 u;
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = pack2(v[8 * h + 2 * i], v[8 * h + 2 * i + 1]);
        *reinterpret_cast<u32x4 *>(y + 8 * h) = u;
    }
}
__device__ __forceinline__ void store16(float *y, const float (&v)[16]) {
#pragma unroll
    for (int h = 0; h < 4; ++h)
        *reinterpret_cast<floatx4 *>(y + 4 * h) =
            floatx4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
}

// Rows of no adapter: base's row (zeros without one), 64 rows a workgroup.
template <class Y>
__device__ void copy_rows(const AdapterRows &o, const int32_t *place, int block, int N, int c0,
                          int c1, const Y *base, Y *y) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int i = wave; i < 64; i += kWaves) {
        const int64_t row = (int64_t)block * 64 + i;
        if (row >= o.rows || place[row] >= 0) continue;
        constexpr int V = 16 / sizeof(Y);
        for (int c = c0 + lane * V; c < c1; c += 64 * V) {
            u32x4 v = {};
            if (base) v = *reinterpret_cast<const u32x4 *>(base + row * N + c);
            *reinterpret_cast<u32x4 *>(y + row * N + c) = v;
        }
    }
}

// The contraction runs over S * rank positions: the S parts of u one behind the
// other, against B's columns as many times.  Chunk c (8 positions) is part
// c / (rank / 8) of u; chunks are padded to whole instructions of four.
// M is the output column (m -> 16 (m / 4) + 4 j + m % 4 for the j-th of four
// instructions, so that a lane ends with 16 consecutive columns of a row), N
// the rows.
template <int RB, int S, class Y>
__global__ __launch_bounds__(64 * kWaves) void expand_kernel(
    AdapterRows o, int rank, int N, const float *__restrict__ p, int splits,
    const bf16_t *__restrict__ w, const float *__restrict__ scale,
    const int32_t *__restrict__ place, const Y *base, Y *y, int tiles, int blocks_per_wg) {
    extern __shared__ char lds[];
    const int c0 = blockIdx.y * blocks_per_wg * 64, c1 = min(N, c0 + blocks_per_wg * 64);
    if ((int)blockIdx.x >= tiles) {
        copy_rows(o, place, (int)blockIdx.x - tiles, N, c0, c1, base, y);
        return;
    }
    const Tile t = find_tile<16 * RB>(o, blockIdx.x);
    if (t.e < 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
    const int rc = rank / 8, chunks = (rc * S + 3) / 4 * 4;
    // u, scaled and cut, in LDS: [row block][chunk][row][8]
    uint16_t *u = reinterpret_cast<uint16_t *>(lds);
    const float f = scale ? scale[t.e] : 1.f;
    for (int i = threadIdx.x; i < 16 * RB * rank; i += 64 * kWaves) {
        const int row = i / rank, r = i % rank;
        float v = 0.f;
        if (row < t.rows)
            for (int q = 0; q < splits; ++q)
                v += p[((int64_t)q * o.rows + t.first + row) * rank + r];
        uint32_t part[S];
        cut<S>(v * f, part);
#pragma unroll
        for (int q = 0; q < S; ++q)
            u[((((row >> 4) * chunks) + q * rc + r / 8) * 16 + (row & 15)) * 8 + r % 8] =
                (uint16_t)part[q];
    }
    for (int i = threadIdx.x; i < RB * (chunks - rc * S) * 128; i += 64 * kWaves) {
        const int b = i / ((chunks - rc * S) * 128), j = i % ((chunks - rc * S) * 128);
        u[(b * chunks + rc * S) * 128 + j] = 0;
    }
    __syncthreads();
    int64_t row[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b)
        row[b] = 16 * b + m < t.rows ? row_at(o, t.first + 16 * b + m) : -1;
    const bf16_t *we = w + (int64_t)t.e * N * rank;
    for (int c = c0 + wave * 64; c < c1; c += kWaves * 64) {
        floatx4 acc[RB][4] = {};
        int ch = g % rc;
        for (int s = 0; s < chunks; s += 4) {
            bf16x8 wv[4], uv[RB];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                wv[j] = load8(we + (int64_t)(c + 16 * (m >> 2) + 4 * j + (m & 3)) * rank + 8 * ch);
                if (s + g >= rc * S) wv[j] = bf16x8{};
            }
#pragma unroll
            for (int b = 0; b < RB; ++b)
                uv[b] = *reinterpret_cast<const bf16x8 *>(u + ((b * chunks + s + g) * 16 + m) * 8);
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[b][j] = mfma(wv[j], uv[b], acc[b][j]);
            ch = (ch + 4) % rc;
        }
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            if (row[b] < 0) continue;
            float v[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = acc[b][j / 4][j % 4];
            const int64_t at = row[b] * N + c + 16 * g;
            if (base) add_base(v, base + at);
            store16(y + at, v);
        }
    }
}

// ---- gradients of A and B ------------------------------------------------

// Rows of a tile of the outer products.
constexpr int kOuterRows = 512;

// 8 x 8 values of 16 bits, rows to columns.
__device__ __forceinline__ void transpose8(const u32x4 (&in)[8], bf16x8 (&out)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {  // columns 2 j and 2 j + 1
        u32x4 lo, hi;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            lo[i] = __builtin_amdgcn_perm(in[2 * i + 1][j], in[2 * i][j], 0x05040100u);
            hi[i] = __builtin_amdgcn_perm(in[2 * i + 1][j], in[2 * i][j], 0x07060302u);
        }
        out[2 * j] = __builtin_bit_cast(bf16x8, lo);
        out[2 * j + 1] = __builtin_bit_cast(bf16x8, hi);
    }
}

// The contraction runs over rows, 32 an instruction.  A lane loads 8 rows x 8
// columns of q and turns them in registers: the operands of eight instructions,
// the j-th of which has column 8 (lane % 16) + j.  M is the rank.
template <int NR>
__global__ __launch_bounds__(64 * kWaves) void outer_kernel(
    AdapterRows o, int rank, int C, const float *__restrict__ p, int splits,
    const bf16_t *__restrict__ q, const float *__restrict__ scale, float *__restrict__ parts,
    int slots, int transposed, int accumulate, float *__restrict__ out) {
    const Tile t = find_tile<kOuterRows>(o, blockIdx.x);
    if (t.e < 0 || (t.tiles > 1 && t.several + t.index >= slots)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
    const int r0 = blockIdx.z * 16 * NR, col = (blockIdx.y * kWaves + wave) * 128 + 8 * m;
    if ((blockIdx.y * kWaves + wave) * 128 >= C) return;
    const int qc = min(col, C - 8);
    const float f = scale ? scale[t.e] : 1.f;
    floatx4 acc[NR][8] = {};
    for (int k0 = 0; k0 < t.rows; k0 += 32) {
        u32x4 raw[8];
        bf16x8 qv[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = row_at(o, t.first + min(k0 + 8 * g + i, t.rows - 1));
            raw[i] = *reinterpret_cast<const u32x4 *>(q + (int64_t)max(row, 0) * C + qc);
        }
        transpose8(raw, qv);
#pragma unroll
        for (int b = 0; b < NR; ++b) {
            const int r = r0 + 16 * b + m;
            uint32_t part[3][8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float v = 0.f;
                if (k0 + 8 * g + i < t.rows && r < rank)
                    for (int s = 0; s < splits; ++s)
                        v += p[((int64_t)s * o.rows + t.first + k0 + 8 * g + i) * rank + r];
                uint32_t c[3];
                cut<3>(v * f, c);
                part[0][i] = c[0];
                part[1][i] = c[1];
                part[2][i] = c[2];
            }
#pragma unroll
            for (int s = 0; s < 3; ++s) {
                u32x4 pk;
#pragma unroll
                for (int i = 0; i < 4; ++i) pk[i] = part[s][2 * i] | (part[s][2 * i + 1] << 16);
                const bf16x8 pv = __builtin_bit_cast(bf16x8, pk);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[b][j] = mfma(pv, qv[j], acc[b][j]);
            }
        }
    }
    if (col >= C) return;
    const bool whole = t.tiles == 1;
    float *to = whole ? out + (int64_t)t.e * rank * C
                      : parts + (int64_t)(t.several + t.index) * rank * C;
    const bool add = whole && accumulate;
#pragma unroll
    for (int b = 0; b < NR; ++b) {
        const int r = r0 + 16 * b + 4 * g;
        if (r >= rank) continue;
        if (transposed) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                floatx4 *d = reinterpret_cast<floatx4 *>(to + (int64_t)(col + j) * rank + r);
                *d = add ? *d + acc[b][j] : acc[b][j];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    floatx4 *d =
                        reinterpret_cast<floatx4 *>(to + (int64_t)(r + i) * C + col + 4 * h);
                    const floatx4 v = {acc[b][4 * h][i], acc[b][4 * h + 1][i],
                                       acc[b][4 * h + 2][i], acc[b][4 * h + 3][i]};
                    *d = add ? *d + v : v;
                }
        }
    }
}

// Adapters of several tiles: their parts, added in order; adapters of no rows:
// zeros (nothing where out accumulates).
__global__ __launch_bounds__(256) void join_kernel(AdapterRows o, int64_t size,
                                                   const float *__restrict__ parts, int slots,
                                                   int accumulate, float *__restrict__ out) {
    const int e = blockIdx.y, lane = threadIdx.x & 63;
    auto tiles_of = [&](int i) {
        if (o.rows == 0) return 0;  // offsets need not be there
        const int a = (int)min((int64_t)max(o.offsets[i], 0), o.rows);
        const int z = (int)min((int64_t)max(o.offsets[i + 1], 0), o.rows);
        return (max(z - a, 0) + kOuterRows - 1) / kOuterRows;
    };
    // tiles of several-tile adapters before e
    int before = 0;
    for (int i = lane; i < e; i += 64) before += tiles_of(i) > 1 ? tiles_of(i) : 0;
    before = __shfl(scan64(before, lane), 63);
    int n = tiles_of(e);
    if (n == 1 || (n == 0 && accumulate)) return;
    n = min(n, slots - before);
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < size;
         i += (int64_t)gridDim.x * 1024) {
        floatx4 v = {};
        for (int j = 0; j < n; ++j)
            v += *reinterpret_cast<const floatx4 *>(parts + (int64_t)(before + j) * size + i);
        floatx4 *d = reinterpret_cast<floatx4 *>(out + (int64_t)e * size + i);
        *d = accumulate ? *d + v : v;
    }
}

// 64 x 64 tiles through LDS.  m or n may be any multiple of 8.
__global__ __launch_bounds__(256) void transpose_kernel(AdapterRows o, int m, int n,
                                                        const bf16_t *__restrict__ w,
                                                        bf16_t *__restrict__ wt) {
    const int e = blockIdx.z;
    if (o.offsets[e + 1] <= o.offsets[e]) return;
    __shared__ uint16_t tile[64][66];
    const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;
    const bf16_t *src = w + (int64_t)e * m * n;
    bf16_t *dst = wt + (int64_t)e * m * n;
    for (int v = threadIdx.x; v < 64 * 8; v += 256) {
        const int i = v / 8, j = v % 8 * 8;
        if (i0 + i < m && j0 + j < n) {
            const u32x4 u = *reinterpret_cast<const u32x4 *>(src + (int64_t)(i0 + i) * n + j0 + j);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                tile[i][j + 2 * q] = (uint16_t)u[q];
                tile[i][j + 2 * q + 1] = (uint16_t)(u[q] >> 16);
            }
        }
    }
    __syncthreads();
    for (int v = threadIdx.x; v < 64 * 8; v += 256) {
        const int j = v / 8, i = v % 8 * 8;
        if (i0 + i < m && j0 + j < n) {
            u32x4 u;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                u[q] = tile[i + 2 * q][j] | ((uint32_t)tile[i + 2 * q + 1][j] << 16);
            *reinterpret_cast<u32x4 *>(dst + (int64_t)(j0 + j) * m + i0 + i) = u;
        }
    }
}

// Tiles of TM rows that `count` adapters can have.
int64_t tile_cap(const AdapterRows &o, int tm) {
    return o.rows / tm + (o.count < o.rows ? o.count : o.rows);
}

// Tall tiles where the adapters' mean rows fill most of one.
bool tall(int64_t rows, int count) { return rows >= (int64_t)48 * count; }

template <int RB>
hipError_t shrink(const AdapterRows &o, int rank, int K, const bf16_t *x, const bf16_t *w, float *p,
                  int splits, hipStream_t s) {
    const unsigned tiles = (unsigned)tile_cap(o, 16 * RB);
    const int nr = rank <= 16 ? 1 : rank <= 32 ? 2 : 4;
    const dim3 grid(tiles, splits, (rank + 16 * nr - 1) / (16 * nr));
    if (nr == 1)
        shrink_kernel<RB, 1><<<grid, 64 * kWaves, 0, s>>>(o, rank, K, x, w, p, splits);
    else if (nr == 2)
        shrink_kernel<RB, 2><<<grid, 64 * kWaves, 0, s>>>(o, rank, K, x, w, p, splits);
    else
        shrink_kernel<RB, 4><<<grid, 64 * kWaves, 0, s>>>(o, rank, K, x, w, p, splits);
    return hipGetLastError();
}

template <int RB, int S, class Y>
hipError_t expand(const AdapterRows &o, int rank, int N, const float *p, int splits,
                  const bf16_t *w, const float *scale, const int32_t *place, const void *base,
                  void *y, hipStream_t s) {
    const int tiles = (int)tile_cap(o, 16 * RB), blocks = N / 64;
    const int64_t copies = base == y ? 0 : (o.rows + 63) / 64;
    // column ranges: enough workgroups for the chip, four blocks (one a wave) at least
    int per = blocks;
    while (per > kWaves && (int64_t)tiles * ((blocks + per - 1) / per) < 1024) per = (per + 1) / 2;
    const size_t lds = (size_t)RB * ((rank / 8 * S + 3) / 4 * 4) * 256;
    if (lds > 65536)
        if (hipError_t e = hipFuncSetAttribute((const void *)expand_kernel<RB, S, Y>,
                                               hipFuncAttributeMaxDynamicSharedMemorySize,
                                               (int)lds))
            return e;
    expand_kernel<RB, S, Y>
        <<<dim3((unsigned)(tiles + copies), (blocks + per - 1) / per), 64 * kWaves, lds, s>>>(
            o, rank, N, p, splits, w, scale, place, (const Y *)base, (Y *)y, tiles, per);
    return hipGetLastError();
}

}  // namespace

int adapter_splits(int64_t rows, int count, int K) {
    const int tm = tall(rows, count) ? 64 : 16;
    const int64_t tiles = rows / tm + (count < rows ? count : rows);
    int64_t splits = (512 + tiles - 1) / tiles;
    const int64_t most = (K / 64 + kWaves - 1) / kWaves;
    if (splits > most) splits = most;
    return (int)(splits < 1 ? 1 : splits > 16 ? 16 : splits);
}

int64_t adapter_outer_slots(int64_t rows) { return 2 * (rows / kOuterRows) + 2; }

hipError_t launch_adapter_shrink(const AdapterRows &o, int rank, int K, const bf16_t *x,
                                 const bf16_t *w, float *p, int splits, hipStream_t s) {
    return tall(o.rows, o.count) ? shrink<4>(o, rank, K, x, w, p, splits, s)
                                 : shrink<1>(o, rank, K, x, w, p, splits, s);
}

hipError_t launch_adapter_expand(const AdapterRows &o, int rank, int N, const float *p, int splits,
                                 const bf16_t *w, const float *scale, const int32_t *place,
                                 const void *base, void *y, int y_type, hipStream_t s) {
    const bool big = tall(o.rows, o.count);
    if (y_type == MOE_FP32)
        return big ? expand<4, 3, float>(o, rank, N, p, splits, w, scale, place, base, y, s)
                   : expand<1, 3, float>(o, rank, N, p, splits, w, scale, place, base, y, s);
    return big ? expand<4, 2, bf16_t>(o, rank, N, p, splits, w, scale, place, base, y, s)
               : expand<1, 2, bf16_t>(o, rank, N, p, splits, w, scale, place, base, y, s);
}

hipError_t launch_adapter_outer(const AdapterRows &o, int rank, int C, const float *p, int splits,
                                const bf16_t *q, const float *scale, float *parts, bool transposed,
                                bool accumulate, float *out, hipStream_t s) {
    const unsigned tiles = (unsigned)tile_cap(o, kOuterRows);
    const int nr = rank <= 16 ? 1 : rank <= 32 ? 2 : 4, slots = (int)adapter_outer_slots(o.rows);
    const dim3 grid(tiles, (C + 128 * kWaves - 1) / (128 * kWaves),
                    (rank + 16 * nr - 1) / (16 * nr));
    if (tiles == 0) {
    } else if (nr == 1) {
        outer_kernel<1><<<grid, 64 * kWaves, 0, s>>>(o, rank, C, p, splits, q, scale, parts, slots,
                                                     transposed, accumulate, out);
    } else if (nr == 2) {
        outer_kernel<2><<<grid, 64 * kWaves, 0, s>>>(o, rank, C, p, splits, q, scale, parts, slots,
                                                     transposed, accumulate, out);
    } else {
        outer_kernel<4><<<grid, 64 * kWaves, 0, s>>>(o, rank, C, p, splits, q, scale, parts, slots,
                                                     transposed, accumulate, out);
    }
    if (hipError_t e = hipGetLastError()) return e;
    const int64_t size = (int64_t)rank * C;
    const unsigned bx = (unsigned)((size + 1023) / 1024);
    join_kernel<<<dim3(bx < 64 ? bx : 64, o.count), 256, 0, s>>>(o, size, parts, slots, accumulate,
                                                               out);
    return hipGetLastError();
}

hipError_t launch_adapter_transpose(const AdapterRows &o, int m, int n, const bf16_t *w,
                                    bf16_t *wt, hipStream_t s) {
    transpose_kernel<<<dim3((n + 63) / 64, (m + 63) / 64, o.count), 256, 0, s>>>(o, m, n, w, wt);
    return hipGetLastError();
}

}  // namespace moe
