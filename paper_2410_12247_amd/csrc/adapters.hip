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

#include <algorithm>

#include "dispatch.h"

namespace moe {
namespace {

constexpr int kWaves = 4;        // of the kernels but shrink
constexpr int kShrinkWaves = 4;  // which share K

__device__ __forceinline__ floatx4 mfma(bf16x8 a, bf16x8 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ bf16x8 load8(const bf16_t *p) {
    return *reinterpret_cast<const bf16x8 *>(p);
}
// At a uniform base and a lane's byte offset.
__device__ __forceinline__ bf16x8 load8(const bf16_t *base, uint32_t off) {
    return *reinterpret_cast<const bf16x8 *>(reinterpret_cast<const char *>(base) + off);
}

// One tile: adapter e's places [first, first + rows), the tile's number among
// the adapter's `tiles`, and the tiles of several-tile adapters before it.
struct Tile {
    int e, rows, index, tiles, several;
    int64_t first;
};

// An offset, cut to [0, rows].
__device__ __forceinline__ int offset_at(const AdapterRows &o, int e) {
    return (int)min((int64_t)max(o.offsets[e], 0), o.rows);
}

// Tile t of all adapters' tiles of 2^sh rows; e < 0 behind the last.  Every lane
// takes four adapters' counts; a scan over the lanes finds the tile's.  The
// result is uniform.
__device__ __forceinline__ Tile find_tile(const AdapterRows &o, int sh, int t) {
    const int lane = threadIdx.x & 63, TM = 1 << sh;
    int at[5], n[4], sum = 0, sev = 0;
#pragma unroll
    for (int i = 0; i < 5; ++i) at[i] = offset_at(o, min(lane * 4 + i, o.count));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        n[i] = (max(at[i + 1] - at[i], 0) + TM - 1) >> sh;
        sum += n[i];
        sev += n[i] > 1 ? n[i] : 0;
    }
    const int incl = wave_inclusive_scan(sum), sincl = wave_inclusive_scan(sev);
    Tile r{-1, 0, 0, 0, 0, 0};
    const uint64_t has = __ballot(incl > t);
    if (!has) return r;
    const int l = __builtin_ctzll(has);
    int left = t - (incl - sum), before = sincl - sev, q = 0, first = at[0], last = at[1];
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (q == i && left >= n[i]) {
            left -= n[i];
            before += n[i] > 1 ? n[i] : 0;
            q = i + 1;
            first = at[i + 1];
            last = at[i + 2];
        }
    r.e = 4 * l + __builtin_amdgcn_readlane(q, l);
    r.index = __builtin_amdgcn_readlane(left, l);
    r.several = __builtin_amdgcn_readlane(before, l);
    const int f = __builtin_amdgcn_readlane(first, l), z = __builtin_amdgcn_readlane(last, l);
    r.tiles = (z - f + TM - 1) >> sh;
    r.first = f + ((int64_t)r.index << sh);
    r.rows = min(TM, (int)(z - r.first));
    return r;
}

// The row of a place, -1 if it is none.
__device__ __forceinline__ int row_at(const AdapterRows &o, int64_t place) {
    const int row = o.order[place];
    return (uint32_t)row < (uint64_t)o.rows ? row : -1;
}

// ---- x A^T ---------------------------------------------------------------

// Sums of `rows` times w [count][rank][K].  The matrix instruction's M is the
// rows, its N the rank; an operand load is 64 bytes of each of 16 rows.  The waves
// (and `splits` workgroups) share K; a wave keeps DEP steps of 64 k in flight.
struct Shrink {
    const bf16_t *x, *w;
    AdapterSums out;
    int K, tiles;
};

template <int RB, int NR>
__device__ __forceinline__ void shrink(const AdapterRows &o, int rank, const Shrink &k, int tile,
                                       int split, int r0, floatx4 (*lds)[RB * NR][64]) {
    constexpr int DEP = RB + NR <= 3 ? 4 : RB + NR <= 5 ? 3 : 2, TM = 16 * RB;
    const Tile t = find_tile(o, RB == 4 ? 6 : 4, tile);
    if (t.e < 0) return;
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // a wave takes every parts-th 128 bytes of a row, so that a workgroup's loads are
    // next to each other
    const int parts = k.out.splits * kShrinkWaves, part = split * kShrinkWaves + wave;
    const int n = (k.K / 64 - part + parts - 1) / parts;
    uint64_t xo[RB];
    uint32_t wo[NR];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int row = row_at(o, t.first + min(16 * b + m, t.rows - 1));
        xo[b] = ((uint64_t)max(row, 0) * k.K + 8 * g) * 2;
    }
#pragma unroll
    for (int c = 0; c < NR; ++c)  // behind the last rank value: the last again, not stored
        wo[c] = ((uint32_t)min(r0 + 16 * c + m, rank - 1) * k.K + 8 * g) * 2;
    const char *xs = (const char *)(k.x + part * 64);
    const char *ws = (const char *)(k.w + (int64_t)t.e * rank * k.K + part * 64);
    floatx4 acc[RB][NR] = {};
    bf16x8 xv[DEP][RB][2], wv[DEP][NR][2];
    // (both halves of a cache line one after the other: it may not stay)
    auto load = [&](int i, int s) {
        const int at = s * parts * 128;
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                xv[i][b][h] = *reinterpret_cast<const bf16x8 *>(xs + at + xo[b] + 64 * h);
#pragma unroll
        for (int c = 0; c < NR; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                wv[i][c][h] = *reinterpret_cast<const bf16x8 *>(ws + at + wo[c] + 64 * h);
    };
    auto use = [&](int i) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
                for (int c = 0; c < NR; ++c)
                    acc[b][c] = mfma(xv[i][b][h], wv[i][c][h], acc[b][c]);
    };
    if (n > 0) {
#pragma unroll
        for (int i = 0; i < DEP; ++i) load(i, min(i, n - 1));
        int s = 0;  // (no branch around a load here: a wait would be for all of them)
        for (; s + DEP <= n; s += DEP) {
#pragma unroll
            for (int i = 0; i < DEP; ++i) {
                use(i);
                load(i, min(s + i + DEP, n - 1));
            }
        }
#pragma unroll
        for (int i = 0; i < DEP; ++i)
            if (s + i < n) use(i);
    }
    // the waves' sums meet in LDS, half of the waves' at a time
#pragma unroll
    for (int half = kShrinkWaves / 2; half >= 1; half /= 2) {
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
                for (int c = 0; c < NR; ++c) lds[wave - half][b * NR + c][lane] = acc[b][c];
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
                for (int c = 0; c < NR; ++c) acc[b][c] += lds[wave][b * NR + c][lane];
        }
        __syncthreads();
    }
    if (wave > 0) return;
    float *p = k.out.p + ((int64_t)tile * k.out.splits + split) * rank * TM;
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int c = 0; c < NR; ++c) {
            const int r = r0 + 16 * c + m;
            if (r < rank) *reinterpret_cast<floatx4 *>(p + r * TM + 16 * b + 4 * g) = acc[b][c];
        }
}

// wt[e] = w[e]^T for the adapters that have rows, w [count][m][n]: 64 x 64 tiles
// through LDS, m and n any multiples of 8.
struct Transpose {
    const bf16_t *w;
    bf16_t *wt;
    int m, n, bx, blocks;  // tiles along n, and of all adapters
};

__device__ __forceinline__ void transpose(const AdapterRows &o, const Transpose &k, int block,
                                          uint16_t (*tile)[66]) {
    const int by = (k.m + 63) / 64, e = block / (k.bx * by), at = block % (k.bx * by);
    if (offset_at(o, e + 1) <= offset_at(o, e)) return;
    const int i0 = at / k.bx * 64, j0 = at % k.bx * 64;
    const bf16_t *src = k.w + (int64_t)e * k.m * k.n;
    bf16_t *dst = k.wt + (int64_t)e * k.m * k.n;
    for (int v = threadIdx.x; v < 64 * 8; v += blockDim.x) {
        const int i = v / 8, j = v % 8 * 8;
        if (i0 + i < k.m && j0 + j < k.n) {
            const u32x4 u =
                *reinterpret_cast<const u32x4 *>(src + (int64_t)(i0 + i) * k.n + j0 + j);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                tile[i][j + 2 * q] = (uint16_t)u[q];
                tile[i][j + 2 * q + 1] = (uint16_t)(u[q] >> 16);
            }
        }
    }
    __syncthreads();
    for (int v = threadIdx.x; v < 64 * 8; v += blockDim.x) {
        const int j = v / 8, i = v % 8 * 8;
        if (i0 + i < k.m && j0 + j < k.n) {
            u32x4 u;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                u[q] = tile[i + 2 * q][j] | ((uint32_t)tile[i + 2 * q + 1][j] << 16);
            *reinterpret_cast<u32x4 *>(dst + (int64_t)(j0 + j) * k.m + i0 + i) = u;
        }
    }
}

// Blocks of the shrink, then of the transposes (of the gradient's first launch).
template <int RB, int NR>
__global__ __launch_bounds__(64 * kShrinkWaves) void shrink_kernel(AdapterRows o, int rank,
                                                                   Shrink k, Transpose ta,
                                                                   Transpose tb) {
    __shared__ union {
        floatx4 sums[kShrinkWaves / 2][RB * NR][64];
        uint16_t tile[64][66];
    } lds;
    int b = blockIdx.x;
    const int groups = (rank + 16 * NR - 1) / (16 * NR), mine = k.tiles * k.out.splits * groups;
    if (b < mine) {
        shrink<RB, NR>(o, rank, k, b % k.tiles, b / k.tiles % k.out.splits,
                       b / (k.tiles * k.out.splits) * 16 * NR, lds.sums);
        return;
    }
    b -= mine;
    if (b < ta.blocks)
        transpose(o, ta, b, lds.tile);
    else
        transpose(o, tb, b - ta.blocks, lds.tile);
}

// ---- + scale u B^T -------------------------------------------------------

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __bf16 x = (__bf16)a, y = (__bf16)b;
    return (uint32_t)__builtin_bit_cast(uint16_t, x) |
           ((uint32_t)__builtin_bit_cast(uint16_t, y) << 16);
}

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
// Eight values' parts, two to a word.
template <int S>
__device__ __forceinline__ void cut8(const float (&v)[8], bf16x8 (&part)[S]) {
    u32x4 w[S] = {};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t c[S];
        cut<S>(v[j], c);
#pragma unroll
        for (int q = 0; q < S; ++q) w[q][j / 2] |= c[q] << (16 * (j & 1));
    }
#pragma unroll
    for (int q = 0; q < S; ++q) part[q] = __builtin_bit_cast(bf16x8, w[q]);
}

// A lane's 16 values of a row's 64 columns from c on: 16-byte pieces, the lane
// groups' next to each other, so that a row's piece is 64 bytes.  column(): the
// output column of the j-th instruction's m (a group has m = 4 g .. 4 g + 3).
// S: bf16 parts of u, two for bf16 outputs (2^-15 of a value at worst, where the
// output's rounding is 2^-8), three for fp32.
template <class Y>
struct Piece;
template <>
struct Piece<bf16_t> {
    static constexpr int N = 2, W = 8, S = 2;
    static __device__ __forceinline__ int column(int j, int m) {
        return 32 * (j >> 1) + 8 * (m >> 2) + 4 * (j & 1) + (m & 3);
    }
    static __device__ __forceinline__ u32x4 add(u32x4 base, const floatx4 (&v)[4], int h) {
        u32x4 u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const floatx4 a = v[2 * h + (i >> 1)];
            u[i] = pack2(__uint_as_float(base[i] << 16) + a[2 * (i & 1)],
                         __uint_as_float(base[i] & 0xFFFF0000u) + a[2 * (i & 1) + 1]);
        }
        return u;
    }
};
template <>
struct Piece<float> {
    static constexpr int N = 4, W = 4, S = 3;
    static __device__ __forceinline__ int column(int j, int m) { return 16 * j + m; }
    static __device__ __forceinline__ u32x4 add(u32x4 base, const floatx4 (&v)[4], int h) {
        return __builtin_bit_cast(u32x4, __builtin_bit_cast(floatx4, base) + v[h]);
    }
};

// y = base + scale w u over N columns, w [count][N][rank].  A workgroup has a tile
// of rows and `span` blocks of 64 columns.
template <class Y>
struct Expand {
    AdapterSums u;
    const bf16_t *w;
    const float *scale;
    const Y *base;
    Y *y;
    int N, tiles, copies, span, ranges;  // ranges: of span blocks
};

// Rows of no adapter: base's row (zeros without one), 64 rows a workgroup.
template <class Y>
__device__ __forceinline__ void copy_rows(const AdapterRows &o, const Expand<Y> &k, int block,
                                          int c0, int c1) {
    constexpr int V = 16 / sizeof(Y);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t mine = (int64_t)block * 64 + lane;
    uint64_t none = __ballot(mine < o.rows && o.place[min(mine, o.rows - 1)] < 0);
    for (int i = 0; none; ++i, none &= none - 1) {
        if (i % kWaves != wave) continue;
        const int64_t at = ((int64_t)block * 64 + __builtin_ctzll(none)) * k.N;
        for (int c = c0 + lane * V; c < c1; c += 64 * V) {
            u32x4 v = {};
            if (k.base) v = *reinterpret_cast<const u32x4 *>(k.base + at + c);
            *reinterpret_cast<u32x4 *>(k.y + at + c) = v;
        }
    }
}

// The contraction runs over S * rank positions: the S parts of u one behind the
// other, against B's columns as many times.  Chunk c (8 positions) is part
// c / (rank / 8) of u; chunks are padded to whole instructions of four.  Where
// rank is a multiple of 32 an operand of B serves all parts.  M is the output
// column, N the rows.  What does not depend on u (base's rows, the first operands
// of B) is on its way before u is cut.
template <int RB, class Y>
__device__ __forceinline__ void expand(const AdapterRows &o, int rank, const Expand<Y> &k,
                                       int block, char *lds) {
    using P = Piece<Y>;
    constexpr int S = P::S, TM = 16 * RB;
    constexpr int WB = RB < 2 ? RB : 2, WR = RB / WB, WC = kWaves / WR;  // a wave's row blocks
    const int tile = block / k.ranges;
    const int c0 = block % k.ranges * k.span * 64, c1 = min(k.N, c0 + k.span * 64);
    if (tile >= k.tiles) {
        copy_rows(o, k, tile - k.tiles, c0, c1);
        return;
    }
    const Tile t = find_tile(o, RB == 4 ? 6 : 4, tile);
    if (t.e < 0) return;
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), b0 = wave % WR * WB;
    const int rc = rank / 8, chunks = (rc * S + 3) / 4 * 4;
    const float *pt = k.u.p + (int64_t)tile * k.u.splits * rank * TM;
    const bf16_t *we = k.w + (int64_t)t.e * k.N * rank;
    uint32_t wo[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) wo[j] = (uint32_t)P::column(j, m) * rank * 2;
    const int step = 4 % rc, ch0 = g % rc;
    int64_t at[WB];
#pragma unroll
    for (int b = 0; b < WB; ++b) {
        const int i = 16 * (b0 + b) + m, row = i < t.rows ? row_at(o, t.first + i) : -1;
        at[b] = row < 0 ? -1 : (int64_t)row * k.N + P::W * g;
    }
    u32x4 old[WB][P::N];
    bf16x8 wv[4];
    auto load_block = [&](int c) {
        if (k.base) {
#pragma unroll
            for (int b = 0; b < WB; ++b)
#pragma unroll
                for (int h = 0; h < P::N; ++h)  // (a place of no row: row 0's, not stored)
                    old[b][h] = *reinterpret_cast<const u32x4 *>(
                        k.base + max(at[b], (int64_t)(P::W * g)) + c + 4 * P::W * h);
        } else {
#pragma unroll
            for (int b = 0; b < WB; ++b)
#pragma unroll
                for (int h = 0; h < P::N; ++h) old[b][h] = u32x4{};
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) wv[j] = load8(we + (int64_t)c * rank, wo[j] + 16 * ch0);
    };
    int c = c0 + wave / WR * 64;
    if (c < c1) load_block(c);
    // u, scaled and cut, in LDS: [row block][chunk][row][8]
    bf16x8 *u = reinterpret_cast<bf16x8 *>(lds);
    const float f = k.scale ? k.scale[t.e] : 1.f;
    for (int i = threadIdx.x; i < TM * (chunks - rc * (S - 1)); i += 64 * kWaves) {
        const int row = i % TM, kc = i / TM;
        bf16x8 part[S] = {};
        if (row < t.rows && kc < rc) {
            float v[8] = {};
            for (int q = 0; q < k.u.splits; ++q)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += pt[((int64_t)q * rank + 8 * kc + j) * TM + row];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= f;
            cut8<S>(v, part);
        }
        // chunks behind the last part's are the padding
#pragma unroll
        for (int q = 0; q < S; ++q)
            if (kc < rc || q + 1 == S)
                u[((row >> 4) * chunks + q * rc + kc) * 16 + (row & 15)] = part[q];
    }
    __syncthreads();
    while (c < c1) {
        const bf16_t *wc = we + (int64_t)c * rank;
        floatx4 acc[WB][4] = {};
        if (rank % 32 == 0) {
            for (int s = 0; s < rc; s += 4) {
                bf16x8 cur[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) cur[j] = wv[j];
                if (s + 4 < rc) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) wv[j] = load8(wc, wo[j] + 16 * (s + 4 + g));
                }
#pragma unroll
                for (int q = 0; q < S; ++q)
#pragma unroll
                    for (int b = 0; b < WB; ++b) {
                        const bf16x8 uv = u[((b0 + b) * chunks + q * rc + s + g) * 16 + m];
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[b][j] = mfma(cur[j], uv, acc[b][j]);
                    }
            }
        } else {
            int ch = ch0;
            for (int s = 0; s < chunks; s += 4) {
                bf16x8 cur[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) cur[j] = s + g < rc * S ? wv[j] : bf16x8{};
                ch += step;
                if (ch >= rc) ch -= rc;
                if (s + 4 < chunks) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) wv[j] = load8(wc, wo[j] + 16 * ch);
                }
#pragma unroll
                for (int b = 0; b < WB; ++b) {
                    const bf16x8 uv = u[((b0 + b) * chunks + s + g) * 16 + m];
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[b][j] = mfma(cur[j], uv, acc[b][j]);
                }
            }
        }
#pragma unroll
        for (int b = 0; b < WB; ++b)
            if (at[b] >= 0) {
#pragma unroll
                for (int h = 0; h < P::N; ++h)
                    *reinterpret_cast<u32x4 *>(k.y + at[b] + c + 4 * P::W * h) =
                        P::add(old[b][h], acc[b], h);
            }
        c += WC * 64;
        if (c < c1) load_block(c);
    }
}

template <int RB, class Y>
__global__ __launch_bounds__(64 * kWaves) void expand_kernel(AdapterRows o, int rank,
                                                             Expand<Y> k) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    expand<RB, Y>(o, rank, k, blockIdx.x, lds);
}

// ---- gradients of A and B ------------------------------------------------

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

// out[e] (+)= scale[e] * sum over the adapter's rows of p^T q: [count][rank][C], or
// transposed [count][C][rank].  A tile is 2^sh rows; adapters of several tiles
// leave them in parts, for the join.
struct Outer {
    AdapterSums p;
    const bf16_t *q;
    float *parts, *out;
    int C, transposed, cb, blocks;  // cb: blocks of 128 columns
};

// Tiles of 2^sh rows before adapter e.
__device__ __forceinline__ int tiles_before(const AdapterRows &o, int sh, int e) {
    int n = 0;
    for (int i = threadIdx.x & 63; i < e; i += 64)
        n += (max(offset_at(o, i + 1) - offset_at(o, i), 0) + (1 << sh) - 1) >> sh;
    return __builtin_amdgcn_readlane(wave_inclusive_scan(n), 63);
}

// The contraction runs over rows, 32 an instruction.  A lane loads 8 rows x 8
// columns of q and turns them in registers: the operands of eight instructions,
// the j-th of which has column 8 (lane % 16) + j.  M is the rank.  The waves take
// steps of 32 rows in turn and join in LDS.  p in three parts: the sums are as
// exact as fp32's.
template <int RB, int NR>
__device__ __forceinline__ void outer(const AdapterRows &o, int rank, const float *scale, int sh,
                                      int slots, bool accumulate, const Outer &k, int block,
                                      char *lds) {
    constexpr int TSH = RB == 4 ? 6 : 4, TM = 16 * RB;
    floatx4(*sums)[NR * 8][64] = reinterpret_cast<floatx4(*)[NR * 8][64]>(lds);
    int *rows = reinterpret_cast<int *>(lds);  // before the sums
    const Tile t = find_tile(o, sh, block / k.cb);
    if (t.e < 0 || (t.tiles > 1 && t.several + t.index >= slots)) return;
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = block % k.cb * 128 + 8 * m, qc = min(col, k.C - 8);
    const int groups = (rank + 16 * NR - 1) / (16 * NR);
    for (int i = threadIdx.x; i < t.rows; i += 64 * kWaves) rows[i] = max(row_at(o, t.first + i), 0);
    const int64_t pt = tiles_before(o, TSH, t.e) + ((int64_t)t.index << (sh - TSH));
    // (offsets out of order may count more tiles than there are sums of)
    if (pt + ((t.rows + TM - 1) >> TSH) > (o.rows >> TSH) + min((int64_t)o.count, o.rows)) return;
    const float f = scale ? scale[t.e] : 1.f;
    __syncthreads();
    const bf16_t *qr = k.q + qc;
    for (int grp = 0; grp < groups; ++grp) {
        const int r0 = grp * 16 * NR;
        floatx4 acc[NR][8] = {};
        u32x4 raw[8];
        floatx4 pv[NR][2];
        auto load = [&](int k0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t row = rows[min(k0 + 8 * g + i, t.rows - 1)];
                raw[i] = *reinterpret_cast<const u32x4 *>(qr + row * k.C);
            }
            // (rows behind the last: of no tile's, cut off below)
            const int at = min(k0 + 8 * g, (t.rows - 1) & ~7);
            const float *src =
                k.p.p + ((pt + (at >> TSH)) * k.p.splits * rank + r0) * TM + (at & (TM - 1));
#pragma unroll
            for (int b = 0; b < NR; ++b) {
                // (a rank value behind the last: another's, not stored)
                const int r = min(16 * b + m, rank - 1 - r0);
                pv[b][0] = pv[b][1] = floatx4{};
                for (int s = 0; s < k.p.splits; ++s)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        pv[b][h] += *reinterpret_cast<const floatx4 *>(
                            src + ((int64_t)s * rank + r) * TM + 4 * h);
            }
        };
        if (32 * wave < t.rows) load(32 * wave);
        for (int k0 = 32 * wave; k0 < t.rows; k0 += 32 * kWaves) {
            bf16x8 qv[8], part[NR][3];
            transpose8(raw, qv);
#pragma unroll
            for (int b = 0; b < NR; ++b) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[i] = k0 + 8 * g + i < t.rows ? pv[b][i / 4][i % 4] * f : 0.f;
                cut8<3>(v, part[b]);
            }
            if (k0 + 32 * kWaves < t.rows) load(k0 + 32 * kWaves);
#pragma unroll
            for (int b = 0; b < NR; ++b)
#pragma unroll
                for (int s = 0; s < 3; ++s)
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[b][j] = mfma(part[b][s], qv[j], acc[b][j]);
        }
        // (rows are read again for another group of rank values: kept behind the sums)
        __syncthreads();
        if (wave >= 2) {
#pragma unroll
            for (int b = 0; b < NR; ++b)
#pragma unroll
                for (int j = 0; j < 8; ++j) sums[wave - 2][b * 8 + j][lane] = acc[b][j];
        }
        __syncthreads();
        if (wave < 2) {
#pragma unroll
            for (int b = 0; b < NR; ++b)
#pragma unroll
                for (int j = 0; j < 8; ++j) sums[wave][b * 8 + j][lane] += acc[b][j];
        }
        __syncthreads();
        const bool whole = t.tiles == 1, add = whole && accumulate;
        float *to = whole ? k.out + (int64_t)t.e * rank * k.C
                          : k.parts + (int64_t)(t.several + t.index) * rank * k.C;
        if (col < k.C && k.transposed) {
            // four rank values of a column: wave w has columns j = w, w + 4
#pragma unroll
            for (int b = 0; b < NR; ++b)
#pragma unroll
                for (int j = 0; j < 8; j += kWaves) {
                    const int r = r0 + 16 * b + 4 * g;
                    if (r >= rank) continue;
                    const floatx4 v =
                        sums[0][b * 8 + j + wave][lane] + sums[1][b * 8 + j + wave][lane];
                    floatx4 *d =
                        reinterpret_cast<floatx4 *>(to + (int64_t)(col + j + wave) * rank + r);
                    *d = add ? *d + v : v;
                }
        } else if (col < k.C) {
            // eight columns of a rank value: wave w has the w-th of a lane's four
            const float *s0 = reinterpret_cast<const float *>(sums[0]) + lane * 4 + wave;
            const float *s1 = reinterpret_cast<const float *>(sums[1]) + lane * 4 + wave;
#pragma unroll
            for (int b = 0; b < NR; ++b) {
                const int r = r0 + 16 * b + 4 * g + wave;
                if (r >= rank) continue;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    floatx4 v;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        v[j] = s0[(b * 8 + 4 * h + j) * 256] + s1[(b * 8 + 4 * h + j) * 256];
                    floatx4 *d = reinterpret_cast<floatx4 *>(to + (int64_t)r * k.C + col + 4 * h);
                    *d = add ? *d + v : v;
                }
            }
        }
        if (grp + 1 < groups) {
            __syncthreads();
            for (int i = threadIdx.x; i < t.rows; i += 64 * kWaves)
                rows[i] = max(row_at(o, t.first + i), 0);
            __syncthreads();
        }
    }
}

// The gradient's last products, one launch: blocks of db, of da, of dx.
template <int RB, int NR, class Y>
__global__ __launch_bounds__(64 * kWaves) void back_kernel(AdapterRows o, int rank,
                                                           const float *scale, int sh, int slots,
                                                           int accumulate, Outer kb, Outer ka,
                                                           Expand<Y> kx) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int b = blockIdx.x;
    if (b < kb.blocks + ka.blocks)
        outer<RB, NR>(o, rank, scale, sh, slots, accumulate, b < kb.blocks ? kb : ka,
                      b < kb.blocks ? b : b - kb.blocks, lds);
    else
        expand<RB, Y>(o, rank, kx, b - kb.blocks - ka.blocks, lds);
}

// Adapters of several tiles: their parts, added in order; adapters of no rows:
// zeros (nothing where out accumulates).  blockIdx.z: da, db.
__global__ __launch_bounds__(256) void join_kernel(AdapterRows o, int sh, int slots, int accumulate,
                                                   Outer ka, Outer kb, int rank) {
    const Outer &k = blockIdx.z ? kb : ka;
    const int e = blockIdx.y, lane = threadIdx.x & 63;
    const int64_t size = (int64_t)rank * k.C;
    auto tiles_of = [&](int i) {
        if (o.rows == 0) return 0;  // offsets need not be there
        return (max(offset_at(o, i + 1) - offset_at(o, i), 0) + (1 << sh) - 1) >> sh;
    };
    int n = tiles_of(e);
    if (n == 1 || (n == 0 && accumulate)) return;
    // tiles of several-tile adapters before e
    int before = 0;
    for (int i = lane; i < e; i += 64) {
        const int q = tiles_of(i);
        before += q > 1 ? q : 0;
    }
    before = __builtin_amdgcn_readlane(wave_inclusive_scan(before), 63);
    n = min(n, slots - before);
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < size;
         i += (int64_t)gridDim.x * 1024) {
        floatx4 v = {};
        for (int j = 0; j < n; ++j)
            v += *reinterpret_cast<const floatx4 *>(k.parts + (int64_t)(before + j) * size + i);
        floatx4 *d = reinterpret_cast<floatx4 *>(k.out + (int64_t)e * size + i);
        *d = accumulate ? *d + v : v;
    }
}

// ---- launches --------------------------------------------------------------

// Tiles of 2^sh rows that `count` adapters can have.
int64_t tile_cap(int64_t rows, int count, int sh) {
    return (rows >> sh) + std::min<int64_t>(count, rows);
}
// Tiles of 64 rows, where they are many and the adapters' mean rows fill most of one.
bool tall(int64_t rows, int count) { return rows >= 4096 && rows >= (int64_t)48 * count; }
int tile_shift(int64_t rows, int count) { return tall(rows, count) ? 6 : 4; }
// Rows of a tile of the outer products, as a power of two: about 16 tiles, which with
// some 60 column blocks fill the chip.
int outer_shift(int64_t rows) { return rows >= 4096 ? 9 : rows >= 2048 ? 8 : 7; }
int64_t outer_slots(int64_t rows) { return 2 * (rows >> outer_shift(rows)) + 2; }

template <int RB, int NR>
hipError_t run_shrink(const AdapterRows &o, int rank, const Shrink &k, const Transpose &ta,
                      const Transpose &tb, hipStream_t s) {
    const unsigned groups = (rank + 16 * NR - 1) / (16 * NR);
    const unsigned grid = (unsigned)k.tiles * k.out.splits * groups + ta.blocks + tb.blocks;
    shrink_kernel<RB, NR><<<grid, 64 * kShrinkWaves, 0, s>>>(o, rank, k, ta, tb);
    return hipGetLastError();
}

hipError_t launch_shrink(const AdapterRows &o, int rank, int K, const bf16_t *x, const bf16_t *w,
                         const AdapterSums &out, const Transpose &ta, const Transpose &tb,
                         hipStream_t s) {
    const Shrink k{x, w, out, K,
                   x ? (int)tile_cap(o.rows, o.count, tile_shift(o.rows, o.count)) : 0};
    auto go = [&](auto fn) { return fn(o, rank, k, ta, tb, s); };
    if (tall(o.rows, o.count))
        return rank <= 16 ? go(run_shrink<4, 1>)
                          : rank <= 32 ? go(run_shrink<4, 2>) : go(run_shrink<4, 4>);
    return rank <= 16 ? go(run_shrink<1, 1>)
                      : rank <= 32 ? go(run_shrink<1, 2>) : go(run_shrink<1, 4>);
}

template <class Y>
Expand<Y> make_expand(const AdapterRows &o, int rank, int N, const AdapterSums &u, const bf16_t *w,
                      const float *scale, const void *base, void *y) {
    Expand<Y> k{u, w, scale, (const Y *)base, (Y *)y, N, 0, 0, 0, 0};
    if (!y) return k;
    k.tiles = (int)tile_cap(o.rows, o.count, tile_shift(o.rows, o.count));
    k.copies = base == y ? 0 : (int)((o.rows + 63) / 64);
    // a block a wave; larger ranks take u's cutting further
    k.span = kWaves * (rank <= 64 ? 1 : rank <= 128 ? 2 : 4);
    k.ranges = (N / 64 + k.span - 1) / k.span;
    return k;
}
template <class Y>
size_t expand_lds(int64_t rows, int count, int rank) {
    return (size_t)(tall(rows, count) ? 4 : 1) * ((rank / 8 * Piece<Y>::S + 3) / 4 * 4) * 256;
}
template <class Y>
int64_t expand_blocks(const Expand<Y> &k) {
    return (int64_t)(k.tiles + k.copies) * k.ranges;
}

// More than 64 KB of LDS are asked for.
hipError_t allow_lds(const void *fn, size_t lds) {
    return lds > 65536 ? hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)lds)
                       : hipSuccess;
}

template <class Y>
hipError_t run_expand(const AdapterRows &o, int rank, const Expand<Y> &k, hipStream_t s) {
    const size_t lds = expand_lds<Y>(o.rows, o.count, rank);
    const unsigned grid = (unsigned)expand_blocks(k);
    const auto fn = tall(o.rows, o.count) ? expand_kernel<4, Y> : expand_kernel<1, Y>;
    if (hipError_t e = allow_lds((const void *)fn, lds)) return e;
    fn<<<grid, 64 * kWaves, lds, s>>>(o, rank, k);
    return hipGetLastError();
}

template <int RB, int NR, class Y>
hipError_t run_back(const AdapterRows &o, int rank, const float *scale, bool accumulate,
                    const Outer &kb, const Outer &ka, const Expand<Y> &kx, hipStream_t s) {
    const int sh = outer_shift(o.rows);
    size_t lds = kx.y ? expand_lds<Y>(o.rows, o.count, rank) : 0;
    if (ka.blocks) lds = std::max(lds, (size_t)(kWaves / 2) * NR * 8 * 64 * sizeof(floatx4));
    const unsigned grid = (unsigned)(kb.blocks + ka.blocks + expand_blocks(kx));
    const auto fn = back_kernel<RB, NR, Y>;
    if (hipError_t e = allow_lds((const void *)fn, lds)) return e;
    fn<<<grid, 64 * kWaves, lds, s>>>(o, rank, scale, sh, (int)outer_slots(o.rows), accumulate, kb,
                                      ka, kx);
    return hipGetLastError();
}

template <class Y>
hipError_t launch_back(const AdapterRows &o, int rank, const float *scale, bool accumulate,
                       const Outer &kb, const Outer &ka, const Expand<Y> &kx, hipStream_t s) {
    auto go = [&](auto fn) { return fn(o, rank, scale, accumulate, kb, ka, kx, s); };
    if (tall(o.rows, o.count))
        return rank <= 16 ? go(run_back<4, 1, Y>)
                          : rank <= 32 ? go(run_back<4, 2, Y>) : go(run_back<4, 4, Y>);
    return rank <= 16 ? go(run_back<1, 1, Y>)
                      : rank <= 32 ? go(run_back<1, 2, Y>) : go(run_back<1, 4, Y>);
}

}  // namespace

int adapter_splits(int64_t rows, int count, int K, int rank) {
    // workgroups for every compute unit; a step of 64 k for every wave
    const int64_t tiles = std::max<int64_t>(tile_cap(rows, count, tile_shift(rows, count)), 1);
    const int64_t want = tall(rows, count) ? 1024 : 512;
    const int64_t most = std::min(std::max(1, K / 64 / kShrinkWaves),
                                  tall(rows, count) ? rank <= 32 ? 4 : 2 : 16);
    return (int)std::max<int64_t>(1, std::min((want + tiles - 1) / tiles, most));
}

size_t adapter_sums_bytes(int64_t rows, int count, int rank) {
    auto bytes = [&](int64_t r) {
        const int sh = tile_shift(r, count);
        const int64_t tiles = tile_cap(r, count, sh);
        // no more than splits * tiles of these rows or fewer
        const int64_t sums = tall(r, count) ? std::max(tiles, std::min<int64_t>(4 * tiles, 2048))
                                            : std::max(tiles, std::min<int64_t>(16 * tiles, 1024));
        return (size_t)sums * rank * sizeof(float) << sh;
    };
    // (the tiles' height changes at one number of rows)
    const int64_t edge = std::max<int64_t>(4096, (int64_t)48 * count);
    return rows >= edge ? std::max(bytes(rows), bytes(edge - 1)) : bytes(rows);
}

size_t adapter_parts_bytes(int64_t rows, int rank, int C) {
    int64_t most = outer_slots(rows);
    for (int64_t r : {2047, 4095})  // the last rows of each tile height
        if (r < rows) most = std::max(most, outer_slots(r));
    return (size_t)most * rank * C * sizeof(float);
}

hipError_t launch_adapter_rows(const AdapterRows &o, const moe_adapters &ad, const bf16_t *x,
                               const void *base, void *y, int y_type, const AdapterSums &u,
                               hipStream_t s) {
    const Transpose none{};
    if (hipError_t e = launch_shrink(o, ad.rank, ad.k, x, ad.a, u, none, none, s)) return e;
    if (y_type == MOE_FP32)
        return run_expand(
            o, ad.rank, make_expand<float>(o, ad.rank, ad.n, u, ad.b, ad.scale, base, y), s);
    return run_expand(o, ad.rank,
                      make_expand<bf16_t>(o, ad.rank, ad.n, u, ad.b, ad.scale, base, y), s);
}

hipError_t launch_adapter_backward(const AdapterRows &o, const moe_adapters &ad,
                                   const AdapterBack &k, hipStream_t s) {
    const int tiles = o.rows ? (int)tile_cap(o.rows, o.count, outer_shift(o.rows)) : 0;
    Outer ka{k.v, k.x, k.pa, k.da, ad.k, 0, (ad.k + 127) / 128, 0};
    Outer kb{k.u, k.dy, k.pb, k.db, ad.n, 1, (ad.n + 127) / 128, 0};
    if (k.da) {
        ka.blocks = tiles * ka.cb;
        kb.blocks = tiles * kb.cb;
    }
    if (o.rows) {
        auto turn = [&](const bf16_t *w, bf16_t *wt, int m, int n) {
            const int bx = (n + 63) / 64;
            return Transpose{w, wt, m, n, bx, o.count * bx * ((m + 63) / 64)};
        };
        // u = A x (for db), B^T, A^T (for dx)
        if (hipError_t e = launch_shrink(o, ad.rank, ad.k, k.da ? k.x : nullptr, ad.a, k.u,
                                         turn(ad.b, k.bt, ad.n, ad.rank),
                                         k.dx ? turn(ad.a, k.at, ad.rank, ad.k) : Transpose{}, s))
            return e;
        // v = B^T dy
        if (hipError_t e = launch_shrink(o, ad.rank, ad.n, k.dy, k.bt, k.v, Transpose{},
                                         Transpose{}, s))
            return e;
        if (k.dx_type == MOE_FP32) {
            const auto kx =
                make_expand<float>(o, ad.rank, ad.k, k.v, k.at, ad.scale, k.base, k.dx);
            if (hipError_t e = launch_back(o, ad.rank, ad.scale, k.accumulate, kb, ka, kx, s))
                return e;
        } else {
            const auto kx =
                make_expand<bf16_t>(o, ad.rank, ad.k, k.v, k.at, ad.scale, k.base, k.dx);
            if (hipError_t e = launch_back(o, ad.rank, ad.scale, k.accumulate, kb, ka, kx, s))
                return e;
        }
    }
    if (!k.da) return hipSuccess;
    const int64_t size = (int64_t)ad.rank * std::max(ad.n, ad.k);
    const unsigned bx = (unsigned)std::min<int64_t>((size + 1023) / 1024, 64);
    join_kernel<<<dim3(bx, o.count, 2), 256, 0, s>>>(o, outer_shift(o.rows),
                                                     (int)outer_slots(o.rows), k.accumulate, ka, kb,
                                                     ad.rank);
    return hipGetLastError();
}

}  // namespace moe
