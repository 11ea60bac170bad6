// Low-rank adapters of many requests beside a shared projection,
//   y = base + scale (x A^T) B^T,
// and their gradient.  Rows are ordered by adapter, as the dispatch orders
// tokens by expert; a tile is up to 16 or 128 rows of one adapter, found on the
// device from the adapters' offsets.
//
// The sums over K of x A^T ("shrink") go through memory in fp32: rank values a
// row, where the rows themselves have thousands.  The products behind it take
// them cut into bf16 parts (hi + mid + lo hold all 24 bits), so that the matrix
// cores multiply bf16 by bf16 without a rounding.  Few rows are bound by latencies, many
// by memory: the matrix cores are busy 1 to 13% of the time.  Times below are of one call among
// others on inputs of their own (4096 x 4096, bf16 y, where nothing else is said).
#include "adapters.h"

#include <algorithm>
#include <limits>
#include <type_traits>

#include "dispatch.h"

namespace moe {
namespace {

constexpr int kWaves = 8;  // of expand (tall tiles: a row block each; short: 64 columns) and
                           // of outer (four column blocks, two halves of the rows)
constexpr int kExpandSpan = 8;  // blocks of 64 columns of expand's workgroups
constexpr int kMostSplits = 8;  // shares of K

// Row blocks of 16 of a tile (1 or 8) -> rows of it, as a power of two.
constexpr int tile_shift_of(int RB) { return RB == 8 ? 7 : 4; }
// The waves of shrink.
constexpr int shrink_waves(int RB) { return RB == 1 ? 4 : RB; }
constexpr int kParts = 3;   // bf16 parts that hold fp32's 24 bits
constexpr int kPitch = 17;  // operands of 16 rows and one: writes of different banks

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

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) {
    return __builtin_amdgcn_perm(b, a, 0x05040100u);
}
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) {
    return __builtin_amdgcn_perm(b, a, 0x07060302u);
}
// Four values of each of two rows `pitch` apart.
__device__ __forceinline__ bf16x8 load_pair(const bf16_t *p, int pitch) {
    const u32x2 a = *reinterpret_cast<const u32x2 *>(p);
    const u32x2 b = *reinterpret_cast<const u32x2 *>(p + pitch);
    return __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]});
}
// The two of each column to word `at` of an operand in LDS, the next column's `step`
// words behind.
__device__ __forceinline__ void put_pair(bf16x8 *to, int at, int step, bf16x8 pair) {
    const u32x4 u = __builtin_bit_cast(u32x4, pair);
    uint32_t *p = reinterpret_cast<uint32_t *>(to) + at;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        p[q * step] = q & 1 ? high_halves(u[q / 2], u[2 + q / 2])
                            : low_halves(u[q / 2], u[2 + q / 2]);
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

// Tile t of all adapters' tiles of 2^sh rows; behind the last e < 0, and index counts on
// from 0.  Every lane takes four adapters' counts; a scan over the lanes finds the
// tile's.  The result is uniform.
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
    if (!has) {
        r.index = t - __builtin_amdgcn_readlane(incl, 63);
        return r;
    }
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
    if (r.rows <= 0) r.e = -1;  // (offsets out of order over so many rows that sums wrapped)
    return r;
}

// The row of a place, -1 if it is none.
__device__ __forceinline__ int row_at(const AdapterRows &o, int64_t place) {
    const int row = o.order[place];
    return (uint32_t)row < (uint64_t)o.rows ? row : -1;
}

// Whether a row is that of a place of an adapter's (offsets that ascend).
__device__ __forceinline__ bool has_place(const AdapterRows &o, int64_t row) {
    const int p = o.place[row];
    const bool in = p >= offset_at(o, 0) && p < offset_at(o, o.count);
    return in && o.order[in ? p : 0] == row;
}

// hi + mid + lo: the leading 8 bits by cutting, the last part rounded.
__device__ __forceinline__ void cut(float v, uint32_t (&part)[kParts]) {
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
        const uint32_t u = __float_as_uint(v);
        if (i + 1 < kParts) {
            part[i] = u >> 16;
            v = (u & 0x7F800000u) == 0x7F800000u ? 0.f : v - __uint_as_float(u & 0xFFFF0000u);
        } else {
            const bool special = (u & 0x7F800000u) == 0x7F800000u;
            part[i] = (special ? u : u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
        }
    }
}
// Eight values' parts, two to a word.
__device__ __forceinline__ void cut8(const float (&v)[8], bf16x8 (&part)[kParts]) {
    u32x4 w[kParts] = {};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t c[kParts];
        cut(v[j], c);
#pragma unroll
        for (int q = 0; q < kParts; ++q) w[q][j / 2] |= c[q] << (16 * (j & 1));
    }
#pragma unroll
    for (int q = 0; q < kParts; ++q) part[q] = __builtin_bit_cast(bf16x8, w[q]);
}

// v[j] += the sum over splits of p[split * pitch + j * TM], four splits' loads at once.
template <int TM>
__device__ __forceinline__ void sum_splits(float (&v)[8], const float *p, int pitch, int splits) {
    for (int q = 0; q < splits; q += 4) {
        float w[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) w[i][j] = p[min(q + i, splits - 1) * pitch + j * TM];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += q + i < splits ? w[i][j] : 0.f;
    }
}

// Sums of tall tiles, scaled and cut once a row for the many workgroups behind: by the
// workgroup that has all of them, or where K is split by a launch of its own.  e:
// parts as operands of expand, [tile][row block][chunk][row][8] with the chunks of
// Expand; q: parts as operands of outer, [tile][part][rank][row].  16384 rows of
// rank 64: 7.2 us, where every workgroup of expand cutting for itself cost 40.
struct Cut {
    bool e, q;
};

__host__ __device__ __forceinline__ int chunks_of(int rank) {
    return (rank / 8 * kParts + 3) / 4 * 4;
}

// p: [split][rank][row], PITCH values a rank value.
template <int RB, int PITCH>
__device__ __forceinline__ void cut_tile(const AdapterRows &o, int rank, const float *scale,
                                         const Cut &k, const AdapterSums &u, const Tile &t,
                                         int tile, const float *p, int splits) {
    constexpr int TM = 16 * RB;
    const int rc = rank / 8, chunks = chunks_of(rank);
    const float f = scale ? scale[t.e] : 1.f;
    bf16x8 *e = reinterpret_cast<bf16x8 *>(u.e) + (int64_t)tile * chunks * TM;
    uint16_t *q = u.q + (int64_t)tile * kParts * rank * TM;
    for (int i = threadIdx.x; i < TM * rc; i += 512) {
        const int row = i % TM, kc = i / TM;
        float v[8] = {};
        if (row < t.rows && row_at(o, t.first + row) >= 0) {
            sum_splits<PITCH>(v, p + 8 * kc * PITCH + row, rank * PITCH, splits);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= f;
        }
        if (k.e) {
            bf16x8 part[kParts];
            cut8(v, part);
#pragma unroll
            for (int s = 0; s < kParts; ++s)
                e[((row >> 4) * chunks + s * rc + kc) * 16 + (row & 15)] = part[s];
        }
        if (k.q) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t c[kParts];
                cut(v[j], c);
#pragma unroll
                for (int s = 0; s < kParts; ++s)
                    q[((int64_t)s * rank + 8 * kc + j) * TM + row] = (uint16_t)c[s];
            }
        }
    }
    // the padding behind the last part
    const int pad = k.e ? chunks - rc * kParts : 0;
    for (int i = threadIdx.x; i < TM * pad; i += 512) {
        const int row = i % TM, c = rc * kParts + i / TM;
        e[((row >> 4) * chunks + c) * 16 + (row & 15)] = bf16x8{};
    }
}

// ---- x A^T ---------------------------------------------------------------

// Sums of `rows` times w [count][rank][K], or where TURNED [count][K][rank] (the
// gradient's).  The matrix instruction's M is the rows, its N the rank.
struct Shrink {
    const bf16_t *x, *w;
    AdapterSums out;
    int K, tiles;
    Cut cut;  // of tall tiles
};

// Short tiles: operands straight to registers, 64 bytes of each of 16 rows a load.
// The four waves (and `splits` workgroups) share K, each taking every so many-th 128
// bytes of a row, and keep DEP steps of them in flight.  A turned w comes a value a
// lane: a load has 16 rank values of four k, side by side where the rank is 16.
// 64 rows of as many adapters, 6144 k, rank 32: 7.4 us, a launch's chain of latencies
// (offsets, order, rows) and 15 MB; both sums of the gradient of 997 rows 10 us (with
// the adapter transposed by a launch before it 11.2 + 3.8).
template <int NR, bool TURNED>
__device__ __forceinline__ void shrink_short(const AdapterRows &o, int rank, const Shrink &k,
                                             int tile, int split, int r0, floatx4 *lds) {
    constexpr int DEP = NR == 1 || (NR == 2 && !TURNED) ? 4 : 2, KG = shrink_waves(1);
    const Tile t = find_tile(o, tile_shift_of(1), tile);
    if (t.e < 0) return;
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int kg = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int parts = k.out.splits * KG, part = split * KG + kg;
    const int n = (k.K / 64 - part + parts - 1) / parts;
    const int row = row_at(o, t.first + min(m, t.rows - 1));
    uint32_t wo[NR];
#pragma unroll
    for (int c = 0; c < NR; ++c)  // behind the last rank value: the last again, not stored
        wo[c] = TURNED ? (uint32_t)(8 * g * rank + min(r0 + 16 * c + m, rank - 1)) * 2
                       : ((uint32_t)min(r0 + 16 * c + m, rank - 1) * k.K + 8 * g) * 2;
    const char *xs = (const char *)(k.x + (int64_t)max(row, 0) * k.K + part * 64 + 8 * g);
    const char *ws =
        (const char *)(k.w + (int64_t)t.e * rank * k.K + (int64_t)part * 64 * (TURNED ? rank : 1));
    floatx4 acc[NR] = {};
    using W = std::conditional_t<TURNED, uint16_t[8], bf16x8>;
    bf16x8 xv[DEP][2];
    W wv[DEP][NR][2];
    // (both halves of a cache line one after the other: it may not stay)
    auto load = [&](int i, int s) {
        const int at = s * parts * 128;
#pragma unroll
        for (int h = 0; h < 2; ++h) xv[i][h] = *reinterpret_cast<const bf16x8 *>(xs + at + 64 * h);
#pragma unroll
        for (int c = 0; c < NR; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if constexpr (TURNED) {
                    const char *p = ws + (int64_t)at * rank + wo[c];
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        wv[i][c][h][q] =
                            *reinterpret_cast<const uint16_t *>(p + (32 * h + q) * rank * 2);
                } else {
                    wv[i][c][h] = *reinterpret_cast<const bf16x8 *>(ws + at + wo[c] + 64 * h);
                }
            }
    };
    auto operand = [&](const W &w) {
        if constexpr (TURNED) {
            u32x4 v;
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = w[2 * q] | (uint32_t)w[2 * q + 1] << 16;
            return __builtin_bit_cast(bf16x8, v);
        } else {
            return w;
        }
    };
    auto use = [&](int i) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int c = 0; c < NR; ++c) acc[c] = mfma(xv[i][h], operand(wv[i][c][h]), acc[c]);
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
    // the waves' sums meet in LDS, half of them at a time
#pragma unroll
    for (int half = KG / 2; half >= 1; half /= 2) {
        floatx4 *at = lds + (kg % half) * NR * 64 + lane;
        if (kg >= half && kg < 2 * half) {
#pragma unroll
            for (int c = 0; c < NR; ++c) at[c * 64] = acc[c];
        }
        __syncthreads();
        if (kg < half) {
#pragma unroll
            for (int c = 0; c < NR; ++c) acc[c] += at[c * 64];
        }
        __syncthreads();
    }
    if (kg > 0) return;
    float *p = k.out.p + ((int64_t)tile * k.out.splits + split) * rank * 16;
#pragma unroll
    for (int c = 0; c < NR; ++c) {
        const int r = r0 + 16 * c + m;
        if (r < rank) *reinterpret_cast<floatx4 *>(p + r * 16 + 4 * g) = acc[c];
    }
}

// Tall tiles: a wave has a row block and all of the rank.  Rows and adapter come in as
// whole lines (eight lanes to the 128 bytes of a row: the cache takes a lane's 16 bytes
// of a row of its own as slowly as 64 of a shared one), AHEAD steps of 64 k in
// registers, and lie in LDS as operands [block][chunk of 8 k][row][8], two steps in
// turn.  `splits` workgroups share K.  16384 rows of rank 64: 45 us, of which reading
// 134 MB of rows not in a cache takes some 40; 55 with lanes on rows of their own.  1, 2
// or 4 to 8 splits in place of 3: 53, 60, 47 to 50.  Of a turned w a thread takes four
// rank values of two k.
template <int RB, int NR>
struct TallShrink {
    static constexpr int TH = 64 * shrink_waves(RB), AHEAD = 3;
    static constexpr int XI = 2, WI = (2 * NR + RB - 1) / RB;  // loads of a thread
    static constexpr int XL = RB * 8 * kPitch, WL = NR * 8 * kPitch;
    static constexpr size_t LDS = (size_t)2 * (XL + WL) * 16;
};

template <int RB, int NR, bool TURNED>
__device__ __forceinline__ void shrink_tall(const AdapterRows &o, int rank, const Shrink &k,
                                            const float *scale, int tile, int split,
                                            char *lds) {
    using C = TallShrink<RB, NR>;
    constexpr int TM = 16 * RB, D = C::AHEAD, XI = C::XI, WI = C::WI;
    const Tile t = find_tile(o, tile_shift_of(RB), tile);
    if (t.e < 0) return;
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int steps = k.K / 64, lo = (int)((int64_t)steps * split / k.out.splits);
    const int n = (int)((int64_t)steps * (split + 1) / k.out.splits) - lo;
    const bf16_t *xp[XI];
    uint32_t wo[WI];
    int xt[XI], wt[WI];  // places in LDS
#pragma unroll
    for (int i = 0; i < XI; ++i) {
        const int item = threadIdx.x + C::TH * i, r = item / 8, ch = item % 8;
        const int row = row_at(o, t.first + min(r, t.rows - 1));
        xp[i] = k.x + (int64_t)max(row, 0) * k.K + lo * 64 + 8 * ch;
        xt[i] = ((r >> 4) * 8 + ch) * kPitch + (r & 15);
    }
#pragma unroll
    for (int i = 0; i < WI; ++i) {  // behind the last rank value: the last again, not stored
        const int at = threadIdx.x + C::TH * i;
        if constexpr (TURNED) {
            const int item = min(at, 8 * rank - 1), kk = item / (rank / 4) * 2;
            const int r = item % (rank / 4) * 4;
            wo[i] = kk * rank + r;
            wt[i] = (C::XL + ((r >> 4) * 8 + (kk >> 3)) * kPitch + (r & 15)) * 4 + (kk & 7) / 2;
        } else {
            const int item = min(at, 16 * NR * 8 - 1), r = item / 8;
            wo[i] = ((uint32_t)min(r, rank - 1) * k.K + 8 * (item % 8)) * 2;
            wt[i] = C::XL + ((r >> 4) * 8 + item % 8) * kPitch + (r & 15);
        }
    }
    const int per_step = 64 * (TURNED ? rank : 1);
    const bf16_t *we = k.w + (int64_t)t.e * rank * k.K + (int64_t)lo * per_step;
    bf16x8 xv[D][XI], wv[D][WI];
    auto load = [&](int i, int s) {
#pragma unroll
        for (int j = 0; j < XI; ++j) xv[i][j] = load8(xp[j] + s * 64);
#pragma unroll
        for (int j = 0; j < WI; ++j) {
            const bf16_t *p = we + (int64_t)s * per_step;
            wv[i][j] = TURNED ? load_pair(p + wo[j], rank) : load8(p, wo[j]);
        }
    };
    floatx4 acc[NR] = {};
    bf16x8 *buf = reinterpret_cast<bf16x8 *>(lds);
    auto put = [&](int i, bf16x8 *to) {
#pragma unroll
        for (int j = 0; j < XI; ++j) to[xt[j]] = xv[i][j];
#pragma unroll
        for (int j = 0; j < WI; ++j) {
            if constexpr (TURNED)
                put_pair(to, wt[j], 4, wv[i][j]);
            else
                to[wt[j]] = wv[i][j];
        }
    };
    auto use = [&](const bf16x8 *from) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const bf16x8 a = from[(wave * 8 + 4 * h + g) * kPitch + m];
#pragma unroll
            for (int c = 0; c < NR; ++c)
                acc[c] = mfma(a, from[C::XL + (c * 8 + 4 * h + g) * kPitch + m], acc[c]);
        }
    };
    constexpr int SZ = C::XL + C::WL;
    if (n > 0) {
#pragma unroll
        for (int i = 0; i < D; ++i) load(i, min(i, n - 1));
        // One barrier a step: who writes a buffer has passed the barrier behind which
        // its last readers were done.
        int s = 0, p = 0;
        for (; s + D <= n; s += D) {
#pragma unroll
            for (int i = 0; i < D; ++i, p ^= 1) {
                put(i, buf + p * SZ);
                load(i, min(s + i + D, n - 1));
                __syncthreads();
                use(buf + p * SZ);
            }
        }
#pragma unroll
        for (int i = 0; i < D; ++i, p ^= 1)
            if (s + i < n) {
                put(i, buf + p * SZ);
                __syncthreads();
                use(buf + p * SZ);
            }
    }
    constexpr int PITCH = TM + 4;
    static_assert((size_t)16 * NR * PITCH * 4 <= C::LDS, "room for the sums");
    const bool whole = k.out.splits == 1;
    float *p = whole ? reinterpret_cast<float *>(lds)
                     : k.out.p + ((int64_t)tile * k.out.splits + split) * rank * TM;
    const int pitch = whole ? PITCH : TM;
    if (whole) __syncthreads();  // the operands have been read
#pragma unroll
    for (int c = 0; c < NR; ++c) {
        const int r = 16 * c + m;
        if (r < rank) *reinterpret_cast<floatx4 *>(p + r * pitch + 16 * wave + 4 * g) = acc[c];
    }
    if (!whole) return;
    __syncthreads();
    cut_tile<RB, PITCH>(o, rank, scale, k.cut, k.out, t, tile,
                        reinterpret_cast<const float *>(lds), 1);
}

// Few rows of few k: every workgroup of expand has its tile's sums itself, which saves
// a launch.  A wave takes every eighth 64 k; rows and adapter come in as whole lines
// and become operands through LDS of the wave's own, DEP steps in flight.  The waves'
// sums lie at the end in lds, [wave][rank][row].
template <int NR>
struct OwnSums {
    static constexpr int DEP = NR == 1 ? 8 : 4, OPERANDS = (1 + NR) * 8 * kPitch;  // a wave's
    static constexpr size_t LDS = (size_t)kWaves * OPERANDS * 16;
    static_assert(LDS >= (size_t)kWaves * 16 * NR * 16 * sizeof(float), "room for the sums");
};

template <int NR>
__device__ __forceinline__ void own_sums(const AdapterRows &o, int rank, const Tile &t,
                                         const bf16_t *x, const bf16_t *a, int K, char *lds) {
    using C = OwnSums<NR>;
    constexpr int DEP = C::DEP;
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int line = lane >> 3, ch = lane & 7;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = (K / 64 - wave + kWaves - 1) / kWaves;
    bf16x8 *own = reinterpret_cast<bf16x8 *>(lds) + wave * C::OPERANDS;
    const bf16_t *xp[2], *ap[2 * NR];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int row = row_at(o, t.first + min(8 * j + line, t.rows - 1));
        xp[j] = x + (int64_t)max(row, 0) * K + wave * 64 + 8 * ch;
    }
#pragma unroll
    for (int j = 0; j < 2 * NR; ++j)  // behind the last rank value: the last again, not stored
        ap[j] = a + ((int64_t)t.e * rank + min(8 * j + line, rank - 1)) * K + wave * 64 + 8 * ch;
    bf16x8 xv[DEP][2], av[DEP][2 * NR];
    auto load = [&](int i, int s) {
#pragma unroll
        for (int j = 0; j < 2; ++j) xv[i][j] = load8(xp[j] + s * kWaves * 64);
#pragma unroll
        for (int j = 0; j < 2 * NR; ++j) av[i][j] = load8(ap[j] + s * kWaves * 64);
    };
    floatx4 acc[NR] = {};
    auto use = [&](int i) {
#pragma unroll
        for (int j = 0; j < 2; ++j) own[ch * kPitch + 8 * j + line] = xv[i][j];
#pragma unroll
        for (int j = 0; j < 2 * NR; ++j)
            own[((1 + j / 2) * 8 + ch) * kPitch + 8 * (j & 1) + line] = av[i][j];
        wave_sync();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const bf16x8 v = own[(4 * h + g) * kPitch + m];
#pragma unroll
            for (int c = 0; c < NR; ++c)
                acc[c] = mfma(v, own[((1 + c) * 8 + 4 * h + g) * kPitch + m], acc[c]);
        }
        wave_sync();
    };
    if (n > 0) {
#pragma unroll
        for (int i = 0; i < DEP; ++i) load(i, min(i, n - 1));
        int s = 0;
        for (; s + DEP < n; s += DEP) {
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
    __syncthreads();
    float *sums = reinterpret_cast<float *>(lds) + wave * rank * 16;
#pragma unroll
    for (int c = 0; c < NR; ++c) {
        const int r = 16 * c + m;
        if (r < rank) *reinterpret_cast<floatx4 *>(sums + r * 16 + 4 * g) = acc[c];
    }
    __syncthreads();
}

// Blocks of one shrink, then of another (of the gradient, whose first is turned).
template <int RB, int NR, bool TURNED>
__global__ __launch_bounds__(64 * shrink_waves(RB), RB == 1 ? 2 : 4) void shrink_kernel(
    AdapterRows o, int rank, const float *scale, Shrink k0, Shrink k1, int blocks0) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const bool first = (int)blockIdx.x < blocks0;
    const Shrink &k = first ? k0 : k1;
    const int b = first ? blockIdx.x : blockIdx.x - blocks0;
    const int split = b % k.out.splits, tile = b / k.out.splits % k.tiles;
    auto run = [&](auto turned) {
        if constexpr (RB == 1)
            shrink_short<NR, turned()>(o, rank, k, tile, split,
                                       b / (k.tiles * k.out.splits) * 16 * NR,
                                       reinterpret_cast<floatx4 *>(lds));
        else
            shrink_tall<RB, NR, turned()>(o, rank, k, scale, tile, split, lds);
    };
    if (TURNED && first)
        run(std::bool_constant<TURNED>());
    else
        run(std::false_type());
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __bf16 x = (__bf16)a, y = (__bf16)b;
    return (uint32_t)__builtin_bit_cast(uint16_t, x) |
           ((uint32_t)__builtin_bit_cast(uint16_t, y) << 16);
}

// Of one sum, then of another (of the gradient).
template <int RB>
__global__ __launch_bounds__(512) void cut_kernel(AdapterRows o, int rank, const float *scale,
                                                  Shrink k0, Shrink k1) {
    const bool first = (int)blockIdx.x < k0.tiles;
    const Shrink &k = first ? k0 : k1;
    const int tile = first ? blockIdx.x : blockIdx.x - k0.tiles, splits = k.out.splits;
    if (splits == 1) return;
    const Tile t = find_tile(o, tile_shift_of(RB), tile);
    if (t.e < 0) return;
    constexpr int TM = 16 * RB;
    cut_tile<RB, TM>(o, rank, scale, k.cut, k.out, t, tile,
                     k.out.p + (int64_t)tile * splits * rank * TM, splits);
}

// A lane's four columns of a row, next to each other (the lanes of a group have 64
// between them).
template <class Y>
struct Four;
template <>
struct Four<bf16_t> {
    typedef u32x2 V;
    static __device__ __forceinline__ V add(V base, floatx4 a) {
        return V{pack2(__uint_as_float(base[0] << 16) + a[0],
                       __uint_as_float(base[0] & 0xFFFF0000u) + a[1]),
                 pack2(__uint_as_float(base[1] << 16) + a[2],
                       __uint_as_float(base[1] & 0xFFFF0000u) + a[3])};
    }
};
template <>
struct Four<float> {
    typedef u32x4 V;
    static __device__ __forceinline__ V add(V base, floatx4 a) {
        return __builtin_bit_cast(u32x4, __builtin_bit_cast(floatx4, base) + a);
    }
};

// y = base + scale w u over N columns, w [count][N][rank], or where TURNED
// [count][rank][N] (the gradient's).  A workgroup has a tile of rows and `span` blocks
// of 64 columns.
template <class Y>
struct Expand {
    AdapterSums u;
    const bf16_t *w;
    const float *scale;
    const Y *base;
    Y *y;
    int N, tiles, copies, span, ranges;  // ranges: of span blocks
    const bf16_t *x, *a;                 // for own_sums
    int K;
};

// Rows of no adapter, or of no place: base's row (zeros without one), 64 rows a workgroup.
template <class Y>
__device__ __forceinline__ void copy_rows(const AdapterRows &o, const Expand<Y> &k, int block,
                                          int c0, int c1) {
    constexpr int V = 16 / sizeof(Y);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t mine = (int64_t)block * 64 + lane;
    uint64_t none = __ballot(mine < o.rows && !has_place(o, min(mine, o.rows - 1)));
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

// The contraction runs over three times the rank's positions: u's parts one behind the
// other, against B's columns as many times.  Chunk c (8 positions) is part
// c / (rank / 8) of u; chunks are padded to whole instructions of four.  Where
// rank is a multiple of 32 an operand of B serves all parts.  M is the rows, N the
// output columns: the j-th of four instructions has columns 4 n + j, so that a lane
// ends with four columns of four rows, and a group's loads and stores are 64 columns
// of a row (lanes side by side on one row: the cache takes a lane's 16 bytes of a row
// of its own as slowly as 64 of a shared one).
//
// Tall tiles: the waves have a row block each and the same columns.  B comes in as
// whole lines, by all of them, and lies in LDS as operands [j][chunk][n][8], two blocks
// of 64 columns in turn, two more on their way.  Short tiles: the waves have columns of
// their own and take B's operands from memory.
//
// 16384 rows of rank 64: 80 us (75 with two parts of u, 66 without the products); a
// linear copy of the base alone takes 61 there.  Gradient of 8192 rows, rank 32, w turned:
// 42.
//
// OWN: rank blocks of own_sums, 0 where the sums come from memory.
template <int RB, class Y, bool TURNED, int OWN = 0>
__device__ __forceinline__ void expand(const AdapterRows &o, int rank, const Expand<Y> &k,
                                       int block, char *lds) {
    using P = Four<Y>;
    using V = typename P::V;
    constexpr int TM = 16 * RB;
    constexpr bool SHARED = RB > 1;
    constexpr int TH = 64 * kWaves, WC = SHARED ? 1 : kWaves;
    const int tile = block / k.ranges;
    const int c0 = block % k.ranges * k.span * 64, c1 = min(k.N, c0 + k.span * 64);
    if (tile >= k.tiles) {
        copy_rows(o, k, tile - k.tiles, c0, c1);
        return;
    }
    const Tile t = find_tile(o, tile_shift_of(RB), tile);
    if (t.e < 0) return;
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), b0 = SHARED ? wave : 0;
    const int rc = rank / 8, chunks = chunks_of(rank);
    const bool whole = rank % 32 == 0;
    const int steps = whole ? rc / 4 : chunks / 4;  // of B's operands
    const bf16_t *we = k.w + (int64_t)t.e * k.N * rank;
    int rows[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int p = 16 * b0 + 4 * g + i;
        rows[i] = p < t.rows ? row_at(o, t.first + p) : -1;
    }
    // (a place of no row: row 0's, not stored)
    auto at = [&](int i, int c) { return (int64_t)max(rows[i], 0) * k.N + 4 * m + c; };
    bf16x8 *u = reinterpret_cast<bf16x8 *>(lds);
    V old[4];
    auto load_base = [&](V(&v)[4], int c) {
        if (k.base) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const V *>(k.base + at(i, c));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = V{};
        }
    };
    floatx4 acc[4];
    auto clear = [&] {
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = floatx4{};
    };
    auto product = [&](const bf16x8(&wv)[4], int st) {
        if (whole) {
#pragma unroll
            for (int q = 0; q < kParts; ++q) {
                const bf16x8 uv = u[(b0 * chunks + q * rc + 4 * st + g) * 16 + m];
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] = mfma(uv, wv[j], acc[j]);
            }
        } else {
            const bool pad = 4 * st + g >= rc * kParts;  // zeros against u's zeros: B may hold inf
            const bf16x8 uv = u[(b0 * chunks + 4 * st + g) * 16 + m];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = mfma(uv, pad ? bf16x8{} : wv[j], acc[j]);
        }
    };
    auto store = [&](const V(&v)[4], int c) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (rows[i] >= 0)
                *reinterpret_cast<V *>(k.y + at(i, c)) =
                    P::add(v[i], floatx4{acc[0][i], acc[1][i], acc[2][i], acc[3][i]});
    };
    auto chunk_of = [&](int st) { return whole ? 4 * st + g : (4 * st + g) % rc; };

    if constexpr (SHARED) {
        bf16x8 *wl = u + RB * chunks * 16;  // two blocks of B
        const int size = 4 * rc * kPitch, items = 64 * rc;
        auto run = [&](auto its) {
            constexpr int IT = its();
            bf16x8 w[2][IT];
            V hold[2][4];
            int from[IT], to[IT];  // a thread's operands of 64 columns, as they lie
#pragma unroll
            for (int it = 0; it < IT; ++it) {
                const int i = min((int)threadIdx.x + TH * it, items - 1), col = i / rc;
                if constexpr (TURNED) {  // four columns of two rank values
                    const int r = i / 16 * 2;
                    from[it] = r * k.N + i % 16 * 4;
                    to[it] = (r / 8 * kPitch + i % 16) * 4 + r % 8 / 2;
                } else {
                    from[it] = 8 * i;
                    to[it] = ((col & 3) * rc + i % rc) * kPitch + (col >> 2);
                }
            }
            auto load_w = [&](bf16x8(&v)[IT], int c) {
                const bf16_t *p = we + (TURNED ? c : (int64_t)c * rank);
#pragma unroll
                for (int it = 0; it < IT; ++it)
                    v[it] = TURNED ? load_pair(p + from[it], k.N) : load8(p + from[it]);
            };
            // (behind the last: the last again)
            auto write_w = [&](const bf16x8(&v)[IT], bf16x8 *p) {
#pragma unroll
                for (int it = 0; it < IT; ++it) {
                    if constexpr (TURNED)
                        put_pair(p, to[it], rc * kPitch * 4, v[it]);
                    else
                        p[to[it]] = v[it];
                }
            };
            auto block_product = [&](const bf16x8 *from) {
                clear();
                for (int st = 0; st < steps; ++st) {
                    const int ch = chunk_of(st);
                    bf16x8 wv[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) wv[j] = from[(j * rc + ch) * kPitch + m];
                    product(wv, st);
                }
            };
            const int nb = (c1 - c0) / 64;  // blocks; two of them on their way
            auto column = [&](int b) { return c0 + 64 * min(b, nb - 1); };
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                load_base(hold[i], column(i));
                load_w(w[i], column(i));
            }
            const bf16x8 *src =
                reinterpret_cast<const bf16x8 *>(k.u.e) + (int64_t)tile * chunks * TM;
            for (int i = threadIdx.x; i < chunks * TM; i += TH) u[i] = src[i];
            write_w(w[0], wl);
            load_w(w[0], column(2));
            __syncthreads();
            // Block b, an even one where I is 0; after: 2 where two more come, 1 one more.
            auto step = [&](auto slot, int b, auto after) {
                constexpr int I = slot();
                block_product(wl + I * size);
                store(hold[I], column(b));
                if constexpr (after() == 2) load_base(hold[I], column(b + 2));
                if constexpr (after() > 0) {
                    write_w(w[I ^ 1], wl + (I ^ 1) * size);
                    if constexpr (after() == 2) load_w(w[I ^ 1], column(b + 3));
                    __syncthreads();
                }
            };
            constexpr std::integral_constant<int, 0> zero{};
            constexpr std::integral_constant<int, 1> one{};
            constexpr std::integral_constant<int, 2> two{};
            int b = 0;
            for (; b + 3 < nb; b += 2) {
                step(zero, b, two);
                step(one, b + 1, two);
            }
            if (nb - b == 3) {
                step(zero, b, two);
                step(one, b + 1, one);
                step(zero, b + 2, zero);
            } else if (nb - b == 2) {
                step(zero, b, one);
                step(one, b + 1, zero);
            } else {
                step(zero, b, zero);
            }
        };
        if (items <= TH)
            run(std::integral_constant<int, 1>());
        else
            run(std::integral_constant<int, 2>());
    } else {
        int c = c0 + wave * 64;
        bf16x8 first[4];
        auto load_w = [&](bf16x8(&wv)[4], int c, int st) {
            const int ch = chunk_of(st);
            if constexpr (TURNED) {  // four columns of eight rank values, turned in registers
                u32x2 v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[i] = *reinterpret_cast<const u32x2 *>(we + (int64_t)(8 * ch + i) * k.N + c +
                                                            4 * m);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    u32x4 u;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        u[i] = j & 1 ? high_halves(v[2 * i][j / 2], v[2 * i + 1][j / 2])
                                     : low_halves(v[2 * i][j / 2], v[2 * i + 1][j / 2]);
                    wv[j] = __builtin_bit_cast(bf16x8, u);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    wv[j] =
                        load8(we + (int64_t)(c + j) * rank, (uint32_t)(4 * m * rank + 8 * ch) * 2);
            }
        };
        // what does not depend on u is on its way before it is cut
        if (c < c1) {
            load_base(old, c);
            load_w(first, c, 0);
        }
        // u, scaled and cut, in LDS: [chunk][row][8]
        const float f = k.scale ? k.scale[t.e] : 1.f;
        const float *pt = k.u.p + (int64_t)tile * k.u.splits * rank * TM;
        if constexpr (OWN > 0) {
            char *at = lds + chunks * 256;
            own_sums<OWN>(o, rank, t, k.x, k.a, k.K, at);
            pt = reinterpret_cast<const float *>(at);
        }
        const int splits = OWN > 0 ? kWaves : k.u.splits;
        for (int i = threadIdx.x; i < TM * (chunks - rc * (kParts - 1)); i += TH) {
            const int row = i % TM, kc = i / TM;
            bf16x8 part[kParts] = {};
            if (row < t.rows && kc < rc) {
                float v[8] = {};
                sum_splits<TM>(v, pt + 8 * kc * TM + row, rank * TM, splits);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] *= f;
                cut8(v, part);
            }
            // chunks behind the last part's are the padding
#pragma unroll
            for (int q = 0; q < kParts; ++q)
                if (kc < rc || q + 1 == kParts) u[(q * rc + kc) * 16 + row] = part[q];
        }
        __syncthreads();
        while (c < c1) {
            clear();
            product(first, 0);
            for (int st = 1; st < steps; ++st) {
                if (4 % rc == 0) {  // (rank 16: the same operands of B)
                    product(first, st);
                    continue;
                }
                bf16x8 wv[4];
                load_w(wv, c, st);
                product(wv, st);
            }
            store(old, c);
            c += WC * 64;
            if (c < c1) {
                load_base(old, c);
                load_w(first, c, 0);
            }
        }
    }
}

template <int RB, class Y, bool TURNED>
__global__ __launch_bounds__(64 * kWaves, 4) void expand_kernel(AdapterRows o, int rank,
                                                             Expand<Y> k) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    expand<RB, Y, TURNED>(o, rank, k, blockIdx.x, lds);
}

template <int OWN, class Y>
__global__ __launch_bounds__(64 * kWaves, 2) void few_kernel(AdapterRows o, int rank, Expand<Y> k) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    expand<1, Y, false, OWN>(o, rank, k, blockIdx.x, lds);
}

// ---- gradients of A and B ------------------------------------------------

// 8 x 8 values of 16 bits, rows to columns.
__device__ __forceinline__ void transpose8(const u32x4 (&in)[8], bf16x8 (&out)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {  // columns 2 j and 2 j + 1
        u32x4 lo, hi;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            lo[i] = low_halves(in[2 * i][j], in[2 * i + 1][j]);
            hi[i] = high_halves(in[2 * i][j], in[2 * i + 1][j]);
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
    int C, transposed, cb, blocks;  // cb: blocks of 512 columns
    int shares;                     // workgroups that share the rank of a block
};

// Tiles of 2^sh rows before adapter e.
__device__ __forceinline__ int tiles_before(const AdapterRows &o, int sh, int e) {
    int n = 0;
    for (int i = threadIdx.x & 63; i < e; i += 64)
        n += (max(offset_at(o, i + 1) - offset_at(o, i), 0) + (1 << sh) - 1) >> sh;
    return __builtin_amdgcn_readlane(wave_inclusive_scan(n), 63);
}

// The n-th adapter without rows, -1 if there are fewer.
__device__ __forceinline__ int empty_adapter(const AdapterRows &o, int n) {
    const int lane = threadIdx.x & 63;
    int mine = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = 4 * lane + i;
        mine += e < o.count && offset_at(o, e + 1) <= offset_at(o, e);
    }
    const int incl = wave_inclusive_scan(mine);
    const uint64_t has = __ballot(incl > n);
    if (!has) return -1;
    const int l = __builtin_ctzll(has);
    int left = n - __builtin_amdgcn_readlane(incl - mine, l);
    for (int e = 4 * l; e < min(4 * l + 4, o.count); ++e)
        if (offset_at(o, e + 1) <= offset_at(o, e) && left-- == 0) return e;
    return -1;
}

// What becomes of da and db.  kZero: workgroups behind the last tile write the zeros of
// adapters without rows (else the join does).
enum { kSet = 0, kAdd = 1, kZero = 2 };

// The contraction runs over rows, 32 an instruction.  A lane loads 8 rows x 8
// columns of q and turns them in registers: the operands of eight instructions,
// the j-th of which has column 8 (lane % 16) + j.  M is the rank.  Four waves stand
// side by side, 128 columns each, and read the same of p; two such rows of waves take
// steps of 32 rows in turn and join in LDS.  p in three parts: the sums are as exact
// as fp32's.  8192 rows, rank 32, both: 38 us for 134 MB of x and dy, 4.7 TB/s with p and
// what it writes; twice the waves with half the registers spill (75 us).  Every 16 NR rank
// values read q anew.
template <int RB, int NR>
__device__ __forceinline__ void outer(const AdapterRows &o, int rank, const float *scale, int sh,
                                      int slots, int mode, const Outer &k, int block,
                                      char *lds) {
    constexpr int TSH = tile_shift_of(RB), TM = 16 * RB, KR = kWaves / 4;
    floatx4 *sums = reinterpret_cast<floatx4 *>(lds);
    int *rows = reinterpret_cast<int *>(sums + 4 * NR * 8 * 64);
    const int share = block % k.shares, at_cb = block / k.shares % k.cb;
    const Tile t = find_tile(o, sh, block / k.shares / k.cb);
    if (t.e < 0) {
        const int e = mode == kZero ? empty_adapter(o, t.index) : -1;
        if (e < 0) return;
        const int c0 = at_cb * 512, C = min(512, k.C - c0), n = C * rank / 4;
        float *to = k.out + (int64_t)e * rank * k.C;
        for (int i = threadIdx.x + 64 * kWaves * share; i < n; i += 64 * kWaves * k.shares) {
            float *d = k.transposed ? to + (int64_t)c0 * rank + 4 * i
                                    : to + (int64_t)(i / (C / 4)) * k.C + c0 + i % (C / 4) * 4;
            *reinterpret_cast<floatx4 *>(d) = floatx4{};
        }
        return;
    }
    if (t.tiles > 1 && t.several + t.index >= slots) return;
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), cw = wave % 4, rw = wave / 4;
    const int col = (at_cb * 4 + cw) * 128 + 8 * m, qc = min(col, k.C - 8);
    const int groups = (rank + 16 * NR - 1) / (16 * NR);
    const int64_t pt = tiles_before(o, TSH, t.e) + ((int64_t)t.index << (sh - TSH));
    // (offsets out of order may count more tiles than there are sums of)
    if (pt + ((t.rows + TM - 1) >> TSH) > (o.rows >> TSH) + min((int64_t)o.count, o.rows)) return;
    const float f = scale ? scale[t.e] : 1.f;
    const bf16_t *qr = k.q + qc;
    bool none = false;
    for (int i = threadIdx.x; i < t.rows; i += 64 * kWaves) {
        rows[i] = row_at(o, t.first + i);
        none |= rows[i] < 0;
    }
    none = __syncthreads_or(none);
    // Rows of one step: the halves take groups of the rank in turn, with nothing to join.
    const bool one = RB == 1 && t.rows <= 32;
    const int from = one ? 0 : 32 * rw;
    for (int grp = share + (one ? rw * k.shares : 0); grp < groups;
         grp += k.shares * (one ? KR : 1)) {
        const int r0 = grp * 16 * NR;
        floatx4 acc[NR][8] = {};
        u32x4 raw[8];
        auto load_q = [&](int k0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t row = max(rows[min(k0 + 8 * g + i, t.rows - 1)], 0);
                raw[i] = *reinterpret_cast<const u32x4 *>(qr + row * k.C);
            }
        };
        constexpr bool AHEAD = RB > 1;  // (of few rows a wave has a step or two)
        if (AHEAD && from < t.rows) load_q(from);
        for (int k0 = from; k0 < t.rows; k0 += 32 * KR) {
            if (!AHEAD) load_q(k0);
            // p of 8 rows, in parts; behind the last row zeros
            const int at = min(k0 + 8 * g, (t.rows - 1) & ~7);
            const int64_t tile = pt + (at >> TSH);
            floatx4 pv[NR][RB == 1 ? 2 : 3];
#pragma unroll
            for (int b = 0; b < NR; ++b) {
                // (a rank value behind the last: another's, not stored)
                const int r = min(r0 + 16 * b + m, rank - 1);
                if constexpr (RB == 1) {
                    const float *src =
                        k.p.p + (tile * k.p.splits * rank + r) * TM + (at & (TM - 1));
                    pv[b][0] = pv[b][1] = floatx4{};
                    for (int s = 0; s < k.p.splits; ++s)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            pv[b][h] += *reinterpret_cast<const floatx4 *>(
                                src + (int64_t)s * rank * TM + 4 * h);
                } else {
                    const bf16_t *src = k.p.q + (tile * 3 * rank + r) * TM + (at & (TM - 1));
#pragma unroll
                    for (int s = 0; s < 3; ++s)
                        pv[b][s] = *reinterpret_cast<const floatx4 *>(src + s * rank * TM);
                }
            }
            if (none) {  // (p has zeros for those: for an infinity of row 0's)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (rows[min(k0 + 8 * g + i, t.rows - 1)] < 0) raw[i] = u32x4{};
            }
            bf16x8 qv[8];
            transpose8(raw, qv);
            if (AHEAD && k0 + 32 * KR < t.rows) load_q(k0 + 32 * KR);
            const bool tail = k0 + 32 > t.rows;
#pragma unroll
            for (int b = 0; b < NR; ++b) {
                bf16x8 part[3];
                if constexpr (RB == 1) {
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        v[i] = k0 + 8 * g + i < t.rows &&
                                       !(none && rows[k0 + 8 * g + i] < 0)
                                   ? pv[b][i / 4][i % 4] * f
                                   : 0.f;
                    cut8(v, part);
                } else {
                    // (a tile's rows behind its last are zeros; eights behind that: no tile's)
#pragma unroll
                    for (int s = 0; s < 3; ++s) part[s] = __builtin_bit_cast(bf16x8, pv[b][s]);
                    if (tail) {
#pragma unroll
                        for (int s = 0; s < 3; ++s)
                            if (k0 + 8 * g >= t.rows) part[s] = bf16x8{};
                    }
                }
#pragma unroll
                for (int s = 0; s < 3; ++s)
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[b][j] = mfma(part[s], qv[j], acc[b][j]);
            }
        }
        if (!one) {
            floatx4 *mine = sums + cw * NR * 8 * 64 + lane;
            if (rw == 1) {
#pragma unroll
                for (int b = 0; b < NR; ++b)
#pragma unroll
                    for (int j = 0; j < 8; ++j) mine[(b * 8 + j) * 64] = acc[b][j];
            }
            __syncthreads();
            if (rw == 0) {
#pragma unroll
                for (int b = 0; b < NR; ++b)
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[b][j] += mine[(b * 8 + j) * 64];
            }
            __syncthreads();
        }
        if ((one || rw == 0) && col < k.C) {
            const bool whole = t.tiles == 1, add = whole && mode == kAdd;
            float *to = whole ? k.out + (int64_t)t.e * rank * k.C
                              : k.parts + (int64_t)(t.several + t.index) * rank * k.C;
#pragma unroll
            for (int b = 0; b < NR; ++b) {
                const int r = r0 + 16 * b + 4 * g;
                if (r >= rank) continue;
                if (k.transposed) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        floatx4 *d =
                            reinterpret_cast<floatx4 *>(to + (int64_t)(col + j) * rank + r);
                        *d = add ? *d + acc[b][j] : acc[b][j];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const floatx4 v = {acc[b][4 * h][i], acc[b][4 * h + 1][i],
                                               acc[b][4 * h + 2][i], acc[b][4 * h + 3][i]};
                            floatx4 *d = reinterpret_cast<floatx4 *>(
                                to + (int64_t)(r + i) * k.C + col + 4 * h);
                            *d = add ? *d + v : v;
                        }
                }
            }
        }
    }
}

// The gradient's products behind u and v: blocks of db, then of da.
template <int RB, int NR>
__global__ __launch_bounds__(64 * kWaves) void outer_kernel(AdapterRows o, int rank,
                                                                 const float *scale, int sh,
                                                                 int slots, int mode,
                                                                 Outer kb, Outer ka) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int b = blockIdx.x;
    outer<RB, NR>(o, rank, scale, sh, slots, mode, b < kb.blocks ? kb : ka,
                  b < kb.blocks ? b : b - kb.blocks, lds);
}

// Of few rows: those and the blocks of dx in one launch.
template <int NR, class Y>
__global__ __launch_bounds__(64 * kWaves, NR == 1 ? 4 : 2) void back_kernel(
    AdapterRows o, int rank, const float *scale, int sh, int slots, int mode, Outer kb,
    Outer ka, Expand<Y> kx) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int b = blockIdx.x;
    if (b < kb.blocks + ka.blocks)
        outer<1, NR>(o, rank, scale, sh, slots, mode, b < kb.blocks ? kb : ka,
                     b < kb.blocks ? b : b - kb.blocks, lds);
    else
        expand<1, Y, true>(o, rank, kx, b - kb.blocks - ka.blocks, lds);
}

// Adapters of several tiles: their parts, added in order; adapters of no rows:
// zeros (nothing where out accumulates).  blockIdx.z: da, db.  8192 rows, rank 32: 5.5 us,
// 18 MB of parts; larger tiles have fewer of them and leave compute units idle.
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
        const float *src = k.parts + before * size + i;
        floatx4 v = {};
        int j = 0;
        for (; j + 4 <= n; j += 4) {
            floatx4 w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                w[q] = *reinterpret_cast<const floatx4 *>(src + (j + q) * size);
#pragma unroll
            for (int q = 0; q < 4; ++q) v += w[q];
        }
        for (; j < n; ++j) v += *reinterpret_cast<const floatx4 *>(src + j * size);
        floatx4 *d = reinterpret_cast<floatx4 *>(k.out + (int64_t)e * size + i);
        *d = accumulate ? *d + v : v;
    }
}

// ---- launches --------------------------------------------------------------

// Tiles of 2^sh rows that `count` adapters can have.
int64_t tile_cap(int64_t rows, int count, int sh) {
    return (rows >> sh) + std::min<int64_t>(count, rows);
}
// Rows from which on tiles are tall.  Those read the adapters' matrices less often and
// rows as whole lines, and take two launches more, some 12 us: worth it from so many
// values of rows and outputs on, in the gradient the earlier the larger the rank, where
// the adapters' mean rows fill half a tile and u's parts of a tile fit LDS.  us, short and
// tall: rank 32, 4096 x 4096, 1800 rows 29 and 31, 3000 rows 42 and 36 (2100 rows, where
// short tiles just need a round more, 38 and 32); 1024 x 2048, 3000 rows 21 and 25, 6000
// rows 33 and 34, 8200 rows 45 and 37.  The gradient: 4096 x 4096, rank 16, 3000 rows 56
// and 59, 6200 rows 104 and 91; rank 128, 1600 rows 158 and 128, 3000 rows 222 and 151.
// Ranks above 128 have short tiles only: rank 256, 8192 rows 344, the gradient 857.
constexpr int64_t kTallValues = 18 << 20, kTallWork = 1 << 30;
int64_t tall_from(const moe_adapters &ad, bool back) {
    if (ad.rank > 128) return std::numeric_limits<int64_t>::max();
    const int64_t width = (int64_t)ad.n + ad.k, work = width * (ad.rank + 24);
    return std::max<int64_t>((int64_t)64 * ad.count, back ? (kTallWork + work - 1) / work
                                                          : (kTallValues + width - 1) / width);
}
// Row blocks of 16 of a tile.
int row_blocks(int64_t rows, const moe_adapters &ad, bool back) {
    return rows >= tall_from(ad, back) ? 8 : 1;
}

// Values of x and A that every workgroup of expand reads itself (own_sums) rather than a
// launch before it, at most: y of 4096 columns, rank 16, with and without it, us in a
// graph: one row of 4096 k 8.4 and 8.9 (called one by one 8.5 and 11.0), of 8192 k 11.4
// and 9.9; 100 rows of 1024 k 8.2 and 9.8.
constexpr int64_t kFewValues = 98304;

int64_t tile_count(const AdapterRows &o) {
    return tile_cap(o.rows, o.count, tile_shift_of(o.blocks));
}
// Rows of a tile of the outer products, as a power of two: about 16 tiles, which with
// some 16 column blocks fill the chip; up to 256 rows of several adapters a tile holds
// any adapter's, which saves the join (200 rows of 8, rank 32: 17.6 -> 15.7 us; of one
// adapter 21.3 -> 22.5).
int outer_shift(int64_t rows, int count) {
    return rows >= 4096 ? 9 : rows >= 2048 || (rows <= 256 && rows > 128 && count > 1) ? 8 : 7;
}
int64_t outer_slots(int64_t rows, int count) {
    return 2 * (rows >> outer_shift(rows, count)) + 2;
}

template <int N>
using Int = std::integral_constant<int, N>;
// More than 64 KB of LDS are asked for.
hipError_t allow_lds(const void *fn, size_t lds) {
    return lds > 65536 ? hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)lds)
                       : hipSuccess;
}

// a, and b unless it has no tiles; a's w is turned where TURNED.
template <bool TURNED>
hipError_t launch_shrink(const AdapterRows &o, int rank, const float *scale, const Shrink &a,
                         const Shrink &b, hipStream_t s) {
    auto go = [&](auto rb, auto nr) {
        const int groups = rb() > 1 ? 1 : (rank + 16 * nr() - 1) / (16 * nr());
        const int na = a.tiles * a.out.splits * groups, nb = b.tiles * b.out.splits * groups;
        const size_t lds = rb() > 1 ? TallShrink<rb(), nr()>::LDS
                                    : (size_t)shrink_waves(1) / 2 * nr() * 64 * sizeof(floatx4);
        const auto fn = shrink_kernel<rb(), nr(), TURNED>;
        if (hipError_t e = allow_lds((const void *)fn, lds)) return e;
        fn<<<(unsigned)(na + nb), 64 * shrink_waves(rb()), lds, s>>>(o, rank, scale, a, b, na);
        if (hipError_t e = hipGetLastError()) return e;
        if (rb() > 1 && std::max(a.out.splits, b.out.splits) > 1) {
            cut_kernel<8><<<(unsigned)(a.tiles + b.tiles), 512, 0, s>>>(o, rank, scale, a, b);
            return hipGetLastError();
        }
        return hipSuccess;
    };
    if (o.blocks == 8)  // one pass over the rows
        return rank <= 16   ? go(Int<8>(), Int<1>())
               : rank <= 32 ? go(Int<8>(), Int<2>())
               : rank <= 64 ? go(Int<8>(), Int<4>())
                            : go(Int<8>(), Int<8>());
    if (rank <= 16) return go(Int<1>(), Int<1>());
    // (a turned w of more needs its registers: 1000 rows of rank 64 27 us, so 21)
    if constexpr (TURNED)
        return go(Int<1>(), Int<2>());
    else
        return rank <= 32 ? go(Int<1>(), Int<2>()) : go(Int<1>(), Int<4>());
}

template <class Y>
Expand<Y> make_expand(const AdapterRows &o, int rank, int N, const AdapterSums &u, const bf16_t *w,
                      const float *scale, const void *base, void *y) {
    Expand<Y> k{};
    k.u = u, k.w = w, k.scale = scale, k.base = (const Y *)base, k.y = (Y *)y;
    k.N = N, k.span = kExpandSpan;
    k.tiles = (int)tile_count(o);
    k.copies = base == y ? 0 : (int)((o.rows + 63) / 64);
    k.ranges = (N / 64 + k.span - 1) / k.span;
    return k;
}
size_t expand_lds(const AdapterRows &o, int rank) {
    const int rb = o.blocks;
    const size_t u = (size_t)rb * chunks_of(rank) * 256;
    return rb > 1 ? u + (size_t)2 * 4 * (rank / 8) * kPitch * 16 : u;  // and B's two blocks
}
template <class Y>
unsigned expand_blocks(const Expand<Y> &k) {
    return (unsigned)((int64_t)(k.tiles + k.copies) * k.ranges);
}

template <bool TURNED, class Y>
hipError_t launch_expand(const AdapterRows &o, int rank, const Expand<Y> &k, hipStream_t s) {
    const size_t lds = expand_lds(o, rank);
    const auto fn = o.blocks == 8 ? expand_kernel<8, Y, TURNED>
                                                           : expand_kernel<1, Y, TURNED>;
    if (hipError_t e = allow_lds((const void *)fn, lds)) return e;
    fn<<<expand_blocks(k), 64 * kWaves, lds, s>>>(o, rank, k);
    return hipGetLastError();
}
template <bool TURNED>
hipError_t launch_expand(const AdapterRows &o, int rank, int N, const AdapterSums &u,
                         const bf16_t *w, const float *scale, const void *base, void *y, int type,
                         hipStream_t s) {
    auto go = [&](auto zero) {
        using Y = decltype(zero);
        return launch_expand<TURNED>(o, rank, make_expand<Y>(o, rank, N, u, w, scale, base, y), s);
    };
    return type == MOE_FP32 ? go(float()) : go(bf16_t());
}

// Whether every workgroup of expand has its sums itself: few values, and one workgroup a
// compute unit.
bool few_rows(const AdapterRows &o, const moe_adapters &ad) {
    const int64_t tiles = tile_count(o);
    const int64_t ranges = (ad.n / 64 + kExpandSpan - 1) / kExpandSpan;
    return o.blocks == 1 && ad.rank <= 32 &&
           (ad.rank + std::min<int64_t>(o.rows, 16)) * ad.k <= kFewValues && tiles * ranges <= 256;
}
template <class Y>
hipError_t launch_few(const AdapterRows &o, const moe_adapters &ad, const bf16_t *x,
                      const void *base, void *y, const AdapterSums &u, hipStream_t s) {
    auto k = make_expand<Y>(o, ad.rank, ad.n, u, ad.b, ad.scale, base, y);
    k.x = x, k.a = ad.a, k.K = ad.k;
    auto go = [&](auto nr) {
        const size_t lds = expand_lds(o, ad.rank) + OwnSums<nr()>::LDS;
        const auto fn = few_kernel<nr(), Y>;
        if (hipError_t e = allow_lds((const void *)fn, lds)) return e;
        fn<<<expand_blocks(k), 64 * kWaves, lds, s>>>(o, ad.rank, k);
        return hipGetLastError();
    };
    return ad.rank <= 16 ? go(Int<1>()) : go(Int<2>());
}

// The sums of half the waves, and the rows of a tile.
size_t outer_lds(int nr) { return (size_t)4 * nr * 8 * 64 * sizeof(floatx4) + 512 * sizeof(int); }

// Blocks of the outer products, which share the rank where they are few; returns the
// rank blocks of a wave.  100 rows of one adapter, rank 128: the gradient 72 us where a
// workgroup has all of the rank, 21 so; 64 adapters of them, rank 64: 78 with two rank
// blocks a wave, 66 with one.
constexpr int kOuterBlocks = 512;
int size_outer(const AdapterRows &o, int rank, Outer &ka, Outer &kb) {
    // (of adapters without rows too)
    const int sh = outer_shift(o.rows, o.count);
    const int tiles = (int)std::max<int64_t>(tile_cap(o.rows, o.count, sh), o.count);
    const int blocks = tiles * (ka.cb + kb.cb);
    const int most = (rank + 15) / 16;
    // one rank block a wave where that makes no more workgroups than are at home at once,
    // or where adapters have a step of rows (more waves at a time)
    const int nr =
        most == 1 || (o.blocks == 1 && (blocks * most <= kOuterBlocks || o.rows <= 32 * o.count))
            ? 1
            : 2;
    const int groups = (most + nr - 1) / nr;
    ka.shares = kb.shares = std::max(1, std::min(groups, kOuterBlocks / blocks));
    ka.blocks = tiles * ka.cb * ka.shares;
    kb.blocks = tiles * kb.cb * kb.shares;
    return nr;
}

hipError_t launch_outer(const AdapterRows &o, int rank, const float *scale, int mode,
                        Outer kb, Outer ka, hipStream_t s) {
    const int sh = outer_shift(o.rows, o.count), slots = (int)outer_slots(o.rows, o.count);
    const int nr = size_outer(o, rank, ka, kb);
    auto go = [&](auto rb, auto nr) {
        const auto fn = outer_kernel<rb(), nr()>;
        const size_t lds = outer_lds(nr());
        if (hipError_t e = allow_lds((const void *)fn, lds)) return e;
        fn<<<(unsigned)(ka.blocks + kb.blocks), 64 * kWaves, lds, s>>>(o, rank, scale, sh, slots,
                                                                       mode, kb, ka);
        return hipGetLastError();
    };
    if (o.blocks == 8) return nr == 1 ? go(Int<8>(), Int<1>()) : go(Int<8>(), Int<2>());
    return nr == 1 ? go(Int<1>(), Int<1>()) : go(Int<1>(), Int<2>());
}

template <class Y>
hipError_t launch_short(const AdapterRows &o, const moe_adapters &ad, const AdapterBack &k,
                        int mode, Outer kb, Outer ka, hipStream_t s) {
    const int sh = outer_shift(o.rows, o.count), slots = (int)outer_slots(o.rows, o.count);
    const int rank = ad.rank, nr = size_outer(o, rank, ka, kb);
    const auto kx = make_expand<Y>(o, rank, ad.k, k.v, ad.a, ad.scale, k.base, k.dx);
    auto go = [&](auto nr) {
        const auto fn = back_kernel<nr(), Y>;
        const size_t lds = std::max(outer_lds(nr()), expand_lds(o, rank));
        if (hipError_t e = allow_lds((const void *)fn, lds)) return e;
        fn<<<ka.blocks + kb.blocks + expand_blocks(kx), 64 * kWaves, lds, s>>>(
            o, rank, ad.scale, sh, slots, mode, kb, ka, kx);
        return hipGetLastError();
    };
    return nr == 1 ? go(Int<1>()) : go(Int<2>());
}

hipError_t launch_join(const AdapterRows &o, int rank, bool accumulate, const Outer &ka,
                       const Outer &kb, hipStream_t s) {
    const int64_t size = (int64_t)rank * std::max(ka.C, kb.C);
    const unsigned bx = (unsigned)std::min<int64_t>((size + 1023) / 1024, 64);
    const int sh = outer_shift(o.rows, o.count), slots = (int)outer_slots(o.rows, o.count);
    join_kernel<<<dim3(bx, o.count, 2), 256, 0, s>>>(o, sh, slots, accumulate, ka, kb, rank);
    return hipGetLastError();
}

// Shares of K that the sums of these rows are cut into: a workgroup for every compute
// unit (twice that: 64 rows of as many adapters, 4096 x 4096, rank 64 22 us in place of 19),
// two where tiles are tall, and a step of 64 k for every wave.  together: sums in the same
// launch.
int splits_of(int64_t rows, int count, int K, int rb, int together) {
    const int64_t tiles = std::max<int64_t>(tile_cap(rows, count, tile_shift_of(rb)), 1);
    const int64_t want = rb > 1 ? 512 / tiles / together : (256 + tiles - 1) / tiles;
    const int64_t most = std::max(1, K / 64 / 4);
    return (int)std::max<int64_t>(1, std::min({want, most, (int64_t)kMostSplits}));
}

// Blocks of 512 threads at most that a launch of expand, or of outer over both
// matrices, has.
int64_t expand_cap(int64_t rows, int64_t tiles, int N) {
    return (tiles + (rows + 63) / 64) * ((N / 64 + kExpandSpan - 1) / kExpandSpan);
}
int64_t outer_cap(int64_t rows, int count, int n, int k) {
    return std::max<int64_t>(tile_cap(rows, count, outer_shift(rows, count)), count) *
           ((n + 511) / 512 + (k + 511) / 512);
}

size_t up(size_t v) { return (v + 255) & ~size_t(255); }

// Bytes of a shrink's sums and their parts (e, q), for these rows.
struct SumsSize {
    size_t p, e, q;
};
SumsSize sums_size(int64_t rows, int count, int rank, int rb) {
    const int sh = tile_shift_of(rb);
    const int64_t tiles = tile_cap(rows, count, sh);
    // no more than splits * tiles of any K
    const int64_t sums = std::max(tiles, std::min<int64_t>(kMostSplits * tiles, 512));
    SumsSize z{up((size_t)sums * rank * sizeof(float) << sh), 0, 0};
    if (rb > 1) {
        z.e = up((size_t)tiles * chunks_of(rank) * 16 << sh);
        z.q = up((size_t)tiles * kParts * rank * sizeof(bf16_t) << sh);
    }
    return z;
}

}  // namespace

bool adapter_launches_fit(int64_t rows, const moe_adapters &ad) {
    const int rb = std::min(row_blocks(rows, ad, false), row_blocks(rows, ad, true));
    const int64_t tiles = tile_cap(rows, ad.count, tile_shift_of(rb));
    // two sums' blocks, those of few tiles in several shares of K
    const int64_t shrink = std::max<int64_t>(tiles, 1024) * 2 * ((ad.rank + 31) / 32);
    const int64_t both = expand_cap(rows, tiles, std::max(ad.n, ad.k)) +
                         outer_cap(rows, ad.count, ad.n, ad.k);
    return std::max(shrink, both) * 64 * kWaves < int64_t(1) << 32;
}

AdapterRows adapter_tiles(AdapterRows o, const moe_adapters &ad, bool back) {
    o.blocks = row_blocks(o.rows, ad, back);
    return o;
}

size_t adapter_sums_bytes(int64_t rows, const moe_adapters &ad, bool back) {
    auto bytes = [&](int64_t r, int rb) {
        const SumsSize z = sums_size(r, ad.count, ad.rank, rb);
        return z.p + z.e + z.q;
    };
    const int64_t edge = tall_from(ad, back);
    return rows >= edge ? std::max(bytes(rows, 8), bytes(edge - 1, 1)) : bytes(rows, 1);
}

AdapterSums adapter_sums(const AdapterRows &o, int rank, int K, int together, void *at) {
    const SumsSize z = sums_size(o.rows, o.count, rank, o.blocks);
    char *p = (char *)at;
    return {(float *)p, splits_of(o.rows, o.count, K, o.blocks, together), (bf16_t *)(p + z.p),
            (bf16_t *)(p + z.p + z.e)};
}

size_t adapter_parts_bytes(int64_t rows, int rank, int C) {
    int64_t most = outer_slots(rows, 1);
    for (int64_t r : {2047, 4095})  // the last rows of each tile height
        if (r < rows) most = std::max(most, outer_slots(r, 1));
    return (size_t)most * rank * C * sizeof(float);
}

hipError_t launch_adapter_rows(const AdapterRows &o, const moe_adapters &ad, const bf16_t *x,
                               const void *base, void *y, int y_type, const AdapterSums &u,
                               hipStream_t s) {
    if (few_rows(o, ad))
        return y_type == MOE_FP32 ? launch_few<float>(o, ad, x, base, y, u, s)
                                  : launch_few<bf16_t>(o, ad, x, base, y, u, s);
    const Shrink ku{x, ad.a, u, ad.k, (int)tile_count(o), Cut{true, false}};
    if (hipError_t e = launch_shrink<false>(o, ad.rank, ad.scale, ku, Shrink{}, s)) return e;
    return launch_expand<false>(o, ad.rank, ad.n, u, ad.b, ad.scale, base, y, y_type, s);
}

hipError_t launch_adapter_backward(const AdapterRows &o, const moe_adapters &ad,
                                   const AdapterBack &k, hipStream_t s) {
    const Outer ka{k.v, k.x, k.pa, k.da, ad.k, 0, (ad.k + 511) / 512, 0, 1};
    const Outer kb{k.u, k.dy, k.pb, k.db, ad.n, 1, (ad.n + 511) / 512, 0, 1};
    // a tile an adapter at most: nothing to join
    const bool joins = o.rows == 0 || o.rows > (int64_t)1 << outer_shift(o.rows, o.count);
    const int mode = k.accumulate ? kAdd : joins ? kSet : kZero;
    if (o.rows) {
        // v = B^T dy, and for db u = A x
        const int tiles = (int)tile_count(o);
        const Cut cv{k.dx != nullptr, k.da != nullptr};
        const Shrink kv{k.dy, ad.b, k.v, ad.n, tiles, cv};
        const Shrink ku = k.da ? Shrink{k.x, ad.a, k.u, ad.k, tiles, Cut{false, true}} : Shrink{};
        if (hipError_t e = launch_shrink<true>(o, ad.rank, ad.scale, kv, ku, s)) return e;
        if (k.dx && k.da && o.blocks == 1) {
            // few rows: one launch for the three products
            if (hipError_t e = k.dx_type == MOE_FP32
                                   ? launch_short<float>(o, ad, k, mode, kb, ka, s)
                                   : launch_short<bf16_t>(o, ad, k, mode, kb, ka, s))
                return e;
        } else {
            if (k.dx)
                if (hipError_t e = launch_expand<true>(o, ad.rank, ad.k, k.v, ad.a, ad.scale,
                                                       k.base, k.dx, k.dx_type, s))
                    return e;
            if (k.da)
                if (hipError_t e = launch_outer(o, ad.rank, ad.scale, mode, kb, ka, s))
                    return e;
        }
    }
    return k.da && joins ? launch_join(o, ad.rank, k.accumulate, ka, kb, s) : hipSuccess;
}

}  // namespace moe
