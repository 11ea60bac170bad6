// Routing by scores: softmax or sigmoid of given logits, a bias for the choice,
// groups of experts, the k best and their weights; and its gradient.
#include <cmath>

#include "dispatch.h"
#include "route_common.h"

namespace moe {
namespace {

constexpr int kWaves = 4;  // of a workgroup
// From so many tokens on eight lanes have one: 65536 tokens of 256 experts 43 us against
// 53 of sixteen; fewer tokens leave waves idle.
constexpr int64_t kManyTokens = 16384;

__device__ __forceinline__ float logit_at(const float *z, int64_t i) { return z[i]; }
__device__ __forceinline__ float logit_at(const bf16_t *z, int64_t i) {
    return __uint_as_float((uint32_t)z[i] << 16);
}

struct Rules {
    int64_t T;
    int E, k, sigmoid, renorm, G, top_groups, pair;
    float scale;
    int per;          // experts of a lane
    uint32_t div_E;   // i / E = i * div_E >> 20 for i < 8 E
    uint32_t div_per; // i / per = i * div_per >> 16 for i < E
    uint32_t div_size;  // i / (E / G) likewise
    int runs;           // groups are runs of lanes
};

// ---- one token by one wave, choices in 64 bits -------------------------------

// Order-preserving bits of a choice; 0 (below every number's) for one that
// cannot be chosen: -inf or NaN.
__device__ __forceinline__ uint64_t choice_key(double c) {
    if (!(c > -INFINITY)) return 0;
    uint64_t u = __builtin_bit_cast(uint64_t, c + 0.0);  // -0 is +0
    return u >> 63 ? ~u : u | (uint64_t(1) << 63);
}

// Order-preserving bits of a logit in the high half, the same rule.
__device__ __forceinline__ uint64_t logit_choice_key(float z) {
    return z > -INFINITY ? (logit_key(z, 0) >> 32) << 32 : 0;
}

__device__ __forceinline__ uint32_t ord32(float v) { return (uint32_t)(logit_key(v, 0) >> 32); }
__device__ __forceinline__ float from_ord32(uint32_t k) { return key_logit((uint64_t)k << 32); }

// Sums and maxima over the LT lanes of a token: 8, 16 or the wave.
template <int LT>
__device__ __forceinline__ double sum_f64(double v) {
    if constexpr (LT == 64) return wave_sum_f64(v);
#pragma unroll
    for (int i = 0; i < (LT == 8 ? 3 : 4); ++i) v = v + dpp_f64(v, i);
    return v;
}
template <int LT>
__device__ __forceinline__ uint32_t max_u32(uint32_t v) {
    if constexpr (LT == 64) return wave_max_u32(v);
    v = max(v, dpp32<0xB1>(v));
    v = max(v, dpp32<0x4E>(v));
    v = max(v, dpp32<0x141>(v));
    return LT == 8 ? v : max(v, dpp32<0x140>(v));
}

// The weight of a lane's chosen expert of logit z_at, before the factor, among the
// lanes of its token (0 where there is none); zmax and sum the softmax's over all.
template <int LT>
__device__ __forceinline__ double chosen_weight(bool sigmoid, bool renorm, bool there, float z_at,
                                                float zmax, double sum) {
    // sigmoids far below 1 are exponentials: taken relative to the largest, so that
    // their sum is not 0
    const float top = renorm ? from_ord32(max_u32<LT>(there ? ord32(z_at) : 0u)) : zmax;
    const bool far = !sigmoid || (renorm && top < -80.f);
    const double x = exp(far ? (double)z_at - top : -(double)z_at);
    double s = there ? far ? x : 1.0 / (1.0 + x) : 0.0;
    if (renorm) sum = sum_f64<LT>(s);
    if (renorm || !sigmoid) s = s / sum;
    return there ? s : 0.0;
}

// By (value descending, number ascending); without a branch.
__device__ __forceinline__ int comes_before(double o, int i, double v, int mine) {
    return (int)(o > v) | ((int)(o == v) & (int)(i < mine));
}

// Bytes of exact_token's LDS.
constexpr int exact_lds(int E) { return 8 * 2 * E; }

// Some 8 us for one token: exponentials and comparisons of doubles, k rounds across the
// wave, which does those of its tokens that come here one after the other.  How many do,
// and what 65536 tokens of 256 experts then take (us, normal logits of deviation D):
//   sigmoid and a bias of 0.1, D = 1             2 in 10000       36
//   a choice beyond 4 (bias of 5, or one of -10) all             229
//   softmax and a bias of 1/256, D = 1, 0.5, 0.3 4, 12, 21%       50, 66, 82
//   no bias, D = 1, 4, 6, 8                      0, 1, 14, 38%    21, 31, 62, 93
// The last for chosen logits more than 8 below the largest; bf16 logits without a bias
// never come here for that (19).  997 tokens of 160 experts: 5.6 us, all of them here 35.
//
// Token t, lane l with experts l, l + 64, l + 128, l + 192; lds: exact_lds(E) bytes.
template <class Z>
__device__ __forceinline__ void exact_token(const Rules &r, int64_t t, const Z *__restrict__ z,
                                            const float *__restrict__ bias,
                                            int32_t *__restrict__ ids, float *__restrict__ w,
                                            void *lds) {
    const int lane = threadIdx.x & 63, E = r.E, G = r.G;
    double *cs = static_cast<double *>(lds), *gs = cs + E;  // choices, groups' values
    float zl[4];
    uint32_t top = 0;
    bool bad = false;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int e = lane + 64 * q;
        zl[q] = e < E ? logit_at(z, t * E + e) : -INFINITY;
        bad |= zl[q] != zl[q] || (!r.sigmoid && zl[q] == INFINITY);
        top = max(top, ord32(zl[q]));
    }
    const bool broken = __ballot(bad) != 0;
    const float zmax = from_ord32(wave_max_u32(top));
    double s[4], sum = 0.0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        s[q] = zl[q] == -INFINITY ? 0.0
               : r.sigmoid        ? 1.0 / (1.0 + exp(-(double)zl[q]))
                                  : exp((double)zl[q] - zmax);
        sum += s[q];
    }
    sum = wave_sum_f64(sum);
    uint64_t key[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int e = lane + 64 * q;
        double c = r.sigmoid ? s[q] : s[q] / sum;
        if (bias && e < E) c += (double)bias[e];
        if (zl[q] == -INFINITY || c != c) c = -INFINITY;
        if (e < E) cs[e] = c;
        // a token with a NaN: by the logits, a NaN as the largest
        key[q] = broken ? logit_choice_key(zl[q] != zl[q] ? INFINITY : zl[q])
                 : bias ? choice_key(c)
                        : logit_choice_key(zl[q]);
    }
    if (G > 1) {
        const int size = E / G;
        wave_sync();
        for (int g = lane; g < G; g += 64) {
            double a = -INFINITY, b = -INFINITY;
            for (int i = 0; i < size; i += 8) {  // eight reads at once
                double c[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) c[j] = cs[g * size + min(i + j, size - 1)];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const double v = i + j < size ? c[j] : -INFINITY;
                    b = v > a ? a : v > b ? v : b;
                    a = v > a ? v : a;
                }
            }
            gs[g] = r.pair && b > -INFINITY ? a + b : a;
        }
        wave_sync();
        if (!broken) {
            double v[4];
            int mine[4], better[4] = {};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                mine[q] = min(lane + 64 * q, E - 1) / size;
                v[q] = gs[mine[q]];
            }
            for (int i = 0; i < G; i += 4) {
                double o[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = gs[min(i + j, G - 1)];
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        better[q] += (int)(i + j < G) & comes_before(o[j], i + j, v[q], mine[q]);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) key[q] = better[q] >= r.top_groups ? 0 : key[q];
        }
        wave_sync();
    }
    float my_z = 0.f;
    int my_e = -1;
    for (int j = 0; j < r.k; ++j) {
        const uint64_t best =
            wave_max_u64(max_u64(max_u64(key[0], key[1]), max_u64(key[2], key[3])));
        if (best == 0) break;
        int e = -1;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint64_t m = __ballot(key[q] == best);
            if (e < 0 && m) {
                const int l = __builtin_ctzll(m);
                e = 64 * q + l;
                if (lane == l) key[q] = 0;
                const float v = __uint_as_float(
                    (uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(zl[q]), l));
                if (lane == j) my_z = v;
            }
        }
        if (lane == j) my_e = e;
    }
    double v = chosen_weight<64>(r.sigmoid, r.renorm, my_e >= 0, my_z, zmax, sum) * r.scale;
    if (broken) v = NAN;
    if (lane < r.k) {
        ids[t * r.k + lane] = my_e;
        w[t * r.k + lane] = (float)v;
    }
}

// ---- several tokens by one wave ------------------------------------------------
// A token has LT lanes (16, or 8 where there are many tokens: fewer steps across
// lanes, twice the work of one), a lane `per` experts next to each other (at most
// NV).  The rows come in as whole cache lines and change places through LDS, where a
// lane's experts are a chunk of NV + 4 floats (16-byte reads of different banks).

template <int LT, int NV>
struct alignas(16) Tokens {
    static constexpr int N = 64 / LT, PITCH = NV + 4;
    float v[64 * PITCH];
    static_assert(exact_lds(LT * NV) <= 4 * 64 * PITCH, "room for exact_token");
    // The place of element i of the tokens' N E.
    static __device__ __forceinline__ int at(const Rules &r, uint32_t i) {
        const uint32_t t = i * r.div_E >> 20, e = i - t * r.E, c = e * r.div_per >> 16;
        return (t * LT + c) * PITCH + (e - c * r.per);
    }
};

__device__ __forceinline__ void load4(const float *p, float (&v)[4]) {
    const floatx4 u = *reinterpret_cast<const floatx4 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = u[i];
}
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void load4(const bf16_t *p, float (&v)[4]) {
    const u32x2 u = *reinterpret_cast<const u32x2 *>(p);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        v[2 * i] = __uint_as_float(u[i] << 16);
        v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ uint32_t bits16(float v) {
    return __builtin_bit_cast(uint16_t, (__bf16)v);
}
__device__ __forceinline__ void store4(float *p, const float (&v)[4]) {
    *reinterpret_cast<floatx4 *>(p) = floatx4{v[0], v[1], v[2], v[3]};
}
__device__ __forceinline__ void store4(bf16_t *p, const float (&v)[4]) {
    *reinterpret_cast<u32x2 *>(p) =
        u32x2{bits16(v[0]) | bits16(v[1]) << 16, bits16(v[2]) | bits16(v[3]) << 16};
}
__device__ __forceinline__ void store1(float *p, float v) { *p = v; }
__device__ __forceinline__ void store1(bf16_t *p, float v) { *p = (uint16_t)bits16(v); }

// n logits (from src, four at a time where ALIGNED) to LDS.
template <int LT, int NV, class Z, bool ALIGNED>
__device__ __forceinline__ void tokens_in(const Rules &r, const Z *__restrict__ src, int n,
                                          Tokens<LT, NV> &q) {
    using Q = Tokens<LT, NV>;
    constexpr int IT = (NV + 3) / 4;
    const int lane = threadIdx.x & 63;
    float v[IT][4];
    if (ALIGNED && n % 4 == 0) {  // (behind the end: the last ones again)
#pragma unroll
        for (int it = 0; it < IT; ++it) load4(src + min(4 * (lane + 64 * it), n - 4), v[it]);
    } else {
#pragma unroll
        for (int it = 0; it < IT; ++it)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                v[it][j] = logit_at(src, min(4 * (lane + 64 * it) + j, n - 1));
    }
    if (r.per % 4 == 0 && r.E % 4 == 0) {
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int i = 4 * (lane + 64 * it);
            if (i < n)
                *reinterpret_cast<floatx4 *>(&q.v[Q::at(r, i)]) =
                    floatx4{v[it][0], v[it][1], v[it][2], v[it][3]};
        }
    } else {
#pragma unroll
        for (int it = 0; it < IT; ++it)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = 4 * (lane + 64 * it) + j;
                if (i < n) q.v[Q::at(r, i)] = v[it][j];
            }
    }
}

// A lane's chunk; experts it does not have get `fill`.
template <int LT, int NV>
__device__ __forceinline__ void tokens_get(const Rules &r, const Tokens<LT, NV> &q, int n,
                                           float fill, float (&v)[NV]) {
    const int lane = threadIdx.x & 63;
    const float *p = q.v + lane * Tokens<LT, NV>::PITCH;
    if constexpr (NV % 4 == 0) {
#pragma unroll
        for (int i = 0; i < NV; i += 4) {
            const floatx4 u = *reinterpret_cast<const floatx4 *>(p + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i + j] = u[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = p[i];
    }
    if (r.E == LT * NV && n == Tokens<LT, NV>::N * r.E) return;
    const int mine = min(r.per, (n > lane / LT * r.E ? r.E : 0) - lane % LT * r.per);
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = i < mine ? v[i] : fill;
}

constexpr float kLog2e = 1.4426950408889634f;

// exp of d <= 0 to some 2^-37: 2^n times a Taylor sum to the ninth power over
// |x| <= ln 2 / 2 (the next term is below 2^-37).
__device__ __forceinline__ double exp_near(double d) {
    d = fmax(d, -1000.0);
    const double n = __builtin_rint(d * 1.4426950408889634);
    const double x = fma(n, -0.6931471805599453, d);
    double s = 1.0 / 362880;
    s = fma(s, x, 1.0 / 40320);
    s = fma(s, x, 1.0 / 5040);
    s = fma(s, x, 1.0 / 720);
    s = fma(s, x, 1.0 / 120);
    s = fma(s, x, 1.0 / 24);
    s = fma(s, x, 1.0 / 6);
    s = fma(s, x, 0.5);
    s = fma(s, x, 1.0);
    s = fma(s, x, 1.0);
    return __builtin_amdgcn_ldexp(s, (int)n);
}

// Keys: 24 bits that fall with the choice above the expert, so that all differ, the
// smallest is the best and ties go to the lowest expert.  kNone and above: an expert
// that cannot be chosen.
constexpr uint32_t kNone = 0xFFFFFF00u;

// Another lane's value (no lane is off).
template <int CTRL>
__device__ __forceinline__ uint32_t lane32(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
template <int CTRL>
__device__ __forceinline__ float lane_f32(float v) {
    return __uint_as_float(lane32<CTRL>(__float_as_uint(v)));
}

__device__ __forceinline__ float dpp_f32(float v, int which) {
    switch (which) {
        case 0: return lane_f32<0xB1>(v);
        case 1: return lane_f32<0x4E>(v);
        case 2: return lane_f32<0x141>(v);
        default: return lane_f32<0x140>(v);
    }
}
template <int LT>
__device__ __forceinline__ float max_f32(float v) {
#pragma unroll
    for (int i = 0; i < (LT == 8 ? 3 : 4); ++i) v = fmaxf(v, dpp_f32(v, i));
    return v;
}
template <int LT>
__device__ __forceinline__ float sum_f32(float v) {
#pragma unroll
    for (int i = 0; i < (LT == 8 ? 3 : 4); ++i) v = v + dpp_f32(v, i);
    return v;
}
// Whether it is true on any lane of the token, and on how many.
template <int LT>
__device__ __forceinline__ uint32_t lanes_true(bool b) {
    return (uint32_t)(__ballot(b) >> (threadIdx.x & (64 - LT))) & ((1u << LT) - 1);
}

__device__ __forceinline__ void order(uint32_t &a, uint32_t &b) {
    const uint32_t lo = min(a, b), hi = max(a, b);
    a = lo;
    b = hi;
}
__device__ __forceinline__ void sort8(uint32_t (&a)[8]) {  // odd-even merge sort
    order(a[0], a[1]), order(a[2], a[3]), order(a[4], a[5]), order(a[6], a[7]);
    order(a[0], a[2]), order(a[1], a[3]), order(a[4], a[6]), order(a[5], a[7]);
    order(a[1], a[2]), order(a[5], a[6]);
    order(a[0], a[4]), order(a[1], a[5]), order(a[2], a[6]), order(a[3], a[7]);
    order(a[2], a[4]), order(a[3], a[5]);
    order(a[1], a[2]), order(a[3], a[4]), order(a[5], a[6]);
}
// a: the eight smallest of both sorted lists, sorted; ninth: the smallest left out.
__device__ __forceinline__ void merge8(uint32_t (&a)[8], const uint32_t (&b)[8], uint32_t &ninth) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        ninth = min(ninth, max(a[i], b[7 - i]));
        a[i] = min(a[i], b[7 - i]);
    }
#pragma unroll
    for (int d = 4; d >= 1; d /= 2)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!(i & d)) order(a[i], a[i + d]);
}
template <int CTRL>
__device__ __forceinline__ void merge_lanes(uint32_t (&a)[8], uint32_t &ninth) {
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = lane32<CTRL>(a[i]);
    ninth = min(ninth, lane32<CTRL>(ninth));
    merge8(a, b, ninth);
}

// A lane's eight smallest keys, sorted, and the ninth.
template <int NV>
__device__ __forceinline__ void lane_best8(const uint32_t (&key)[NV], uint32_t (&a)[8],
                                           uint32_t &ninth) {
    ninth = ~0u;
#pragma unroll
    for (int o = 0; o < NV; o += 8) {
        uint32_t b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = o + i < NV ? key[o + i < NV ? o + i : 0] : ~0u;
        sort8(b);
        if (o == 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = b[i];
        } else {
            merge8(a, b, ninth);
        }
    }
}

template <int CTRL>
__device__ __forceinline__ int above(float other, float v) {
    return lane_f32<CTRL>(other) > v ? 1 : 0;
}
// Lanes of the token with a larger value.
template <int LT>
__device__ __forceinline__ int lanes_above(float v) {
    if constexpr (LT == 8) {
        const float o = lane_f32<0x141>(v);  // the other four lanes, mirrored
        return above<0x39>(v, v) + above<0x4E>(v, v) + above<0x93>(v, v) + (o > v ? 1 : 0) +
               above<0x39>(o, v) + above<0x4E>(o, v) + above<0x93>(o, v);
    }
    return above<0x121>(v, v) + above<0x122>(v, v) + above<0x123>(v, v) + above<0x124>(v, v) +
           above<0x125>(v, v) + above<0x126>(v, v) + above<0x127>(v, v) + above<0x128>(v, v) +
           above<0x129>(v, v) + above<0x12A>(v, v) + above<0x12B>(v, v) + above<0x12C>(v, v) +
           above<0x12D>(v, v) + above<0x12E>(v, v) + above<0x12F>(v, v);
}

// How many of a token's other first eight lanes are chosen before this one, by
// (c descending, id ascending); lanes behind them keep their own number.
template <int CTRL>
__device__ __forceinline__ int before(double c, int id, double mc, int mid) {
    const uint64_t b = __builtin_bit_cast(uint64_t, c);
    const double oc = __builtin_bit_cast(
        double, (uint64_t)lane32<CTRL>((uint32_t)(b >> 32)) << 32 | lane32<CTRL>((uint32_t)b));
    const int oid = (int)lane32<CTRL>((uint32_t)id);
    return comes_before(oc, oid, mc, mid);
}
__device__ __forceinline__ int eight_rank(double c, int id, int l) {
    const uint64_t b = __builtin_bit_cast(uint64_t, c);
    const double o = __builtin_bit_cast(  // the other four, mirrored
        double, (uint64_t)lane32<0x141>((uint32_t)(b >> 32)) << 32 | lane32<0x141>((uint32_t)b));
    const int oid = (int)lane32<0x141>((uint32_t)id);
    const int n = before<0x39>(c, id, c, id) + before<0x4E>(c, id, c, id) +
                  before<0x93>(c, id, c, id) + before<0x39>(o, oid, c, id) +
                  before<0x4E>(o, oid, c, id) + before<0x93>(o, oid, c, id) +
                  comes_before(o, oid, c, id);
    return l < 8 ? n : l;
}

// The two largest of a run of lanes.
__device__ __forceinline__ void run_top2(float &x, float &y, int run) {
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (run >= 2 << i) {
            const float x2 = dpp_f32(x, i), y2 = dpp_f32(y, i);
            y = fmaxf(fminf(x, x2), fmaxf(y, y2));
            x = fmaxf(x, x2);
        }
}

// Choices in fp32 with their error's bound: a token whose choice could come out
// otherwise in 64 bits (a gap below the bound, a NaN, values out of range) is done
// again by exact_token.  Bounds, for |c| <= 4: sigmoid within 2^-22 (exponent, sum
// and reciprocal together below 4 * 2^-24), softmax within 2^-18.7 (a sum of NV terms
// by LT lanes: 35 roundings of 2^-24 at most, and the terms' own), the bias' addition
// 2^-22, the key's step 2^-23.
// Groups are best as whole runs of lanes: G divides LT, and LT the experts.
//
// 65536 tokens of 256 experts in 8 groups by two, sigmoid and bias, 8 of them: 36.4 us,
// bound by the vector units (1720 instructions a wave of eight tokens; the logits alone
// are 13 us of memory) and by the last exact tokens' 5 us.  One token a wave with all
// choices in 64 bits: 153; sixteen lanes a token: 53.  Groups that are no runs of lanes
// (200 experts in 5): 58, by the exact way 131.  997 tokens of 160: 5.8.
template <int LT, int NV, class Z, bool ALIGNED>
__global__ __launch_bounds__(64 * kWaves, 4) void scores_kernel(Rules r, const Z *__restrict__ z,
                                                             const float *__restrict__ bias,
                                                             int32_t *__restrict__ ids,
                                                             float *__restrict__ w) {
    using Q = Tokens<LT, NV>;
    __shared__ Q quads[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane % LT;
    const int64_t t0 = ((int64_t)blockIdx.x * kWaves + wave) * Q::N;
    if (t0 >= r.T) return;
    Q &q = quads[wave];
    const int n = (int)min((int64_t)Q::N, r.T - t0) * r.E;
    const int64_t t = t0 + lane / LT;
    tokens_in<LT, NV, Z, ALIGNED>(r, z + t0 * r.E, n, q);
    float b[NV];
    if (bias) {
#pragma unroll
        for (int i = 0; i < NV; ++i) b[i] = bias[min(l * r.per + i, r.E - 1)];
    }
    wave_sync();
    float v[NV];  // logits, then what the choice is by
    tokens_get(r, q, n, -INFINITY, v);
    // infinities and NaN: a sum of zeros, or not
    float odd = 0.f, zmax = v[0];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        odd = fmaf(v[i], 0.f, odd);
        zmax = fmaxf(zmax, v[i]);
    }
    zmax = max_f32<LT>(zmax);
    const bool masks = __ballot(odd != 0.f) != 0;
    // infinite, or so large that the exponent's rounding (of the size of zmax) overflows
    bool bad = !(fabsf(zmax) < 0x1p24f);
    if (masks) {
#pragma unroll
        for (int i = 0; i < NV; ++i) bad |= v[i] != v[i];
    }
    const bool groups = r.G > 1, by_score = bias || (groups && r.pair);
    double sum = 1.0;
    if (!r.sigmoid && !r.renorm) {
        sum = 0.0;
#pragma unroll
        for (int i = 0; i < NV; ++i) sum += exp_near((double)v[i] - zmax);
        sum = sum_f64<LT>(sum);
    }
    float s[NV] = {};
    if (by_score) {
        if (r.sigmoid) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                s[i] = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * v[i]));
        } else {
            float total = 0.f;
            const float far = -kLog2e * zmax;  // (its rounding is every term's)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                s[i] = __builtin_amdgcn_exp2f(fmaf(v[i], kLog2e, far));
                total += s[i];
            }
            const float f = __builtin_amdgcn_rcpf(sum_f32<LT>(total));
#pragma unroll
            for (int i = 0; i < NV; ++i) s[i] *= f;
        }
        if (bias) {
            float out = 0.f, most = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                s[i] += b[i];
                out = fmaf(s[i], 0.f, out);
                most = fmaxf(most, fabsf(s[i]));
            }
            // a bias that is no number, or out of the bounds' range; -inf is a mask
            if (__ballot(out != 0.f || !(most <= 4.f))) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    if (!(s[i] > -INFINITY)) s[i] = -INFINITY;
                    bad |= s[i] > 4.f || (s[i] < -4.f && s[i] > -INFINITY);
                }
            }
        }
        if (masks) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (v[i] == -INFINITY) s[i] = -INFINITY;
        }
    }
    bool keep = true;  // all of a lane's experts
    if (groups) {
        const int run = r.runs ? LT / r.G : 1;  // lanes of a group
        float in, out;  // the worst group kept, the best one left out
        int kept;
        if (r.runs) {
            float x = -INFINITY, y = -INFINITY;  // the two largest
            if (by_score) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    y = __builtin_amdgcn_fmed3f(x, y, s[i]);
                    x = fmaxf(x, s[i]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < NV; ++i) x = fmaxf(x, v[i]);
            }
            run_top2(x, y, run);
            if (r.pair && y > -INFINITY) x += y;
            const int rank = lanes_above<LT>(x);  // (by every lane)
            keep = x > -INFINITY && rank < r.top_groups * run;
            in = -max_f32<LT>(keep ? -x : -INFINITY);
            out = max_f32<LT>(keep ? -INFINITY : x);
            kept = __popc(lanes_true<LT>(keep));
        } else {
            // any groups: through LDS, a lane takes every LT-th; a group's value, then
            // whether it is kept, lies at its first expert
            const int size = r.E / r.G, first = lane / LT * r.E;
            float *own = q.v + lane * Q::PITCH;
            if (by_score) {
#pragma unroll
                for (int i = 0; i < NV; ++i) own[i] = s[i];
                wave_sync();
            }
            const int mine = (r.G - l + LT - 1) / LT;  // at most 32
            float low = INFINITY, high = -INFINITY;
            int n_kept = 0;
            for (int j = 0; j < mine; ++j) {
                const int at = first + (l + j * LT) * size;
                float x = -INFINITY, y = -INFINITY;
                for (int i = 0; i < size; ++i) {
                    const float c = q.v[Q::at(r, at + i)];
                    y = fmaxf(y, fminf(x, c));
                    x = fmaxf(x, c);
                }
                if (r.pair && y > -INFINITY) x += y;
                q.v[Q::at(r, at)] = x;
            }
            wave_sync();
            uint32_t keeps = 0;  // bit j: the lane's j-th group
            for (int j = 0; j < mine; ++j) {
                const float x = q.v[Q::at(r, first + (l + j * LT) * size)];
                int above = 0;
                for (int g = 0; g < r.G; ++g) above += q.v[Q::at(r, first + g * size)] > x;
                const bool k = x > -INFINITY && above < r.top_groups;
                keeps |= (uint32_t)k << j;
                n_kept += k;
                low = fminf(low, k ? x : INFINITY);
                high = fmaxf(high, k ? -INFINITY : x);
            }
            wave_sync();
            for (int j = 0; j < mine; ++j)
                q.v[Q::at(r, first + (l + j * LT) * size)] = keeps >> j & 1 ? 1.f : 0.f;
            wave_sync();
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const uint32_t e = min(l * r.per + i, r.E - 1);
                const float k = q.v[Q::at(r, first + (e * r.div_size >> 16) * size)];
                v[i] = k != 0.f ? v[i] : -INFINITY;
                s[i] = k != 0.f ? s[i] : -INFINITY;
            }
            in = -max_f32<LT>(-low);
            out = max_f32<LT>(high);
            kept = (int)sum_f32<LT>((float)n_kept);
        }
        // a group's value (two choices and their sum) is within 2^-17.5, of sigmoids
        // 2^-19.6; logits are exact
        const float gap = r.sigmoid ? 0x1p-18f : 0x1p-16f;
        bad |= out > -INFINITY && !(by_score ? in - out > gap : in > out);
        // (logits so far out that 64 bits hold the same score for several)
        if (!by_score)
            bad |= out > -INFINITY &&
                   (r.sigmoid ? out > 20.f || in < -700.f : in < zmax - 700.f);
        bad |= kept > r.top_groups * run;  // equal ones
    }
    // keys: steps below the largest, of 2^-23 for choices, of 2^-21 for logits, whose
    // differences are within half a step; bf16 logits keep their own bits
    const bool bits = !bias && sizeof(Z) == 2;
    uint32_t key[NV];
    if (bits) {
#pragma unroll
        for (int i = 0; i < NV; ++i) key[i] = 0xFFFFu - (ord32(v[i]) >> 16);
    } else {
        float top = zmax;
        if (bias) {
            top = s[0];
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                v[i] = s[i];
                top = fmaxf(top, s[i]);
            }
            top = max_f32<LT>(top);
        }
        const float step = bias ? 0x1p23f : 0x1p21f;
        top *= step;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            key[i] = (uint32_t)fminf(fmaf(v[i], -step, top), 16777214.f);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) key[i] = (key[i] << 8) + (uint32_t)(l * r.per) + i;
    if (masks || bias || !r.runs) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (v[i] == -INFINITY) key[i] = ~0u;
    }
    uint32_t a[8], ninth;
    lane_best8(key, a, ninth);
    if (groups) {
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = keep ? a[i] : ~0u;
        ninth = keep ? ninth : ~0u;
    }
    merge_lanes<0xB1>(a, ninth);
    merge_lanes<0x4E>(a, ninth);
    merge_lanes<0x141>(a, ninth);
    if constexpr (LT == 16) merge_lanes<0x140>(a, ninth);
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) mine = l == i ? a[i] : mine;
    const bool found = l < 8 && mine < kNone;
    const uint32_t e = found ? mine & 255u : 0u;
    const float z_at = r.runs ? q.v[Q::at(r, lane / LT * r.E + e)]
                              : logit_at(z, min(t, r.T - 1) * r.E + e);
    int rank = l;
    if (!bits) {
        const uint32_t gap = (bias ? (r.sigmoid ? 12u : 65u) : 4u) << 8;
        bool near = false;  // among the eight
#pragma unroll
        for (int i = 0; i < 7; ++i)
            near |= a[i + 1] - a[i] < (i < r.k && a[i + 1] < kNone ? gap : 0u);
        // the ninth may be one of the k: by itself, or by a chain of near ones
        uint32_t kth = a[7];
#pragma unroll
        for (int i = 0; i < 7; ++i) kth = r.k == i + 1 ? a[i] : kth;
        bad |= ninth < kNone && ninth - a[7] < gap && a[7] - kth < 8 * gap;
        bad |= kth >= kNone;  // fewer than k: rare, not looked into here
        if (bias && !r.sigmoid) {
            bad |= near;
        } else if (__ballot(near)) {  // the eight in 64 bits
            double c = z_at;
            if (bias) c = 1.0 / (1.0 + exp(-(double)z_at)) + (double)bias[e];
            if (!found) c = -INFINITY;
            const int id = found ? (int)e : 256 + l;
            rank = eight_rank(c, id, l);
        }
    }
    const bool there = found && rank < r.k;
    const double weight = chosen_weight<LT>(r.sigmoid, r.renorm, there, z_at, zmax, sum) * r.scale;
    bad = lanes_true<LT>(bad && t < r.T) != 0;
    if (t < r.T && l < 8 && rank < r.k && !bad) {
        ids[t * r.k + rank] = there ? (int32_t)e : -1;
        w[t * r.k + rank] = (float)weight;
    }
    const uint64_t redo = __ballot(bad);
    if (!redo) return;
    wave_sync();
#pragma unroll 1
    for (int i = 0; i < Q::N; ++i)
        if (redo >> (LT * i) & 1)
            exact_token(r, t0 + i, z, bias, ids, w, q.v);
}

// ---- gradient ---------------------------------------------------------------

template <int I>
__device__ __forceinline__ uint32_t row_lane(uint32_t v) {  // lane I of the row
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x150 + I, 0xF, 0xF, false);
}
template <int I>
__device__ __forceinline__ double row_lane_f64(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, (uint64_t)row_lane<I>((uint32_t)(b >> 32)) << 32 |
                                          row_lane<I>((uint32_t)b));
}
// fn(I) for each of the row's first eight lanes.
template <class F>
__device__ __forceinline__ void each_slot(F fn) {
    fn(std::integral_constant<int, 0>()), fn(std::integral_constant<int, 1>());
    fn(std::integral_constant<int, 2>()), fn(std::integral_constant<int, 3>());
    fn(std::integral_constant<int, 4>()), fn(std::integral_constant<int, 5>());
    fn(std::integral_constant<int, 6>()), fn(std::integral_constant<int, 7>());
}
// Sum of v over those with the same id.
__device__ __forceinline__ double same_id_sum(int id, double v) {
    double s = 0.0;
    each_slot([&](auto i) {
        const double o = row_lane_f64<i()>(v);
        const int o_id = (int)row_lane<i()>((uint32_t)id);
        s += o_id == id ? o : 0.0;
    });
    return s;
}
// Whether the lane is the first of its id.
__device__ __forceinline__ bool first_of_id(int id, int l) {
    bool first = true;
    each_slot([&](auto i) {
        const int o = (int)row_lane<i()>((uint32_t)id);  // (by all lanes: none is off)
        first &= i() >= l | o != id;
    });
    return first;
}
// Sum of p_i (g - g_i) over those i.
__device__ __forceinline__ double weighted_gaps(double p, double g) {
    double s = 0.0;
    each_slot([&](auto i) { s = fma(row_lane_f64<i()>(p), g - row_lane_f64<i()>(g), s); });
    return s;
}

// dz of four tokens.  Lane j < k of a token works out the chosen expert j's part:
//   softmax over all      dz_e = s_e (U g_e + sum p_i (g_e - g_i)) over the chosen experts
//                         i, g_i the sum of their G, U the other experts' share; at those
//                         -s_e D, D = sum G_j s_j
//   softmax, renormalised dz_j = p_j sum p_i (G_j - G_i)      p: softmax over the chosen
//   sigmoid               dz_j = G_j s (1 - s)
//   sigmoid, renormalised dz_j = q_j (1 - s_j) sum q_i (G_j - G_i)   q: s over their sum
// with G = scale dw, in 64 bits: G - D and 1 - s, which the sums stand for, would lose
// what is left of them where one expert has nearly all.  The other experts' -s_e D is
// a product of fp32 values.
// 65536 tokens of 256 experts, sigmoid: 18.5 us, 5.7 TB/s (a wave a token, without the rows
// through LDS: 53).  Softmax over all: 40, of which the exponentials in doubles, whose sum
// without the chosen ones is U, are 10 (138 MB: 27).
template <int NV, class Z, bool ALIGNED>
__global__ __launch_bounds__(64 * kWaves) void scores_back_kernel(
    Rules r, const Z *__restrict__ z, const int32_t *__restrict__ ids,
    const float *__restrict__ dw, Z *__restrict__ dz) {
    using Q = Tokens<16, NV>;
    __shared__ Q quads[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15;
    const int64_t t0 = ((int64_t)blockIdx.x * kWaves + wave) * Q::N;
    if (t0 >= r.T) return;
    Q &q = quads[wave];
    const int n = (int)min((int64_t)Q::N, r.T - t0) * r.E;
    const int64_t t = t0 + (lane >> 4);
    const bool slot = t < r.T && l < r.k;
    int id = slot ? ids[t * r.k + l] : -1;
    if (id >= r.E || id < 0) id = -1;
    const bool there = id >= 0;
    const double G = there ? (double)dw[t * r.k + l] * r.scale : 0.0;
    const float zj = there ? logit_at(z, t * r.E + id) : 0.f;
    const bool all = !r.sigmoid && !r.renorm;
    float *mine = q.v + lane * Q::PITCH;
    float s[NV];
    float zmax = 0.f;
    double sum = 1.0, rest = 0.0;
    if (all) {
        uint32_t chosen = 0;  // of the lane's experts
        each_slot([&](auto i) {
            const uint32_t at = row_lane<i()>((uint32_t)id) - (uint32_t)(l * r.per);
            chosen |= at < (uint32_t)r.per ? 1u << at : 0u;
        });
        tokens_in<16, NV, Z, ALIGNED>(r, z + t0 * r.E, n, q);
        wave_sync();
        tokens_get(r, q, n, -INFINITY, s);
        zmax = -INFINITY;
        bool nan = false;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            zmax = fmaxf(zmax, s[i]);
            nan |= s[i] != s[i];
        }
        zmax = max_f32<16>(zmax);
        const bool bad = lanes_true<16>(nan) != 0 || zmax == INFINITY;
        if (zmax == -INFINITY) zmax = 0.f;  // every expert switched off: all s are 0
        double total = 0.0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const double e = exp_near((double)s[i] - zmax);
            total += e;
            rest += chosen >> i & 1 ? 0.0 : e;
            s[i] = (float)e;
        }
        total = sum_f64<16>(total);
        sum = bad ? (double)NAN : total > 0.0 ? total : 1.0;
        rest = sum_f64<16>(rest) / sum;
    }
    const double p = chosen_weight<16>(r.sigmoid, r.renorm, there, zj, zmax, sum);
    const double D = sum_f64<16>(G * p);
    double c;
    if (all) {
        const double g = same_id_sum(id, G);
        c = p * fma(rest, g, weighted_gaps(first_of_id(id, l) ? p : 0.0, g));
    } else {
        c = r.renorm ? p * weighted_gaps(p, G) : G * p;
        if (r.sigmoid) c *= 1.0 / (1.0 + exp((double)zj));  // 1 - s
        c = same_id_sum(id, there ? c : 0.0);
    }
    const float f = all ? (float)(-D / sum) : 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) s[i] = all ? s[i] * f : 0.f;
    if constexpr (NV % 4 == 0) {
#pragma unroll
        for (int i = 0; i < NV; i += 4)
            *reinterpret_cast<floatx4 *>(mine + i) = floatx4{s[i], s[i + 1], s[i + 2], s[i + 3]};
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) mine[i] = s[i];
    }
    wave_sync();
    if (there)  // (lanes of one id write the same value)
        q.v[Q::at(r, (lane >> 4) * r.E + id)] = (float)c;
    wave_sync();
    Z *dst = dz + t0 * r.E;
    constexpr int IT = (NV + 3) / 4;
    const bool whole = r.per % 4 == 0 && r.E % 4 == 0;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        const int i = 4 * (lane + 64 * it);
        if (i >= n) continue;
        float o[4];
        if (whole) {
            const floatx4 u = *reinterpret_cast<const floatx4 *>(&q.v[Q::at(r, i)]);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = u[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = i + j < n ? q.v[Q::at(r, i + j)] : 0.f;
        }
        if (ALIGNED && i + 4 <= n) {
            store4(dst + i, o);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (i + j < n) store1(dst + i + j, o[j]);
        }
    }
}

// Sixteen lanes a token, of 2^32 in a launch.
moe_status check_tokens(const char *fn, const moe_dims *d) {
    MOE_TRY(check_dims(d));
    return d->tokens < (int64_t(1) << 28)
               ? MOE_OK
               : fail(MOE_ERR_UNSUPPORTED, "%s: 2^28 tokens or more", fn);
}

moe_status check_routing(const char *fn, const moe_dims *d, const moe_routing *r, int32_t type) {
    MOE_TRY(check_tokens(fn, d));
    if (!r) return fail(MOE_ERR_INVALID, "%s: routing is NULL", fn);
    if (r->score != MOE_SCORE_SOFTMAX && r->score != MOE_SCORE_SIGMOID)
        return fail(MOE_ERR_INVALID, "%s: score %d", fn, r->score);
    if (r->group_score != MOE_GROUP_MAX && r->group_score != MOE_GROUP_TOP_TWO)
        return fail(MOE_ERR_INVALID, "%s: group_score %d", fn, r->group_score);
    if (r->groups < 1 || d->experts % r->groups)
        return fail(MOE_ERR_INVALID, "%s: %d experts in %d groups", fn, d->experts, r->groups);
    if (r->top_groups < 1 || r->top_groups > r->groups)
        return fail(MOE_ERR_INVALID, "%s: top_groups %d outside [1, %d]", fn, r->top_groups,
                    r->groups);
    if (r->top_groups * (d->experts / r->groups) < d->top_k)
        return fail(MOE_ERR_INVALID, "%s: %d experts in the groups kept, top_k %d", fn,
                    r->top_groups * (d->experts / r->groups), d->top_k);
    if (!std::isfinite(r->scale)) return fail(MOE_ERR_INVALID, "%s: scale is not finite", fn);
    if (type != MOE_BF16 && type != MOE_FP32)
        return fail(MOE_ERR_INVALID, "%s: logits_type %d", fn, type);
    return MOE_OK;
}

moe_status check_at(const char *fn, const char *name, const void *p, uintptr_t a) {
    if (!p) return fail(MOE_ERR_INVALID, "%s: %s is NULL", fn, name);
    if ((uintptr_t)p % a)
        return fail(MOE_ERR_INVALID, "%s: %s is not %d-byte aligned", fn, name, (int)a);
    return MOE_OK;
}

Rules rules(const moe_dims &d, const moe_routing &r) {
    Rules q{};
    q.T = d.tokens;
    q.E = d.experts, q.k = d.top_k;
    q.sigmoid = r.score == MOE_SCORE_SIGMOID, q.renorm = d.renormalize;
    q.G = r.groups, q.top_groups = r.top_groups, q.pair = r.group_score == MOE_GROUP_TOP_TWO;
    q.scale = r.scale;
    return q;
}
Rules with_lanes(Rules r, int lanes) {
    r.per = (r.E + lanes - 1) / lanes;
    r.div_E = ((1u << 20) + r.E - 1) / r.E;
    r.div_per = ((1u << 16) + r.per - 1) / r.per;
    const int size = r.E / r.G;
    r.div_size = ((1u << 16) + size - 1) / size;
    r.runs = r.G == 1 || (lanes % r.G == 0 && r.E % lanes == 0);
    return r;
}

template <int N>
using Int = std::integral_constant<int, N>;
// fn(the most experts of a lane, whether four elements load at once).
template <class F>
hipError_t by_size(const Rules &r, bool aligned, F fn) {
    auto go = [&](auto nv) {
        return aligned ? fn(nv, std::true_type()) : fn(nv, std::false_type());
    };
    if (r.per <= 1) return go(Int<1>());
    if (r.per <= 4) return go(Int<4>());
    if (r.per <= 8) return go(Int<8>());
    if (r.per <= 10) return go(Int<10>());
    return go(Int<16>());
}

template <class Z>
bool aligned4(const Z *p) { return (uintptr_t)p % (4 * sizeof(Z)) == 0; }

unsigned grid_of(const Rules &r, int tokens) {  // of a wave
    return (unsigned)((r.T + kWaves * tokens - 1) / (kWaves * tokens));
}

template <class Z>
hipError_t launch_scores(Rules r, const Z *z, const float *bias, int32_t *ids, float *w,
                         hipStream_t s) {
    const bool runs16 = with_lanes(r, 16).runs;
    if (r.T >= kManyTokens && r.E > 64 && aligned4(z) && (with_lanes(r, 8).runs || !runs16)) {
        r = with_lanes(r, 8);
        auto go = [&](auto nv) {
            scores_kernel<8, nv(), Z, true><<<grid_of(r, 8), 64 * kWaves, 0, s>>>(r, z, bias, ids,
                                                                                  w);
            return hipGetLastError();
        };
        return r.per <= 16 ? go(Int<16>()) : r.per <= 20 ? go(Int<20>()) : go(Int<32>());
    }
    r = with_lanes(r, 16);
    return by_size(r, aligned4(z), [&](auto nv, auto al) {
        scores_kernel<16, nv(), Z, al()><<<grid_of(r, 4), 64 * kWaves, 0, s>>>(r, z, bias, ids, w);
        return hipGetLastError();
    });
}

template <class Z>
hipError_t launch_back(Rules r, const Z *z, const int32_t *ids, const float *dw, Z *dz,
                       hipStream_t s) {
    r = with_lanes(r, 16);
    return by_size(r, aligned4(z) && aligned4(dz), [&](auto nv, auto al) {
        scores_back_kernel<nv(), Z, al()><<<grid_of(r, 4), 64 * kWaves, 0, s>>>(r, z, ids, dw, dz);
        return hipGetLastError();
    });
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" {

moe_status moe_route_logits(const moe_dims *dims, const moe_bf16 *x, const float *w_router,
                            float *logits, void *stream) {
    const char *fn = "moe_route_logits";
    MOE_TRY(check_tokens(fn, dims));
    if (dims->tokens == 0) return MOE_OK;
    MOE_TRY(check_at(fn, "x", x, 16));
    MOE_TRY(check_at(fn, "w_router", w_router, 4));
    MOE_TRY(check_at(fn, "logits", logits, 4));
    MOE_HIP(launch_route_logits(*dims, x, w_router, logits, (hipStream_t)stream));
    return MOE_OK;
}

moe_status moe_route_scores(const moe_dims *dims, const moe_routing *routing, const void *logits,
                            int32_t logits_type, const float *bias, int32_t *topk_ids,
                            float *topk_w, void *stream) {
    const char *fn = "moe_route_scores";
    MOE_TRY(check_routing(fn, dims, routing, logits_type));
    if (dims->tokens == 0) return MOE_OK;
    MOE_TRY(check_at(fn, "logits", logits, logits_type == MOE_FP32 ? 4 : 2));
    if (bias) MOE_TRY(check_at(fn, "bias", bias, 4));
    MOE_TRY(check_at(fn, "topk_ids", topk_ids, 4));
    MOE_TRY(check_at(fn, "topk_w", topk_w, 4));
    const Rules r = rules(*dims, *routing);
    hipStream_t s = (hipStream_t)stream;
    MOE_HIP(logits_type == MOE_FP32
                ? launch_scores(r, (const float *)logits, bias, topk_ids, topk_w, s)
                : launch_scores(r, (const bf16_t *)logits, bias, topk_ids, topk_w, s));
    return MOE_OK;
}

moe_status moe_route_scores_backward(const moe_dims *dims, const moe_routing *routing,
                                     const void *logits, int32_t logits_type,
                                     const int32_t *topk_ids, const float *dtopk_w, void *dlogits,
                                     void *stream) {
    const char *fn = "moe_route_scores_backward";
    MOE_TRY(check_routing(fn, dims, routing, logits_type));
    if (dims->tokens == 0) return MOE_OK;
    const uintptr_t a = logits_type == MOE_FP32 ? 4 : 2;
    MOE_TRY(check_at(fn, "logits", logits, a));
    MOE_TRY(check_at(fn, "topk_ids", topk_ids, 4));
    MOE_TRY(check_at(fn, "dtopk_w", dtopk_w, 4));
    MOE_TRY(check_at(fn, "dlogits", dlogits, a));
    const Rules r = rules(*dims, *routing);
    hipStream_t s = (hipStream_t)stream;
    MOE_HIP(logits_type == MOE_FP32 ? launch_back(r, (const float *)logits, topk_ids, dtopk_w,
                                                  (float *)dlogits, s)
                                    : launch_back(r, (const bf16_t *)logits, topk_ids, dtopk_w,
                                                  (bf16_t *)dlogits, s));
    return MOE_OK;
}

}  // extern "C"
