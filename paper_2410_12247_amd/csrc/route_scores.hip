// Routing by scores: softmax or sigmoid of given logits, a bias for the choice,
// groups of experts, the k best and their weights; and its gradient.
#include <cmath>

#include "route_common.h"

namespace moe {
namespace {

constexpr int kTokens = 4;  // of a workgroup: one a wave

__device__ __forceinline__ float logit_at(const float *z, int64_t i) { return z[i]; }
__device__ __forceinline__ float logit_at(const bf16_t *z, int64_t i) {
    return __uint_as_float((uint32_t)z[i] << 16);
}

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

// fp64 exp of the argument, 0 for -inf.
__device__ __forceinline__ double exp64(double v) { return exp(v); }

// The weights of a token's chosen experts, by lanes 0 .. k - 1 (e < 0: no
// expert); z_at the lane's chosen logit, zmax and sum the softmax's over all.
__device__ __forceinline__ double chosen_weight(bool sigmoid, bool renorm, bool there, float z_at,
                                                float zmax, double sum) {
    if (!renorm) {
        if (!there) return 0.0;
        return sigmoid ? 1.0 / (1.0 + exp64(-(double)z_at)) : exp64((double)z_at - zmax) / sum;
    }
    // relative to the largest, so that no sum is 0
    const float v = sigmoid ? fminf(z_at, 0.f) : z_at;
    const uint32_t key = there ? (uint32_t)(logit_key(v, 0) >> 32) : 0u;
    const uint32_t top = wave_max_u32(key);
    const float m = key_logit((uint64_t)top << 32);
    double s = 0.0;
    if (there) {
        s = exp64((double)v - m);
        if (sigmoid) s /= 1.0 + exp64(-fabs((double)z_at));
    }
    const double S = wave_sum_f64(s);
    return there ? s / S : 0.0;
}

// One wave a token; lane l has experts l, l + 64, l + 128, l + 192.
template <class Z>
__global__ __launch_bounds__(64 * kTokens) void scores_kernel(
    const Z *__restrict__ z, const float *__restrict__ bias, int64_t T, int E, int k, int sigmoid,
    int renorm, int G, int top_groups, int pair, float scale, int32_t *__restrict__ ids,
    float *__restrict__ w) {
    __shared__ double cs[kTokens][kMaxExperts], gs[kTokens][kMaxExperts];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t t = (int64_t)blockIdx.x * kTokens + wave;
    const bool live = t < T;
    float zl[4];
    uint32_t top = 0;
    bool bad = false;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int e = lane + 64 * q;
        zl[q] = live && e < E ? logit_at(z, t * E + e) : -INFINITY;
        bad |= zl[q] != zl[q] || (!sigmoid && zl[q] == INFINITY);
        top = max(top, (uint32_t)(logit_key(zl[q], 0) >> 32));
    }
    const bool broken = __ballot(bad) != 0;
    const float zmax = key_logit((uint64_t)wave_max_u32(top) << 32);
    double s[4], sum = 0.0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        s[q] = zl[q] == -INFINITY ? 0.0
               : sigmoid          ? 1.0 / (1.0 + exp64(-(double)zl[q]))
                                  : exp64((double)zl[q] - zmax);
        sum += s[q];
    }
    sum = wave_sum_f64(sum);
    uint64_t key[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int e = lane + 64 * q;
        double c = sigmoid ? s[q] : s[q] / sum;
        if (bias && e < E) c += (double)bias[e];
        if (zl[q] == -INFINITY || c != c) c = -INFINITY;
        if (e < E) cs[wave][e] = c;
        // a token with a NaN: by the logits, a NaN as the largest
        key[q] = broken ? logit_choice_key(zl[q] != zl[q] ? INFINITY : zl[q])
                 : bias ? choice_key(c)
                        : logit_choice_key(zl[q]);
    }
    if (G > 1) {
        const int size = E / G;
        __syncthreads();
        for (int g = lane; g < G; g += 64) {
            double a = -INFINITY, b = -INFINITY;
            for (int i = 0; i < size; ++i) {
                const double c = cs[wave][g * size + i];
                if (c > a) b = a, a = c;
                else if (c > b) b = c;
            }
            gs[wave][g] = pair && b > -INFINITY ? a + b : a;
        }
        __syncthreads();
        if (!broken) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int e = lane + 64 * q;
                if (e >= E) continue;
                const int g = e / size;
                const double v = gs[wave][g];
                int better = 0;
                for (int i = 0; i < G; ++i) {
                    const double o = gs[wave][i];
                    better += o > v || (o == v && i < g);
                }
                if (better >= top_groups) key[q] = 0;
            }
        }
    }
    float my_z = 0.f;
    int my_e = -1;
    for (int j = 0; j < k; ++j) {
        const uint64_t best = wave_max_u64(
            max_u64(max_u64(key[0], key[1]), max_u64(key[2], key[3])));
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
    double v = chosen_weight(sigmoid, renorm, my_e >= 0, my_z, zmax, sum) * scale;
    if (broken) v = NAN;
    if (live && lane < k) {
        ids[t * k + lane] = my_e;
        w[t * k + lane] = (float)v;
    }
}

__device__ __forceinline__ void store_logit(float *z, int64_t i, float v) { z[i] = v; }
__device__ __forceinline__ void store_logit(bf16_t *z, int64_t i, float v) {
    z[i] = __builtin_bit_cast(uint16_t, (__bf16)v);
}

// dz of a token, by one wave.  Lane j < k works out the chosen expert j's part:
//   softmax over all     dz_e = s_e (sum over j with id e of G_j - D), D = sum G_j s_j
//   softmax, renormalised dz_j = p_j (G_j - sum G p)      p: softmax over the chosen
//   sigmoid              dz_j = G_j s (1 - s)
//   sigmoid, renormalised dz_j = q_j (1 - s_j) (G_j - sum G q)   q: s over their sum
// with G = scale dw.
template <class Z>
__global__ __launch_bounds__(64 * kTokens) void scores_back_kernel(
    const Z *__restrict__ z, const int32_t *__restrict__ ids, const float *__restrict__ dw,
    int64_t T, int E, int k, int sigmoid, int renorm, float scale, Z *__restrict__ dz) {
    const int lane = threadIdx.x & 63;
    const int64_t t = (int64_t)blockIdx.x * kTokens + (threadIdx.x >> 6);
    if (t >= T) return;
    const bool all = !sigmoid && !renorm;
    float zl[4] = {};
    double s[4] = {}, sum = 1.0;
    float zmax = 0.f;
    if (all) {
        uint32_t top = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int e = lane + 64 * q;
            zl[q] = e < E ? logit_at(z, t * E + e) : -INFINITY;
            top = max(top, (uint32_t)(logit_key(zl[q], 0) >> 32));
        }
        zmax = key_logit((uint64_t)wave_max_u32(top) << 32);
        double part = 0.0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            s[q] = zl[q] == -INFINITY ? 0.0 : exp64((double)zl[q] - zmax);
            part += s[q];
        }
        sum = wave_sum_f64(part);
        if (sum == 0.0) sum = 1.0;  // every expert switched off: all s are 0
    }
    int id = lane < k ? ids[t * k + lane] : -1;
    if (id >= E) id = -1;
    const bool there = id >= 0;
    const double G = there ? (double)dw[t * k + lane] * scale : 0.0;
    const float zj = there ? logit_at(z, t * E + id) : 0.f;
    double p = chosen_weight(sigmoid, renorm, there, zj, zmax, sum), c;
    if (sigmoid) {
        const double rest = 1.0 / (1.0 + exp64((double)zj));  // 1 - s
        c = renorm ? p * rest * (G - wave_sum_f64(G * p)) : G * p * rest;
    } else {
        const double D = wave_sum_f64(G * p);
        c = renorm ? p * (G - D) : G * p;
        if (all) {
#pragma unroll
            for (int q = 0; q < 4; ++q) s[q] = -(s[q] / sum) * D;
        }
    }
    if (!there) c = 0.0;
    double v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = all ? s[q] : 0.0;
    for (int j = 0; j < k; ++j) {
        const int e = __builtin_amdgcn_readlane(id, j);
        const double cj =
            __builtin_bit_cast(double, readlane64(__builtin_bit_cast(uint64_t, c), j));
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (e == lane + 64 * q) v[q] += cj;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
        if (lane + 64 * q < E) store_logit(dz, t * E + lane + 64 * q, (float)v[q]);
}

moe_status check_routing(const char *fn, const moe_dims *d, const moe_routing *r, int32_t type) {
    MOE_TRY(check_dims(d));
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

unsigned blocks(int64_t tokens) { return (unsigned)((tokens + kTokens - 1) / kTokens); }

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" {

moe_status moe_route_logits(const moe_dims *dims, const moe_bf16 *x, const float *w_router,
                            float *logits, void *stream) {
    const char *fn = "moe_route_logits";
    MOE_TRY(check_dims(dims));
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
    const moe_dims &d = *dims;
    const moe_routing &r = *routing;
    hipStream_t s = (hipStream_t)stream;
    const int sigmoid = r.score == MOE_SCORE_SIGMOID, pair = r.group_score == MOE_GROUP_TOP_TWO;
    if (logits_type == MOE_FP32)
        scores_kernel<float><<<blocks(d.tokens), 64 * kTokens, 0, s>>>(
            (const float *)logits, bias, d.tokens, d.experts, d.top_k, sigmoid, d.renormalize,
            r.groups, r.top_groups, pair, r.scale, topk_ids, topk_w);
    else
        scores_kernel<bf16_t><<<blocks(d.tokens), 64 * kTokens, 0, s>>>(
            (const bf16_t *)logits, bias, d.tokens, d.experts, d.top_k, sigmoid, d.renormalize,
            r.groups, r.top_groups, pair, r.scale, topk_ids, topk_w);
    MOE_HIP(hipGetLastError());
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
    const moe_dims &d = *dims;
    hipStream_t s = (hipStream_t)stream;
    const int sigmoid = routing->score == MOE_SCORE_SIGMOID;
    if (logits_type == MOE_FP32)
        scores_back_kernel<float><<<blocks(d.tokens), 64 * kTokens, 0, s>>>(
            (const float *)logits, topk_ids, dtopk_w, d.tokens, d.experts, d.top_k, sigmoid,
            d.renormalize, routing->scale, (float *)dlogits);
    else
        scores_back_kernel<bf16_t><<<blocks(d.tokens), 64 * kTokens, 0, s>>>(
            (const bf16_t *)logits, topk_ids, dtopk_w, d.tokens, d.experts, d.top_k, sigmoid,
            d.renormalize, routing->scale, (bf16_t *)dlogits);
    MOE_HIP(hipGetLastError());
    return MOE_OK;
}

}  // extern "C"
