// C-ABI entry points of the block-scaled 8-bit operators: argument checks,
// workspace layout, and the layer that runs them one after another.
#include <algorithm>
#include <cmath>

#include "scaled.h"

using namespace moe;

namespace {

bool width_ok(int32_t v) { return v > 0 && v % kDimAlign == 0 && v <= kMaxWidth; }
bool type_ok(int32_t t) { return t == MOE_BF16 || t == MOE_FP32; }
bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// 16-byte loads and stores of tensors, 4-byte ones of scale rows.
moe_status check_tensor(const char *fn, const char *name, const void *p, uintptr_t a = 16) {
    if (!p) return fail(MOE_ERR_INVALID, "%s: %s is NULL", fn, name);
    if (!aligned(p, a))
        return fail(MOE_ERR_INVALID, "%s: %s is not %d-byte aligned", fn, name, (int)a);
    return MOE_OK;
}
moe_status check_pair(const char *fn, const char *name, const void *q, const void *s) {
    MOE_TRY(check_tensor(fn, name, q));
    return check_tensor(fn, "a scale tensor", s, 4);
}

// Products of `rows` rows in `experts` groups: the kernels count rows and
// tiles in 32 bits.
moe_status check_product(const char *fn, int64_t rows, int64_t experts, int32_t n, int32_t k) {
    if (!width_ok(n) || !width_ok(k))
        return fail(MOE_ERR_INVALID, "%s: widths %d, %d not multiples of %d up to 2^20", fn, n, k,
                    kDimAlign);
    if (rows >= (int64_t(1) << 31))
        return fail(MOE_ERR_UNSUPPORTED, "%s: 2^31 rows or more", fn);
    if ((rows / 32 + experts + 1) * ((int64_t)n / 128 + 1) >= (int64_t(1) << 31))
        return fail(MOE_ERR_UNSUPPORTED, "%s: %lld rows of %d columns are too many tiles", fn,
                    (long long)rows, n);
    return MOE_OK;
}

int64_t row_cap(const moe_dims *d) {
    return d->tokens * std::min<int64_t>(d->top_k, d->local_count);
}

// Grouped calls' common arguments.
moe_status check_group(const char *fn, const moe_dims *d, int32_t e_first, int32_t e_count,
                       const int32_t *offsets, const int32_t *sorted_slot, int32_t k) {
    if (e_first < 0 || e_count < 0 || e_first > d->local_count - e_count)
        return fail(MOE_ERR_INVALID, "%s: expert range outside [0, local_count)", fn);
    if (d->tokens == 0 || e_count == 0) return MOE_OK;
    if (!offsets) return fail(MOE_ERR_INVALID, "%s: offsets is NULL", fn);
    if (sorted_slot && (uint64_t)d->tokens * (uint64_t)k >= kMaxOffset)
        return fail(MOE_ERR_UNSUPPORTED, "%s: a gathered token matrix of 4 GiB or more", fn);
    return MOE_OK;
}

// The load of the local experts under uniform routing.  It picks the form of a
// launch, over whatever range of them, so that a range has the bits of the
// whole.
ScaledLoad expected_load(const moe_dims &d) {
    ScaledLoad l;
    const double p = (double)d.top_k / d.experts;
    l.rows = (double)d.tokens * p * d.local_count;
    l.active = d.local_count * (1.0 - std::pow(1.0 - p, (double)d.tokens));
    l.max_rows = d.tokens;  // a token routes to an expert at most once
    l.experts = d.local_count;
    return l;
}

ScaledLoad dense_load(int64_t rows) { return {(double)rows, 1.0, rows, 1}; }

hipError_t product(const ScaledGemm &g, int y_type, const ScaledLoad &load, hipStream_t s) {
    if (scaled_stream_product_fits(g.N, g.K, load))
        return launch_stream_scaled(g, y_type, false, load, s);
    return scaled_mid_fits(g.N, load) ? launch_mid_scaled(g, y_type, load.max_rows, s)
                                      : launch_scaled_gemm(g, y_type, load, s);
}

size_t up(size_t v) { return (v + 255) & ~size_t(255); }

// The SwiGLU rows between an FFN's two products: quantised, or fp32 where the
// launches of few rows run.  few: the most rows that those can be chosen for.
// A workspace holds either, so that one made for some tokens serves fewer.
struct FfnWs {
    bool stream;
    size_t act, act_s, total;
};
FfnWs ffn_ws(int64_t rows, int64_t few, int32_t inter, const ScaledLoad &load) {
    FfnWs w;
    w.stream = rows > 0 && scaled_stream_fits(scaled_tiles(true, inter), load);
    w.act = 0;
    w.act_s = up((size_t)rows * inter);
    w.total = std::max(w.act_s + up((size_t)rows * scale_pitch(inter)),
                       up((size_t)std::min(rows, few) * inter * sizeof(float)));
    return w;
}
FfnWs ffn_ws(const moe_dims *d) {
    const int64_t few_tokens = std::min(kStreamTokens, kStreamRows * d->experts / d->top_k);
    return ffn_ws(row_cap(d), few_tokens * std::min(d->top_k, d->local_count), d->inter,
                  expected_load(*d));
}
FfnWs shared_ws(const moe_dims *d) {
    return ffn_ws(d->tokens, kStreamRows, d->shared_inter, dense_load(d->tokens));
}

struct Matrix {
    const uint8_t *q, *s;
};
// Both products of an FFN; `rows` holds the rows of the first (offsets, x,
// row_map, ..), weights of width `inter`.
moe_status ffn(ScaledGemm rows, int32_t hidden, int32_t inter, Matrix gate, Matrix up_,
               Matrix down, void *y, int32_t y_type, const FfnWs &L, char *ws,
               const ScaledLoad &load, hipStream_t s) {
    uint8_t *act = (uint8_t *)ws + L.act, *act_s = (uint8_t *)ws + L.act_s;
    ScaledGemm g = rows;
    g.w0 = gate.q, g.s0 = gate.s;
    g.w1 = up_.q, g.s1 = up_.s;
    g.N = inter, g.K = hidden;
    g.out = act, g.out_s = act_s;
    MOE_HIP(L.stream ? launch_stream_swiglu(g, load, s) : launch_scaled_swiglu(g, load, s));
    ScaledGemm h = rows;
    h.x = act, h.xs = act_s;
    h.row_map = nullptr;
    h.w0 = down.q, h.s0 = down.s;
    h.N = hidden, h.K = inter;
    h.out = y;
    MOE_HIP(L.stream ? launch_stream_scaled(h, y_type, true, load, s)
                     : product(h, y_type, load, s));
    return MOE_OK;
}

// Workspace of the whole layer.
struct LayerWs {
    WsLayout perm;  // the dispatch's own regions, at offset 0
    FfnWs routed, shared;
    size_t y, q, s, ids, weights, logits, counts, offsets, sorted_slot, slot_row, ffn, y_perm,
        total;
};
LayerWs layer_ws(const moe_dims *d) {
    LayerWs w;
    w.perm = ws_layout(d, nullptr);
    w.routed = ffn_ws(d);
    w.shared = d->shared_inter > 0 ? shared_ws(d) : FfnWs{};
    size_t o = up(w.perm.total);
    auto take = [&](size_t bytes) {
        const size_t at = o;
        o += up(bytes);
        return at;
    };
    const size_t T = (size_t)d->tokens, slots = T * d->top_k, H = (size_t)d->hidden;
    w.y = take(T * H * sizeof(bf16_t));
    w.q = take(T * H);
    w.s = take(T * scale_pitch(d->hidden));
    w.ids = take(slots * sizeof(int32_t));
    w.weights = take(slots * sizeof(float));
    w.logits = d->experts > 16 && d->tokens <= kRouteLogitsMaxTokens
                   ? take(T * d->experts * sizeof(float))
                   : 0;
    w.counts = take(d->local_count * sizeof(int32_t));
    w.offsets = take((d->local_count + 1) * sizeof(int32_t));
    w.sorted_slot = take((size_t)row_cap(d) * sizeof(int32_t));
    w.slot_row = take(slots * sizeof(int32_t));
    w.ffn = take(std::max(w.routed.total, w.shared.total));  // one FFN after the other
    w.y_perm = take((size_t)row_cap(d) * H * sizeof(bf16_t));
    w.total = o;
    return w;
}

}  // namespace

extern "C" {

size_t moe_scale_pitch(int32_t k) { return width_ok(k) ? (size_t)scale_pitch(k) : 0; }

moe_status moe_quant_rows(int64_t rows, int32_t cols, const void *x, int32_t x_type, moe_e4m3 *q,
                          moe_scale *scales, void *stream) {
    const char *fn = "moe_quant_rows";
    if (rows < 0) return fail(MOE_ERR_INVALID, "%s: rows < 0", fn);
    if (!width_ok(cols))
        return fail(MOE_ERR_INVALID, "%s: cols %d not a multiple of %d up to 2^20", fn, cols,
                    kDimAlign);
    if (!type_ok(x_type)) return fail(MOE_ERR_INVALID, "%s: x_type %d", fn, x_type);
    if (rows == 0) return MOE_OK;
    MOE_TRY(check_tensor(fn, "x", x));
    MOE_TRY(check_pair(fn, "q", q, scales));
    MOE_HIP(launch_norm_quant(rows, cols, x, x_type, nullptr, false, nullptr, 0.f, nullptr,
                              nullptr, q, scales, (hipStream_t)stream));
    return MOE_OK;
}

moe_status moe_quant_weights(int32_t experts, int32_t n, int32_t k, const moe_bf16 *w,
                             moe_e4m3 *q, moe_scale *scales, void *stream) {
    const char *fn = "moe_quant_weights";
    if (experts < 0) return fail(MOE_ERR_INVALID, "%s: experts < 0", fn);
    if (experts > kMaxExperts)
        return fail(MOE_ERR_UNSUPPORTED, "%s: experts %d > %d", fn, experts, kMaxExperts);
    if (!width_ok(n) || !width_ok(k))
        return fail(MOE_ERR_INVALID, "%s: widths %d, %d not multiples of %d up to 2^20", fn, n, k,
                    kDimAlign);
    if (experts == 0) return MOE_OK;
    MOE_TRY(check_tensor(fn, "w", w));
    MOE_TRY(check_pair(fn, "q", q, scales));
    MOE_HIP(launch_quant_weights(experts, n, k, w, q, scales, (hipStream_t)stream));
    return MOE_OK;
}

moe_status moe_norm_quant(int64_t rows, int32_t hidden, const void *x, int32_t x_type,
                          const moe_bf16 *residual, const moe_bf16 *weight, float eps,
                          moe_bf16 *total, moe_bf16 *y, moe_e4m3 *q, moe_scale *scales,
                          void *stream) {
    const char *fn = "moe_norm_quant";
    if (rows < 0) return fail(MOE_ERR_INVALID, "%s: rows < 0", fn);
    if (!width_ok(hidden))
        return fail(MOE_ERR_INVALID, "%s: hidden %d not a multiple of %d up to 2^20", fn, hidden,
                    kDimAlign);
    if (!type_ok(x_type)) return fail(MOE_ERR_INVALID, "%s: x_type %d", fn, x_type);
    if (!(eps >= 0.f) || std::isinf(eps))
        return fail(MOE_ERR_INVALID, "%s: eps is negative or not finite", fn);
    if (!y && !q) return fail(MOE_ERR_INVALID, "%s: neither y nor q is given", fn);
    if ((q == nullptr) != (scales == nullptr))
        return fail(MOE_ERR_INVALID, "%s: q and scales go together", fn);
    if (rows == 0) return MOE_OK;
    MOE_TRY(check_tensor(fn, "x", x));
    if (residual) MOE_TRY(check_tensor(fn, "residual", residual));
    if (weight) MOE_TRY(check_tensor(fn, "weight", weight));
    if (total) MOE_TRY(check_tensor(fn, "total", total));
    if (y) MOE_TRY(check_tensor(fn, "y", y));
    if (q) MOE_TRY(check_pair(fn, "q", q, scales));
    MOE_HIP(launch_norm_quant(rows, hidden, x, x_type, residual, true, weight, eps, total, y, q,
                              scales, (hipStream_t)stream));
    return MOE_OK;
}

moe_status moe_gemm_scaled(int64_t rows, int32_t n, int32_t k, const moe_e4m3 *x,
                           const moe_scale *x_scales, const moe_e4m3 *w,
                           const moe_scale *w_scales, void *y, int32_t y_type, void *stream) {
    const char *fn = "moe_gemm_scaled";
    if (rows < 0) return fail(MOE_ERR_INVALID, "%s: rows < 0", fn);
    MOE_TRY(check_product(fn, rows, 1, n, k));
    if (!type_ok(y_type)) return fail(MOE_ERR_INVALID, "%s: y_type %d", fn, y_type);
    if (rows == 0) return MOE_OK;
    MOE_TRY(check_pair(fn, "x", x, x_scales));
    MOE_TRY(check_pair(fn, "w", w, w_scales));
    MOE_TRY(check_tensor(fn, "y", y));
    ScaledGemm g{};
    g.e_count = 1;
    g.rows_one = rows;
    g.x = x, g.xs = x_scales;
    g.slot_div = 1;
    g.w0 = w, g.s0 = w_scales;
    g.N = n, g.K = k;
    g.out = y;
    MOE_HIP(product(g, y_type, dense_load(rows), (hipStream_t)stream));
    return MOE_OK;
}

moe_status moe_gemm_group_scaled(const moe_dims *dims, int32_t e_first, int32_t e_count,
                                 const int32_t *offsets, const int32_t *sorted_slot, int32_t n,
                                 int32_t k, const moe_e4m3 *x, const moe_scale *x_scales,
                                 const moe_e4m3 *w, const moe_scale *w_scales, void *y,
                                 int32_t y_type, void *stream) {
    const char *fn = "moe_gemm_group_scaled";
    MOE_TRY(check_dims(dims));
    MOE_TRY(check_product(fn, row_cap(dims), dims->local_count, n, k));
    if (!type_ok(y_type)) return fail(MOE_ERR_INVALID, "%s: y_type %d", fn, y_type);
    MOE_TRY(check_group(fn, dims, e_first, e_count, offsets, sorted_slot, k));
    if (dims->tokens == 0 || e_count == 0) return MOE_OK;
    MOE_TRY(check_pair(fn, "x", x, x_scales));
    MOE_TRY(check_pair(fn, "w", w, w_scales));
    MOE_TRY(check_tensor(fn, "y", y));
    ScaledGemm g{};
    g.offsets = offsets;
    g.e_first = e_first, g.e_count = e_count;
    g.x = x, g.xs = x_scales;
    g.row_map = sorted_slot;
    g.slot_div = dims->top_k;
    g.w0 = w, g.s0 = w_scales;
    g.N = n, g.K = k;
    g.out = y;
    MOE_HIP(product(g, y_type, expected_load(*dims), (hipStream_t)stream));
    return MOE_OK;
}

size_t moe_scaled_workspace_bytes(const moe_dims *dims) {
    if (check_dims(dims) != MOE_OK) return 0;
    return std::max<size_t>(ffn_ws(dims).total, 256);
}

moe_status moe_ffn_group_scaled(const moe_dims *dims, int32_t e_first, int32_t e_count,
                                const int32_t *offsets, const int32_t *sorted_slot,
                                const moe_e4m3 *x, const moe_scale *x_scales,
                                const moe_e4m3 *w_gate, const moe_scale *gate_scales,
                                const moe_e4m3 *w_up, const moe_scale *up_scales,
                                const moe_e4m3 *w_down, const moe_scale *down_scales,
                                void *y_perm, int32_t y_type, void *ws, size_t ws_bytes,
                                void *stream) {
    const char *fn = "moe_ffn_group_scaled";
    MOE_TRY(check_dims(dims));
    MOE_TRY(check_product(fn, row_cap(dims), dims->local_count,
                          std::max(dims->hidden, dims->inter), kDimAlign));
    if (!type_ok(y_type)) return fail(MOE_ERR_INVALID, "%s: y_type %d", fn, y_type);
    MOE_TRY(check_group(fn, dims, e_first, e_count, offsets, sorted_slot, dims->hidden));
    if (dims->tokens == 0 || e_count == 0) return MOE_OK;
    MOE_TRY(check_pair(fn, "x", x, x_scales));
    MOE_TRY(check_pair(fn, "w_gate", w_gate, gate_scales));
    MOE_TRY(check_pair(fn, "w_up", w_up, up_scales));
    MOE_TRY(check_pair(fn, "w_down", w_down, down_scales));
    MOE_TRY(check_tensor(fn, "y_perm", y_perm));
    const FfnWs L = ffn_ws(dims);
    if (!ws || ws_bytes < L.total)
        return fail(MOE_ERR_WORKSPACE, "%s: workspace %zu < %zu bytes", fn, ws_bytes, L.total);
    MOE_TRY(check_tensor(fn, "ws", ws));
    ScaledGemm g{};
    g.offsets = offsets;
    g.e_first = e_first, g.e_count = e_count;
    g.x = x, g.xs = x_scales;
    g.row_map = sorted_slot;
    g.slot_div = dims->top_k;
    return ffn(g, dims->hidden, dims->inter, {w_gate, gate_scales}, {w_up, up_scales},
               {w_down, down_scales}, y_perm, y_type, L, (char *)ws, expected_load(*dims),
               (hipStream_t)stream);
}

moe_status moe_combine_rows(const moe_dims *dims, int32_t e_first, int32_t e_count,
                            const void *y_perm, int32_t y_type, const int32_t *topk_ids,
                            const int32_t *slot_row, const float *topk_w, float *y,
                            int32_t accumulate, void *stream) {
    const char *fn = "moe_combine_rows";
    MOE_TRY(check_dims(dims));
    if (!type_ok(y_type)) return fail(MOE_ERR_INVALID, "%s: y_type %d", fn, y_type);
    if (y_type == MOE_FP32)
        return moe_combine(dims, e_first, e_count, (const float *)y_perm, topk_ids, slot_row,
                           topk_w, y, accumulate, stream);
    if (e_first < 0 || e_count < 0 || e_first > dims->local_count - e_count)
        return fail(MOE_ERR_INVALID, "%s: expert range outside [0, local_count)", fn);
    if (accumulate != 0 && accumulate != 1)
        return fail(MOE_ERR_INVALID, "%s: accumulate must be 0 or 1", fn);
    if (dims->tokens == 0) return MOE_OK;
    if (!topk_ids || !slot_row || !topk_w)
        return fail(MOE_ERR_INVALID, "%s: NULL index tensor", fn);
    MOE_TRY(check_tensor(fn, "y", y));
    if (e_count > 0) MOE_TRY(check_tensor(fn, "y_perm", y_perm, 8));
    MOE_HIP(launch_combine(*dims, e_first, e_count, 0, dims->tokens, (const bf16_t *)y_perm,
                           topk_ids, slot_row, topk_w, y, accumulate, (hipStream_t)stream));
    return MOE_OK;
}

size_t moe_forward_scaled_bytes(const moe_dims *dims) {
    if (check_dims(dims) != MOE_OK) return 0;
    // (more tokens than that need no router logits)
    moe_dims few = *dims;
    few.tokens = std::min(few.tokens, kRouteLogitsMaxTokens);
    return std::max(layer_ws(dims).total, layer_ws(&few).total);
}

moe_status moe_forward_scaled(const moe_dims *dims, const void *x, int32_t x_type,
                              const moe_bf16 *residual, const moe_bf16 *norm_weight, float eps,
                              moe_bf16 *total, const float *w_router, const float *bias,
                              const moe_scaled_weights *weights, float *y, int32_t *topk_ids,
                              float *topk_w, int32_t *counts, void *ws, size_t ws_bytes,
                              void *stream) {
    const char *fn = "moe_forward_scaled";
    MOE_TRY(check_dims(dims));
    MOE_TRY(check_product(fn, row_cap(dims), dims->local_count,
                          std::max({dims->hidden, dims->inter, dims->shared_inter}), kDimAlign));
    if (!type_ok(x_type)) return fail(MOE_ERR_INVALID, "%s: x_type %d", fn, x_type);
    if (!norm_weight && (x_type != MOE_BF16 || residual || total))
        return fail(MOE_ERR_INVALID,
                    "%s: without norm_weight x is bf16 rows normalised before, with no residual "
                    "and no total",
                    fn);
    if (norm_weight && (!(eps >= 0.f) || std::isinf(eps)))
        return fail(MOE_ERR_INVALID, "%s: eps is negative or not finite", fn);
    if (!weights) return fail(MOE_ERR_INVALID, "%s: weights is NULL", fn);
    if ((uint64_t)dims->tokens * (uint64_t)dims->hidden >= kMaxOffset)
        return fail(MOE_ERR_UNSUPPORTED, "%s: a quantised token matrix of 4 GiB or more", fn);
    if (dims->tokens == 0) return MOE_OK;
    MOE_TRY(check_tensor(fn, "x", x));
    if (residual) MOE_TRY(check_tensor(fn, "residual", residual));
    if (norm_weight) MOE_TRY(check_tensor(fn, "norm_weight", norm_weight));
    if (total) MOE_TRY(check_tensor(fn, "total", total));
    if (!w_router) return fail(MOE_ERR_INVALID, "%s: w_router is NULL", fn);
    const moe_scaled_weights &w = *weights;
    MOE_TRY(check_pair(fn, "w_gate", w.gate, w.gate_scales));
    MOE_TRY(check_pair(fn, "w_up", w.up, w.up_scales));
    MOE_TRY(check_pair(fn, "w_down", w.down, w.down_scales));
    if (dims->shared_inter > 0) {
        MOE_TRY(check_pair(fn, "shared_gate", w.shared_gate, w.shared_gate_scales));
        MOE_TRY(check_pair(fn, "shared_up", w.shared_up, w.shared_up_scales));
        MOE_TRY(check_pair(fn, "shared_down", w.shared_down, w.shared_down_scales));
    }
    MOE_TRY(check_tensor(fn, "y", y));
    const LayerWs L = layer_ws(dims);
    if (!ws || ws_bytes < L.total)
        return fail(MOE_ERR_WORKSPACE, "%s: workspace %zu < %zu bytes", fn, ws_bytes, L.total);
    MOE_TRY(check_tensor(fn, "ws", ws));

    const moe_dims &d = *dims;
    char *base = (char *)ws;
    hipStream_t s = (hipStream_t)stream;
    uint8_t *q = (uint8_t *)base + L.q, *qs = (uint8_t *)base + L.s;
    // rows: normalised ones go through the workspace to the router
    const bf16_t *rows = (const bf16_t *)x;
    if (norm_weight) {
        bf16_t *yn = (bf16_t *)(base + L.y);
        MOE_HIP(launch_norm_quant(d.tokens, d.hidden, x, x_type, residual, true, norm_weight, eps,
                                  total, yn, q, qs, s));
        rows = yn;
    } else {
        MOE_HIP(launch_norm_quant(d.tokens, d.hidden, x, x_type, nullptr, false, nullptr, 0.f,
                                  nullptr, nullptr, q, qs, s));
    }
    // routing and dispatch indices
    int32_t *ids = topk_ids ? topk_ids : (int32_t *)(base + L.ids);
    float *wts = topk_w ? topk_w : (float *)(base + L.weights);
    int32_t *cnt = counts ? counts : (int32_t *)(base + L.counts);
    int32_t *off = (int32_t *)(base + L.offsets), *slot = (int32_t *)(base + L.sorted_slot);
    int32_t *slot_row = (int32_t *)(base + L.slot_row);
    float *logits = L.logits ? (float *)(base + L.logits) : nullptr;
    const bool fused = route_dispatches(d, rows, logits);
    const DispatchOut disp = dispatch_out(d, L.perm, 0, cnt, off, nullptr, slot, slot_row);
    MOE_HIP(launch_route(d, rows, w_router, bias, ids, wts, logits, s, fused ? &disp : nullptr));
    if (!fused)
        MOE_HIP(launch_permute(d, ids, base, L.perm, 0, cnt, off, nullptr, slot, slot_row, s));
    // the shared experts are one expert of all tokens and write y
    ScaledGemm g{};
    g.x = q, g.xs = qs;
    g.slot_div = d.top_k;
    if (d.shared_inter > 0) {
        g.e_count = 1;
        g.rows_one = d.tokens;
        MOE_TRY(ffn(g, d.hidden, d.shared_inter, {w.shared_gate, w.shared_gate_scales},
                    {w.shared_up, w.shared_up_scales}, {w.shared_down, w.shared_down_scales}, y,
                    MOE_FP32, L.shared, base + L.ffn, dense_load(d.tokens), s));
    }
    g.offsets = off;
    g.e_count = d.local_count;
    g.row_map = slot;
    // The routed rows wait for the combine in bf16, half the bytes of fp32 (16384 x
    // 4096 of two rows 143 -> 100 us): at most 2^-8 of a value, where the quantisation of
    // its inputs and weights costs the layer 6.6%.  moe_ffn_group_scaled and
    // moe_combine_rows do the same in fp32.
    bf16_t *y_perm = (bf16_t *)(base + L.y_perm);
    MOE_TRY(ffn(g, d.hidden, d.inter, {w.gate, w.gate_scales}, {w.up, w.up_scales},
                {w.down, w.down_scales}, y_perm, MOE_BF16, L.routed, base + L.ffn,
                expected_load(d), s));
    MOE_HIP(launch_combine(d, 0, d.local_count, 0, d.tokens, y_perm, ids, slot_row, wts, y,
                           d.shared_inter > 0 ? 1 : 0, s));
    return MOE_OK;
}

}  // extern "C"
