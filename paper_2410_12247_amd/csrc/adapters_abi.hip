// C-ABI entry points of the low-rank adapters: argument checks, workspace
// layout, and the launches of a call.
#include <algorithm>

#include "adapters.h"

using namespace moe;

namespace {

bool width_ok(int32_t v) { return v > 0 && v % kDimAlign == 0 && v <= kMaxWidth; }

moe_status check_at(const char *fn, const char *name, const void *p, uintptr_t a = 16) {
    if (!p) return fail(MOE_ERR_INVALID, "%s: %s is NULL", fn, name);
    if ((uintptr_t)p % a)
        return fail(MOE_ERR_INVALID, "%s: %s is not %d-byte aligned", fn, name, (int)a);
    return MOE_OK;
}

moe_status check_adapters(const char *fn, int64_t rows, const moe_adapters *ad) {
    if (rows < 0) return fail(MOE_ERR_INVALID, "%s: rows < 0", fn);
    if (rows >= (int64_t(1) << 31)) return fail(MOE_ERR_UNSUPPORTED, "%s: 2^31 rows or more", fn);
    if (!ad) return fail(MOE_ERR_INVALID, "%s: adapters is NULL", fn);
    if (ad->count < 1) return fail(MOE_ERR_INVALID, "%s: count %d", fn, ad->count);
    if (ad->count > kMaxExperts)
        return fail(MOE_ERR_UNSUPPORTED, "%s: count %d > %d", fn, ad->count, kMaxExperts);
    if (ad->rank < 1 || ad->rank % kRankAlign)
        return fail(MOE_ERR_INVALID, "%s: rank %d not a positive multiple of %d", fn, ad->rank,
                    kRankAlign);
    if (ad->rank > kMaxRank)
        return fail(MOE_ERR_UNSUPPORTED, "%s: rank %d > %d", fn, ad->rank, kMaxRank);
    if (!width_ok(ad->n) || !width_ok(ad->k))
        return fail(MOE_ERR_INVALID, "%s: widths %d, %d not multiples of %d up to 2^20", fn, ad->n,
                    ad->k, kDimAlign);
    if (!adapter_launches_fit(rows, *ad))
        return fail(MOE_ERR_UNSUPPORTED, "%s: %lld rows of %d and %d values need 2^32 lanes", fn,
                    (long long)rows, ad->n, ad->k);
    return MOE_OK;
}

moe_status check_weights(const char *fn, const moe_adapters *ad) {
    MOE_TRY(check_at(fn, "a", ad->a));
    MOE_TRY(check_at(fn, "b", ad->b));
    if (ad->scale) MOE_TRY(check_at(fn, "scale", ad->scale, 4));
    return MOE_OK;
}

moe_status check_rows(const char *fn, const int32_t *offsets, const int32_t *sorted_slot) {
    MOE_TRY(check_at(fn, "offsets", offsets, 4));
    return check_at(fn, "sorted_slot", sorted_slot, 4);
}

size_t up(size_t v) { return (v + 255) & ~size_t(255); }

size_t sums_bytes(int64_t rows, const moe_adapters *ad, bool back) {
    return up(adapter_sums_bytes(rows, *ad, back));
}

struct BackWs {
    size_t u, v, pa, pb, total;
};
BackWs back_ws(int64_t rows, const moe_adapters *ad) {
    BackWs w;
    size_t o = 0;
    auto take = [&](size_t bytes) {
        const size_t at = o;
        o += up(bytes);
        return at;
    };
    w.u = take(sums_bytes(rows, ad, true));
    w.v = take(sums_bytes(rows, ad, true));
    w.pa = take(adapter_parts_bytes(rows, ad->rank, ad->k));
    w.pb = take(adapter_parts_bytes(rows, ad->rank, ad->n));
    w.total = o;
    return w;
}

}  // namespace

extern "C" {

size_t moe_adapter_workspace_bytes(int64_t rows, const moe_adapters *adapters) {
    if (check_adapters("moe_adapter_workspace_bytes", rows, adapters) != MOE_OK) return 0;
    return std::max<size_t>(sums_bytes(rows, adapters, false), 256);
}

moe_status moe_adapter_rows(int64_t rows, const moe_adapters *adapters, const int32_t *offsets,
                            const int32_t *sorted_slot, const int32_t *slot_row,
                            const moe_bf16 *x, const void *base, void *y, int32_t y_type, void *ws,
                            size_t ws_bytes, void *stream) {
    const char *fn = "moe_adapter_rows";
    MOE_TRY(check_adapters(fn, rows, adapters));
    if (y_type != MOE_BF16 && y_type != MOE_FP32)
        return fail(MOE_ERR_INVALID, "%s: y_type %d", fn, y_type);
    if (rows == 0) return MOE_OK;
    MOE_TRY(check_weights(fn, adapters));
    MOE_TRY(check_rows(fn, offsets, sorted_slot));
    MOE_TRY(check_at(fn, "x", x));
    if (base) MOE_TRY(check_at(fn, "base", base));
    MOE_TRY(check_at(fn, "y", y));
    if (base != y) MOE_TRY(check_at(fn, "slot_row", slot_row, 4));
    const moe_adapters &ad = *adapters;
    const size_t need = sums_bytes(rows, &ad, false);
    if (!ws || ws_bytes < need)
        return fail(MOE_ERR_WORKSPACE, "%s: workspace %zu < %zu bytes", fn, ws_bytes, need);
    MOE_TRY(check_at(fn, "ws", ws));
    const AdapterRows o =
        adapter_tiles({offsets, sorted_slot, slot_row, rows, ad.count, 0}, ad, false);
    MOE_HIP(launch_adapter_rows(o, ad, x, base, y, y_type, adapter_sums(o, ad.rank, ad.k, 1, ws),
                                (hipStream_t)stream));
    return MOE_OK;
}

size_t moe_adapter_backward_bytes(int64_t rows, const moe_adapters *adapters) {
    if (check_adapters("moe_adapter_backward_bytes", rows, adapters) != MOE_OK) return 0;
    // (the forward pass has tall tiles, which need more, from fewer rows on at small ranks)
    return std::max<size_t>(
        {back_ws(rows, adapters).total, sums_bytes(rows, adapters, false), 256});
}

moe_status moe_adapter_backward(int64_t rows, const moe_adapters *adapters,
                                const int32_t *offsets, const int32_t *sorted_slot,
                                const int32_t *slot_row, const moe_bf16 *x, const moe_bf16 *dy,
                                const void *dx_base, void *dx, int32_t dx_type, float *da,
                                float *db, int32_t accumulate, void *ws, size_t ws_bytes,
                                void *stream) {
    const char *fn = "moe_adapter_backward";
    MOE_TRY(check_adapters(fn, rows, adapters));
    if (dx_type != MOE_BF16 && dx_type != MOE_FP32)
        return fail(MOE_ERR_INVALID, "%s: dx_type %d", fn, dx_type);
    if (accumulate != 0 && accumulate != 1)
        return fail(MOE_ERR_INVALID, "%s: accumulate must be 0 or 1", fn);
    if ((da == nullptr) != (db == nullptr))
        return fail(MOE_ERR_INVALID, "%s: da and db go together", fn);
    if (!dx && !da) return fail(MOE_ERR_INVALID, "%s: neither dx nor da is given", fn);
    if (!dx && dx_base) return fail(MOE_ERR_INVALID, "%s: dx_base without dx", fn);
    if (da) {
        MOE_TRY(check_at(fn, "da", da));
        MOE_TRY(check_at(fn, "db", db));
    }
    const moe_adapters &ad = *adapters;
    const AdapterRows o =
        adapter_tiles({offsets, sorted_slot, slot_row, rows, ad.count, 0}, ad, true);
    AdapterBack k{};
    k.x = x, k.dy = dy;
    k.base = dx_base, k.dx = dx, k.dx_type = dx_type;
    k.da = da, k.db = db, k.accumulate = accumulate != 0;
    if (rows == 0) {  // gradients of nothing are zeros
        MOE_HIP(launch_adapter_backward(o, ad, k, (hipStream_t)stream));
        return MOE_OK;
    }
    MOE_TRY(check_weights(fn, adapters));
    MOE_TRY(check_rows(fn, offsets, sorted_slot));
    if (da) MOE_TRY(check_at(fn, "x", x));
    MOE_TRY(check_at(fn, "dy", dy));
    if (dx) {
        if (dx_base) MOE_TRY(check_at(fn, "dx_base", dx_base));
        MOE_TRY(check_at(fn, "dx", dx));
        if (dx_base != dx) MOE_TRY(check_at(fn, "slot_row", slot_row, 4));
    }
    const BackWs L = back_ws(rows, adapters);
    if (!ws || ws_bytes < L.total)
        return fail(MOE_ERR_WORKSPACE, "%s: workspace %zu < %zu bytes", fn, ws_bytes, L.total);
    MOE_TRY(check_at(fn, "ws", ws));
    char *base = (char *)ws;
    k.u = adapter_sums(o, ad.rank, ad.k, 2, base + L.u);
    k.v = adapter_sums(o, ad.rank, ad.n, 2, base + L.v);
    k.pa = (float *)(base + L.pa), k.pb = (float *)(base + L.pb);
    MOE_HIP(launch_adapter_backward(o, ad, k, (hipStream_t)stream));
    return MOE_OK;
}

}  // extern "C"
