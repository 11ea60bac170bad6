// Low-rank adapters: what their kernels and entry points share.
#pragma once

#include "common.h"

namespace moe {

constexpr int kMaxRank = 256;
constexpr int kRankAlign = 8;  // a 16-byte load of an adapter row

// The rows of a launch, ordered by adapter (moe_permute's outputs): places
// [offsets[e], offsets[e + 1]) belong to adapter e, place p is row order[p];
// place[row] is row's, < 0 for a row of no adapter.
struct AdapterRows {
    const int32_t *offsets, *order, *place;
    int64_t rows;
    int count;
    int blocks;  // of 16 rows of a tile, 1 or 8
};
// With the tiles' height, of the forward pass or the gradient.
AdapterRows adapter_tiles(AdapterRows o, const moe_adapters &ad, bool back);

// Sums over K of rows times a low-rank matrix, in fp32: [tile][split][rank][rows of
// a tile], tiles as the device numbers them, a split a share of K; for many rows also
// scaled and cut into bf16 parts, as operands (e, q).
struct AdapterSums {
    float *p;
    int splits;
    bf16_t *e, *q;
};
// Their layout at an address (together: how many sums share a launch), and its bytes
// (no fewer than any fewer rows need).
AdapterSums adapter_sums(const AdapterRows &o, int rank, int K, int together, void *at);
size_t adapter_sums_bytes(int64_t rows, const moe_adapters &ad, bool back);

// Whether every launch of these rows and widths (both directions') is one the device
// takes.
bool adapter_launches_fit(int64_t rows, const moe_adapters &ad);

// Bytes of the buffer of the outer products' parts over C columns (likewise).
size_t adapter_parts_bytes(int64_t rows, int rank, int C);

// The forward pass: y[row] = base[row] + scale[e] * b[e] (a[e] x_row).
hipError_t launch_adapter_rows(const AdapterRows &o, const moe_adapters &ad, const bf16_t *x,
                               const void *base, void *y, int y_type, const AdapterSums &u,
                               hipStream_t s);

// Its gradient; dx, or da and db, may be NULL.  pa, pb: the parts of da and db.
struct AdapterBack {
    const bf16_t *x, *dy;
    const void *base;
    void *dx;
    int dx_type;
    float *da, *db;
    bool accumulate;
    AdapterSums u, v;
    float *pa, *pb;
};
hipError_t launch_adapter_backward(const AdapterRows &o, const moe_adapters &ad,
                                   const AdapterBack &k, hipStream_t s);

}  // namespace moe
