// Low-rank adapters: what their kernels and entry points share.
#pragma once

#include "common.h"

namespace moe {

constexpr int kMaxRank = 256;
constexpr int kRankAlign = 8;  // a 16-byte load of an adapter row

// The rows of a launch, ordered by adapter (moe_permute's outputs): places
// [offsets[e], offsets[e + 1]) belong to adapter e, place p is row order[p].
struct AdapterRows {
    const int32_t *offsets, *order;
    int64_t rows;
    int count;
};

// p[split][place][rank] = partial sums over K of w[e] x_row (w [count][rank][K]):
// split s of `splits` takes its share of K.
hipError_t launch_adapter_shrink(const AdapterRows &o, int rank, int K, const bf16_t *x,
                                 const bf16_t *w, float *p, int splits, hipStream_t s);
// y[row] = base[row] + scale[e] * w[e] (sum over splits of p[.][place]) (w [count][N][rank]);
// rows of no adapter (place[row] < 0) get base's row, unless base is y.
hipError_t launch_adapter_expand(const AdapterRows &o, int rank, int N, const float *p, int splits,
                                 const bf16_t *w, const float *scale, const int32_t *place,
                                 const void *base, void *y, int y_type, hipStream_t s);
// out[e] (+)= scale[e] * sum over the adapter's rows of p[place]^T q_row: out
// [count][rank][C], or transposed [count][C][rank].  parts: adapter_outer_slots()
// buffers of rank * C floats.
hipError_t launch_adapter_outer(const AdapterRows &o, int rank, int C, const float *p, int splits,
                                const bf16_t *q, const float *scale, float *parts, bool transposed,
                                bool accumulate, float *out, hipStream_t s);
// wt[e] = w[e]^T for the adapters that have rows; w [count][m][n].
hipError_t launch_adapter_transpose(const AdapterRows &o, int m, int n, const bf16_t *w,
                                    bf16_t *wt, hipStream_t s);

// Shares of K that a shrink of these rows is cut into.
int adapter_splits(int64_t rows, int count, int K);
int64_t adapter_outer_slots(int64_t rows);

}  // namespace moe
