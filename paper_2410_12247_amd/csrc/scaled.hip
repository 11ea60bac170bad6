// Products over block-scaled 8-bit tensors on the gfx950 matrix cores:
//   y[r][n] = sum over blocks b of 128 k of
//             2^(sx[r][b] + sw[n/128][b] - 254) sum_{k in b} x[r][k] w[n][k],
// or Q(silu(g) u) of two such products.  The scaled matrix instruction takes
// both scale bytes as operands, so a block's scaling costs nothing: the token
// row's scale is a lane's own byte, the weight's one for all.  Weights are its A
// operand and tokens its B, so a lane holds runs of four output columns of one
// token row.
//
// Large launches are bound by the matrix cores, and those by the board's power:
// the chip runs at 1.55 to 1.9 GHz under them, and a launch's time depends on what
// ran before it.  16384 x 5120 x 4096 takes 263 us, 2.61 PFLOP/s (a library's 8-bit
// product of 8192^3 2.71), the cores busy in 65% of the cycles; the Mixtral FFN of
// 16384 tokens 1.22 ms, 2.36 PFLOP/s (1.34 under launches of its own only); DBRX gate
// of 8192 tokens 253 to 259 us, 2.1 (N is 5.25 tiles of 256: 15% of the products are
// padding).  Few rows are bound by the weights' stream: DBRX FFN of 64 tokens 91
// us, 4.4 TB/s; DeepSeekV2 gate product of 61 tokens (20 experts, 157 MB) 31 us, 5.1
// TB/s; its down product of 4099 tokens with a Zipf load 66 to 75 us, 4.0 TB/s and 1.2
// PFLOP/s, between the two, its second round of tiles part full.
#include <algorithm>

#include "lds_dma.h"
#include "scaled.h"

namespace moe {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// buffer resource word 3 for raw (untyped, unswizzled) access on gfx9 parts
constexpr int kBufferFlags = 0x00020000;
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

// ---------------------------------------------------------------------------
// Tile of BN weight rows x BM token rows, four waves (one per SIMD) in a 2 x 2
// arrangement, each with a BN/2 x BM/2 accumulator block of 32 x 32 MFMAs (the
// blocks' token rows alternate by 32, so a tile of few rows keeps all waves
// busy).
// K advances by pairs of 64 (one MFMA's K, so a pair is a scale block) through
// two to four LDS buffers filled by LDS-DMA with whole 128-byte lines of the rows.
// One workgroup per CU stays for the whole launch, and the next tile's requests
// are on their way under a tile's epilogue.
// ---------------------------------------------------------------------------
template <int MODE, int BM_, int BN_>
struct Cfg {
    static constexpr int BM = BM_, BN = BN_;                 // token and weight rows of the tile
    static constexpr int BNOUT = MODE == SWIGLU ? 128 : BN;  // output columns
    static_assert(BN == 256 || (BN == 128 && MODE != SWIGLU), "whole scale blocks per tile");
    static constexpr int THREADS = 256;
    static constexpr int BK = 128;  // bytes of a row per pair
    // LDS buffers: 96 to 128 KB
    static constexpr int NS = BM + BN > 320 ? 2 : BM + BN > 192 ? 3 : 4;
    static constexpr int WTN = BN / 2, WTM = BM / 2;
    static constexpr int TN = WTN / 32, TM = WTM / 32;
    static constexpr int WI = BN / 8 / 4, XI = BM / 8 / 4;  // LDS-DMA requests per wave and pair
    static constexpr int LPS = WI + XI;
    static constexpr int STAGE_W = BN * BK, STAGE = (BN + BM) * BK;
    static constexpr int ES = MODE == OUT_F32 ? 4 : 2;
    // LDS: ring | token scales [SG][256] words | row indices [2][256] | tiles
    // ahead [4 waves][PLAN][8] | epilogue scratch | expert offsets
    static constexpr int SG = NS < 4 ? 4 : 8;  // more than NS
    static constexpr int SCALES = NS * STAGE;
    static constexpr int IDX = SCALES + SG * 1024;
    static constexpr int PLAN = 8;
    static constexpr int PLANS = IDX + 2 * 1024;
    static constexpr int SCRATCH = PLANS + 4 * PLAN * 32;
    static constexpr int SC_COLS = MODE == OUT_F32 ? 32 : 64;  // columns of a scratch block
    static constexpr int SC_ROW = (MODE == SWIGLU ? 64 : SC_COLS * ES) + 16;
    static constexpr int SC_WAVE = 32 * SC_ROW;
    // 16-byte stores of a tile's epilogue per wave (all are issued, whatever is valid)
    static constexpr int STORES = MODE == SWIGLU ? 2 * TM : TN * TM * (ES == 4 ? 4 : 2);
    static constexpr int SMAX = SCRATCH + 4 * SC_WAVE;
    static constexpr int INTS = SMAX + (MODE == SWIGLU ? 2 * BM * 4 : 0);
    static constexpr int LDS_BYTES = INTS + 3 * (kMaxExperts + 1) * 4;
    static_assert(LDS_BYTES <= 160 * 1024, "LDS of a compute unit");
};

struct Tile {
    int e;           // expert of the launch
    int64_t r0, n0;  // first product row, first output column
    int m_valid, n_valid;
};

// The tiles of all experts, BM token rows high.  TAIL: an expert's last rows,
// where they fill at most half a tile and are all it has or follow at least
// four whole tiles, are no tile of it but a tail; the tails run behind the
// tiles, as tiles of half the height and a fraction of the time, and are dealt
// out from the first workgroup that the tiles' last round leaves without one.
// So experts of few rows cost less, and the last round is a short one instead
// of a whole one: DBRX gate of 8192 tokens (768 tiles, 54 tails, 256
// workgroups) 288 -> 275 us.  Behind fewer tiles, reading the weights again
// costs more than it saves: DeepSeekV2 FFN of 8192 tokens (a tile and some 50
// rows per expert) 241 -> 256.
template <class C, bool TAIL>
struct Walk {
    int *s_off, *s_tile, *s_tail;  // e_count + 1 ints each in LDS
    int NT, tiles, tails;
    static __device__ __forceinline__ int tile_rows(int cnt) {
        const int n = cnt / C::BM, rest = cnt % C::BM;
        const bool tail = TAIL && rest <= C::BM / 2 && (n == 0 || n >= 4);
        return n + (rest > 0 && !tail);
    }
    __device__ __forceinline__ Walk(const ScaledGemm &g, int *lds) {
        s_off = lds;
        s_tile = lds + kMaxExperts + 1;
        s_tail = lds + 2 * (kMaxExperts + 1);
        NT = (g.N + C::BNOUT - 1) / C::BNOUT;
        const int tid = threadIdx.x, lane = tid & 63;
        for (int i = tid; i <= g.e_count; i += C::THREADS)
            s_off[i] = g.offsets ? g.offsets[g.e_first + i] : (i == 0 ? 0 : (int)g.rows_one);
        __syncthreads();
        // inclusive prefix sums over the experts, one per thread
        int f = 0, h = 0;
        if (tid < g.e_count) {
            const int cnt = s_off[tid + 1] - s_off[tid];
            const int n = tile_rows(cnt);
            f = n * NT;
            h = ((cnt + C::BM - 1) / C::BM - n) * NT;
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int uf = __shfl_up(f, d), uh = __shfl_up(h, d);
            if (lane >= d) f += uf, h += uh;
        }
        s_tile[tid + 1] = f;
        s_tail[tid + 1] = h;
        if (tid == 0) s_tile[0] = s_tail[0] = 0;
        if (g.e_count > 64) {
            __syncthreads();
            for (int w = 64; w <= tid - lane; w += 64) f += s_tile[w], h += s_tail[w];
            __syncthreads();
            s_tile[tid + 1] = f;
            s_tail[tid + 1] = h;
        }
        __syncthreads();
        tiles = __builtin_amdgcn_readfirstlane(s_tile[g.e_count]);
        tails = __builtin_amdgcn_readfirstlane(s_tail[g.e_count]);
    }
    // Tails of 128 columns instead of BNOUT.
    __device__ __forceinline__ int narrow_tails(const ScaledGemm &g) const {
        return tails / NT * ((g.N + 127) / 128);
    }
    __device__ __forceinline__ void narrow(const ScaledGemm &g) {
        const int n = (g.N + 127) / 128;
        __syncthreads();
        for (int i = threadIdx.x; i <= g.e_count; i += C::THREADS) s_tail[i] = s_tail[i] / NT * n;
        __syncthreads();
        tails = tails / NT * n;
    }
    // tile tau of the tiles (tail false) or of the tails, of BN columns
    template <int BN>
    __device__ __forceinline__ Tile tile(const ScaledGemm &g, int tau, bool tail) const {
        auto lds = [](const int &v) { return __builtin_amdgcn_readfirstlane(v); };
        const int *pre = tail ? s_tail : s_tile;
        int lo = 0, hi = g.e_count - 1;  // the last expert with pre[e] <= tau
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (lds(pre[mid]) <= tau) lo = mid; else hi = mid - 1;
        }
        const int row0 = lds(s_off[lo]);
        const int cnt = lds(s_off[lo + 1]) - row0;
        int mt = cnt / C::BM, nt = tau - lds(pre[lo]);
        if (!tail) {
            const int MT = tile_rows(cnt), per_sc = GROUP_N * MT;
            const int sc = nt / per_sc, q = nt - sc * per_sc;
            const int width = min(GROUP_N, NT - sc * GROUP_N);
            mt = q / width;
            nt = sc * GROUP_N + (q - mt * width);
        }
        Tile t;
        t.e = lo;
        t.r0 = (int64_t)row0 + (int64_t)mt * C::BM;
        t.n0 = (int64_t)nt * BN;
        t.m_valid = min(C::BM, cnt - mt * C::BM);
        t.n_valid = min(BN, (int)(g.N - t.n0));
        return t;
    }
};

typedef const __attribute__((address_space(4))) uint32_t *scalar_words;

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// TAIL: the tiles are the walk's tails.
template <int MODE, int BM_, int BN_, bool TAIL, class W>
struct TileLoop {
    using C = Cfg<MODE, BM_, BN_>;
    struct FragsA {
        u32x4 v[C::TN][2];
    };
    struct FragsB {
        u32x4 v[C::TM][2];
    };

    const ScaledGemm &g;
    const W &walk;
    char *smem;
    const int total;
    uint32_t lds0;
    int lane, wave, wn, wm, K, SK, np, G;

    // load side: the tile whose pairs are being requested, and its number
    int l_tau, l_n, l_kp, l_slot, l_group, l_idx;
    u32x4 wres, xres, sres;
    uint32_t woff[C::WI], xoff[C::XI], soff, upper;

    // compute side
    int c_slot, c_group, c_byte;
    floatx16 acc[C::TN][C::TM];
    int sx[C::TM], sxn[C::TM];

    __device__ __forceinline__ TileLoop(const ScaledGemm &g_, const W &w_, char *sm)
        : g(g_), walk(w_), smem(sm), total(TAIL ? w_.tails : w_.tiles) {
        lds0 = (uint32_t)(uintptr_t)(lds_void_t *)sm;
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        wn = wave & 1, wm = wave >> 1;
        K = g.K, SK = scale_pitch(K), np = scale_blocks(K);
        G = gridDim.x;
        l_slot = l_group = l_idx = 0;
        c_slot = c_group = c_byte = 0;
    }

    // The workgroup's n-th tile is found once, ahead of its first request, and
    // kept in LDS (each wave for itself: no barrier); the gather's row indices
    // (behind the last row: the last one's) are requested with it.
    __device__ __forceinline__ int *plan(int n) const {
        return reinterpret_cast<int *>(smem + C::PLANS) +
               (wave * C::PLAN + (n & (C::PLAN - 1))) * 8;
    }
    __device__ __forceinline__ void plan_tile(int tau, int n, int which) {
        if (tau >= total) return;
        const Tile t = walk.template tile<C::BNOUT>(g, tau, TAIL);
        int *p = plan(n);
        p[0] = t.e;
        p[1] = (int)t.r0;
        p[2] = (int)t.n0;
        p[3] = t.m_valid;
        p[4] = t.n_valid;
        if (!g.row_map) return;
        const uint32_t r = (uint32_t)min(wave * 64 + lane, t.m_valid - 1) * 4u;
        buf4_to_lds(buf_rsrc(g.row_map + t.r0), r, 0,
                    lds0 + C::IDX + which * 1024 + wave * 256);
    }
    __device__ __forceinline__ Tile planned(int n) const {
        const int *p = plan(n);
        auto at = [&](int i) { return __builtin_amdgcn_readfirstlane(p[i]); };
        return Tile{at(0), at(1), at(2), at(3), at(4)};
    }

    // Operand addresses of tile l_tau.  A request copies 8 rows of 128 bytes;
    // the 16-byte chunks of LDS row r are stored at chunk ^ (r / 2 % 8), so
    // the 16 lanes of a fragment read that are served together find all banks.
    __device__ __forceinline__ void bind() {
        const Tile t = planned(l_n);
        const int64_t we = (int64_t)(g.e_first + t.e) * g.N + t.n0;
        const bool up = MODE == SWIGLU && wave >= 2;
        const int wrow0 = (MODE == SWIGLU ? wave & 1 : wave) * (C::BN / 4);
        wres = buf_rsrc((up ? g.w1 : g.w0) + we * K);
        int ln = threadIdx.x & 63;  // opaque: its products are not kept over the K loop
        asm volatile("" : "+v"(ln));
        const int drow = ln >> 3;
        // LDS rows 8 i + drow: r / 2 % 8 is drow / 2 + 4 (i % 2)
        const uint32_t c0 = (uint32_t)((ln & 7) ^ (drow >> 1)), c1 = c0 ^ 4u;
#pragma unroll
        for (int i = 0; i < C::WI; ++i)
            woff[i] = (uint32_t)(min(wrow0 + i * 8 + drow, t.n_valid - 1) * K) +
                      (i & 1 ? c1 : c0) * 16u;
        // where K ends inside a pair: how far a chunk of the missing half is
        // moved back (one of the two chunks c0, c1 always is)
        upper = c0 & 4u;
        const int srow = min(wave * 64 + ln, t.m_valid - 1);
        if (g.row_map) {
            const int *idx = reinterpret_cast<const int *>(smem + C::IDX + l_idx * 1024);
            xres = buf_rsrc(g.x);
            sres = buf_rsrc(g.xs);
#pragma unroll
            for (int i = 0; i < C::XI; ++i)
                xoff[i] = (uint32_t)(idx[(wave * C::XI + i) * 8 + drow] / g.slot_div) *
                              (uint32_t)K + (i & 1 ? c1 : c0) * 16u;
            soff = (uint32_t)(idx[srow] / g.slot_div) * (uint32_t)SK;
        } else {
            xres = buf_rsrc(g.x + t.r0 * K);
            sres = buf_rsrc(g.xs + t.r0 * SK);
#pragma unroll
            for (int i = 0; i < C::XI; ++i)
                xoff[i] = (uint32_t)(min((wave * C::XI + i) * 8 + drow, t.m_valid - 1) * K) +
                          (i & 1 ? c1 : c0) * 16u;
            soff = (uint32_t)(srow * SK);
        }
        l_kp = 0;
    }
    __device__ __forceinline__ static int next(int slot) {
        return slot == C::NS - 1 ? 0 : slot + 1;
    }
    // Behind a pair's requests: the next tile's first pair follows the last one
    // (behind the last tile: its last pair again, which nothing reads).
    __device__ __forceinline__ void advance() {
        l_slot = next(l_slot);
        if (++l_kp < np) return;
        if (l_tau + G >= total) {
            l_kp = np - 1;
            return;
        }
        l_tau += G;
        l_n += 1;
        l_idx ^= 1;
        // Its indices were requested at the last crossing, np pairs ago; the waits in
        // between let AHEAD requests stay on their way, those of NS - 2 pairs and a
        // token tile.  So they cover the indices only where np >= NS - 1.
        if (np < C::NS - 1 && g.row_map) landed<0>();
        bind();
        plan_tile(l_tau + G, l_n + 1, l_idx ^ 1);
    }
    __device__ __forceinline__ void request_scales() {
        if (l_kp & 3) return;
        buf4_to_lds(sres, soff, (uint32_t)l_kp,
                    lds0 + C::SCALES + l_group * 1024 + wave * 256);
        l_group = (l_group + 1) & (C::SG - 1);
    }
    // Where the pair has one half only, the other half's chunks read that one
    // (nothing uses them): how far back, for even and odd requests.
    __device__ __forceinline__ void backs(uint32_t &back0, uint32_t &back1) const {
        const bool half = (l_kp + 1) * C::BK > K;
        back0 = half ? upper * 16u : 0u;
        back1 = half ? (upper ^ 4u) * 16u : 0u;
    }
    __device__ __forceinline__ void request_w(int i, uint32_t back0, uint32_t back1) {
        buf16_to_lds(wres, woff[i] - (i & 1 ? back1 : back0), (uint32_t)l_kp * C::BK,
                     lds0 + (uint32_t)l_slot * C::STAGE + (wave * C::WI + i) * 1024);
    }
    __device__ __forceinline__ void request_x(int i, uint32_t back0, uint32_t back1) {
        buf16_to_lds(xres, xoff[i] - (i & 1 ? back1 : back0), (uint32_t)l_kp * C::BK,
                     lds0 + (uint32_t)l_slot * C::STAGE + C::STAGE_W +
                         (wave * C::XI + i) * 1024);
    }
    __device__ __forceinline__ void request_all_x() {
        request_scales();
        uint32_t b0, b1;
        backs(b0, b1);
#pragma unroll
        for (int i = 0; i < C::XI; ++i) request_x(i, b0, b1);
    }
    __device__ __forceinline__ void request_pair() {
        request_all_x();
        uint32_t b0, b1;
        backs(b0, b1);
#pragma unroll
        for (int i = 0; i < C::WI; ++i) request_w(i, b0, b1);
        advance();
    }

    // first token row of the wave's fragment j
    __device__ __forceinline__ int row0(int j) const { return (2 * j + wm) * 32; }
    // 16 bytes (h of 2) of a fragment, half `hf` of the pair in c_slot
    __device__ __forceinline__ u32x4 read(int lds_row, int h, int hf) const {
        const int row = lane & 31;
        const int chunk = ((hf * 4 + (lane >> 5) * 2 + h) ^ ((row >> 1) & 7)) * 16;
        return *reinterpret_cast<const u32x4 *>(smem + c_slot * C::STAGE +
                                                (lds_row + row) * C::BK + chunk);
    }
    __device__ __forceinline__ void read_a(FragsA &f, int r, int hf) const {
        const int i = r >> 1;
        const int w0 = MODE == SWIGLU ? (i >= 2 ? 128 : 0) + wn * 64 + (i & 1) * 32
                                      : wn * C::WTN + i * 32;
        f.v[i][r & 1] = read(w0, r & 1, hf);
    }
    __device__ __forceinline__ void read_b(FragsB &f, int r, int hf) const {
        f.v[r >> 1][r & 1] = read(C::BN + row0(r >> 1), r & 1, hf);
    }
    __device__ __forceinline__ void read_scales(int (&s)[C::TM]) {
        const uint8_t *p = reinterpret_cast<const uint8_t *>(smem) + C::SCALES +
                           c_group * 1024 + c_byte;
#pragma unroll
        for (int j = 0; j < C::TM; ++j) s[j] = p[(row0(j) + (lane & 31)) * 4];
    }
    __device__ __forceinline__ static v8i whole(const u32x4 (&v)[2]) {
        return v8i{(int)v[0][0], (int)v[0][1], (int)v[0][2], (int)v[0][3],
                   (int)v[1][0], (int)v[1][1], (int)v[1][2], (int)v[1][3]};
    }

    // The gate/up launch of few rows per expert (64-row tiles) is bound by the
    // weight stream, so its products can be exact: e4m3 widened to bf16, in which
    // products and sums are exact to fp32, at half the rate.  An error of 2e-5 of
    // a sum, which the 8-bit instruction has, moves one quantised value in
    // some thousands to its neighbour, which a row of few large values shows
    // (DBRX FFN of 64 tokens: off by 1.9 to 3.7e-3 with it, 1.7e-3 without, all of
    // that the output's bf16), at 3% of the time (93.8 -> 96.7 us); with more rows
    // the matrix cores are the bound, and the 8-bit products stay (the FFN's rows are
    // off by 2.0 to 2.5e-3 then).
    static constexpr bool EXACT = MODE == SWIGLU && BM_ == 64;
    // e4m3 values of a lane's 32 bytes, 8 (part) to 8 (part) + 7, times scale
    __device__ __forceinline__ static bf16x8 widen(const u32x4 (&v)[2], int part, float scale) {
        const uint32_t lo = v[part >> 1][2 * (part & 1)], hi = v[part >> 1][2 * (part & 1) + 1];
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
        const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
        const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
        return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    // A scale byte as the float whose exponent it is.  Both operands carry their
    // own: as one factor the product of two could leave the exponent's range.
    __device__ __forceinline__ static float scale(int s) {
        return __uint_as_float((uint32_t)s << 23);
    }
    // e4m3 values are 2^-9 to 448, so with bytes of 10 to 246 they are normal bf16
    // numbers.  Rows that meet another byte in a tile (a block whose largest value is
    // below 2^-108 or above 2^119; far: their lanes) get sums taken from memory again,
    // the scales applied to each block's fp32 sums as the few rows' kernels do.
    // Watching for them costs 1%, a few such rows 80% (DBRX FFN of 64 tokens 103 -> 187
    // us; a byte of every row 245): a chain of loads as long as K.  (Scaling every block's sums in the loop, or a branch
    // there to the 8-bit instruction, moves the accumulators about in every half: DBRX
    // FFN of 64 tokens 89 -> 121 to 127 us.)
    uint64_t far;
    __device__ __forceinline__ void note_far(int sw0, int sw1) {
        auto out = [](int s) { return (uint32_t)(s - 10) > 236u; };
        far |= __builtin_amdgcn_ballot_w64(out(sx[0]) || out(sw0) || out(sw1));
    }
    __device__ __forceinline__ void sums_of_far(const Tile &t) {
        const int row = min(row0(0) + (lane & 31), t.m_valid - 1);
        const int64_t src = g.row_map ? g.row_map[t.r0 + row] / g.slot_div : t.r0 + row;
        const int64_t we = (int64_t)(g.e_first + t.e) * g.N + t.n0;
        const int64_t se = (int64_t)(g.e_first + t.e) * scale_blocks(g.N) + t.n0 / kScaleBlock;
        const uint8_t *xp = g.x + src * K + (lane >> 5) * 32;
        const uint8_t *wp[C::TN];
        floatx16 sum[C::TN];
#pragma unroll
        for (int i = 0; i < C::TN; ++i) {
            const int wrow = min(wn * 64 + (i & 1) * 32 + (lane & 31), t.n_valid - 1);
            wp[i] = (i >= 2 ? g.w1 : g.w0) + (we + wrow) * K + (lane >> 5) * 32;
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[i][r] = 0.f;
        }
        for (int kb = 0; kb < np; ++kb) {
            const int st = g.xs[src * SK + kb];
            const int k[2] = {kb * C::BK, min(kb * C::BK + 64, K - 64)};
            const bool one = k[0] == k[1];  // half a block: its one half again, unused
            u32x4 b[2][2], a[C::TN][2][2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    b[h][c] = reinterpret_cast<const u32x4 *>(xp + k[h])[c];
#pragma unroll
                    for (int i = 0; i < C::TN; ++i)
                        a[i][h][c] = reinterpret_cast<const u32x4 *>(wp[i] + k[h])[c];
                }
#pragma unroll
            for (int i = 0; i < C::TN; ++i) {
                const int sw = (i >= 2 ? g.s1 : g.s0)[se * SK + kb];
                floatx16 p;
#pragma unroll
                for (int r = 0; r < 16; ++r) p[r] = 0.f;
#pragma unroll
                for (int h = 0; h < 8; ++h)
                    if (h < 4 || !one)
                        p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            widen(a[i][h >> 2], h & 3, 1.f), widen(b[h >> 2], h & 3, 1.f), p, 0, 0,
                            0);
                const float nan = sw == 255 || st == 255 ? __builtin_nanf("") : 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    sum[i][r] += __builtin_amdgcn_ldexpf(p[r] + nan, st + sw - 254);
            }
        }
        const bool mine = far >> lane & 1;
#pragma unroll
        for (int i = 0; i < C::TN; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][0][r] = mine ? sum[i][r] : acc[i][0][r];
    }
    // One half's MFMAs, and between them the parts f(m) of NM of its reads and
    // requests.  (The sums count as used behind them: the compiler would move the
    // MFMAs behind branches that follow, away from those.)
    static constexpr int NM = C::TN * C::TM * (EXACT ? 4 : 1);
    template <class F>
    __device__ __forceinline__ void half(const FragsA &a, const FragsB &b, int sw0, int sw1,
                                         F &&f) {
        if constexpr (EXACT) {
            static_assert(C::TM == 1, "one token fragment");
            const float st = scale(sx[0]), sg = scale(sw0), su = scale(sw1);
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const bf16x8 bt = widen(b.v[0], h, st);
#pragma unroll
                for (int i = 0; i < C::TN; ++i) {
                    acc[i][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        widen(a.v[i], h, i >= 2 ? su : sg), bt, acc[i][0], 0, 0, 0);
                    f(h * C::TN + i);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        } else {
#pragma unroll
            for (int m = 0; m < NM; ++m) {
                const int i = m / C::TM, j = m % C::TM;
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                    whole(a.v[i]), whole(b.v[j]), acc[i][j], 0, 0, 0,
                    MODE == SWIGLU && i >= 2 ? sw1 : sw0, 0, sx[j]);
                f(m);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int i = 0; i < C::TN; ++i)
#pragma unroll
            for (int j = 0; j < C::TM; ++j) asm volatile("" : "+a"(acc[i][j]));
    }
    // requests younger than the next pair's once a pair's token rows are requested
    static constexpr int AHEAD = C::XI + (C::NS - 2) * C::LPS;
    // Part m of NM of N things; EARLY: all of them in the first three quarters
    // (the last MFMAs then hide the reads' latency).
    template <int N, bool EARLY, class F>
    __device__ __forceinline__ static void part(int m, F &&f) {
        constexpr int M = EARLY ? NM * 3 / 4 : NM;
        if (m >= M) return;
#pragma unroll
        for (int q = m * N / M; q < (m + 1) * N / M; ++q) f(q);
    }

    // The first half of a pair.  The token rows of its buffer are in registers
    // (both halves' fragments), so those of the pair NS ahead are
    // requested into it; the other half's weight fragments are read.  Behind
    // it no wave needs the pair's buffer, and the next pair has landed for
    // every wave.  stored: the epilogue's stores, younger than that pair's
    // requests, may still be on their way.
    __device__ __forceinline__ void first_half(const FragsA &a, const FragsB &b,
                                               FragsA &a2, int sw0, int sw1, bool stored) {
        request_scales();
        uint32_t b0, b1;
        backs(b0, b1);
        half(a, b, sw0, sw1, [&](int m) {
            part<2 * C::TN, true>(m, [&](int r) { read_a(a2, r, 1); });
            part<C::XI, false>(m, [&](int q) { request_x(q, b0, b1); });
        });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (stored)
            wait_vmcnt<(AHEAD + C::STORES < 63 ? AHEAD + C::STORES : 63)>();
        else
            wait_vmcnt<AHEAD>();
        __builtin_amdgcn_s_barrier();
    }
    // The second half: the weights of the pair NS ahead are requested,
    // and the next pair's token fragments read for both halves (b, b2) and its
    // weights' for the first (a).  Behind it every wave has its token rows.
    __device__ __forceinline__ void second_half(const FragsA &ca, const FragsB &cb,
                                                FragsA &a, FragsB &b, FragsB &b2, int sw0,
                                                int sw1) {
        uint32_t b0, b1;
        backs(b0, b1);
        if constexpr (EXACT) note_far(sw0, sw1);
        c_slot = next(c_slot);
        half(ca, cb, sw0, sw1, [&](int m) {
            part<2 * C::TN + 4 * C::TM, true>(m, [&](int r) {
                if (r < 4 * C::TM)
                    read_b(r & 1 ? b2 : b, r >> 1, r & 1);
                else
                    read_a(a, r - 4 * C::TM, 0);
            });
            part<C::WI, false>(m, [&](int q) { request_w(q, b0, b1); });
        });
        advance();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
    }
    // Every wave's requests so far but the youngest N have landed, and its LDS
    // reads are done.
    template <int N>
    __device__ __forceinline__ void landed() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        wait_vmcnt<N>();
        __builtin_amdgcn_s_barrier();
    }
};

// Between the steps of an epilogue block: a wave's LDS accesses stay in order,
// and no later block's accumulators are taken up early.
__device__ __forceinline__ void block_end() {
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_sched_barrier(0);
}

// Keeps an accumulator in the matrix cores' registers up to here: the ones of
// all blocks do not fit the others beside the next tile's fragments.
__device__ __forceinline__ void in_place(floatx16 &v) { asm volatile("" : "+a"(v)); }

template <int MODE, class L>
__device__ __forceinline__ void epilogue(const ScaledGemm &g, const Tile &t, L &loop, char *smem) {
    using C = typename L::C;
    int lane = threadIdx.x & 63;  // opaque: its products are not kept over the K loop
    asm volatile("" : "+v"(lane));
    const int wave = loop.wave, wn = loop.wn, half = lane >> 5;
    auto &acc = loop.acc;
    // The lane holds, of token row row0(j) + lane % 32, the weight rows
    // 32 i + 8 (r / 4) + 4 (lane / 32) + r % 4.
    char *sc = smem + C::SCRATCH + wave * C::SC_WAVE;
    // every store is issued, since the waits count them: what is not valid gets
    // an offset past the resource's range, which drops it
    constexpr uint32_t RANGE = 0xFFFFFFF0u, DROP = 0xFFFFFFF8u;
    const __amdgpu_buffer_rsrc_t ores = __builtin_amdgcn_make_buffer_rsrc(
        (char *)g.out + (t.r0 * g.N + t.n0) * (MODE == SWIGLU ? 1 : C::ES), 0, (int)RANGE,
        kBufferFlags);
    auto store = [&](const u32x4 &v, bool valid, uint32_t off) {
        __builtin_amdgcn_raw_buffer_store_b128(v, ores, valid ? off : DROP, 0, 0);
    };
    if constexpr (MODE == SWIGLU) {
        float *smax = reinterpret_cast<float *>(smem + C::SMAX);  // [2][BM]
#pragma unroll
        for (int j = 0; j < C::TM; ++j) {
            float m = 0.f;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                in_place(acc[i][j]);
                in_place(acc[i + 2][j]);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float h = wn * 64 + i * 32 < t.n_valid
                                        ? silu_mul(acc[i][j][r], acc[i + 2][j][r])
                                        : 0.f;
                    acc[i][j][r] = h;
                    m = fmaxf(m, fabsf(h));
                }
                in_place(acc[i][j]);
            }
            m = fmaxf(m, __shfl_xor(m, 32));
            if (half == 0) smax[wn * C::BM + loop.row0(j) + lane] = m;
            __builtin_amdgcn_sched_barrier(0);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
#pragma unroll
        for (int j = 0; j < C::TM; ++j) {
            const int row = loop.row0(j) + (lane & 31);
            const int e = scale_exponent(fmaxf(smax[row], smax[C::BM + row]));
            const float inv = scale_inverse(e);
            if (wn == 0 && half == 0 && row < t.m_valid)
                g.out_s[(t.r0 + row) * scale_pitch(g.N) + t.n0 / kScaleBlock] = scale_byte(e);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                in_place(acc[i][j]);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    *reinterpret_cast<uint32_t *>(sc + (lane & 31) * C::SC_ROW + i * 32 + r * 8 +
                                                  half * 4) =
                        pack_e4m3(acc[i][j][4 * r], acc[i][j][4 * r + 1], acc[i][j][4 * r + 2],
                                  acc[i][j][4 * r + 3], inv);
            }
            block_end();
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int rr = q * 16 + (lane >> 2), chunk = lane & 3;
                const u32x4 v = *reinterpret_cast<const u32x4 *>(sc + rr * C::SC_ROW + chunk * 16);
                const int orow = loop.row0(j) + rr;
                store(v, orow < t.m_valid && wn * 64 < t.n_valid,
                      (uint32_t)(orow * g.N + wn * 64 + chunk * 16));
            }
            block_end();
        }
        // (the next tile's maxima are written many barriers from here)
    } else {
        constexpr int IB = C::SC_COLS / 32;                  // fragments of a scratch block
        constexpr int CPR = C::SC_COLS * C::ES / 16, RPI = 64 / CPR;  // chunks per row, rows a pass
#pragma unroll
        for (int j = 0; j < C::TM; ++j)
#pragma unroll
            for (int ib = 0; ib < C::TN; ib += IB) {
#pragma unroll
                for (int i = 0; i < IB; ++i) {
                    in_place(acc[ib + i][j]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const floatx16 &v = acc[ib + i][j];
                        char *p = sc + (lane & 31) * C::SC_ROW + (i * 32 + r * 8 + half * 4) * C::ES;
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
                }
                block_end();
#pragma unroll
                for (int q = 0; q < 32 / RPI; ++q) {
                    const int rr = q * RPI + lane / CPR, chunk = lane % CPR;
                    const int row = loop.row0(j) + rr;
                    const int col = wn * C::WTN + ib * 32 + chunk * (16 / C::ES);
                    const u32x4 v =
                        *reinterpret_cast<const u32x4 *>(sc + rr * C::SC_ROW + chunk * 16);
                    store(v, row < t.m_valid && col < t.n_valid,
                          (uint32_t)(row * g.N + col) * C::ES);
                }
                block_end();
            }
    }
}

// The workgroup's share of the tiles, or of the tails: `first` and every
// gridDim.x-th one behind it.
template <int MODE, int BM_, int BN_, bool TAIL, class W>
__device__ __forceinline__ void run_tiles(const ScaledGemm &g, const W &walk, int first,
                                          char *smem) {
    using L = TileLoop<MODE, BM_, BN_, TAIL, W>;
    using C = typename L::C;
    L t(g, walk, smem);
    if (first >= t.total) return;
    t.l_tau = first;
    t.l_n = 0;
    // Where a tile has at most NS pairs, the first requests reach the second tile
    // and those behind it.  So the second tile's indices are waited for with the
    // first one's; the third tile's, which take the first one's place, are requested
    // once every wave has read those; and a wait behind each pair covers the ones
    // requested on the way.
    t.plan_tile(first, 0, 0);
    t.plan_tile(first + t.G, 1, 1);
    t.template landed<0>();
    t.bind();
    if (g.row_map && t.np <= C::NS) t.template landed<0>();
#pragma unroll
    for (int i = 0; i < C::NS; ++i) {
        t.request_pair();
        if (i == C::NS - 1 || (g.row_map && t.np < C::NS)) t.template landed<0>();
    }
    typename L::FragsA a0, a1;
    typename L::FragsB b0, b1, n1;
#pragma unroll
    for (int r = 0; r < 2 * C::TN; ++r) t.read_a(a0, r, 0);
#pragma unroll
    for (int r = 0; r < 2 * C::TM; ++r) {
        t.read_b(b0, r, 0);
        t.read_b(b1, r, 1);
    }
    t.read_scales(t.sx);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();

    // a tile's weight scales, a word for four pairs, and the first words
    scalar_words ws0, ws1 = nullptr;
    uint32_t w0, w1 = 0;
    auto first_words = [&](const Tile &tile) {
        const int64_t nb = (int64_t)(g.e_first + tile.e) * scale_blocks(g.N) +
                           min((int)(tile.n0 / kScaleBlock) + (C::WTN == 128 && MODE != SWIGLU ? t.wn : 0),
                               scale_blocks(g.N) - 1);
        auto words = [&](const uint8_t *s) {
            const uint64_t a = (uint64_t)(uintptr_t)(s + nb * t.SK);
            return (scalar_words)(uintptr_t)(
                (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)a) |
                (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32)) << 32);
        };
        ws0 = words(g.s0);
        w0 = ws0[0];
        if (MODE == SWIGLU) {
            ws1 = words(g.s1);
            w1 = ws1[0];
        }
    };
    first_words(t.planned(0));

    for (int tau = first, n = 0; tau < t.total; tau += t.G, ++n) {
        // the next pair's scales of the tokens, and behind the pair of the weights
        auto next_scales = [&](int p) {
            if (p + 1 >= t.np || t.c_byte == 3) {
                t.c_byte = 0;
                t.c_group = (t.c_group + 1) & (C::SG - 1);
            } else {
                t.c_byte += 1;
            }
            t.read_scales(t.sxn);
        };
        auto next_words = [&](int p) {
            w0 >>= 8, w1 >>= 8;
            if ((p & 3) == 3 && p + 1 < t.np) {
                w0 = ws0[(p + 1) >> 2];
                if (MODE == SWIGLU) w1 = ws1[(p + 1) >> 2];
            }
#pragma unroll
            for (int j = 0; j < C::TM; ++j) t.sx[j] = t.sxn[j];
        };
#pragma unroll
        for (int i = 0; i < C::TN; ++i)
#pragma unroll
            for (int j = 0; j < C::TM; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) t.acc[i][j][r] = 0.f;
        t.far = 0;
        // b1: the pair's second half's token fragments, n1: the next one's
        auto pair = [&](int p, typename L::FragsB &b1, typename L::FragsB &n1) {
            const int s0 = w0 & 255, s1 = w1 & 255;
            t.first_half(a0, b0, a1, s0, s1, p == 0 && tau != first);
            next_scales(p);
            t.second_half(a1, b1, a0, b0, n1, s0, s1);
            next_words(p);
        };
        const int whole = t.K / C::BK;
        int p = 0;
        for (; p + 1 < whole; p += 2) {
            pair(p, b1, n1);
            pair(p + 1, n1, b1);
        }
        if (p < whole) {
            pair(p, b1, n1);
            b1 = n1;
        }
        if (whole < t.np) {  // half a pair
            t.request_all_x();
            t.template landed<L::AHEAD>();
            next_scales(whole);
            a1 = a0;
            typename L::FragsB c0 = b0;
            t.second_half(a1, c0, a0, b0, b1, w0 & 255, w1 & 255);
            next_words(whole);
        }
        const Tile tile = t.planned(n);
        if (tau + t.G < t.total) first_words(t.planned(n + 1));  // (bound by now)
        if constexpr (L::EXACT)
            if (t.far) t.sums_of_far(tile);
        epilogue<MODE>(g, tile, t, smem);
    }
    t.template landed<0>();  // requests behind the last pair
}

template <int MODE, int BM_, int BN_>
__global__ __launch_bounds__(256, 1) void tile_kernel(ScaledGemm g) {
    using C = Cfg<MODE, BM_, BN_>;
    constexpr bool TAILS = BM_ > 128;
    __shared__ __attribute__((aligned(16))) char smem[C::LDS_BYTES];
    using W = Walk<C, TAILS>;
    W walk(g, reinterpret_cast<int *>(smem + C::INTS));
    // neighbouring tiles on one XCD
    const int G = gridDim.x;  // a multiple of NXCD
    const int slot = (blockIdx.x % NXCD) * (G / NXCD) + blockIdx.x / NXCD;
    run_tiles<MODE, BM_, BN_, false>(g, walk, slot, smem);
    if constexpr (TAILS) {
        static_assert(Cfg<MODE, 128, BN_>::INTS <= C::INTS, "the offsets lie behind every layout");
        if (walk.tails == 0) return;
        const int used = walk.tiles % G, left = used ? G - used : 0;
        const int from = slot >= used ? slot - used : slot + G - used;
        // Where the tails need a round of their own, ones of half the columns that
        // fit into it shorten it (DBRX gate of 8192 tokens 270 -> 253 us).  Where
        // they do not fit, or run beside the last tiles, whole ones do less work.
        // (The SwiGLU tile's columns are one scale block: it has no half.)
        if constexpr (MODE != SWIGLU && BM_ == 256) {
            static_assert(Cfg<MODE, 128, 128>::INTS <= C::INTS, "and this one");
            if (walk.tails > left && walk.narrow_tails(g) <= G + left) {
                walk.narrow(g);
                run_tiles<MODE, 128, 128, true>(g, walk, from, smem);
                return;
            }
        }
        run_tiles<MODE, 128, BN_, true>(g, walk, from, smem);
    }
}

// Tile rows of all experts at a height of bm, expected under uniform routing: an
// expert's rows are then about normal with the mean m and the variance v.
double expected_tile_rows(const ScaledLoad &l, int bm) {
    if (l.rows <= 0) return 0;
    const double m = l.rows / l.experts, p = std::min(1.0, m / (double)l.max_rows);
    const double v = m * (1 - p);
    if (v < 1e-9 || m > 64.0 * bm)
        return l.experts * (v < 1e-9 ? std::ceil(m / bm) : m / bm + 0.5);
    double rows = l.active / l.experts;  // P(any)
    for (int j = 1; j * (double)bm < m + 6 * std::sqrt(v) + 1; ++j)  // + P(more than j bm)
        rows += 0.5 * std::erfc((j * (double)bm + 0.5 - m) / std::sqrt(2 * v));
    return l.experts * rows;
}

// The tile of a launch: the one whose rounds over the chip are expected to take
// least, from the measured us per pair of K (a round of full tiles) and per tile.
// 256 x 256 (weight x token rows) does 1.0 of the work per time, 256 x 192 0.95,
// 256 x 128 0.8, 128 x 128 0.7 and 128 x 64 0.5, but more and smaller tiles fill
// the chip:
// 1500 x 4096 x 4096 (96, 192, 384 and 768 tiles) 52.2, 33.0, 36.3 and 41.7 us,
// 300 x 5120 x 1536 (40, 60, 120 and 200) 23.2, 15.8, 11.4 and 10.2.  A smaller
// tile has to promise an eighth less: a large one's rounds take less than
// counted where its rows are not all valid (DeepSeekV2 FFN of 8192 tokens, 307
// rows per expert: 239 us, with 128-row tiles counted 7% less 261).
// 192 token rows are for one group of rows, whose number is known: 5000 x 2048 x
// 2048 31.3 -> 25.8 us, 2500 x 4096 x 4096 53.4 -> 43.4, 1501 x 5120 x 1536 24.8 ->
// 20.6.  Over experts they gain while the loads are even (DeepSeekV2 FFN of 8192
// tokens 233 -> 215 us) and lose more where they are not, for the rounds that the
// fuller experts add (the same with exponents of 0.3 and, 4099 tokens, 1.1: 236 ->
// 266 and 213 -> 222).
struct Form {
    int bm, bn;
    double pair, tile;
};
int pick_form(const Form *forms, int count, const ScaledGemm &g, int columns,
              const ScaledLoad &load, unsigned grid) {
    int best = 0;
    double least = 0;
    for (int i = 0; i < count; ++i) {
        const Form &f = forms[i];
        if (f.bm == 192 && load.experts > 1) continue;
        const int nt = (g.N + (columns ? columns : f.bn) - 1) / (columns ? columns : f.bn);
        const double tiles = expected_tile_rows(load, f.bm) * nt;
        const double us = std::ceil(tiles / grid) * (scale_blocks(g.K) * f.pair + f.tile);
        if (i == 0 || us < 0.875 * least) {
            best = i;
            least = us;
        }
    }
    return best;
}

template <int MODE, int BM, int BN>
hipError_t go(const ScaledGemm &g, unsigned grid, hipStream_t s) {
    tile_kernel<MODE, BM, BN><<<grid, 256, 0, s>>>(g);
    return hipGetLastError();
}
unsigned tile_grid() { return (unsigned)std::max(NXCD, device_cu_count() / NXCD * NXCD); }

template <int MODE>
hipError_t go_out(const ScaledGemm &g, const ScaledLoad &load, hipStream_t s) {
    static const Form forms[] = {
        {256, 256, 1.48, 3.5}, {192, 256, 1.16, 3.3}, {128, 256, 0.90, 3.0},
        {128, 128, 0.55, 1.6}, {64, 128, 0.39, 1.6}};
    const unsigned grid = tile_grid();
    switch (pick_form(forms, 5, g, 0, load, grid)) {
        case 0: return go<MODE, 256, 256>(g, grid, s);
        case 1: return go<MODE, 192, 256>(g, grid, s);
        case 2: return go<MODE, 128, 256>(g, grid, s);
        case 3: return go<MODE, 128, 128>(g, grid, s);
        default: return go<MODE, 64, 128>(g, grid, s);
    }
}

}  // namespace

hipError_t launch_scaled_gemm(const ScaledGemm &g, int y_type, const ScaledLoad &load,
                              hipStream_t s) {
    return y_type == MOE_FP32 ? go_out<OUT_F32>(g, load, s) : go_out<OUT_BF16>(g, load, s);
}
hipError_t launch_scaled_swiglu(const ScaledGemm &g, const ScaledLoad &load, hipStream_t s) {
    static const Form forms[] = {
        {256, 256, 1.48, 4.5}, {128, 256, 0.90, 3.5}, {64, 256, 0.73, 3.0}};
    const unsigned grid = tile_grid();
    switch (pick_form(forms, 3, g, 128, load, grid)) {  // 128 gate and 128 up rows
        case 0: return go<SWIGLU, 256, 256>(g, grid, s);
        case 1: return go<SWIGLU, 128, 256>(g, grid, s);
        default: return go<SWIGLU, 64, 256>(g, grid, s);
    }
}

}  // namespace moe
