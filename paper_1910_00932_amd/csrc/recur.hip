// Gated linear recurrence over the frames of a clip, forward and backward.
//
//   a = sigmoid(g), k = 1 - a = sigmoid(-g);   h_t = a_t h_{t-1} + k_t x_t,  y_t = h_t
//   D_t = dy_t + E_{t+1},  E_t = a_t D_t (E_T = dh_last);   dx_t = k_t D_t,  dg_t = E_t k_t (h_{t-1} - x_t),  dh_0 = E_0
//
// Every value of a frame is a recurrence of its own ("column"), so both memory orders are the same [N][T][M] tensor, M = C*H*W.
// Both passes are bound by memory: forward reads x, g and writes y, backward reads x, g, dy and writes dx, dg.  The steps of a
// column are maps h -> A h + B, which join associatively: a block takes a tile of SEG segments of 8 steps times LC*4 columns, one
// thread per segment and four columns, holds the tile in registers, joins the segments' maps through LDS and runs every segment
// again from its true start.  Tiles follow one another in time with the state carried along, so each tensor is read once.  The
// state, the maps and what is carried are fp32 throughout; only y, dx and dg are rounded to the storage type.
// The backward pass needs h inside a tile: it starts from the states that the forward pass left every 128 steps (1.6 % of a bf16
// tensor), and forms h again from x and g, which it reads anyway, instead of reading y, which is rounded.
#include "internal.h"
#include "args.h"
#include "vec_any.h"

namespace tsm {

static constexpr int RC_NT = 256, RC_V = 4, RC_K = 8;     // threads, columns per thread, steps per thread
static constexpr int RC_SAVE = 128;                       // steps between saved states

struct RecurArgs {
    const void *x, *g, *dy;
    void *y, *dx, *dg;
    const float *h0, *dh_last;
    float *h_last, *dh0;
    float* saved;         // [N][(T-1)/RC_SAVE][M]: the state in front of step RC_SAVE*(j+1)
    float* maps;          // spans > 1: [N][spans][2][M], the spans' maps; behind them [N][M], the state in front of the first
    long M, cblocks, jobs;
    int N, T, spans, tiles_per_span;
};

// sigmoid(g) and 1 - sigmoid(g), neither by subtraction: e = exp(-|g|), 1/(1+e) and e/(1+e).  exp as 2^(hi+lo) with the product's
// rounding carried in lo (the low part of log2 e included), so that large |g| keep their relative precision; beyond 120 exp is
// zero in fp32 whatever it is.
__device__ __forceinline__ void gate(float g, float& a, float& k) {
    const float L2E = 1.44269502f, L2E_LO = 1.92596299e-8f, LN2 = 0.693147182f;
    const float m = fabsf(g) > 120.f ? 120.f : fabsf(g);
    const float hi = -m * L2E, lo = fmaf(-m, L2E, -hi) - m * L2E_LO;
    const float p = __builtin_amdgcn_exp2f(hi);
    const float e = fmaf(p, lo * LN2, p);
    const float big = __builtin_amdgcn_rcpf(1.f + e), small = e * big;
    a = g < 0.f ? small : big;
    k = g < 0.f ? big : small;
}

// The maps of the tile's segments, one parity per tile so that one barrier per tile is enough.
template <int SEG, int PLANES>
struct RecurLds {
    float4 m[2][SEG > 1 ? PLANES : 1][SEG > 1 ? SEG : 1][SEG > 1 ? RC_NT / SEG : 1];
};

__device__ __forceinline__ float4 pack4(const float (&f)[4]) { return make_float4(f[0], f[1], f[2], f[3]); }
__device__ __forceinline__ void load_state(const float* p, int nv, float (&f)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = p && e < nv ? p[e] : 0.f;
}
__device__ __forceinline__ void store_state(float* p, int nv, const float (&f)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < nv) p[e] = f[e];
}

template <typename T, int SEG>
__global__ void __launch_bounds__(RC_NT) recur_fwd_kernel(RecurArgs a) {
    constexpr int LC = RC_NT / SEG, STEPS = SEG * RC_K;
    typedef typename RawVec<T, RC_V>::type Raw;
    __shared__ RecurLds<SEG, 2> lds;
    const int lc = threadIdx.x % LC, seg = SEG == 1 ? 0 : threadIdx.x / LC;
    const int nsaved = (a.T - 1) / RC_SAVE;
    const int tiles = (a.T + STEPS - 1) / STEPS;
    int par = 0;
    for (long job = blockIdx.x; job < a.jobs; job += gridDim.x) {
        const long cb = job % a.cblocks;
        const int span = (int)(job / a.cblocks % a.spans);
        const long n = job / a.cblocks / a.spans;
        const long col = (cb * LC + lc) * RC_V;
        const int nv = (int)(a.M - col < RC_V ? a.M - col : RC_V);      // columns of this thread, none if not positive
        const T* x = (const T*)a.x + n * a.T * a.M + col;
        const T* g = (const T*)a.g + n * a.T * a.M + col;
        T* y = (T*)a.y + n * a.T * a.M + col;
        float c[4];                                                     // the state in front of the tile
        if (a.spans > 1) {
            const float* maps = a.maps + n * a.spans * 2 * a.M + col;
            load_state(a.maps + ((long)a.N * a.spans * 2 + n) * a.M + col, nv, c);
            for (int s = 0; s < span; ++s) {
                float A[4], B[4];
                load_state(maps + (long)s * 2 * a.M, nv, A);
                load_state(maps + ((long)s * 2 + 1) * a.M, nv, B);
#pragma unroll
                for (int e = 0; e < 4; ++e) c[e] = fmaf(A[e], c[e], B[e]);
            }
        } else {
            load_state(a.h0 ? a.h0 + n * a.M + col : nullptr, nv, c);
        }
        const int tile0 = span * a.tiles_per_span, tile1 = tile0 + a.tiles_per_span < tiles ? tile0 + a.tiles_per_span : tiles;
        for (int tile = tile0; tile < tile1; ++tile) {
            const int t0 = tile * STEPS + seg * RC_K;
            Raw rx[RC_K], rg[RC_K];
#pragma unroll
            for (int i = 0; i < RC_K; ++i) {
                const int n1 = t0 + i < a.T ? nv : 0;
                rx[i] = raw_load<T, RC_V>(x + (long)(t0 + i) * a.M, n1);
                rg[i] = raw_load<T, RC_V>(g + (long)(t0 + i) * a.M, n1);
            }
            float av[RC_K][4], kx[RC_K][4];
#pragma unroll
            for (int i = 0; i < RC_K; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float ga, gk;
                    gate(raw_get<T>(rg[i], e), ga, gk);
                    av[i][e] = t0 + i < a.T ? ga : 1.f;                 // steps beyond the clip change nothing
                    kx[i][e] = t0 + i < a.T ? gk * raw_get<T>(rx[i], e) : 0.f;
                }
            float h[4];
            if constexpr (SEG > 1) {
                float A[4] = {1.f, 1.f, 1.f, 1.f}, B[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < RC_K; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        A[e] *= av[i][e];
                        B[e] = fmaf(av[i][e], B[e], kx[i][e]);
                    }
                lds.m[par][0][seg][lc] = pack4(A);
                lds.m[par][1][seg][lc] = pack4(B);
                __syncthreads();
#pragma unroll
                for (int s = 0; s < SEG; ++s) {
                    const float4 fa = lds.m[par][0][s][lc], fb = lds.m[par][1][s][lc];
                    if (s == seg) { h[0] = c[0]; h[1] = c[1]; h[2] = c[2]; h[3] = c[3]; }
                    c[0] = fmaf(fa.x, c[0], fb.x); c[1] = fmaf(fa.y, c[1], fb.y);
                    c[2] = fmaf(fa.z, c[2], fb.z); c[3] = fmaf(fa.w, c[3], fb.w);
                }
                par ^= 1;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) h[e] = c[e];
            }
            if (a.saved && t0 > 0 && t0 % RC_SAVE == 0 && t0 < a.T) store_state(a.saved + (n * nsaved + t0 / RC_SAVE - 1) * a.M + col, nv, h);
#pragma unroll
            for (int i = 0; i < RC_K; ++i) {
#pragma unroll
                for (int e = 0; e < 4; ++e) h[e] = fmaf(av[i][e], h[e], kx[i][e]);
                if (t0 + i < a.T) raw_store<T, RC_V>(y + (long)(t0 + i) * a.M, h, nv);
            }
            if constexpr (SEG == 1) {
#pragma unroll
                for (int e = 0; e < 4; ++e) c[e] = h[e];
            }
        }
        if (a.h_last && span == a.spans - 1 && seg == 0) store_state(a.h_last + n * a.M + col, nv, c);
    }
}

// The tiles of a span from the last to the first.  STEPS is a multiple of RC_SAVE or T does not exceed it, so that the state in
// front of every tile is at hand.
template <typename T, int SEG>
__global__ void __launch_bounds__(RC_NT) recur_bwd_kernel(RecurArgs a) {
    constexpr int LC = RC_NT / SEG, STEPS = SEG * RC_K;
    typedef typename RawVec<T, RC_V>::type Raw;
    __shared__ RecurLds<SEG, 3> lds;
    const int lc = threadIdx.x % LC, seg = SEG == 1 ? 0 : threadIdx.x / LC;
    const int nsaved = (a.T - 1) / RC_SAVE;
    const int tiles = (a.T + STEPS - 1) / STEPS;
    int par = 0;
    for (long job = blockIdx.x; job < a.jobs; job += gridDim.x) {
        const long cb = job % a.cblocks;
        const int span = (int)(job / a.cblocks % a.spans);
        const long n = job / a.cblocks / a.spans;
        const long col = (cb * LC + lc) * RC_V;
        const int nv = (int)(a.M - col < RC_V ? a.M - col : RC_V);
        const long base = n * a.T * a.M + col;
        float e1[4];                                                    // E behind the tile
        load_state(a.dh_last ? a.dh_last + n * a.M + col : nullptr, nv, e1);
        for (int s = a.spans - 1; s > span; --s) {
            float A[4], B[4];
            load_state(a.maps + ((n * a.spans + s) * 2) * a.M + col, nv, A);
            load_state(a.maps + ((n * a.spans + s) * 2 + 1) * a.M + col, nv, B);
#pragma unroll
            for (int e = 0; e < 4; ++e) e1[e] = fmaf(A[e], e1[e], B[e]);
        }
        const int tile0 = span * a.tiles_per_span, tile1 = tile0 + a.tiles_per_span < tiles ? tile0 + a.tiles_per_span : tiles;
        for (int tile = tile1 - 1; tile >= tile0; --tile) {
            const int t0 = tile * STEPS + seg * RC_K;
            Raw rx[RC_K], rg[RC_K], rd[RC_K];
#pragma unroll
            for (int i = 0; i < RC_K; ++i) {
                const int n1 = t0 + i < a.T ? nv : 0;
                const long at = base + (long)(t0 + i) * a.M;
                rx[i] = raw_load<T, RC_V>((const T*)a.x + at, n1);
                rg[i] = raw_load<T, RC_V>((const T*)a.g + at, n1);
                rd[i] = raw_load<T, RC_V>((const T*)a.dy + at, n1);
            }
            float h[4];                                                 // the state in front of the tile, then of the segment
            if (tile == 0) load_state(a.h0 ? a.h0 + n * a.M + col : nullptr, nv, h);
            else load_state(a.saved + (n * nsaved + tile * (STEPS / RC_SAVE) - 1) * a.M + col, nv, h);
            float av[RC_K][4], kv[RC_K][4];
#pragma unroll
            for (int i = 0; i < RC_K; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float ga, gk;
                    gate(raw_get<T>(rg[i], e), ga, gk);
                    av[i][e] = t0 + i < a.T ? ga : 1.f;
                    kv[i][e] = t0 + i < a.T ? gk : 0.f;
                }
            float en[4];                                                // E behind the segment
            if constexpr (SEG > 1) {
                float A[4] = {1.f, 1.f, 1.f, 1.f}, B[4] = {0.f, 0.f, 0.f, 0.f}, C[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < RC_K; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        A[e] *= av[i][e];
                        B[e] = fmaf(av[i][e], B[e], kv[i][e] * raw_get<T>(rx[i], e));
                    }
#pragma unroll
                for (int i = RC_K - 1; i >= 0; --i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) C[e] = av[i][e] * (raw_get<T>(rd[i], e) + C[e]);   // (dy is zero beyond the clip)
                lds.m[par][0][seg][lc] = pack4(A);
                lds.m[par][1][seg][lc] = pack4(B);
                lds.m[par][2][seg][lc] = pack4(C);
                __syncthreads();
#pragma unroll
                for (int s = 0; s < SEG - 1; ++s) {
                    if (s < seg) {
                        const float4 fa = lds.m[par][0][s][lc], fb = lds.m[par][1][s][lc];
                        h[0] = fmaf(fa.x, h[0], fb.x); h[1] = fmaf(fa.y, h[1], fb.y);
                        h[2] = fmaf(fa.z, h[2], fb.z); h[3] = fmaf(fa.w, h[3], fb.w);
                    }
                }
#pragma unroll
                for (int s = SEG - 1; s >= 0; --s) {
                    const float4 fa = lds.m[par][0][s][lc], fc = lds.m[par][2][s][lc];
                    if (s == seg) { en[0] = e1[0]; en[1] = e1[1]; en[2] = e1[2]; en[3] = e1[3]; }
                    e1[0] = fmaf(fa.x, e1[0], fc.x); e1[1] = fmaf(fa.y, e1[1], fc.y);
                    e1[2] = fmaf(fa.z, e1[2], fc.z); e1[3] = fmaf(fa.w, e1[3], fc.w);
                }
                par ^= 1;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) en[e] = e1[e];
            }
            float before[RC_K][4];                                      // the state in front of every step
#pragma unroll
            for (int i = 0; i < RC_K; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    before[i][e] = h[e];
                    h[e] = fmaf(av[i][e], h[e], kv[i][e] * raw_get<T>(rx[i], e));
                }
#pragma unroll
            for (int i = RC_K - 1; i >= 0; --i) {
                float ox[4], og[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float D = raw_get<T>(rd[i], e) + en[e];
                    ox[e] = kv[i][e] * D;
                    en[e] = av[i][e] * D;
                    og[e] = en[e] * kv[i][e] * (before[i][e] - raw_get<T>(rx[i], e));
                }
                if (t0 + i < a.T) {
                    const long at = base + (long)(t0 + i) * a.M;
                    raw_store<T, RC_V>((T*)a.dx + at, ox, nv);
                    raw_store<T, RC_V>((T*)a.dg + at, og, nv);
                }
            }
            if constexpr (SEG == 1) {
#pragma unroll
                for (int e = 0; e < 4; ++e) e1[e] = en[e];
            }
        }
        if (a.dh0 && span == 0 && seg == 0) store_state(a.dh0 + n * a.M + col, nv, e1);
    }
}

// The map of every span but the one that nothing follows, for launches that split the time axis: h behind the span as a map of h
// in front of it, or (BWD) E in front of it as a map of E behind it.  A segment keeps its own running map: the segments of a
// tile are joined per tile, as in the passes above.
template <typename T, bool BWD>
__global__ void __launch_bounds__(RC_NT) recur_span_kernel(RecurArgs a, int steps_per_span) {
    constexpr int SEG = 16, LC = RC_NT / SEG, STEPS = SEG * RC_K;
    __shared__ RecurLds<SEG, 2> lds;
    const int lc = threadIdx.x % LC, seg = threadIdx.x / LC;
    const long cblocks = (a.M + LC * RC_V - 1) / (LC * RC_V), jobs = cblocks * a.spans * a.N;
    int par = 0;
    for (long job = blockIdx.x; job < jobs; job += gridDim.x) {
        const long cb = job % cblocks;
        const int span = (int)(job / cblocks % a.spans);
        const long n = job / cblocks / a.spans;
        const long col = (cb * LC + lc) * RC_V;
        const int nv = (int)(a.M - col < RC_V ? a.M - col : RC_V);
        if (!BWD && span == 0 && seg == 0) {    // a copy of the first state: h_last may be the same memory
            float h[4];
            load_state(a.h0 ? a.h0 + n * a.M + col : nullptr, nv, h);
            store_state(a.maps + ((long)a.N * a.spans * 2 + n) * a.M + col, nv, h);
        }
        if (span == (BWD ? 0 : a.spans - 1)) continue;
        const int begin = span * steps_per_span, end = begin + steps_per_span < a.T ? begin + steps_per_span : a.T;
        const int tiles = (end - begin + STEPS - 1) / STEPS;
        const long base = n * a.T * a.M + col;
        float A1[4] = {1.f, 1.f, 1.f, 1.f}, B1[4] = {0.f, 0.f, 0.f, 0.f};
        for (int q = 0; q < tiles; ++q) {
            const int t0 = begin + (BWD ? tiles - 1 - q : q) * STEPS + seg * RC_K;
            typename RawVec<T, RC_V>::type rb[RC_K], rg[RC_K];
#pragma unroll
            for (int i = 0; i < RC_K; ++i) {
                const int n1 = t0 + i < end ? nv : 0;
                rb[i] = raw_load<T, RC_V>((const T*)(BWD ? a.dy : a.x) + base + (long)(t0 + i) * a.M, n1);
                rg[i] = raw_load<T, RC_V>((const T*)a.g + base + (long)(t0 + i) * a.M, n1);
            }
            float A[4] = {1.f, 1.f, 1.f, 1.f}, B[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < RC_K; ++j) {
                const int i = BWD ? RC_K - 1 - j : j;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float ga, gk;
                    gate(raw_get<T>(rg[i], e), ga, gk);
                    if (t0 + i < end) {
                        A[e] *= ga;
                        B[e] = BWD ? ga * (raw_get<T>(rb[i], e) + B[e]) : fmaf(ga, B[e], gk * raw_get<T>(rb[i], e));
                    }
                }
            }
            lds.m[par][0][seg][lc] = pack4(A);
            lds.m[par][1][seg][lc] = pack4(B);
            __syncthreads();
            if (seg == 0) {
#pragma unroll
                for (int s = 0; s < SEG; ++s) {
                    const float4 fa = lds.m[par][0][BWD ? SEG - 1 - s : s][lc], fb = lds.m[par][1][BWD ? SEG - 1 - s : s][lc];
                    A1[0] *= fa.x; A1[1] *= fa.y; A1[2] *= fa.z; A1[3] *= fa.w;
                    B1[0] = fmaf(fa.x, B1[0], fb.x); B1[1] = fmaf(fa.y, B1[1], fb.y);
                    B1[2] = fmaf(fa.z, B1[2], fb.z); B1[3] = fmaf(fa.w, B1[3], fb.w);
                }
            }
            par ^= 1;
        }
        if (seg == 0) {
            store_state(a.maps + ((n * a.spans + span) * 2) * a.M + col, nv, A1);
            store_state(a.maps + ((n * a.spans + span) * 2 + 1) * a.M + col, nv, B1);
        }
    }
}

// ---- host --------------------------------------------------------------------------------
struct RecurPlan {
    int seg;              // segments per tile
    int spans, tiles_per_span;
    long cblocks, jobs;
};

// Segments: as few as hold the clip (8 steps each), so that threads lie along the columns, where a row of memory is; of long clips
// 16 (128-byte rows) while the columns fill the chip, 32 (64-byte rows) for fewer.  What still leaves CUs idle splits the time
// axis into spans, whose maps a launch of their own takes first.
static RecurPlan recur_plan(const tsm_recur_desc* d) {
    RecurPlan p;
    const long M = (long)d->C * d->H * d->W;
    auto jobs = [&](int seg) { return (M + RC_NT / seg * RC_V - 1) / (RC_NT / seg * RC_V) * d->N; };
    p.seg = d->T <= RC_K ? 1 : d->T <= 4 * RC_K ? 4 : jobs(16) >= 512 ? 16 : 32;
    const int steps = p.seg * RC_K, tiles = cdiv(d->T, steps);
    p.cblocks = jobs(p.seg) / d->N;
    long want = jobs(p.seg) < 256 ? 256 / jobs(p.seg) : 1;
    if (want > 64) want = 64;
    if (want > tiles) want = tiles;
    p.tiles_per_span = cdiv(tiles, want);
    p.spans = cdiv(tiles, p.tiles_per_span);
    p.jobs = p.cblocks * d->N * p.spans;
    return p;
}

static int recur_check(const tsm_recur_desc* d, const char* who) {
    if (!d) return fail(TSM_ERR_NULLPTR, "%s: null descriptor", who);
    if (d->dtype != TSM_F32 && d->dtype != TSM_BF16) return fail(TSM_ERR_DTYPE, "%s: unknown dtype %d", who, d->dtype);
    if (d->N <= 0 || d->T <= 0 || d->C <= 0 || d->H <= 0 || d->W <= 0) return fail(TSM_ERR_SHAPE, "%s: non-positive dimension", who);
    const double n = (double)d->N * d->T * d->C * d->H * d->W;
    if (n > 1e17 || (double)d->C * d->H * d->W > 1e15 || d->T > 0x7fff0000) return fail(TSM_ERR_SHAPE, "%s: tensor too large", who);
    return TSM_OK;
}

static size_t recur_saved(const tsm_recur_desc* d) { return (size_t)d->N * ((d->T - 1) / RC_SAVE) * d->C * d->H * d->W * sizeof(float); }
static size_t recur_ws(const tsm_recur_desc* d, const RecurPlan& p) {
    return p.spans > 1 ? align_up((size_t)d->N * (2 * p.spans + 1) * d->C * d->H * d->W * sizeof(float)) : 0;
}

static RecurArgs recur_args(const tsm_recur_desc* d, const RecurPlan& p) {
    RecurArgs a{};
    a.M = (long)d->C * d->H * d->W;
    a.cblocks = p.cblocks;
    a.jobs = p.jobs;
    a.N = d->N;
    a.T = d->T;
    a.spans = p.spans;
    a.tiles_per_span = p.tiles_per_span;
    return a;
}

template <typename T>
static int recur_run(const RecurArgs& a, const RecurPlan& p, bool bwd, hipStream_t s) {
    const unsigned cap = 1u << 22;
    const dim3 block(RC_NT), grid((unsigned)(a.jobs < cap ? a.jobs : cap));
    if (p.spans > 1) {
        const long jobs = (a.M + 63) / 64 * a.N * a.spans;
        const dim3 sgrid((unsigned)(jobs < cap ? jobs : cap));
        const int steps = a.tiles_per_span * p.seg * RC_K;
        if (bwd) recur_span_kernel<T, true><<<sgrid, block, 0, s>>>(a, steps);
        else recur_span_kernel<T, false><<<sgrid, block, 0, s>>>(a, steps);
        TSM_TRY(check_launch(bwd ? "recur_bwd_spans" : "recur_fwd_spans"));
    }
#define CALL(SEG)                                                        \
    do {                                                                 \
        if (bwd) recur_bwd_kernel<T, SEG><<<grid, block, 0, s>>>(a);     \
        else recur_fwd_kernel<T, SEG><<<grid, block, 0, s>>>(a);         \
    } while (0)
    if (p.seg == 1) CALL(1);
    else if (p.seg == 4) CALL(4);
    else if (p.seg == 16) CALL(16);
    else CALL(32);
#undef CALL
    return check_launch(bwd ? "recur_bwd" : "recur_fwd");
}

}  // namespace tsm

using namespace tsm;

extern "C" {

size_t tsm_recur_saved_bytes(const tsm_recur_desc* d) { return recur_check(d, "tsm_recur_saved_bytes") == TSM_OK ? recur_saved(d) : 0; }

size_t tsm_recur_workspace_bytes(const tsm_recur_desc* d) {
    return recur_check(d, "tsm_recur_workspace_bytes") == TSM_OK ? recur_ws(d, recur_plan(d)) : 0;
}

int tsm_recur_fwd(const tsm_recur_desc* d, const void* x, const void* g, const float* h0, void* y, float* h_last, void* saved, void* ws,
                  size_t ws_bytes, void* stream) {
    const char* who = "tsm_recur_fwd";
    TSM_TRY(recur_check(d, who));
    if (!x || !g || !y) return fail(TSM_ERR_NULLPTR, "%s: null tensor pointer", who);
    const RecurPlan p = recur_plan(d);
    const size_t need = recur_ws(d, p);
    if (ws_bytes < need) return fail(TSM_ERR_WORKSPACE, "%s: workspace %zu bytes, need %zu", who, ws_bytes, need);
    if (need && !ws) return fail(TSM_ERR_NULLPTR, "%s: null workspace", who);
    RecurArgs a = recur_args(d, p);
    const size_t n = (size_t)d->N * d->T * a.M * dtype_size(d->dtype), st = (size_t)d->N * a.M * 4;
    // (h_last may be h0: the state of a stream, carried in place)
    const Span in[] = {{x, n, "x"}, {g, n, "g"}, {h0 == h_last ? nullptr : h0, st, "h0"}};
    const Span out[] = {{y, n, "y"}, {h_last, st, "h_last"}, {saved, recur_saved(d), "saved"}, {ws, need, "the workspace"}};
    TSM_TRY(check_spans(who, in, 3, out, 4));
    a.x = x; a.g = g; a.h0 = h0; a.y = y; a.h_last = h_last; a.saved = (float*)saved; a.maps = (float*)ws;
    return d->dtype == TSM_BF16 ? recur_run<bf16_t>(a, p, false, (hipStream_t)stream) : recur_run<float>(a, p, false, (hipStream_t)stream);
}

int tsm_recur_bwd(const tsm_recur_desc* d, const void* x, const void* g, const float* h0, const void* saved, const void* dy, const float* dh_last,
                  void* dx, void* dg, float* dh0, void* ws, size_t ws_bytes, void* stream) {
    const char* who = "tsm_recur_bwd";
    TSM_TRY(recur_check(d, who));
    if (!x || !g || !dy || !dx || !dg) return fail(TSM_ERR_NULLPTR, "%s: null tensor pointer", who);
    const RecurPlan p = recur_plan(d);
    const size_t need = recur_ws(d, p), sv = recur_saved(d);
    if (sv && !saved) return fail(TSM_ERR_NULLPTR, "%s: null saved buffer", who);
    if (ws_bytes < need) return fail(TSM_ERR_WORKSPACE, "%s: workspace %zu bytes, need %zu", who, ws_bytes, need);
    if (need && !ws) return fail(TSM_ERR_NULLPTR, "%s: null workspace", who);
    RecurArgs a = recur_args(d, p);
    const size_t n = (size_t)d->N * d->T * a.M * dtype_size(d->dtype), st = (size_t)d->N * a.M * 4;
    const Span in[] = {{x, n, "x"}, {g, n, "g"}, {h0, st, "h0"}, {saved, sv, "saved"}, {dy, n, "dy"}, {dh_last, st, "dh_last"}};
    const Span out[] = {{dx, n, "dx"}, {dg, n, "dg"}, {dh0, st, "dh0"}, {ws, need, "the workspace"}};
    TSM_TRY(check_spans(who, in, 6, out, 4));
    a.x = x; a.g = g; a.h0 = h0; a.saved = (float*)saved; a.dy = dy; a.dh_last = dh_last; a.dx = dx; a.dg = dg; a.dh0 = dh0; a.maps = (float*)ws;
    return d->dtype == TSM_BF16 ? recur_run<bf16_t>(a, p, true, (hipStream_t)stream) : recur_run<float>(a, p, true, (hipStream_t)stream);
}

}  // extern "C"
