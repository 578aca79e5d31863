// Gated linear recurrence over the frames of a clip, forward and backward.
//
//   a = sigmoid(g), k = 1 - a = sigmoid(-g);   h_t = a_t h_{t-1} + k_t x_t,  y_t = h_t
//   D_t = dy_t + E_{t+1},  E_t = a_t D_t (E_T = dh_last);   dx_t = k_t D_t,  dg_t = E_t k_t (h_{t-1} - x_t),  dh_0 = E_0
//
// Every value of a frame is a recurrence of its own ("column"), so both memory orders are the same [N][T][M] tensor, M = C*H*W.
// Both passes are bound by memory: forward reads x, g and writes y, backward reads x, g, dy and writes dx, dg.  The steps of a
// column are maps h -> A h + B, which join associatively: a block takes a tile of SEG segments of 8 steps times LC*4 columns, one
// thread per segment and four columns, holds the tile in registers, joins the segments' maps through LDS and runs every segment
// again from its true start.  Tiles follow one another in time with the state carried along, so each tensor is read once (twice
// where few columns make several blocks share the time axis).  The
// state, the maps and what is carried are fp32 throughout; only y, dx and dg are rounded to the storage type.
// The backward pass needs h inside a tile: it starts from the states that the forward pass left every 128 steps (1.6 % of a bf16
// tensor), and forms h again from x and g, which it reads anyway, instead of reading y, which is rounded.
#include <algorithm>
#include <type_traits>
#include "internal.h"
#include "args.h"
#include "vec_any.h"

namespace tsm {

static constexpr int RC_NT = 256, RC_V = 4, RC_STEPS = 8;   // threads, columns per thread (one where there are fewer), steps per thread (fewer for the shortest clips)
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

// sigmoid(g) and 1 - sigmoid(g), neither by subtraction: e = exp(-|g|), 1/(1+e) and e/(1+e).  (The product with log2 e is rounded, which
// makes e off by |g| units of its last place: half a unit of the sum 1 + e at most.)
__device__ __forceinline__ void gate(float g, float& a, float& k) {
    const float e = __builtin_amdgcn_exp2f(-fabsf(g) * 1.44269502f);
    const float big = __builtin_amdgcn_rcpf(1.f + e), small = e * big;
    a = g < 0.f ? small : big;
    k = g < 0.f ? big : small;
}

// The columns of a thread: V from `col`, of which the first `skip` belong to the thread before.  Columns that would lie behind the last are
// moved back onto it, so that loads need no condition (one under a condition is awaited where the branches join); only what a
// thread owns is stored.
template <typename T, int V>
struct RecurCols {
    long col;
    int skip;
    __device__ __forceinline__ RecurCols(long c, long M) {
        col = c < M - V ? c : M - V;
        skip = (int)(c - col < V ? c - col : V);
    }
    typedef typename std::conditional<V == 1, T, typename RawVec<T, V == 1 ? 4 : V>::type>::type Raw;
    __device__ __forceinline__ static Raw load(const T* p) {
        if constexpr (V == 1) return *p;
        else return *(const typename RawVec<T, V>::mem*)p;
    }
    __device__ __forceinline__ static float get(const Raw& r, int e) {
        if constexpr (V == 1) return Elem<T>::ld(r);
        else return raw_get<T>(r, e);
    }
    __device__ __forceinline__ void store(T* p, const float (&f)[V]) const {
        if constexpr (V > 1) {
            if (skip == 0) {
                raw_store<T, V>(p, f, V);
                return;
            }
        }
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e >= skip) p[e] = Elem<T>::st(f[e]);
    }
    __device__ __forceinline__ void load_state(const float* p, float (&f)[V]) const {       // p: of column 0, or null
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = p ? p[col + e] : 0.f;
    }
    __device__ __forceinline__ void store_state(float* p, const float (&f)[V]) const {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e >= skip) p[col + e] = f[e];
    }
};

// The maps of the tile's segments, one parity per tile so that one barrier per tile is enough.
template <int SEG, int PLANES, int V>
struct RecurLds {
    struct alignas(V * 4) Vec { float f[V]; };
    Vec m[2][SEG > 1 ? PLANES : 1][SEG > 1 ? SEG : 1][SEG > 1 ? RC_NT / SEG : 1];
    Vec carry[2][SEG > 1 ? RC_NT / SEG : 1];                            // what one tile hands to the next
    __device__ __forceinline__ static void put(Vec& to, const float (&f)[V]) {
        Vec v;
#pragma unroll
        for (int e = 0; e < V; ++e) v.f[e] = f[e];
        to = v;
    }
    __device__ __forceinline__ static void get(const Vec& from, float (&f)[V]) {
        const Vec v = from;
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = v.f[e];
    }
    // f through the maps (A in plane 0, B in `plane`) of the segments in front of (UP) or behind `seg`, in order.  Those in front of all
    // segments of the wavefront need no condition.
    template <bool UP>
    __device__ __forceinline__ void through(int par, int plane, int seg, int lc, float (&f)[V]) const {
        constexpr int PER = 64 / (RC_NT / SEG) < 1 ? 1 : 64 / (RC_NT / SEG);        // segments of a wavefront
        const int own = __builtin_amdgcn_readfirstlane(UP ? seg : SEG - 1 - seg) / PER * PER;   // segments that all of them pass
        const int mine = UP ? seg : SEG - 1 - seg;
#pragma unroll 4
        for (int q = 0; q < own; ++q) {
            const int s = UP ? q : SEG - 1 - q;
            const Vec fa = m[par][0][s][lc], fb = m[par][plane][s][lc];
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] = fmaf(fa.f[e], f[e], fb.f[e]);
        }
#pragma unroll
        for (int q = 0; q < PER - 1; ++q) {
            const int s = UP ? own + q : SEG - 1 - own - q;
            const Vec fa = m[par][0][s][lc], fb = m[par][plane][s][lc];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float o = fmaf(fa.f[e], f[e], fb.f[e]);
                f[e] = own + q < mine ? o : f[e];
            }
        }
    }
};

template <typename T, int V, int SEG, int RC_K = RC_STEPS>
__global__ void __launch_bounds__(RC_NT) recur_fwd_kernel(RecurArgs a) {
    constexpr int LC = RC_NT / SEG, STEPS = SEG * RC_K;
    typedef RecurCols<T, V> Cols;
    typedef RecurLds<SEG, 2, V> Lds;
    __shared__ Lds lds;
    const int lc = threadIdx.x % LC, seg = SEG == 1 ? 0 : threadIdx.x / LC;
    const int nsaved = (a.T - 1) / RC_SAVE;
    const int tiles = (a.T + STEPS - 1) / STEPS;
    int par = 0;
    for (long job = blockIdx.x; job < a.jobs; job += gridDim.x) {
        const long cb = job % a.cblocks;
        const int span = (int)(job / a.cblocks % a.spans);
        const long n = job / a.cblocks / a.spans;
        const Cols cols((cb * LC + lc) * V, a.M);
        const T* x = (const T*)a.x + n * a.T * a.M + cols.col;
        const T* g = (const T*)a.g + n * a.T * a.M + cols.col;
        T* y = (T*)a.y + n * a.T * a.M + cols.col;
        float c[V];                                                     // the state in front of the tile
        if (a.spans > 1) {
            const float* maps = a.maps + n * a.spans * 2 * a.M;
            cols.load_state(a.maps + ((long)a.N * a.spans * 2 + n) * a.M, c);
            for (int s = 0; s < span; ++s) {
                float A[V], B[V];
                cols.load_state(maps + (long)s * 2 * a.M, A);
                cols.load_state(maps + ((long)s * 2 + 1) * a.M, B);
#pragma unroll
                for (int e = 0; e < V; ++e) c[e] = fmaf(A[e], c[e], B[e]);
            }
        } else {
            cols.load_state(a.h0 ? a.h0 + n * a.M : nullptr, c);
        }
        const int tile0 = span * a.tiles_per_span, tile1 = tile0 + a.tiles_per_span < tiles ? tile0 + a.tiles_per_span : tiles;
        typename Cols::Raw rx[RC_K], rg[RC_K];
        auto load = [&](int tile) {                                     // (steps behind the last one read it again)
#pragma unroll
            for (int i = 0; i < RC_K; ++i) {
                const int t = tile * STEPS + seg * RC_K + i;
                const long at = (long)(t < a.T ? t : a.T - 1) * a.M;
                rx[i] = Cols::load(x + at);
                rg[i] = Cols::load(g + at);
            }
        };
        load(tile0);
        for (int tile = tile0; tile < tile1; ++tile) {
            const int t0 = tile * STEPS + seg * RC_K;
            const bool full = (tile + 1) * STEPS <= a.T;                // of all segments
            float av[RC_K][V], kx[RC_K][V];
#pragma unroll
            for (int i = 0; i < RC_K; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float k;
                    gate(Cols::get(rg[i], e), av[i][e], k);
                    kx[i][e] = k * Cols::get(rx[i], e);
                }
            if (tile + 1 < tile1) load(tile + 1);                       // on its way while this tile is joined and stored
            if (!full) {                                                // steps beyond the clip change nothing
#pragma unroll
                for (int i = 0; i < RC_K; ++i)
                    if (t0 + i >= a.T)
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            av[i][e] = 1.f;
                            kx[i][e] = 0.f;
                        }
            }
            float h[V];
            if constexpr (SEG > 1) {
                float A[V], B[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    A[e] = av[0][e];
                    B[e] = kx[0][e];
                }
#pragma unroll
                for (int i = 1; i < RC_K; ++i)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        A[e] *= av[i][e];
                        B[e] = fmaf(av[i][e], B[e], kx[i][e]);
                    }
                Lds::put(lds.m[par][0][seg][lc], A);
                Lds::put(lds.m[par][1][seg][lc], B);
                __syncthreads();
                if (tile > tile0) Lds::get(lds.carry[par ^ 1][lc], c);
#pragma unroll
                for (int e = 0; e < V; ++e) h[e] = c[e];
                lds.template through<true>(par, 1, seg, lc, h);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) h[e] = c[e];
            }
            if (a.saved && t0 > 0 && t0 % RC_SAVE == 0 && t0 < a.T) cols.store_state(a.saved + (n * nsaved + t0 / RC_SAVE - 1) * a.M, h);
#pragma unroll
            for (int i = 0; i < RC_K; ++i) {
#pragma unroll
                for (int e = 0; e < V; ++e) h[e] = fmaf(av[i][e], h[e], kx[i][e]);
                if (full || t0 + i < a.T) cols.store(y + (long)(t0 + i) * a.M, h);
            }
            if constexpr (SEG > 1) {
                if (seg == SEG - 1) Lds::put(lds.carry[par][lc], h);
                par ^= 1;
            }
#pragma unroll
            for (int e = 0; e < V; ++e) c[e] = h[e];
        }
        if (a.h_last && span == a.spans - 1 && seg == SEG - 1) cols.store_state(a.h_last + n * a.M, c);
    }
}

// The tiles of a span from the last to the first.  STEPS is a multiple of RC_SAVE or T does not exceed it, so that the state in
// front of every tile is at hand.
template <typename T, int V, int SEG, int RC_K = RC_STEPS>
__global__ void __launch_bounds__(RC_NT) recur_bwd_kernel(RecurArgs a) {
    constexpr int LC = RC_NT / SEG, STEPS = SEG * RC_K;
    typedef RecurCols<T, V> Cols;
    typedef RecurLds<SEG, 3, V> Lds;
    __shared__ Lds lds;
    const int lc = threadIdx.x % LC, seg = SEG == 1 ? 0 : threadIdx.x / LC;
    const int nsaved = (a.T - 1) / RC_SAVE;
    const int tiles = (a.T + STEPS - 1) / STEPS;
    int par = 0;
    for (long job = blockIdx.x; job < a.jobs; job += gridDim.x) {
        const long cb = job % a.cblocks;
        const int span = (int)(job / a.cblocks % a.spans);
        const long n = job / a.cblocks / a.spans;
        const Cols cols((cb * LC + lc) * V, a.M);
        const long base = n * a.T * a.M + cols.col;
        float e1[V];                                                    // E behind the tile
        cols.load_state(a.dh_last ? a.dh_last + n * a.M : nullptr, e1);
        for (int s = a.spans - 1; s > span; --s) {
            float A[V], B[V];
            cols.load_state(a.maps + (n * a.spans + s) * 2 * a.M, A);
            cols.load_state(a.maps + ((n * a.spans + s) * 2 + 1) * a.M, B);
#pragma unroll
            for (int e = 0; e < V; ++e) e1[e] = fmaf(A[e], e1[e], B[e]);
        }
        const int tile0 = span * a.tiles_per_span, tile1 = tile0 + a.tiles_per_span < tiles ? tile0 + a.tiles_per_span : tiles;
        typename Cols::Raw rx[RC_K], rg[RC_K], rd[RC_K];
        auto load = [&](int tile) {                                     // (steps behind the last one read it again)
#pragma unroll
            for (int i = 0; i < RC_K; ++i) {
                const int t = tile * STEPS + seg * RC_K + i;
                const long at = base + (long)(t < a.T ? t : a.T - 1) * a.M;
                rx[i] = Cols::load((const T*)a.x + at);
                rg[i] = Cols::load((const T*)a.g + at);
                rd[i] = Cols::load((const T*)a.dy + at);
            }
        };
        for (int tile = tile1 - 1; tile >= tile0; --tile) {
            const int t0 = tile * STEPS + seg * RC_K;
            const bool full = (tile + 1) * STEPS <= a.T;
            load(tile);
            float h[V];                                                 // the state in front of the tile, then of the segment
            cols.load_state(tile == 0 ? (a.h0 ? a.h0 + n * a.M : nullptr) : a.saved + (n * nsaved + tile * (STEPS / RC_SAVE) - 1) * a.M, h);
            float av[RC_K][V], kv[RC_K][V];
#pragma unroll
            for (int i = 0; i < RC_K; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) gate(Cols::get(rg[i], e), av[i][e], kv[i][e]);
            if (!full) {                                                // steps beyond the clip change nothing
#pragma unroll
                for (int i = 0; i < RC_K; ++i)
                    if (t0 + i >= a.T) {
                        rx[i] = rd[i] = typename Cols::Raw{};
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            av[i][e] = 1.f;
                            kv[i][e] = 0.f;
                        }
                    }
            }
            float en[V];                                                // E behind the segment
            if constexpr (SEG > 1) {
                float A[V], B[V], C[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    A[e] = av[0][e];
                    B[e] = kv[0][e] * Cols::get(rx[0], e);
                    C[e] = av[RC_K - 1][e] * Cols::get(rd[RC_K - 1], e);
                }
#pragma unroll
                for (int i = 1; i < RC_K; ++i)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        A[e] *= av[i][e];
                        B[e] = fmaf(av[i][e], B[e], kv[i][e] * Cols::get(rx[i], e));
                        C[e] = av[RC_K - 1 - i][e] * (Cols::get(rd[RC_K - 1 - i], e) + C[e]);
                    }
                Lds::put(lds.m[par][0][seg][lc], A);
                Lds::put(lds.m[par][1][seg][lc], B);
                Lds::put(lds.m[par][2][seg][lc], C);
                __syncthreads();
                if (tile + 1 < tile1) Lds::get(lds.carry[par ^ 1][lc], e1);
#pragma unroll
                for (int e = 0; e < V; ++e) en[e] = e1[e];
                lds.template through<true>(par, 1, seg, lc, h);
                lds.template through<false>(par, 2, seg, lc, en);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) en[e] = e1[e];
            }
            float u[RC_K][V];                                           // the state in front of every step less its input
#pragma unroll
            for (int i = 0; i < RC_K; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    u[i][e] = h[e] - Cols::get(rx[i], e);
                    h[e] = fmaf(av[i][e], h[e], kv[i][e] * Cols::get(rx[i], e));
                }
#pragma unroll
            for (int i = RC_K - 1; i >= 0; --i) {
                float ox[V], og[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float D = Cols::get(rd[i], e) + en[e];
                    ox[e] = kv[i][e] * D;
                    en[e] = av[i][e] * D;
                    og[e] = en[e] * (kv[i][e] * u[i][e]);
                }
                if (full || t0 + i < a.T) {
                    const long at = base + (long)(t0 + i) * a.M;
                    cols.store((T*)a.dx + at, ox);
                    cols.store((T*)a.dg + at, og);
                }
            }
            if constexpr (SEG > 1) {
                if (seg == 0) Lds::put(lds.carry[par][lc], en);
                par ^= 1;
            }
#pragma unroll
            for (int e = 0; e < V; ++e) e1[e] = en[e];
        }
        if (a.dh0 && span == 0 && seg == 0) cols.store_state(a.dh0 + n * a.M, e1);
    }
}

// The map of every span but the one that nothing follows, for launches that split the time axis: h behind the span as a map of h
// in front of it, or (BWD) E in front of it as a map of E behind it.
template <typename T, int V, bool BWD>
__global__ void __launch_bounds__(RC_NT) recur_span_kernel(RecurArgs a, int steps_per_span) {
    constexpr int SEG = 16, LC = RC_NT / SEG, RC_K = RC_STEPS, STEPS = SEG * RC_K;
    typedef RecurCols<T, V> Cols;
    typedef RecurLds<SEG, 2, V> Lds;
    __shared__ Lds lds;
    const int lc = threadIdx.x % LC, seg = threadIdx.x / LC;
    const long cblocks = (a.M + LC * V - 1) / (LC * V), jobs = cblocks * a.spans * a.N;
    int par = 0;
    for (long job = blockIdx.x; job < jobs; job += gridDim.x) {
        const long cb = job % cblocks;
        const int span = (int)(job / cblocks % a.spans);
        const long n = job / cblocks / a.spans;
        const Cols cols((cb * LC + lc) * V, a.M);
        if (!BWD && span == 0 && seg == 0) {    // a copy of the first state: h_last may be the same memory
            float h[V];
            cols.load_state(a.h0 ? a.h0 + n * a.M : nullptr, h);
            cols.store_state(a.maps + ((long)a.N * a.spans * 2 + n) * a.M, h);
        }
        if (span == (BWD ? 0 : a.spans - 1)) continue;
        const int begin = span * steps_per_span, end = begin + steps_per_span < a.T ? begin + steps_per_span : a.T;
        const int tiles = (end - begin + STEPS - 1) / STEPS;
        const long base = n * a.T * a.M + cols.col;
        float A1[V], B1[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            A1[e] = 1.f;
            B1[e] = 0.f;
        }
        for (int q = 0; q < tiles; ++q) {
            const int t0 = begin + (BWD ? tiles - 1 - q : q) * STEPS + seg * RC_K;
            typename Cols::Raw rb[RC_K], rg[RC_K];
#pragma unroll
            for (int i = 0; i < RC_K; ++i) {
                const long at = base + (long)(t0 + i < end ? t0 + i : end - 1) * a.M;
                rb[i] = Cols::load((const T*)(BWD ? a.dy : a.x) + at);
                rg[i] = Cols::load((const T*)a.g + at);
            }
            float A[V], B[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                A[e] = 1.f;
                B[e] = 0.f;
            }
#pragma unroll
            for (int j = 0; j < RC_K; ++j) {
                const int i = BWD ? RC_K - 1 - j : j;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float ga, gk;
                    gate(Cols::get(rg[i], e), ga, gk);
                    const float b = Cols::get(rb[i], e), nb = BWD ? ga * (b + B[e]) : fmaf(ga, B[e], gk * b);
                    A[e] = t0 + i < end ? A[e] * ga : A[e];
                    B[e] = t0 + i < end ? nb : B[e];
                }
            }
            Lds::put(lds.m[par][0][seg][lc], A);
            Lds::put(lds.m[par][1][seg][lc], B);
            __syncthreads();
            if (seg == 0) {
#pragma unroll
                for (int s = 0; s < SEG; ++s) {
                    const typename Lds::Vec fa = lds.m[par][0][BWD ? SEG - 1 - s : s][lc], fb = lds.m[par][1][BWD ? SEG - 1 - s : s][lc];
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        A1[e] *= fa.f[e];
                        B1[e] = fmaf(fa.f[e], B1[e], fb.f[e]);
                    }
                }
            }
            par ^= 1;
        }
        if (seg == 0) {
            cols.store_state(a.maps + (n * a.spans + span) * 2 * a.M, A1);
            cols.store_state(a.maps + ((n * a.spans + span) * 2 + 1) * a.M, B1);
        }
    }
}

// ---- host --------------------------------------------------------------------------------
struct RecurPlan {
    int v, seg;           // columns per thread, segments per tile
    int spans, tiles_per_span;
    long cblocks, jobs;
};

// Segments: as few as hold the clip (8 steps each), so that threads lie along the columns, where a row of memory is, up to 16 with rows of
// 64 columns.  What then leaves CUs idle splits the time axis into spans, whose maps a launch of their own takes first, at the price of
// reading two tensors twice.  us in one span and in 1024 blocks of them, bf16, 2048 columns per clip: forward 4 clips of 4096 frames (128
// blocks in one span) 84, 62, 5 of 2048 45, 45, 6 of 2048 45, 47, 8 of 2048 47, 59; backward 170, 94; 70, 56; 73, 65; 99, 91; 12 of 1024 50, 63.
static RecurPlan recur_plan(const tsm_recur_desc* d, bool bwd) {
    RecurPlan p;
    const long M = (long)d->C * d->H * d->W;
    p.v = M < RC_V ? 1 : RC_V;
    p.seg = d->T <= RC_STEPS ? 1 : d->T <= 4 * RC_STEPS ? 4 : d->T <= 8 * RC_STEPS ? 8 : 16;
    const int steps = p.seg * RC_STEPS, tiles = cdiv(d->T, steps), width = RC_NT / p.seg * p.v;
    p.cblocks = (M + width - 1) / width;
    const long blocks = p.cblocks * d->N;
    long want = blocks <= (bwd ? 224 : 160) ? 1024 / blocks : 1;
    if (want > 64) want = 64;
    if (want > tiles) want = tiles;
    p.tiles_per_span = cdiv(tiles, want);
    p.spans = cdiv(tiles, p.tiles_per_span);
    p.jobs = blocks * p.spans;
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

template <typename T, int V>
static int recur_run(const RecurArgs& a, const RecurPlan& p, bool bwd, hipStream_t s) {
    const unsigned cap = 1u << 22;
    const dim3 block(RC_NT), grid((unsigned)(a.jobs < cap ? a.jobs : cap));
    if (p.spans > 1) {
        const long jobs = (a.M + 16 * V - 1) / (16 * V) * a.N * a.spans;
        const dim3 sgrid((unsigned)(jobs < cap ? jobs : cap));
        const int steps = a.tiles_per_span * p.seg * RC_STEPS;
        if (bwd) recur_span_kernel<T, V, true><<<sgrid, block, 0, s>>>(a, steps);
        else recur_span_kernel<T, V, false><<<sgrid, block, 0, s>>>(a, steps);
        TSM_TRY(check_launch(bwd ? "recur_bwd_spans" : "recur_fwd_spans"));
    }
#define CALL(...)                                                                \
    do {                                                                         \
        if (bwd) recur_bwd_kernel<T, V, __VA_ARGS__><<<grid, block, 0, s>>>(a);  \
        else recur_fwd_kernel<T, V, __VA_ARGS__><<<grid, block, 0, s>>>(a);      \
    } while (0)
    if (a.T == 1) CALL(1, 1);
    else if (a.T <= 4) CALL(1, 4);
    else if (p.seg == 1) CALL(1);
    else if (p.seg == 4) CALL(4);
    else if (p.seg == 8) CALL(8);
    else CALL(16);
#undef CALL
    return check_launch(bwd ? "recur_bwd" : "recur_fwd");
}

static int recur_any(const RecurArgs& a, const RecurPlan& p, int dtype, bool bwd, hipStream_t s) {
    if (dtype == TSM_BF16) return p.v == 1 ? recur_run<bf16_t, 1>(a, p, bwd, s) : recur_run<bf16_t, RC_V>(a, p, bwd, s);
    return p.v == 1 ? recur_run<float, 1>(a, p, bwd, s) : recur_run<float, RC_V>(a, p, bwd, s);
}

}  // namespace tsm

using namespace tsm;

extern "C" {

size_t tsm_recur_saved_bytes(const tsm_recur_desc* d) { return recur_check(d, "tsm_recur_saved_bytes") == TSM_OK ? recur_saved(d) : 0; }

size_t tsm_recur_workspace_bytes(const tsm_recur_desc* d) {
    return recur_check(d, "tsm_recur_workspace_bytes") == TSM_OK ? std::max(recur_ws(d, recur_plan(d, false)), recur_ws(d, recur_plan(d, true))) : 0;
}

int tsm_recur_fwd(const tsm_recur_desc* d, const void* x, const void* g, const float* h0, void* y, float* h_last, void* saved, void* ws,
                  size_t ws_bytes, void* stream) {
    const char* who = "tsm_recur_fwd";
    TSM_TRY(recur_check(d, who));
    if (!x || !g || !y) return fail(TSM_ERR_NULLPTR, "%s: null tensor pointer", who);
    const RecurPlan p = recur_plan(d, false);
    const size_t need = tsm_recur_workspace_bytes(d);
    if (ws_bytes < need) return fail(TSM_ERR_WORKSPACE, "%s: workspace %zu bytes, need %zu", who, ws_bytes, need);
    if (need && !ws) return fail(TSM_ERR_NULLPTR, "%s: null workspace", who);
    RecurArgs a = recur_args(d, p);
    const size_t n = (size_t)d->N * d->T * a.M * dtype_size(d->dtype), st = (size_t)d->N * a.M * 4;
    // (h_last may be h0: the state of a stream, carried in place)
    const Span in[] = {{x, n, "x"}, {g, n, "g"}, {h0 == h_last ? nullptr : h0, st, "h0"}};
    const Span out[] = {{y, n, "y"}, {h_last, st, "h_last"}, {saved, recur_saved(d), "saved"}, {ws, need, "the workspace"}};
    TSM_TRY(check_spans(who, in, 3, out, 4));
    a.x = x; a.g = g; a.h0 = h0; a.y = y; a.h_last = h_last; a.saved = (float*)saved; a.maps = (float*)ws;
    return recur_any(a, p, d->dtype, false, (hipStream_t)stream);
}

int tsm_recur_bwd(const tsm_recur_desc* d, const void* x, const void* g, const float* h0, const void* saved, const void* dy, const float* dh_last,
                  void* dx, void* dg, float* dh0, void* ws, size_t ws_bytes, void* stream) {
    const char* who = "tsm_recur_bwd";
    TSM_TRY(recur_check(d, who));
    if (!x || !g || !dy || !dx || !dg) return fail(TSM_ERR_NULLPTR, "%s: null tensor pointer", who);
    const RecurPlan p = recur_plan(d, true);
    const size_t need = tsm_recur_workspace_bytes(d), sv = recur_saved(d);
    if (sv && !saved) return fail(TSM_ERR_NULLPTR, "%s: null saved buffer", who);
    if (ws_bytes < need) return fail(TSM_ERR_WORKSPACE, "%s: workspace %zu bytes, need %zu", who, ws_bytes, need);
    if (need && !ws) return fail(TSM_ERR_NULLPTR, "%s: null workspace", who);
    RecurArgs a = recur_args(d, p);
    const size_t n = (size_t)d->N * d->T * a.M * dtype_size(d->dtype), st = (size_t)d->N * a.M * 4;
    const Span in[] = {{x, n, "x"}, {g, n, "g"}, {h0, st, "h0"}, {saved, sv, "saved"}, {dy, n, "dy"}, {dh_last, st, "dh_last"}};
    const Span out[] = {{dx, n, "dx"}, {dg, n, "dg"}, {dh0, st, "dh0"}, {ws, need, "the workspace"}};
    TSM_TRY(check_spans(who, in, 6, out, 4));
    a.x = x; a.g = g; a.h0 = h0; a.saved = (float*)saved; a.dy = dy; a.dh_last = dh_last; a.dx = dx; a.dg = dg; a.dh0 = dh0; a.maps = (float*)ws;
    return recur_any(a, p, d->dtype, true, (hipStream_t)stream);
}

}  // extern "C"
