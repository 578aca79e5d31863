// Gated linear recurrence over the frames of a clip, forward and backward.
//
//   a = sigmoid(g), k = 1 - a = sigmoid(-g);   h_t = a_t h_{t-1} + k_t x_t,  y_t = h_t
//   D_t = dy_t + E_{t+1},  E_t = a_t D_t (E_T = dh_last);   dx_t = k_t D_t,  dg_t = E_t k_t (h_{t-1} - x_t),  dh_0 = E_0
//
// Every value of a frame is a recurrence of its own ("column"), so both memory orders are the same [N][T][M] tensor, M = C*H*W.
// Both passes are bound by memory: forward reads x, g and writes y, backward reads x, g, dy and writes dx, dg.  The steps of a
// column are maps h -> A h + B, which join associatively: a block takes a tile of SEG segments of 8 steps times LC*4 columns, one
// thread per segment and four columns, holds the tile in registers, joins the segments' maps through LDS and runs every segment
// again from its true start, so each tensor is read once.  Tiles follow one another in time with the state carried along; where few
// columns would leave CUs idle, a column's tiles run side by side and hand their maps on through memory (JOIN).  The
// state, the maps and what is carried are fp32 throughout; only y, dx and dg are rounded to the storage type.
// The backward pass needs h inside a tile: it starts from the states that the forward pass left every 128 steps (1.6 % of a bf16
// tensor), and forms h again from x and g, which it reads anyway, instead of reading y, which is rounded.
// Measured, bf16: 64 clips of 8 frames of 7 x 7 x 2048: forward 53.5 us (5.8 TB/s), backward 82 us (6.3 TB/s); 4 clips of 4096 frames
// of 2048 values: 46 and 76 us (4.4 TB/s; a copy of that size reaches 6.7: a tile waits on loads, on the tiles in front and on its
// stores in turn, with four and three tiles per CU to cover for one another).
#include <algorithm>
#include <type_traits>
#include "internal.h"
#include "args.h"
#include "vec_any.h"

namespace tsm {

static constexpr int RC_NT = 256, RC_V = 4, RC_STEPS = 8;   // threads, columns per thread (one where there are fewer), steps per thread (fewer for the shortest clips)
static constexpr int RC_SAVE = 128;                       // steps between saved states
static constexpr int RC_GROUP = 64, RC_TICKET = 16;       // JOIN: tiles from one whole state to the next; words (64 bytes) of a ticket counter

struct RecurArgs {
    const void *x, *g, *dy;
    void *y, *dx, *dg;
    const float *h0, *dh_last;
    float *h_last, *dh0;
    float* saved;         // [N][(T-1)/RC_SAVE][M]: the state in front of step RC_SAVE*(j+1)
    uint64_t* slots;      // JOIN: [N][tiles + groups][M], see recur_join; in front of them
    uint32_t* tickets;    // [N][cblocks], one in RC_TICKET words: how many tiles have been taken
    long M, cblocks, jobs, ws_bytes;
    int N, T, tiles, groups;
    bool runs;            // the jobs in runs per XCD
};

// a = sigmoid(g) and k = 1 - a, neither by subtraction: e = exp(-|g|), 1/(1+e) and e/(1+e).  (The product with log2 e is rounded, which
// makes e off by |g| units of its last place: half a unit of the sum 1 + e at most.)  PACKED: in one register, the smaller under the sign
// of g; the larger is 1 less that, off by half a unit of its last place.
template <bool PACKED> struct Gate {
    float av, kv;
    __device__ __forceinline__ static Gate of(float g) {
        const float e = __builtin_amdgcn_exp2f(-fabsf(g) * 1.44269502f), big = __builtin_amdgcn_rcpf(1.f + e), small = e * big;
        return g < 0.f ? Gate{small, big} : Gate{big, small};
    }
    __device__ __forceinline__ float a() const { return av; }
    __device__ __forceinline__ float k() const { return kv; }
    __device__ __forceinline__ void open() {                            // a step that changes nothing
        av = 1.f;
        kv = 0.f;
    }
    __device__ __forceinline__ void renew() {}
};
template <> struct Gate<true> {
    float s;
    __device__ __forceinline__ static Gate of(float g) {
        const float e = __builtin_amdgcn_exp2f(-fabsf(g) * 1.44269502f);
        return Gate{copysignf(e * __builtin_amdgcn_rcpf(1.f + e), g)};
    }
    __device__ __forceinline__ bool closed() const { return (int)__float_as_uint(s) < 0; }
    __device__ __forceinline__ float a() const { return closed() ? -s : 1.f - s; }
    __device__ __forceinline__ float k() const { return closed() ? 1.f + s : s; }
    __device__ __forceinline__ void open() { s = 0.f; }
    __device__ __forceinline__ void renew() { asm volatile("" : "+v"(s)); }     // to the compiler, another value: taken apart again, not held apart
};

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
    __device__ __forceinline__ static void renew(Raw& r) {     // to the compiler, another value
        if constexpr (V > 1)
#pragma unroll
            for (int i = 0; i < (int)(sizeof(Raw) / 4); ++i) {
                uint32_t w = r[i];
                asm volatile("" : "+v"(w));
                r[i] = w;
            }
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

// Every XCD takes a run of the jobs, so that blocks beside one another share the lines of memory that lie across their border in its L2
// (3 x 301 x 4995 fp32: forward 16.6 -> 13.9 us, backward 30.8 -> 25.3), and tiles side by side read neighbouring memory at one time (4 x
// 4096 x 2048 142 -> 130).  Rows of whole lines in turn are better off without: 64 x 8 frames 142 -> 146.
__device__ __forceinline__ long xcd_run(long job, long jobs) {
    const long xcd = job & 7;
    return xcd * (jobs / 8) + (xcd < jobs % 8 ? xcd : jobs % 8) + (job >> 3);
}

// A job's block of columns and what is left of its number; the division in 32 bits where they suffice.
struct RecurJob {
    long cb, n;
    __device__ __forceinline__ RecurJob(const RecurArgs& a, long job) {
        if (a.jobs >> 32 == 0) {
            n = (uint32_t)job / (uint32_t)a.cblocks;
            cb = (uint32_t)job - (uint32_t)n * (uint32_t)a.cblocks;
        } else {
            n = job / a.cblocks;
            cb = job - n * a.cblocks;
        }
    }
};

// Where the values of a step lie, from the clip's first one; NEAR: from the tile's, in 32 bits, which cost a register less per address.
// (Tiles lie side by side for few columns only: 128 steps of them are far below 2^32 bytes.)
template <bool NEAR> struct RecurRows {
    typedef typename std::conditional<NEAR, uint32_t, long>::type At;
    long origin;
    int t0;
    At M, col;
    __device__ __forceinline__ RecurRows(const RecurArgs& a, long n, int first, long c) : origin((n * a.T + first) * a.M), t0(first), M((At)a.M), col((At)c) {}
    __device__ __forceinline__ At at(int t) const { return (At)(t - t0) * M + col; }
    template <typename T> __device__ __forceinline__ T* of(const void* p, At at) const { return (T*)((char*)((T*)p + origin) + at * (At)sizeof(T)); }
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

// ---- JOIN: too few columns to fill the chip; a block takes one tile, and the tiles of a column run side by side ------------
// A tile's map goes into a slot, one 64-bit word (A below, B above) per column, which says by itself that it is there: all slots are
// filled with ones first, a NaN that no published A is.  A block then waits for the maps in front of it, joins them in an order that does
// not depend on which came first, and runs its tile, which has stayed in registers.  The last tile of every RC_GROUP also leaves the
// state behind it, where those of the next group begin.  A block of columns hands out its tiles by ticket, in their order: whoever
// a tile waits for was taken before it, by a block that is on a CU and that waits for still earlier tiles only, so every wait ends.  (It is
// bounded all the same, for callers that share a workspace between streams: what is missing then enters as the NaN of an empty
// slot.)  One ticket counter for all columns costs 15 ns a tile in turn: 4 x 4096 frames of 2048 values forward, again and again
// on the same tensors, 77 us, with a counter per block of columns 43; a launch of its own for the maps, which reads x and g twice, 61.
static constexpr int RC_TRIES = 1 << 22;

__global__ void __launch_bounds__(256) recur_clear_kernel(any_u32x4* p, long n) {
    for (long i = blockIdx.x * 256L + threadIdx.x; i < n; i += gridDim.x * 256L) p[i] = any_u32x4{~0u, ~0u, ~0u, ~0u};
}

// The next tile, in their order, of column block `at`.
__device__ __forceinline__ int recur_ticket(const RecurArgs& a, long at, int* shared) {
    __syncthreads();                                                    // (LDS of the block's last tile is free)
    if (threadIdx.x == 0) *shared = (int)(__hip_atomic_fetch_add(a.tickets + at * RC_TICKET, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1);   // (from all ones)
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(*shared);
}

__device__ __forceinline__ void recur_publish(uint64_t* slot, float A, float B) {
    const uint32_t lo = __float_as_uint(A);
    __hip_atomic_store(slot, (uint64_t)__float_as_uint(B) << 32 | (lo == ~0u ? 0x7fc00000u : lo), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// What precedes the tile that is `order`-th of its columns (block `cb` of n), from the segments' maps in lds: f.  A lane per column:
// the first wavefront joins the tile's own map and publishes it, then each of the four joins a quarter of the maps in front.
// first: what precedes the first tile, or null.  It is read by the lane that publishes what depends on it, before it does.
template <bool UP, typename T, int V, typename Lds>
__device__ __forceinline__ void recur_join(const RecurArgs& a, long n, long cb, int order, const float* first, Lds& lds, int plane, int lc, float (&f)[V]) {
    constexpr int SEG = 16, W = 16 * V, BATCH = 8;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x % W, e = l % V;
    const RecurCols<T, V> cols((cb * 16 + l / V) * V, a.M);
    const bool owner = threadIdx.x < W && e >= cols.skip;
    uint64_t* slots = a.slots + n * (a.tiles + a.groups) * a.M + cols.col + e;
    float A = order == 0 ? 0.f : 1.f, B = 0.f;                          // (a tile with nothing in front has a state behind it, not a map)
    if (wave == 0) {
        if (order == 0) {
            B = first ? first[cols.col + e] : 0.f;
            if (threadIdx.x < W) lds.m[1][1][0][l / V].f[e] = B;
        }
#pragma unroll 4
        for (int i = 0; i < SEG; ++i) {
            const int s = UP ? i : SEG - 1 - i;
            const float fa = lds.m[0][0][s][l / V].f[e];
            B = fmaf(fa, B, lds.m[0][plane][s][l / V].f[e]);
            A *= fa;
        }
        if (owner) recur_publish(slots + (long)order * a.M, A, B);
    }
    // the state behind the last group, if there is one, and the maps of this group's tiles
    const int group = order / RC_GROUP, lead = group > 0, count = order % RC_GROUP + lead, per = (count + 3) / 4;
    const int i0 = wave * per, i1 = i0 + per < count ? i0 + per : count;
    if (i0 < i1 && e >= cols.skip) {                                    // (columns that are not stored wait for none)
        float PA = 1.f, PB = 0.f;
        for (int b = i0; b < i1; b += BATCH) {
            uint64_t v[BATCH];
            bool there;
            int tries = 0;
            do {
                there = true;
#pragma unroll
                for (int k = 0; k < BATCH; ++k) {
                    const int i = b + k < i1 ? b + k : i1 - 1;
                    v[k] = __hip_atomic_load(slots + (lead && i == 0 ? a.tiles + group - 1L : (long)group * RC_GROUP + i - lead) * a.M, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
#pragma unroll
                for (int k = 0; k < BATCH; ++k) there = there && (uint32_t)v[k] != ~0u;
            } while (!there && ++tries < RC_TRIES);
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                if (b + k >= i1) break;
                const float fa = __uint_as_float((uint32_t)v[k]);
                PB = fmaf(fa, PB, __uint_as_float((uint32_t)(v[k] >> 32)));
                PA *= fa;
            }
        }
        if (threadIdx.x % 64 < W) {
            lds.m[1][0][wave][l / V].f[e] = PA;
            lds.m[1][1][wave][l / V].f[e] = PB;
        }
    }
    __syncthreads();
    const int parts = order == 0 ? 1 : (count + per - 1) / per;
    Lds::get(lds.m[1][1][0][lc], f);
    for (int w = 1; w < parts; ++w) {
        float fa[V], fb[V];
        Lds::get(lds.m[1][0][w][lc], fa);
        Lds::get(lds.m[1][1][w][lc], fb);
#pragma unroll
        for (int k = 0; k < V; ++k) f[k] = fmaf(fa[k], f[k], fb[k]);
    }
    if (wave == 0 && order % RC_GROUP == RC_GROUP - 1 && order + 1 < a.tiles) {
        float c = lds.m[1][1][0][l / V].f[e];
        for (int w = 1; w < parts; ++w) c = fmaf(lds.m[1][0][w][l / V].f[e], c, lds.m[1][1][w][l / V].f[e]);
        if (owner) recur_publish(slots + (a.tiles + (long)group) * a.M, 0.f, fmaf(A, c, B));
    }
}

template <typename T, int V, int SEG, int RC_K = RC_STEPS, bool JOIN = false>
__global__ void __launch_bounds__(RC_NT, JOIN ? 4 : 1) recur_fwd_kernel(RecurArgs a) {
    constexpr int LC = RC_NT / SEG, STEPS = SEG * RC_K;
    typedef RecurCols<T, V> Cols;
    typedef RecurRows<JOIN> Rows;
    typedef RecurLds<SEG, 2, V> Lds;
    __shared__ Lds lds;
    const int lc = threadIdx.x % LC, seg = SEG == 1 ? 0 : threadIdx.x / LC;
    const int nsaved = (a.T - 1) / RC_SAVE;
    const int tiles = (a.T + STEPS - 1) / STEPS;
    __shared__ int s_tile;
    int par = 0;
    for (long job = blockIdx.x; job < a.jobs; job += gridDim.x) {
        const RecurJob j(a, a.runs ? xcd_run(job, a.jobs) : job);
        const long cb = j.cb, n = JOIN ? j.n % (uint32_t)a.N : j.n;
        const int order = JOIN ? recur_ticket(a, n * a.cblocks + cb, &s_tile) : 0;
        if (JOIN && (unsigned)order >= (unsigned)tiles) return;         // (a workspace that another call writes to)
        const Cols cols((cb * LC + lc) * V, a.M);
        const Rows rows(a, n, JOIN ? order * STEPS : 0, cols.col);
        float c[V];                                                     // the state in front of the tile
        if constexpr (!JOIN) cols.load_state(a.h0 ? a.h0 + n * a.M : nullptr, c);
        const int tile0 = JOIN ? order : 0, tile1 = JOIN ? order + 1 : tiles;
        typename Cols::Raw rx[RC_K], rg[RC_K];
        auto load = [&](int tile) {                                     // (steps behind the last one read it again)
#pragma unroll
            for (int i = 0; i < RC_K; ++i) {
                const int t = tile * STEPS + seg * RC_K + i;
                const auto at = rows.at(t < a.T ? t : a.T - 1);
                rx[i] = Cols::load(rows.template of<T>(a.x, at));
                rg[i] = Cols::load(rows.template of<T>(a.g, at));
            }
        };
        load(tile0);
        for (int tile = tile0; tile < tile1; ++tile) {
            const int t0 = tile * STEPS + seg * RC_K;
            const bool full = (tile + 1) * STEPS <= a.T;                // of all segments
            Gate<JOIN> gt[RC_K][V];
            typename Cols::Raw xv[RC_K];
#pragma unroll
            for (int i = 0; i < RC_K; ++i) {
                xv[i] = rx[i];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    gt[i][e] = Gate<JOIN>::of(Cols::get(rg[i], e));
                    if constexpr (!JOIN) gt[i][e].kv *= Cols::get(rx[i], e);
                }
            }
            if (tile + 1 < tile1) load(tile + 1);                       // on its way while this tile is joined and stored
            if (!full) {                                                // steps beyond the clip change nothing
#pragma unroll
                for (int i = 0; i < RC_K; ++i)
                    if (t0 + i >= a.T) {
                        xv[i] = typename Cols::Raw{};
#pragma unroll
                        for (int e = 0; e < V; ++e) gt[i][e].open();
                    }
            }
            auto kx = [&](int i, int e) {
                if constexpr (JOIN) return gt[i][e].k() * Cols::get(xv[i], e);
                else return gt[i][e].kv;
            };
            float h[V];
            if constexpr (SEG > 1) {
                float A[V], B[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    A[e] = gt[0][e].a();
                    B[e] = kx(0, e);
                }
#pragma unroll
                for (int i = 1; i < RC_K; ++i)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        A[e] *= gt[i][e].a();
                        B[e] = fmaf(gt[i][e].a(), B[e], kx(i, e));
                    }
                Lds::put(lds.m[par][0][seg][lc], A);
                Lds::put(lds.m[par][1][seg][lc], B);
                __syncthreads();
                if constexpr (JOIN) {
                    recur_join<true, T, V>(a, n, cb, order, a.h0 ? a.h0 + n * a.M : nullptr, lds, 1, lc, c);
#pragma unroll
                    for (int i = 0; i < RC_K; ++i) {
                        Cols::renew(xv[i]);
#pragma unroll
                        for (int e = 0; e < V; ++e) gt[i][e].renew();
                    }
                } else if (tile > tile0) {
                    Lds::get(lds.carry[par ^ 1][lc], c);
                }
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
                for (int e = 0; e < V; ++e) h[e] = fmaf(gt[i][e].a(), h[e], kx(i, e));
                if (full || t0 + i < a.T) cols.store(rows.template of<T>(a.y, rows.at(t0 + i)), h);
            }
            if constexpr (SEG > 1 && !JOIN) {
                if (seg == SEG - 1) Lds::put(lds.carry[par][lc], h);
                par ^= 1;
            }
#pragma unroll
            for (int e = 0; e < V; ++e) c[e] = h[e];
        }
        if (a.h_last && tile1 == tiles && seg == SEG - 1) cols.store_state(a.h_last + n * a.M, c);
    }
}

// The tiles from the last to the first.  STEPS is a multiple of RC_SAVE or T does not exceed it, so that the state in
// front of every tile is at hand.
template <typename T, int V, int SEG, int RC_K = RC_STEPS, bool JOIN = false>
__global__ void __launch_bounds__(RC_NT, JOIN ? 2 : 1) recur_bwd_kernel(RecurArgs a) {
    constexpr int LC = RC_NT / SEG, STEPS = SEG * RC_K;
    typedef RecurCols<T, V> Cols;
    typedef RecurRows<JOIN> Rows;
    typedef RecurLds<SEG, 3, V> Lds;
    __shared__ Lds lds;
    const int lc = threadIdx.x % LC, seg = SEG == 1 ? 0 : threadIdx.x / LC;
    const int nsaved = (a.T - 1) / RC_SAVE;
    const int tiles = (a.T + STEPS - 1) / STEPS;
    __shared__ int s_tile;
    int par = 0;
    for (long job = blockIdx.x; job < a.jobs; job += gridDim.x) {
        const RecurJob j(a, a.runs ? xcd_run(job, a.jobs) : job);
        const long cb = j.cb, n = JOIN ? j.n % (uint32_t)a.N : j.n;
        const int order = JOIN ? recur_ticket(a, n * a.cblocks + cb, &s_tile) : 0;
        if (JOIN && (unsigned)order >= (unsigned)tiles) return;         // (a workspace that another call writes to)
        const Cols cols((cb * LC + lc) * V, a.M);
        float e1[V];                                                    // E behind the tile
        if constexpr (!JOIN) cols.load_state(a.dh_last ? a.dh_last + n * a.M : nullptr, e1);
        const int tile0 = JOIN ? tiles - 1 - order : 0, tile1 = JOIN ? tiles - order : tiles;
        const Rows rows(a, n, JOIN ? tile0 * STEPS : 0, cols.col);
        typename Cols::Raw rx[RC_K], rg[RC_K], rd[RC_K];
        auto load = [&](int tile) {                                     // (steps behind the last one read it again)
#pragma unroll
            for (int i = 0; i < RC_K; ++i) {
                const int t = tile * STEPS + seg * RC_K + i;
                const auto at = rows.at(t < a.T ? t : a.T - 1);
                rx[i] = Cols::load(rows.template of<T>(a.x, at));
                rg[i] = Cols::load(rows.template of<T>(a.g, at));
                rd[i] = Cols::load(rows.template of<T>(a.dy, at));
            }
        };
        for (int tile = tile1 - 1; tile >= tile0; --tile) {
            const int t0 = tile * STEPS + seg * RC_K;
            const bool full = (tile + 1) * STEPS <= a.T;
            load(tile);
            float h[V];                                                 // the state in front of the tile, then of the segment
            cols.load_state(tile == 0 ? (a.h0 ? a.h0 + n * a.M : nullptr) : a.saved + (n * nsaved + tile * (STEPS / RC_SAVE) - 1) * a.M, h);
            Gate<JOIN> gt[RC_K][V];
#pragma unroll
            for (int i = 0; i < RC_K; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) gt[i][e] = Gate<JOIN>::of(Cols::get(rg[i], e));
            if (!full) {                                                // steps beyond the clip change nothing
#pragma unroll
                for (int i = 0; i < RC_K; ++i)
                    if (t0 + i >= a.T) {
                        rx[i] = rd[i] = typename Cols::Raw{};
#pragma unroll
                        for (int e = 0; e < V; ++e) gt[i][e].open();
                    }
            }
            float en[V];                                                // E behind the segment
            if constexpr (SEG > 1) {
                float A[V], B[V], C[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    A[e] = gt[0][e].a();
                    B[e] = gt[0][e].k() * Cols::get(rx[0], e);
                    C[e] = A[e] * Cols::get(rd[0], e);
                }
#pragma unroll
                for (int i = 1; i < RC_K; ++i)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        A[e] *= gt[i][e].a();
                        B[e] = fmaf(gt[i][e].a(), B[e], gt[i][e].k() * Cols::get(rx[i], e));
                        C[e] = fmaf(A[e], Cols::get(rd[i], e), C[e]);
                    }
                Lds::put(lds.m[par][0][seg][lc], A);
                Lds::put(lds.m[par][1][seg][lc], B);
                Lds::put(lds.m[par][2][seg][lc], C);
                __syncthreads();
                if constexpr (JOIN) {
                    recur_join<false, T, V>(a, n, cb, order, a.dh_last ? a.dh_last + n * a.M : nullptr, lds, 2, lc, e1);
#pragma unroll
                    for (int i = 0; i < RC_K; ++i) {
                        Cols::renew(rx[i]);
                        Cols::renew(rd[i]);
#pragma unroll
                        for (int e = 0; e < V; ++e) gt[i][e].renew();
                    }
                } else if (tile + 1 < tile1) {
                    Lds::get(lds.carry[par ^ 1][lc], e1);
                }
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
                    h[e] = fmaf(gt[i][e].a(), h[e], gt[i][e].k() * Cols::get(rx[i], e));
                    gt[i][e].renew();
                }
#pragma unroll
            for (int i = RC_K - 1; i >= 0; --i) {
                float ox[V], og[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float D = Cols::get(rd[i], e) + en[e];
                    ox[e] = gt[i][e].k() * D;
                    en[e] = gt[i][e].a() * D;
                    og[e] = en[e] * (gt[i][e].k() * u[i][e]);
                }
                if (full || t0 + i < a.T) {
                    const auto at = rows.at(t0 + i);
                    cols.store(rows.template of<T>(a.dx, at), ox);
                    cols.store(rows.template of<T>(a.dg, at), og);
                }
            }
            if constexpr (SEG > 1 && !JOIN) {
                if (seg == 0) Lds::put(lds.carry[par][lc], en);
                par ^= 1;
            }
#pragma unroll
            for (int e = 0; e < V; ++e) e1[e] = en[e];
        }
        if (a.dh0 && tile0 == 0 && seg == 0) cols.store_state(a.dh0 + n * a.M, e1);
    }
}

// ---- host --------------------------------------------------------------------------------
struct RecurPlan {
    int v, seg;           // columns per thread, segments per tile
    bool join;            // the tiles of a column side by side
    int tiles, groups;
    long cblocks, jobs;
};

// Segments: as few as hold the clip (8 steps each), so that threads lie along the columns, where a row of memory is, up to 16 with rows of
// 64 columns.  Tiles of a column run side by side where a block or less per CU would take four tiles and more in turn (backward three, at
// half a block).  us in turn and side by
// side, bf16, 2048 columns per clip: 4 clips of 300 frames (3 tiles) forward 10.5, 11.3, backward 13.7, 13.1; of 512 12.7, 11.3 and
// 17.7, 13.7; of 1024 22.6, 14.3 and 35.3, 23.2; 8 clips of 1024 25.8, 23.7 and 42.7, 38.4; 16 clips 36.6, 38.6 and 58.4, 67.3.  fp32 forward,
// which has registers for fewer tiles at a time: 4 clips of 512 13.5, 15.5, 8 clips of 1024 34.0, 41.7.  Three tiles, both passes, in turn, the backward pass side by side, both: 1 clip
// of 300 bf16 23.6, 23.5, 25.8, 2 clips 23.7, 22.8, 25.0, 4 clips 25.4, 24.8, 25.0, fp32 22.7, 22.4, 27.7, 25.0, 23.2, 24.9, 26.1, 26.8, 28.8.
static RecurPlan recur_plan(const tsm_recur_desc* d, bool bwd) {
    RecurPlan p;
    const long M = (long)d->C * d->H * d->W;
    p.v = M < RC_V ? 1 : RC_V;
    p.seg = d->T <= RC_STEPS ? 1 : d->T <= 4 * RC_STEPS ? 4 : d->T <= 8 * RC_STEPS ? 8 : 16;
    const int width = RC_NT / p.seg * p.v;
    p.tiles = cdiv(d->T, p.seg * RC_STEPS);
    p.groups = (p.tiles - 1) / RC_GROUP;
    p.cblocks = (M + width - 1) / width;
    p.jobs = p.cblocks * d->N;
    p.join = (p.tiles >= 4 && p.jobs <= (!bwd && d->dtype == TSM_F32 ? 128 : 256)) || (bwd && p.tiles == 3 && p.jobs <= 128);
    if (p.join) p.jobs *= p.tiles;
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
static size_t recur_tickets(const tsm_recur_desc* d, const RecurPlan& p) { return align_up((size_t)d->N * p.cblocks * RC_TICKET * 4); }
static size_t recur_ws(const tsm_recur_desc* d, const RecurPlan& p) {
    return p.join ? recur_tickets(d, p) + align_up((size_t)d->N * (p.tiles + p.groups) * d->C * d->H * d->W * sizeof(uint64_t)) : 0;
}

static RecurArgs recur_args(const tsm_recur_desc* d, const RecurPlan& p) {
    RecurArgs a{};
    a.M = (long)d->C * d->H * d->W;
    a.cblocks = p.cblocks;
    a.jobs = p.jobs;
    a.N = d->N;
    a.T = d->T;
    a.tiles = p.tiles;
    a.groups = p.groups;
    a.runs = p.join || (p.seg > 1 && a.M * dtype_size(d->dtype) % 128 != 0);
    return a;
}

static void recur_slots(const tsm_recur_desc* d, const RecurPlan& p, RecurArgs& a, void* ws) {
    a.tickets = (uint32_t*)ws;
    a.slots = (uint64_t*)((char*)ws + recur_tickets(d, p));
    a.ws_bytes = recur_ws(d, p);
}

template <typename T, int V>
static int recur_run(const RecurArgs& a, const RecurPlan& p, bool bwd, hipStream_t s) {
    const long cap = 1 << 22;
    const dim3 block(RC_NT), grid((unsigned)std::min(a.jobs, cap));
    if (p.join) {
        const long n = a.ws_bytes / 16;
        recur_clear_kernel<<<dim3((unsigned)std::min((n + 255) / 256, 2048L)), dim3(256), 0, s>>>((any_u32x4*)a.tickets, n);
        TSM_TRY(check_launch("recur_clear"));
    }
#define CALL(...)                                                                \
    do {                                                                         \
        if (bwd) recur_bwd_kernel<T, V, __VA_ARGS__><<<grid, block, 0, s>>>(a);  \
        else recur_fwd_kernel<T, V, __VA_ARGS__><<<grid, block, 0, s>>>(a);      \
    } while (0)
    if (p.join) CALL(16, RC_STEPS, true);
    else if (a.T == 1) CALL(1, 1);
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
    a.x = x; a.g = g; a.h0 = h0; a.y = y; a.h_last = h_last; a.saved = (float*)saved;
    recur_slots(d, p, a, ws);
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
    a.x = x; a.g = g; a.h0 = h0; a.saved = (float*)saved; a.dy = dy; a.dh_last = dh_last; a.dx = dx; a.dg = dg; a.dh0 = dh0;
    recur_slots(d, p, a, ws);
    return recur_any(a, p, d->dtype, true, (hipStream_t)stream);
}

}  // extern "C"
