// Layer norm over rows of C consecutive values and its backward pass with the weights' gradients.
//
//   mean = sum x / C, rstd = 1 / sqrt(sum (x - mean)^2 / C + eps), xhat = (x - mean) * rstd, y = gamma * xhat + beta
//   v = gamma * dy;  dx = rstd * (v - sum v / C - xhat * sum (v * xhat) / C);  dgamma = sum_rows dy * xhat, dbeta = sum_rows dy
//
// Both passes are bound by memory: x -> y forward, x, dy -> dx backward.  A row lives in the registers of L lanes from its
// one read on (R vectors of 16 bytes per lane), so mean, centred variance and result cost one pass; all sums are fp32.  The
// weights' gradients are column sums over all rows: every block keeps its rows' share in registers, writes one row of a
// partial buffer at its end, and a second launch adds the rows in a fixed order.
#include <algorithm>
#include "internal.h"
#include "args.h"
#include "vec_any.h"
#include "long_sum.h"

namespace tsm {

static constexpr int LN_NT = 256;

// N values of a row vector from c0, zero behind the C-th
template <int N>
__device__ __forceinline__ void ln_params(const float* p, int c0, int C, float (&f)[N]) {
#pragma unroll
    for (int h = 0; h < N; h += 4) {
        const auto v = raw_load<float, 4>(p + c0 + h, C - c0 - h);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[h + e] = raw_get<float>(v, e);
    }
}

// Sum over L adjacent lanes (L <= 64), or over the block's wavefronts as well (L == LN_NT; red: one slot per wavefront and
// parity, so that two sums in a row need one barrier each).
template <int L>
__device__ __forceinline__ float ln_sum(float v, float* red) {
#pragma unroll
    for (int o = (L < 64 ? L : 64) / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    if constexpr (L > 64) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < L / 64; ++w) v += red[w];
    }
    return v;
}

template <typename T, int L, int R>
__global__ void __launch_bounds__(LN_NT) ln_fwd_kernel(const T* __restrict__ x, const float* __restrict__ gamma, const float* __restrict__ beta,
                                                       T* __restrict__ y, float* __restrict__ mean_out, float* __restrict__ rstd_out, long rows,
                                                       int C, float eps) {
    constexpr int VE = Elem<T>::VEC;
    __shared__ float red[2][L > 64 ? LN_NT / 64 : 1];
    const int lane = threadIdx.x % L;
    float gm[R][VE], bt[R][VE];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        ln_params<VE>(gamma, (lane + r * L) * VE, C, gm[r]);
        ln_params<VE>(beta, (lane + r * L) * VE, C, bt[r]);
    }
    for (long row = (long)blockIdx.x * (LN_NT / L) + threadIdx.x / L; row < rows; row += (long)gridDim.x * (LN_NT / L)) {
        const T* xr = x + row * C;
        typename RawVec<T, VE>::type raw[R];
#pragma unroll
        for (int r = 0; r < R; ++r) raw[r] = raw_load<T, VE>(xr + (lane + r * L) * VE, C - (lane + r * L) * VE);
        float s = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < VE; ++e) s += raw_get<T>(raw[r], e);
        // (a quotient, not a product with 1 / C, which the compiler would fuse into x - mean: of a constant row that is zero then)
        const float mean = ln_sum<L>(s, red[0]) / (float)C;
        float q = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float d = (lane + r * L) * VE + e < C ? raw_get<T>(raw[r], e) - mean : 0.f;
                q = fmaf(d, d, q);
            }
        const float rstd = 1.f / sqrtf(ln_sum<L>(q, red[1]) / (float)C + eps);
        if (lane == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
        T* yr = y + row * C;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c0 = (lane + r * L) * VE;
            if (c0 >= C) break;
            float f[VE];
#pragma unroll
            for (int e = 0; e < VE; ++e) f[e] = fmaf((raw_get<T>(raw[r], e) - mean) * rstd, gm[r][e], bt[r][e]);
            raw_store<T, VE>(yr + c0, f, C - c0);
        }
    }
}

// Rows longer than the registers of a block: one block per row, which reads it three times (from L2 after the first).  (One register for a
// thread's share lets a row of 2^23 times 0.3 lose 3e-4 of its mean, of 2^25 1e-3, and the variance with it.)
template <typename T>
__global__ void __launch_bounds__(LN_NT) ln_fwd_long_kernel(const T* __restrict__ x, const float* __restrict__ gamma, const float* __restrict__ beta,
                                                            T* __restrict__ y, float* __restrict__ mean_out, float* __restrict__ rstd_out,
                                                            long rows, int C, float eps) {
    constexpr int VE = Elem<T>::VEC;
    __shared__ float red[2][LN_NT / 64];
    for (long row = blockIdx.x; row < rows; row += gridDim.x) {
        const T* xr = x + row * C;
        LongSum s;
        for (int c0 = threadIdx.x * VE; c0 < C; c0 += LN_NT * VE) {
            const auto raw = raw_load<T, VE>(xr + c0, C - c0);
            float t = 0.f;
#pragma unroll
            for (int e = 0; e < VE; ++e) t += raw_get<T>(raw, e);
            s.add(t);
        }
        const float mean = ln_sum<LN_NT>(s.get(), red[0]) / (float)C;
        LongSum q;
        for (int c0 = threadIdx.x * VE; c0 < C; c0 += LN_NT * VE) {
            const auto raw = raw_load<T, VE>(xr + c0, C - c0);
            float t = 0.f;
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float d = c0 + e < C ? raw_get<T>(raw, e) - mean : 0.f;
                t = fmaf(d, d, t);
            }
            q.add(t);
        }
        const float rstd = 1.f / sqrtf(ln_sum<LN_NT>(q.get(), red[1]) / (float)C + eps);
        if (threadIdx.x == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
        for (int c0 = threadIdx.x * VE; c0 < C; c0 += LN_NT * VE) {
            const auto raw = raw_load<T, VE>(xr + c0, C - c0);
            float f[VE];
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const int c = c0 + e < C ? c0 + e : C - 1;
                f[e] = fmaf((raw_get<T>(raw, e) - mean) * rstd, gamma[c], beta[c]);
            }
            raw_store<T, VE>(y + row * C + c0, f, C - c0);
        }
    }
}

// dgamma's and dbeta's shares of a block's rows, `step` values from block to block.
template <typename T, int L, int R>
__global__ void __launch_bounds__(LN_NT) ln_bwd_kernel(const T* __restrict__ x, const T* __restrict__ dy, const float* __restrict__ gamma,
                                                       const float* __restrict__ mean_in, const float* __restrict__ rstd_in, T* __restrict__ dx,
                                                       float* __restrict__ dgamma, float* __restrict__ dbeta, long step, long rows, int C) {
    constexpr int VE = Elem<T>::VEC;
    constexpr int G = LN_NT / L;                        // rows in flight per block
    __shared__ float red[2][L > 64 ? LN_NT / 64 : 1];
    __shared__ float share[G > 1 ? (G - 1) * L * R * VE : 1];
    const int lane = threadIdx.x % L, grp = threadIdx.x / L;
    const float inv = 1.f / (float)C;
    float gm[R][VE], ag[R][VE], ab[R][VE];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        ln_params<VE>(gamma, (lane + r * L) * VE, C, gm[r]);
#pragma unroll
        for (int e = 0; e < VE; ++e) ag[r][e] = ab[r][e] = 0.f;
    }
    for (long row = (long)blockIdx.x * G + grp; row < rows; row += (long)gridDim.x * G) {
        typename RawVec<T, VE>::type rx[R], rd[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c0 = (lane + r * L) * VE;
            rx[r] = raw_load<T, VE>(x + row * C + c0, C - c0);
            rd[r] = raw_load<T, VE>(dy + row * C + c0, C - c0);
        }
        const float mean = mean_in[row], rstd = rstd_in[row];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float d = raw_get<T>(rd[r], e), xh = (raw_get<T>(rx[r], e) - mean) * rstd, v = d * gm[r][e];
                const bool in = (lane + r * L) * VE + e < C;      // (rd and gm are zero outside, but 0 * NaN is not)
                s1 += v;
                s2 += in ? v * xh : 0.f;
                ag[r][e] += in ? d * xh : 0.f;
                ab[r][e] += d;
            }
        const float m1 = ln_sum<L>(s1, red[0]) * inv, m2 = ln_sum<L>(s2, red[1]) * inv;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c0 = (lane + r * L) * VE;
            if (c0 >= C) break;
            float f[VE];
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float xh = (raw_get<T>(rx[r], e) - mean) * rstd;
                f[e] = rstd * (fmaf(raw_get<T>(rd[r], e), gm[r][e], -m1) - xh * m2);
            }
            raw_store<T, VE>(dx + row * C + c0, f, C - c0);
        }
    }
    // the rows in flight meet in LDS, in a fixed order, one sum at a time
    for (int which = 0; which < 2; ++which) {
        float* out = (which ? dbeta : dgamma) + blockIdx.x * step;
        if constexpr (G > 1) {
            __syncthreads();
            if (grp > 0) {
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int e = 0; e < VE; ++e) share[((grp - 1) * R * VE + r * VE + e) * L + lane] = which ? ab[r][e] : ag[r][e];
            }
            __syncthreads();
        }
        if (grp == 0) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const int c = (lane + r * L) * VE + e;
                    float t = which ? ab[r][e] : ag[r][e];
                    if constexpr (G > 1) {
#pragma unroll 4
                        for (int g = 0; g < G - 1; ++g) t += share[(g * R * VE + r * VE + e) * L + lane];
                    }
                    if (c < C) out[c] = t;
                }
        }
    }
}

// Rows longer than the registers of a block: dx by one block per row (two reads, the second from L2) ...
template <typename T>
__global__ void __launch_bounds__(LN_NT) ln_bwd_long_kernel(const T* __restrict__ x, const T* __restrict__ dy, const float* __restrict__ gamma,
                                                            const float* __restrict__ mean_in, const float* __restrict__ rstd_in,
                                                            T* __restrict__ dx, long rows, int C) {
    constexpr int VE = Elem<T>::VEC;
    __shared__ float red[2][LN_NT / 64];
    for (long row = blockIdx.x; row < rows; row += gridDim.x) {
        const float mean = mean_in[row], rstd = rstd_in[row];
        LongSum s1, s2;
        for (int c0 = threadIdx.x * VE; c0 < C; c0 += LN_NT * VE) {
            const auto rx = raw_load<T, VE>(x + row * C + c0, C - c0);
            const auto rd = raw_load<T, VE>(dy + row * C + c0, C - c0);
            float t1 = 0.f, t2 = 0.f;
#pragma unroll
            for (int e = 0; e < VE; ++e)
                if (c0 + e < C) {
                    const float v = raw_get<T>(rd, e) * gamma[c0 + e];
                    t1 += v;
                    t2 = fmaf(v, (raw_get<T>(rx, e) - mean) * rstd, t2);
                }
            s1.add(t1);
            s2.add(t2);
        }
        const float m1 = ln_sum<LN_NT>(s1.get(), red[0]) / (float)C, m2 = ln_sum<LN_NT>(s2.get(), red[1]) / (float)C;
        for (int c0 = threadIdx.x * VE; c0 < C; c0 += LN_NT * VE) {
            const auto rx = raw_load<T, VE>(x + row * C + c0, C - c0);
            const auto rd = raw_load<T, VE>(dy + row * C + c0, C - c0);
            float f[VE];
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float g = gamma[c0 + e < C ? c0 + e : C - 1];
                f[e] = rstd * (fmaf(raw_get<T>(rd, e), g, -m1) - (raw_get<T>(rx, e) - mean) * rstd * m2);
            }
            raw_store<T, VE>(dx + row * C + c0, f, C - c0);
        }
    }
}
// ... and the weights' gradients by blocks of 64 vectors of columns times a share of the rows.
template <typename T>
__global__ void __launch_bounds__(LN_NT) ln_bwd_cols_kernel(const T* __restrict__ x, const T* __restrict__ dy, const float* __restrict__ mean_in,
                                                            const float* __restrict__ rstd_in, float* __restrict__ dgamma, float* __restrict__ dbeta, long step, long rows,
                                                            int C) {
    constexpr int VE = Elem<T>::VEC;
    __shared__ float share[3 * 64 * VE];
    const int lane = threadIdx.x & 63, grp = threadIdx.x >> 6;
    const long cblocks = (C + 64 * VE - 1) / (64 * VE);
    for (long cb = blockIdx.x; cb < cblocks; cb += gridDim.x) {
        const int c0 = (int)((cb * 64 + lane) * VE);
        float ag[VE], ab[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) ag[e] = ab[e] = 0.f;
        if (c0 < C)
            for (long row = (long)blockIdx.y * 4 + grp; row < rows; row += (long)gridDim.y * 4) {
                const auto rx = raw_load<T, VE>(x + row * C + c0, C - c0);
                const auto rd = raw_load<T, VE>(dy + row * C + c0, C - c0);
                const float mean = mean_in[row], rstd = rstd_in[row];
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const float d = raw_get<T>(rd, e);
                    ag[e] = fmaf(d, (raw_get<T>(rx, e) - mean) * rstd, ag[e]);
                    ab[e] += d;
                }
            }
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
            if (grp > 0)
#pragma unroll
                for (int e = 0; e < VE; ++e) share[((grp - 1) * VE + e) * 64 + lane] = which ? ab[e] : ag[e];
            __syncthreads();
            if (grp == 0)
#pragma unroll
                for (int e = 0; e < VE; ++e)
                    if (c0 + e < C) {
                        float t = which ? ab[e] : ag[e];
                        for (int g = 0; g < 3; ++g) t += share[(g * VE + e) * 64 + lane];
                        (which ? dbeta : dgamma)[blockIdx.y * step + c0 + e] = t;
                    }
        }
    }
}

// dgamma, dbeta = the sums of the partial rows: 64 columns x 16 row lanes per block and turn.
__global__ void __launch_bounds__(1024) ln_join_kernel(const float* __restrict__ partial, int nrows, int C, float* __restrict__ dgamma,
                                                       float* __restrict__ dbeta) {
    __shared__ float red[16][64];
    const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
    const long w2 = 2L * C;
    for (long w0 = blockIdx.x * 64L; w0 < w2; w0 += gridDim.x * 64L) {
        const long w = w0 + tx;
        float s = 0.f;
        if (w < w2)
#pragma unroll 4
            for (int r = ty; r < nrows; r += 16) s += partial[(size_t)r * w2 + w];
        if (w0 != blockIdx.x * 64L) __syncthreads();            // (the turn before has been read)
        red[ty][tx] = s;
        __syncthreads();
        if (ty == 0 && w < w2) {
            float t = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) t += red[r][tx];
            if (w < C) dgamma[w] = t;
            else dbeta[w - C] = t;
        }
    }
}

// ---- host --------------------------------------------------------------------------------
// Blocks keep gamma and beta over their rows (200704 x 256 bf16: 512 52, 1024 37, 2048 36, 4096 48, 8192 67 us; inputs
// from HBM, 1024, 2048, 4096: 43, 38, 38, 400000 x 64 34, 30, 29, 25088 x 2048 42, 38, 38, 6000 x 8192 36, 37, 41).
static constexpr int LN_FWD_BLOCKS = 2048;
// Rows that a thread adds up in turn for dgamma and dbeta, at most; of more rows there are more blocks and partial rows.  (512 blocks for all: 2^26
// rows of 8 channels, 8192 in turn, lose 1.2e-4 of a sum of one sign, and twice that of twice the rows.)
static constexpr int64_t LN_CHAIN = 512;
static constexpr long LN_JOIN_BLOCKS = 1 << 16;      // (2^32 threads are more than a launch has: 2 x 2^27 columns in one turn)
static constexpr int LN_BLOCKS = 512;     // of the backward pass: two per CU, each writes one partial row (25088 x 2048 bf16: 256 73, 512 56, 1024 63 us; both
                                          // passes of 6000 x 4096 76, 67, 75, of 200704 x 256 153, 111, 97, of 400000 x 64 144, 98, 76)

// Lanes and vectors per lane of a row; 0 lanes: the row exceeds a block's registers.  Few vectors per lane keep many rows in
// flight, up to four they cost no barrier.
static void ln_shape(int C, int dtype, int* L, int* R) {
    const int nv = cdiv(C, dtype == TSM_BF16 ? 8 : 4);
    if (nv <= 16) { *L = 16; *R = 1; }
    else if (nv <= 32) { *L = 32; *R = 1; }
    else if (nv <= 64) { *L = 64; *R = 1; }
    else if (nv <= 128) { *L = 64; *R = 2; }
    else if (nv <= 256) { *L = 64; *R = 4; }
    else if (nv <= 512) { *L = 256; *R = 2; }
    else if (nv <= 1024) { *L = 256; *R = 4; }
    else *L = *R = 0;
}

#define LN_DISPATCH(T, CALL)                                  \
    do {                                                      \
        if (L == 16) CALL(T, 16, 1);                          \
        else if (L == 32) CALL(T, 32, 1);                     \
        else if (L == 64 && R == 1) CALL(T, 64, 1);           \
        else if (L == 64 && R == 2) CALL(T, 64, 2);           \
        else if (L == 64) CALL(T, 64, 4);                     \
        else if (R == 2) CALL(T, 256, 2);                     \
        else CALL(T, 256, 4);                                 \
    } while (0)

static int ln_check(const tsm_layernorm_desc* d, const char* who) {
    if (!d) return fail(TSM_ERR_NULLPTR, "%s: null descriptor", who);
    if (d->dtype != TSM_F32 && d->dtype != TSM_BF16) return fail(TSM_ERR_DTYPE, "%s: unknown dtype %d", who, d->dtype);
    if (d->rows <= 0 || d->C <= 0) return fail(TSM_ERR_SHAPE, "%s: non-positive dimension", who);
    if (d->rows > ((int64_t)1 << 60) / d->C || d->C > (1 << 30)) return fail(TSM_ERR_SHAPE, "%s: tensor too large", who);
    if (!(d->eps >= 0.f)) return fail(TSM_ERR_SHAPE, "%s: eps must not be negative or NaN", who);
    return TSM_OK;
}

static int ln_bwd_blocks(const tsm_layernorm_desc* d) {
    int L, R;
    ln_shape(d->C, d->dtype, &L, &R);
    if (L == 0)     // row shares of ln_bwd_cols_kernel, by four wavefronts each
        return (int)std::min(std::max(std::min((d->rows + 31) / 32, (int64_t)16), (d->rows + 4 * LN_CHAIN - 1) / (4 * LN_CHAIN)), (int64_t)65535);
    const int64_t groups = (d->rows + LN_NT / L - 1) / (LN_NT / L);
    return groups <= 2 ? 1 : (int)std::min(std::max(std::min(groups, (int64_t)LN_BLOCKS), (groups + LN_CHAIN - 1) / LN_CHAIN), (int64_t)1 << 22);
}

static size_t ln_ws_bytes(const tsm_layernorm_desc* d) { return align_up((size_t)ln_bwd_blocks(d) * 2 * d->C * sizeof(float)); }

template <typename T>
static int ln_fwd(const tsm_layernorm_desc* d, const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd, hipStream_t s) {
    int L, R;
    ln_shape(d->C, d->dtype, &L, &R);
    const int64_t jobs = L ? (d->rows + LN_NT / L - 1) / (LN_NT / L) : d->rows;
    const dim3 grid((unsigned)(jobs < LN_FWD_BLOCKS ? jobs : LN_FWD_BLOCKS)), block(LN_NT);
#define CALL(T, L, R) ln_fwd_kernel<T, L, R><<<grid, block, 0, s>>>((const T*)x, gamma, beta, (T*)y, mean, rstd, d->rows, d->C, d->eps)
    if (L == 0) ln_fwd_long_kernel<T><<<dim3((unsigned)(jobs < (1 << 22) ? jobs : (1 << 22))), block, 0, s>>>((const T*)x, gamma, beta, (T*)y, mean, rstd, d->rows, d->C, d->eps);
    else LN_DISPATCH(T, CALL);
#undef CALL
    return check_launch("layernorm_fwd");
}

template <typename T>
static int ln_bwd(const tsm_layernorm_desc* d, const void* x, const void* dy, const float* gamma, const float* mean, const float* rstd, void* dx,
                  float* dgamma, float* dbeta, float* partial, hipStream_t s) {
    int L, R;
    ln_shape(d->C, d->dtype, &L, &R);
    const int nb = ln_bwd_blocks(d);
    const dim3 grid((unsigned)nb), block(LN_NT);
    // one block's shares are the result (16 rows of 43, call after call: 10.2 -> 8.3 us)
    float *pg = nb > 1 ? partial : dgamma, *pb = nb > 1 ? partial + d->C : dbeta;
    const long step = 2L * d->C;
#define CALL(T, L, R) ln_bwd_kernel<T, L, R><<<grid, block, 0, s>>>((const T*)x, (const T*)dy, gamma, mean, rstd, (T*)dx, pg, pb, step, d->rows, d->C)
    if (L == 0) {
        const dim3 rgrid((unsigned)(d->rows < (1 << 22) ? d->rows : (1 << 22)));
        ln_bwd_long_kernel<T><<<rgrid, block, 0, s>>>((const T*)x, (const T*)dy, gamma, mean, rstd, (T*)dx, d->rows, d->C);
        TSM_TRY(check_launch("layernorm_bwd_rows"));
        const int64_t cb = cdiv(d->C, 64 * Elem<T>::VEC);
        ln_bwd_cols_kernel<T><<<dim3((unsigned)cb, (unsigned)nb), block, 0, s>>>((const T*)x, (const T*)dy, mean, rstd, pg, pb, step, d->rows, d->C);
    } else {
        LN_DISPATCH(T, CALL);
    }
#undef CALL
    TSM_TRY(check_launch("layernorm_bwd"));
    if (nb == 1) return TSM_OK;
    ln_join_kernel<<<dim3((unsigned)std::min((2L * d->C + 63) / 64, LN_JOIN_BLOCKS)), dim3(1024), 0, s>>>(partial, nb, d->C, dgamma, dbeta);
    return check_launch("layernorm_join");
}

}  // namespace tsm

using namespace tsm;

extern "C" {

size_t tsm_layernorm_workspace_bytes(const tsm_layernorm_desc* d) {
    return ln_check(d, "tsm_layernorm_workspace_bytes") == TSM_OK ? ln_ws_bytes(d) : 0;
}

int tsm_layernorm_fwd(const tsm_layernorm_desc* d, const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd,
                      void* stream) {
    const char* who = "tsm_layernorm_fwd";
    TSM_TRY(ln_check(d, who));
    if (!x || !gamma || !beta || !y) return fail(TSM_ERR_NULLPTR, "%s: null pointer", who);
    const size_t n = (size_t)d->rows * d->C * dtype_size(d->dtype), cb = (size_t)d->C * 4, rb = (size_t)d->rows * 4;
    const Span in[] = {{x, n, "x"}, {gamma, cb, "gamma"}, {beta, cb, "beta"}}, out[] = {{y, n, "y"}, {mean, rb, "mean"}, {rstd, rb, "rstd"}};
    TSM_TRY(check_spans(who, in, 3, out, 3));
    const hipStream_t s = (hipStream_t)stream;
    return d->dtype == TSM_BF16 ? ln_fwd<bf16_t>(d, x, gamma, beta, y, mean, rstd, s) : ln_fwd<float>(d, x, gamma, beta, y, mean, rstd, s);
}

int tsm_layernorm_bwd(const tsm_layernorm_desc* d, const void* x, const void* dy, const float* gamma, const float* mean, const float* rstd,
                      void* dx, float* dgamma, float* dbeta, void* ws, size_t ws_bytes, void* stream) {
    const char* who = "tsm_layernorm_bwd";
    TSM_TRY(ln_check(d, who));
    if (!x || !dy || !gamma || !mean || !rstd || !dx || !dgamma || !dbeta) return fail(TSM_ERR_NULLPTR, "%s: null pointer", who);
    const size_t need = ln_ws_bytes(d);
    if (ws_bytes < need) return fail(TSM_ERR_WORKSPACE, "%s: workspace %zu bytes, need %zu", who, ws_bytes, need);
    if (!ws) return fail(TSM_ERR_NULLPTR, "%s: null workspace", who);
    const size_t n = (size_t)d->rows * d->C * dtype_size(d->dtype), cb = (size_t)d->C * 4, rb = (size_t)d->rows * 4;
    const Span in[] = {{x, n, "x"}, {dy, n, "dy"}, {gamma, cb, "gamma"}, {mean, rb, "mean"}, {rstd, rb, "rstd"}};
    const Span out[] = {{dx, n, "dx"}, {dgamma, cb, "dgamma"}, {dbeta, cb, "dbeta"}, {ws, need, "the workspace"}};
    TSM_TRY(check_spans(who, in, 5, out, 4));
    const hipStream_t s = (hipStream_t)stream;
    return d->dtype == TSM_BF16 ? ln_bwd<bf16_t>(d, x, dy, gamma, mean, rstd, dx, dgamma, dbeta, (float*)ws, s)
                                : ln_bwd<float>(d, x, dy, gamma, mean, rstd, dx, dgamma, dbeta, (float*)ws, s);
}

}  // extern "C"
