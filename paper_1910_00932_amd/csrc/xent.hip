// Linear classifier with softmax cross entropy whose logits are never stored, and its gradients.
//
//   s = x w^T + b;  lse_r = log sum_v exp s_rv;  loss_r = lse_r - s_r,label  (0 for rows whose label is no class)
//   G_rv = dloss_r (exp(s_rv - lse_r) - [v == label_r]);  dx = G w;  dw = G^T x;  db_v = sum_r G_rv
//
// Forward: tiles of s stay in registers; each leaves the maximum and the sum of exponentials of its columns per row (a softmax
// joined over the tiles) and the label's logit.  Backward: s is formed again in pieces of the classes, a piece of G in the storage
// type lives in the workspace for the two products that read it.  G is rounded once to the storage type, as the operands of the
// matrix cores are; lse, the losses, db (from G before that rounding) and all sums are fp32.
#include <type_traits>
#include "internal.h"
#include "args.h"
#include "vec_any.h"

namespace tsm {

typedef float x_f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 x_bf16x8 __attribute__((ext_vector_type(8)));

struct XentEpi {
    // STATS
    float2* part;            // [N tiles][M]: maximum and sum of exp(s - maximum) of a tile's columns
    float* picked;           // [M]: the label's logit
    // STATS and GRAD: columns are classes col0 + n of `classes`
    const float* bias;
    const int32_t* labels;
    long col0, classes;
    // GRAD
    const float *lse, *dloss;
    void* G;                 // [M][ldg], zero behind the last column; the main tiles': blocks (X_GROWS), ldg elements per row tile
    long ldg;
    float* dbias_part;       // [M tiles][lddb], nullable
    long lddb;
    // OUT
    const float* acc;        // fp32 [M][N] added to the result, nullable
    float* out_f32;          // [splits][M][N], or
    void* out;               // [M][N] in the storage type
};

struct XentArgs {
    const void *A, *B;
    long lda, ldb, M, N, K, ksplit;    // ksplit: K of one split (grid.z)
    const int32_t* klabels;            // rows k of B whose label is no class of `classes` count as zero; nullable
    XentEpi e;
};

enum { XE_STATS = 0, XE_GRAD = 1, XE_OUT = 2 };

__device__ __forceinline__ bool is_class(int label, long classes) { return label >= 0 && label < classes; }

// exp(v - m) with exp(-inf - -inf) = 0: a column without any weight
__device__ __forceinline__ float exp_below(float v, float m) { return v == -__builtin_inff() && v == m ? 0.f : __expf(v - m); }
// joins (m, s) with (m2, s2)
__device__ __forceinline__ void join_softmax(float& m, float& s, float m2, float s2) {
    const float t = fmaxf(m, m2);
    s = (m == t ? s : s * __expf(m - t)) + (m2 == t ? s2 : s2 * __expf(m2 - t));
    m = t;
}

// ---- the plain tile: 64 x 64 results, the four wavefronts take every fourth step of K ---------------------------------
// AK / BK: the operand has K consecutive in memory ([rows][K]), else its rows are K ([K][rows]).
template <typename T, bool KC>
__device__ __forceinline__ void plain_frag(const T* P, long ld, long row, long rows, long k, long K, const int32_t* klabels, long classes,
                                           typename RawVec<T, 16 / sizeof(T)>::type& f) {
    constexpr int VE = 16 / sizeof(T);
    if constexpr (KC) {
        f = raw_load<T, VE>(P + row * ld + k, row < rows ? (int)(K - k < VE ? K - k : VE) : 0);
    } else {
        f = typename RawVec<T, VE>::type{};
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            if (row < rows && k + e < K && (!klabels || is_class(klabels[k + e], classes))) {
                if constexpr (sizeof(T) == 2) f[e >> 1] |= (uint32_t)P[(k + e) * ld + row] << (16 * (e & 1));
                else f[e] = __float_as_uint(P[(k + e) * ld + row]);
            }
        }
    }
}

template <typename T, int MODE, bool AK, bool BK>
__global__ void __launch_bounds__(256) xent_plain_kernel(XentArgs a) {
    constexpr int VE = 16 / sizeof(T), KSTEP = 2 * VE;
    __shared__ float red[4][64][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hi = lane >> 5, lo = lane & 31;
    const long ntiles = (a.N + 63) / 64, total = ntiles * ((a.M + 63) / 64);
    const long kb = blockIdx.z * a.ksplit, ke = kb + a.ksplit < a.K ? kb + a.ksplit : a.K;
    const T *A = (const T*)a.A, *B = (const T*)a.B;
    for (long tile = blockIdx.x; tile < total; tile += gridDim.x) {
    const long mt = tile / ntiles, nt = tile % ntiles;
    const long m0 = mt * 64, n0 = nt * 64;
    x_f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    for (long k0 = kb + wave * KSTEP; k0 < ke; k0 += 4 * KSTEP) {
        typename RawVec<T, VE>::type fa[2], fb[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            plain_frag<T, AK>(A, a.lda, m0 + 32 * i + lo, a.M, k0 + hi * VE, ke, nullptr, 0, fa[i]);
            plain_frag<T, BK>(B, a.ldb, n0 + 32 * i + lo, a.N, k0 + hi * VE, ke, a.klabels, a.e.classes, fb[i]);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if constexpr (sizeof(T) == 2)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(x_bf16x8, fa[i]), __builtin_bit_cast(x_bf16x8, fb[j]), acc[i][j], 0, 0, 0);
                else
#pragma unroll
                    for (int e = 0; e < VE; ++e)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(fa[i][e]), __uint_as_float(fb[j][e]), acc[i][j], 0, 0, 0);
            }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) red[wave][i * 32 + 8 * (r / 4) + 4 * hi + r % 4][j * 32 + lo] = acc[i][j][r];
    __syncthreads();
    // one row of the tile at a time per wavefront, a column per lane
    const long n = n0 + lane;
    const long v = a.e.col0 + n;
    const bool in = n < a.N;
    const float bias = MODE != XE_OUT && in && a.e.bias ? a.e.bias[v] : 0.f;
    float dbias = 0.f;
    for (int q = 0; q < 16; ++q) {
        const int row = wave * 16 + q;
        const long m = m0 + row;
        if (m >= a.M) break;
        float s = (red[0][row][lane] + red[1][row][lane]) + (red[2][row][lane] + red[3][row][lane]);
        if constexpr (MODE == XE_STATS) {
            s = in ? s + bias : -__builtin_inff();
            if (in && a.e.labels[m] == v) a.e.picked[m] = s;
            float mx = s;
            for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
            float t = in ? exp_below(s, mx) : 0.f;
            for (int o = 32; o > 0; o >>= 1) t += __shfl_xor(t, o, 64);
            if (lane == 0) a.e.part[nt * a.M + m] = make_float2(mx, t);
        } else if constexpr (MODE == XE_GRAD) {
            const int label = a.e.labels[m];
            float g = 0.f;
            if (in && is_class(label, a.e.classes)) {
                const float p = __expf(s + bias - a.e.lse[m]);
                g = a.e.dloss[m] * (label == v ? p - 1.f : p);
            }
            dbias += g;
            if (n < a.e.ldg) ((T*)a.e.G)[m * a.e.ldg + n] = Elem<T>::st(g);
        } else if (in) {
            if (a.e.acc) s += a.e.acc[m * a.N + n];
            if (a.e.out_f32) a.e.out_f32[(blockIdx.z * a.M + m) * a.N + n] = s;
            else ((T*)a.e.out)[m * a.N + n] = Elem<T>::st(s);
        }
    }
    if constexpr (MODE == XE_GRAD) {
        if (a.e.dbias_part) {
            __syncthreads();
            red[0][wave][lane] = dbias;
            __syncthreads();
            if (wave == 0 && in) a.e.dbias_part[mt * a.e.lddb + n] = (red[0][0][lane] + red[0][1][lane]) + (red[0][2][lane] + red[0][3][lane]);
        }
    }
    __syncthreads();
    }
}

// ---- the main tile: bf16, BM x BN results, eight wavefronts that share the operands through LDS -------------------------
// Operands come 64 steps of K at a time, straight from memory into one of two LDS stages while the other is multiplied.  An
// operand with consecutive K lies there as rows of 128 bytes whose eight 16-byte pieces are permuted by the row (piece ^ (row/2)%8),
// so that the 32 rows of a fragment read spread over all banks; one whose rows are K lies there as it does in memory, its
// 32-byte granules permuted by K, and fragments are read through the transposing LDS read, four K of 16 columns at a time.
static constexpr int XBK = 64;
static constexpr int X_GTILE = 256;                // rows of a block of G, and columns of the tiles that write them
static constexpr uint32_t X_OOB = 0x80000000u;     // beyond every buffer: such lanes of a load leave zeros

__device__ __forceinline__ __amdgpu_buffer_rsrc_t x_rsrc(const void* base) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, 0x7fffffff, 0x00020000);
}
__device__ __forceinline__ void x_load_lds16(__amdgpu_buffer_rsrc_t r, unsigned char* at, uint32_t voff, int soff) {
#if defined(__HIP_DEVICE_COMPILE__)   // (the host pass of the compiler knows no such address space)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)at, 16, (int)voff, soff, 0, 0);
#endif
}
template <int VM> __device__ __forceinline__ void x_wait() {     // at most VM memory operations and no LDS access outstanding
    __builtin_amdgcn_s_waitcnt((VM & 15) | (7 << 4) | (0 << 8) | ((VM >> 4) << 14));
}
__device__ __forceinline__ void x_wait_lds() {                    // no LDS access outstanding
    __builtin_amdgcn_s_waitcnt(0xf | (7 << 4) | (0 << 8) | (3 << 14));
}
__device__ __forceinline__ void x_barrier() {
    asm volatile("" ::: "memory");   // (a fence would also wait for every load into LDS in flight)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
typedef short x_s16x4 __attribute__((ext_vector_type(4)));
typedef short x_s16x8 __attribute__((ext_vector_type(8)));

// How an operand lies in memory.  The blocks of G: [row tile][64 columns][256 rows], 32 KB each, so that a step of either product
// reads stretches of 8 KB and more, where rows of G as such would be a 64 KB apart.
enum { X_ROWS = 0, X_COLS = 1, X_GROWS = 2, X_GCOLS = 3 };     // [rows][K], [K][rows], G with its columns as K, with its rows as K

// One operand of a tile: ROWS rows of the result's side.
template <int ROWS, int KIND, int NT>
struct XOperand {
    static constexpr bool KC = KIND == X_ROWS || KIND == X_GROWS;     // K consecutive in LDS
    static constexpr int BYTES = ROWS * XBK * 2;
    static constexpr int PIECES = BYTES / (NT * 16);          // per thread and step
    static constexpr int RPP = KC ? NT / 8 : NT / (ROWS / 8); // rows of the LDS image per pass
    static constexpr int PITCH = KC ? XBK * 2 : ROWS * 2;     // its bytes
    static constexpr int GMASK = ROWS / 16 - 1;               // granules of 16 columns
    uint32_t off[PIECES];         // byte offset in the step's window of this thread's pieces
    int kfirst;                   // KC: K of the piece, else K of the thread's row in a pass
    const char* base;             // of the step's window
    long step;                    // bytes from one step to the next
    int quarter;                  // X_GCOLS: steps into a row tile

    __device__ __forceinline__ static int swz(int k) { return ((((k & 3) << 1) | (((k >> 3) & 1) << 3))) & GMASK; }

    // row0: first row of the tile, rows: of the matrix; k0: first K.  ld: elements from row to row, for G from one row tile to the next.
    __device__ __forceinline__ void init(const bf16_t* p, long ld, long row0, long rows, long k0, int tid) {
        quarter = 0;
        if constexpr (KC) {
            const int r = tid / 8;
            const int kv = (tid % 8) ^ ((r >> 1) & 7);
            kfirst = kv * 8;
            const long pitch = KIND == X_GROWS ? XBK : ld;
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
                off[i] = row0 + i * RPP + r < rows ? (uint32_t)((i * RPP + r) * pitch * 2 + kv * 16) : X_OOB;
            base = KIND == X_GROWS ? (const char*)(p + row0 / ROWS * ld + k0 * ROWS) : (const char*)(p + row0 * ld + k0);
            step = KIND == X_GROWS ? ROWS * XBK * 2 : XBK * 2;
        } else {
            const int k = tid / (ROWS / 8), slot = tid % (ROWS / 8);
            kfirst = k;
            const int col = (((slot >> 1) ^ swz(k)) << 4) + (slot & 1) * 8;
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const long at = KIND == X_GCOLS ? col / XBK * (X_GTILE * XBK) + (i * RPP + k) * XBK + col % XBK : (i * RPP + k) * ld + col;
                off[i] = row0 + col < rows ? (uint32_t)(at * 2) : X_OOB;
            }
            if constexpr (KIND == X_GCOLS) {
                quarter = (int)(k0 % X_GTILE / XBK);
                base = (const char*)(p + k0 / X_GTILE * ld + row0 * X_GTILE + k0 % X_GTILE * XBK);
                step = (ld - (X_GTILE - XBK) * XBK) * 2;       // into the next row tile
            } else {
                base = (const char*)(p + k0 * ld + row0);
                step = XBK * 2 * ld;
            }
        }
    }
    __device__ __forceinline__ void advance() {
        if constexpr (KIND == X_GCOLS) {
            const bool last = quarter == X_GTILE / XBK - 1;
            base += last ? step : (long)XBK * XBK * 2;
            quarter = last ? 0 : quarter + 1;
        } else {
            base += step;
        }
    }
    // Piece i of the step at the window: left = K from its start to the end; mask: bit k clear for rows k that count as zero.
    __device__ __forceinline__ void load(unsigned char* stage, int i, int left, uint64_t mask, int wave_u) const {
        const int k = KC ? kfirst : i * RPP + kfirst;
        const bool in = k < left && (KC || (mask >> k) & 1);
        x_load_lds16(x_rsrc(base), stage + i * (NT * 16) + wave_u * 1024, in ? off[i] : X_OOB, 0);
    }
    // Where a lane reads the fragment of the 32 rows from row0 (a multiple of 32), K consecutive: of slice ks, else of slice 0.
    __device__ __forceinline__ static uint32_t frag_at(int row0, int ks, int lane) {
        if constexpr (KC) {
            const int r = lane & 31, hi = lane >> 5;
            return (row0 + r) * PITCH + (((2 * ks + hi) ^ ((r >> 1) & 7)) * 16);
        } else {
            const int c = lane & 3, e = (lane >> 2) & 3, mblk = (lane >> 4) & 1, kg = lane >> 5;
            return (8 * kg + e) * PITCH + ((row0 / 16 + mblk) ^ swz(8 * kg + e)) * 32 + c * 8;
        }
    }
};

// The fragments of a K slice, four of A and two of B, read and waited for in one block: as separate reads the compiler, which
// cannot tell the stage being read from the one that loads are on their way to, waits for those loads first.
__device__ __forceinline__ x_bf16x8 x_join(x_s16x4 lo, x_s16x4 up) {
    return __builtin_bit_cast(x_bf16x8, (x_s16x8)__builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7));
}
// both with consecutive K: one address each, fragments 32 rows apart
__device__ __forceinline__ void read_frags(uint32_t a, uint32_t b, x_bf16x8 (&fa)[4], x_bf16x8 (&fb)[2]) {
    asm volatile("ds_read_b128 %0, %6\n ds_read_b128 %4, %7\n ds_read_b128 %1, %6 offset:4096\n ds_read_b128 %5, %7 offset:4096\n"
                 "ds_read_b128 %2, %6 offset:8192\n ds_read_b128 %3, %6 offset:12288\n s_waitcnt lgkmcnt(0)"
                 : "=&v"(fa[0]), "=&v"(fa[1]), "=&v"(fa[2]), "=&v"(fa[3]), "=&v"(fb[0]), "=&v"(fb[1])
                 : "v"(a), "v"(b) : "memory");
}
// B through the transposing read: one address per fragmnt, slice OFF, its K 4 to 7 at OFF2
template <int OFF, int OFF2>
__device__ __forceinline__ void read_frags(uint32_t a, const uint32_t (&b)[2], x_bf16x8 (&fa)[4], x_bf16x8 (&fb)[2]) {
    x_s16x4 l0, l1, u0, u1;
    asm volatile("ds_read_b128 %0, %8\n ds_read_b64_tr_b16 %4, %9 offset:%11\n ds_read_b64_tr_b16 %5, %9 offset:%12\n"
                 "ds_read_b128 %1, %8 offset:4096\n ds_read_b64_tr_b16 %6, %10 offset:%11\n ds_read_b64_tr_b16 %7, %10 offset:%12\n"
                 "ds_read_b128 %2, %8 offset:8192\n ds_read_b128 %3, %8 offset:12288\n s_waitcnt lgkmcnt(0)"
                 : "=&v"(fa[0]), "=&v"(fa[1]), "=&v"(fa[2]), "=&v"(fa[3]), "=&v"(l0), "=&v"(u0), "=&v"(l1), "=&v"(u1)
                 : "v"(a), "v"(b[0]), "v"(b[1]), "n"(OFF), "n"(OFF2) : "memory");
    fb[0] = x_join(l0, u0);
    fb[1] = x_join(l1, u1);
}
// both through it
template <int OFF, int OFF2>
__device__ __forceinline__ void read_frags(const uint32_t (&a)[4], const uint32_t (&b)[2], x_bf16x8 (&fa)[4], x_bf16x8 (&fb)[2]) {
    x_s16x4 l[6], u[6];
    asm volatile("ds_read_b64_tr_b16 %0, %12 offset:%18\n ds_read_b64_tr_b16 %1, %12 offset:%19\n ds_read_b64_tr_b16 %8, %16 offset:%18\n"
                 "ds_read_b64_tr_b16 %9, %16 offset:%19\n ds_read_b64_tr_b16 %2, %13 offset:%18\n ds_read_b64_tr_b16 %3, %13 offset:%19\n"
                 "ds_read_b64_tr_b16 %10, %17 offset:%18\n ds_read_b64_tr_b16 %11, %17 offset:%19\n ds_read_b64_tr_b16 %4, %14 offset:%18\n"
                 "ds_read_b64_tr_b16 %5, %14 offset:%19\n ds_read_b64_tr_b16 %6, %15 offset:%18\n ds_read_b64_tr_b16 %7, %15 offset:%19\n"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(l[0]), "=&v"(u[0]), "=&v"(l[1]), "=&v"(u[1]), "=&v"(l[2]), "=&v"(u[2]), "=&v"(l[3]), "=&v"(u[3]), "=&v"(l[4]), "=&v"(u[4]),
                   "=&v"(l[5]), "=&v"(u[5])
                 : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(b[0]), "v"(b[1]), "n"(OFF), "n"(OFF2) : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) fa[i] = x_join(l[i], u[i]);
#pragma unroll
    for (int j = 0; j < 2; ++j) fb[j] = x_join(l[4 + j], u[4 + j]);
}

// Two words that the two halves of a wavefront hold of adjacent column quads, x of quads 0 | 1, y of quads 2 | 3: afterwards the lower
// half has quads 0, 1 and the upper half quads 2, 3.
__device__ __forceinline__ void swap_halves(uint32_t& x, uint32_t& y) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(x, y, false, false));
    x = r[0];
    y = r[1];
}

// Sum over the 32 lanes of a half, in its last lane: within rows of 16 lanes by data-parallel moves, then across the two rows.
template <int CTRL> __device__ __forceinline__ float dpp_add(float v) {
    return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float sum32(float v) {
    v = dpp_add<0xB1>(v);         // quad_perm 1 0 3 2
    v = dpp_add<0x4E>(v);         // quad_perm 2 3 0 1
    v = dpp_add<0x141>(v);        // row_half_mirror
    v = dpp_add<0x140>(v);        // row_mirror
    return v + __shfl_xor(v, 16, 64);
}

static constexpr int X_BM = 256, X_BN = 256, X_WM = 2, X_WN = 4, X_NT = X_WM * X_WN * 64, X_BLOCKS = 1 << 22;   // of one launch, at most
static constexpr int X_STAGE = (X_BM + X_BN) * XBK * 2;
static constexpr int X_SMEM = 2 * X_STAGE + X_WN * X_BM * 8 + X_BN * 4;   // two stages, row statistics, biases

// One block per CU at a time.  (Persistent blocks that load a tile's first steps behind the epilogue of the tile before are no faster: the
// epilogue is 3 of 58 us at 2048 features.)
// DB: the column sums of G are wanted.
template <int MODE, int AKIND, int BKIND, bool DB>
__global__ void __launch_bounds__(X_NT) xent_tile_kernel(XentArgs a, const uint64_t* __restrict__ kmask, long job0) {
    constexpr int BM = X_BM, BN = X_BN, WM = X_WM, WN = X_WN, NT = X_NT, MI = BM / (WM * 32), NJ = BN / (WN * 32);
    typedef XOperand<BM, AKIND, NT> OpA;
    typedef XOperand<BN, BKIND, NT> OpB;
    constexpr int NP = OpA::PIECES + OpB::PIECES;
    constexpr float L2E = 1.44269502f;
    static_assert(MI == 4 && NJ == 2 && XBK == 64, "read_frags");
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    float2* s_part = (float2*)(smem + 2 * X_STAGE);             // [WN][BM]; the column sums of G as floats [WM][BN]
    float* s_bias = (float*)(smem + 2 * X_STAGE + WN * BM * 8); // [BN]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, hi = lane >> 5, lo = lane & 31;
    const int wave_u = __builtin_amdgcn_readfirstlane(wave);
    const int wm = wave_u / WN, wn = wave_u % WN;

    // Jobs: the tiles of every split of K, four row tiles at a time (eight where the classes run along columns), column by column.
    // Every XCD takes a stretch of that order, so that the tiles it works on at one time share their operands in its L2 (bands
    // of 2, 4, 8, 16, 32 row tiles: dw 4.23, 4.19, 4.42, 4.98, 5.24 ms of 8192 x 2048 x 131072, statistics 3.95, 3.89, 3.80, 3.90, 4.35).
    constexpr int BAND = MODE == XE_OUT ? 4 : 8;
    const long mtiles = (a.M + BM - 1) / BM, ntiles = (a.N + BN - 1) / BN, tiles = mtiles * ntiles;
    const int njobs = gridDim.x;
    const int xcd = blockIdx.x & 7;
    const long job = job0 + xcd * (njobs / 8) + (xcd < njobs % 8 ? xcd : njobs % 8) + (blockIdx.x >> 3), tile = job % tiles, z = job / tiles;
    const long band = tile / (BAND * ntiles), rest = tile - band * BAND * ntiles;
    const long high = mtiles - band * BAND < BAND ? mtiles - band * BAND : BAND;
    const long mt = band * BAND + rest % high, nt = rest / high;
    const long m0 = mt * BM, n0 = nt * BN;
    const long kb = z * a.ksplit, ke = kb + a.ksplit < a.K ? kb + a.ksplit : a.K;
    const int steps = ke > kb ? (int)((ke - kb + XBK - 1) / XBK) : 0;
    OpA pa;
    OpB pb;
    auto load_step = [&](int stage, int kc) {                   // the step at the operands' windows
        unsigned char* st = smem + stage * X_STAGE;
        const long l = ke - kb - (long)kc * XBK;
        const int left = l < XBK ? (int)l : XBK;
        uint64_t mask = ~0ull;
        if constexpr (AKIND == X_GCOLS) mask = ((const __attribute__((address_space(4))) uint64_t*)kmask)[kb / XBK + kc];
#pragma unroll
        for (int q = 0; q < OpA::PIECES; ++q) pa.load(st, q, left, ~0ull, wave_u);
#pragma unroll
        for (int q = 0; q < OpB::PIECES; ++q) pb.load(st + OpA::BYTES, q, left, mask, wave_u);
    };
    auto next_step = [&](int stage, int kc) {
        pa.advance();
        pb.advance();
        load_step(stage, kc);
    };

    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const unsigned char*)smem;
    uint32_t aat[4], bat[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        aat[q] = lds0 + (OpA::KC ? OpA::frag_at(wm * (BM / WM), q, lane) : OpA::frag_at(wm * (BM / WM) + q * 32, 0, lane));
        if (OpB::KC || q < NJ) bat[q] = lds0 + OpA::BYTES + (OpB::KC ? OpB::frag_at(wn * (BN / WN), q, lane) : OpB::frag_at(wn * (BN / WN) + q * 32, 0, lane));
    }
    x_bf16x8 af[2][MI], bf[2][NJ];
    auto read = [&](auto slice, int stage) {
        constexpr int ks = decltype(slice)::value, f = ks & 1;
        const uint32_t so = stage * X_STAGE;
        if constexpr (OpA::KC && OpB::KC) {
            read_frags(aat[ks] + so, bat[ks] + so, af[f], bf[f]);
        } else {
            const uint32_t b[2] = {bat[0] + so, bat[1] + so};
            if constexpr (OpA::KC) {
                read_frags<16 * ks * OpB::PITCH, (16 * ks + 4) * OpB::PITCH>(aat[ks] + so, b, af[f], bf[f]);
            } else {
                const uint32_t q[4] = {aat[0] + so, aat[1] + so, aat[2] + so, aat[3] + so};
                read_frags<16 * ks * OpB::PITCH, (16 * ks + 4) * OpB::PITCH>(q, b, af[f], bf[f]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    x_f32x16 acc[MI][NJ];
    auto multiply = [&](int f) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j)      // the result's columns run along registers, its rows along lanes
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bf[f][j], af[f][i], acc[i][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    typedef std::integral_constant<int, 0> S0;
    typedef std::integral_constant<int, 1> S1;
    typedef std::integral_constant<int, 2> S2;
    typedef std::integral_constant<int, 3> S3;

#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

        // One barrier per step, in front of its last group of products: behind it the next step is complete and this stage is
        // free, and the loads of the step after next go to it, a whole step ahead of their barrier.  The reads of a slice wait on their
        // own; of the two wavefronts of a SIMD one multiplies meanwhile.  ms of the largest listed pass: loads spread over the
        // groups of the step before 19.5, at its start 17.6, behind its barrier 16.3, with the reads in one block each 15.5;
        // stages of 32 K, up to four steps ahead, gained nothing (18.0 against 17.6), four wavefronts of 128 x 128 lose (20.4).
        if (steps > 0) {
            pa.init((const bf16_t*)a.A, a.lda, m0, a.M, kb, tid);
            pb.init((const bf16_t*)a.B, a.ldb, n0, a.N, kb, tid);
            load_step(0, 0);
            if (steps > 1) {
                next_step(1, 1);
                x_wait<NP>();
            } else {
                x_wait<0>();
            }
            x_barrier();
            read(S0{}, 0);
        }
        for (int kc = 0; kc < steps; ++kc) {
            const int cur = kc & 1, nxt = cur ^ 1;
            multiply(0);
            read(S1{}, cur);
            multiply(1);
            read(S2{}, cur);
            multiply(0);
            read(S3{}, cur);
            x_wait<0>();
            x_barrier();
            multiply(1);
            if (kc + 2 < steps) next_step(cur, kc + 2);
            __builtin_amdgcn_sched_barrier(0);
            if (kc + 1 < steps) read(S0{}, nxt);
        }

        // ---- epilogue: rows mrow(i), columns nw + ncol(j, q) .. + 3
        const int wrow = wm * (BM / WM) + lo;
        auto mrow = [&](int i) { return m0 + wrow + i * 32; };
        int label[MI];
        float lse[MI], up[MI];
        if constexpr (MODE != XE_OUT) {
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const long m = mrow(i) < a.M ? mrow(i) : a.M - 1;
                label[i] = a.e.labels[m];
                if constexpr (MODE == XE_GRAD) {
                    lse[i] = a.e.lse[m];
                    up[i] = a.e.dloss[m];
                }
            }
            if (tid < BN) s_bias[tid] = a.e.bias && n0 + tid < a.N ? a.e.bias[a.e.col0 + n0 + tid] : 0.f;
            __syncthreads();
        }
        const long nw = n0 + wn * (BN / WN);
        const int cols = (int)(a.N - nw < BN / WN ? a.N - nw : BN / WN);     // of the wavefront's, those that there are
        // where row i's label is among them, else below zero
        auto label_col = [&](int i) {
            const long ln = (long)label[i] - a.e.col0 - nw;
            return mrow(i) < a.M && is_class(label[i], a.e.classes) && ln >= 0 && ln < cols ? (int)ln : -1;
        };
        auto ncol = [&](int j, int q) { return j * 32 + 8 * q + 4 * hi; };
        if constexpr (MODE != XE_OUT) {
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float4 b = *(const float4*)(s_bias + wn * (BN / WN) + ncol(j, q));
#pragma unroll
                    for (int i = 0; i < MI; ++i) {
                        acc[i][j][4 * q] += b.x;
                        acc[i][j][4 * q + 1] += b.y;
                        acc[i][j][4 * q + 2] += b.z;
                        acc[i][j][4 * q + 3] += b.w;
                    }
                }
            if (n0 + BN > a.N) {                                // the last column tile: nothing behind the last class
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (ncol(j, r / 4) + r % 4 >= cols)
#pragma unroll
                            for (int i = 0; i < MI; ++i) acc[i][j][r] = -__builtin_inff();
            }
        }
        if constexpr (MODE == XE_STATS) {
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                __builtin_amdgcn_sched_barrier(0);               // one row at a time, within the registers
                const long m = mrow(i);
                const int ln = label_col(i);
                if (__any(ln >= 0)) {
#pragma unroll
                    for (int j = 0; j < NJ; ++j)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (ln == ncol(j, r / 4) + r % 4) a.e.picked[m] = acc[i][j][r];
                }
                float mx = -__builtin_inff();
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, acc[i][j][r]);
                mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                const float from = mx == -__builtin_inff() ? 0.f : mx;       // (a row of minus infinities sums to zero)
                float s = 0.f;
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s += __builtin_amdgcn_exp2f((acc[i][j][r] - from) * L2E);
                s += __shfl_xor(s, 32, 64);
                if (hi == 0) s_part[wn * BM + wrow + i * 32] = make_float2(mx, s);
            }
            x_wait_lds();
            x_barrier();
            if (tid < BM && m0 + tid < a.M) {
                float2 p = s_part[tid];
#pragma unroll
                for (int w = 1; w < WN; ++w) join_softmax(p.x, p.y, s_part[w * BM + tid].x, s_part[w * BM + tid].y);
                a.e.part[nt * a.M + m0 + tid] = p;
            }
        } else if constexpr (MODE == XE_GRAD) {
            bf16_t* G = (bf16_t*)a.e.G + mt * a.e.ldg + nw * X_GTILE + wrow * XBK;      // the wavefront's block, this lane's row
            static_assert(BM == X_GTILE && BN / WN == XBK, "a wavefront's columns are those of a block of G");
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                __builtin_amdgcn_sched_barrier(0);               // one row at a time, within the registers
                const bool use = mrow(i) < a.M && is_class(label[i], a.e.classes);
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r)                             // (zero behind the last class: s is minus infinity there)
                        acc[i][j][r] = use ? up[i] * __builtin_amdgcn_exp2f((acc[i][j][r] - lse[i]) * L2E) : 0.f;
                const int ln = label_col(i);
                if (__any(ln >= 0)) {
#pragma unroll
                    for (int j = 0; j < NJ; ++j)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (ln == ncol(j, r / 4) + r % 4) acc[i][j][r] -= up[i];
                }
            }
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int q = 0; q < 4; q += 2) {
                        uint32_t w0 = pack_bf16x2(acc[i][j][4 * q], acc[i][j][4 * q + 1]), w1 = pack_bf16x2(acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
                        uint32_t w2 = pack_bf16x2(acc[i][j][4 * q + 4], acc[i][j][4 * q + 5]), w3 = pack_bf16x2(acc[i][j][4 * q + 6], acc[i][j][4 * q + 7]);
                        swap_halves(w0, w2);
                        swap_halves(w1, w3);
                        *(any_u32x4*)(G + i * 32 * XBK + j * 32 + 8 * (q + hi)) = any_u32x4{w0, w1, w2, w3};
                    }
            if constexpr (DB) {
                // sums over the wavefront's rows, then over the wavefronts
                float* s_sum = (float*)s_part;
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float t = sum32((acc[0][j][r] + acc[1][j][r]) + (acc[2][j][r] + acc[3][j][r]));
                        if (lo == 31) s_sum[wm * BN + wn * (BN / WN) + ncol(j, r / 4) + r % 4] = t;
                    }
                x_wait_lds();
                x_barrier();
                if (tid < BN && n0 + tid < a.N) a.e.dbias_part[mt * a.e.lddb + n0 + tid] = s_sum[tid] + s_sum[BN + tid];
            }
        } else {
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const long m = mrow(i);
                if (m >= a.M) continue;
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const long n = nw + ncol(j, q);       // (N is a multiple of 8)
                        if (n >= a.N) continue;
                        float4 v = make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
                        if (a.e.acc) {
                            const float4 o = *(const float4*)(a.e.acc + m * a.N + n);
                            v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
                        }
                        if (a.e.out_f32) *(float4*)(a.e.out_f32 + (z * a.M + m) * a.N + n) = v;
                        else *(uint2*)((bf16_t*)a.e.out + m * a.N + n) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
                    }
            }
        }
}

// bit r of word r / 64: row r has a label
__global__ void __launch_bounds__(256) xent_mask_kernel(const int32_t* __restrict__ labels, long rows, long classes, uint64_t* __restrict__ mask) {
    for (long r = (long)blockIdx.x * 256 + threadIdx.x; r < (rows + 63) / 64 * 64; r += (long)gridDim.x * 256) {
        const uint64_t b = __ballot(r < rows && is_class(labels[r], classes));
        if ((threadIdx.x & 63) == 0) mask[r / 64] = b;
    }
}

// lse and loss of a row from its tiles: one wavefront per row
__global__ void __launch_bounds__(256) xent_finish_kernel(const float2* __restrict__ part, const float* __restrict__ picked,
                                                          const int32_t* __restrict__ labels, float* __restrict__ loss, float* __restrict__ lse,
                                                          long M, long ntiles, long classes) {
    const int lane = threadIdx.x & 63;
    for (long m = (long)blockIdx.x * 4 + (threadIdx.x >> 6); m < M; m += (long)gridDim.x * 4) {
        float mx = -__builtin_inff(), s = 0.f;
        for (long t = lane; t < ntiles; t += 64) {
            const float2 p = part[t * M + m];
            join_softmax(mx, s, p.x, p.y);
        }
        for (int o = 32; o > 0; o >>= 1) {
            const float m2 = __shfl_xor(mx, o, 64), s2 = __shfl_xor(s, o, 64);
            join_softmax(mx, s, m2, s2);
        }
        if (lane == 0) {
            const float l = mx + logf(s);
            lse[m] = l;
            loss[m] = is_class(labels[m], classes) ? l - picked[m] : 0.f;
        }
    }
}

// out[c] = sum of the rows of part [rows][ld]
__global__ void __launch_bounds__(256) xent_colsum_kernel(const float* __restrict__ part, long rows, long ld, long n, float* __restrict__ out) {
    const long c = (long)blockIdx.x * 256 + threadIdx.x;
    if (c >= n) return;
    float s = 0.f;
    for (long r = 0; r < rows; ++r) s += part[r * ld + c];
    out[c] = s;
}

// out = sum of the splits' results, rounded once
template <typename T>
__global__ void __launch_bounds__(256) xent_join_kernel(const float* __restrict__ part, int splits, long n, T* __restrict__ out) {
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long)gridDim.x * 256) {
        float s = 0.f;
        for (int z = 0; z < splits; ++z) s += part[z * n + i];
        out[i] = Elem<T>::st(s);
    }
}

// ---- host --------------------------------------------------------------------------------
struct XentPlan {
    long piece, pieces;           // classes of a piece of G, number of pieces
    long ldg, lddb;               // elements from row (main: row tile) to row of G, of the partial sums of db
    long ntiles;                  // column tiles of the forward pass
    long mtiles;                  // row tiles of G
    int zdx, zdw;                 // splits of K of the two products
    size_t fwd_bytes, bwd_bytes;
    size_t o_part, o_picked, o_G, o_acc, o_dw, o_dbias, o_mask;
    bool main;                    // on the main tiles
};

static constexpr size_t XENT_G_BYTES = (size_t)512 << 20;   // of a piece of G, at most (a piece has 1024 classes at least)

static int splits_of(long tiles, long K, long fill) {
    long z = tiles < fill ? fill / tiles : 1;
    const long most = K / 512 > 1 ? K / 512 : 1;
    if (z > most) z = most;
    return (int)(z > 64 ? 64 : z);
}

static XentPlan xent_plan(const tsm_xent_desc* d) {
    XentPlan p{};
    const long R = d->rows, D = d->features, V = d->classes, es = (long)dtype_size(d->dtype);
    p.main = d->dtype == TSM_BF16 && D % 8 == 0 && D <= (1 << 21);
    const long bm = p.main ? X_BM : 64, bn = p.main ? X_BN : 64, fill = p.main ? 256 : 512;
    p.ntiles = (V + bn - 1) / bn;
    p.mtiles = (R + bm - 1) / bm;
    Arena f(nullptr, 0);
    p.o_part = f.used; f.take((size_t)p.ntiles * R * 8);
    p.o_picked = f.used; f.take((size_t)R * 4);
    p.fwd_bytes = f.used;
    long piece = (long)(XENT_G_BYTES / es) / R / 1024 * 1024;
    if (piece < 1024) piece = 1024;
    if (piece > V) piece = V;
    p.piece = piece;
    p.pieces = (V + piece - 1) / piece;
    p.lddb = (piece + 7) / 8 * 8;
    p.ldg = p.main ? (piece + X_GTILE - 1) / X_GTILE * X_GTILE * X_GTILE : p.lddb;
    const long dt = (D + bn - 1) / bn;
    p.zdx = p.pieces > 1 ? 1 : splits_of(p.mtiles * dt, V, fill);
    p.zdw = splits_of((piece + bm - 1) / bm * dt, R, fill);
    Arena b(nullptr, 0);
    p.o_G = b.used; b.take((size_t)(p.main ? p.mtiles : R) * p.ldg * es);
    p.o_acc = b.used; b.take(p.pieces > 1 || p.zdx > 1 ? (size_t)p.zdx * R * D * 4 : 0);
    p.o_dw = b.used; b.take(p.zdw > 1 ? (size_t)p.zdw * piece * D * 4 : 0);
    p.o_dbias = b.used; b.take((size_t)p.mtiles * p.lddb * 4);
    p.o_mask = b.used; b.take((size_t)(R + 63) / 64 * 8);
    p.bwd_bytes = b.used;
    return p;
}

static int xent_check(const tsm_xent_desc* d, const char* who) {
    if (!d) return fail(TSM_ERR_NULLPTR, "%s: null descriptor", who);
    if (d->dtype != TSM_F32 && d->dtype != TSM_BF16) return fail(TSM_ERR_DTYPE, "%s: unknown dtype %d", who, d->dtype);
    if (d->rows <= 0 || d->features <= 0 || d->classes <= 0) return fail(TSM_ERR_SHAPE, "%s: non-positive dimension", who);
    if ((double)d->rows * d->features > 1e14 || (double)d->classes * d->features > 1e14) return fail(TSM_ERR_SHAPE, "%s: tensor too large", who);
    return TSM_OK;
}

static size_t xent_ws(const XentPlan& p) { return p.fwd_bytes > p.bwd_bytes ? p.fwd_bytes : p.bwd_bytes; }

template <typename T, int MODE, bool AK, bool BK, bool DB = false>
static int xent_product(const XentArgs& a, const XentPlan& p, int splits, const uint64_t* kmask, const char* what, hipStream_t s) {
    XentArgs b = a;
    if constexpr (sizeof(T) == 2) {
        if (p.main) {
            const long jobs = ((a.N + X_BN - 1) / X_BN) * ((a.M + X_BM - 1) / X_BM) * splits;
            auto kernel = xent_tile_kernel<MODE, MODE != XE_OUT ? X_ROWS : AK ? X_GROWS : X_GCOLS, BK ? X_ROWS : X_COLS, DB>;
            static bool configured = false;
            if (!configured) {
                if (hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) != hipSuccess)
                    return fail(TSM_ERR_LAUNCH, "%s: cannot raise dynamic LDS limit", what);
                configured = true;
            }
            b.ksplit = ((a.K + splits - 1) / splits + 63) / 64 * 64;
            for (long j = 0; j < jobs; j += X_BLOCKS)
                kernel<<<dim3((unsigned)(jobs - j < X_BLOCKS ? jobs - j : X_BLOCKS)), dim3(X_NT), X_SMEM, s>>>(b, kmask, j);
            return check_launch(what);
        }
    }
    const long nt = (a.N + 63) / 64, mt = (a.M + 63) / 64;
    b.ksplit = ((a.K + splits - 1) / splits + 63) / 64 * 64;
    xent_plain_kernel<T, MODE, AK, BK><<<dim3((unsigned)(nt * mt < 65536 ? nt * mt : 65536), 1, (unsigned)splits), dim3(256), 0, s>>>(b);
    return check_launch(what);
}

template <typename T>
static int xent_join(const float* part, int splits, long n, void* out, const char* what, hipStream_t s) {
    const long blocks = (n + 255) / 256;
    xent_join_kernel<T><<<dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, s>>>(part, splits, n, (T*)out);
    return check_launch(what);
}

template <typename T>
static int xent_fwd(const tsm_xent_desc* d, const XentPlan& p, const void* x, const void* w, const float* bias, const int32_t* labels, float* loss,
                    float* lse, char* ws, hipStream_t s) {
    XentArgs a{};
    a.A = x; a.B = w;
    a.lda = a.ldb = a.K = d->features;
    a.M = d->rows; a.N = d->classes;
    a.e.part = (float2*)(ws + p.o_part);
    a.e.picked = (float*)(ws + p.o_picked);
    a.e.bias = bias; a.e.labels = labels; a.e.classes = d->classes;
    TSM_TRY((xent_product<T, XE_STATS, true, true>(a, p, 1, nullptr, "xent_stats", s)));
    const long blocks = (a.M + 3) / 4;
    xent_finish_kernel<<<dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, s>>>(a.e.part, a.e.picked, labels, loss, lse, a.M, p.ntiles, d->classes);
    return check_launch("xent_finish");
}

template <typename T>
static int xent_bwd(const tsm_xent_desc* d, const XentPlan& p, const void* x, const void* w, const float* bias, const int32_t* labels,
                    const float* lse, const float* dloss, void* dx, void* dw, float* dbias, char* ws, hipStream_t s) {
    const long R = d->rows, D = d->features, V = d->classes;
    void* G = ws + p.o_G;
    float *acc = (float*)(ws + p.o_acc), *dwp = (float*)(ws + p.o_dw), *dbp = (float*)(ws + p.o_dbias);
    uint64_t* mask = nullptr;
    if (dw && p.main) {
        mask = (uint64_t*)(ws + p.o_mask);
        const long blocks = (R + 255) / 256;
        xent_mask_kernel<<<dim3((unsigned)(blocks < 1024 ? blocks : 1024)), dim3(256), 0, s>>>(labels, R, V, mask);
        TSM_TRY(check_launch("xent_mask"));
    }
    for (long c = 0; c < p.pieces; ++c) {
        const long v0 = c * p.piece, n = V - v0 < p.piece ? V - v0 : p.piece;
        const T* wc = (const T*)w + v0 * D;
        XentArgs a{};
        a.A = x; a.B = wc;
        a.lda = a.ldb = a.K = D;
        a.M = R; a.N = n;
        a.e.bias = bias; a.e.labels = labels; a.e.classes = V; a.e.col0 = v0;
        a.e.lse = lse; a.e.dloss = dloss; a.e.G = G; a.e.ldg = p.ldg; a.e.dbias_part = dbias ? dbp : nullptr;
        a.e.lddb = p.lddb;
        if (dbias) TSM_TRY((xent_product<T, XE_GRAD, true, true, true>(a, p, 1, nullptr, "xent_grad", s)));
        else TSM_TRY((xent_product<T, XE_GRAD, true, true>(a, p, 1, nullptr, "xent_grad", s)));
        if (dbias) {
            xent_colsum_kernel<<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s>>>(dbp, p.mtiles, p.lddb, n, dbias + v0);
            TSM_TRY(check_launch("xent_dbias"));
        }
        if (dx) {
            XentArgs b{};
            b.A = G; b.lda = p.ldg; b.B = wc; b.ldb = D;
            b.M = R; b.N = D; b.K = n;
            b.e.acc = c > 0 ? acc : nullptr;
            if (p.zdx > 1 || c + 1 < p.pieces) b.e.out_f32 = acc;
            else b.e.out = dx;
            TSM_TRY((xent_product<T, XE_OUT, true, false>(b, p, p.zdx, nullptr, "xent_dx", s)));
            if (p.zdx > 1) TSM_TRY(xent_join<T>(acc, p.zdx, R * D, dx, "xent_dx_join", s));
        }
        if (dw) {
            XentArgs b{};
            b.A = G; b.lda = p.ldg; b.B = x; b.ldb = D;
            b.M = n; b.N = D; b.K = R;
            b.klabels = labels; b.e.classes = V;
            T* out = (T*)dw + v0 * D;
            if (p.zdw > 1) b.e.out_f32 = dwp;
            else b.e.out = out;
            TSM_TRY((xent_product<T, XE_OUT, false, false>(b, p, p.zdw, mask, "xent_dw", s)));
            if (p.zdw > 1) TSM_TRY(xent_join<T>(dwp, p.zdw, n * D, out, "xent_dw_join", s));
        }
    }
    return TSM_OK;
}

}  // namespace tsm

using namespace tsm;

extern "C" {

size_t tsm_xent_workspace_bytes(const tsm_xent_desc* d) {
    return xent_check(d, "tsm_xent_workspace_bytes") == TSM_OK ? xent_ws(xent_plan(d)) : 0;
}

int tsm_xent_fwd(const tsm_xent_desc* d, const void* x, const void* w, const float* bias, const int32_t* labels, float* loss, float* lse, void* ws,
                 size_t ws_bytes, void* stream) {
    const char* who = "tsm_xent_fwd";
    TSM_TRY(xent_check(d, who));
    if (!x || !w || !labels || !loss || !lse) return fail(TSM_ERR_NULLPTR, "%s: null pointer", who);
    const XentPlan p = xent_plan(d);
    const size_t need = xent_ws(p);
    if (ws_bytes < need) return fail(TSM_ERR_WORKSPACE, "%s: workspace %zu bytes, need %zu", who, ws_bytes, need);
    if (!ws) return fail(TSM_ERR_NULLPTR, "%s: null workspace", who);
    const size_t es = dtype_size(d->dtype), rb = (size_t)d->rows * 4;
    const Span in[] = {{x, (size_t)d->rows * d->features * es, "x"}, {w, (size_t)d->classes * d->features * es, "w"},
                       {bias, (size_t)d->classes * 4, "bias"}, {labels, rb, "labels"}};
    const Span out[] = {{loss, rb, "loss"}, {lse, rb, "lse"}, {ws, need, "the workspace"}};
    TSM_TRY(check_spans(who, in, 4, out, 3));
    const hipStream_t s = (hipStream_t)stream;
    return d->dtype == TSM_BF16 ? xent_fwd<bf16_t>(d, p, x, w, bias, labels, loss, lse, (char*)ws, s)
                                : xent_fwd<float>(d, p, x, w, bias, labels, loss, lse, (char*)ws, s);
}

int tsm_xent_bwd(const tsm_xent_desc* d, const void* x, const void* w, const float* bias, const int32_t* labels, const float* lse,
                 const float* dloss, void* dx, void* dw, float* dbias, void* ws, size_t ws_bytes, void* stream) {
    const char* who = "tsm_xent_bwd";
    TSM_TRY(xent_check(d, who));
    if (!x || !w || !labels || !lse || !dloss) return fail(TSM_ERR_NULLPTR, "%s: null pointer", who);
    if (!dx && !dw && !dbias) return fail(TSM_ERR_NULLPTR, "%s: no gradient asked for", who);
    const XentPlan p = xent_plan(d);
    const size_t need = xent_ws(p);
    if (ws_bytes < need) return fail(TSM_ERR_WORKSPACE, "%s: workspace %zu bytes, need %zu", who, ws_bytes, need);
    if (!ws) return fail(TSM_ERR_NULLPTR, "%s: null workspace", who);
    const size_t es = dtype_size(d->dtype), rb = (size_t)d->rows * 4;
    const size_t xb = (size_t)d->rows * d->features * es, wb = (size_t)d->classes * d->features * es, bb = (size_t)d->classes * 4;
    const Span in[] = {{x, xb, "x"}, {w, wb, "w"}, {bias, bb, "bias"}, {labels, rb, "labels"}, {lse, rb, "lse"}, {dloss, rb, "dloss"}};
    const Span out[] = {{dx, xb, "dx"}, {dw, wb, "dw"}, {dbias, bb, "dbias"}, {ws, need, "the workspace"}};
    TSM_TRY(check_spans(who, in, 6, out, 4));
    const hipStream_t s = (hipStream_t)stream;
    return d->dtype == TSM_BF16 ? xent_bwd<bf16_t>(d, p, x, w, bias, labels, lse, dloss, dx, dw, dbias, (char*)ws, s)
                                : xent_bwd<float>(d, p, x, w, bias, labels, lse, dloss, dx, dw, dbias, (char*)ws, s);
}

}  // extern "C"
