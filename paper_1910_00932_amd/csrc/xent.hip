// Linear classifier with softmax cross entropy whose logits are never stored, and its gradients.
//
//   s = x w^T + b;  lse_r = log sum_v exp s_rv;  loss_r = lse_r - s_r,label  (0 for rows whose label is no class)
//   G_rv = dloss_r (exp(s_rv - lse_r) - [v == label_r]);  dx = G w;  dw = G^T x;  db_v = sum_r G_rv
//
// Forward: tiles of s stay in registers; each leaves the maximum and the sum of exponentials of its columns per row (a softmax
// joined over the tiles) and the label's logit.  Backward: s is formed again in pieces of the classes, a piece of G lives in the
// workspace for the two products that read it.  Four products of rows x features x classes in all, on the bf16 matrix cores.
//
// bf16: G, but for a factor (XScale), is rounded once, to the type of the matrix cores' operands, or of few rows or classes cut into two parts
// (X_GTWO); lse, the losses, db (from G before that) and all sums are fp32.  fp32: x, w and G are cut into three bf16 parts each, exactly (8 + 8 + 8 bits), and a product is the sum of the
// six largest part products (the method of Henry, Tang and Heinecke, "Leveraging the bfloat16 artificial intelligence datatype for
// higher-precision computations", 2019; what is left out is at most 2^-24 of it), the small ones first.
#include <algorithm>
#include <type_traits>
#include "internal.h"
#include "args.h"
#include "vec_any.h"
#include "long_sum.h"

namespace tsm {

typedef float x_f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 x_bf16x8 __attribute__((ext_vector_type(8)));

struct XentEpi {
    // STATS
    float2* part;            // [column tiles][M]: maximum and sum of exp(s - maximum) of a tile's columns
    float* picked;           // [M]: the label's logit
    // STATS and GRAD: columns are classes col0 + n of `classes`
    const float* bias;
    const int32_t* labels;
    long col0, classes;
    // GRAD
    const float *lse, *dloss;     // (dloss for OUT too, with labels and classes)
    const float* scale;      // GRAD and OUT, bf16: XScale's factor, where a wavefront does not look for it itself
    long rows;               // OUT: of the whole pass
    bf16_t* G;               // in blocks (X_GROWS): ldg elements per 256 rows, gplane from one part to the next
    long ldg, gplane;
    float* dbias_part;       // [row tiles][lddb]
    long lddb;
    uint64_t* mask;          // bit r % 64 of word r / 64: row r has a label; nullable
    // OUT: [M][N]
    const float* acc;        // fp32 [splits][M][N], added to the result, nullable
    float* out_f32;          // [splits][M][N], or
    bf16_t* out;
};

struct XentArgs {
    const bf16_t *A, *B;
    long lda, ldb, aplane, bplane;     // elements from row to row (G: per 256 rows), from part to part
    long M, N, K, ksplit;              // ksplit: K of one split, a multiple of 64
    const uint64_t* kmask;             // OUT over the rows of G: rows of B that count as zero
    long job0;
    XentEpi e;
};

enum { X_TINY = 0, X_SMALL = 1, X_MID = 2, X_BIG = 3 };      // tiles of 32 (of s only), 64, 128, 256
enum { XE_STATS = 0, XE_GRAD = 1, XE_OUT = 2 };

__device__ __forceinline__ bool is_class(int label, long classes) { return label >= 0 && label < classes; }

// joins (m, s) with (m2, s2)
__device__ __forceinline__ void join_softmax(float& m, float& s, float m2, float s2) {
    const float t = fmaxf(m, m2);
    s = (m == t ? s : s * __expf(m - t)) + (m2 == t ? s2 : s2 * __expf(m2 - t));
    m = t;
}

// The factor in [1, 2) that bf16 G of one part leaves out of dloss, and what reads G puts back: the mantissa of the first ordinary dloss among the
// rows with a label, the same in every tile.  A mean's dloss is one number for all rows, and the entry of a row's label, by far
// its largest, is almost that number: rounded with it, all of them would be off alike, by up to 2^-9 of the whole gradient.
// Of up to 512 rows every wavefront looks for itself, 64 at a time, most often once; of more, a launch of one block does (4.7 us at 1777 rows,
// 5.3 at 8192; a pass of 128 x 2048 x 1000, 29 us, would be 3 to 4 longer with it), which passes over any number of rows.
__device__ __forceinline__ bool ordinary(float v) {
    const uint32_t exponent = (__float_as_uint(v) >> 23) & 0xff;
    return exponent != 0 && exponent != 0xff;
}
__device__ __forceinline__ float mantissa(float v) { return __uint_as_float((__float_as_uint(v) & 0x7fffffu) | 0x3f800000u); }
static constexpr int X_SCALE_ROWS = 512, X_SCALE_TURN = 4;      // rows that a wavefront looks through; rows per thread and turn of the launch
struct XScale {
    float up;
    bool ok, found;
    __device__ __forceinline__ void rows(const XentEpi& e, long from, long M) {
        const long r = from + (threadIdx.x & 63), at = r < M ? r : M - 1;       // (the last one again)
        up = e.dloss[at];
        ok = is_class(e.labels[at], e.classes);
    }
    __device__ __forceinline__ void load(const XentEpi& e, long M) {            // ahead of get()
        found = e.scale != nullptr;
        if (found) up = *(const __attribute__((address_space(4))) float*)e.scale;
        else rows(e, 0, M);
    }
    __device__ __forceinline__ float get(const XentEpi& e, long M) {
        if (found) return up;
        uint64_t count = __ballot(ok && ordinary(up));
        for (long from = 64; count == 0 && from < M; from += 64) {
            rows(e, from, M);
            count = __ballot(ok && ordinary(up));
        }
        const float first = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(up), count ? __builtin_ctzll(count) : 0));
        return count ? mantissa(first) : 1.f;
    }
};
__global__ void __launch_bounds__(1024) xent_scale_kernel(const float* __restrict__ dloss, const int32_t* __restrict__ labels, int rows, long classes,
                                                          float* __restrict__ scale) {
    __shared__ int s_first;
    if (threadIdx.x == 0) s_first = rows;
    __syncthreads();
    for (long base = 0; base < rows; base += 1024 * X_SCALE_TURN) {
        bool use[X_SCALE_TURN];
#pragma unroll
        for (int i = 0; i < X_SCALE_TURN; ++i) {
            const long r = base + i * 1024 + threadIdx.x, at = r < rows ? r : rows - 1;
            use[i] = is_class(labels[at], classes) && ordinary(dloss[at]) && r < rows;
        }
#pragma unroll
        for (int i = 0; i < X_SCALE_TURN; ++i) {
            const uint64_t count = __ballot(use[i]);
            if (count) {                                        // the wavefront's first; one LDS access for all of it
                if ((threadIdx.x & 63) == 0) atomicMin(&s_first, (int)(base + i * 1024 + threadIdx.x + __builtin_ctzll(count)));
                break;
            }
        }
        __syncthreads();
        if (s_first < rows) break;                              // (the same for all: the next turn writes behind another barrier)
        __syncthreads();
    }
    if (threadIdx.x == 0) *scale = s_first < rows ? mantissa(dloss[s_first]) : 1.f;
}

// ---- tiles: BM x BN results of wavefronts that share the operands through LDS ---------------------------------------------
// Operands come 64 steps of K at a time (32 for those in three parts), straight from memory into an LDS stage while another is
// multiplied.  An operand with consecutive K lies there as rows of 128 bytes whose eight 16-byte pieces are permuted by the row,
// so that the 32 rows of a fragment read spread over all banks; one whose rows are K lies there as it does in memory, its
// 32-byte granules permuted by K, and fragments are read through the transposing LDS read, four K of 16 columns at a time.
static constexpr int X_GTILE = 256, X_GCOLUMNS = 64;        // rows and columns of a block of G
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

// How an operand lies in memory.  The blocks of G: [256 rows][64 columns], 32 KB each, those of 256 rows after one another, so that a
// step of either product reads stretches of 8 KB, where rows of G as such would lie 64 KB apart.
enum { X_ROWS = 0, X_COLS = 1, X_GROWS = 2, X_GCOLS = 3 };     // [rows][K], [K][rows], G with its columns as K, with its rows as K

// One operand of a tile: ROWS rows of the result's side, BK steps of K at a time, loaded by NT threads.
template <int ROWS, int KIND, int NT, int BK>
struct XOperand {
    static constexpr bool KC = KIND == X_ROWS || KIND == X_GROWS;     // K consecutive in LDS
    static constexpr int BYTES = ROWS * BK * 2;
    static constexpr int PIECES = BYTES / (NT * 16);          // per thread and step
    static constexpr int KV = BK / 8;                         // KC: 16-byte pieces of a row
    static constexpr int RPP = KC ? NT / KV : NT / (ROWS / 8);// rows of the LDS image per pass
    static constexpr int PITCH = KC ? BK * 2 : ROWS * 2;      // its bytes
    uint32_t off[PIECES];         // byte offset in the step's window of this thread's pieces
    int kfirst;                   // KC: K of the first piece, else K of the thread's row in a pass
    const char *base, *base0;     // of the step's window, of the first one of the first part
    long step;                    // bytes from one step to the next
    int part, part0;              // G: steps into a block (X_GROWS), into 256 rows (X_GCOLS)
    static constexpr int PARTS = KIND == X_GROWS ? X_GCOLUMNS / BK : X_GTILE / BK;

    // XOR of the piece number in a row of consecutive K: the rows of a fragment read spread over all banks
    __device__ __forceinline__ static int kswz(int r) { return (r / (16 / KV)) & (KV - 1); }
    // XOR of the granule number: four consecutive K and the two granules of a fragment fall on different banks
    __device__ __forceinline__ static int swz(int k) {
        return ROWS == 64 ? ((k >> 1) & 1) << 1 : ((((k & 3) << 1) | (((k >> 3) & 1) << 3))) & (ROWS / 16 - 1);
    }

    // row0: first row of the tile, rows: of the matrix; k0: first K, a multiple of 64.
    __device__ __forceinline__ void init(const bf16_t* p, long ld, long row0, long rows, long k0, int tid) {
        part0 = 0;
        if constexpr (KC) {
            const int r = tid / KV;
            const int kv = (tid % KV) ^ kswz(r);
            kfirst = kv * 8;
            const long pitch = KIND == X_GROWS ? X_GCOLUMNS : ld;
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
                off[i] = row0 + i * RPP + r < rows ? (uint32_t)((i * RPP + r) * pitch * 2 + (kv ^ kswz(i * RPP)) * 16) : X_OOB;
            base0 = (const char*)(KIND == X_GROWS ? p + row0 / X_GTILE * ld + row0 % X_GTILE * X_GCOLUMNS + k0 * X_GTILE : p + row0 * ld + k0);
            step = KIND == X_GROWS ? (X_GTILE * X_GCOLUMNS - (X_GCOLUMNS - BK)) * 2 : BK * 2;      // (into the next block)
        } else {
            const int k = tid / (ROWS / 8), slot = tid % (ROWS / 8);
            kfirst = k;
            const int col = (((slot >> 1) ^ swz(k)) << 4) + (slot & 1) * 8;
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const long at = KIND == X_GCOLS ? col / X_GCOLUMNS * (X_GTILE * X_GCOLUMNS) + (i * RPP + k) * X_GCOLUMNS + col % X_GCOLUMNS : (i * RPP + k) * ld + col;
                off[i] = row0 + col < rows ? (uint32_t)(at * 2) : X_OOB;
            }
            if constexpr (KIND == X_GCOLS) {
                part0 = (int)(k0 % X_GTILE / BK);
                base0 = (const char*)(p + k0 / X_GTILE * ld + row0 * X_GTILE + k0 % X_GTILE * X_GCOLUMNS);
                step = (ld - (X_GTILE - BK) * X_GCOLUMNS) * 2;         // into the next 256 rows
            } else {
                base0 = (const char*)(p + k0 * ld + row0);
                step = BK * 2 * ld;
            }
        }
        // (the same in all lanes, which the compiler has to know for a load's descriptor)
        base0 = (const char*)uniform((uint64_t)base0);
        step = (long)uniform((uint64_t)step);
        part0 = __builtin_amdgcn_readfirstlane(part0);
        restart(0);
    }
    __device__ __forceinline__ static uint64_t uniform(uint64_t v) {
        return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)v);
    }
    __device__ __forceinline__ void restart(long elements) {   // the first step again, of another part
        base = base0 + elements * 2;
        part = part0;
    }
    __device__ __forceinline__ void advance() {
        if constexpr ((KIND == X_GROWS && PARTS > 1) || KIND == X_GCOLS) {
            const bool last = part == PARTS - 1;
            base += last ? step : (long)(KIND == X_GROWS ? BK : BK * X_GCOLUMNS) * 2;
            part = last ? 0 : part + 1;
        } else {
            base += step;
        }
    }
    // Piece i of the step at the window, `more` bytes behind it: left = K from its start to the end; mask: bit k clear for rows k that
    // count as zero.
    __device__ __forceinline__ void load(unsigned char* stage, int i, int left, uint64_t mask, int wave_u, long more = 0) const {
        const int k = KC ? kfirst ^ kswz(i * RPP) * 8 : i * RPP + kfirst;
        const bool in = k < left && (KC || (mask >> k) & 1);
        x_load_lds16(x_rsrc(base + more), stage + i * (NT * 16) + wave_u * 1024, in ? off[i] : X_OOB, 0);
    }
    // Whole fp32: the q-th of a lane's four reads of four values, two of either slice of 16 values.
    __device__ __forceinline__ static uint32_t whole_at(int row0, int q, int lane) {
        const int r = lane & 31, hi = lane >> 5;
        return (row0 + r) * PITCH + (((q / 2 * 4 + hi * 2 + q % 2) ^ kswz(r)) * 16);
    }
    // Where a lane reads the fragment of the 32 rows from row0 (a multiple of 32), K consecutive: of slice ks, else of slice 0.
    __device__ __forceinline__ static uint32_t frag_at(int row0, int ks, int lane) {
        if constexpr (KC) {
            const int r = lane & 31, hi = lane >> 5;
            return (row0 + r) * PITCH + (((2 * ks + hi) ^ kswz(r)) * 16);
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

// the middle tiles' two and two
__device__ __forceinline__ void read_frags(uint32_t a, uint32_t b, x_bf16x8 (&fa)[2], x_bf16x8 (&fb)[2]) {
    asm volatile("ds_read_b128 %0, %4\n ds_read_b128 %2, %5\n ds_read_b128 %1, %4 offset:4096\n ds_read_b128 %3, %5 offset:4096\n s_waitcnt lgkmcnt(0)"
                 : "=&v"(fa[0]), "=&v"(fa[1]), "=&v"(fb[0]), "=&v"(fb[1]) : "v"(a), "v"(b) : "memory");
}
template <int OFF, int OFF2>
__device__ __forceinline__ void read_frags(uint32_t a, const uint32_t (&b)[2], x_bf16x8 (&fa)[2], x_bf16x8 (&fb)[2]) {
    x_s16x4 l0, l1, u0, u1;
    asm volatile("ds_read_b128 %0, %6\n ds_read_b64_tr_b16 %2, %7 offset:%9\n ds_read_b64_tr_b16 %3, %7 offset:%10\n"
                 "ds_read_b128 %1, %6 offset:4096\n ds_read_b64_tr_b16 %4, %8 offset:%9\n ds_read_b64_tr_b16 %5, %8 offset:%10\n s_waitcnt lgkmcnt(0)"
                 : "=&v"(fa[0]), "=&v"(fa[1]), "=&v"(l0), "=&v"(u0), "=&v"(l1), "=&v"(u1)
                 : "v"(a), "v"(b[0]), "v"(b[1]), "n"(OFF), "n"(OFF2) : "memory");
    fb[0] = x_join(l0, u0);
    fb[1] = x_join(l1, u1);
}
template <int OFF, int OFF2>
__device__ __forceinline__ void read_frags(const uint32_t (&a)[2], const uint32_t (&b)[2], x_bf16x8 (&fa)[2], x_bf16x8 (&fb)[2]) {
    x_s16x4 l[4], u[4];
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%12\n ds_read_b64_tr_b16 %1, %8 offset:%13\n ds_read_b64_tr_b16 %4, %10 offset:%12\n"
                 "ds_read_b64_tr_b16 %5, %10 offset:%13\n ds_read_b64_tr_b16 %2, %9 offset:%12\n ds_read_b64_tr_b16 %3, %9 offset:%13\n"
                 "ds_read_b64_tr_b16 %6, %11 offset:%12\n ds_read_b64_tr_b16 %7, %11 offset:%13\n s_waitcnt lgkmcnt(0)"
                 : "=&v"(l[0]), "=&v"(u[0]), "=&v"(l[1]), "=&v"(u[1]), "=&v"(l[2]), "=&v"(u[2]), "=&v"(l[3]), "=&v"(u[3])
                 : "v"(a[0]), "v"(a[1]), "v"(b[0]), "v"(b[1]), "n"(OFF), "n"(OFF2) : "memory");
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        fa[i] = x_join(l[i], u[i]);
        fb[i] = x_join(l[2 + i], u[2 + i]);
    }
}
// The small tiles' wavefronts have one fragment of each operand per slice: the four slices of a step in one block.
__device__ __forceinline__ void read_step(const uint32_t (&a)[4], const uint32_t (&b)[4], x_bf16x8 (&fa)[4], x_bf16x8 (&fb)[4]) {
    asm volatile("ds_read_b128 %0, %8\n ds_read_b128 %4, %12\n ds_read_b128 %1, %9\n ds_read_b128 %5, %13\n"
                 "ds_read_b128 %2, %10\n ds_read_b128 %6, %14\n ds_read_b128 %3, %11\n ds_read_b128 %7, %15\n s_waitcnt lgkmcnt(0)"
                 : "=&v"(fa[0]), "=&v"(fa[1]), "=&v"(fa[2]), "=&v"(fa[3]), "=&v"(fb[0]), "=&v"(fb[1]), "=&v"(fb[2]), "=&v"(fb[3])
                 : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]) : "memory");
}
// (PITCH of 128 bytes: slices 2048 bytes apart, K 4 to 7 at 512)
__device__ __forceinline__ void read_step(const uint32_t (&a)[4], uint32_t b, x_bf16x8 (&fa)[4], x_bf16x8 (&fb)[4]) {
    x_s16x4 l[4], u[4];
    asm volatile("ds_read_b128 %0, %12\n ds_read_b64_tr_b16 %4, %16\n ds_read_b64_tr_b16 %5, %16 offset:512\n"
                 "ds_read_b128 %1, %13\n ds_read_b64_tr_b16 %6, %16 offset:2048\n ds_read_b64_tr_b16 %7, %16 offset:2560\n"
                 "ds_read_b128 %2, %14\n ds_read_b64_tr_b16 %8, %16 offset:4096\n ds_read_b64_tr_b16 %9, %16 offset:4608\n"
                 "ds_read_b128 %3, %15\n ds_read_b64_tr_b16 %10, %16 offset:6144\n ds_read_b64_tr_b16 %11, %16 offset:6656\n s_waitcnt lgkmcnt(0)"
                 : "=&v"(fa[0]), "=&v"(fa[1]), "=&v"(fa[2]), "=&v"(fa[3]), "=&v"(l[0]), "=&v"(u[0]), "=&v"(l[1]), "=&v"(u[1]), "=&v"(l[2]), "=&v"(u[2]),
                   "=&v"(l[3]), "=&v"(u[3])
                 : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(b) : "memory");
#pragma unroll
    for (int k = 0; k < 4; ++k) fb[k] = x_join(l[k], u[k]);
}
__device__ __forceinline__ void read_step(uint32_t a, uint32_t b, x_bf16x8 (&fa)[4], x_bf16x8 (&fb)[4]) {
    x_s16x4 l[8], u[8];
    asm volatile("ds_read_b64_tr_b16 %0, %16\n ds_read_b64_tr_b16 %1, %16 offset:512\n ds_read_b64_tr_b16 %8, %17\n ds_read_b64_tr_b16 %9, %17 offset:512\n"
                 "ds_read_b64_tr_b16 %2, %16 offset:2048\n ds_read_b64_tr_b16 %3, %16 offset:2560\n ds_read_b64_tr_b16 %10, %17 offset:2048\n"
                 "ds_read_b64_tr_b16 %11, %17 offset:2560\n ds_read_b64_tr_b16 %4, %16 offset:4096\n ds_read_b64_tr_b16 %5, %16 offset:4608\n"
                 "ds_read_b64_tr_b16 %12, %17 offset:4096\n ds_read_b64_tr_b16 %13, %17 offset:4608\n ds_read_b64_tr_b16 %6, %16 offset:6144\n"
                 "ds_read_b64_tr_b16 %7, %16 offset:6656\n ds_read_b64_tr_b16 %14, %17 offset:6144\n ds_read_b64_tr_b16 %15, %17 offset:6656\n s_waitcnt lgkmcnt(0)"
                 : "=&v"(l[0]), "=&v"(u[0]), "=&v"(l[1]), "=&v"(u[1]), "=&v"(l[2]), "=&v"(u[2]), "=&v"(l[3]), "=&v"(u[3]), "=&v"(l[4]), "=&v"(u[4]),
                   "=&v"(l[5]), "=&v"(u[5]), "=&v"(l[6]), "=&v"(u[6]), "=&v"(l[7]), "=&v"(u[7])
                 : "v"(a), "v"(b) : "memory");
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        fa[k] = x_join(l[k], u[k]);
        fb[k] = x_join(l[4 + k], u[4 + k]);
    }
}

// Three parts of a slice, two fragments of A and one of B each: f[part]; parts 8192 bytes apart.  KC: slices at addresses of their own.
__device__ __forceinline__ void read_parts(uint32_t a, uint32_t b, x_bf16x8 (&fa)[3][2], x_bf16x8 (&fb)[3]) {
    asm volatile("ds_read_b128 %0, %9\n ds_read_b128 %6, %10\n ds_read_b128 %1, %9 offset:2048\n ds_read_b128 %2, %9 offset:8192\n"
                 "ds_read_b128 %7, %10 offset:8192\n ds_read_b128 %3, %9 offset:10240\n ds_read_b128 %4, %9 offset:16384\n"
                 "ds_read_b128 %8, %10 offset:16384\n ds_read_b128 %5, %9 offset:18432\n s_waitcnt lgkmcnt(0)"
                 : "=&v"(fa[0][0]), "=&v"(fa[0][1]), "=&v"(fa[1][0]), "=&v"(fa[1][1]), "=&v"(fa[2][0]), "=&v"(fa[2][1]), "=&v"(fb[0]), "=&v"(fb[1]), "=&v"(fb[2])
                 : "v"(a), "v"(b) : "memory");
}
// (the transposing read: rows of 256 bytes, OFF of the slice)
template <int OFF>
__device__ __forceinline__ void read_parts(uint32_t a, uint32_t b, x_bf16x8 (&fa)[3][2], x_bf16x8 (&fb)[3]) {
    x_s16x4 l[3], u[3];
    asm volatile("ds_read_b128 %0, %12\n ds_read_b64_tr_b16 %6, %13 offset:%14\n ds_read_b64_tr_b16 %7, %13 offset:%15\n ds_read_b128 %1, %12 offset:2048\n"
                 "ds_read_b128 %2, %12 offset:8192\n ds_read_b64_tr_b16 %8, %13 offset:%16\n ds_read_b64_tr_b16 %9, %13 offset:%17\n"
                 "ds_read_b128 %3, %12 offset:10240\n ds_read_b128 %4, %12 offset:16384\n ds_read_b64_tr_b16 %10, %13 offset:%18\n"
                 "ds_read_b64_tr_b16 %11, %13 offset:%19\n ds_read_b128 %5, %12 offset:18432\n s_waitcnt lgkmcnt(0)"
                 : "=&v"(fa[0][0]), "=&v"(fa[0][1]), "=&v"(fa[1][0]), "=&v"(fa[1][1]), "=&v"(fa[2][0]), "=&v"(fa[2][1]), "=&v"(l[0]), "=&v"(u[0]),
                   "=&v"(l[1]), "=&v"(u[1]), "=&v"(l[2]), "=&v"(u[2])
                 : "v"(a), "v"(b), "n"(OFF), "n"(OFF + 1024), "n"(OFF + 8192), "n"(OFF + 9216), "n"(OFF + 16384), "n"(OFF + 17408) : "memory");
#pragma unroll
    for (int k = 0; k < 3; ++k) fb[k] = x_join(l[k], u[k]);
}
template <int OFF>
__device__ __forceinline__ void read_parts(const uint32_t (&a)[2], uint32_t b, x_bf16x8 (&fa)[3][2], x_bf16x8 (&fb)[3]) {
    x_s16x4 l[9], u[9];
    asm volatile("ds_read_b64_tr_b16 %0, %18 offset:%21\n ds_read_b64_tr_b16 %1, %18 offset:%22\n ds_read_b64_tr_b16 %12, %20 offset:%21\n"
                 "ds_read_b64_tr_b16 %13, %20 offset:%22\n ds_read_b64_tr_b16 %2, %19 offset:%21\n ds_read_b64_tr_b16 %3, %19 offset:%22\n"
                 "ds_read_b64_tr_b16 %4, %18 offset:%23\n ds_read_b64_tr_b16 %5, %18 offset:%24\n ds_read_b64_tr_b16 %14, %20 offset:%23\n"
                 "ds_read_b64_tr_b16 %15, %20 offset:%24\n ds_read_b64_tr_b16 %6, %19 offset:%23\n ds_read_b64_tr_b16 %7, %19 offset:%24\n"
                 "ds_read_b64_tr_b16 %8, %18 offset:%25\n ds_read_b64_tr_b16 %9, %18 offset:%26\n ds_read_b64_tr_b16 %16, %20 offset:%25\n"
                 "ds_read_b64_tr_b16 %17, %20 offset:%26\n ds_read_b64_tr_b16 %10, %19 offset:%25\n ds_read_b64_tr_b16 %11, %19 offset:%26\n s_waitcnt lgkmcnt(0)"
                 : "=&v"(l[0]), "=&v"(u[0]), "=&v"(l[1]), "=&v"(u[1]), "=&v"(l[2]), "=&v"(u[2]), "=&v"(l[3]), "=&v"(u[3]), "=&v"(l[4]), "=&v"(u[4]),
                   "=&v"(l[5]), "=&v"(u[5]), "=&v"(l[6]), "=&v"(u[6]), "=&v"(l[7]), "=&v"(u[7]), "=&v"(l[8]), "=&v"(u[8])
                 : "v"(a[0]), "v"(a[1]), "v"(b), "n"(OFF), "n"(OFF + 1024), "n"(OFF + 8192), "n"(OFF + 9216), "n"(OFF + 16384), "n"(OFF + 17408) : "memory");
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        fa[k][0] = x_join(l[2 * k], u[2 * k]);
        fa[k][1] = x_join(l[2 * k + 1], u[2 * k + 1]);
        fb[k] = x_join(l[6 + k], u[6 + k]);
    }
}

// fp32 operands that lie in LDS as they are (WHOLE): eight consecutive K of a lane, cut into their three parts in registers.
struct XCut {
    x_bf16x8 part[3];
    __device__ __forceinline__ explicit XCut(const float (&v)[8]) {
        float f[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) f[t] = v[t];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            uint32_t w[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                // (a finite value that would round to infinity is cut off instead)
                constexpr float MOST = 0x1.fep127f;
                w[t] = k == 0 ? pack_bf16x2(__builtin_amdgcn_fmed3f(f[2 * t], -MOST, MOST), __builtin_amdgcn_fmed3f(f[2 * t + 1], -MOST, MOST))
                              : pack_bf16x2(f[2 * t], f[2 * t + 1]);
                if (k < 2) {
                    f[2 * t] -= __uint_as_float(w[t] << 16);
                    f[2 * t + 1] -= __uint_as_float(w[t] & 0xffff0000u);
                }
            }
            part[k] = __builtin_bit_cast(x_bf16x8, any_u32x4{w[0], w[1], w[2], w[3]});
        }
    }
    __device__ __forceinline__ static XCut of(const x_bf16x8& lo, const x_bf16x8& up) {     // (two reads of four values)
        const any_f32x4 l = __builtin_bit_cast(any_f32x4, lo), u = __builtin_bit_cast(any_f32x4, up);
        const float f[8] = {l[0], l[1], l[2], l[3], u[0], u[1], u[2], u[3]};
        return XCut(f);
    }
};
// A slice of G's parts, 4096 bytes apart, and of a whole fp32 operand whose rows, of 256 bytes, are K.
template <int KS>
__device__ __forceinline__ void read_whole(uint32_t a, const uint32_t (&b)[4], x_bf16x8 (&fa)[3], float (&fb)[8]) {
    asm volatile("ds_read_b128 %0, %11\n ds_read_b32 %3, %12 offset:%16\n ds_read_b32 %4, %13 offset:%16\n ds_read_b32 %5, %14 offset:%16\n"
                 "ds_read_b32 %6, %15 offset:%16\n ds_read_b128 %1, %11 offset:4096\n ds_read_b32 %7, %12 offset:%17\n ds_read_b32 %8, %13 offset:%17\n"
                 "ds_read_b32 %9, %14 offset:%17\n ds_read_b32 %10, %15 offset:%17\n ds_read_b128 %2, %11 offset:8192\n s_waitcnt lgkmcnt(0)"
                 : "=&v"(fa[0]), "=&v"(fa[1]), "=&v"(fa[2]), "=&v"(fb[0]), "=&v"(fb[1]), "=&v"(fb[2]), "=&v"(fb[3]), "=&v"(fb[4]), "=&v"(fb[5]),
                   "=&v"(fb[6]), "=&v"(fb[7])
                 : "v"(a), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "n"(KS * 4096), "n"(KS * 4096 + 1024) : "memory");
}
// (G through the transposing read, rows of 128 bytes)
template <int KS>
__device__ __forceinline__ void read_whole_tr(uint32_t a, const uint32_t (&b)[4], x_bf16x8 (&fa)[3], float (&fb)[8]) {
    x_s16x4 l[3], u[3];
    constexpr int OFF = KS * 2048;
    asm volatile("ds_read_b64_tr_b16 %0, %14 offset:%21\n ds_read_b64_tr_b16 %1, %14 offset:%22\n ds_read_b32 %6, %15 offset:%19\n"
                 "ds_read_b32 %7, %16 offset:%19\n ds_read_b32 %8, %17 offset:%19\n ds_read_b32 %9, %18 offset:%19\n"
                 "ds_read_b64_tr_b16 %2, %14 offset:%23\n ds_read_b64_tr_b16 %3, %14 offset:%24\n ds_read_b32 %10, %15 offset:%20\n"
                 "ds_read_b32 %11, %16 offset:%20\n ds_read_b32 %12, %17 offset:%20\n ds_read_b32 %13, %18 offset:%20\n"
                 "ds_read_b64_tr_b16 %4, %14 offset:%25\n ds_read_b64_tr_b16 %5, %14 offset:%26\n s_waitcnt lgkmcnt(0)"
                 : "=&v"(l[0]), "=&v"(u[0]), "=&v"(l[1]), "=&v"(u[1]), "=&v"(l[2]), "=&v"(u[2]), "=&v"(fb[0]), "=&v"(fb[1]), "=&v"(fb[2]), "=&v"(fb[3]),
                   "=&v"(fb[4]), "=&v"(fb[5]), "=&v"(fb[6]), "=&v"(fb[7])
                 : "v"(a), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "n"(KS * 4096), "n"(KS * 4096 + 1024), "n"(OFF), "n"(OFF + 512), "n"(OFF + 4096),
                   "n"(OFF + 4608), "n"(OFF + 8192), "n"(OFF + 8704) : "memory");
#pragma unroll
    for (int k = 0; k < 3; ++k) fa[k] = x_join(l[k], u[k]);
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

// The shapes of a tile.  Large: eight wavefronts of 128 x 64, one block per CU, for whatever fills the chip with it.  Middle: four of
// 64 x 64, two blocks per CU.  Small: four of 32 x 32, two blocks per CU, loads three steps ahead.  Deep: a small one by four groups of
// wavefronts that take every fourth step of K each and add their sums up at the end, for fewer tiles than CUs.  Parts: for operands in three
// parts, all of which a stage holds, so that each is loaded once for the six products: eight wavefronts of 64 x 32, one block per CU.
// fp32 operands of small and deep tiles lie in LDS whole and are cut where they are multiplied, each value by two wavefronts: that
// saves the pass that cuts them, for products that wait for memory and on one another's steps anyway (us of a training pass: 15 x 772 x 69968,
// where that pass was most of it, 683 -> 310, 157 x 3377 x 285, whose steps are few now, 242 -> 152).  Tiny, for the fewest tiles: eight
// wavefronts take every eighth step of a tile of 32 x 32 (128 x 2048 x 1000 34.4 -> 28.1); in fp32 sixteen take theirs straight from memory,
// which spreads the cutting over more CUs (152 -> 102; in bf16 the rows of 16-byte reads cost what that saves).
struct XBig { static constexpr int BM = 256, BN = 256, WM = 2, WN = 4, NS = 2, KG = 1, BK = 64, PARTS = 1; static constexpr bool DIRECT = false; };
struct XMid { static constexpr int BM = 128, BN = 128, WM = 2, WN = 2, NS = 2, KG = 1, BK = 64, PARTS = 1; static constexpr bool DIRECT = false; };
struct XSmall { static constexpr int BM = 64, BN = 64, WM = 2, WN = 2, NS = 4, KG = 1, BK = 64, PARTS = 1; static constexpr bool DIRECT = false; };
struct XDeep { static constexpr int BM = 64, BN = 64, WM = 2, WN = 2, NS = 2, KG = 4, BK = 64, PARTS = 1; static constexpr bool DIRECT = false; };
struct XTiny { static constexpr int BM = 32, BN = 32, WM = 1, WN = 1, NS = 2, KG = 8, BK = 64, PARTS = 1; static constexpr bool DIRECT = false; };
struct XTinyWhole { static constexpr int BM = 32, BN = 32, WM = 1, WN = 1, NS = 1, KG = 16, BK = 64, PARTS = 1; static constexpr bool DIRECT = true; };
struct XParts { static constexpr int BM = 128, BN = 128, WM = 2, WN = 4, NS = 2, KG = 1, BK = 32, PARTS = 3; static constexpr bool DIRECT = false; };
// What a stage holds of each operand: parts of K steps each.  WHOLE: fp32 as it is, which to its loads is twice as many bf16 along K, or,
// of the operand whose rows are K (OUT's second), along its columns; G is in parts.
template <typename C, int MODE, bool SPLIT>
struct XStage {
    static constexpr bool WHOLE = SPLIT && C::PARTS == 1, WOUT = WHOLE && MODE == XE_OUT;
    static constexpr int BK = WOUT ? 32 : C::BK, APARTS = WOUT ? 3 : C::PARTS, BPARTS = C::PARTS, BROWS = WOUT ? 2 * C::BN : C::BN;
    static constexpr int NS = WOUT ? 3 : C::NS;
    static constexpr int BYTES = (C::BM * APARTS + BROWS * BPARTS) * BK * 2;
    static constexpr int STAGES = C::DIRECT ? C::KG * C::BM * C::BN * 4 : C::KG * NS * BYTES;      // (direct: the groups' sums)
    static constexpr int SMEM = STAGES + C::WN * C::BM * 8 + C::BN * 4;       // stages, row statistics, biases
};
static constexpr int X_LAUNCH = 1 << 22;   // blocks of one launch, at most

// GP: the parts of G, 3 for fp32, whose operands are in three parts too (SPLIT), 2 or 1 for bf16.  DB: the column sums of G are wanted.
template <typename C, int MODE, int AKIND, int BKIND, int GP, bool DB>
__device__ __forceinline__ void xent_tile(const XentArgs& a, int block, int njobs) {
    constexpr bool SPLIT = GP == 3, TWICE = GP == 2 && MODE == XE_OUT;      // TWICE: every step of K once per part of G
    constexpr int BM = C::BM, BN = C::BN, WM = C::WM, WN = C::WN, NT = WM * WN * 64, MI = BM / (WM * 32), NJ = BN / (WN * 32);
    constexpr bool BIG = NJ == 2;
    static_assert((BIG && (MI == 4 || MI == 2)) || (MI == 1 && NJ == 1) || (C::PARTS == 3 && MI == 2 && NJ == 1 && SPLIT), "read_frags, read_step, read_parts");
    typedef XStage<C, MODE, SPLIT> S;
    constexpr int TM = BM / WM, TN = BN / WN, NS = S::NS, KG = C::KG, STAGE = S::BYTES;
    static_assert(KG == 1 || (AKIND == X_ROWS && BKIND == X_ROWS && MODE != XE_OUT), "groups skip steps");
    constexpr int BK = S::BK, PARTS = C::PARTS;
    constexpr bool WHOLE = S::WHOLE, WOUT = S::WOUT;
    typedef XOperand<BM, AKIND, NT, BK> OpA;
    typedef XOperand<S::BROWS, BKIND, NT, BK> OpB;
    constexpr int NP = OpA::PIECES * S::APARTS + OpB::PIECES * S::BPARTS;
    constexpr float L2E = 1.44269502f;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    float2* s_part = (float2*)(smem + S::STAGES);               // [WN][BM]; the column sums of G as floats [WM][BN]
    float* s_bias = (float*)(smem + S::STAGES + WN * BM * 8);   // [BN]
    const int group = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / NT), tid = threadIdx.x % NT;      // within the group
    const int lane = tid & 63, wave = tid >> 6, hi = lane >> 5, lo = lane & 31;
    const int wave_u = __builtin_amdgcn_readfirstlane(wave);
    const int wm = wave_u / WN, wn = wave_u % WN;

    // Jobs: the tiles of every split of K, four row tiles at a time, column by column.
    // Every XCD takes a stretch of that order, so that the tiles it works on at one time share their operands in its L2 (bands
    // of 2, 4, 8, 16, 32 row tiles: dw 4.23, 4.19, 4.42, 4.98, 5.24 ms of 8192 x 2048 x 131072, statistics, with the final loop, at 4, 8, 16 3.61, 3.66, 3.76).
    constexpr int BAND = 4;
    const long mtiles = (a.M + BM - 1) / BM, ntiles = (a.N + BN - 1) / BN, tiles = mtiles * ntiles;
    const int xcd = block & 7;
    const long job = a.job0 + xcd * (njobs / 8) + (xcd < njobs % 8 ? xcd : njobs % 8) + (block >> 3), tile = job % tiles, z = job / tiles;
    const long band = tile / (BAND * ntiles), rest = tile - band * BAND * ntiles;
    const long high = mtiles - band * BAND < BAND ? mtiles - band * BAND : BAND;
    const long mt = band * BAND + rest % high, nt = rest / high;
    const long m0 = mt * BM, n0 = nt * BN;
    const long kb = z * a.ksplit, ke = kb + a.ksplit < a.K ? kb + a.ksplit : a.K;
    const int steps = ke > kb ? (int)((ke - kb + BK - 1) / BK) * (TWICE ? 2 : 1) : 0;
    OpA pa;
    OpB pb;
    int kc = 0;                                                 // the step at the operands' windows
    int part0 = TWICE ? 1 : 0;                                  // the part of A that it takes, of those the first
    auto load_step = [&](int stage) {
        unsigned char* st = smem + (group * NS + stage) * STAGE;
        const long l = ke - kb - (long)kc * BK;
        const int left = l < BK ? (int)l : BK;
        uint64_t mask = ~0ull;
        if constexpr (AKIND == X_GCOLS) {
            const long k = kb + (long)kc * BK;
            mask = ((const __attribute__((address_space(4))) uint64_t*)a.kmask)[k / 64] >> (BK < 64 ? k % 64 : 0);
        }
#pragma unroll
        for (int part = 0; part < S::APARTS; ++part) {
#pragma unroll
            for (int q = 0; q < OpA::PIECES; ++q) pa.load(st + part * OpA::BYTES, q, left, ~0ull, wave_u, (part0 + part) * a.aplane * 2);
            if (part < S::BPARTS)
#pragma unroll
                for (int q = 0; q < OpB::PIECES; ++q) pb.load(st + S::APARTS * OpA::BYTES + part * OpB::BYTES, q, left, mask, wave_u, part * a.bplane * 2);
        }
    };
    auto next_step = [&](int stage) {
        if constexpr (KG > 1) {                                 // this group's next step: KG further on
            kc += KG;
            pa.restart((long)kc * BK);
            pb.restart((long)kc * BK);
        } else if (TWICE && part0 == 1) {                       // the same K of the large part (B comes from L2 this time)
            part0 = 0;
        } else {
            if (TWICE) part0 = 1;
            ++kc;
            pa.advance();
            pb.advance();
        }
        load_step(stage);
    };

    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const unsigned char*)smem;
    uint32_t aat[4], bat[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (OpA::KC ? q < BK / 16 : q < MI) aat[q] = lds0 + (OpA::KC ? OpA::frag_at(wm * TM, q, lane) : OpA::frag_at(wm * TM + q * 32, 0, lane));
        if (OpB::KC ? q < BK / 16 : q < NJ) bat[q] = lds0 + S::APARTS * OpA::BYTES + (OpB::KC ? OpB::frag_at(wn * TN, q, lane) : OpB::frag_at(wn * TN + q * 32, 0, lane));
    }
    if constexpr (WHOLE) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (OpA::KC && OpB::KC) {                           // two reads of four values per slice
                aat[q] = lds0 + OpA::whole_at(wm * TM, q, lane);
                bat[q] = lds0 + OpA::BYTES + OpB::whole_at(wn * TN, q, lane);
            } else {                                            // rows 8 hi + q of the lane's column
                const int k = 8 * hi + q, n = wn * TN + lo;
                bat[q] = lds0 + S::APARTS * OpA::BYTES + k * OpB::PITCH + ((n / 8) ^ OpB::swz(k)) * 32 + n % 8 * 4;
            }
        }
    }
    x_f32x16 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    constexpr bool SCALE = GP == 1 && MODE != XE_STATS;
    XScale scale;
    float factor = 1.f;
    if constexpr (SCALE && MODE == XE_OUT) scale.load(a.e, a.e.rows);      // (awaited behind the first steps' loads)
    if (!C::DIRECT && steps > 0) {
        pa.init(a.A, a.lda, m0, a.M, kb, tid);
        pb.init(a.B, a.ldb, WOUT ? 2 * n0 : n0, WOUT ? 2 * a.N : a.N, kb, tid);
        if constexpr (KG == 1) load_step(0);
    }
    constexpr int PA[6] = {2, 0, 1, 1, 0, 0}, PB[6] = {0, 2, 1, 0, 1, 0};      // of three parts, the small products first
    auto multiply_parts = [&](const x_bf16x8 (&fa)[3], const x_bf16x8 (&fb)[3]) {
#pragma unroll
        for (int k = 0; k < 6; ++k) acc[0][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[PB[k]], fa[PA[k]], acc[0][0], 0, 0, 0);
    };
    // fp32 logits: every 8 steps what the matrix cores have added up is added to a sum outside of them, which rounds to the nearest.  Theirs
    // lean to minus infinity, each addition by a little: of 2^21 features lse by 6e-6 of itself, of 65536 by 2e-7, now 4e-7 and 0.9e-7 (us of a pass of
    // 192 x 1024 x 30000 437 and 442, 512 x 1024 x 10007 322 and 323).
    constexpr bool SETTLE = SPLIT && MODE != XE_OUT;
    constexpr int CHAIN = 8;
    x_f32x16 settled[SETTLE && !C::DIRECT ? MI : 1][NJ];
    if constexpr (SETTLE && !C::DIRECT) {
#pragma unroll
        for (int i = 0; i < MI; ++i) settled[i][0] = acc[i][0];
    }
    auto settle = [&](int n, bool last) {                       // behind the n-th step
        if constexpr (SETTLE && !C::DIRECT) {
            if (!last && n % CHAIN != CHAIN - 1) return;
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                asm volatile("s_nop 11" : "+v"(acc[i][0]));     // (12 states between a product and what reads it: behind this branch the compiler leaves 3)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    settled[i][0][r] += acc[i][0][r];
                    acc[i][0][r] = last ? settled[i][0][r] : 0.f;
                }
            }
        }
    };
    auto join_groups = [&]() {                                  // the sums of all groups, in the first one
        float4* sums = (float4*)smem;                           // [KG - 1][4][NT]
        if (group > 0) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                sums[((group - 1) * 4 + r) * NT + tid] = make_float4(acc[0][0][4 * r], acc[0][0][4 * r + 1], acc[0][0][4 * r + 2], acc[0][0][4 * r + 3]);
        }
        __syncthreads();
        if (group > 0) return;
#pragma unroll 3
        for (int g = 0; g < KG - 1; ++g)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float4 o = sums[(g * 4 + r) * NT + tid];
                acc[0][0][4 * r] += o.x; acc[0][0][4 * r + 1] += o.y; acc[0][0][4 * r + 2] += o.z; acc[0][0][4 * r + 3] += o.w;
            }
    };
    if constexpr (BIG) {
        x_bf16x8 af[2][MI], bf[2][NJ];
        auto read = [&](auto slice, int stage) {
            constexpr int ks = decltype(slice)::value, f = ks & 1;
            const uint32_t so = stage * STAGE;
            if constexpr (OpA::KC && OpB::KC) {
                read_frags(aat[ks] + so, bat[ks] + so, af[f], bf[f]);
            } else {
                const uint32_t b[2] = {bat[0] + so, bat[1] + so};
                if constexpr (OpA::KC) {
                    read_frags<16 * ks * OpB::PITCH, (16 * ks + 4) * OpB::PITCH>(aat[ks] + so, b, af[f], bf[f]);
                } else {
                    uint32_t q[MI];
#pragma unroll
                    for (int i = 0; i < MI; ++i) q[i] = aat[i] + so;
                    read_frags<16 * ks * OpB::PITCH, (16 * ks + 4) * OpB::PITCH>(q, b, af[f], bf[f]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        };
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
        // One barrier per step, in front of its last group of products: behind it the next step is complete and this stage is
        // free, and the loads of the step after next go to it, a whole step ahead of their barrier.  The reads of a slice wait on their
        // own; of the two wavefronts of a SIMD one multiplies meanwhile.  ms of a training pass of 8192 x 2048 x 131072: loads spread over the
        // groups of the step before 19.5, at its start 17.6, behind its barrier 16.3, with the reads in one block each 15.5;
        // stages of 32 K, up to four steps ahead, gained nothing (18.0 against 17.6), four wavefronts of 128 x 128 lose (20.4).  Persistent
        // blocks that load a tile's first steps behind the epilogue before are no faster (that epilogue is 3 of 58 us at 2048 features).
        if (steps > 1) next_step(1);
        if constexpr (SCALE && MODE == XE_OUT) factor = scale.get(a.e, a.e.rows);
        if (steps > 0) {
            if (steps > 1) x_wait<NP>();
            else x_wait<0>();
            x_barrier();
            read(S0{}, 0);
        }
        for (int s = 0; s < steps; ++s) {
            const int cur = s & 1, nxt = cur ^ 1;
            multiply(0);
            read(S1{}, cur);
            multiply(1);
            read(S2{}, cur);
            multiply(0);
            read(S3{}, cur);
            x_wait<0>();
            x_barrier();
            multiply(1);
            if (s + 2 < steps) next_step(cur);
            __builtin_amdgcn_sched_barrier(0);
            if (s + 1 < steps) read(S0{}, nxt);
        }
    } else if constexpr (C::DIRECT) {
        static_assert(WHOLE, "fp32");
        // a wavefront's fragments come from memory as they are, those of its next step before this one's are multiplied
        const __amdgpu_buffer_rsrc_t ra = x_rsrc((const void*)OpA::uniform((uint64_t)(a.A + m0 * a.lda))), rb = x_rsrc((const void*)OpA::uniform((uint64_t)(a.B + n0 * a.ldb)));
        const uint32_t rowa = m0 + lo < a.M ? (uint32_t)(lo * a.lda * 2) : X_OOB, rowb = n0 + lo < a.N ? (uint32_t)(lo * a.ldb * 2) : X_OOB;
        x_bf16x8 fa[2][4], fb[2][4];
        auto fetch = [&](int s, int f) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {                       // two reads of four values per slice
                const long k = (long)s * BK + q / 2 * 32 + hi * 16 + q % 2 * 8;
                const uint32_t out = k < a.K ? 0 : X_OOB;
                fa[f][q] = __builtin_bit_cast(x_bf16x8, __builtin_amdgcn_raw_buffer_load_b128(ra, (int)((rowa + (uint32_t)(k * 2)) | out | (rowa & X_OOB)), 0, 0));
                fb[f][q] = __builtin_bit_cast(x_bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rb, (int)((rowb + (uint32_t)(k * 2)) | out | (rowb & X_OOB)), 0, 0));
            }
        };
        auto take = [&](int f) {
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) multiply_parts(XCut::of(fa[f][2 * ks], fa[f][2 * ks + 1]).part, XCut::of(fb[f][2 * ks], fb[f][2 * ks + 1]).part);
        };
        // (no registers are left for another sum: it lies in LDS, where the groups' meet)
        float4* sums = (float4*)smem;                           // [KG][4][NT]
        auto put = [&](bool first) {
            asm volatile("s_nop 11" : "+v"(acc[0][0]));         // (as above)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float4* at = sums + (group * 4 + r) * NT + tid;
                const float4 o = first ? make_float4(0.f, 0.f, 0.f, 0.f) : *at;
                *at = make_float4(o.x + acc[0][0][4 * r], o.y + acc[0][0][4 * r + 1], o.z + acc[0][0][4 * r + 2], o.w + acc[0][0][4 * r + 3]);
                acc[0][0][4 * r] = acc[0][0][4 * r + 1] = acc[0][0][4 * r + 2] = acc[0][0][4 * r + 3] = 0.f;
            }
        };
        bool first = true;
        if (group < steps) fetch(group, 0);
        for (int s = group, n = 0; s < steps; s += 2 * KG, n += 2) {
            if (s + KG < steps) fetch(s + KG, 1);
            take(0);
            if (s + KG < steps) {
                if (s + 2 * KG < steps) fetch(s + 2 * KG, 0);
                take(1);
            }
            if (n % CHAIN == CHAIN - 2) {
                put(first);
                first = false;
            }
        }
        if (group > 0 || !first) put(first);
        __syncthreads();
        if (group == 0) {
#pragma unroll 3
            for (int g = first ? 1 : 0; g < KG; ++g)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float4 o = sums[(g * 4 + r) * NT + tid];
                    acc[0][0][4 * r] += o.x; acc[0][0][4 * r + 1] += o.y; acc[0][0][4 * r + 2] += o.z; acc[0][0][4 * r + 3] += o.w;
                }
        }
    } else if constexpr (KG > 1) {
        kc = group - KG;
        if (group < steps) next_step(0);
        for (int s = 0; s < steps; s += KG) {                   // (as many barriers for every group)
            const int stage = s / KG & 1;
            x_wait<0>();
            x_barrier();
            if (s + KG + group < steps) next_step(stage ^ 1);
            if (s + group < steps) {
                x_bf16x8 fa[4], fb[4];
                const uint32_t so = (group * NS + stage) * STAGE;
                const uint32_t q[4] = {aat[0] + so, aat[1] + so, aat[2] + so, aat[3] + so}, b[4] = {bat[0] + so, bat[1] + so, bat[2] + so, bat[3] + so};
                read_step(q, b, fa, fb);
                if constexpr (WHOLE) {
#pragma unroll
                    for (int ks = 0; ks < 2; ++ks) multiply_parts(XCut::of(fa[2 * ks], fa[2 * ks + 1]).part, XCut::of(fb[2 * ks], fb[2 * ks + 1]).part);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[0][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[k], fa[k], acc[0][0], 0, 0, 0);
                }
            }
            settle(s / KG, false);
        }
        settle(0, true);
        x_wait<0>();
        x_barrier();
        join_groups();
    } else if constexpr (PARTS > 1) {
        static_assert(NS == 2, "two stages");
        for (int s = 0; s < steps; ++s) {                       // (three stages instead of two: the same time)
            const int stage = s & 1;
            x_wait<0>();
            x_barrier();
            if (s + 1 < steps) next_step(stage ^ 1);
            __builtin_amdgcn_sched_barrier(0);
            const uint32_t so = stage * STAGE;
            auto slice = [&](auto number) {
                constexpr int ks = decltype(number)::value, OFF = ks * 16 * OpB::PITCH;
                x_bf16x8 fa[3][2], fb[3];
                if constexpr (OpA::KC && OpB::KC) {
                    read_parts(aat[ks] + so, bat[ks] + so, fa, fb);
                } else if constexpr (OpA::KC) {
                    read_parts<OFF>(aat[ks] + so, bat[0] + so, fa, fb);
                } else {
                    const uint32_t q[2] = {aat[0] + so, aat[1] + so};
                    read_parts<OFF>(q, bat[0] + so, fa, fb);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int k = 0; k < 6; ++k)
#pragma unroll
                    for (int i = 0; i < MI; ++i) acc[i][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[PB[k]], fa[PA[k]][i], acc[i][0], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            };
            slice(std::integral_constant<int, 0>{});
            slice(std::integral_constant<int, 1>{});
            settle(s, false);
        }
        settle(0, true);
    } else {
        // One barrier per step: in front of it every wavefront waits for its loads of this step, behind it the stage of the step
        // before is free.
        if (steps > 1) next_step(1);
        if (NS > 3 && steps > 2) next_step(2);
        if constexpr (SCALE && MODE == XE_OUT) factor = scale.get(a.e, a.e.rows);
        int stage = 0;
        for (int s = 0; s < steps;) {                           // (a chain at a time: a branch in every step costs 3 % of 192 x 1024 x 30000)
            const int to = SETTLE && steps - s > CHAIN ? s + CHAIN : steps;
            for (; s < to; ++s) {
                if (s + NS - 2 < steps) x_wait<(NS - 2) * NP>();
                else x_wait<0>();
                x_barrier();
                if (s + NS - 1 < steps) next_step(stage == 0 ? NS - 1 : stage - 1);
                const uint32_t so = stage * STAGE;
                if constexpr (WOUT) {
                    const uint32_t b[4] = {bat[0] + so, bat[1] + so, bat[2] + so, bat[3] + so};
                    auto slice = [&](auto number) {
                        constexpr int ks = decltype(number)::value;
                        x_bf16x8 fa[3];
                        float fb[8];
                        if constexpr (OpA::KC) read_whole<ks>(aat[ks] + so, b, fa, fb);
                        else read_whole_tr<ks>(aat[0] + so, b, fa, fb);
                        multiply_parts(fa, XCut(fb).part);
                    };
                    slice(std::integral_constant<int, 0>{});
                    slice(std::integral_constant<int, 1>{});
                } else {
                    x_bf16x8 fa[4], fb[4];
                    const uint32_t q[4] = {aat[0] + so, aat[OpA::KC ? 1 : 0] + so, aat[OpA::KC ? 2 : 0] + so, aat[OpA::KC ? 3 : 0] + so};
                    const uint32_t b[4] = {bat[0] + so, bat[OpB::KC ? 1 : 0] + so, bat[OpB::KC ? 2 : 0] + so, bat[OpB::KC ? 3 : 0] + so};
                    if constexpr (OpA::KC && OpB::KC) read_step(q, b, fa, fb);
                    else if constexpr (OpA::KC) read_step(q, b[0], fa, fb);
                    else read_step(q[0], b[0], fa, fb);
                    if constexpr (WHOLE) {
#pragma unroll
                        for (int ks = 0; ks < 2; ++ks) multiply_parts(XCut::of(fa[2 * ks], fa[2 * ks + 1]).part, XCut::of(fb[2 * ks], fb[2 * ks + 1]).part);
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k) acc[0][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[k], fa[k], acc[0][0], 0, 0, 0);
                    }
                }
                stage = stage + 1 == NS ? 0 : stage + 1;
            }
            settle(CHAIN - 1, to == steps);
        }
    }

    if (KG > 1 && group > 0) return;                            // (barriers are among the wavefronts that are left)

    // ---- epilogue: this lane has rows mrow(i), columns nw + ncol(j, q) .. + 3
    const int wrow = wm * TM + lo;
    auto mrow = [&](int i) { return m0 + wrow + i * 32; };
    const long nw = n0 + wn * TN;
    const int cols = (int)(a.N - nw < TN ? a.N - nw : TN);       // of the wavefront's, those that there are
    auto ncol = [&](int j, int q) { return j * 32 + 8 * q + 4 * hi; };
    int label[MI];
    float lse[MI], up[MI];
    // where row i's label is among the columns, else below zero
    auto label_col = [&](int i) {
        const long ln = (long)label[i] - a.e.col0 - nw;
        return mrow(i) < a.M && is_class(label[i], a.e.classes) && ln >= 0 && ln < cols ? (int)ln : -1;
    };
    if constexpr (MODE != XE_OUT) {
        if constexpr (SCALE) {
            scale.load(a.e, a.M);
            factor = scale.get(a.e, a.M);
        }
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const long m = mrow(i) < a.M ? mrow(i) : a.M - 1;
            label[i] = a.e.labels[m];
            if constexpr (MODE == XE_GRAD) {
                lse[i] = a.e.lse[m];
                up[i] = SCALE ? a.e.dloss[m] / factor : a.e.dloss[m];      // (exact where they differ by a power of two)
            }
        }
        if (tid < BN) s_bias[tid] = a.e.bias && n0 + tid < a.N ? a.e.bias[a.e.col0 + n0 + tid] : 0.f;
        if (MODE == XE_GRAD && a.e.mask && nt == 0 && tid < BM) {
            const uint64_t b = __ballot(m0 + tid < a.M && is_class(a.e.labels[m0 + tid < a.M ? m0 + tid : 0], a.e.classes));
            if (lane == 0) {
                if (BM >= 64) a.e.mask[(m0 + tid) / 64] = b;
                else ((uint32_t*)a.e.mask)[m0 / 32] = (uint32_t)b;
            }
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float4 b = *(const float4*)(s_bias + wn * TN + ncol(j, q));
#pragma unroll
                for (int i = 0; i < MI; ++i) {
                    acc[i][j][4 * q] += b.x;
                    acc[i][j][4 * q + 1] += b.y;
                    acc[i][j][4 * q + 2] += b.z;
                    acc[i][j][4 * q + 3] += b.w;
                }
            }
        if (n0 + BN > a.N) {                                     // the last column tile: nothing behind the last class
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
            __builtin_amdgcn_sched_barrier(0);                   // one row at a time, within the registers
            const int ln = label_col(i);
            if (__any(ln >= 0)) {
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (ln == ncol(j, r / 4) + r % 4) a.e.picked[mrow(i)] = acc[i][j][r];
            }
            float mx = -__builtin_inff();
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) mx = fmaxf(mx, acc[i][j][r]);
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            const float from = mx == -__builtin_inff() ? 0.f : mx;           // (a row of minus infinities sums to zero)
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
        // this lane's first row in the block of G that has the wavefront's columns
        bf16_t* G = a.e.G + m0 / X_GTILE * a.e.ldg + nw / X_GCOLUMNS * (X_GTILE * X_GCOLUMNS) + (m0 % X_GTILE + wrow) * X_GCOLUMNS + nw % X_GCOLUMNS;
        static_assert(TN == X_GCOLUMNS || TN == 32, "a wavefront's columns are of one block of G");
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            __builtin_amdgcn_sched_barrier(0);                   // one row at a time, within the registers
            const bool use = mrow(i) < a.M && is_class(label[i], a.e.classes);
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r)                                 // (zero behind the last class: s is minus infinity there)
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
        if constexpr (DB) {
            // sums over the wavefront's rows, then over the wavefronts
            float* s_sum = (float*)s_part;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float t = acc[0][j][r];
#pragma unroll
                    for (int i = 1; i < MI; ++i) t += acc[i][j][r];
                    t = sum32(t);
                    if (lo == 31) s_sum[wm * BN + wn * TN + ncol(j, r / 4) + r % 4] = t;
                }
        }
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int q = 0; q < 4; q += 2) {
                    float f[8];
#pragma unroll
                    for (int t = 0; t < 8; ++t) f[t] = acc[i][j][4 * q + t];
#pragma unroll
                    for (int part = 0; part < GP; ++part) {
                        uint32_t w[4];
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            w[t] = pack_bf16x2(f[2 * t], f[2 * t + 1]);
                            if (part + 1 < GP) {
                                f[2 * t] -= __uint_as_float(w[t] << 16);
                                f[2 * t + 1] -= __uint_as_float(w[t] & 0xffff0000u);
                                if (GP == 2) {                          // (what is infinite or NaN is so in its first part alone)
                                    f[2 * t] = f[2 * t] == f[2 * t] ? f[2 * t] : 0.f;
                                    f[2 * t + 1] = f[2 * t + 1] == f[2 * t + 1] ? f[2 * t + 1] : 0.f;
                                }
                            }
                        }
                        swap_halves(w[0], w[2]);
                        swap_halves(w[1], w[3]);
                        *(any_u32x4*)(G + part * a.e.gplane + i * 32 * X_GCOLUMNS + j * 32 + 8 * (q + hi)) = any_u32x4{w[0], w[1], w[2], w[3]};
                    }
                }
        if constexpr (DB) {
            const float* s_sum = (const float*)s_part;
            x_wait_lds();
            x_barrier();
            if (tid < BN && n0 + tid < a.N) {
                float t = s_sum[tid];
#pragma unroll
                for (int w = 1; w < WM; ++w) t += s_sum[w * BN + tid];
                a.e.dbias_part[mt * a.e.lddb + n0 + tid] = t * factor;
            }
        }
    } else {
        // 32 rows of the wavefront at a time through LDS (behind the last barrier the stages are free, the small tiles' but for their last
        // step), so that rows are stored in stretches of its columns, results past the caches (dw of 4 x 2048 x 65536, which is little
        // but its store, 110 -> 65 us).
        if constexpr (!BIG) x_barrier();
        constexpr int Q = TN / 4;                                // quads of a row, permuted by the row
        float4* mine = (float4*)smem + wave_u * (32 * Q);
#pragma unroll
        for (int i = 0; i < MI; ++i) {
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    mine[lo * Q + ((j * 8 + 2 * q + hi) ^ (lo & (Q - 1)))] = make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
            // the quad c of row r with what is added to it; `there` columns of it and more
            auto quad = [&](int r, int c, long at, int there, float* f) {
                const float4 v = mine[r * Q + (c ^ (r & (Q - 1)))];
                f[0] = v.x * factor; f[1] = v.y * factor; f[2] = v.z * factor; f[3] = v.w * factor;
                if (a.e.acc) {
                    const any_u32x4 o = raw_load<float, 4>(a.e.acc + z * a.M * a.N + at, there);
#pragma unroll
                    for (int t = 0; t < 4; ++t) f[t] += raw_get<float>(o, t);
                }
            };
            if (a.e.out_f32) {
#pragma unroll
                for (int t = 0; t < 32 * Q / 64; ++t) {
                    const int r = (t * 64 + lane) / Q, c = (t * 64 + lane) % Q, there = cols - c * 4;
                    const long m = m0 + wm * TM + i * 32 + r, at = m * a.N + nw + c * 4;
                    if (m >= a.M || there <= 0) continue;
                    float f[4];
                    quad(r, c, at, there, f);
                    float* to = a.e.out_f32 + z * a.M * a.N + at;
                    if (a.ksplit < a.K && there >= 4) *(any_f32x4_at4*)to = any_f32x4{f[0], f[1], f[2], f[3]};      // (read again soon)
                    else raw_store<float, 4>(to, f, there);
                }
            } else {
#pragma unroll
                for (int t = 0; t < 16 * Q / 64; ++t) {
                    const int r = (t * 64 + lane) / (Q / 2), c = (t * 64 + lane) % (Q / 2), there = cols - c * 8;
                    const long m = m0 + wm * TM + i * 32 + r, at = m * a.N + nw + c * 8;
                    if (m >= a.M || there <= 0) continue;
                    float f[8];
                    quad(r, 2 * c, at, there, f);
                    quad(r, 2 * c + 1, at + 4, there - 4, f + 4);
                    raw_store<bf16_t, 8>(a.e.out + at, f, there);
                }
            }
        }
    }
}

template <typename C, int MODE, int AKIND, int BKIND, int GP, bool DB>
__global__ void __launch_bounds__(C::WM * C::WN * C::KG * 64) xent_tile_kernel(XentArgs a) {
    xent_tile<C, MODE, AKIND, BKIND, GP, DB>(a, blockIdx.x, gridDim.x);
}
// out[c] = sum of the rows of part [rows][ld], eight and then any number of them at a time
__device__ __forceinline__ void column_sum(const float* __restrict__ part, long rows, long ld, long n, float* __restrict__ out, long block) {
    const long c = block * 256 + threadIdx.x;
    if (c >= n) return;
    LongSum s;
    for (long r = 0; r < rows; r += 8) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) t += r + i < rows ? part[(r + i) * ld + c] : 0.f;
        s.add(t);
    }
    out[c] = s.get();
}
struct XColumns {
    const float* part;
    long rows, ld, n;
    float* out;
};
// The two products that read G, where both have small tiles: dx by the first nx blocks, dw by nw, the sums of dbias by any others.
template <int GP>
__global__ void __launch_bounds__(XSmall::WM * XSmall::WN * 64) xent_both_kernel(XentArgs dx, XentArgs dw, int nx, int nw, XColumns sums) {
    const int b = blockIdx.x;
    if (b < nx) xent_tile<XSmall, XE_OUT, X_GROWS, X_COLS, GP, false>(dx, b, nx);
    else if (b < nx + nw) xent_tile<XSmall, XE_OUT, X_GCOLS, X_COLS, GP, false>(dw, b - nx, nw);
    else column_sum(sums.part, sums.rows, sums.ld, sums.n, sums.out, b - nx - nw);
}

// Rows of C fp32 values as rows of Cp, zero behind the C-th.  Two tensors in a launch.
__global__ void __launch_bounds__(256) xent_pad_kernel(const float* __restrict__ in0, long rows0, float* __restrict__ out0, const float* __restrict__ in1,
                                                       long rows1, float* __restrict__ out1, int C, int Cp) {
    const long quads = (rows0 + rows1) * (Cp / 4);
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < quads; i += (long)gridDim.x * 256) {
        const long row = i / (Cp / 4);
        const int c = (int)(i % (Cp / 4)) * 4;
        const bool second = row >= rows0;
        const long r = second ? row - rows0 : row;
        *(any_u32x4*)((second ? out1 : out0) + r * Cp + c) = raw_load<float, 4>((second ? in1 : in0) + r * C + c, C - c);
    }
}

// Rows of C values as operands: PARTS bf16 parts (fp32: three, exact), rows of Cp values, zero behind the C-th.  Two tensors in a launch.
template <typename T, int PARTS>
__global__ void __launch_bounds__(256) xent_parts_kernel(const T* __restrict__ in0, long rows0, bf16_t* __restrict__ out0, long plane0,
                                                         const T* __restrict__ in1, long rows1, bf16_t* __restrict__ out1, long plane1, int C, int Cp) {
    const long pieces = (rows0 + rows1) * (Cp / 8);
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (long)gridDim.x * 256) {
        const long row = i / (Cp / 8);
        const int c = (int)(i % (Cp / 8)) * 8;
        const bool second = row >= rows0;
        const long r = second ? row - rows0 : row, plane = second ? plane1 : plane0;
        bf16_t* out = second ? out1 : out0;
        const T* p = (second ? in1 : in0) + r * C + c;
        float f[8];
        if constexpr (sizeof(T) == 2) {
            const auto v = raw_load<T, 8>(p, C - c);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = raw_get<T>(v, e);
        } else {
            const auto v = raw_load<T, 4>(p, C - c), w = raw_load<T, 4>(p + 4, C - c - 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[e] = raw_get<T>(v, e);
                f[4 + e] = raw_get<T>(w, e);
            }
        }
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
            any_u32x4 o;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t w = pack_bf16x2(f[2 * q], f[2 * q + 1]);
                if constexpr (PARTS > 1) {
                    // A finite value that rounds to infinity is cut off instead; what is infinite or NaN is so in its first part alone.
                    float lo = __uint_as_float(w << 16), hi = __uint_as_float(w & 0xffff0000u);
                    if (__builtin_isinf(lo) && !__builtin_isinf(f[2 * q])) w = (w & 0xffff0000u) | (__float_as_uint(f[2 * q]) >> 16);
                    if (__builtin_isinf(hi) && !__builtin_isinf(f[2 * q + 1])) w = (w & 0xffffu) | (__float_as_uint(f[2 * q + 1]) & 0xffff0000u);
                    lo = f[2 * q] - __uint_as_float(w << 16);
                    hi = f[2 * q + 1] - __uint_as_float(w & 0xffff0000u);
                    f[2 * q] = lo == lo ? lo : 0.f;
                    f[2 * q + 1] = hi == hi ? hi : 0.f;
                }
                o[q] = w;
            }
            *(any_u32x4*)(out + part * plane + r * Cp + c) = o;
        }
    }
}

// lse and loss of a row from its tiles: WAVES wavefronts per row
template <int WAVES>
__global__ void __launch_bounds__(256) xent_finish_kernel(const float2* __restrict__ part, const float* __restrict__ picked,
                                                          const int32_t* __restrict__ labels, float* __restrict__ loss, float* __restrict__ lse,
                                                          long M, long ntiles, long classes) {
    constexpr int PER = 4 / WAVES;
    __shared__ float2 s_part[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (long m0 = (long)blockIdx.x * PER; m0 < M; m0 += (long)gridDim.x * PER) {
        const long m = m0 + wave / WAVES;
        float mx = -__builtin_inff(), s = 0.f;
        if (m < M)
#pragma unroll 4
            for (long t = threadIdx.x % (WAVES * 64); t < ntiles; t += WAVES * 64) {
                const float2 p = part[t * M + m];
                join_softmax(mx, s, p.x, p.y);
            }
        for (int o = 32; o > 0; o >>= 1) {
            const float m2 = __shfl_xor(mx, o, 64), s2 = __shfl_xor(s, o, 64);
            join_softmax(mx, s, m2, s2);
        }
        if constexpr (WAVES > 1) {
            __syncthreads();
            if (lane == 0) s_part[wave] = make_float2(mx, s);
            __syncthreads();
            mx = s_part[0].x;
            s = s_part[0].y;
#pragma unroll
            for (int w = 1; w < WAVES; ++w) join_softmax(mx, s, s_part[w].x, s_part[w].y);
        }
        if (lane == 0 && wave % WAVES == 0 && m < M) {
            const float l = mx + logf(s);
            lse[m] = l;
            loss[m] = is_class(labels[m], classes) ? l - picked[m] : 0.f;
        }
    }
}

__global__ void __launch_bounds__(256) xent_colsum_kernel(const float* __restrict__ part, long rows, long ld, long n, float* __restrict__ out) {
    column_sum(part, rows, ld, n, out, blockIdx.x);
}
// out = sum of the splits' results, rounded once
template <typename T>
__global__ void __launch_bounds__(256) xent_join_kernel(const float* __restrict__ part, int splits, long n, T* __restrict__ out) {
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long)gridDim.x * 256) {
        float s = 0.f;
#pragma unroll 8
        for (int z = 0; z < splits; ++z) s += part[z * n + i];
        out[i] = Elem<T>::st(s);
    }
}

// ---- host --------------------------------------------------------------------------------
struct XentPlan {
    long piece, pieces;           // classes of a piece of G, number of pieces
    int gparts;                   // bf16 parts of G
    long Cp;                      // row pitch of x and w as operands
    bool whole;                   // fp32 operands as they are (small tiles only)
    bool cut;                     // x and w are made into operands in the workspace
    long pitch, depth;            // as the tiles see them: from row to row of x and w, features
    int size;                     // the tiles of s
    int sizedx, sizedw;           // of the two products that read G
    int zdx, zdw;                 // their splits of K
    long ntiles, mtiles;          // tiles of s: of all columns, of the rows, at most
    long ldg, gplane, xplane, wplane, lddb;
    size_t fwd_bytes, bwd_bytes;
    size_t o_x, o_w, o_part, o_picked, o_G, o_acc, o_dw, o_dbias, o_mask, o_scale;
};

// In bf16 G is one bf16 number per entry, or two, of 16 bits in all.  With few rows or classes a gradient is made of few entries, whose
// roundings do not average: of one row it is off by up to 2.0 times what the rounding of the results costs (1 x 76 x 3: 0.0033 of its norm, with
// two parts 0.0016), of more than 64 rows and classes by 1.0 to 1.2 times.  And there the second part costs little, since the products wait
// for what they read (us of a pass with one part and two: 64 x 2048 x 400 29 and 29, 8192 x 2048 x 10 67 and 67, 4 x 2048 x 65536 223 and
// 242, 64 x 2048 x 65536 240 and 270), where those of 1777 x 1000 x 32003, 235 of 538 us, would take twice as long.
static constexpr int X_GTWO = 64;
static constexpr size_t XENT_G_BYTES = (size_t)512 << 20;   // of a piece of G, at most (a piece has 1024 classes at least)

static long x_tiles(long M, long N, int t) { return ((M + t - 1) / t) * ((N + t - 1) / t); }

static int x_tile(int size) { return size == X_BIG ? 256 : size == X_MID ? 128 : size == X_SMALL ? 64 : 32; }
static int x_room(int size, bool parts) { return size == X_BIG || (size == X_MID && parts) ? 256 : 512; }      // blocks that run at one time

// Splits of K that fill the chip, each of 512 products per result at least (fp32: of parts).
static int x_splits(int size, long M, long N, long K, bool parts) {
    const long tiles = x_tiles(M, N, x_tile(size)), fill = x_room(size, parts);
    long z = tiles < fill ? fill / tiles : 1;
    const long most = std::max(1L, K * (parts ? 6 : 1) / 512);
    if (z > most) z = most;
    return (int)(z > 64 ? 64 : z);
}

// The largest tiles that fill half the chip, K split (split) or not, and are not more than half empty where the matrix is narrow.
// us of the products with small, middle, large tiles: statistics of 1777 x 1000 x 32003 244, 150, 144, of 4 x 2048 x 65536 (w read from HBM)
// 61, 69, 75, of 64 x 2048 x 400 17, 28, 50; dx of the first 231, 131 + 11, 110 + 18.  fp32, 2048 x 1024 x 10000: large tiles, with the
// pairs of parts one after the other along K, 288, middle ones that take them together 222.
static int x_size(long M, long N, long K, bool split, bool parts) {
    const long narrow = M < N ? M : N;
    for (int size = narrow > 128 && !parts ? X_BIG : narrow > 64 ? X_MID : X_SMALL; size > X_SMALL; --size)
        if (x_tiles(M, N, x_tile(size)) * (split ? x_splits(size, M, N, K, parts) : 1) >= x_room(size, parts) / 2) return size;
    return X_SMALL;
}

// The columns of s that fill whole rounds of tiles, and the tiles of the rest: where the last round would be at most half full, smaller
// ones that need one round of their own.  (A round of large, middle, small tiles at 1000 features: 36, 21, 9 us; in fp32 at 1024 41 for the
// middle ones, 18 for deep ones.  At fewer features there is less to win than the second launch costs, us of a pass without and with it:
// bf16 1777 x 128 x 32003 179, 182, x 256 254, 264, x 384 276, 274, 1030 x 128 x 14000 83, 85, x 256 128, 121, x 384 156, 143; fp32 512 x 128 x 8500
// 97, 98, x 256 127, 125, x 384 156, 147; from 512 on 1030 x 520 x 14000 172, 153.)
struct XRest {
    long columns;
    int size;
};
static XRest x_rest(const XentPlan& p, long M, long N, long D, bool f32) {
    const long t = x_tile(p.size), room = x_room(p.size, f32), mt = (M + t - 1) / t, whole = x_tiles(M, N, (int)t) / room * room / mt * t;
    if (whole > 0 && whole < N && D >= 512 && !(f32 && D % 4 != 0))
        for (int size = X_SMALL; size < p.size; ++size)
            if (x_tiles(M, N - whole, x_tile(size)) <= (f32 ? 256 : 512)) return {whole, size};
    return {N, p.size};
}
static long x_column_tiles(const XentPlan& p, long M, long N, long D, bool f32) {
    const XRest r = x_rest(p, M, N, D, f32);
    return (r.columns + x_tile(p.size) - 1) / x_tile(p.size) + (N - r.columns + x_tile(r.size) - 1) / x_tile(r.size);
}

static XentPlan xent_plan(const tsm_xent_desc* d) {
    XentPlan p{};
    const long R = d->rows, D = d->features, V = d->classes;
    const int parts = d->dtype == TSM_F32 ? 3 : 1;
    p.gparts = parts == 3 ? 3 : std::min(R, V) <= X_GTWO ? 2 : 1;
    const long grows = (R + X_GTILE - 1) / X_GTILE * X_GTILE;   // of G, whole blocks
    long piece = (long)(XENT_G_BYTES / (2 * p.gparts)) / grows / 1024 * 1024;
    if (piece < 1024) piece = 1024;
    if (piece > V) piece = V;
    p.piece = piece;
    p.pieces = (V + piece - 1) / piece;
    const bool f32 = parts == 3;
    // fp32 of few rows or classes: cutting x and w first costs more than larger tiles save (us of a pass of 100 x 3000 x 20000 with middle and
    // small tiles 921, 610, of 192 x 1024 x 30000 461, 435, of 256 x 1024 x 30000 513, 555)
    p.size = f32 && std::min(R, V) <= 192 ? X_SMALL : x_size(R, piece, D, false, f32);
    if ((f32 || D >= 512) && p.size == X_SMALL && x_tiles(R, V, 32) <= 256) p.size = X_TINY;
    p.whole = f32 && p.size <= X_SMALL;
    p.cut = p.whole ? D % 4 != 0 : f32 || D % 8 != 0;
    p.Cp = p.whole ? (D + 3) / 4 * 4 : (D + 7) / 8 * 8;
    p.pitch = p.whole ? 2 * p.Cp : p.Cp;
    p.depth = p.whole ? 2 * p.Cp : D;
    const int copies = p.whole ? 2 : parts;                     // of two bytes
    const long t = x_tile(p.size);
    const long last = V - (p.pieces - 1) * piece;
    p.ntiles = p.cut ? (p.pieces - 1) * x_column_tiles(p, R, piece, D, f32) + x_column_tiles(p, R, last, D, f32) : x_column_tiles(p, R, V, D, f32);
    p.mtiles = (R + t - 1) / t;
    for (const long n : {piece, last}) p.mtiles = std::max(p.mtiles, (R + x_tile(x_rest(p, R, n, D, f32).size) - 1) / x_tile(x_rest(p, R, n, D, f32).size));
    p.xplane = R * p.Cp;
    p.wplane = piece * p.Cp;
    p.ldg = (piece + std::max(t, 64L) - 1) / std::max(t, 64L) * std::max(t, 64L) * X_GTILE;
    p.gplane = grows / X_GTILE * p.ldg;
    p.lddb = (piece + 7) / 8 * 8;
    Arena f(nullptr, 0);
    p.o_x = f.used; f.take(p.cut ? (size_t)copies * p.xplane * 2 : 0);
    p.o_w = f.used; f.take(p.cut ? (size_t)copies * p.wplane * 2 : 0);
    Arena b = f;
    p.o_part = f.used; f.take((size_t)p.ntiles * R * 8);
    p.o_picked = f.used; f.take((size_t)R * 4);
    p.fwd_bytes = f.used;
    // (where s has larger tiles, its operands are in parts, and a whole one is the caller's own)
    const int least = f32 && !p.whole && D % 4 != 0 ? X_MID : X_SMALL;
    p.sizedx = p.whole ? X_SMALL : std::max(least, x_size(R, D, piece, true, f32));
    p.zdx = x_splits(p.sizedx, R, D, piece, f32);
    p.sizedw = p.whole ? X_SMALL : std::max(least, x_size(piece, D, R, true, f32));
    p.zdw = x_splits(p.sizedw, piece, D, R, f32);
    p.o_G = b.used; b.take((size_t)p.gparts * p.gplane * 2);
    p.o_acc = b.used; b.take((parts == 1 && p.pieces > 1) || p.zdx > 1 ? (size_t)p.zdx * R * D * 4 : 0);
    p.o_dw = b.used; b.take(p.zdw > 1 ? (size_t)p.zdw * piece * D * 4 : 0);
    p.o_dbias = b.used; b.take((size_t)p.mtiles * p.lddb * 4);
    p.o_mask = b.used; b.take((size_t)(R + 255) / 256 * 4 * 8);
    p.o_scale = b.used; b.take(p.gparts > 1 || R <= X_SCALE_ROWS ? 0 : 4);
    p.bwd_bytes = b.used;
    return p;
}

static int xent_check(const tsm_xent_desc* d, const char* who) {
    if (!d) return fail(TSM_ERR_NULLPTR, "%s: null descriptor", who);
    if (d->dtype != TSM_F32 && d->dtype != TSM_BF16) return fail(TSM_ERR_DTYPE, "%s: unknown dtype %d", who, d->dtype);
    if (d->rows <= 0 || d->features <= 0 || d->classes <= 0) return fail(TSM_ERR_SHAPE, "%s: non-positive dimension", who);
    if (d->features > (1 << 21)) return fail(TSM_ERR_SHAPE, "%s: more than 2^21 features", who);   // (a tile's offsets have 31 bits)
    if ((double)d->rows * d->features > 1e14 || (double)d->classes * d->features > 1e14) return fail(TSM_ERR_SHAPE, "%s: tensor too large", who);
    return TSM_OK;
}

static size_t xent_ws(const XentPlan& p) { return p.fwd_bytes > p.bwd_bytes ? p.fwd_bytes : p.bwd_bytes; }

static long x_ksplit(long K, int splits) { return ((K + splits - 1) / splits + 63) / 64 * 64; }

template <typename C, int MODE, int AKIND, int BKIND, int GP, bool DB>
static int x_launch(XentArgs a, int splits, const char* what, hipStream_t s) {
    auto kernel = xent_tile_kernel<C, MODE, AKIND, BKIND, GP, DB>;
    static OncePerDevice lds;
    TSM_TRY(raise_lds_limit((const void*)kernel, lds, what));
    const long jobs = x_tiles(a.M, a.N, C::BM) * splits;
    a.ksplit = x_ksplit(a.K, splits);
    for (a.job0 = 0; a.job0 < jobs; a.job0 += X_LAUNCH) {
        const long n = jobs - a.job0;
        kernel<<<dim3((unsigned)(n < X_LAUNCH ? n : X_LAUNCH)), dim3(C::WM * C::WN * C::KG * 64), XStage<C, MODE, GP == 3>::SMEM, s>>>(a);
        TSM_TRY(check_launch(what));
    }
    return TSM_OK;
}

template <int MODE, int AKIND, int BKIND, int GP, bool DB = false>
static int x_product(int size, const XentArgs& a, int splits, const char* what, hipStream_t s) {
    constexpr bool SPLIT = GP == 3;
    if constexpr (SPLIT) {
        if (size == X_MID) return x_launch<XParts, MODE, AKIND, BKIND, GP, DB>(a, splits, what, s);
    } else if constexpr (GP == 1 || MODE == XE_OUT) {           // (two parts: s is at most 64 rows or columns, and has small tiles)
        if (size == X_BIG) return x_launch<XBig, MODE, AKIND, BKIND, GP, DB>(a, splits, what, s);
        if (size == X_MID) return x_launch<XMid, MODE, AKIND, BKIND, GP, DB>(a, splits, what, s);
    }
    if constexpr (MODE != XE_OUT)
        if (size == X_TINY) return x_launch<typename std::conditional<SPLIT, XTinyWhole, XTiny>::type, MODE, AKIND, BKIND, GP, DB>(a, splits, what, s);
    if constexpr (MODE != XE_OUT)      // (us at 64 x 2048 x 400: 14.2 with small tiles, 10.3 with deep ones)
        if (x_tiles(a.M, a.N, 64) <= 256 && a.K >= 512) return x_launch<XDeep, MODE, AKIND, BKIND, GP, DB>(a, splits, what, s);
    return x_launch<XSmall, MODE, AKIND, BKIND, GP, DB>(a, splits, what, s);
}

// dx, dw and what is left of dbias in one launch: small ones would otherwise wait for one another's.
template <int GP>
static int x_both(XentArgs dx, int zdx, XentArgs dw, int zdw, const XColumns& sums, const char* what, hipStream_t s) {
    auto kernel = xent_both_kernel<GP>;
    static OncePerDevice lds;
    TSM_TRY(raise_lds_limit((const void*)kernel, lds, what));
    const long nx = x_tiles(dx.M, dx.N, XSmall::BM) * zdx, nw = x_tiles(dw.M, dw.N, XSmall::BM) * zdw;
    dx.ksplit = x_ksplit(dx.K, zdx);
    dw.ksplit = x_ksplit(dw.K, zdw);
    kernel<<<dim3((unsigned)(nx + nw + (sums.n + 255) / 256)), dim3(XSmall::WM * XSmall::WN * 64), XStage<XSmall, XE_OUT, GP == 3>::SMEM, s>>>(dx, dw, (int)nx, (int)nw, sums);
    return check_launch(what);
}

template <typename T>
static int xent_join(const float* part, int splits, long n, void* out, const char* what, hipStream_t s) {
    const long blocks = (n + 255) / 256;
    xent_join_kernel<T><<<dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, s>>>(part, splits, n, (T*)out);
    return check_launch(what);
}

// x (with the first piece) and a piece of w as operands: the caller's own where they can be, else made in the workspace.
template <typename T>
static int x_operands(const XentPlan& p, const void* x, long R, const void* w, long n, int C, char* ws, bool first, const bf16_t** xo, const bf16_t** wo,
                      hipStream_t s) {
    *xo = (const bf16_t*)x;
    *wo = (const bf16_t*)w;
    if (!p.cut) return TSM_OK;
    *xo = (const bf16_t*)(ws + p.o_x);
    *wo = (const bf16_t*)(ws + p.o_w);
    const long rows = first ? R : 0, blocks = ((rows + n) * (p.Cp / 8) + 255) / 256;
    if (sizeof(T) == 4 && p.whole) {
        const long quads = (rows + n) * (p.Cp / 4);
        xent_pad_kernel<<<dim3((unsigned)std::min((quads + 255) / 256, 8192L)), dim3(256), 0, s>>>((const float*)x, rows, (float*)(ws + p.o_x), (const float*)w, n,
                                                                                                   (float*)(ws + p.o_w), C, (int)p.Cp);
        return check_launch("xent_pad");
    }
    xent_parts_kernel<T, sizeof(T) == 2 ? 1 : 3><<<dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(256), 0, s>>>(
        (const T*)x, rows, (bf16_t*)(ws + p.o_x), p.xplane, (const T*)w, n, (bf16_t*)(ws + p.o_w), p.wplane, C, (int)p.Cp);
    return check_launch("xent_parts");
}

// The same for columns `from` to n of a piece; whole fp32 operands are the caller's own.
template <typename T>
static void x_columns(const XentPlan& p, XentArgs& a, long from, long n, const void* x, const T* w, long D) {
    a.N = n - from;
    a.e.col0 += from;
    a.B += from * p.pitch;
    if (sizeof(T) == 4) {
        a.A = (const bf16_t*)x;
        a.B = (const bf16_t*)(w + from * D);
        a.lda = a.ldb = a.K = 2 * D;
    }
}

template <typename T>
static int xent_fwd(const tsm_xent_desc* d, const XentPlan& p, const void* x, const void* w, const float* bias, const int32_t* labels, float* loss,
                    float* lse, char* ws, hipStream_t s) {
    constexpr bool F32 = sizeof(T) == 4;
    const long D = d->features, V = d->classes;
    XentArgs a{};
    a.lda = a.ldb = p.pitch;
    a.K = p.depth;
    a.M = d->rows;
    a.aplane = p.xplane;
    a.bplane = p.wplane;
    a.e.picked = (float*)(ws + p.o_picked);
    a.e.bias = bias; a.e.labels = labels; a.e.classes = V;
    // (nothing of the pieces' size but the operands of w: where the caller's own serve, the classes go in one piece)
    const long piece = p.cut ? p.piece : V;
    long tiles = 0;
    for (long v0 = 0; v0 < V; v0 += piece) {
        const long n = V - v0 < piece ? V - v0 : piece;
        TSM_TRY(x_operands<T>(p, x, a.M, (const T*)w + v0 * D, n, (int)D, ws, v0 == 0, &a.A, &a.B, s));
        const XRest rest = x_rest(p, a.M, n, D, F32);
        XentArgs b = a;
        b.N = rest.columns;
        b.e.col0 = v0;
        b.e.part = (float2*)(ws + p.o_part) + tiles * a.M;
        TSM_TRY((x_product<XE_STATS, X_ROWS, X_ROWS, F32 ? 3 : 1>(p.size, b, 1, "xent_stats", s)));
        tiles += (b.N + x_tile(p.size) - 1) / x_tile(p.size);
        if (b.N < n) {
            x_columns<T>(p, b, b.N, n, x, (const T*)w + v0 * D, D);
            b.e.part = (float2*)(ws + p.o_part) + tiles * a.M;
            TSM_TRY((x_product<XE_STATS, X_ROWS, X_ROWS, F32 ? 3 : 1>(rest.size, b, 1, "xent_stats_rest", s)));
            tiles += (b.N + x_tile(rest.size) - 1) / x_tile(rest.size);
        }
    }
    // few rows: four wavefronts each (4 rows x 1024 tiles: 65.0 -> 61.0 us for the whole call)
    const float2* part = (const float2*)(ws + p.o_part);
    const bool wide = a.M < 1024;
    const long blocks = wide ? a.M : std::min((a.M + 3) / 4, 65536L);
    if (wide) xent_finish_kernel<4><<<dim3((unsigned)blocks), dim3(256), 0, s>>>(part, a.e.picked, labels, loss, lse, a.M, tiles, V);
    else xent_finish_kernel<1><<<dim3((unsigned)blocks), dim3(256), 0, s>>>(part, a.e.picked, labels, loss, lse, a.M, tiles, V);
    return check_launch("xent_finish");
}

template <typename T, int GP>
static int xent_bwd(const tsm_xent_desc* d, const XentPlan& p, const void* x, const void* w, const float* bias, const int32_t* labels,
                    const float* lse, const float* dloss, void* dx, void* dw, float* dbias, char* ws, hipStream_t s) {
    constexpr bool F32 = sizeof(T) == 4;
    const long R = d->rows, D = d->features, V = d->classes;
    bf16_t* G = (bf16_t*)(ws + p.o_G);
    // fp32 results are added up where they go
    float *acc = F32 && p.zdx == 1 ? (float*)dx : (float*)(ws + p.o_acc), *dwp = (float*)(ws + p.o_dw), *dbp = (float*)(ws + p.o_dbias);
    uint64_t* mask = (uint64_t*)(ws + p.o_mask);
    const float* scale = nullptr;
    if (GP == 1 && R > X_SCALE_ROWS) {
        scale = (const float*)(ws + p.o_scale);
        xent_scale_kernel<<<dim3(1), dim3(1024), 0, s>>>(dloss, labels, d->rows, V, (float*)(ws + p.o_scale));
        TSM_TRY(check_launch("xent_scale"));
    }
    const bf16_t *xo, *wo;
    for (long c = 0; c < p.pieces; ++c) {
        const long v0 = c * p.piece, n = V - v0 < p.piece ? V - v0 : p.piece;
        TSM_TRY(x_operands<T>(p, x, R, (const T*)w + v0 * D, n, (int)D, ws, c == 0, &xo, &wo, s));
        XentArgs a{};
        a.A = xo; a.B = wo;
        a.lda = a.ldb = p.pitch;
        a.aplane = p.xplane; a.bplane = p.wplane;
        a.M = R; a.N = n; a.K = p.depth;
        a.e.bias = bias; a.e.labels = labels; a.e.classes = V; a.e.col0 = v0;
        a.e.lse = lse; a.e.dloss = dloss; a.e.scale = scale; a.e.G = G; a.e.ldg = p.ldg; a.e.gplane = p.gplane;
        a.e.mask = dw && c == 0 ? mask : nullptr;
        const bool both = dx && dw && p.sizedx == X_SMALL && p.sizedw == X_SMALL && x_tiles(R, D, 64) * p.zdx + x_tiles(n, D, 64) * p.zdw + n / 256 < X_LAUNCH;
        XColumns sums{};
        const XRest rest = x_rest(p, R, n, D, F32);
        for (int part = 0; part < (rest.columns < n ? 2 : 1); ++part) {
            const int size = part ? rest.size : p.size;
            const long mtiles = (R + x_tile(size) - 1) / x_tile(size);
            if (part) {
                x_columns<T>(p, a, rest.columns, n, x, (const T*)w + v0 * D, D);
                a.e.G += rest.columns / X_GCOLUMNS * (X_GTILE * X_GCOLUMNS);
                a.e.mask = nullptr;
            } else {
                a.N = rest.columns;
            }
            if (dbias) {
                // one row tile: its sums are the result
                a.e.dbias_part = mtiles == 1 ? dbias + a.e.col0 : dbp;
                a.e.lddb = p.lddb;
                TSM_TRY((x_product<XE_GRAD, X_ROWS, X_ROWS, GP, true>(size, a, 1, part ? "xent_grad_rest" : "xent_grad", s)));
                if (mtiles > 1 && both && rest.columns == n) {
                    sums = XColumns{dbp, mtiles, p.lddb, n, dbias + v0};
                } else if (mtiles > 1) {
                    xent_colsum_kernel<<<dim3((unsigned)((a.N + 255) / 256)), dim3(256), 0, s>>>(dbp, mtiles, p.lddb, a.N, dbias + a.e.col0);
                    TSM_TRY(check_launch("xent_dbias"));
                }
            } else {
                TSM_TRY((x_product<XE_GRAD, X_ROWS, X_ROWS, GP>(size, a, 1, part ? "xent_grad_rest" : "xent_grad", s)));
            }
        }
        XentArgs gx{}, gw{};
        gx.A = gw.A = G;
        gx.lda = gw.lda = p.ldg;
        gx.aplane = gw.aplane = p.gplane;
        gx.e.labels = gw.e.labels = labels;
        gx.e.dloss = gw.e.dloss = dloss;
        gx.e.scale = gw.e.scale = scale;
        gx.e.classes = gw.e.classes = V;
        gx.e.rows = gw.e.rows = R;
        gx.ldb = gw.ldb = p.pitch;
        T* out = (T*)dw + v0 * D;
        if (dx) {
            gx.B = wo; gx.bplane = p.wplane;
            if (F32 && p.sizedx == X_SMALL && !p.whole) {
                gx.B = (const bf16_t*)((const T*)w + v0 * D);
                gx.ldb = 2 * D;
            }
            gx.M = R; gx.N = D; gx.K = n;
            gx.e.acc = c > 0 ? acc : nullptr;
            if (F32 || p.zdx > 1 || c + 1 < p.pieces) gx.e.out_f32 = acc;
            else gx.e.out = (bf16_t*)dx;
        }
        if (dw) {
            gw.B = xo; gw.bplane = p.xplane;
            if (F32 && p.sizedw == X_SMALL && !p.whole) {
                gw.B = (const bf16_t*)x;
                gw.ldb = 2 * D;
            }
            gw.M = n; gw.N = D; gw.K = R;
            gw.kmask = mask;
            if (F32 || p.zdw > 1) gw.e.out_f32 = p.zdw > 1 ? dwp : (float*)out;
            else gw.e.out = (bf16_t*)out;
        }
        if (both) {
            TSM_TRY((x_both<GP>(gx, p.zdx, gw, p.zdw, sums, "xent_dx_dw", s)));
        } else {
            if (dx) TSM_TRY((x_product<XE_OUT, X_GROWS, X_COLS, GP>(p.sizedx, gx, p.zdx, "xent_dx", s)));
            if (dw) TSM_TRY((x_product<XE_OUT, X_GCOLS, X_COLS, GP>(p.sizedw, gw, p.zdw, "xent_dw", s)));
        }
        if (dx && p.zdx > 1 && c + 1 == p.pieces) TSM_TRY(xent_join<T>(acc, p.zdx, R * D, dx, "xent_dx_join", s));      // (each has added up its pieces)
        if (dw && p.zdw > 1) TSM_TRY(xent_join<T>(dwp, p.zdw, n * D, out, "xent_dw_join", s));
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
    const auto run = d->dtype == TSM_F32 ? xent_bwd<float, 3> : p.gparts == 2 ? xent_bwd<bf16_t, 2> : xent_bwd<bf16_t, 1>;
    return run(d, p, x, w, bias, labels, lse, dloss, dx, dw, dbias, (char*)ws, s);
}

}  // extern "C"
