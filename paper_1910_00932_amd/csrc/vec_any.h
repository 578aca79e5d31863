// Vectors of consecutive elements at any element address (odd row lengths): whole vectors go through one wide access, which the
// hardware takes at any alignment, the rest of a row element by element.
#pragma once
#include "common.h"

namespace tsm {

typedef uint32_t any_u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t any_u32x4 __attribute__((ext_vector_type(4)));
typedef any_u32x2 any_u32x2_at2 __attribute__((aligned(2)));
typedef any_u32x4 any_u32x4_at2 __attribute__((aligned(2)));
typedef any_u32x4 any_u32x4_at4 __attribute__((aligned(4)));
typedef float any_f32x4 __attribute__((ext_vector_type(4)));
typedef any_f32x4 any_f32x4_at4 __attribute__((aligned(4)));

// N elements of T as they lie in memory.
template <typename T, int N> struct RawVec;
template <> struct RawVec<bf16_t, 4> { typedef any_u32x2 type; typedef any_u32x2_at2 mem; };
template <> struct RawVec<bf16_t, 8> { typedef any_u32x4 type; typedef any_u32x4_at2 mem; };
template <> struct RawVec<float, 4> { typedef any_u32x4 type; typedef any_u32x4_at4 mem; };

template <typename T> __device__ __forceinline__ float raw_get(const any_u32x2& r, int i);
template <> __device__ __forceinline__ float raw_get<bf16_t>(const any_u32x2& r, int i) {
    return __uint_as_float(i & 1 ? r[i >> 1] & 0xffff0000u : r[i >> 1] << 16);
}
template <typename T> __device__ __forceinline__ float raw_get(const any_u32x4& r, int i);
template <> __device__ __forceinline__ float raw_get<bf16_t>(const any_u32x4& r, int i) {
    return __uint_as_float(i & 1 ? r[i >> 1] & 0xffff0000u : r[i >> 1] << 16);
}
template <> __device__ __forceinline__ float raw_get<float>(const any_u32x4& r, int i) { return __uint_as_float(r[i]); }

// n valid elements of N from p (n may exceed N or be below 1); the others are zero.
template <typename T, int N>
__device__ __forceinline__ typename RawVec<T, N>::type raw_load(const T* p, int n) {
    typedef typename RawVec<T, N>::type R;
    if (n >= N) return *(const typename RawVec<T, N>::mem*)p;
    R r{};
    constexpr int PER = 4 / sizeof(T);
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < n) {
            if constexpr (PER == 2) r[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
            else r[i] = __float_as_uint(p[i]);
        }
    return r;
}

// Stores the first n of the N values, rounded to T.  Whole vectors go past the caches (nontemporal), which leaves those to what is read:
// the recurrence over 64 x 8 frames 148 -> 127 us, over 4 x 4096 171 -> 148.
template <typename T, int N>
__device__ __forceinline__ void raw_store(T* p, const float (&f)[N], int n) {
    typedef typename RawVec<T, N>::type R;
    if (n >= N) {
        R r;
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) r[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) r[i] = __float_as_uint(f[i]);
        }
        __builtin_nontemporal_store(r, (typename RawVec<T, N>::mem*)p);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < n) p[i] = Elem<T>::st(f[i]);
}

}  // namespace tsm
