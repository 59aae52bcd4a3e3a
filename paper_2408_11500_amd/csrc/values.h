// Element types of token and block rows, accesses of several elements, and sums over groups of lanes.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "slicegcn_train.h"

namespace slicegcn {

using bf16 = __bf16;
using f16 = _Float16;

inline int type_bytes(int32_t type) { return type == SLICEGCN_F32 ? 4 : 2; }
inline bool known_type(int32_t type) { return type == SLICEGCN_F32 || type == SLICEGCN_BF16 || type == SLICEGCN_F16; }
// every element on a boundary of its size: accesses of 16 bytes start at any such boundary
inline bool aligned_for(const void *p, int32_t type) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(type_bytes(type) - 1)) == 0; }

// Whether rows are stored past the caches: where they exceed the last-level cache (256 MB).  A lookup of 128-wide fp32 rows alone, and with a
// pass that reads its output, through / past the caches: 64 MB 21.2 / 20.6 and 41.5 / 42.7 us, 128 MB 41.1 / 39.3 and 86.9 / 89.0, 256 MB 89.1 / 76.8 and
// 185.8 / 180.2, 1 GB 334 / 294 and 686 / 680; 2.4 M rows of 100 columns that lie 128 apart (lines written in part) 412 / 263 alone.
inline bool past_cache(int64_t rows, int64_t ld, int32_t type) { return rows * ld * type_bytes(type) >= (int64_t)256 << 20; }

// V elements that one access moves (16 bytes at most), at any element boundary
template <class T, int V> struct VecOf {
    typedef T type __attribute__((ext_vector_type(V)));
    typedef T packed __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};
template <class T> struct VecOf<T, 1> {
    struct type { T v; __device__ T &operator[](int) { return v; } __device__ T operator[](int) const { return v; } };
    typedef type packed;
};

template <class T, int V> __device__ inline typename VecOf<T, V>::type load_vec(const T *p)
{
    return *reinterpret_cast<const typename VecOf<T, V>::packed *>(p);
}

template <class T, int V> __device__ inline void store_vec(T *p, const float (&v)[V])
{
    typename VecOf<T, V>::type r;
#pragma unroll
    for (int i = 0; i < V; ++i) r[i] = (T)v[i]; // to nearest, ties to even: the one rounding of a result
    *reinterpret_cast<typename VecOf<T, V>::packed *>(p) = r;
}

// The same past the caches, for results too large to be found there by whoever reads them next: see past_cache.  (Which of the two is a
// template argument: of a branch between them the compiler makes one plain store.)
template <class T, int V> __device__ inline void store_vec_past_cache(T *p, const float (&v)[V])
{
    if constexpr (V == 1) {
        store_vec<T, V>(p, v);
    } else {
        typename VecOf<T, V>::type r;
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = (T)v[i];
        __builtin_nontemporal_store(r, reinterpret_cast<typename VecOf<T, V>::packed *>(p));
    }
}

template <bool PAST, class T, int V> __device__ inline void store_result(T *p, const float (&v)[V])
{
    if constexpr (PAST) store_vec_past_cache<T, V>(p, v);
    else store_vec<T, V>(p, v);
}

template <int CTRL> __device__ inline float dpp(float v)
{
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, true));
}

// Sum over groups of `lanes` (a power of two up to 64) neighbouring lanes, in every lane of a group the same bits: each step adds
// two sums that hold disjoint lanes, and both of their owners form the same sum.
__device__ inline float group_sum(float v, int lanes)
{
    if (lanes > 1) v += dpp<0xB1>(v);  // quad_perm [1,0,3,2]
    if (lanes > 2) v += dpp<0x4E>(v);  // quad_perm [2,3,0,1]
    if (lanes > 4) v += dpp<0x141>(v); // row_half_mirror
    if (lanes > 8) v += dpp<0x140>(v); // row_mirror
    if (lanes > 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (lanes > 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return v;
}

// Calls f with std::true_type or std::false_type
template <class F> inline auto with_flag(bool flag, F f) { return flag ? f(std::true_type()) : f(std::false_type()); }

// Calls f with a value of the element type `type`
template <class F> inline auto with_type(int32_t type, F f)
{
    return type == SLICEGCN_F32 ? f(float()) : type == SLICEGCN_BF16 ? f(bf16()) : f(f16());
}

} // namespace slicegcn
