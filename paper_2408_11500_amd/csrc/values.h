// Element types of token and block rows, accesses of several elements, and sums over groups of lanes.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "slicegcn_train.h"

namespace slicegcn {

using bf16 = __bf16;
using f16 = _Float16;

inline int type_bytes(int32_t type) { return type == SLICEGCN_F32 ? 4 : 2; }
inline bool known_type(int32_t type) { return type == SLICEGCN_F32 || type == SLICEGCN_BF16 || type == SLICEGCN_F16; }
// every element on a boundary of its size: accesses of 16 bytes start at any such boundary
inline bool aligned_for(const void *p, int32_t type) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(type_bytes(type) - 1)) == 0; }

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

// Calls f with a value of the element type `type`
template <class F> inline auto with_type(int32_t type, F f)
{
    return type == SLICEGCN_F32 ? f(float()) : type == SLICEGCN_BF16 ? f(bf16()) : f(f16());
}

} // namespace slicegcn
