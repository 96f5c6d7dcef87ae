// Rows of a matrix moved E elements at a time (embed.cu, route.cu, clip.cu).
#pragma once

#include <type_traits>

#include "tokens.cuh"

namespace pdb {

template <int BYTES>
struct Raw;
template <>
struct Raw<2> { using type = uint16_t; };
template <>
struct Raw<4> { using type = uint32_t; };
template <>
struct Raw<8> { using type = uint2; };

template <typename T, int E>
struct alignas(E * sizeof(T)) Pack {
    T e[E];
};

// volatile: the loads of a batch are issued where they are written, all before the first is used
template <typename T, int E>
__device__ __forceinline__ Pack<T, E> load_pack(const T *p)
{
    constexpr int BYTES = E * sizeof(T);
    Pack<T, E> v;
    uint32_t *w = reinterpret_cast<uint32_t *>(&v);
    if constexpr (BYTES == 32)
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
    else if constexpr (BYTES == 16)
        asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
    else if constexpr (BYTES == 8)
        asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
    else if constexpr (BYTES == 4)
        asm volatile("ld.global.b32 %0, [%1];" : "=r"(w[0]) : "l"(p));
    else
        asm volatile("ld.global.b16 %0, [%1];" : "=h"(*reinterpret_cast<uint16_t *>(&v)) : "l"(p));
    return v;
}
template <typename T, int E>
__device__ __forceinline__ void store_pack(T *p, const Pack<T, E> &v)
{
    if constexpr (E * sizeof(T) == 32) {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(&v);
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                     "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
    } else if constexpr (E * sizeof(T) == 16) {
        __stcs(reinterpret_cast<uint4 *>(p), *reinterpret_cast<const uint4 *>(&v));
    } else {
        using R = typename Raw<E * sizeof(T)>::type;
        *reinterpret_cast<R *>(p) = *reinterpret_cast<const R *>(&v);
    }
}

// the elements in fp32 and back, 16-bit ones by the pair
template <typename T, int E>
__device__ __forceinline__ void to_floats(const Pack<T, E> &v, float (&f)[E])
{
    if constexpr (sizeof(T) == 2 && E % 2 == 0) {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(&v);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            if constexpr (std::is_same_v<T, __half>) {
                const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(w + i));
                f[2 * i] = x.x, f[2 * i + 1] = x.y;
            } else {
                f[2 * i] = __uint_as_float(w[i] << 16), f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) f[i] = to_float(v.e[i]);
    }
}
template <typename T, int E>
__device__ __forceinline__ Pack<T, E> of_floats(const float (&f)[E])
{
    Pack<T, E> v;
    if constexpr (sizeof(T) == 2 && E % 2 == 0) {
        uint32_t *w = reinterpret_cast<uint32_t *>(&v);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            if constexpr (std::is_same_v<T, __half>) {
                const __half2 x = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t *>(&x);
            } else {
                const __nv_bfloat162 x = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t *>(&x);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) v.e[i] = from_float<T>(f[i]);
    }
    return v;
}

// whether E elements of each row can be moved as one piece (up to 32 bytes: a lane's whole sector in one instruction)
inline bool fits(const pdb_mat *m, int E)
{
    const int bytes = E * type_bytes(m->type);
    return m->cols % E == 0 && (uintptr_t)m->data % bytes == 0 &&
           (m->rows < 2 || m->stride * type_bytes(m->type) % bytes == 0);
}

}  // namespace pdb
