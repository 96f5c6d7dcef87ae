// Rows of a matrix moved E elements at a time (embed.cu, route.cu, clip.cu).
#pragma once

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

// whether E elements of each row can be moved as one piece (up to 32 bytes: a lane's whole sector in one instruction)
inline bool fits(const pdb_mat *m, int E)
{
    const int bytes = E * type_bytes(m->type);
    return m->cols % E == 0 && (uintptr_t)m->data % bytes == 0 &&
           (m->rows < 2 || m->stride * type_bytes(m->type) % bytes == 0);
}

}  // namespace pdb
