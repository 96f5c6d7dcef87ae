// One pass over a row of logits with the running maximum and sum of its softmax,
// shared by logprobs.cu and distill.cu.
//
// A row is worked on by a cluster of 1 to 8 blocks, one share each.  From the
// row's first 16-byte boundary on it is a body of vectors of 16 bytes, split
// evenly over the cluster's blocks; the fewer than 8 elements before the first
// and after the last vector (rows of odd lengths start anywhere) go to the
// first and the last block, one element a thread.
//
// Thread t of a block holds the vectors t, t + THREADS, ... of its share, UNROLL
// of them in registers at a time (64 bytes in flight per thread); what lies past
// the share's end is filled with -inf, which adds nothing.
#pragma once

#include <cooperative_groups.h>

#include "tokens.cuh"

namespace pdb {

constexpr int UNROLL = 4;
constexpr int MAX_CLUSTER = 8;
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// maximum that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// logits are read through L2 only: the first pass leaves them there for the second,
// the last pass marks them first to go
__device__ __forceinline__ uint4 ld_keep(const uint4 *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint4 ld_last(const uint4 *p)
{
    uint4 v;
    asm volatile("ld.global.cs.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

// 16 bytes of elements: unpacking, packing, maximum
template <typename T>
struct Vec;

template <>
struct Vec<float> {
    static constexpr int E = 4;
    static constexpr uint32_t NEG_INF = 0xff800000u;
    using Max = float;                          // running maximum in the elements' own form
    static __device__ __forceinline__ Max max_init() { return -INFINITY; }
    static __device__ __forceinline__ void unpack(const uint4 &v, float (&f)[E])
    {
        f[0] = __uint_as_float(v.x), f[1] = __uint_as_float(v.y), f[2] = __uint_as_float(v.z), f[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[E])
    {
        return {__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
    static __device__ __forceinline__ Max vmax(Max m, const uint4 &v)
    {
        float f[E];
        unpack(v, f);
        return fmaxf(m, fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3])));
    }
    static __device__ __forceinline__ float max_float(Max m) { return m; }
};

template <>
struct Vec<__nv_bfloat16> {
    static constexpr int E = 8;
    static constexpr uint32_t NEG_INF = 0xff80ff80u;
    using Max = __nv_bfloat162;
    static __device__ __forceinline__ Max of(uint32_t u) { return *reinterpret_cast<const Max *>(&u); }
    static __device__ __forceinline__ Max max_init() { return of(NEG_INF); }
    static __device__ __forceinline__ void unpack(const uint4 &v, float (&f)[E])
    {
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[2 * i] = __uint_as_float(u[i] << 16), f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[E])
    {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Max p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            u[i] = *reinterpret_cast<const uint32_t *>(&p);
        }
        return {u[0], u[1], u[2], u[3]};
    }
    static __device__ __forceinline__ Max vmax(Max m, const uint4 &v)
    {
        return __hmax2(m, __hmax2(__hmax2(of(v.x), of(v.y)), __hmax2(of(v.z), of(v.w))));
    }
    static __device__ __forceinline__ float max_float(Max m) { return fmaxf(__low2float(m), __high2float(m)); }
};

template <>
struct Vec<__half> {
    static constexpr int E = 8;
    static constexpr uint32_t NEG_INF = 0xfc00fc00u;
    using Max = __half2;
    static __device__ __forceinline__ Max of(uint32_t u) { return *reinterpret_cast<const Max *>(&u); }
    static __device__ __forceinline__ Max max_init() { return of(NEG_INF); }
    static __device__ __forceinline__ void unpack(const uint4 &v, float (&f)[E])
    {
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 p = __half22float2(of(u[i]));
            f[2 * i] = p.x, f[2 * i + 1] = p.y;
        }
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[E])
    {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Max p = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
            u[i] = *reinterpret_cast<const uint32_t *>(&p);
        }
        return {u[0], u[1], u[2], u[3]};
    }
    static __device__ __forceinline__ Max vmax(Max m, const uint4 &v)
    {
        return __hmax2(m, __hmax2(__hmax2(of(v.x), of(v.y)), __hmax2(of(v.z), of(v.w))));
    }
    static __device__ __forceinline__ float max_float(Max m) { return fmaxf(__low2float(m), __high2float(m)); }
};

// a block's share of a row: elements [j0, j1); in them vectors v0..v1 of the body (vector v starts at
// element head + v * E), before and after them edge elements
struct Share {
    int head;        // elements of the row before its first vector
    int v0, v1;      // the share's vectors
    int j0, j1;      // the share's elements, edges included
    int b0, b1;      // its vectors' elements
    __device__ __forceinline__ int edges() const { return (b0 - j0) + (j1 - b1); }
    // the i-th edge element
    __device__ __forceinline__ int edge(int i) const { return i < b0 - j0 ? j0 + i : b1 + (i - (b0 - j0)); }
};

template <typename T>
__device__ __forceinline__ Share share_of(const T *row, int cols, int rank, int blocks)
{
    constexpr int E = Vec<T>::E;
    Share s;
    s.head = min(cols, (int)(((16 - ((uintptr_t)row & 15)) & 15) / sizeof(T)));
    const int nv = (cols - s.head) / E;
    const int log = __ffs(blocks) - 1;            // a power of two
    s.v0 = (int)((int64_t)nv * rank >> log);
    s.v1 = (int)((int64_t)nv * (rank + 1) >> log);
    s.b0 = s.head + s.v0 * E;
    s.b1 = s.head + s.v1 * E;
    s.j0 = rank == 0 ? 0 : s.b0;
    s.j1 = rank == blocks - 1 ? cols : s.b1;
    return s;
}

// running softmax statistics: maximum m, s = sum of 2^x, w = sum of 2^x x with
// x = (z - m) c, c = scale * log2(e).  m starts at the lowest float, not at -inf,
// so that no difference is inf - inf: a row of -inf alone ends with s = 0.
template <bool ENT>
struct Stat {
    float m = -3.402823466e38f, s = 0.0f, w = 0.0f;
    __device__ __forceinline__ void rebase(float to, float c)
    {
        const float x = __fmul_rn(__fsub_rn(m, to), c), f = ex2(x);
        if (ENT) w = __fmul_rn(f, __fmaf_rn(fmaxf(x, -1e30f), s, w));
        s = __fmul_rn(s, f);
        m = to;
    }
    __device__ __forceinline__ void join(float m2, float s2, float w2, float c)
    {
        Stat o;
        o.m = m2, o.s = s2, o.w = w2;
        const float to = fmaxf(m, m2);
        rebase(to, c);
        o.rebase(to, c);
        s = __fadd_rn(s, o.s);
        if (ENT) w = __fadd_rn(w, o.w);
    }
    // over groups of LANES lanes: all to the largest m, then plain sums
    template <int LANES>
    __device__ __forceinline__ void warp_join(float c)
    {
        float to = m;
#pragma unroll
        for (int off = LANES / 2; off >= 1; off >>= 1) to = fmaxf(to, __shfl_xor_sync(FULL, to, off));
        rebase(to, c);
#pragma unroll
        for (int off = LANES / 2; off >= 1; off >>= 1) {
            s = __fadd_rn(s, __shfl_xor_sync(FULL, s, off));
            if (ENT) w = __fadd_rn(w, __shfl_xor_sync(FULL, w, off));
        }
    }
};

// adds a thread's UNROLL vectors.  Per element: unpacking, (z - m) c in two roundings,
// the exponential, its sum and, with ENT, the sum of e x (x held above -200, where e = 0, so
// that e x of a token masked by -inf is 0 and not a NaN).
template <typename T, bool ENT>
__device__ __forceinline__ void add_vectors(Stat<ENT> &a, const uint4 (&v)[UNROLL], float c, float &top)
{
    constexpr int E = Vec<T>::E;
    typename Vec<T>::Max mx = Vec<T>::max_init();
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) mx = Vec<T>::vmax(mx, v[u]);
    const float cm = Vec<T>::max_float(mx);
    top = fmaxf(top, cm);
    a.rebase(fmaxf(a.m, cm), c);
    const float m = a.m;
    float ps[UNROLL], pw[UNROLL];                 // UNROLL short chains of sums
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        float f[E];
        Vec<T>::unpack(v[u], f);
        ps[u] = pw[u] = 0.0f;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            float x = __fmul_rn(__fsub_rn(f[i], m), c);
            if (ENT) x = max_nan(x, -200.0f);
            const float e = ex2(x);
            ps[u] = __fadd_rn(ps[u], e);
            if (ENT) pw[u] = __fmaf_rn(e, x, pw[u]);
        }
    }
    a.s = __fadd_rn(a.s, __fadd_rn(__fadd_rn(ps[0], ps[1]), __fadd_rn(ps[2], ps[3])));
    if (ENT) a.w = __fadd_rn(a.w, __fadd_rn(__fadd_rn(pw[0], pw[1]), __fadd_rn(pw[2], pw[3])));
}

// one more element
template <bool ENT>
__device__ __forceinline__ void add_element(Stat<ENT> &a, float z, float c)
{
    a.rebase(fmaxf(a.m, z), c);
    const float x = max_nan(__fmul_rn(__fsub_rn(z, a.m), c), -200.0f);
    const float e = ex2(x);
    a.s = __fadd_rn(a.s, e);
    if (ENT) a.w = __fmaf_rn(e, x, a.w);
}

// the vectors base + threadIdx.x + u * THREADS below `end`
template <typename T, int THREADS>
__device__ __forceinline__ void load_vectors(uint4 (&v)[UNROLL], const uint4 *__restrict__ body, int base, int end)
{
    constexpr uint32_t N = Vec<T>::NEG_INF;
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const int i = base + (int)threadIdx.x + u * THREADS;
        v[u] = i < end ? ld_keep(body + i) : uint4{N, N, N, N};
    }
}

// joins the threads' statistics over the block, on every thread; `part` holds 3 * 32 floats
template <int THREADS, bool ENT>
__device__ __forceinline__ void block_join(Stat<ENT> &a, float c, float *part)
{
    constexpr int W = THREADS / 32;
    a.template warp_join<32>(c);
    if ((threadIdx.x & 31) == 0) {
        const int w = threadIdx.x >> 5;
        part[w] = a.m, part[32 + w] = a.s, part[64 + w] = a.w;
    }
    __syncthreads();
    const int lane = threadIdx.x & (W - 1);
    a.m = part[lane], a.s = part[32 + lane], a.w = part[64 + lane];
    a.template warp_join<W>(c);
}

// How many blocks share a row, and how many threads a block has.
//   threads  one for every four vectors of a row, 128 to 512
//   blocks   as long as the grid then still is at most two blocks per SM and each
//            thread keeps a vector: a row alone on one SM is bound by that SM's loads
struct Shape {
    int blocks, threads;
};
inline Shape row_shape(int64_t rows, int64_t cols, int vec, int sms)
{
    const int64_t nv = (cols + vec - 1) / vec;
    Shape s;
    s.threads = nv >= 2048 ? 512 : nv >= 1024 ? 256 : 128;
    s.blocks = 1;
    while (s.blocks < MAX_CLUSTER && rows * s.blocks * 2 <= (int64_t)sms * 2 && nv / (s.blocks * 2) >= s.threads) s.blocks *= 2;
    return s;
}

// f called with the number of threads as a type
template <typename F>
inline auto with_threads(int threads, F f)
{
    if (threads == 512) return f(Num<512>());
    if (threads == 256) return f(Num<256>());
    return f(Num<128>());
}

// launch of `rows` clusters
template <typename... P, typename... A>
inline int launch_rows(void (*kernel)(P...), int64_t rows, Shape shape, size_t smem, cudaStream_t s, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * shape.blocks));
    cfg.blockDim = dim3((unsigned)shape.threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {(unsigned)shape.blocks, 1, 1};
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, P(args)...);
    note_launch();
    if (e != cudaSuccess) cudaGetLastError();
    return e == cudaSuccess ? PDB_OK : PDB_ECUDA;
}

}  // namespace pdb
