// Shared by the token operators (embed.cu, logprobs.cu, distill.cu): element
// types, argument checks, the handle.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "common.cuh"

struct pdb_tokens {
    int device, sms;
    int64_t max_tokens, max_dim;
    unsigned tries;            // of a wait of k_distill_grad
    int *status;               // device: [0] first error recorded by a kernel; [1] always 0 (the radix
                               // sort's kernels return at once when their status word is set); [2] long runs (embed.cu)
    uint32_t *skey;            // [max_tokens] ids as sort keys in sorted order
    int32_t *spos;             // [max_tokens] their positions
    uint32_t *key, *tkey;      // [max_tokens] beyond what a cluster sorts: keys, and the radix sort's scratch
    int32_t *tpos;
    float *part;               // pieces of long runs (embed.cu)
    int4 *run_list;            // where they start, their pieces, their id
    pdb::Block arrays;         // holds the device arrays
    cudaEvent_t ev_use;        // recorded after the last work any call enqueued on the handle
};

namespace pdb {

// every call on a handle records ev_use when it returns; not while a graph is
// recorded, whose event could not be waited for (the graph's owner keeps the handle)
struct TokensUse {
    const pdb_tokens *t;
    cudaStream_t s;
    ~TokensUse()
    {
        cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
        if (cudaStreamIsCapturing(s, &capturing) != cudaSuccess || capturing != cudaStreamCaptureStatusNone) return;
        if (t->ev_use) cudaEventRecord(t->ev_use, s);
    }
};

// lets a kernel have all of an SM's shared memory as dynamic one; once per kernel and device
bool allow_smem(const void *kernel);

// PDB_OK where the current device is the handle's
inline int check_device(const pdb_tokens *t)
{
    int device = -1;
    if (cudaGetDevice(&device) != cudaSuccess) return PDB_ECUDA;
    return device == t->device ? PDB_OK : PDB_EINVAL;
}

inline int type_bytes(int type) { return type == PDB_TYPE_FLOAT ? 4 : 2; }

// elements from the first row's start to the last one's: what any memory holds, and far from the 64-bit range's end
constexpr int64_t MOST_EXTENT = (int64_t)1 << 58;

// PDB_OK for a matrix that the calls accept
inline int check_mat(const pdb_mat *m)
{
    if (!m || m->rows < 0 || m->cols < 0) return PDB_EINVAL;
    if (m->type != PDB_TYPE_FLOAT && m->type != PDB_TYPE_BFLOAT && m->type != PDB_TYPE_HALF) return PDB_EINVAL;
    if (m->rows > 1 && m->stride < m->cols) return PDB_EINVAL;
    if (m->rows > 0 && m->cols > 0 && (!m->data || (uintptr_t)m->data % type_bytes(m->type) != 0)) return PDB_EINVAL;
    if (m->cols > INT32_MAX / 2 || m->rows > INT32_MAX) return PDB_ETOOBIG;
    if (m->rows > 1 && m->stride > MOST_EXTENT / (m->rows - 1)) return PDB_EINVAL;
    return PDB_OK;
}

// ids of n rows of k each (pdb_ids.stride then is that of the rows)
inline int check_ids(const pdb_ids *ids, int64_t n, int64_t k = 1)
{
    if (!ids || ids->n != n * k) return PDB_EINVAL;
    if (n > 1 && ids->stride < k) return PDB_EINVAL;
    if (n * k > 0 && (!ids->data || (uintptr_t)ids->data % (ids->wide ? 8 : 4) != 0)) return PDB_EINVAL;
    if (n > 1 && ids->stride > MOST_EXTENT / (n - 1)) return PDB_EINVAL;
    return PDB_OK;
}

// the ids as the kernels take them
struct Ids {
    const void *data;
    int64_t stride;
    int wide;
};
inline Ids ids_of(const pdb_ids *ids, bool given = true)
{
    if (!given) return {nullptr, 0, 0};
    return {ids->data, ids->n > 1 ? ids->stride : 0, ids->wide};
}

// stride of a matrix whose stride may be unset (fewer than two rows)
inline int64_t stride_of(const pdb_mat *m) { return m->rows > 1 ? m->stride : m->cols; }

// whether `bytes` bytes at p share memory with rows of m
inline bool meets_rows(const char *p, int64_t bytes, const pdb_mat *m)
{
    const int64_t width = m->cols * type_bytes(m->type), step = stride_of(m) * type_bytes(m->type);
    // the first row that ends behind p is the one to look at
    const int64_t from = p - (const char *)m->data - width;
    const int64_t row = from < 0 ? 0 : from / step + 1;
    return row < m->rows && (const char *)m->data + row * step < p + bytes;
}

// whether two matrices share memory; rows of the one may lie between rows of the other
inline bool overlap(const pdb_mat *a, const pdb_mat *b)
{
    if (a->rows == 0 || b->rows == 0 || a->cols == 0 || b->cols == 0) return false;
    const char *a0 = (const char *)a->data, *b0 = (const char *)b->data;
    const int64_t sa = stride_of(a) * type_bytes(a->type), sb = stride_of(b) * type_bytes(b->type);
    const int64_t wa = a->cols * type_bytes(a->type), wb = b->cols * type_bytes(b->type);
    if (a0 + (a->rows - 1) * sa + wa <= b0 || b0 + (b->rows - 1) * sb + wb <= a0) return false;
    if (a->rows > 1 && b->rows > 1 && sa == sb) {
        // row i of a against row j of b: k = i - j decides, and any k of the range that lies where they meet
        const int64_t d = b0 - a0;
        const auto down = [&](int64_t x) { return x >= 0 ? x / sa : -((-x + sa - 1) / sa); };
        const int64_t first = std::max(down(d - wa) + 1, 1 - b->rows), last = std::min(-down(-(d + wb)) - 1, a->rows - 1);
        return first <= last;
    }
    const pdb_mat *few = a->rows <= b->rows ? a : b, *other = few == a ? b : a;
    for (int64_t i = 0; i < few->rows; ++i)
        if (meets_rows((const char *)few->data + i * (few == a ? sa : sb), few == a ? wa : wb, other)) return true;
    return false;
}

// a result that may be written over its input: the same matrix, or one apart
inline bool same_or_apart(const pdb_mat *a, const pdb_mat *b)
{
    if (!overlap(a, b)) return true;
    return a->data == b->data && a->type == b->type && stride_of(a) == stride_of(b);
}

// id k of row i
__device__ __forceinline__ int64_t load_id(Ids ids, int64_t i, int k = 0)
{
    const int64_t at = i * ids.stride + k;
    return ids.wide ? ((const int64_t *)ids.data)[at] : (int64_t)((const int *)ids.data)[at];
}

// the same in two steps, so that the warp does not wait for the load before it needs the id
__device__ __forceinline__ int2 fetch_id(Ids ids, int64_t i, int k = 0)
{
    const int64_t at = i * ids.stride + k;
    // (volatile: several of them are issued before the first is used)
    int2 raw = {0, 0};
    if (ids.wide) asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(raw.x), "=r"(raw.y) : "l"((const int2 *)ids.data + at));
    else asm volatile("ld.global.b32 %0, [%1];" : "=r"(raw.x) : "l"((const int *)ids.data + at));
    return raw;
}
__device__ __forceinline__ int64_t id_of(Ids ids, int2 raw)
{
    return ids.wide ? (int64_t)((uint64_t)(uint32_t)raw.y << 32 | (uint32_t)raw.x) : (int64_t)raw.x;
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }

template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// Every kernel of the token operators starts with this: it is launched while the kernel before it in the stream still
// runs (launch below), and waits here until that one has ended and its writes are visible.  Takes the launch's latency out
// of a sequence of calls (500 x 256 gradient, three kernels: 16.4 us a call -> 10.7).
// What these kernels read is read by plain loads: the read-only ones (.nc, __ldg, what the compiler makes of a
// const __restrict__ parameter) are for data that nobody writes while the kernel lives, and it lives while the kernel
// before it still writes; the compiler may also move them over the wait.
__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// lets the next kernel of the stream take its place on the SMs now (it waits for this one's end all the same)
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// `cluster` > 1: blocks of a cluster (grid is a multiple)
template <typename... P, typename... A>
inline int launch(void (*kernel)(P...), int64_t grid, int threads, size_t smem, int cluster, cudaStream_t s, A... args)
{
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, P(args)...);
    note_launch();
    if (e != cudaSuccess) cudaGetLastError();
    return e == cudaSuccess ? PDB_OK : PDB_ECUDA;
}

// a number as a type
template <int N>
struct Num {
    static constexpr int value = N;
};

// f called with a null pointer of the element type
template <typename F>
inline auto with_type(int type, F f)
{
    if (type == PDB_TYPE_FLOAT) return f((float *)nullptr);
    if (type == PDB_TYPE_BFLOAT) return f((__nv_bfloat16 *)nullptr);
    return f((__half *)nullptr);
}

}  // namespace pdb
