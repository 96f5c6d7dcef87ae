// Rows of logits for logprobs.cu and distill.cu: shares of a row, running softmax
// statistics, and the stream that brings the rows into shared memory.
//
// A row is worked on by a cluster of 1 to 8 blocks, one share each.  From the
// row's first 16-byte boundary on it is a body of vectors of 16 bytes, split
// evenly over the cluster's blocks; the fewer than 8 elements before the first
// and after the last vector (rows of odd lengths start anywhere) go to the
// first and the last block, one element a thread.
//
// A share is worked on in chunks of THREADS * UNROLL vectors; warp w of the block has the chunk's vectors from 32 UNROLL w on,
// UNROLL rows of 32.  Where a row is visited once they are loaded into registers, a chunk
// ahead, and many small blocks share an SM: what one waits for at its row's end the others fill.
// Where a row is visited twice (statistics, then gradient) clusters are persistent, cluster i taking the
// rows i, i + clusters, ..., and the vectors travel by bulk copies through a ring in shared memory that keeps
// as much of the row as fits for the second visit; the copies run over row ends, so that while a
// row's statistics are joined the next row's first chunks arrive.
#pragma once

#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>

#include "tokens.cuh"

namespace pdb {

constexpr int UNROLL = 4;               // vectors of a thread under way in registers
constexpr int MAX_CLUSTER = 8;
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// whether logits can be scaled by it: positive, and c = scale * log2(e) finite (0 * c is 0 then, for the row's maximum)
inline bool usable_scale(float scale) { return scale > 0.0f && std::isfinite(scale * LOG2E); }

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

// two fp32 operations in one instruction
__device__ __forceinline__ uint64_t pair(float lo, float hi)
{
    uint64_t p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(lo), "f"(hi));
    return p;
}
__device__ __forceinline__ void unpair(uint64_t p, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t y;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b));
    return y;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t y;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b));
    return y;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t y;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(y) : "l"(a), "l"(b), "l"(c));
    return y;
}

// ---- transaction barriers in shared memory, and bulk copies that complete on them
__device__ __forceinline__ unsigned shared_addr(const void *p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t *bar, unsigned count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(shared_addr(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t *bar)
{
    asm volatile("{ .reg .b64 t; mbarrier.arrive.shared::cta.b64 t, [%0]; }" ::"r"(shared_addr(bar)) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t *bar, unsigned bytes)
{
    asm volatile("{ .reg .b64 t; mbarrier.arrive.expect_tx.shared::cta.b64 t, [%0], %1; }" ::"r"(shared_addr(bar)), "r"(bytes)
                 : "memory");
}
__device__ __forceinline__ bool bar_done(uint64_t *bar, unsigned parity)
{
    unsigned ok;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                 : "=r"(ok) : "r"(shared_addr(bar)), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ uint4 ld_shared(unsigned at)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
// four floats into shared memory of block `rank` of the cluster at the place that `to` has in this one, completing on that
// block's barrier at `bar`'s place
__device__ __forceinline__ void send_async(float *to, uint64_t *bar, int rank, float a, float b, float c, float d)
{
    unsigned dst, dbar;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(dst) : "r"(shared_addr(to)), "r"(rank));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(dbar) : "r"(shared_addr(bar)), "r"(rank));
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(dst), "f"(a),
                 "f"(b), "f"(c), "f"(d), "r"(dbar)
                 : "memory");
}
// `bytes` (a multiple of 16, both ends 16-byte aligned) from global to this block's shared memory
__device__ __forceinline__ void bulk_copy(void *to, const void *from, unsigned bytes, uint64_t *bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(shared_addr(to)),
                 "l"(from), "r"(bytes), "r"(shared_addr(bar))
                 : "memory");
}

// logits that are read once, or again by few threads, come through L2 only
__device__ __forceinline__ uint4 ld_keep(const uint4 *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
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

// Adds a thread's N vectors.  Per two elements: unpacking, (z - m) c in two roundings, two
// exponentials, their sum and, with ENT, the sum of e x (x held above -200, where e = 0, so that e x
// of a token masked by -inf is 0 and not a NaN).  The reference m moves only when the vectors'
// maximum passes it by 2^8: e <= 2^8 until then costs no precision.
template <typename T, bool ENT, int N>
__device__ __forceinline__ void add_vectors(Stat<ENT> &a, const uint4 (&v)[N], float c, float &top)
{
    constexpr int E = Vec<T>::E;
    typename Vec<T>::Max mx = Vec<T>::max_init();
#pragma unroll
    for (int u = 0; u < N; ++u) mx = Vec<T>::vmax(mx, v[u]);
    const float cm = Vec<T>::max_float(mx);
    top = fmaxf(top, cm);
    if (__fmul_rn(__fsub_rn(cm, a.m), c) > 8.0f) a.rebase(cm, c);
    const uint64_t m2 = pair(-a.m, -a.m), c2 = pair(c, c);
    uint64_t ps[2] = {0, 0}, pw[2] = {0, 0};      // short chains of sums
#pragma unroll
    for (int u = 0; u < N; ++u) {
        float f[E];
        Vec<T>::unpack(v[u], f);
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            uint64_t x = mul2(add2(pair(f[i], f[i + 1]), m2), c2);
            float x0, x1;
            unpair(x, x0, x1);
            if (ENT) {
                x0 = max_nan(x0, -200.0f), x1 = max_nan(x1, -200.0f);
                x = pair(x0, x1);
            }
            const uint64_t e = pair(ex2(x0), ex2(x1));
            const int k = (i >> 1) & 1;
            ps[k] = add2(ps[k], e);
            if (ENT) pw[k] = fma2(e, x, pw[k]);
        }
    }
    float lo, hi;
    unpair(add2(ps[0], ps[1]), lo, hi);
    a.s = __fadd_rn(a.s, __fadd_rn(lo, hi));
    if (ENT) {
        unpair(add2(pw[0], pw[1]), lo, hi);
        a.w = __fadd_rn(a.w, __fadd_rn(lo, hi));
    }
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

// where a thread's vectors of a chunk start; they are 32 apart
__device__ __forceinline__ int lane_start() { return (int)(threadIdx.x & ~31u) * UNROLL + (int)(threadIdx.x & 31); }

// a thread's vectors of the chunk at `base` of a share of `end` vectors, -inf past it: `first`, and every STEP-th
template <typename T, int THREADS, int STEP>
__device__ __forceinline__ void load_vectors(uint4 (&v)[UNROLL], const uint4 *share, int base, int first, int end)
{
    constexpr uint32_t N = Vec<T>::NEG_INF;
    const uint4 *from = share + base + first;
    if (base + UNROLL * THREADS <= end) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) v[u] = ld_keep(from + u * STEP);
    } else {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            v[u] = uint4{N, N, N, N};
            if (base + first + u * STEP < end) v[u] = ld_keep(from + u * STEP);
        }
    }
}

// barrier of the block's first THREADS threads (a kernel may have a warp more, which brings its rows)
template <int THREADS>
__device__ __forceinline__ void team_sync()
{
    asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
}

// joins the threads' statistics over the block, on every thread, with one barrier; `part` holds 3 * 32 floats and is
// not used again before another barrier
template <int THREADS, bool ENT>
__device__ __forceinline__ void block_join(Stat<ENT> &a, float c, float *part)
{
    constexpr int W = THREADS / 32;
    a.template warp_join<32>(c);
    if ((threadIdx.x & 31) == 0) {
        const int w = threadIdx.x >> 5;
        part[w] = a.m, part[32 + w] = a.s, part[64 + w] = a.w;
    }
    team_sync<THREADS>();
    const int lane = threadIdx.x & (W - 1);
    a.m = part[lane], a.s = part[32 + lane], a.w = part[64 + lane];
    a.template warp_join<W>(c);
}

constexpr int MOST_SLOTS = 16;
constexpr unsigned WAIT_TRIES = 1u << 22;   // of a wait, unless the handle has a lower limit; one takes some 20 ns to a microsecond

// One block's shares of its cluster's rows, chunk after chunk of SPAN = THREADS * UNROLL vectors, each row twice.
// A warp of its own brings the chunks by bulk copies into `slots` places, in turn (issued by one of the reading threads
// between its own chunks, 4096 x 128,000 bf16 took 419 us instead of 381); a place is free again
// when each of the THREADS / 32 other warps has given it back.  A row's last `hold` chunks stay in their places after the
// first visit and come again from there; the ones before are brought once more, after the held ones (L2 has seen them
// a few microseconds ago).  Every wait has a limit, after which the status word holds PDB_ETIMEOUT and no
// wait of the thread waits again.  A reader that has given up gives no place back; so the bringing thread runs out of
// places and of its own tries, brings nothing more, and waits for what it has under way before it ends.
template <typename T, int THREADS>
struct Stream {
    static constexpr int SPAN = THREADS * UNROLL;
    static constexpr unsigned LIMIT = WAIT_TRIES;
    uint4 *place;                       // slots * SPAN vectors
    uint64_t *full, *empty;             // a barrier for each place
    int *status;
    int slots, hold;
    int slot;                           // the next place to take or to fill
    unsigned parity;                    // its full barrier's
    unsigned tries;                     // of a wait
    bool gave_up;

    // whether it is done after so many tries
    __device__ __forceinline__ bool tried(uint64_t *bar, unsigned par, unsigned n)
    {
#pragma unroll 1
        for (unsigned i = 0; i < n; ++i)
            if (bar_done(bar, par)) return true;
        set_status(status, PDB_ETIMEOUT);
        return false;
    }
    __device__ __forceinline__ void wait(uint64_t *bar, unsigned par)
    {
        if (bar_done(bar, par) || gave_up) return;
        gave_up = !tried(bar, par, tries);
    }
    // A wait for the cluster's other blocks, each of which sends its numbers once it has done with its own waits, given up
    // or not: these must not be left out, so the limit is one that no run of another block's tries reaches
    __device__ __forceinline__ void wait_blocks(uint64_t *bar, unsigned par)
    {
        if (bar_done(bar, par)) return;
        gave_up |= !tried(bar, par, 4 * LIMIT);
    }
    // `bars` holds 2 * MOST_SLOTS barriers; a barrier of the block follows before the first use.  Without a try (tries_ == 0)
    // the readers have given up before they start; the bringing thread has more tries than they have
    __device__ __forceinline__ void start(uint4 *place_, uint64_t *bars, int slots_, int hold_, unsigned tries_, int *status_)
    {
        place = place_, full = bars, empty = bars + MOST_SLOTS, status = status_, slots = slots_, hold = hold_;
        slot = 0, parity = 0, tries = threadIdx.x < THREADS ? tries_ : tries_ + 1024, gave_up = tries == 0;
        if (gave_up) set_status(status, PDB_ETIMEOUT);
        if (threadIdx.x == 0) {
#pragma unroll 1
            for (int i = 0; i < slots; ++i) {
                bar_init(full + i, 1);
                bar_init(empty + i, THREADS / 32);
            }
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
    }
    __device__ __forceinline__ void next()
    {
        if (++slot == slots) slot = 0, parity ^= 1;
    }
    // chunks of a share that pass through, before the held ones (a row without vectors has one empty chunk)
    __device__ __forceinline__ int passing(int n_vec) const { return max(0, (max(n_vec, 1) + SPAN - 1) / SPAN - hold); }
    // the bringing thread, all of its work
    __device__ __forceinline__ void bring_rows(const T *logits, int64_t stride, int64_t rows, int cols, int64_t first,
                                               int64_t step, int rank, int blocks)
    {
        int brought = 0;
#pragma unroll 1
        for (int64_t r = first; r < rows && !gave_up; r += step) {
            const T *row = logits + r * stride;
            const Share sh = share_of(row, cols, rank, blocks);
            const uint4 *body = reinterpret_cast<const uint4 *>(row + sh.b0);
            const int n_vec = sh.v1 - sh.v0;
            int end = n_vec;
#pragma unroll 1
            for (int sweep = 0; sweep < 2 && !gave_up; ++sweep) {
#pragma unroll 1
                for (int v = 0; v < end || (sweep == 0 && v == 0); v += SPAN) {
                    wait(empty + slot, parity ^ 1);         // a place never used is free
                    if (gave_up) break;                     // it may still be in use, its copy under way
                    const int n = min(SPAN, end - v);
                    bar_expect(full + slot, n * 16);
                    if (n > 0) bulk_copy(place + slot * SPAN, body + v, n * 16, full + slot);
                    next();
                    ++brought;
                }
                end = passing(n_vec) * SPAN;                // the passing chunks once more
            }
        }
        // nothing is under way when the block ends, whatever became of the other warps and of the waits above
#pragma unroll 1
        for (int i = 0; i < min(slots, brought); ++i) {
            if (slot == 0) slot = slots, parity ^= 1;
            --slot;
            tried(full + slot, parity, LIMIT);
        }
    }
    // the next chunk's place, once it is there
    __device__ __forceinline__ int take()
    {
        wait(full + slot, parity);
        const int p = slot;
        next();
        return p;
    }
    // this thread's vectors in place p
    __device__ __forceinline__ void read(uint4 (&x)[UNROLL], int p) const
    {
        const unsigned at = shared_addr(place) + (unsigned)(p * SPAN + lane_start()) * 16;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) x[u] = ld_shared(at + u * 512);
    }
    __device__ __forceinline__ uint4 read_one(int p, int u) const
    {
        return ld_shared(shared_addr(place) + (unsigned)(p * SPAN + lane_start() + u * 32) * 16);
    }
    // the place of the chunk taken n takes ago
    __device__ __forceinline__ int before(int n) const { return slot - n < 0 ? slot - n + slots : slot - n; }
    // this warp has done with place p; not after a wait that ran out, behind which a copy may be under way to any place
    __device__ __forceinline__ void give_back(int p)
    {
        __syncwarp();
        if ((threadIdx.x & 31) == 0 && !gave_up) bar_arrive(empty + p);
    }
};

// How a call is cut: blocks of a cluster, threads of a block, clusters, dynamic shared memory; for the stream also its
// places, and how many chunks of a row are held.
struct Shape {
    int blocks, threads, map_bytes, bit_bytes;
    int64_t clusters;
    size_t smem;
    int slots, hold;
};
constexpr size_t SMEM_PER_SM = 228 << 10, STATIC_SMEM = 3072;

// blocks of a cluster: while they still find room on the SMs all at once (`room`: clusters of so many blocks) and each
// thread has a vector.  A row alone on one SM is bound by what that SM can have under way (4 x 128,000 bf16: 8 blocks
// 8.9 us, one 11.7)
template <typename F>
inline int cluster_of(int64_t rows, int64_t nv, int threads, F room)
{
    int blocks = 1;
    while (blocks < MAX_CLUSTER && rows <= room(blocks * 2) && nv / (blocks * 2) >= threads) blocks *= 2;
    return blocks;
}

// a share's marks: a bit per vector, in whole chunks, then a byte per vector
inline void set_maps(Shape &s, int64_t vectors)
{
    const int64_t chunk = s.threads * UNROLL;
    s.bit_bytes = (int)((vectors + chunk - 1) / chunk * chunk / 8);
    s.map_bytes = s.bit_bytes + (int)((vectors + 15) / 16 * 16);
}

// One visit per row: a cluster per row.  Many rows: small blocks, whose waits at a row's ends overlap (1024 x 32,000 fp16:
// 128 threads 16 us, 256 19, 512 27), 256 threads for rows of 128 KB and more (4096 x 128,000 bf16: 5 us of 157).
// Few rows: as many threads as have two vectors each, up to 512.
inline Shape once_shape(int64_t rows, int64_t cols, int vec, int sms, size_t extra, bool map)
{
    const int64_t nv = cols / vec + 1;
    Shape s = {};
    s.threads = rows < sms ? (nv < 1024 ? 128 : nv < 2048 ? 256 : 512) : nv < 8192 ? 128 : 256;
    s.blocks = cluster_of(rows, nv, s.threads, [&](int blocks) { return sms / blocks; });
    while (map && nv / s.blocks > 65536 && s.blocks < MAX_CLUSTER) s.blocks *= 2;      // room for the marks
    if (map) set_maps(s, nv / s.blocks + 1);
    s.smem = extra + s.map_bytes;
    s.clusters = rows;
    return s;
}

// how many blocks of so many threads, and the warp that brings their rows, an SM takes by their 96 registers a thread
constexpr int blocks_per_sm(int threads) { return threads == 64 ? 6 : 512 / threads; }

// shared memory of a block where `per` of them share an SM, which keeps 1 KB for each
constexpr size_t block_smem(int per) { return SMEM_PER_SM / per - 1024 - STATIC_SMEM; }

// Clusters of 1, 2, 4 and 8 blocks of k_distill_grad that run at once on a device (0: none of that size), as the device says it: an SM
// more or less in one of its groups takes more than its share of the larger clusters.
struct Room {
    static constexpr int ALONE = 3;
    int clusters[4][4];                 // by blocks of 256, 128, 64 threads, and one block an SM
};

// Two visits per row: persistent clusters of blocks of 64, 128 or 256 threads, each block with its warp that brings its
// rows and its part of the SM's shared memory for the stream.  A row goes to one block of 64 up to 20 KB (where `k` slots are one for
// a thread), to one of 128 up to 72, to two up to 144, then to two of 256, to four from 288 KB.  Measured with gradient (all of them 1% faster than since a wait that runs out stops the cluster), us, by
// 1 x 64, 1 x 128, 2 x 128, 1 x 256, 2 x 256, 4 x 256:
// 8000 x 2000 bf16 42, 57; 4000 x 10,000 bf16 44, 48; 8000 x 16,000 bf16 123, 113; 8000 x 32,000 bf16 -, 176, 212, 203, 308, 521;
// 4000 x 64,000 bf16 -, 222, 177, 174, 212, 320; 3000 x 40,000 fp32 -, 212, 181, 181, 160, 232;
// 4096 x 128,000 bf16 -, 475, 450, 447, 356, 451; 3000 x 90,000 fp32 -, 479, 470, 469, 398, 354.  Larger shares go to memory for
// their second visit (more than L2 keeps is under way); smaller ones leave too little work between a row's waits.
// No more clusters than run at once (room): one cluster more, and the others wait for its rows (76 clusters of 4 where 74
// have room: 3000 x 128,000 fp32 733 us, 487 by 74).
inline Shape twice_shape(int64_t rows, int64_t cols, int vec, const Room &room, size_t extra, int k)
{
    const int64_t nv = cols / vec + 1;
    Shape s = {};
    s.threads = nv <= 1280 && k <= 64 ? 64 : nv <= 9216 ? 128 : 256;
    const int per = blocks_per_sm(s.threads), kind = 8 - __builtin_ctz(s.threads);
    s.blocks = cluster_of(rows, nv, s.threads, [&](int blocks) { return room.clusters[kind][__builtin_ctz(blocks)]; });
    while (nv / s.blocks > s.threads * 36 && s.blocks < MAX_CLUSTER && room.clusters[kind][__builtin_ctz(s.blocks * 2)] > 0)
        s.blocks *= 2;
    set_maps(s, nv / s.blocks + 1);
    const size_t chunk = (size_t)UNROLL * 16 * s.threads, fixed = extra + s.map_bytes, most = block_smem(per);
    const int64_t chunks = std::max<int64_t>(1, (nv / s.blocks + UNROLL * s.threads) / (UNROLL * s.threads));
    const int64_t fit = fixed < most ? (int64_t)((most - fixed) / chunk) : 0;
    s.slots = (int)std::max<int64_t>(3, std::min({fit, 2 * chunks + 2, (int64_t)MOST_SLOTS}));
    s.hold = (int)std::max<int64_t>(1, std::min<int64_t>(chunks, s.slots - 2));
    s.smem = fixed + s.slots * chunk;
    s.clusters = std::min<int64_t>(rows, room.clusters[s.smem > most ? Room::ALONE : kind][__builtin_ctz(s.blocks)]);
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

template <typename... P, typename... A>
inline int launch_rows(void (*kernel)(P...), const Shape &shape, cudaStream_t s, A... args)
{
    if (!allow_smem((const void *)kernel)) return PDB_ECUDA;
    return launch(kernel, shape.clusters * shape.blocks, shape.threads, shape.smem, shape.blocks, s, args...);
}

}  // namespace pdb
