// Rows of a table by token id, and the table's gradient by sorted ids
// (pdb_embed, pdb_embed_grad), and the handle of the token operators.
#include <algorithm>
#include <mutex>
#include <new>

#include "rows.cuh"

using namespace pdb;
namespace cg = cooperative_groups;

namespace {

// ------------------------------------------------------------------ E elements at a time
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

// ------------------------------------------------------------------ lookup
// A warp moves one piece of LOOKUP_UNROLL * 32 packs of one row: all its loads are issued before the
// first store.  Bound by memory; the id's and the row's latency are covered by the other warps.  16,384 rows of 4096
// bf16, word-like ids: 33.4 us, 189 MB at 5.6 TB/s; 8 rows of 1024: 1.6 us, launch and two latencies.
constexpr int LOOKUP_UNROLL = 4;

template <typename T, typename O, int E>
__global__ __launch_bounds__(256) void k_embed(const T *table, int64_t vocab, int64_t stride, Ids ids,
                                               int64_t n, int dim, int pieces, float scale, int64_t pad,
                                               O *__restrict__ out, int64_t out_stride, int *status)
{
    after_previous();
    const int lane = threadIdx.x & 31;
    const int64_t total = n * pieces, step = (int64_t)gridDim.x * 8;
    for (int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); w < total; w += step) {
        const int64_t i = total <= UINT32_MAX ? (int64_t)((uint32_t)w / (uint32_t)pieces) : w / pieces;
        const int piece = (int)(w - i * pieces);
        const int64_t v = load_id(ids, i);
        const bool there = v != pad && v >= 0 && v < vocab;
        if (!there && v != pad && lane == 0 && piece == 0) set_status(status, PDB_ERANGE);
        const T *from = table + v * stride;
        O *to = out + i * out_stride;
        const int j0 = (piece * LOOKUP_UNROLL * 32 + lane) * E;
        Pack<T, E> x[LOOKUP_UNROLL];
#pragma unroll
        for (int u = 0; u < LOOKUP_UNROLL; ++u)
            if (there && j0 + u * 32 * E < dim) x[u] = load_pack<T, E>(from + j0 + u * 32 * E);
#pragma unroll
        for (int u = 0; u < LOOKUP_UNROLL; ++u) {
            const int j = j0 + u * 32 * E;
            if (j >= dim) break;
            Pack<O, E> y;
#pragma unroll
            for (int e = 0; e < E; ++e) y.e[e] = from_float<O>(there ? __fmul_rn(scale, to_float(x[u].e[e])) : 0.0f);
            store_pack<O, E>(to + j, y);
        }
    }
}

// ------------------------------------------------------------------ sorted ids
// an id as a sort key; those left out (pad, out of range) sort last
__device__ __forceinline__ uint32_t embed_key(Ids ids, int2 raw, int64_t vocab, int64_t pad, int *status)
{
    const int64_t v = id_of(ids, raw);
    const bool there = v != pad && v >= 0 && v < vocab;
    if (!there && v != pad) set_status(status, PDB_ERANGE);
    return there ? (uint32_t)v : (uint32_t)vocab;
}

// more than SORT_MAX ids: the keys for the library's radix sort
__global__ void k_embed_keys(Ids ids, int64_t n, int64_t vocab, int64_t pad, uint32_t *__restrict__ key, int *long_runs,
                             int *status)
{
    after_previous();
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i == 0) *long_runs = 0;          // for k_embed_sum
    if (i < n) key[i] = embed_key(ids, fetch_id(ids, i), vocab, pad, status);
}

// Up to RANK_MAX ids: each id's place is the number of smaller ids and of equal ones before it,
// counted against all of them in shared memory.  A block places RANK_IDS ids, its
// threads in RANK_SLICES slices of the others.  n^2 comparisons over the whole GPU: the least latency for few ids.
constexpr int RANK_MAX = 2048, RANK_IDS = 64, RANK_SLICES = 8, RANK_THREADS = RANK_IDS * RANK_SLICES;

__global__ __launch_bounds__(RANK_THREADS) void k_embed_rank(Ids ids, int n, int64_t vocab, int64_t pad,
                                                             uint32_t *__restrict__ skey, int32_t *__restrict__ spos,
                                                             int *long_runs, int *status)
{
    after_previous();
    let_next_start();
    extern __shared__ __align__(16) uint32_t s_key[];       // n, rounded up to 4 * RANK_SLICES
    __shared__ int count[RANK_IDS];
    if (blockIdx.x == 0 && threadIdx.x == 0) *long_runs = 0;      // for k_embed_sum
    const int padded = (n + 4 * RANK_SLICES - 1) / (4 * RANK_SLICES) * (4 * RANK_SLICES);
    constexpr int EACH = RANK_MAX / RANK_THREADS;
    int2 raw[EACH];
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        const int i = j * RANK_THREADS + threadIdx.x;
        raw[j] = i < n ? fetch_id(ids, i) : int2{0, 0};
    }
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        const int i = j * RANK_THREADS + threadIdx.x;
        if (i < padded) s_key[i] = i < n ? embed_key(ids, raw[j], vocab, pad, status) : 0xffffffffu;   // the fill counts for nobody
    }
    if (threadIdx.x < RANK_IDS) count[threadIdx.x] = 0;
    __syncthreads();
    const int mine = blockIdx.x * RANK_IDS + threadIdx.x % RANK_IDS, slice = threadIdx.x / RANK_IDS;
    const int first = blockIdx.x * RANK_IDS, last = first + RANK_IDS;
    const int j0 = padded / RANK_SLICES * slice, j1 = padded / RANK_SLICES * (slice + 1);
    if (mine < n) {
        const uint32_t k = s_key[mine];
        int c = 0;
        // before the block's own ids equal ones count, behind them they do not
        for (int j = j0; j < min(j1, first); j += 4) {
            const uint4 o = *reinterpret_cast<const uint4 *>(s_key + j);
            c += (o.x <= k) + (o.y <= k) + (o.z <= k) + (o.w <= k);
        }
        for (int j = max(j0, first); j < min(j1, last); ++j) c += s_key[j] < k || (s_key[j] == k && j < mine) ? 1 : 0;
        for (int j = max(j0, last); j < j1; j += 4) {
            const uint4 o = *reinterpret_cast<const uint4 *>(s_key + j);
            c += (o.x < k) + (o.y < k) + (o.z < k) + (o.w < k);
        }
        if (c) atomicAdd(&count[threadIdx.x % RANK_IDS], c);
    }
    __syncthreads();
    if (slice == 0 && mine < n) {
        skey[count[threadIdx.x]] = s_key[mine];
        spos[count[threadIdx.x]] = mine;
    }
}

// Up to SORT_MAX ids: the whole stable sort in one launch, by a cluster of 1 to 8 blocks that keep the pairs (key, position)
// in their shared memory.  Least significant digit first, passes of up to 10 bits: one for a table of fewer than 2^10 rows, two
// below 2^20, three below 2^30, four above.  A warp ranks its pairs by one ballot per digit bit and running counts per digit; the
// counts are summed over the warps, then over the cluster; the pairs are put in order within the block
// and then stored where they belong, in whichever block's shared memory that is, neighbours together (stored one by
// one from their places, 65,536 pairs took 19 us a pass).
constexpr int SORT_THREADS = 512, SORT_WARPS = SORT_THREADS / 32, SORT_CLUSTER = 8, SORT_MAX = 65536, SORT_BITS = 10;

inline size_t sort_smem(int ipt)
{
    return sizeof(uint2) * 2 * SORT_THREADS * ipt + sizeof(uint32_t) * 3 * (1 << SORT_BITS) +
           sizeof(uint16_t) * SORT_WARPS * (1 << SORT_BITS);
}

// Rows of the gradient that the SMs which have nothing to sort fill with zeros meanwhile (k_embed_sum then writes those that
// do occur): `row` pieces of 16 bytes each, `stride` bytes apart.
struct Fill {
    char *to;
    int64_t rows, stride;
    int row;
};

template <int IPT>
__global__ __launch_bounds__(SORT_THREADS) void k_embed_sort(Ids ids, int n, int64_t vocab, int64_t pad, int passes, int bits,
                                                             uint32_t *__restrict__ skey, int32_t *__restrict__ spos,
                                                             int *long_runs, Fill fill, int *status)
{
    after_previous();
    let_next_start();
    constexpr int SPAN = SORT_THREADS * IPT;
    extern __shared__ __align__(16) uint2 s_pair[];         // [SPAN] this block's part of the order: key, position
    uint2 *s_local = s_pair + SPAN;                         // [SPAN] its pairs by digit
    uint32_t *s_hist = reinterpret_cast<uint32_t *>(s_local + SPAN);   // [1 << SORT_BITS] its count of each digit
    uint32_t *s_first = s_hist + (1 << SORT_BITS);          // where each digit starts in s_local
    uint32_t *s_move = s_first + (1 << SORT_BITS);          // from there to its place in the whole order
    uint16_t *s_warp = reinterpret_cast<uint16_t *>(s_move + (1 << SORT_BITS));   // [warp][digit]
    __shared__ uint32_t s_total[2][SORT_WARPS];
    cg::cluster_group cluster = cg::this_cluster();
    const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (blockIdx.x >= blocks) {          // another cluster's block: a warp a row
        for (int64_t r = (int64_t)(blockIdx.x - blocks) * SORT_WARPS + warp; r < fill.rows;
             r += (int64_t)(gridDim.x - blocks) * SORT_WARPS)
            for (int j = lane; j < fill.row; j += 32)
                __stcs(reinterpret_cast<uint4 *>(fill.to + r * fill.stride) + j, uint4{0, 0, 0, 0});
        return;
    }
    const unsigned lt = lanemask_lt();
    const int radix = 1 << bits;
    if (rank == 0 && tid == 0) *long_runs = 0;              // for k_embed_sum
    uint32_t key[IPT];
    int32_t pos[IPT];
    int2 raw[IPT];
#pragma unroll
    for (int i = 0; i < IPT; ++i) {
        pos[i] = rank * SPAN + warp * (32 * IPT) + i * 32 + lane;
        raw[i] = pos[i] < n ? fetch_id(ids, pos[i]) : int2{0, 0};
    }
#pragma unroll
    for (int i = 0; i < IPT; ++i)
        key[i] = pos[i] < n ? embed_key(ids, raw[i], vocab, pad, status) : 0xffffffffu;      // the fill sorts behind all
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = pass * bits;
        uint16_t *count = s_warp + warp * radix;
        for (int d = lane; d < radix; d += 32) count[d] = 0;
        __syncwarp();
        uint32_t place[IPT];
#pragma unroll
        for (int i = 0; i < IPT; ++i) {
            const uint32_t d = key[i] >> shift & (radix - 1);
            unsigned peers = FULL;
            for (int b = 0; b < bits; ++b) {
                const unsigned m = __ballot_sync(FULL, d >> b & 1);
                peers &= d >> b & 1 ? m : ~m;
            }
            place[i] = __popc(peers & lt) | __popc(peers) << 16;
        }
#pragma unroll
        for (int i = 0; i < IPT; ++i) {
            const uint32_t d = key[i] >> shift & (radix - 1);
            const uint32_t c = count[d];
            __syncwarp();
            if ((place[i] & 0xffff) == 0) count[d] = (uint16_t)(c + (place[i] >> 16));
            place[i] = c + (place[i] & 0xffff);
            __syncwarp();
        }
        __syncthreads();
        // digits 2 tid, 2 tid + 1: counts by warp become places, their sums the block's counts
        uint32_t own[2] = {0, 0};
        if (2 * tid < radix) {
#pragma unroll
            for (int w = 0; w < SORT_WARPS; ++w) {
                uint32_t *at = reinterpret_cast<uint32_t *>(s_warp + w * radix + 2 * tid);
                const uint32_t c = *at;
                *at = own[1] << 16 | own[0];
                own[0] += c & 0xffff, own[1] += c >> 16;
            }
            s_hist[2 * tid] = own[0], s_hist[2 * tid + 1] = own[1];
        }
        cluster.sync();                  // every block has its pairs in registers and its counts in place
        // pairs of the two digits in all blocks, and in those before this one
        uint32_t all[2] = {0, 0}, before[2] = {0, 0};
        if (2 * tid < radix) {
            uint2 h[SORT_CLUSTER];
#pragma unroll
            for (int b = 0; b < SORT_CLUSTER; ++b)
                h[b] = *reinterpret_cast<const uint2 *>(cluster.map_shared_rank(s_hist, min(b, blocks - 1)) + 2 * tid);
#pragma unroll
            for (int b = 0; b < SORT_CLUSTER; ++b)
                if (b < blocks) {
                    all[0] += h[b].x, all[1] += h[b].y;
                    if (b < rank) before[0] += h[b].x, before[1] += h[b].y;
                }
        }
        uint32_t x = all[0] + all[1], y = own[0] + own[1];
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const uint32_t u = __shfl_up_sync(FULL, x, off), v = __shfl_up_sync(FULL, y, off);
            if (lane >= off) x += u, y += v;
        }
        if (lane == 31) s_total[0][warp] = x, s_total[1][warp] = y;
        __syncthreads();
        x -= all[0] + all[1], y -= own[0] + own[1];
#pragma unroll
        for (int w = 0; w < SORT_WARPS; ++w)
            if (w < warp) x += s_total[0][w], y += s_total[1][w];
        if (2 * tid < radix) {
            s_first[2 * tid] = y, s_move[2 * tid] = x + before[0] - y;
            s_first[2 * tid + 1] = y + own[0], s_move[2 * tid + 1] = x + all[0] + before[1] - y - own[0];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < IPT; ++i) {
            const uint32_t d = key[i] >> shift & (radix - 1);
            s_local[s_first[d] + s_warp[warp * radix + d] + place[i]] = make_uint2(key[i], (uint32_t)pos[i]);
        }
        __syncthreads();
        const bool last = pass == passes - 1;
#pragma unroll
        for (int i = 0; i < IPT; ++i) {
            const uint32_t at = i * SORT_THREADS + tid;
            const uint2 p = s_local[at];
            const uint32_t to = at + s_move[p.x >> shift & (radix - 1)];
            if (last) {
                if (to < (uint32_t)n) skey[to] = p.x, spos[to] = (int32_t)p.y;
            } else {
                cluster.map_shared_rank(s_pair, to / SPAN)[to % SPAN] = p;
            }
        }
        cluster.sync();                  // every pair has arrived, every count been read
        if (!last)
#pragma unroll
            for (int i = 0; i < IPT; ++i) {
                const uint2 p = s_pair[warp * (32 * IPT) + i * 32 + lane];
                key[i] = p.x, pos[i] = (int32_t)p.y;
            }
    }
}

// ------------------------------------------------------------------ sums of runs
// A run of equal ids is cut into pieces of 32 positions from its start.  The sorted positions are cut into windows of 32, or of 8
// where those would be too few to fill the SMs, and a warp sums the pieces that start in its window (31 positions more
// than a window at most), 32 * E columns of them: rows are
// loaded SUM_UNROLL at a time, a run that is one piece is written at once, and a piece of a longer run
// is left in `part`: of the pieces that start at positions 32 w to 32 w + 31, row 2w + 1 for the first piece of a long run, row 2w
// for a later piece (there cannot be two of one kind).  k_embed_join adds a long run's
// pieces.  So the work is even whatever the ids: a hot id of 6000 rows is 188 pieces.
// Bound by memory: each row is read once, each result written once, and `part` is written and read for runs
// over 32 only, 1/8 (fp32 rows) or 1/4 (16-bit rows) of those runs' bytes in all.  65,536 x 2048 bf16 into 50,000 rows of
// fp32: 582 MB (and some of the zeros earlier, below) in 104 us, 5.6 TB/s (copies 6.7).
constexpr int PIECE = 32, SUM_WARPS = 8;

template <typename O, int E, bool ACC>
__device__ __forceinline__ void write_sum(O *at, const float (&sum)[E], const Pack<O, E> &old, float scale)
{
    Pack<O, E> y;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float v = __fmul_rn(scale, sum[e]);
        y.e[e] = from_float<O>(ACC ? __fadd_rn(to_float(old.e[e]), v) : v);
    }
    store_pack<O, E>(at, y);
}

// number of sorted keys below v, by the whole warp: 32 probes at a time
__device__ __forceinline__ int64_t keys_below(const uint32_t *key, int64_t n, uint32_t v)
{
    const int lane = threadIdx.x & 31;
    int64_t lo = 0, hi = n;              // the answer lies in [lo, hi]
#pragma unroll 1
    while (lo < hi) {
        const int64_t step = (hi - lo + 31) / 32, at = lo + lane * step;
        const int below = __popc(__ballot_sync(FULL, at < hi && key[at] < v));
        // probes 0 .. below - 1 are below v
        hi = min64(hi, lo + below * step);
        if (below) lo = lo + (below - 1) * step + 1;
    }
    return lo;
}

// zeros in the rows of 32 ids from v0 on that do not occur: every `parts`-th of them from the part-th on
template <typename O, int E>
__device__ __forceinline__ void zero_rows(const uint32_t *key, int64_t n, int64_t vocab, int64_t v0,
                                          int part, int parts, O *__restrict__ dtable, int64_t stride, int dim)
{
    const int lane = threadIdx.x & 31;
    const uint32_t first = (uint32_t)v0, end = (uint32_t)min64(vocab, v0 + 32);
    unsigned present = 0;
#pragma unroll 1
    for (int64_t at = keys_below(key, n, first); at < n;) {
        const uint32_t k = at + lane < n ? key[at + lane] : 0xffffffffu;
        present |= __reduce_or_sync(FULL, k < end ? 1u << (k - first) : 0u);
        const uint32_t last = __shfl_sync(FULL, k, 31);
        if (last >= end) break;
        // a run that fills the lanes is passed over by a search
        at = __shfl_sync(FULL, k, 0) == last ? keys_below(key, n, last + 1) : at + 32;
    }
    unsigned absent = ~present & (end - first == 32 ? FULL : (1u << (end - first)) - 1);
    Pack<O, E> zero;
#pragma unroll
    for (int e = 0; e < E; ++e) zero.e[e] = from_float<O>(0.0f);
#pragma unroll 1
    for (int i = 0; absent; ++i) {
        O *row = dtable + (v0 + __ffs(absent) - 1) * stride;
        absent &= absent - 1;
        if ((i & (parts - 1)) != part) continue;
#pragma unroll 1
        for (int j = lane * E; j < dim; j += 32 * E) store_pack<O, E>(row + j, zero);
    }
}

template <typename T, typename O, int E, bool ACC>
__global__ __launch_bounds__(SUM_WARPS * 32, ACC ? 2 : 4) void k_embed_sum(const uint32_t *key,
                                                              const int32_t *pos, int64_t n, int64_t vocab,
                                                              const T *dout, int64_t stride, int dim,
                                                              int tiles, int log_window, int64_t sum_blocks,
                                                              int64_t zero_first, int64_t zero_groups, int log_parts, float scale,
                                                              O *__restrict__ dtable, int64_t out_stride,
                                                              float *__restrict__ part, int *__restrict__ long_runs,
                                                              int4 *__restrict__ run_list)
{
    after_previous();
    constexpr int SUM_UNROLL = ACC ? 4 : 8;          // rows under way, with the rows they are added to
    const int lane = threadIdx.x & 31, size = 1 << log_window;
    // without ACC some of the blocks, spread among the others, write zeros in the rows of ids that do not occur
    const uint64_t zero_blocks = gridDim.x - sum_blocks, zeros_before = blockIdx.x * zero_blocks / gridDim.x;
    if (!ACC && (blockIdx.x + 1) * zero_blocks / gridDim.x != zeros_before) {
        const int64_t zero = zeros_before * SUM_WARPS + (threadIdx.x >> 5), group = zero_first + (zero >> log_parts);
        const int parts = 1 << log_parts;
        if (group < zero_groups)
            zero_rows<O, E>(key, n, vocab, group * 32, (int)(zero & (parts - 1)), parts, dtable, out_stride, dim);
        return;
    }
    const int64_t w = (blockIdx.x - zeros_before) * SUM_WARPS + (threadIdx.x >> 5);
    const int64_t window = w / tiles, p0 = window << log_window;
    if (p0 >= n) return;
    const int tile = (int)(w - window * tiles), col = tile * 32 * E + lane * E;
    const bool on = col < dim;
    // keys and rows of the window and behind it, 64 positions in all
    uint32_t k[2];
    int32_t row[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t i = p0 + h * 32 + lane;
        k[h] = i < n ? key[i] : 0xffffffffu;
        row[h] = i < n ? pos[i] : 0;
    }
    const uint32_t before = p0 > 0 ? key[p0 - 1] : 0xffffffffu;
    const uint32_t left0 = __shfl_up_sync(FULL, k[0], 1), left1 = __shfl_up_sync(FULL, k[1], 1);
    const uint32_t end0 = __shfl_sync(FULL, k[0], 31), first = __shfl_sync(FULL, k[0], 0);
    // positions (of 64) where a run starts; those behind the last id that counts make one of their own
    const uint64_t heads = (uint64_t)__ballot_sync(FULL, k[1] != (lane == 0 ? end0 : left1)) << 32 |
                           __ballot_sync(FULL, k[0] != (lane == 0 ? before : left0));
    const uint64_t counts = (uint64_t)__ballot_sync(FULL, k[1] < (uint32_t)vocab) << 32 | __ballot_sync(FULL, k[0] < (uint32_t)vocab);
    const int limit = __popcll(counts);  // sorted: the ids that count come first
    if (limit == 0) return;
    // pieces that start in the window: at its heads, and one of the run that comes in
    uint32_t starts = (uint32_t)heads & (uint32_t)counts & (0xffffffffu >> (32 - size));
    int later = -1;                      // where a later piece of a run starts
    if (!(heads & 1)) {
        const int64_t origin = keys_below(key, n, first);
        const int q = (int)(-(p0 - origin) & (PIECE - 1));
        if (q < size && (heads & ((2ull << q) - 1)) == 0 && q < limit) later = q, starts |= 1u << q;
    }
    if (starts == 0) return;
    const int s0 = __ffs(starts) - 1, last = 31 - __clz(starts);
    const uint64_t behind = heads >> last >> 1;
    const int run_end = behind ? last + __ffsll((long long)behind) : 64;
    const int end = min(min(last + PIECE, run_end), limit);
    float sum[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = 0.0f;
    int from = s0;                       // start of the current piece
    const int safe = on ? col : 0;       // lanes past the columns load what they do not use
    auto id_at = [&](int i) {
        const uint32_t a = __shfl_sync(FULL, k[0], i & 31), b = __shfl_sync(FULL, k[1], i & 31);
        return i < 32 ? a : b;
    };
#pragma unroll 1
    for (int i0 = s0; i0 < end; i0 += SUM_UNROLL) {
        Pack<T, E> x[SUM_UNROLL];
        Pack<O, E> old[ACC ? SUM_UNROLL : 1];
#pragma unroll
        for (int u = 0; u < SUM_UNROLL; ++u) {
            const int i = min(i0 + u, end - 1);
            const int32_t ra = __shfl_sync(FULL, row[0], i & 31), rb = __shfl_sync(FULL, row[1], i & 31);
            x[u] = load_pack<T, E>(dout + (i < 32 ? ra : rb) * stride + safe);
            if (ACC) old[u] = load_pack<O, E>(dtable + (int64_t)id_at(i) * out_stride + safe);
        }
#pragma unroll
        for (int u = 0; u < SUM_UNROLL; ++u) {
            const int i = i0 + u;
            if (i >= end) break;
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] = __fadd_rn(sum[e], to_float(x[u].e[e]));
            if (i + 1 == end || (heads >> (i + 1) & 1)) {
                // longer than a piece: the same id stands 32 positions behind the start, or it is a later piece
                const bool first_of_long = from != later && i + 1 == from + PIECE && p0 + from + PIECE < n &&
                                           (i + 1 < 64 ? !(heads >> (i + 1) & 1) : false);
                const uint32_t id = id_at(i);
                if (from == later || first_of_long) {
                    if (on) {
                        float *at = part + (2 * ((p0 + from) / PIECE) + (first_of_long ? 1 : 0)) * dim + col;
#pragma unroll
                        for (int e = 0; e < E; ++e) at[e] = sum[e];
                    }
                    if (first_of_long && tile == 0) {
                        const int64_t length = keys_below(key, n, id + 1) - (p0 + from);
                        if (lane == 0)
                            run_list[atomicAdd(long_runs, 1)] =
                                make_int4((int)(p0 + from), (int)((length + PIECE - 1) / PIECE), (int)id, 0);
                    }
                } else if (on) {
                    write_sum<O, E, ACC>(dtable + (int64_t)id * out_stride + col, sum, old[ACC ? u : 0], scale);
                }
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] = 0.0f;
                from = i + 1;
            }
        }
    }
}

// Runs over 32 positions: blocks take (run, 128 columns) in turn; a warp holds four columns a lane of every
// 8th piece, four loads under way; the warps' sums are added in order.  The order of a run's sum depends on its length alone.
constexpr int JOIN_COLS = 128, JOIN_WARPS = 8;

// JE: columns that one load brings (4, or 1 where the columns are no multiple of 4)
template <typename O, int JE, bool ACC>
__global__ __launch_bounds__(JOIN_WARPS * 32) void k_embed_join(int dim, int tiles, float scale, O *__restrict__ dtable,
                                                                int64_t out_stride, const float *part,
                                                                const int *long_runs,
                                                                const int4 *run_list)
{
    after_previous();
    __shared__ float s_sum[JOIN_WARPS][JOIN_COLS];
    const int set = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t items = (int64_t)*long_runs * tiles;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int4 run = run_list[item / tiles];            // start, pieces, id
        const int64_t window = run.x / PIECE;
        const int pieces = run.y, base = (int)(item % tiles) * JOIN_COLS, col0 = base + lane * 4;
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int b0 = set; b0 < pieces; b0 += 4 * JOIN_WARPS) {
            Pack<float, JE> x[4][4 / JE];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int b = min(b0 + u * JOIN_WARPS, pieces - 1);
                const float *at = part + (2 * (window + b) + (b == 0 ? 1 : 0)) * dim;
#pragma unroll
                for (int e = 0; e < 4; e += JE) x[u][e / JE] = load_pack<float, JE>(at + min(col0 + e, dim - JE));
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (b0 + u * JOIN_WARPS < pieces)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[e] = __fadd_rn(sum[e], x[u][e / JE].e[e % JE]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) s_sum[set][lane * 4 + e] = sum[e];
        __syncthreads();
        const int col = base + (int)threadIdx.x;
        if (threadIdx.x < JOIN_COLS && col < dim) {
            float total[1] = {0.0f};
            for (int i = 0; i < min(JOIN_WARPS, pieces); ++i) total[0] = __fadd_rn(total[0], s_sum[i][threadIdx.x]);
            O *at = dtable + (int64_t)run.z * out_stride + col;
            Pack<O, 1> old;
            if (ACC) old.e[0] = *at;
            write_sum<O, 1, ACC>(at, total, old, scale);
        }
        __syncthreads();
    }
}

}  // namespace

namespace pdb {

bool allow_smem(const void *kernel)
{
    // (kernel, device) pairs told already; beyond the table, told again at every call
    static std::mutex lock;
    static struct { const void *kernel; int device; } done[256];
    static int n_done = 0;
    int device = 0, most = 0;
    cudaGetDevice(&device);
    std::lock_guard<std::mutex> guard(lock);
    for (int i = 0; i < n_done; ++i)
        if (done[i].kernel == kernel && done[i].device == device) return true;
    cudaFuncAttributes at;
    if (cudaDeviceGetAttribute(&most, cudaDevAttrMaxSharedMemoryPerBlockOptin, device) != cudaSuccess ||
        cudaFuncGetAttributes(&at, kernel) != cudaSuccess ||
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most - (int)at.sharedSizeBytes) !=
            cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    if (n_done < 256) done[n_done++] = {kernel, device};
    return true;
}

}  // namespace pdb

extern "C" {

void pdb_tokens_free(pdb_tokens *t)
{
    if (!t) return;
    if (t->ev_use) cudaEventSynchronize(t->ev_use);
    release(t->arrays, own_stream());
    if (t->ev_use) cudaEventDestroy(t->ev_use);
    delete t;
}

int pdb_tokens_create(int64_t max_tokens, int64_t max_dim, pdb_tokens **out, void *stream)
{
    ApiScope scope("pdb_tokens_create", nullptr, nullptr, nullptr, nullptr, false);
    if (!out) return PDB_EINVAL;
    *out = nullptr;
    if (max_tokens < 0 || max_dim < 0) return PDB_EINVAL;
    if (max_tokens > INT32_MAX || max_dim > INT32_MAX / 2) return PDB_ETOOBIG;
    cudaStream_t s = (cudaStream_t)stream;
    pdb_tokens *t = new (std::nothrow) pdb_tokens();
    if (!t) return PDB_ENOMEM;
    const Launch l = launch_info();
    t->device = l.device;
    t->sms = l.sms;
    t->max_tokens = max_tokens;
    t->max_dim = max_dim;
    t->tries = WAIT_TRIES;
    int rc = cudaEventCreateWithFlags(&t->ev_use, cudaEventDisableTiming) == cudaSuccess ? PDB_OK : PDB_ECUDA;
    const size_t words = sizeof(uint32_t) * max_tokens, radix = max_tokens > SORT_MAX ? words : 0;   // of the radix sort only
    rc = rc ? rc : alloc_block(t->arrays, {{(void **)&t->status, 3 * sizeof(int)},
                                           {(void **)&t->key, radix},
                                           {(void **)&t->tkey, radix},
                                           {(void **)&t->tpos, radix},
                                           {(void **)&t->skey, words},
                                           {(void **)&t->spos, words},
                                           // two rows of columns in fp32 for each 32 positions
                                           {(void **)&t->part, sizeof(float) * 2 * ((max_tokens + PIECE - 1) / PIECE) * max_dim},
                                           {(void **)&t->run_list, sizeof(int4) * (max_tokens / (PIECE + 1))}}, s);
    rc = rc ? rc : fill_words(t->status, 0u, 3 * sizeof(int), s);
    if (rc != PDB_OK) {
        cudaGetLastError();
        cudaStreamSynchronize(s);
        pdb_tokens_free(t);
        return rc;
    }
    cudaEventRecord(t->ev_use, s);
    *out = t;
    return PDB_OK;
}

int pdb_tokens_status(const pdb_tokens *t, void *stream)
{
    if (!t) return PDB_EINVAL;
    if (const int rc = check_device(t)) return rc;
    int st = 0;
    if (read_words(&st, t->status, sizeof(int), (cudaStream_t)stream) != PDB_OK) return PDB_ECUDA;
    return st;
}

int pdb_tokens_set_wait_limit(pdb_tokens *t, int64_t tries)
{
    if (!t || tries < 0 || tries > (int64_t)WAIT_TRIES) return PDB_EINVAL;
    t->tries = (unsigned)tries;
    return PDB_OK;
}

int pdb_embed(pdb_tokens *t, const pdb_mat *table, const pdb_ids *ids, float scale, int64_t pad, const pdb_mat *out,
              void *stream)
{
    ApiScope scope("pdb_embed", nullptr, nullptr, nullptr, nullptr, false);
    if (!t) return PDB_EINVAL;
    int rc = check_mat(table);
    rc = rc ? rc : check_mat(out);
    rc = rc ? rc : check_ids(ids, out->rows);
    if (rc != PDB_OK) return rc;
    if (table->cols != out->cols || overlap(table, out)) return PDB_EINVAL;
    if (out->rows == 0 || out->cols == 0) return PDB_OK;
    if ((rc = check_device(t)) != PDB_OK) return rc;
    cudaStream_t s = (cudaStream_t)stream;
    TokensUse use{t, s};
    const auto run = [&](auto *a, auto *b, auto e) {
        using T = std::remove_pointer_t<decltype(a)>;
        using O = std::remove_pointer_t<decltype(b)>;
        constexpr int E = decltype(e)::value;
        const int dim = (int)out->cols, pieces = (dim + LOOKUP_UNROLL * 32 * E - 1) / (LOOKUP_UNROLL * 32 * E);
        const int64_t blocks = std::min<int64_t>((out->rows * pieces + 7) / 8, (int64_t)1 << 24);
        rc = launch(k_embed<T, O, E>, blocks, 256, 0, 1, s, (const T *)table->data, table->rows, stride_of(table),
                    ids_of(ids), out->rows, dim, pieces, scale, pad, (O *)out->data, stride_of(out), t->status);
    };
    with_type(table->type, [&](auto *a) {
        with_type(out->type, [&](auto *b) {
            // the widest moves that the columns' number and both matrices' alignment allow
            if (fits(table, 8) && fits(out, 8)) run(a, b, Num<8>());
            else if (fits(table, 4) && fits(out, 4)) run(a, b, Num<4>());
            else if (fits(table, 2) && fits(out, 2)) run(a, b, Num<2>());
            else run(a, b, Num<1>());
        });
    });
    return rc;
}

int pdb_embed_grad(pdb_tokens *t, const pdb_ids *ids, const pdb_mat *dout, float scale, int64_t pad, int accumulate,
                   const pdb_mat *dtable, void *stream)
{
    ApiScope scope("pdb_embed_grad", nullptr, nullptr, nullptr, nullptr, false);
    if (!t) return PDB_EINVAL;
    int rc = check_mat(dout);
    rc = rc ? rc : check_mat(dtable);
    rc = rc ? rc : check_ids(ids, dout->rows);
    if (rc != PDB_OK) return rc;
    if (dout->cols != dtable->cols || overlap(dout, dtable)) return PDB_EINVAL;
    if (dout->rows > t->max_tokens || dout->cols > t->max_dim || dtable->rows >= INT32_MAX) return PDB_ETOOBIG;
    const int64_t n = dout->rows, vocab = dtable->rows;
    const int dim = (int)dout->cols;
    if (vocab == 0 && n == 0) return PDB_OK;
    if ((rc = check_device(t)) != PDB_OK) return rc;
    cudaStream_t s = (cudaStream_t)stream;
    TokensUse use{t, s};
    // What the sort leaves idle writes zeros: about as many bytes as go to memory in its time (the 25 us of 65,536 ids: 148 us
    // -> 142 with 50,000 rows of 8 KB), none for the short sorts and rows that are not whole 16-byte pieces.
    Fill fill = {};
    const int64_t row_bytes = (int64_t)dim * type_bytes(dtable->type), step = stride_of(dtable) * type_bytes(dtable->type);
    if (!accumulate && n > RANK_MAX && n <= SORT_MAX && row_bytes > 0 && row_bytes % 16 == 0 && step % 16 == 0 &&
        (uintptr_t)dtable->data % 16 == 0) {
        const int64_t rows = (n < 16384 ? 24 << 20 : 96 << 20) / row_bytes;
        fill = Fill{(char *)dtable->data, std::min(rows, vocab) / 32 * 32, step, (int)(row_bytes / 16)};
    }
    const bool nothing = dim == 0 || vocab == 0;            // the ids are looked at all the same
    if (n > 0 && n <= RANK_MAX) {
        const size_t smem = sizeof(uint32_t) * ((n + 4 * RANK_SLICES - 1) / (4 * RANK_SLICES) * (4 * RANK_SLICES));
        rc = launch(k_embed_rank, (n + RANK_IDS - 1) / RANK_IDS, RANK_THREADS, smem, 1, s, ids_of(ids), (int)n, vocab, pad,
                    t->skey, t->spos, t->status + 2, t->status);
    } else if (n > 0 && n <= SORT_MAX) {
        // blocks of 1024 to 8192 pairs, as many of a cluster as it takes
        const int b = bits_for(vocab), passes = (b + SORT_BITS - 1) / SORT_BITS, bits = std::max(5, (b + passes - 1) / passes);
        const auto sort = [&](auto i) {
            constexpr int IPT = decltype(i)::value;
            int blocks = 1;
            while (blocks * SORT_THREADS * IPT < n) blocks *= 2;
            Shape shape = {};
            shape.blocks = blocks, shape.threads = SORT_THREADS, shape.smem = sort_smem(IPT);
            shape.clusters = fill.rows > 0 ? t->sms / blocks : 1;
            return launch_rows(k_embed_sort<IPT>, shape, s, ids_of(ids), (int)n, vocab, pad, passes, bits, t->skey, t->spos,
                               t->status + 2, fill, t->status);
        };
        constexpr int UNIT = SORT_THREADS * SORT_CLUSTER;
        rc = n <= 2 * UNIT ? sort(Num<2>()) : n <= 4 * UNIT ? sort(Num<4>()) : n <= 8 * UNIT ? sort(Num<8>()) : sort(Num<16>());
    } else if (n > 0) {
        rc = launch(k_embed_keys, (n + 255) / 256, 256, 0, 1, s, ids_of(ids), n, vocab, pad, t->key, t->status + 2, t->status);
        if (!nothing && rc == PDB_OK)
            rc = radix_sort(t->key, nullptr, t->skey, t->spos, t->tkey, t->tpos, n, bits_for(vocab), t->status + 1, s);
    }
    if (rc != PDB_OK || nothing) return rc;
    const auto run = [&](auto *a, auto *b, auto e) {
        using T = std::remove_pointer_t<decltype(a)>;
        using O = std::remove_pointer_t<decltype(b)>;
        constexpr int E = decltype(e)::value;
        // windows of 8 below 16 warps an SM (8191 x 320: 512 warps otherwise)
        const int tiles = (dim + 32 * E - 1) / (32 * E);
        const int log_window = (n + PIECE - 1) / PIECE * tiles < (int64_t)t->sms * 16 ? 3 : 5;
        const int64_t windows = (n + (1 << log_window) - 1) >> log_window;
        const int64_t sum_blocks = (windows * tiles + SUM_WARPS - 1) / SUM_WARPS;
        const int64_t zero_first = fill.rows / 32, zero_groups = accumulate ? 0 : (vocab + 31) / 32;
        // A warp zeroes the absent ones of 32 rows, or a part of them (8 KB at least) up to 32 warps an SM: 14 x 880 fp32
        // into 9045 rows 17 us -> 7, 65,536 x 2048 bf16 into 50,000 fp32 rows 156 -> 143 (with parts of 2 KB 500 x 256
        // into 10,000 rows take 10.2 us instead of 9.4: each part looks the keys up again).
        int log_parts = 0;
        while (log_parts < 5 && (zero_groups - zero_first) << log_parts < (int64_t)t->sms * 32 &&
               32 * row_bytes >> log_parts >= 16384)
            ++log_parts;
        const int64_t zero_warps = (zero_groups - zero_first) << log_parts;
        const int64_t blocks = sum_blocks + (accumulate ? 0 : (zero_warps + SUM_WARPS - 1) / SUM_WARPS);
        if (blocks > 0) {
            const auto kernel = accumulate ? k_embed_sum<T, O, E, true> : k_embed_sum<T, O, E, false>;
            rc = launch(kernel, blocks, SUM_WARPS * 32, 0, 1, s, t->skey, t->spos, n, vocab, (const T *)dout->data,
                        stride_of(dout), dim, tiles, log_window, sum_blocks, zero_first, zero_groups, log_parts, scale,
                        (O *)dtable->data, stride_of(dtable), t->part, t->status + 2, t->run_list);
        }
        if (n > PIECE && rc == PDB_OK) {                 // else no run is longer than a piece
            const bool four = dim % 4 == 0;
            const auto kernel = accumulate ? (four ? k_embed_join<O, 4, true> : k_embed_join<O, 1, true>)
                                           : (four ? k_embed_join<O, 4, false> : k_embed_join<O, 1, false>);
            const int tiles = (dim + JOIN_COLS - 1) / JOIN_COLS;
            const int64_t most = n / (PIECE + 1) * tiles;
            rc = launch(kernel, std::max<int64_t>(1, std::min<int64_t>(most, t->sms * 8)), JOIN_WARPS * 32, 0, 1, s, dim, tiles,
                        scale, (O *)dtable->data, stride_of(dtable), t->part, t->status + 2, t->run_list);
        }
    };
    with_type(dout->type, [&](auto *a) {
        with_type(dtable->type, [&](auto *b) {
            constexpr int E = 16 / sizeof(*a);
            if (fits(dout, E) && fits(dtable, E)) run(a, b, Num<E>());
            else if (fits(dout, E / 2) && fits(dtable, E / 2)) run(a, b, Num<E / 2>());
            else run(a, b, Num<1>());
        });
    });
    return rc;
}

}  // extern "C"
