// Tokens to experts and back (pdb_route, pdb_route_rows, pdb_route_join,
// pdb_route_join_grad).
//
// n tokens have k slots each; slot f = i k + j of token i names an expert e_f, or none.  The experts' rows lie one expert after the
// other, an expert's slots in ascending order:
//   place_f = first(e_f) + |{f' < f : e_f' = e_f}|,   first(e) = |{f : e_f < e}|, or e * capacity
// a stable counting sort by expert.  With it rows go there, come back weighted and summed, and their gradients the other way.
#include <algorithm>

#include "pack.cuh"
#include "rows.cuh"

using namespace pdb;
namespace cg = cooperative_groups;

namespace {

// ------------------------------------------------------------------ places
constexpr int MAX_EXPERTS = 4096, MAX_ROUTE_SLOTS = 64, ROUTE_THREADS = 512, ROUTE_WARPS = ROUTE_THREADS / 32;

struct Slots {
    Ids ids;
    uint32_t n, k;                      // slots in all, of a token
    int experts;
};

// the expert of slot f, or `experts` for none
__device__ __forceinline__ int expert_of(const Slots &s, int2 raw, int *status)
{
    const int64_t e = id_of(s.ids, raw);
    if (e >= s.experts) set_status(status, PDB_ERANGE);
    return e >= 0 && e < s.experts ? (int)e : s.experts;
}
__device__ __forceinline__ int2 fetch_slot(const Slots &s, uint32_t f)
{
    const uint32_t i = f / s.k;
    return fetch_id(s.ids, i, (int)(f - i * s.k));
}

// More than a cluster's slots: how often each expert occurs among a block's slots, for the places' launch, whose blocks each add up the
// counts of all.  131,072 slots, 64 experts: 5.3 and 8.4 us, chains of latencies (ids, counts, barriers).
template <int IPT>
__global__ __launch_bounds__(ROUTE_THREADS) void k_route_count(Slots s, uint32_t *__restrict__ counts, int *status)
{
    after_previous();
    let_next_start();
    extern __shared__ uint32_t s_count[];
    for (int e = threadIdx.x; e < s.experts; e += ROUTE_THREADS) s_count[e] = 0;
    const uint32_t f0 = blockIdx.x * (uint32_t)(ROUTE_THREADS * IPT);
    int2 raw[IPT];
#pragma unroll
    for (int i = 0; i < IPT; ++i) {
        const uint32_t f = f0 + i * ROUTE_THREADS + threadIdx.x;
        raw[i] = f < s.n ? fetch_slot(s, f) : int2{-1, -1};
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < IPT; ++i) {
        const int e = expert_of(s, raw[i], status);
        // one addition for the lanes of one expert
        const unsigned peers = __match_any_sync(FULL, e);
        if (e < s.experts && (peers & lanemask_lt()) == 0) atomicAdd(&s_count[e], __popc(peers));
    }
    __syncthreads();
    for (int e = threadIdx.x; e < s.experts; e += ROUTE_THREADS) counts[(int64_t)blockIdx.x * s.experts + e] = s_count[e];
}

// A block's slots, warp after warp, 32 at a time: a lane's rank is the lower lanes of its expert, its warp's slots before
// them, the lower warps', and the lower blocks'.  Up to CLUSTER_SLOTS slots the blocks are a cluster and take one another's counts from
// shared memory (ONE: a launch alone; 8198 slots, 32 experts: 9.7 us instead of 14.3 in two).
constexpr int CLUSTER_SLOTS = 65536;

template <int IPT, bool ONE>
__global__ __launch_bounds__(ROUTE_THREADS) void k_route_place(Slots s, const uint32_t *counts, int64_t capacity,
                                                               int32_t *__restrict__ place, int32_t *__restrict__ source,
                                                               int32_t *__restrict__ ends, int *status)
{
    after_previous();
    let_next_start();
    extern __shared__ uint32_t s_first[];                                       // [experts] of all and of lower blocks, then
    uint32_t *s_total = s_first + s.experts;                                    // [experts] slots of the expert in all
    uint32_t *s_block = s_total + s.experts;                                    // [experts] the block's (ONE)
    uint16_t *s_warp = reinterpret_cast<uint16_t *>(s_block + (ONE ? s.experts : 0));      // [warp][experts] the expert's slots by warp
    __shared__ uint32_t s_sum[ROUTE_WARPS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, experts = s.experts;
    const uint32_t f0 = blockIdx.x * (uint32_t)(ROUTE_THREADS * IPT) + warp * (32 * IPT) + lane;
    int2 raw[IPT];
#pragma unroll
    for (int i = 0; i < IPT; ++i) raw[i] = f0 + i * 32 < s.n ? fetch_slot(s, f0 + i * 32) : int2{-1, -1};
    for (int e = tid; e < experts; e += ROUTE_THREADS) s_first[e] = s_total[e] = 0;
    for (int e = tid; e < ROUTE_WARPS * experts; e += ROUTE_THREADS) s_warp[e] = 0;
    __syncthreads();
    // the blocks' counts, every `sets`-th of them by one thread
    if (!ONE) {
        const int sets = max(1, ROUTE_THREADS / experts);
        for (int x = tid; x < sets * experts; x += ROUTE_THREADS) {
            const int set = x / experts, e = x - set * experts;
            uint32_t all = 0, before = 0;
#pragma unroll 8
            for (int b = set; b < (int)gridDim.x; b += sets) {
                const uint32_t c = counts[(int64_t)b * experts + e];
                all += c;
                before += b < (int)blockIdx.x ? c : 0;
            }
            atomicAdd(&s_total[e], all);
            atomicAdd(&s_first[e], before);
        }
    }
    int expert[IPT], rank[IPT];
    uint16_t *own = s_warp + warp * experts;
#pragma unroll
    for (int i = 0; i < IPT; ++i) {
        expert[i] = expert_of(s, raw[i], status);
        const unsigned peers = __match_any_sync(FULL, expert[i]);
        const bool there = expert[i] < experts;
        const int c = there ? own[expert[i]] : 0;
        __syncwarp();
        rank[i] = c + __popc(peers & lanemask_lt());
        if (there && (peers & lanemask_lt()) == 0) own[expert[i]] = (uint16_t)(c + __popc(peers));
        __syncwarp();
    }
    __syncthreads();
    // experts tid * per ..: the warps' counts become places, the totals are summed up over the experts
    const int per = (experts + ROUTE_THREADS - 1) / ROUTE_THREADS, e0 = min(experts, tid * per), e1 = min(experts, e0 + per);
    for (int e = e0; e < e1; ++e) {
        uint32_t sum = 0;
#pragma unroll
        for (int w = 0; w < ROUTE_WARPS; ++w) {
            const uint32_t c = s_warp[w * experts + e];
            s_warp[w * experts + e] = (uint16_t)sum;
            sum += c;
        }
        if (ONE) s_block[e] = sum;
    }
    uint32_t mine = 0;
    if (ONE) {
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        for (int e = e0; e < e1; ++e) {
            uint32_t all = 0, before = 0;
            for (int b = 0; b < (int)gridDim.x; ++b) {
                const uint32_t c = cluster.map_shared_rank(s_block, b)[e];
                all += c;
                before += b < (int)blockIdx.x ? c : 0;
            }
            s_total[e] = all, s_first[e] = before;
        }
    }
    for (int e = e0; e < e1; ++e) mine += s_total[e];
    uint32_t up = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const uint32_t u = __shfl_up_sync(FULL, up, off);
        if (lane >= off) up += u;
    }
    if (lane == 31) s_sum[warp] = up;
    __syncthreads();
    up -= mine;
    for (int w = 0; w < warp; ++w) up += s_sum[w];
    for (int e = e0; e < e1; ++e) {
        const uint32_t total = s_total[e];
        const uint32_t first = capacity ? (uint32_t)(e * capacity) : up;
        const uint32_t end = first + (capacity ? (uint32_t)min64(total, capacity) : total);
        if (blockIdx.x == 0) ends[e] = (int32_t)end;
        s_total[e] = end;
        s_first[e] += first;
        up += total;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < IPT; ++i) {
        const uint32_t f = f0 + i * 32;
        if (f >= s.n) break;
        int32_t at = -1;
        if (expert[i] < experts) {
            const uint32_t p = s_first[expert[i]] + own[expert[i]] + rank[i];
            if (p < s_total[expert[i]]) at = (int32_t)p;          // with a capacity, slots behind it have no row
        }
        place[f] = at;
        if (at >= 0) source[at] = (int32_t)f;
    }
    // rows that no slot takes
    const int64_t rows = capacity ? experts * capacity : (int64_t)s.n;
    for (int64_t r = (int64_t)blockIdx.x * ROUTE_THREADS + tid; r < rows; r += (int64_t)gridDim.x * ROUTE_THREADS)
        if (r >= s_total[capacity ? (int)(r / capacity) : experts - 1]) source[r] = -1;
    if (ONE) cg::this_cluster().sync();              // the others have read this block's counts
}

inline size_t place_smem(int experts, bool one) { return (size_t)experts * ((one ? 12 : 8) + 2 * ROUTE_WARPS); }

// w / pieces
__device__ __forceinline__ int64_t row_of(int64_t w, int pieces)
{
    return w <= UINT32_MAX ? (int64_t)((uint32_t)w / (uint32_t)pieces) : w / pieces;
}

// ------------------------------------------------------------------ rows there
// zeros in the rows of `rows` (ZERO_ROWS of them from r0 on) that no slot takes, by a warp: few, since a warp that finds all of its
// rows unused is the launch's last (9600 rows of 1001 fp32 for 8198 slots: 12 us, with 8 to a warp 16)
constexpr int ZERO_ROWS = 2;

template <typename O, int E>
__device__ __forceinline__ void zero_unused(const int32_t *source, int64_t r0, int64_t rows, int dim, O *out, int64_t stride)
{
    const int lane = threadIdx.x & 31;
    unsigned unused = __ballot_sync(FULL, lane < ZERO_ROWS && r0 + lane < rows && source[r0 + lane] < 0);
    Pack<O, E> zero;
#pragma unroll
    for (int e = 0; e < E; ++e) zero.e[e] = from_float<O>(0.0f);
    for (; unused; unused &= unused - 1) {
        O *row = out + (r0 + __ffs(unused) - 1) * stride;
        for (int j = lane * E; j < dim; j += 32 * E) store_pack<O, E>(row + j, zero);
    }
}

// A warp moves one piece of ROWS_UNROLL * 32 packs of a token's row, read once, to the rows of its slots; the warps behind
// those write zeros where no slot is.  Bound by memory: 16,384 rows of 2048 bf16 to 8 places each 96 us, 605 MB at 6.3 TB/s (by
// place, each token's row would be read 8 times).  Rows that start at any 4 bytes are moved element by element, 4099 x 1001 fp32 into 9600 rows 12 us, 55
// MB at 4.6 TB/s.
template <int E>
constexpr int ROWS_UNROLL = E > 1 ? 4 : 16;

template <typename T, typename O, int E>
__global__ __launch_bounds__(256) void k_route_rows(const T *x, int64_t stride, int64_t n, int k, int dim, int pieces,
                                                    const int32_t *place, const int32_t *source, int64_t rows,
                                                    O *__restrict__ out, int64_t out_stride, int *status)
{
    after_previous();
    const int lane = threadIdx.x & 31;
    const int64_t copies = n * pieces, w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (w >= copies) {
        zero_unused<O, E>(source, (w - copies) * ZERO_ROWS, rows, dim, out, out_stride);
        return;
    }
    const int64_t i = row_of(w, pieces);
    const int piece = (int)(w - i * pieces), j0 = (piece * ROWS_UNROLL<E> * 32 + lane) * E;
    const T *from = x + i * stride;
    int32_t mine = lane < k ? place[i * k + lane] : -1;          // on its way beside the row
    Pack<T, E> v[ROWS_UNROLL<E>];
#pragma unroll
    for (int u = 0; u < ROWS_UNROLL<E>; ++u)
        if (j0 + u * 32 * E < dim) v[u] = load_pack<T, E>(from + j0 + u * 32 * E);
    Pack<O, E> y[ROWS_UNROLL<E>];
#pragma unroll
    for (int u = 0; u < ROWS_UNROLL<E>; ++u) {
        float f[E];
        to_floats(v[u], f);
        y[u] = of_floats<O>(f);
    }
    for (int s0 = 0; s0 < k; s0 += 32) {
        if (s0) mine = s0 + lane < k ? place[i * k + s0 + lane] : -1;
        if (mine >= rows) set_status(status, PDB_ERANGE);
        unsigned there = __ballot_sync(FULL, mine >= 0 && mine < rows);
        for (; there; there &= there - 1) {
            O *to = out + (int64_t)__shfl_sync(FULL, mine, __ffs(there) - 1) * out_stride;
#pragma unroll
            for (int u = 0; u < ROWS_UNROLL<E>; ++u)
                if (j0 + u * 32 * E < dim) store_pack<O, E>(to + j0 + u * 32 * E, y[u]);
        }
    }
}

// ------------------------------------------------------------------ and back
// a lane's slot: its row (-1: none), its weight
struct Slot {
    int32_t at;
    float weight;
};
__device__ __forceinline__ Slot load_slot(const int32_t *place, const float *weight, int64_t i, int k, int j, bool on)
{
    Slot s = {-1, 1.0f};
    if (on && j < k) {
        s.at = place[i * k + j];
        if (weight) s.weight = weight[i * k + j];
    }
    return s;
}
// the lanes' slots that have a row
__device__ __forceinline__ unsigned slots_there(const Slot &s, int64_t rows, int *status)
{
    if (s.at >= rows) set_status(status, PDB_ERANGE);
    return __ballot_sync(FULL, s.at >= 0 && s.at < rows);
}

// A warp sums one piece of JOIN_UNROLL * 32 packs of a token's row over its slots in ascending order, JOIN_SLOTS rows under way
// at once, and takes the next piece; that one's first 32 places are on their way meanwhile.  Bound by memory: 8192 tokens of 4 slots,
// 4096 bf16, 48 us, 336 MB at 7.0 TB/s (a warp a piece, 106 registers a thread: 91 us; pieces of half the size: 65).
template <int E>
constexpr int JOIN_UNROLL = E > 2 ? 2 : 4;
constexpr int JOIN_SLOTS = 4, JOIN_BLOCKS = 3;

template <typename T, typename O, int E>
__global__ __launch_bounds__(256, JOIN_BLOCKS) void k_route_join(const T *in, int64_t stride, int64_t rows, int k,
                                                                 const int32_t *place, const float *weight, int64_t n, int dim,
                                                                 int pieces, O *__restrict__ out, int64_t out_stride, int *status)
{
    after_previous();
    constexpr int U = JOIN_UNROLL<E>;
    const int lane = threadIdx.x & 31;
    const int64_t items = n * pieces, step = (int64_t)gridDim.x * 8;
    int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), i = row_of(w, pieces);
    Slot ahead = load_slot(place, weight, i, k, lane, w < items);
    for (; w < items; w += step) {
        const int64_t token = i;
        const int j0 = ((int)(w - i * pieces) * U * 32 + lane) * E;
        Slot slot = ahead;
        i = row_of(w + step, pieces);
        ahead = load_slot(place, weight, i, k, lane, w + step < items);
        float sum[U][E];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) sum[u][e] = 0.0f;
        for (int s0 = 0; s0 < k; s0 += 32) {
            if (s0) slot = load_slot(place, weight, token, k, s0 + lane, true);
            unsigned there = slots_there(slot, rows, status);
            while (there) {
                Pack<T, E> v[JOIN_SLOTS][U];
                float ws[JOIN_SLOTS];
                const int batch = min(JOIN_SLOTS, __popc(there));
#pragma unroll
                for (int s = 0; s < JOIN_SLOTS; ++s) {
                    const int at = there ? __ffs(there) - 1 : 0;
                    ws[s] = __shfl_sync(FULL, slot.weight, at);
                    const T *from = in + (int64_t)__shfl_sync(FULL, slot.at, at) * stride;
                    if (s < batch)
#pragma unroll
                        for (int u = 0; u < U; ++u)
                            if (j0 + u * 32 * E < dim) v[s][u] = load_pack<T, E>(from + j0 + u * 32 * E);
                    there &= there - 1;
                }
#pragma unroll
                for (int s = 0; s < JOIN_SLOTS; ++s)
                    if (s < batch)
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            float f[E];
                            to_floats(v[s][u], f);
#pragma unroll
                            for (int e = 0; e < E; ++e) sum[u][e] = __fmaf_rn(ws[s], f[e], sum[u][e]);
                        }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + u * 32 * E;
            if (j >= dim) break;
            store_pack<O, E>(out + token * out_stride + j, of_floats<O>(sum[u]));
        }
    }
}

// Gradients of the join: drows[p_j] = w_j dy, dw_j = <dy, rows[p_j]>.  `team` warps of a block (a power of two) have a token, whose columns
// they take in turn: each holds its packs of dy and goes over the slots, GRAD_SLOTS rows under way at once; the dot products are summed over
// the lanes, then over the team's warps in order.  The next token's places, weights and first packs of dy are on their way meanwhile.
// At the end the warps write zeros in rows that no slot takes.  Bound by memory: 8192 tokens of 4 slots, 4096 bf16, 107 us, 604 MB at 5.6 TB/s
// (half of it written; a block a token: 186 us; packs of 1 instead of 4 of a lane: 150).
constexpr int GRAD_UNROLL = 4, GRAD_WARPS = 8, GRAD_SLOTS = 4, GRAD_BLOCKS = 2;

template <typename T, typename D, int E>
__global__ __launch_bounds__(GRAD_WARPS * 32, GRAD_BLOCKS) void k_route_join_grad(const T *in, int64_t stride, int64_t rows, int k,
                                                                                  const int32_t *place, const int32_t *source,
                                                                                  const float *weight, const D *dy, int64_t dy_stride,
                                                                                  int64_t n, int dim, int team, T *drows,
                                                                                  int64_t out_stride, float *__restrict__ dweight,
                                                                                  int *status)
{
    after_previous();
    constexpr int U = GRAD_UNROLL, SPAN = U * 32 * E;
    __shared__ float s_dot[2][GRAD_WARPS][MAX_ROUTE_SLOTS];     // of two tokens in turn
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per = GRAD_WARPS / team, part = warp & (team - 1);
    const int64_t step = (int64_t)gridDim.x * per;
    int64_t first = (int64_t)blockIdx.x * per;
    const auto load_dy = [&](int64_t i, int c0, Pack<D, E> (&d)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i < n && c0 + u * 32 * E + lane * E < dim) d[u] = load_pack<D, E>(dy + i * dy_stride + c0 + u * 32 * E + lane * E);
    };
    Slot ahead = load_slot(place, weight, first + warp / team, k, lane, first + warp / team < n);
    Pack<D, E> d_ahead[U];
    load_dy(first + warp / team, part * SPAN, d_ahead);
    for (int turn = 0; first < n; first += step, turn ^= 1) {
        const int64_t i = first + warp / team;
        const Slot slot0 = ahead;
        Pack<D, E> d[U];
#pragma unroll
        for (int u = 0; u < U; ++u) d[u] = d_ahead[u];
        ahead = load_slot(place, weight, i + step, k, lane, i + step < n);
        load_dy(i + step, part * SPAN, d_ahead);
        float *dots = s_dot[turn][warp];
        if (dweight)
            for (int j = lane; j < k; j += 32) dots[j] = 0.0f;
        __syncwarp();
        if (i < n)
            for (int c0 = part * SPAN; c0 < dim; c0 += team * SPAN) {
                const int j0 = c0 + lane * E;
                if (c0 != part * SPAN) load_dy(i, c0, d);
                for (int s0 = 0; s0 < k; s0 += 32) {
                    const Slot slot = s0 ? load_slot(place, weight, i, k, s0 + lane, true) : slot0;
                    unsigned left = slots_there(slot, rows, status);
                    while (left) {
                        Pack<T, E> v[GRAD_SLOTS][U];
                        int which[GRAD_SLOTS];
                        int64_t row[GRAD_SLOTS];
                        const int batch = min(GRAD_SLOTS, __popc(left));
#pragma unroll
                        for (int s = 0; s < GRAD_SLOTS; ++s) {
                            which[s] = left ? __ffs(left) - 1 : 0;
                            left &= left - 1;
                            row[s] = __shfl_sync(FULL, slot.at, which[s]);
                            if (dweight && s < batch)
#pragma unroll
                                for (int u = 0; u < U; ++u)
                                    if (j0 + u * 32 * E < dim) v[s][u] = load_pack<T, E>(in + row[s] * stride + j0 + u * 32 * E);
                        }
                        // drows may be the rows' own memory: what is loaded is loaded before anything is stored there
                        asm volatile("" ::: "memory");
                        float dot[GRAD_SLOTS];
#pragma unroll
                        for (int s = 0; s < GRAD_SLOTS; ++s) {
                            dot[s] = 0.0f;
                            const float ws = __shfl_sync(FULL, slot.weight, which[s]);
                            if (s >= batch) continue;
#pragma unroll
                            for (int u = 0; u < U; ++u) {
                                const int j = j0 + u * 32 * E;
                                if (j >= dim) break;
                                float g[E], f[E];
                                to_floats(d[u], g);
                                if (dweight) {
                                    to_floats(v[s][u], f);
#pragma unroll
                                    for (int e = 0; e < E; ++e) dot[s] = __fmaf_rn(g[e], f[e], dot[s]);
                                }
#pragma unroll
                                for (int e = 0; e < E; ++e) g[e] = __fmul_rn(ws, g[e]);
                                store_pack<T, E>(drows + row[s] * out_stride + j, of_floats<T>(g));
                            }
                        }
                        if (dweight) {
                            // lanes of one half keep half of the slots' sums, then a quarter: lane 8 s has slot s
                            static_assert(GRAD_SLOTS == 4, "two halvings");
                            const bool high = lane & 16, odd = lane & 8;
                            float a = high ? dot[2] : dot[0], b = high ? dot[3] : dot[1];
                            a = __fadd_rn(a, __shfl_xor_sync(FULL, high ? dot[0] : dot[2], 16));
                            b = __fadd_rn(b, __shfl_xor_sync(FULL, high ? dot[1] : dot[3], 16));
                            float x = __fadd_rn(odd ? b : a, __shfl_xor_sync(FULL, odd ? a : b, 8));
#pragma unroll
                            for (int off = 4; off >= 1; off >>= 1) x = __fadd_rn(x, __shfl_xor_sync(FULL, x, off));
                            const int s = lane >> 3, at = s0 + (s == 0 ? which[0] : s == 1 ? which[1] : s == 2 ? which[2] : which[3]);
                            if ((lane & 7) == 0 && s < batch) dots[at] = __fadd_rn(dots[at], x);
                            __syncwarp();
                        }
                    }
                }
            }
        if (!dweight) continue;
        __syncthreads();                 // (the next token's sums go to the other half)
        for (int x = threadIdx.x; x < per * k; x += GRAD_WARPS * 32) {
            const int who = x / k, j = x - who * k;
            if (first + who >= n) break;
            float sum = s_dot[turn][who * team][j];
            for (int p = 1; p < team; ++p) sum = __fadd_rn(sum, s_dot[turn][who * team + p][j]);
            dweight[(first + who) * k + j] = sum;
        }
    }
    if (dim > 0)
        for (int64_t r0 = ((int64_t)blockIdx.x * GRAD_WARPS + warp) * ZERO_ROWS; r0 < rows; r0 += (int64_t)gridDim.x * GRAD_WARPS * ZERO_ROWS)
            zero_unused<T, E>(source, r0, rows, dim, drows, out_stride);
}

// n tokens of k slots each and their places, or PDB_EINVAL
int check_places(int64_t n, int64_t k, const int32_t *place)
{
    if (k < 1) return PDB_EINVAL;
    if (k > MAX_ROUTE_SLOTS) return PDB_ETOOBIG;
    if (n > 0 && (!place || (uintptr_t)place % 4 != 0)) return PDB_EINVAL;
    return n * k > INT32_MAX ? PDB_ETOOBIG : PDB_OK;
}
int check_words(const void *p, int64_t n) { return n > 0 && (!p || (uintptr_t)p % 4 != 0) ? PDB_EINVAL : PDB_OK; }

int64_t zero_warps(int64_t rows, int dim) { return dim > 0 ? (rows + ZERO_ROWS - 1) / ZERO_ROWS : 0; }

}  // namespace

extern "C" {

int pdb_route(pdb_tokens *t, const pdb_ids *ids, int64_t k, int64_t n_experts, int64_t capacity, int32_t *place,
              int32_t *source, int32_t *ends, void *stream)
{
    ApiScope scope("pdb_route", nullptr, nullptr, nullptr, nullptr, false);
    if (!t || !ids || k < 1 || n_experts < 1 || capacity < 0 || ids->n < 0 || ids->n % k != 0) return PDB_EINVAL;
    const int64_t n = ids->n / k;
    if (k > MAX_ROUTE_SLOTS || n_experts > MAX_EXPERTS || ids->n > INT32_MAX || capacity > INT32_MAX / n_experts)
        return PDB_ETOOBIG;
    const int64_t rows = capacity ? capacity * n_experts : ids->n;
    int rc = check_ids(ids, n, k);
    rc = rc ? rc : check_words(place, ids->n);
    rc = rc ? rc : check_words(source, rows);
    rc = rc ? rc : check_words(ends, n_experts);
    if (rc != PDB_OK) return rc;
    if (ids->n > t->max_tokens) return PDB_ETOOBIG;
    if ((rc = check_device(t)) != PDB_OK) return rc;
    cudaStream_t s = (cudaStream_t)stream;
    TokensUse use{t, s};
    const Slots slots{{ids->data, n > 1 ? ids->stride : 0, ids->wide}, (uint32_t)ids->n, (uint32_t)k, (int)n_experts};
    const auto run = [&](auto ipt, auto one) {
        constexpr int IPT = decltype(ipt)::value;
        constexpr bool ONE = decltype(one)::value;
        int64_t blocks = std::max<int64_t>(1, (ids->n + ROUTE_THREADS * IPT - 1) / (ROUTE_THREADS * IPT));
        int got = PDB_OK;
        if (ONE) {
            int cluster = 1;
            while (cluster < blocks) cluster *= 2;
            blocks = cluster;
        } else {
            // the blocks' counts: no more words than slots, since blocks * experts <= slots above CLUSTER_SLOTS
            got = launch(k_route_count<IPT>, blocks, ROUTE_THREADS, sizeof(uint32_t) * n_experts, 1, s, slots, t->skey, t->status);
            if (got != PDB_OK) return got;
        }
        const auto kernel = k_route_place<IPT, ONE>;
        if (!allow_smem((const void *)kernel)) return (int)PDB_ECUDA;
        return launch(kernel, blocks, ROUTE_THREADS, place_smem((int)n_experts, ONE), ONE ? (int)blocks : 1, s, slots, t->skey, capacity,
                      place, source, ends, t->status);
    };
    static_assert(CLUSTER_SLOTS == ROUTE_THREADS * 16 * MAX_CLUSTER, "sixteen slots a thread");
    // blocks of 2048 slots while there are few of them: each adds up the counts of all
    if (ids->n <= ROUTE_THREADS * 4 * MAX_CLUSTER) return run(Num<4>(), Num<1>());
    if (ids->n <= CLUSTER_SLOTS) return run(Num<16>(), Num<1>());
    return n_experts <= 1024 && ids->n <= 2048 * (int64_t)t->sms ? run(Num<4>(), Num<0>()) : run(Num<16>(), Num<0>());
}

int pdb_route_rows(pdb_tokens *t, const pdb_mat *x, const int32_t *place, int64_t k, const int32_t *source,
                   const pdb_mat *rows, void *stream)
{
    ApiScope scope("pdb_route_rows", nullptr, nullptr, nullptr, nullptr, false);
    if (!t) return PDB_EINVAL;
    int rc = check_mat(x);
    rc = rc ? rc : check_mat(rows);
    rc = rc ? rc : check_places(x->rows, k, place);
    rc = rc ? rc : check_words(source, rows->rows);
    if (rc != PDB_OK) return rc;
    if (x->cols != rows->cols || overlap(x, rows)) return PDB_EINVAL;
    const int dim = (int)x->cols;
    if (dim == 0 || rows->rows == 0) return PDB_OK;
    if ((rc = check_device(t)) != PDB_OK) return rc;
    cudaStream_t s = (cudaStream_t)stream;
    TokensUse use{t, s};
    const auto run = [&](auto *a, auto *b, auto e) {
        using T = std::remove_pointer_t<decltype(a)>;
        using O = std::remove_pointer_t<decltype(b)>;
        constexpr int E = decltype(e)::value;
        const int pieces = (dim + ROWS_UNROLL<E> * 32 * E - 1) / (ROWS_UNROLL<E> * 32 * E);
        const int64_t blocks = (x->rows * pieces + zero_warps(rows->rows, dim) + 7) / 8;
        if (blocks > INT32_MAX) return (int)PDB_ETOOBIG;
        return launch(k_route_rows<T, O, E>, blocks, 256, 0, 1, s, (const T *)x->data, stride_of(x), x->rows, (int)k, dim, pieces,
                      place, source, rows->rows, (O *)rows->data, stride_of(rows), t->status);
    };
    return with_type(x->type, [&](auto *a) {
        return with_type(rows->type, [&](auto *b) {
            // the widest moves that the columns' number and both matrices' alignment allow
            if (fits(x, 8) && fits(rows, 8)) return run(a, b, Num<8>());
            if (fits(x, 4) && fits(rows, 4)) return run(a, b, Num<4>());
            return run(a, b, Num<1>());
        });
    });
}

int pdb_route_join(pdb_tokens *t, const pdb_mat *rows, const int32_t *place, int64_t k, const float *weight,
                   const pdb_mat *y, void *stream)
{
    ApiScope scope("pdb_route_join", nullptr, nullptr, nullptr, nullptr, false);
    if (!t) return PDB_EINVAL;
    int rc = check_mat(rows);
    rc = rc ? rc : check_mat(y);
    rc = rc ? rc : check_places(y->rows, k, place);
    if (rc == PDB_OK && weight) rc = check_words(weight, y->rows * k);
    if (rc != PDB_OK) return rc;
    if (y->cols != rows->cols || overlap(rows, y)) return PDB_EINVAL;
    const int dim = (int)y->cols;
    if (dim == 0 || y->rows == 0) return PDB_OK;
    if ((rc = check_device(t)) != PDB_OK) return rc;
    cudaStream_t s = (cudaStream_t)stream;
    TokensUse use{t, s};
    const auto run = [&](auto *a, auto *b, auto e) {
        using T = std::remove_pointer_t<decltype(a)>;
        using O = std::remove_pointer_t<decltype(b)>;
        constexpr int E = decltype(e)::value;
        const int pieces = (dim + JOIN_UNROLL<E> * 32 * E - 1) / (JOIN_UNROLL<E> * 32 * E);
        const int64_t blocks = std::min<int64_t>((y->rows * pieces + 7) / 8, (int64_t)t->sms * JOIN_BLOCKS);
        return launch(k_route_join<T, O, E>, blocks, 256, 0, 1, s, (const T *)rows->data, stride_of(rows), rows->rows, (int)k,
                      place, weight, y->rows, dim, pieces, (O *)y->data, stride_of(y), t->status);
    };
    return with_type(rows->type, [&](auto *a) {
        return with_type(y->type, [&](auto *b) {
            constexpr int E = 16 / sizeof(*a);
            if (fits(rows, E) && fits(y, E)) return run(a, b, Num<E>());
            if (fits(rows, E / 2) && fits(y, E / 2)) return run(a, b, Num<E / 2>());
            return run(a, b, Num<1>());
        });
    });
}

int pdb_route_join_grad(pdb_tokens *t, const pdb_mat *rows, const int32_t *place, int64_t k, const int32_t *source,
                        const float *weight, const pdb_mat *dy, const pdb_mat *drows, float *dweight, void *stream)
{
    ApiScope scope("pdb_route_join_grad", nullptr, nullptr, nullptr, nullptr, false);
    if (!t || (dweight && !rows)) return PDB_EINVAL;
    int rc = rows ? check_mat(rows) : PDB_OK;
    rc = rc ? rc : check_mat(dy);
    rc = rc ? rc : check_mat(drows);
    rc = rc ? rc : check_places(dy->rows, k, place);
    rc = rc ? rc : check_words(source, drows->rows);
    if (rc == PDB_OK && weight) rc = check_words(weight, dy->rows * k);
    if (rc == PDB_OK && rows) rc = check_words(dweight, dy->rows * k);
    if (rc != PDB_OK) return rc;
    if (dy->cols != drows->cols || overlap(dy, drows)) return PDB_EINVAL;
    if (rows && (rows->rows != drows->rows || rows->cols != drows->cols || rows->type != drows->type ||
                 !same_or_apart(rows, drows)))
        return PDB_EINVAL;
    const int dim = (int)dy->cols;
    if (dy->rows == 0 && (drows->rows == 0 || dim == 0)) return PDB_OK;
    if ((rc = check_device(t)) != PDB_OK) return rc;
    cudaStream_t s = (cudaStream_t)stream;
    TokensUse use{t, s};
    const auto run = [&](auto *a, auto *b, auto e) {
        using T = std::remove_pointer_t<decltype(a)>;
        using D = std::remove_pointer_t<decltype(b)>;
        constexpr int E = decltype(e)::value;
        int team = 1;
        while (team < GRAD_WARPS && team * GRAD_UNROLL * 32 * E < dim) team *= 2;
        const int64_t token_blocks = (dy->rows + GRAD_WARPS / team - 1) / (GRAD_WARPS / team);
        const int64_t zero_blocks = (zero_warps(drows->rows, dim) + GRAD_WARPS - 1) / GRAD_WARPS;
        const int64_t blocks = std::min<int64_t>(std::max(token_blocks, zero_blocks), (int64_t)t->sms * GRAD_BLOCKS);
        return launch(k_route_join_grad<T, D, E>, blocks, GRAD_WARPS * 32, 0, 1, s, rows ? (const T *)rows->data : (const T *)nullptr,
                      rows ? stride_of(rows) : 0, drows->rows, (int)k, place, source, weight, (const D *)dy->data, stride_of(dy),
                      dy->rows, dim, team, (T *)drows->data, stride_of(drows), dweight, t->status);
    };
    return with_type(drows->type, [&](auto *a) {
        return with_type(dy->type, [&](auto *b) {
            constexpr int E = 16 / sizeof(*a);
            const auto all_fit = [&](int n) { return fits(dy, n) && fits(drows, n) && (!rows || fits(rows, n)); };
            if (all_fit(E)) return run(a, b, Num<E>());
            if (all_fit(E / 2)) return run(a, b, Num<E / 2>());
            return run(a, b, Num<1>());
        });
    });
}

}  // extern "C"
