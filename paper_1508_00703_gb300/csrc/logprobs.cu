// Log probabilities of given tokens with entropy and the most probable
// alternatives, and their gradient (pdb_logprobs, pdb_logprobs_grad).
//
// Per row of logits z, c = scale * log2(e), in one pass over the row (rows.cuh):
//   m = max z,  s = sum 2^((z - m) c),  w = sum 2^((z - m) c) (z - m) c
//   log p_j = (z_j - m) scale - ln s,  lse = m scale + ln s,  entropy = ln s - ln2 w / s
// The row's blocks hand (m, s, w) to the cluster's first one through its shared memory.
//
// Alternatives.  The pass keeps the maximum of each of 64 or 128 groups of
// neighbouring threads.  A value tau that k of them reach is at most the k-th largest
// logit, since k different logits reach it, and the groups that reach tau hold every logit that
// does.  Only those groups' vectors are read again (from L2, dealt out over the block: a warp per group
// waited for one group after the other, 3472 x 18,034 bf16 with 32 alternatives 54 us, 48 now), their logits
// >= tau collected (a few more than k as a rule) and ranked by counting.  A thread's vectors are the block's
// size apart, so that short shares have as many groups as long ones (8 x 4372 bf16, 32 alternatives: 17 us by
// contiguous warps, whose few groups let too much through, 8 now).  Where more
// than the buffer reach tau (ties, rows with fewer unmasked tokens than alternatives) or a NaN hides from the maxima, a radix
// selection over the block's share takes over: four counting passes, exact for
// any order of the row, at its own price (4 x 128,000 bf16, 20 alternatives: 45 us with 8 tokens left in each row, 8.4 with
// half of them).  The pass itself pays one maximum per thread and 64 bytes.
//
// Measured: 2039 x 50,001 bf16, entropy and 5 alternatives 48 us, 204 MB at 4.2 TB/s: 59% of the issue slots
// taken (51 instructions per 8 logits), the rest waits at the rows' ends; 4096 x 128,000
// bf16 without alternatives 154 us of 460 with the gradient, 6.8 TB/s; 4 x 128,000 with 20 alternatives 8.4 us, a chain of
// latencies (two launches' worth of barriers, three reads).
#include <algorithm>
#include <cmath>

#include "rows.cuh"

using namespace pdb;
namespace cg = cooperative_groups;

namespace {

constexpr int MAX_TOP = 64;
constexpr int GROUPS = 128;             // most groups of threads
constexpr int BUFFER = 1024;            // candidates of a block; also the lists of a cluster: MAX_CLUSTER * MAX_TOP
static_assert(MAX_CLUSTER * MAX_TOP <= BUFFER, "the cluster's lists are ranked in one buffer");

// a logit as a word that orders like it: NaN above all, -0 = +0
__device__ __forceinline__ uint32_t order_of(float z)
{
    const uint32_t b = __float_as_uint(z);
    return z != z ? 0xfffffffeu : z == 0.0f ? 0x80000000u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float order_value(uint32_t o)
{
    return __uint_as_float((o & 0x80000000u) ? o ^ 0x80000000u : ~o);
}
// with its token: larger logits first, then lower tokens
__device__ __forceinline__ uint64_t key_of(uint32_t order, int j) { return (uint64_t)order << 32 | (uint32_t)~j; }

struct TopShared {
    alignas(16) float group[GROUPS];
    int list[GROUPS];                   // groups that reach tau
    uint64_t key[BUFFER];               // candidates
    uint64_t best[MAX_TOP];             // the block's best, in order
    int hist[256];
    int warp_count[16];
    int n, n_list, need, digit;
    float tau;
};

// best[0..min(k, n)) = the largest of key[0..n), in order (keys differ)
template <int THREADS>
__device__ __forceinline__ void rank_keys(TopShared &t, int n, int k)
{
    for (int i = threadIdx.x; i < n; i += THREADS) {
        const uint64_t mine = t.key[i];
        int above = 0;
        for (int j = 0; j < n; ++j) above += t.key[j] > mine ? 1 : 0;
        if (above < k) t.best[above] = mine;
    }
    __syncthreads();
}

// the k largest of row[j0..j1) into key[0..k) by radix selection, for any contents (j1 - j0 > k)
template <typename T, int THREADS>
__device__ __noinline__ void select_keys(TopShared &t, const T *row, int j0, int j1, int k)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t masked = order_of(-INFINITY);
    uint32_t prefix = 0, fixed = 0;
    int need = k;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = threadIdx.x; i < 256; i += THREADS) t.hist[i] = 0;
        __syncthreads();
        int n_masked = 0;                // the one value that whole rows hold is counted apart
        for (int j = j0 + threadIdx.x; j < j1; j += THREADS) {
            const uint32_t o = order_of(to_float(row[j]));
            if ((o & fixed) != prefix) continue;
            if (o == masked) ++n_masked;
            else atomicAdd(&t.hist[(o >> shift) & 255], 1);
        }
        if (n_masked) atomicAdd(&t.hist[(masked >> shift) & 255], n_masked);
        __syncthreads();
        if (threadIdx.x == 0) {
            int d = 255;
            while (d > 0 && t.hist[d] < need) need -= t.hist[d--];
            t.digit = d;
            t.need = need;
            t.n = 0;
        }
        __syncthreads();
        prefix |= (uint32_t)t.digit << shift;
        fixed |= 255u << shift;
        need = t.need;
    }
    // prefix is the k-th largest value: everything above it, and the first `need` that equal it
    int taken = 0;
    for (int base = j0; base < j1; base += THREADS) {
        const int j = base + threadIdx.x;
        const uint32_t o = j < j1 ? order_of(to_float(row[j])) : 0u;
        if (j < j1 && o > prefix) t.key[atomicAdd(&t.n, 1)] = key_of(o, j);
        const bool equal = j < j1 && o == prefix;
        if (__syncthreads_or(equal && taken < need)) {
            const unsigned b = __ballot_sync(FULL, equal);
            if (lane == 0) t.warp_count[warp] = __popc(b);
            __syncthreads();
            int at = taken + __popc(b & lanemask_lt()), all = 0;
            for (int w = 0; w < THREADS / 32; ++w) {
                const int x = t.warp_count[w];
                at += w < warp ? x : 0;
                all += x;
            }
            if (equal && at < need) t.key[k - need + at] = key_of(o, j);   // behind the k - need above it
            taken += all;
            __syncthreads();
        }
    }
    __syncthreads();
}

// best[0..k) = the block's share's k largest; returns how many there are
template <typename T, int THREADS>
__device__ __forceinline__ int top_of_share(TopShared &t, const T *row, const uint4 *share, const Share &sh, float top,
                                            bool odd, int k)
{
    constexpr int E = Vec<T>::E;
    const int n_share = sh.j1 - sh.j0, have = min(k, n_share);
    if (n_share <= k) {
        for (int j = sh.j0 + threadIdx.x; j < sh.j1; j += THREADS) t.key[j - sh.j0] = key_of(order_of(to_float(row[j])), j);
        __syncthreads();
        rank_keys<THREADS>(t, n_share, k);
        return have;
    }
    if (!odd) {
        // groups of `per` neighbouring threads: fewer for few alternatives
        const int per = THREADS / (k <= 16 ? GROUPS / 2 : GROUPS), groups = THREADS / per;
        for (int off = per >> 1; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, off));
        if (threadIdx.x % (unsigned)per == 0) t.group[threadIdx.x / (unsigned)per] = top;
        if (threadIdx.x == 0) t.n = t.n_list = 0;
        __syncthreads();
        if (threadIdx.x < 32) {
            // tau by bisection over the orders of the groups' maxima: any value that k groups reach will do, the higher
            // the better; it stops when hardly more than k do
            uint32_t o[GROUPS / 32], lo = 0xffffffffu, hi = 0;
#pragma unroll
            for (int i = 0; i < GROUPS / 32; ++i) {
                o[i] = i * 32 < groups ? order_of(t.group[i * 32 + threadIdx.x]) : 0u;
                hi = max(hi, o[i]);
                if (i * 32 < groups) lo = min(lo, o[i]);
            }
            hi = __reduce_max_sync(FULL, hi) + 1;          // no group reaches hi; all reach lo
            lo = __reduce_min_sync(FULL, lo);
            while (hi - lo > 1) {
                const uint32_t mid = lo + (hi - lo) / 2;
                int n = 0;
#pragma unroll
                for (int i = 0; i < GROUPS / 32; ++i) n += __popc(__ballot_sync(FULL, o[i] >= mid));
                if (n >= k) lo = mid;
                else hi = mid;
                if (n >= k && n <= k + 1 + k / 8) break;
            }
            if (threadIdx.x == 0) t.tau = order_value(lo);
        }
        __syncthreads();
        const float tau = t.tau;
        if ((int)threadIdx.x < groups && t.group[threadIdx.x] >= tau) t.list[atomicAdd(&t.n_list, 1)] = threadIdx.x;
        __syncthreads();
        const int n_list = t.n_list;    // k, or somewhat more
        const int n_vec = sh.v1 - sh.v0, turns = (n_vec + THREADS - 1) / THREADS;
        auto take = [&](float z, int j) {
            if (z >= tau) {
                const int at = atomicAdd(&t.n, 1);
                if (at < BUFFER) t.key[at] = key_of(order_of(z), j);
            }
        };
        // the groups' vectors, dealt out over the block, UNROLL of a thread under way; those side by side go together
#pragma unroll 1
        for (int i0 = threadIdx.x; i0 < n_list * turns * per; i0 += THREADS * UNROLL) {
            uint4 x[UNROLL];
            int at[UNROLL];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int i = i0 + u * THREADS, pair = i / (unsigned)per, g = pair / (unsigned)turns;
                at[u] = n_vec;
                if (g < n_list) at[u] = (pair - g * turns) * THREADS + t.list[g] * per + (i & (per - 1));
                if (at[u] < n_vec) x[u] = ld_keep(share + at[u]);
            }
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                if (at[u] >= n_vec || Vec<T>::max_float(Vec<T>::vmax(Vec<T>::max_init(), x[u])) < tau) continue;
                float f[E];
                Vec<T>::unpack(x[u], f);
#pragma unroll
                for (int e = 0; e < E; ++e) take(f[e], sh.b0 + at[u] * E + e);
            }
        }
        if ((int)threadIdx.x < sh.edges()) take(to_float(row[sh.edge(threadIdx.x)]), sh.edge(threadIdx.x));
        __syncthreads();
        const int n = t.n;
        if (n <= BUFFER) {
            rank_keys<THREADS>(t, n, k);
            return have;
        }
        __syncthreads();
    }
    select_keys<T, THREADS>(t, row, sh.j0, sh.j1, k);
    rank_keys<THREADS>(t, k, k);
    return have;
}

struct LogprobsOut {
    float *logp, *lse, *entropy, *top_logp;
    int32_t *top_ids;
};

template <typename T, bool ENT, bool TOP, int THREADS>
__global__ __launch_bounds__(THREADS, 1024 / THREADS) void k_logprobs(const T *logits, int cols, int64_t stride, Ids ids,
                                                      float scale, int64_t ignore, int k, LogprobsOut out, int *status)
{
    after_previous();
    __shared__ float part[96];
    __shared__ float own[4];            // this block's m, s, w, number of alternatives
    __shared__ __align__(16) unsigned char top_raw[TOP ? sizeof(TopShared) : 16];
    TopShared &t = *reinterpret_cast<TopShared *>(top_raw);
    cg::cluster_group cluster = cg::this_cluster();
    const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int64_t r = blockIdx.x / (unsigned)blocks;
    const T *row = logits + r * stride;
    const Share sh = share_of(row, cols, rank, blocks);
    const uint4 *body = reinterpret_cast<const uint4 *>(row + sh.b0);
    const int n_vec = sh.v1 - sh.v0;
    const float c = __fmul_rn(scale, LOG2E);

    // the given token, then its logit, on their way while the row is read
    const bool asks = out.logp && rank == 0 && threadIdx.x == 0;
    int2 raw = {0, 0};
    if (asks) raw = fetch_id(ids, r);
    T z_given = from_float<T>(0.0f);
    bool there = false;
    auto ask = [&]() {
        const int64_t given = id_of(ids, raw);
        there = given != ignore && given >= 0 && given < cols;
        if (!there && given != ignore) set_status(status, PDB_ERANGE);
        if (there) z_given = row[given];
    };
    const bool has_edge = (int)threadIdx.x < sh.edges();
    T z_edge = from_float<T>(0.0f);
    if (has_edge) z_edge = row[sh.edge(threadIdx.x)];
    Stat<ENT> a;
    float top = -INFINITY;
    {
        uint4 v[UNROLL];
        load_vectors<T, THREADS, THREADS>(v, body, 0, threadIdx.x, n_vec);
        for (int base = 0; base < n_vec; base += THREADS * UNROLL) {
            uint4 next[UNROLL];
            load_vectors<T, THREADS, THREADS>(next, body, base + THREADS * UNROLL, threadIdx.x, n_vec);
            add_vectors<T, ENT>(a, v, c, top);
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) v[u] = next[u];
            if (base == 0 && asks) ask();
        }
        if (n_vec == 0 && asks) ask();
    }
    if (has_edge) add_element(a, to_float(z_edge), c);
    block_join<THREADS>(a, c, part);
    int have = 0;
    if (TOP) have = top_of_share<T, THREADS>(t, row, body, sh, top, !(a.s < INFINITY), k);
    if (blocks > 1) {
        if (threadIdx.x == 0) own[0] = a.m, own[1] = a.s, own[2] = a.w, own[3] = (float)have;
        cluster.sync();
        if (rank == 0) {
            for (int b = 1; b < blocks; ++b) {
                const float *o = cluster.map_shared_rank(own, b);
                a.join(o[0], o[1], ENT ? o[2] : 0.0f, c);
            }
            if (TOP) {
                // the blocks' lists, one after the other, ranked together
                if (threadIdx.x == 0) t.n = 0;
                __syncthreads();
                for (int i = threadIdx.x; i < blocks * k; i += THREADS) {
                    const int b = i / k, at = i % k;
                    if (at < (int)cluster.map_shared_rank(own, b)[3])
                        t.key[atomicAdd(&t.n, 1)] = cluster.map_shared_rank(&t, b)->best[at];
                }
                __syncthreads();
                rank_keys<THREADS>(t, t.n, k);
            }
        }
        cluster.sync();                  // the others' shared memory has been read
        if (rank != 0) return;
    }
    const bool none = a.s == 0.0f;
    const float ref = none ? 0.0f : a.m, logs = logf(a.s);
    if (threadIdx.x == 0) {
        if (out.lse) out.lse[r] = none ? -INFINITY : __fmaf_rn(ref, scale, logs);
        if (out.entropy) out.entropy[r] = none ? 0.0f : __fmaf_rn(-LN2, __fdiv_rn(a.w, a.s), logs);
        if (out.logp)
            out.logp[r] = !there ? 0.0f : none ? -INFINITY : __fmaf_rn(__fsub_rn(to_float(z_given), ref), scale, -logs);
    }
    if (TOP)
        for (int i = threadIdx.x; i < k; i += THREADS) {
            const uint64_t key = t.best[i];
            if (out.top_ids) out.top_ids[r * k + i] = (int)~(uint32_t)key;
            if (out.top_logp)
                out.top_logp[r * k + i] =
                    none ? -INFINITY : __fmaf_rn(__fsub_rn(order_value((uint32_t)(key >> 32)), ref), scale, -logs);
        }
}

// m and s (rows.cuh) of a whole row, on every thread of the block; `part` holds 96 floats
template <typename T, int THREADS>
__device__ __noinline__ float2 row_statistics(const T *row, int cols, float c, float *part)
{
    const Share sh = share_of(row, cols, 0, 1);
    const uint4 *body = reinterpret_cast<const uint4 *>(row + sh.b0);
    const int n_vec = sh.v1 - sh.v0;
    Stat<false> a;
    float unused = 0.0f;
#pragma unroll 1
    for (int base = 0; base < n_vec; base += THREADS * UNROLL) {
        uint4 v[UNROLL];
        load_vectors<T, THREADS, 32>(v, body, base, lane_start(), n_vec);
        add_vectors<T, false>(a, v, c, unused);
    }
    if ((int)threadIdx.x < sh.edges()) add_element(a, to_float(row[sh.edge(threadIdx.x)]), c);
    block_join<THREADS>(a, c, part);
    return {a.m, a.s};
}

// dlogits = -p (A + B x) (+ scale g at the given token), x = (z - lse / scale) c, p = 2^x,
// A = scale (g + h entropy), B = scale h ln2.  One pass, every element read and written once: bound by
// memory.  A block takes one piece of a row; pieces of a row need nothing from one another.
//
// lse is rounded to 32 bits, which moves p by 2^-24 |lse|: a row masked by the type's lowest value from end to end would have
// lse = that value, and p = 1 for all.  From |lse| = 256 on (p good to 2^-15 below), and where lse has left fp32's
// range, the row's first block alone takes the whole row, with its maximum and sum formed again: x = (z - m) c - log2 s.
// 4096 x 128,000 bf16: 303 us, 433 where every row is such a one; 1 x 128,000, in 64 pieces: 2.6 us, 14 by one block.
constexpr float FAR_LSE = 256.0f;

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void k_logprobs_grad(const T *logits, int cols, int64_t stride, int pieces, Ids ids,
                                                           float scale, int64_t ignore, const float *lse,
                                                           const float *entropy,
                                                           const float *dlogp,
                                                           const float *dentropy, T *dlogits,
                                                           int64_t out_stride, int *status)
{
    after_previous();
    constexpr int E = Vec<T>::E;
    __shared__ float part[96];
    const int64_t r = blockIdx.x / (unsigned)pieces;
    const int piece = (int)(blockIdx.x - r * pieces);
    const T *row = logits + r * stride;
    T *drow = dlogits + r * out_stride;
    Share sh = share_of(row, cols, piece, pieces);
    const uint4 *body = reinterpret_cast<const uint4 *>(row + sh.b0);
    int n_vec = sh.v1 - sh.v0;
    uint4 v[UNROLL];
    load_vectors<T, THREADS, 32>(v, body, 0, lane_start(), n_vec);          // on their way while the row's numbers arrive

    float g = dlogp ? dlogp[r] : 0.0f;
    const float h = dentropy ? dentropy[r] : 0.0f;
    int t = -1;
    if (dlogp) {
        const int64_t id = load_id(ids, r);
        const bool there = id != ignore && id >= 0 && id < cols;
        if (!there && id != ignore && threadIdx.x == 0 && piece == 0) set_status(status, PDB_ERANGE);
        if (there) t = (int)id;
        else g = 0.0f;
    }
    const float l = lse[r];
    // up to a scale of 1 no finite logits have an lse of -inf
    bool zero = (g == 0.0f && h == 0.0f) || (l == -INFINITY && scale <= 1.0f);
    const float H = h != 0.0f ? entropy[r] : 0.0f;
    const float c = __fmul_rn(scale, LOG2E);
    float ref = __fdiv_rn(l, scale), log2s = 0.0f;
    if (!zero && !(fabsf(l) < FAR_LSE && fabsf(ref) < INFINITY)) {
        if (piece != 0) return;
        const float2 ms = row_statistics<T, THREADS>(row, cols, c, part);
        ref = ms.x, log2s = log2f(ms.y), zero = ms.y == 0.0f;
        sh = share_of(row, cols, 0, 1);
        body = reinterpret_cast<const uint4 *>(row + sh.b0);
        n_vec = sh.v1 - sh.v0;
        load_vectors<T, THREADS, 32>(v, body, 0, lane_start(), n_vec);
    }
    const float A = -__fmul_rn(scale, __fmaf_rn(h, H, g)), B = -__fmul_rn(__fmul_rn(scale, h), LN2);
    const float at_t = __fmul_rn(scale, g);
    auto slope = [&](float z) {
        // x held above -200, where p = 0: B x p of a token masked by -inf is 0
        const float x = max_nan(__fmaf_rn(__fsub_rn(z, ref), c, -log2s), -200.0f);
        return __fmul_rn(ex2(x), __fmaf_rn(B, x, A));
    };
    const bool aligned = ((uintptr_t)(drow + sh.b0) & 15) == 0;
    for (int base = 0; base < n_vec; base += THREADS * UNROLL) {
        uint4 next[UNROLL];
        load_vectors<T, THREADS, 32>(next, body, base + THREADS * UNROLL, lane_start(), n_vec);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int i = base + lane_start() + u * 32;
            if (i < n_vec) {
                float f[E];
                Vec<T>::unpack(v[u], f);
                const int j = sh.b0 + i * E;
#pragma unroll
                for (int e = 0; e < E; ++e) f[e] = zero ? 0.0f : slope(f[e]);
                if ((unsigned)(t - j) < (unsigned)E && !zero)
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (j + e == t) f[e] = __fadd_rn(f[e], at_t);
                if (aligned) {
                    __stcs(reinterpret_cast<uint4 *>(drow + j), Vec<T>::pack(f));
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) drow[j + e] = from_float<T>(f[e]);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) v[u] = next[u];
    }
    if ((int)threadIdx.x < sh.edges()) {
        const int j = sh.edge(threadIdx.x);
        const float x = slope(to_float(row[j]));
        drow[j] = from_float<T>(zero ? 0.0f : j == t ? __fadd_rn(x, at_t) : x);
    }
}

}  // namespace

extern "C" {

int pdb_logprobs(pdb_tokens *t, const pdb_mat *logits, const pdb_ids *ids, float scale, int64_t ignore, float *logp,
                 float *lse, float *entropy, int64_t k, float *top_logp, int32_t *top_ids, void *stream)
{
    ApiScope scope("pdb_logprobs", nullptr, nullptr, nullptr, nullptr, false);
    if (!t) return PDB_EINVAL;
    int rc = check_mat(logits);
    if (rc == PDB_OK && logp) rc = check_ids(ids, logits->rows);
    if (rc != PDB_OK) return rc;
    if (!usable_scale(scale) || k < 0 || k > logits->cols) return PDB_EINVAL;
    if (k > MAX_TOP) return PDB_ETOOBIG;
    if (logits->rows == 0) return PDB_OK;
    if ((rc = check_device(t)) != PDB_OK) return rc;
    cudaStream_t s = (cudaStream_t)stream;
    TokensUse use{t, s};
    const bool top = k > 0 && (top_logp || top_ids);
    const LogprobsOut out{logp, lse, entropy, top_logp, top_ids};
    return with_type(logits->type, [&](auto *a) {
        using T = std::remove_pointer_t<decltype(a)>;
        const Shape shape = once_shape(logits->rows, logits->cols, Vec<T>::E, t->sms, 0, false);
        return with_threads(shape.threads, [&](auto n) {
            constexpr int N = decltype(n)::value;
            const auto kernel = entropy ? (top ? k_logprobs<T, true, true, N> : k_logprobs<T, true, false, N>)
                                        : (top ? k_logprobs<T, false, true, N> : k_logprobs<T, false, false, N>);
            return launch_rows(kernel, shape, s, (const T *)logits->data, (int)logits->cols, stride_of(logits),
                               ids_of(ids, logp), scale, ignore, (int)k, out, t->status);
        });
    });
}

int pdb_logprobs_grad(pdb_tokens *t, const pdb_mat *logits, const pdb_ids *ids, float scale, int64_t ignore,
                      const float *lse, const float *entropy, const float *dlogp, const float *dentropy,
                      const pdb_mat *dlogits, void *stream)
{
    ApiScope scope("pdb_logprobs_grad", nullptr, nullptr, nullptr, nullptr, false);
    if (!t) return PDB_EINVAL;
    int rc = check_mat(logits);
    rc = rc ? rc : check_mat(dlogits);
    if (rc == PDB_OK && dlogp) rc = check_ids(ids, logits->rows);
    if (rc != PDB_OK) return rc;
    if (!usable_scale(scale)) return PDB_EINVAL;
    if (dlogits->rows != logits->rows || dlogits->cols != logits->cols || dlogits->type != logits->type ||
        !same_or_apart(logits, dlogits))
        return PDB_EINVAL;
    if (logits->rows == 0 || logits->cols == 0) return PDB_OK;
    if (!lse || (dentropy && !entropy)) return PDB_EINVAL;
    if ((rc = check_device(t)) != PDB_OK) return rc;
    cudaStream_t s = (cudaStream_t)stream;
    TokensUse use{t, s};
    return with_type(logits->type, [&](auto *a) {
        using T = std::remove_pointer_t<decltype(a)>;
        // pieces of about 4 vectors a thread and, for few rows, as many as there are SMs
        const int64_t nv = logits->cols / Vec<T>::E + 1;
        const int threads = nv < 1024 ? 128 : nv < 4096 ? 256 : 512;
        int pieces = 1;
        while (pieces < 64 && logits->rows * pieces < t->sms && nv / (2 * pieces) >= threads) pieces *= 2;
        return with_threads(threads, [&](auto n) {
            constexpr int N = decltype(n)::value;
            return launch(k_logprobs_grad<T, N>, logits->rows * pieces, N, 0, 1, s, (const T *)logits->data,
                          (int)logits->cols, stride_of(logits), pieces, ids_of(ids, dlogp), scale, ignore, lse, entropy,
                          dlogp, dentropy, (T *)dlogits->data, stride_of(dlogits), t->status);
        });
    });
}

}  // extern "C"
