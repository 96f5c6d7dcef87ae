// Distillation from a teacher's top logits: loss and gradient (pdb_distill).
//
// Per row, with x_j = (z_j - m) / T and q_k the teacher's probability of slot k:
//   loss / T^2 = sum_k q_k (log q_k - x_k + ln s)   (s = sum_j e^x_j)
//                + q_t (ln q_t - ln p_t)              (bucket: p_t the probability in no slot)
//   dlogits / (w T) = p_j - q_t p_j / p_t  in no slot,  p_j - sum of q_k  in a slot
//
// One cluster of blocks per row (rows.cuh).  The tokens in the slots are marked in a
// bitmap in shared memory, a byte per vector of the row.  With the bucket the pass leaves marked
// tokens out, so that p_t is a sum of its own: one minus the slots' probabilities would
// lose it to rounding for a student as sure as its teacher, and sums relative to the
// outside's own maximum keep it from underflowing.  For the gradient the row is
// read a second time, from L2, where the first pass has left it: e^x is formed again
// rather than kept, each vector written once, and the slots' few elements are
// written over after that by the block that holds them.
#include <algorithm>
#include <cmath>

#include "rows.cuh"

using namespace pdb;
namespace cg = cooperative_groups;

namespace {

constexpr int MAX_SLOTS = 1024;
constexpr float LEAST_REST = 1e-6f;     // a teacher's rest below this is the rounding of its lse
constexpr int MAP_VECTORS = 1 << 15;    // vectors that a block's bitmap covers at a time

__device__ __forceinline__ float load_float(const void *p, int type, int64_t i)
{
    return type == PDB_TYPE_FLOAT    ? ((const float *)p)[i]
           : type == PDB_TYPE_BFLOAT ? __bfloat162float(((const __nv_bfloat16 *)p)[i])
                                     : __half2float(((const __half *)p)[i]);
}

struct Teacher {
    Ids ids;
    const void *top;
    int type, K;
    int64_t stride;
    const float *lse;                   // nullptr: the slots renormalised
};

// sums of N values over the block, on every thread
template <int THREADS, int N>
__device__ __forceinline__ void block_sums(float (&v)[N], float *part)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) v[i] = __fadd_rn(v[i], __shfl_xor_sync(FULL, v[i], off));
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) part[i * 32 + (threadIdx.x >> 5)] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < THREADS / 32; ++w) v[i] = __fadd_rn(v[i], part[i * 32 + w]);
    }
}

// Shared memory: K slots of (token, teacher logit / T, student logit), then the bitmap.
// Slot phase, per slot: token (-1: empty), t = teacher / T (-inf: empty), z = the student's logit.
template <typename T, bool BUCKET, bool GRAD, int THREADS>
__global__ __launch_bounds__(THREADS) void k_distill(const T *logits, int cols, int64_t stride, Teacher teach,
                                                     float temperature, float *loss, const float *__restrict__ weight,
                                                     T *dlogits, int64_t out_stride, int map_words, int *status)
{
    constexpr int E = Vec<T>::E;
    constexpr bool MAP = BUCKET || GRAD;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float part[128];
    __shared__ float own[3];            // this block's m, s, whether its share holds a token of two slots
    __shared__ int twice;               // a token stands in more than one slot
    __shared__ unsigned edge_map;       // marked edge elements
    const int K = teach.K;
    int *s_id = reinterpret_cast<int *>(smem);
    float *s_t = reinterpret_cast<float *>(s_id + K), *s_z = s_t + K;
    unsigned *s_map = reinterpret_cast<unsigned *>(smem + ((size_t)K * 12 + 15) / 16 * 16);
    const unsigned char *map = reinterpret_cast<const unsigned char *>(s_map);

    cg::cluster_group cluster = cg::this_cluster();
    const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int64_t r = blockIdx.x / (unsigned)blocks;
    const T *row = logits + r * stride;
    const Share sh = share_of(row, cols, rank, blocks);
    const uint4 *body = reinterpret_cast<const uint4 *>(row + sh.head);
    const float inv = __fdiv_rn(1.0f, temperature), c = __fmul_rn(inv, LOG2E);

    uint4 v[UNROLL];
    load_vectors<T, THREADS>(v, body, sh.v0, sh.v1);
    const float teacher_lse = BUCKET ? teach.lse[r] : 0.0f;
    const float w = GRAD && weight ? weight[r] : 1.0f;
    // the slots
    if (threadIdx.x == 0) twice = 0, edge_map = 0;
    if (MAP)
        for (int i = threadIdx.x; i < map_words; i += THREADS) s_map[i] = 0;
    float peak = -INFINITY, peak_z = -3.402823466e38f;
    bool odd = false;                   // a NaN among the teacher's logits
    for (int k = threadIdx.x; k < K; k += THREADS) {
        int64_t id = load_id(teach.ids, r, k);
        const float t = load_float(teach.top, teach.type, r * teach.stride + k);
        if (id >= cols) {
            if (rank == 0) set_status(status, PDB_ERANGE);
            id = -1;
        }
        const bool used = id >= 0;
        s_id[k] = used ? (int)id : -1;
        s_t[k] = used ? __fmul_rn(t, inv) : -INFINITY;
        const float z = used ? to_float(row[id]) : 0.0f;
        s_z[k] = z;
        if (used) {
            peak_z = fmaxf(peak_z, z);
            peak = fmaxf(peak, __fmul_rn(t, inv));
            odd |= t != t;
        }
    }
    __syncthreads();
    auto mark = [&](int first) {        // marks the slots' tokens in the map of vectors first .. first + MAP_VECTORS
        for (int k = threadIdx.x; k < K; k += THREADS) {
            const int j = s_id[k];
            if (j < sh.j0 || j >= sh.j1) continue;
            unsigned old, bit;
            if (j < sh.b0 || j >= sh.b1) {
                if (first != sh.v0) continue;
                bit = 1u << (j < sh.b0 ? j - sh.j0 : sh.b0 - sh.j0 + j - sh.b1);
                old = atomicOr(&edge_map, bit);
            } else {
                const int e = j - sh.head - first * E, vec = e / E;
                if (e < 0 || vec >= MAP_VECTORS) continue;
                bit = 1u << (8 * (vec & 3) + e % E);
                old = atomicOr(&s_map[vec >> 2], bit);
            }
            if (old & bit) twice = 1;
        }
    };
    // the pass over the row: all tokens, or with the bucket those in no slot
    Stat<false> a;
    float unused = 0.0f;
    for (int first = sh.v0; first == sh.v0 || first < sh.v1; first += MAP_VECTORS) {
        const int end = min(sh.v1, first + MAP_VECTORS);
        if (MAP) {
            if (first != sh.v0) {
                __syncthreads();
                for (int i = threadIdx.x; i < map_words; i += THREADS) s_map[i] = 0;
                __syncthreads();
            }
            mark(first);
            __syncthreads();
        }
        for (int base = first; base < end; base += THREADS * UNROLL) {
            uint4 next[UNROLL];
            load_vectors<T, THREADS>(next, body, base + THREADS * UNROLL, sh.v1);
            if (BUCKET) {
                unsigned any[UNROLL];
#pragma unroll
                for (int u = 0; u < UNROLL; ++u) {
                    const int i = base + (int)threadIdx.x + u * THREADS;
                    any[u] = i < end ? map[i - first] : 0u;
                }
                if (any[0] | any[1] | any[2] | any[3]) {
#pragma unroll
                    for (int u = 0; u < UNROLL; ++u)
                        if (any[u]) {
                            float f[E];
                            Vec<T>::unpack(v[u], f);
#pragma unroll
                            for (int e = 0; e < E; ++e)
                                if (any[u] >> e & 1) f[e] = -INFINITY;
                            v[u] = Vec<T>::pack(f);
                        }
                }
            }
            add_vectors<T, false>(a, v, c, unused);
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) v[u] = next[u];
        }
    }
    if ((int)threadIdx.x < sh.edges() && !(BUCKET && (edge_map >> threadIdx.x & 1)))
        add_element(a, to_float(row[sh.edge(threadIdx.x)]), c);
    block_join<THREADS>(a, c, part);
    bool repeated = twice;
    if (blocks > 1) {
        if (threadIdx.x == 0) own[0] = a.m, own[1] = a.s, own[2] = (float)twice;
        cluster.sync();
        a = Stat<false>();
        for (int b = 0; b < blocks; ++b) {
            const float *o = cluster.map_shared_rank(own, b);
            a.join(o[0], o[1], 0.0f, c);
            repeated |= o[2] != 0.0f;
        }
        cluster.sync();                  // read by all, and every block has its slots' logits
    }
    // maxima over the slots
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) {
        peak = fmaxf(peak, __shfl_xor_sync(FULL, peak, off));
        peak_z = fmaxf(peak_z, __shfl_xor_sync(FULL, peak_z, off));
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = peak, part[32 + (threadIdx.x >> 5)] = peak_z;
    odd = __syncthreads_or(odd);
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) peak = fmaxf(peak, part[w]), peak_z = fmaxf(peak_z, part[32 + w]);
    const bool live = odd || peak != -INFINITY;
    const bool dup = MAP && repeated;
    auto first_of = [&](int k) {        // slot k is the first of its token
        bool first = true;
        for (int i = 0; i < (dup ? k : 0); ++i) first &= s_id[i] != s_id[k];
        return first;
    };
    const float m = BUCKET ? fmaxf(a.m, peak_z) : a.m;
    // log q = (t - base) - logt: the slots' own log-sum-exp in two parts, each exact to its own size
    const float base = BUCKET ? teacher_lse : peak == -INFINITY ? 0.0f : peak;
    float logt = 0.0f;
    auto logq_of = [&](int k) { return __fsub_rn(__fsub_rn(s_t[k], base), logt); };
    auto q_of = [&](int k) { return s_t[k] == -INFINITY ? 0.0f : expf(logq_of(k)); };
    // sums over the slots: the teacher's weights and, with the bucket, the student's exponentials
    float sums[BUCKET ? 2 : 1] = {};
    for (int k = threadIdx.x; k < K; k += THREADS) {
        sums[0] = __fadd_rn(sums[0], q_of(k));
        if (BUCKET && s_id[k] >= 0 && first_of(k)) sums[1] = __fadd_rn(sums[1], ex2(__fmul_rn(__fsub_rn(s_z[k], m), c)));
    }
    block_sums<THREADS>(sums, part);
    float rest = 0.0f;
    if (BUCKET) {
        rest = __fsub_rn(1.0f, sums[0]);
        if (rest <= LEAST_REST) rest = 0.0f;
    } else {
        logt = logf(sums[0]);
    }
    // s: all tokens relative to m; the outside: a.s relative to a.m
    const float lift = BUCKET ? ex2(__fmul_rn(__fsub_rn(a.m, m), c)) : 1.0f;
    const float s = BUCKET ? __fmaf_rn(a.s, lift, sums[BUCKET ? 1 : 0]) : a.s;
    const bool none = s == 0.0f;
    const float logs = logf(s);
    if (loss && rank == 0 && threadIdx.x < 32) {
        // slot by slot: the sums of q log q and q x alone are many times their difference
        float kl = 0.0f;
        for (int k = threadIdx.x; k < K; k += 32) {
            const float q = q_of(k), x = __fmaf_rn(__fsub_rn(s_z[k], m), inv, -logs);
            if (q != 0.0f) kl = __fmaf_rn(q, __fsub_rn(logq_of(k), x), kl);
        }
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) kl = __fadd_rn(kl, __shfl_xor_sync(FULL, kl, off));
        if (BUCKET && rest > 0.0f) {
            // ln(q_t / p_t): of the quotient, near 1 as a rule; by logarithms where p_t is out of fp32's range
            const float out = __fmul_rn(a.s, lift), p_t = __fdiv_rn(out, __fadd_rn(out, sums[BUCKET ? 1 : 0]));
            const float ratio = p_t > 1e-30f ? logf(__fdiv_rn(rest, p_t))
                                             : __fsub_rn(logf(rest), __fadd_rn(__fsub_rn(logf(a.s), logs),
                                                                              __fmul_rn(__fsub_rn(a.m, m), inv)));
            kl = __fmaf_rn(rest, ratio, kl);
        }
        if (threadIdx.x == 0) loss[r] = !live ? 0.0f : none ? INFINITY : __fmul_rn(__fmul_rn(temperature, temperature), kl);
    }
    if (!GRAD) return;
    // the second pass.  Outside of the slots p_j - q_t p_j / p_t = 2^x_j part, x_j relative to the outside's own
    // maximum, so that neither p_j nor p_t need be representable.
    const bool zero = w == 0.0f || !live || none;
    const float wt = __fmul_rn(w, temperature);
    const float one = __fdiv_rn(1.0f, s);
    const float factor = BUCKET ? (a.s == 0.0f ? 0.0f : __fmul_rn(wt, __fsub_rn(__fmul_rn(lift, one), __fdiv_rn(rest, a.s))))
                                : __fmul_rn(wt, one);
    const float ref = a.m;
    T *drow = dlogits + r * out_stride;
    const bool aligned = ((uintptr_t)(drow + sh.head) & 15) == 0;
    auto slope = [&](float z) { return __fmul_rn(ex2(__fmul_rn(__fsub_rn(z, ref), c)), factor); };
    auto load_again = [&](int at) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int i = at + (int)threadIdx.x + u * THREADS;
            if (i < sh.v1) v[u] = ld_last(body + i);
        }
    };
    for (int at = sh.v0; at < sh.v1; at += THREADS * UNROLL) {
        load_again(at);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int i = at + (int)threadIdx.x + u * THREADS;
            if (i < sh.v1) {
                float f[E];
                Vec<T>::unpack(v[u], f);
#pragma unroll
                for (int e = 0; e < E; ++e) f[e] = zero ? 0.0f : slope(f[e]);
                T *to = drow + sh.head + i * E;
                if (aligned) {
                    __stcs(reinterpret_cast<uint4 *>(to), Vec<T>::pack(f));
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) to[e] = from_float<T>(f[e]);
                }
            }
        }
    }
    if ((int)threadIdx.x < sh.edges()) {
        const int j = sh.edge(threadIdx.x);
        drow[j] = from_float<T>(zero ? 0.0f : slope(to_float(row[j])));
    }
    if (zero) return;
    __syncthreads();
    for (int k = threadIdx.x; k < K; k += THREADS) {
        const int j = s_id[k];
        if (j < sh.j0 || j >= sh.j1 || !first_of(k)) continue;
        float q = 0.0f;
        for (int i = k; i < (dup ? K : k + 1); ++i)
            if (s_id[i] == j) q = __fadd_rn(q, q_of(i));
        const float p = __fmul_rn(ex2(__fmul_rn(__fsub_rn(s_z[k], m), c)), one);
        drow[j] = from_float<T>(__fmul_rn(wt, __fsub_rn(p, q)));
    }
}

}  // namespace

extern "C" int pdb_distill(pdb_tokens *t, const pdb_mat *logits, const pdb_ids *top_ids, const pdb_mat *top_logits,
                           const float *teacher_lse, float temperature, float *loss, const float *weight,
                           const pdb_mat *dlogits, void *stream)
{
    ApiScope scope("pdb_distill", nullptr, nullptr, nullptr, nullptr, false);
    if (!t) return PDB_EINVAL;
    int rc = check_mat(logits);
    rc = rc ? rc : check_mat(top_logits);
    if (rc == PDB_OK && dlogits) rc = check_mat(dlogits);
    if (rc == PDB_OK && top_logits->cols > MAX_SLOTS) rc = PDB_ETOOBIG;
    rc = rc ? rc : check_ids(top_ids, logits->rows, top_logits->cols);
    if (rc != PDB_OK) return rc;
    if (top_logits->rows != logits->rows || (!loss && !dlogits)) return PDB_EINVAL;
    if (!(temperature > 0.0f) || std::isinf(temperature)) return PDB_EINVAL;
    if (dlogits && (dlogits->rows != logits->rows || dlogits->cols != logits->cols || dlogits->type != logits->type ||
                    !same_or_apart(logits, dlogits)))
        return PDB_EINVAL;
    if (logits->rows == 0) return PDB_OK;
    cudaStream_t s = (cudaStream_t)stream;
    TokensUse use{t, s};
    const Teacher teach{ids_of(top_ids), top_logits->data, top_logits->type, (int)top_logits->cols, stride_of(top_logits),
                        teacher_lse};
    return with_type(logits->type, [&](auto *a) {
        using T = std::remove_pointer_t<decltype(a)>;
        const Shape shape = row_shape(logits->rows, logits->cols, Vec<T>::E, t->sms);
        const int64_t share = (logits->cols / Vec<T>::E + shape.blocks) / shape.blocks;     // vectors of a block, at most
        const int map_words = teacher_lse || dlogits ? (int)(std::min<int64_t>(share, MAP_VECTORS) + 3) / 4 : 0;
        const size_t smem = ((size_t)teach.K * 12 + 15) / 16 * 16 + sizeof(unsigned) * map_words;
        return with_threads(shape.threads, [&](auto n) {
            constexpr int N = decltype(n)::value;
            const auto kernel = teacher_lse ? (dlogits ? k_distill<T, true, true, N> : k_distill<T, true, false, N>)
                                            : (dlogits ? k_distill<T, false, true, N> : k_distill<T, false, false, N>);
            return launch_rows(kernel, logits->rows, shape, smem, s, (const T *)logits->data, (int)logits->cols,
                               stride_of(logits), teach, temperature, loss, weight,
                               dlogits ? (T *)dlogits->data : (T *)nullptr, dlogits ? stride_of(dlogits) : (int64_t)0,
                               map_words, t->status);
        });
    });
}
