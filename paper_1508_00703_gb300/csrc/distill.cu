// Distillation from a teacher's top logits: loss and gradient (pdb_distill).
//
// Per row, with x_j = (z_j - m) / T and q_k the teacher's probability of slot k:
//   loss / T^2 = sum_k q_k (log q_k - x_k + ln s)   (s = sum_j e^x_j)
//                + q_t (ln q_t - ln p_t)              (bucket: p_t the probability in no slot)
//   dlogits / (w T) = p_j - q_t p_j / p_t  in no slot,  p_j - sum of q_k  in a slot
//
// One cluster of blocks per row (rows.cuh).  The tokens in the slots are marked in
// shared memory, a bit and a byte per vector of the row.  With the bucket the pass leaves vectors with a marked token
// out (one word of bits tests a warp's chunk), and a thread per slot adds the vector's other
// tokens, so that p_t is a sum of its own: one minus the slots' probabilities would
// lose it to rounding for a student as sure as its teacher, and sums relative to the
// outside's own maximum keep it from underflowing.  For the gradient the row is
// visited a second time, from shared memory as far as that holds it and else from L2: e^x is formed again
// rather than kept, each vector written once, and the slots' few elements are
// written over after that by the block that holds them.
//
// Measured: the loss alone, 1024 x 32,000 fp16, 64 slots, 15.6 us (66 MB, 4.2 TB/s: one round of blocks, of whose time
// start, joins and end are 6 us); with gradient 4096 x 128,000 bf16 360 us (2.1 GB, 5.8 TB/s; DRAM moves little more
// than that, the rest is time per row), 1501 x 50,001 fp32 114 us (5.3 TB/s), 3000 x 128,000 fp32 484 us (6.3 TB/s).  Many short
// rows are bound by the chain of barriers and joins of each: 8000 x 2000 bf16 42 us, four times what their bytes take.
#include <algorithm>
#include <cmath>
#include <mutex>

#include "rows.cuh"

using namespace pdb;
namespace cg = cooperative_groups;

namespace {

constexpr int MAX_SLOTS = 1024;
constexpr float LEAST_REST = 1e-6f;     // a teacher's rest below this is the rounding of its lse
constexpr int64_t MAX_COLS = 1 << 21;   // a block's marks then take 73,872 bytes at most (fp32, clusters of 8)

// an element of a matrix of any type, fetched and converted in two steps (as fetch_id)
__device__ __forceinline__ uint32_t fetch_element(const void *p, int type, int64_t i)
{
    return type == PDB_TYPE_FLOAT ? ((const uint32_t *)p)[i] : (uint32_t)((const uint16_t *)p)[i];
}
__device__ __forceinline__ float element_of(int type, uint32_t raw)
{
    return type == PDB_TYPE_FLOAT    ? __uint_as_float(raw)
           : type == PDB_TYPE_BFLOAT ? __uint_as_float(raw << 16)
                                     : __half2float(__ushort_as_half((unsigned short)raw));
}

struct Teacher {
    Ids ids;
    const void *top;
    int type, K;
    int64_t stride;
    const float *lse;                   // nullptr: the slots renormalised
};

// sums of N values over the block, on every thread, with one barrier (`part` as for block_join)
template <int THREADS, int N>
__device__ __forceinline__ void block_sums(float (&v)[N], float *part)
{
    constexpr int W = THREADS / 32;
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) v[i] = __fadd_rn(v[i], __shfl_xor_sync(FULL, v[i], off));
        if ((threadIdx.x & 31) == 0) part[i * 32 + (threadIdx.x >> 5)] = v[i];
    }
    team_sync<THREADS>();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = part[i * 32 + (threadIdx.x & (W - 1))];
#pragma unroll
        for (int off = W / 2; off >= 1; off >>= 1) v[i] = __fadd_rn(v[i], __shfl_xor_sync(FULL, v[i], off));
    }
}

// ------------------------------------------------------------------ parts of both kernels
// The K slots of a row in shared memory: token (-1: empty), teacher logit / T (-inf: empty), student's logit.
struct Slots {
    int *id;
    float *t, *z;
    __device__ __forceinline__ Slots(void *at, int K) : id((int *)at), t((float *)at + K), z((float *)at + 2 * K) {}
};
constexpr int SLOT_BYTES = 12;

// Marks of the tokens in slots: per vector of the share a bit (some token of it) and a byte (which), and a word for the
// share's edges.
struct Marks {
    unsigned *bits, *bytes, *edge;
    // the place of token j's mark; false: not in this share.  vec: its vector, -1 on an edge
    template <int E>
    __device__ __forceinline__ bool place(const Share &sh, int j, unsigned *&word, unsigned &bit, int &vec) const
    {
        if (j < sh.j0 || j >= sh.j1) return false;
        if (j < sh.b0 || j >= sh.b1) {
            bit = 1u << (j < sh.b0 ? j - sh.j0 : sh.b0 - sh.j0 + j - sh.b1);
            word = edge, vec = -1;
        } else {
            const int e = j - sh.b0;
            vec = e / E;
            bit = 1u << (8 * (vec & 3) + e % E);
            word = bytes + (vec >> 2);
        }
        return true;
    }
    // marks it; true if it was marked before
    template <int E>
    __device__ __forceinline__ bool set(const Share &sh, int j) const
    {
        unsigned *word, bit;
        int vec;
        if (!place<E>(sh, j, word, bit, vec)) return false;
        if (vec >= 0) atomicOr(bits + (vec >> 5), 1u << (vec & 31));
        return (atomicOr(word, bit) & bit) != 0;
    }
    template <int E>
    __device__ __forceinline__ void clear(const Share &sh, int j) const
    {
        unsigned *word, bit;
        int vec;
        if (place<E>(sh, j, word, bit, vec) && vec >= 0) *word = 0, bits[vec >> 5] = 0;
    }
    __device__ __forceinline__ unsigned of_vector(int vec) const { return bytes[vec >> 2] >> (8 * (vec & 3)) & 255u; }
    // a thread's vectors of the chunk at base: those with a marked token become -inf altogether
    template <typename T>
    __device__ __forceinline__ void leave_out(uint4 (&x)[UNROLL], int base) const
    {
        static_assert(UNROLL == 4, "a warp's bits of a chunk are one 16-byte word");
        constexpr uint32_t N = Vec<T>::NEG_INF;
        const uint4 w = *reinterpret_cast<const uint4 *>(bits + (base + (int)(threadIdx.x & ~31u) * UNROLL) / 32);
        if (w.x | w.y | w.z | w.w) {
            const int lane = threadIdx.x & 31;
            const unsigned m[UNROLL] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int u = 0; u < UNROLL; ++u)
                if (m[u] >> lane & 1) x[u] = uint4{N, N, N, N};
        }
    }
};

// slot k of a row as fetched; then its token (-1: empty; an id past the vocabulary is recorded and counts as empty) and
// the teacher's logit / T
struct RawSlot {
    int2 id;
    uint32_t t;
    __device__ __forceinline__ void fetch(const Teacher &teach, int64_t r, int k)
    {
        id = fetch_id(teach.ids, r, k);
        t = fetch_element(teach.top, teach.type, r * teach.stride + k);
    }
    __device__ __forceinline__ int token(const Teacher &teach, int cols, bool tell, int *status) const
    {
        const int64_t j = id_of(teach.ids, id);
        if (j >= cols && tell) set_status(status, PDB_ERANGE);
        return j < 0 || j >= cols ? -1 : (int)j;
    }
    __device__ __forceinline__ float logit(const Teacher &teach, float inv) const { return __fmul_rn(element_of(teach.type, t), inv); }
};

// the 16 bytes around token j's logit where it lies in the share's body, else the logit alone in their first bytes; and
// the logit in them
template <typename T>
__device__ __forceinline__ uint4 fetch_around(const T *row, const Share &sh, int j)
{
    uint4 x = {0, 0, 0, 0};
    if (j >= sh.b0 && j < sh.b1) x = ld_keep(reinterpret_cast<const uint4 *>(row + sh.b0) + (j - sh.b0) / Vec<T>::E);
    else if (sizeof(T) == 2) x.x = *reinterpret_cast<const uint16_t *>(row + j);
    else x.x = *reinterpret_cast<const uint32_t *>(row + j);
    return x;
}
template <typename T>
__device__ __forceinline__ float logit_in(const uint4 &x, const Share &sh, int j)
{
    constexpr int E = Vec<T>::E;
    const int at = j >= sh.b0 && j < sh.b1 ? (j - sh.b0) % E : 0;
    float f[E], z = 0.0f;
    Vec<T>::unpack(x, f);
#pragma unroll
    for (int i = 0; i < E; ++i) z = i == at ? f[i] : z;
    return z;
}

// The loss of a row whose sum came out infinite at a temperature below 1, with every term times T^2: (z - m) / T of a token masked
// by the type's lowest value passes fp32's range, T (z - m) does not.  A call of its own, for the sake of the others.
__device__ __noinline__ float loss_of_lowest(const float *t, const float *z, int K, float T, float base, float logt, float m,
                                             float logs, float rest, float out_m, float out_logs)
{
    const float square = __fmul_rn(T, T);
    float kl = 0.0f;
#pragma unroll 1
    for (int k = threadIdx.x & 31; k < K; k += 32) {
        if (t[k] == -INFINITY) continue;
        const float logq = __fsub_rn(__fsub_rn(t[k], base), logt), q = expf(logq);
        const float x = __fmaf_rn(__fsub_rn(z[k], m), T, -__fmul_rn(logs, square));
        if (q != 0.0f) kl = __fmaf_rn(q, __fsub_rn(__fmul_rn(logq, square), x), kl);
    }
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) kl = __fadd_rn(kl, __shfl_xor_sync(FULL, kl, off));
    if (rest > 0.0f) {
        const float logp = __fmaf_rn(__fsub_rn(out_m, m), T, __fmul_rn(__fsub_rn(out_logs, logs), square));
        kl = __fmaf_rn(rest, __fsub_rn(__fmul_rn(logf(rest), square), logp), kl);
    }
    return kl;
}

// What the slots and the pass over the row come to.
template <bool BUCKET>
struct Row {
    Stat<false> a;                      // all tokens, or with the bucket those in no slot
    float m;                            // maximum over all
    float base, logt;                   // log q = (t - base) - logt, each part exact to its own size
    float peak, peak_z;                 // largest teacher logit / T, largest student logit in a slot
    bool odd;                           // a NaN among the teacher's logits
    bool repeated;                      // a token stands in more than one slot
    bool live;                          // there is a slot to learn from
    float s, lift, in_slots, rest;      // sum of exponentials relative to m; a.s * lift + in_slots = s; the teacher's rest

    __device__ __forceinline__ float logq(const Slots &S, int k) const { return __fsub_rn(__fsub_rn(S.t[k], base), logt); }
    __device__ __forceinline__ float q(const Slots &S, int k) const { return S.t[k] == -INFINITY ? 0.0f : expf(logq(S, k)); }
    // slot k is the first of its token
    __device__ __forceinline__ bool first_of(const Slots &S, int k) const
    {
        bool is = true;
#pragma unroll 1
        for (int i = 0; i < (repeated ? k : 0); ++i) is &= S.id[i] != S.id[k];
        return is;
    }

    // adds the unmarked tokens of the vector around slot k's token j, once for each such vector (by the slot of its first
    // marked token): the pass has left the whole vector out
    template <typename T>
    __device__ __forceinline__ void add_around(const Slots &S, const Marks &marks, const Share &sh, int k, const uint4 &around,
                                               float c)
    {
        constexpr int E = Vec<T>::E;
        const int j = S.id[k];
        if (j < sh.b0 || j >= sh.b1) return;
        const int e = (j - sh.b0) % E;
        const unsigned m = marks.of_vector((j - sh.b0) / E);
        if ((m & ((1u << e) - 1)) != 0 || !first_of(S, k)) return;
        float f[E], unused = 0.0f;
        Vec<T>::unpack(around, f);
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (m >> i & 1) f[i] = -INFINITY;
        const uint4 x[1] = {Vec<T>::pack(f)};
        add_vectors<T, false>(a, x, c, unused);
    }

    // joins the threads' statistics and slot maxima; `part` holds 192 floats; one barrier
    template <int THREADS>
    __device__ __forceinline__ void join(float c, int K, float *part)
    {
        const int warp = threadIdx.x >> 5;
        if (warp * 32 < K) {
#pragma unroll
            for (int off = 16; off >= 1; off >>= 1) {
                peak = fmaxf(peak, __shfl_xor_sync(FULL, peak, off));
                peak_z = fmaxf(peak_z, __shfl_xor_sync(FULL, peak_z, off));
            }
            odd = __any_sync(FULL, odd);
            if ((threadIdx.x & 31) == 0) part[96 + warp] = peak, part[128 + warp] = peak_z, part[160 + warp] = odd ? 1.0f : 0.0f;
        }
        block_join<THREADS>(a, c, part);
        peak = -INFINITY, peak_z = -3.402823466e38f, odd = false;
#pragma unroll 1
        for (int i = 0; i < THREADS / 32 && i * 32 < K; ++i) {
            peak = fmaxf(peak, part[96 + i]);
            peak_z = fmaxf(peak_z, part[128 + i]);
            odd |= part[160 + i] != 0.0f;
        }
        live = odd || peak != -INFINITY;
    }
    // with the cluster's other blocks
    __device__ __forceinline__ void join_cluster(cg::cluster_group &cluster, float c, float *own)
    {
        if (threadIdx.x == 0) own[0] = a.m, own[1] = a.s, own[2] = repeated ? 1.0f : 0.0f;
        cluster.sync();
        a = Stat<false>();
#pragma unroll 1
        for (int b = 0; b < (int)cluster.num_blocks(); ++b) {
            const float *o = cluster.map_shared_rank(own, b);
            a.join(o[0], o[1], 0.0f, c);
            repeated |= o[2] != 0.0f;
        }
    }
    // the same without a barrier of the cluster, which would wait for the stores of the row before: every block sends its
    // numbers to every block, 16 bytes each, that complete on `bar`; `own` holds 4 * MAX_CLUSTER floats.  With them goes
    // whether a wait of the block has run out, so that all blocks stop after the same row, with no numbers on their way;
    // true then
    template <typename In>
    __device__ __forceinline__ bool exchange(In &in, int blocks, int rank, float c, float *own, uint64_t *bar, unsigned parity,
                                             bool stop)
    {
        if (threadIdx.x == 0) bar_expect(bar, 16 * blocks);
        if ((int)threadIdx.x < blocks)
            send_async(own + 4 * rank, bar, threadIdx.x, a.m, a.s, repeated ? 1.0f : 0.0f, stop ? 1.0f : 0.0f);
        in.wait_blocks(bar, parity);
        stop = in.gave_up;
        a = Stat<false>();
#pragma unroll 1
        for (int b = 0; b < blocks; ++b) {
            a.join(own[4 * b], own[4 * b + 1], 0.0f, c);
            repeated |= own[4 * b + 2] != 0.0f;
            stop |= own[4 * b + 3] != 0.0f;
        }
        return stop;
    }
    // sums over the slots: the teacher's weights and, with the bucket, the student's exponentials; `part` holds 64 floats;
    // one barrier
    template <int THREADS>
    __device__ __forceinline__ void sum_slots(const Slots &S, int K, float teacher_lse, float c, float *part)
    {
        m = BUCKET ? fmaxf(a.m, peak_z) : a.m;
        base = BUCKET ? teacher_lse : peak == -INFINITY ? 0.0f : peak;
        logt = 0.0f;
        float sums[BUCKET ? 2 : 1] = {};
#pragma unroll 1
        for (int k = threadIdx.x; k < K; k += THREADS) {
            sums[0] = __fadd_rn(sums[0], q(S, k));
            if (BUCKET && S.id[k] >= 0 && first_of(S, k)) sums[1] = __fadd_rn(sums[1], ex2(__fmul_rn(__fsub_rn(S.z[k], m), c)));
        }
        block_sums<THREADS>(sums, part);
        rest = 0.0f, lift = 1.0f, in_slots = 0.0f, s = a.s;
        if (BUCKET) {
            rest = __fsub_rn(1.0f, sums[0]);
            if (rest <= LEAST_REST) rest = 0.0f;
            lift = ex2(__fmul_rn(__fsub_rn(a.m, m), c));
            in_slots = sums[BUCKET ? 1 : 0];
            s = __fmaf_rn(a.s, lift, in_slots);
        } else {
            logt = logf(sums[0]);
        }
    }
    // the row's loss, by one warp
    __device__ __forceinline__ float loss(const Slots &S, int K, float temperature, float inv) const
    {
        // slot by slot: the sums of q log q and q x alone are many times their difference
        const float logs = logf(s);
        float kl = 0.0f;
#pragma unroll 1
        for (int k = threadIdx.x & 31; k < K; k += 32) {
            const float p = q(S, k), x = __fmaf_rn(__fsub_rn(S.z[k], m), inv, -logs);
            if (p != 0.0f) kl = __fmaf_rn(p, __fsub_rn(logq(S, k), x), kl);
        }
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) kl = __fadd_rn(kl, __shfl_xor_sync(FULL, kl, off));
        if (BUCKET && rest > 0.0f) {
            // ln(q_t / p_t): of the quotient, near 1 as a rule; by logarithms where p_t is out of fp32's range
            const float out = __fmul_rn(a.s, lift), p_t = __fdiv_rn(out, __fadd_rn(out, in_slots));
            const float ratio = p_t > 1e-30f ? logf(__fdiv_rn(rest, p_t))
                                             : __fsub_rn(logf(rest), __fadd_rn(__fsub_rn(logf(a.s), logs),
                                                                              __fmul_rn(__fsub_rn(a.m, m), inv)));
            kl = __fmaf_rn(rest, ratio, kl);
        }
        if (kl == INFINITY && temperature < 1.0f && live && s != 0.0f)
            return loss_of_lowest(S.t, S.z, K, temperature, base, logt, m, logs, BUCKET ? rest : 0.0f, a.m, logf(a.s));
        return !live ? 0.0f : s == 0.0f ? INFINITY : __fmul_rn(__fmul_rn(temperature, temperature), kl);
    }
};

// ------------------------------------------------------------------ the loss alone: a cluster per row
// Shared memory: the slots, then (bucket) the marks.
template <typename T, bool BUCKET, int THREADS>
__global__ __launch_bounds__(THREADS, 1024 / THREADS) void k_distill_loss(const T *logits, int cols,
                                                                          int64_t stride, Teacher teach, float temperature,
                                                                          float *__restrict__ loss, int map_bytes,
                                                                          int bit_bytes, int *status)
{
    constexpr int E = Vec<T>::E;
    after_previous();
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float part[192], part2[64], own[4];
    __shared__ int twice;
    __shared__ unsigned edge_map;
    const int K = teach.K;
    const Slots S(smem, K);
    unsigned *map = reinterpret_cast<unsigned *>(smem + ((size_t)K * SLOT_BYTES + 15) / 16 * 16);
    const Marks marks{map, map + bit_bytes / 4, &edge_map};
    cg::cluster_group cluster = cg::this_cluster();
    const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int64_t r = blockIdx.x / (unsigned)blocks;
    const T *row = logits + r * stride;
    const Share sh = share_of(row, cols, rank, blocks);
    const uint4 *body = reinterpret_cast<const uint4 *>(row + sh.b0);
    const int n_vec = sh.v1 - sh.v0;
    const float inv = __fdiv_rn(1.0f, temperature), c = __fmul_rn(inv, LOG2E);

    RawSlot slot = {};
    if ((int)threadIdx.x < K) slot.fetch(teach, r, threadIdx.x);
    uint4 x[UNROLL];
    load_vectors<T, THREADS, 32>(x, body, 0, lane_start(), n_vec);
    const bool has_edge = (int)threadIdx.x < sh.edges();
    T z_edge = from_float<T>(0.0f);
    if (has_edge) z_edge = row[sh.edge(threadIdx.x)];
    const float teacher_lse = BUCKET ? teach.lse[r] : 0.0f;
    if (threadIdx.x == 0) twice = 0, edge_map = 0;
    if (BUCKET) {
#pragma unroll 1
        for (int i = threadIdx.x; i < map_bytes / 16; i += THREADS) reinterpret_cast<uint4 *>(map)[i] = uint4{0, 0, 0, 0};
        __syncthreads();
    }
    Row<BUCKET> R;
    R.peak = -INFINITY, R.peak_z = -3.402823466e38f, R.odd = false;
    uint4 around = {0, 0, 0, 0};        // of slot threadIdx.x: used when the pass is over
#pragma unroll 1
    for (int k = threadIdx.x; k < K; k += THREADS) {
        if (k >= THREADS) slot.fetch(teach, r, k);
        const int j = slot.token(teach, cols, rank == 0, status);
        const float t = j < 0 ? -INFINITY : slot.logit(teach, inv);
        S.id[k] = j, S.t[k] = t;
        R.odd |= t != t;
        R.peak = fmaxf(R.peak, t);
        if (BUCKET && marks.set<E>(sh, j)) twice = 1;
        if (k < THREADS && j >= 0) around = fetch_around(row, sh, j);
    }
    if (BUCKET) __syncthreads();
    float unused = 0.0f;
    for (int base = 0; base < n_vec; base += THREADS * UNROLL) {
        uint4 next[UNROLL];
        load_vectors<T, THREADS, 32>(next, body, base + THREADS * UNROLL, lane_start(), n_vec);
        if (BUCKET) marks.leave_out<T>(x, base);
        add_vectors<T, false>(R.a, x, c, unused);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) x[u] = next[u];
    }
    if (has_edge && !(BUCKET && (edge_map >> threadIdx.x & 1))) add_element(R.a, to_float(z_edge), c);
    R.repeated = twice;
#pragma unroll 1
    for (int k = threadIdx.x; k < K; k += THREADS) {
        const int j = S.id[k];
        if (k >= THREADS && j >= 0) around = fetch_around(row, sh, j);
        const float z = j < 0 ? -INFINITY : logit_in<T>(around, sh, j);
        S.z[k] = z;
        R.peak_z = fmaxf(R.peak_z, z);
        if (BUCKET) R.template add_around<T>(S, marks, sh, k, around, c);
    }
    R.template join<THREADS>(c, K, part);
    if (blocks > 1) R.join_cluster(cluster, c, own);
    R.template sum_slots<THREADS>(S, K, teacher_lse, c, part2);
    if (rank == 0 && threadIdx.x < 32) {
        const float value = R.loss(S, K, temperature, inv);
        if (threadIdx.x == 0) loss[r] = value;
    }
    if (blocks > 1) cluster.sync();     // every block's shared memory has been read
}

// ------------------------------------------------------------------ loss and gradient: persistent clusters
// Per row: the pass for the statistics, their join (a barrier), the slots' sums (a barrier), the pass that writes
// the gradient, and after the barrier that opens the next row the slots' own elements.  The next row's slots
// are read and marked, and its student logits fetched, before the second pass.
// Shared memory: the slots of two rows in turn, the marks, the stream's places.
// An SM's blocks are at different places of the kernel at any time, so its size counts: with the loops whose length is not known
// left rolled it is 54 KB, and 8000 x 32,000 bf16 take 176 us; unrolled by the compiler's choice 97 KB and 219 us.

template <typename T, bool BUCKET, int THREADS>
__global__ __launch_bounds__(THREADS + 32, blocks_per_sm(THREADS)) void k_distill_grad(
    const T *logits, int64_t rows, int cols, int64_t stride, Teacher teach, float temperature, float *loss,
    const float *weight, T *dlogits, int64_t out_stride, int slots, int hold, int map_bytes, int bit_bytes,
    unsigned tries, int *status)
{
    constexpr int E = Vec<T>::E;
    constexpr uint32_t NEG_INF = Vec<T>::NEG_INF;
    after_previous();
    using In = Stream<T, THREADS>;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float part[2][192], part2[2][64];
    __shared__ __align__(16) float own[2][4 * MAX_CLUSTER];
    __shared__ int twice[2];
    __shared__ int stopped;             // a wait has run out: the row under work is the last
    __shared__ unsigned edge_map[2];
    __shared__ uint64_t bars[2 * MOST_SLOTS], joined[2];
    const int K = teach.K;
    unsigned *map = reinterpret_cast<unsigned *>(smem + ((size_t)K * SLOT_BYTES * 2 + 15) / 16 * 16);
    cg::cluster_group cluster = cg::this_cluster();
    const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int64_t first = blockIdx.x / (unsigned)blocks, step = gridDim.x / (unsigned)blocks;
    const float inv = __fdiv_rn(1.0f, temperature), c = __fmul_rn(inv, LOG2E);

    if (threadIdx.x == 0) bar_init(&joined[0], 1), bar_init(&joined[1], 1);
    In in;
    in.start(reinterpret_cast<uint4 *>(reinterpret_cast<unsigned char *>(map) + map_bytes), bars, slots, hold, tries,
             status);
#pragma unroll 1
    for (int i = threadIdx.x; i < map_bytes / 16; i += THREADS + 32) reinterpret_cast<uint4 *>(map)[i] = uint4{0, 0, 0, 0};
    if (threadIdx.x < 2) twice[threadIdx.x] = 0, edge_map[threadIdx.x] = 0;
    if (threadIdx.x == 0) stopped = 0;

    if (blocks > 1) cluster.sync();     // every block's barriers are there
    else __syncthreads();               // the map is clear
    if (threadIdx.x >= THREADS) {
        if (threadIdx.x == THREADS) in.bring_rows(logits, stride, rows, cols, first, step, rank, blocks);
        __syncwarp();
        if (blocks > 1) cluster.sync();
        return;
    }
    // a row's numbers, fetched a row ahead; its first THREADS slots two rows ahead
    RawSlot slot = {};
    auto fetch_slots = [&](int64_t r) {
        if (r < rows && (int)threadIdx.x < K) slot.fetch(teach, r, threadIdx.x);
    };
    float teacher_lse = 0.0f, w = 1.0f;
    T z_edge = from_float<T>(0.0f);
    uint4 around = {0, 0, 0, 0};
    Row<BUCKET> R;
    float peak = -INFINITY;
    bool odd = false;
    auto open_row = [&](int64_t r, int turn) {
        const T *row = logits + r * stride;
        const Share sh = share_of(row, cols, rank, blocks);
        const Slots S(smem + turn * SLOT_BYTES * K, K);
        const Marks marks{map, map + bit_bytes / 4, &edge_map[turn]};
        peak = -INFINITY, odd = false;
#pragma unroll 1
        for (int k = threadIdx.x; k < K; k += THREADS) {
            RawSlot here = slot;
            if (k >= THREADS) here.fetch(teach, r, k);
            const int j = here.token(teach, cols, rank == 0, status);
            const float t = j < 0 ? -INFINITY : here.logit(teach, inv);
            S.id[k] = j, S.t[k] = t;
            odd |= t != t;
            peak = fmaxf(peak, t);
            if (marks.set<E>(sh, j)) twice[turn] = 1;
            if (k < THREADS && j >= 0) around = fetch_around(row, sh, j);
        }
        if ((int)threadIdx.x < sh.edges()) z_edge = row[sh.edge(threadIdx.x)];
        teacher_lse = BUCKET ? teach.lse[r] : 0.0f;
        w = weight ? weight[r] : 1.0f;
        fetch_slots(r + step);
    };
    // the slots' own elements of row r, when the rest of the row is written
    float wt = 0.0f, one = 0.0f;
    bool zero = true;
    auto write_slots = [&](int64_t r, int turn) {
        const Share sh = share_of(logits + r * stride, cols, rank, blocks);
        const Slots S(smem + turn * SLOT_BYTES * K, K);
#pragma unroll 1
        for (int k = threadIdx.x; k < (zero ? 0 : K); k += THREADS) {
            const int j = S.id[k];
            if (j < sh.j0 || j >= sh.j1 || !R.first_of(S, k)) continue;
            float q = 0.0f;
#pragma unroll 1
            for (int i = k; i < (R.repeated ? K : k + 1); ++i)
                if (S.id[i] == j) q = __fadd_rn(q, R.q(S, i));
            const float p = __fmul_rn(ex2(__fmul_rn(__fsub_rn(S.z[k], R.m), c)), one);
            dlogits[r * out_stride + j] = from_float<T>(__fmul_rn(wt, __fsub_rn(p, q)));
        }
    };
    fetch_slots(first);
    if (first < rows) open_row(first, 0);

    int turn = 0;
    unsigned joins = 0;                 // rows joined so far
    bool stop = false;                  // the same on all threads, and with the blocks' exchange on all blocks
#pragma unroll 1
    for (int64_t r = first; r < rows && !stop; r += step, turn ^= 1) {
        team_sync<THREADS>();           // the marks are set; the row before is written
        if (threadIdx.x == 0) twice[turn ^ 1] = 0, edge_map[turn ^ 1] = 0;
        if (r != first) write_slots(r - step, turn ^ 1);
        const T *row = logits + r * stride;
        const Share sh = share_of(row, cols, rank, blocks);
        const Slots S(smem + turn * SLOT_BYTES * K, K);
        const Marks marks{map, map + bit_bytes / 4, &edge_map[turn]};
        const bool has_edge = (int)threadIdx.x < sh.edges();
        const float lse = teacher_lse, w_own = w;
        const T z_own_edge = z_edge;
        R.a = Stat<false>();
        const int n_vec = sh.v1 - sh.v0, passing = in.passing(n_vec);
        int chunks = 0;
        float unused = 0.0f;
#pragma unroll 1
        for (int base = 0;; ) {
            const int p = in.take();
            uint4 x[UNROLL];
            in.read(x, p);
            if (base + In::SPAN > n_vec)
#pragma unroll
                for (int u = 0; u < UNROLL; ++u)
                    if (base + lane_start() + u * 32 >= n_vec) x[u] = uint4{NEG_INF, NEG_INF, NEG_INF, NEG_INF};
            if (BUCKET) marks.leave_out<T>(x, base);
            add_vectors<T, false>(R.a, x, c, unused);
            if (chunks < passing) in.give_back(p);
            ++chunks;
            base += In::SPAN;
            if (base >= n_vec) break;
        }
        if (has_edge && !(BUCKET && (edge_map[turn] >> threadIdx.x & 1))) add_element(R.a, to_float(z_own_edge), c);
        R.repeated = twice[turn];
        R.peak = peak, R.peak_z = -3.402823466e38f, R.odd = odd;
#pragma unroll 1
        for (int k = threadIdx.x; k < K; k += THREADS) {
            const int j = S.id[k];
            if (k >= THREADS && j >= 0) around = fetch_around(row, sh, j);
            const float z = j < 0 ? -INFINITY : logit_in<T>(around, sh, j);
            S.z[k] = z;
            R.peak_z = fmaxf(R.peak_z, z);
            if (BUCKET) R.template add_around<T>(S, marks, sh, k, around, c);
        }
        if (in.gave_up) stopped = 1;
        R.template join<THREADS>(c, K, part[turn]);
#pragma unroll 1
        for (int k = threadIdx.x; k < K; k += THREADS) marks.clear<E>(sh, S.id[k]);          // for the next row
        if (blocks > 1 &&
            R.exchange(in, blocks, rank, c, own[turn], &joined[turn], joins++ >> 1 & 1, *(volatile int *)&stopped != 0))
            stopped = 1;
        R.template sum_slots<THREADS>(S, K, lse, c, part2[turn]);
        stop = *(volatile int *)&stopped != 0;      // not written again before the next row's first barrier
        if (loss && rank == 0 && threadIdx.x >= THREADS - 32) {
            const float value = R.loss(S, K, temperature, inv);
            if (threadIdx.x == THREADS - 1) loss[r] = value;
        }
        // The second pass.  Outside of the slots p_j - q_t p_j / p_t = 2^x_j factor / (w T), x_j relative to the outside's
        // own maximum, so that neither p_j nor p_t need be representable.
        zero = w_own == 0.0f || !R.live || R.s == 0.0f;
        wt = __fmul_rn(w_own, temperature);
        // A NaN among the student's logits or the teacher's is one in the whole row: the teacher's shows in the rest or in the
        // slots' sum alone, and one in a slot not outside of the slots where nothing is left there
        const float known = __fadd_rn(R.s, BUCKET ? R.rest : R.logt);
        one = known != known ? known : __fdiv_rn(1.0f, R.s);
        const float factor =
            BUCKET ? (R.a.s == 0.0f ? __fmul_rn(0.0f, one)
                                    : __fmul_rn(wt, __fsub_rn(__fmul_rn(R.lift, one), __fdiv_rn(R.rest, R.a.s))))
                   : __fmul_rn(wt, one);
        T *drow = dlogits + r * out_stride, *dbody = drow + sh.b0;
        if (has_edge) {
            const float x = __fmul_rn(ex2(__fmul_rn(__fsub_rn(to_float(z_own_edge), R.a.m), c)), factor);
            drow[sh.edge(threadIdx.x)] = from_float<T>(zero ? 0.0f : x);
        }
        if (r + step < rows) open_row(r + step, turn ^ 1);
        const uint64_t m2 = pair(-R.a.m, -R.a.m), c2 = pair(c, c), f2 = pair(factor, factor);
        // element by element where dlogits is not aligned as the logits are, and for rows of zeros whatever they hold
        const bool aligned = ((uintptr_t)dbody & 15) == 0;
        auto write_any = [&](const uint4 &x, int i) {
            float f[E];
            Vec<T>::unpack(x, f);
#pragma unroll
            for (int e = 0; e < E; ++e) f[e] = zero ? 0.0f : __fmul_rn(ex2(__fmul_rn(__fsub_rn(f[e], R.a.m), c)), factor);
            if (aligned) {
                __stcs(reinterpret_cast<uint4 *>(dbody) + i, Vec<T>::pack(f));
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) dbody[i * E + e] = from_float<T>(f[e]);
            }
        };
        // 16-bit results: (z - m) c by one fused operation, whose m c is rounded to 2^-16 at most, against half a
        // unit of 2^-12 of the result; m is the row's, so that only rows of logits beyond 170 take the general form
        const bool fused = sizeof(T) == 2 && fabsf(R.a.m) * c < 256.0f;
        const uint64_t mc2 = fused ? pair(-__fmul_rn(R.a.m, c), -__fmul_rn(R.a.m, c)) : 0;
        auto write = [&](const uint4 &x, int i) {
            float f[E];
            Vec<T>::unpack(x, f);
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                float x0, x1;
                const uint64_t z = pair(f[e], f[e + 1]);
                unpair(sizeof(T) == 2 ? fma2(z, c2, mc2) : mul2(add2(z, m2), c2), x0, x1);
                unpair(mul2(pair(ex2(x0), ex2(x1)), f2), f[e], f[e + 1]);
            }
            __stcs(reinterpret_cast<uint4 *>(dbody) + i, Vec<T>::pack(f));
        };
        const bool plain = !zero && (fused || sizeof(T) == 4) && aligned;
        // the held chunks first, while the others are brought again
        const int held = chunks - passing;
#pragma unroll 1
        for (int n = 0; n < chunks; ++n) {
            const int p = n < held ? in.before(held - n) : in.take();
            const int base = (n < held ? passing + n : n - held) * In::SPAN, i = base + lane_start();
            if (plain && base + In::SPAN <= n_vec) {
                uint4 x[UNROLL];
                in.read(x, p);
#pragma unroll
                for (int u = 0; u < UNROLL; ++u) write(x[u], i + u * 32);
            } else {
#pragma unroll 1
                for (int u = 0; u < UNROLL && i + u * 32 < n_vec; ++u) write_any(in.read_one(p, u), i + u * 32);
            }
            in.give_back(p);
        }
    }
    team_sync<THREADS>();
    if (first < rows && !stop) {
        const int64_t last = first + (rows - 1 - first) / step * step;
        write_slots(last, turn ^ 1);
    }
    if (blocks > 1) cluster.sync();      // nothing is on its way to this block's shared memory any more
}

}  // namespace

namespace {

// asked at a device's first call with gradient, then kept: 16 queries
Room room_of(int device, int sms)
{
    static std::mutex lock;
    static bool known[64];
    static Room rooms[64];
    std::lock_guard<std::mutex> guard(lock);
    const bool kept = device >= 0 && device < 64;
    if (kept && known[device]) return rooms[device];
    Room room = {};
    const auto kernel = k_distill_grad<__nv_bfloat16, true, 256>;
    if (!allow_smem((const void *)kernel)) return room;
    cudaLaunchAttribute at = {};
    at.id = cudaLaunchAttributeClusterDimension;
    cudaLaunchConfig_t cfg = {};
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    for (int i = 0; i <= Room::ALONE; ++i)
        for (int log = 0; log < 4; ++log) {
            const int threads = i == Room::ALONE ? 256 : 256 >> i;
            at.val.clusterDim.x = 1u << log;
            at.val.clusterDim.y = at.val.clusterDim.z = 1;
            cfg.gridDim = dim3((unsigned)sms * 8);
            cfg.blockDim = dim3(threads + 32);
            cfg.dynamicSmemBytes = block_smem(i == Room::ALONE ? 1 : blocks_per_sm(threads));
            int n = 0;
            if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess) room.clusters[i][log] = n;
            else cudaGetLastError();
        }
    if (kept && room.clusters[0][0] > 0) rooms[device] = room, known[device] = true;
    return room;
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
    if (!(temperature > 0.0f) || !usable_scale(1.0f / temperature) || std::isinf(temperature * temperature)) return PDB_EINVAL;
    if (dlogits && (dlogits->rows != logits->rows || dlogits->cols != logits->cols || dlogits->type != logits->type ||
                    !same_or_apart(logits, dlogits)))
        return PDB_EINVAL;
    if (logits->cols > MAX_COLS) return PDB_ETOOBIG;
    if (logits->rows == 0) return PDB_OK;
    if ((rc = check_device(t)) != PDB_OK) return rc;
    cudaStream_t s = (cudaStream_t)stream;
    TokensUse use{t, s};
    const Teacher teach{ids_of(top_ids), top_logits->data, top_logits->type, (int)top_logits->cols, stride_of(top_logits),
                        teacher_lse};
    return with_type(logits->type, [&](auto *a) {
        using T = std::remove_pointer_t<decltype(a)>;
        if (!dlogits) {
            const size_t slot_bytes = ((size_t)teach.K * SLOT_BYTES + 15) / 16 * 16;
            const Shape shape = once_shape(logits->rows, logits->cols, Vec<T>::E, t->sms, slot_bytes, teacher_lse != nullptr);
            return with_threads(shape.threads, [&](auto n) {
                constexpr int N = decltype(n)::value;
                return launch_rows(teacher_lse ? k_distill_loss<T, true, N> : k_distill_loss<T, false, N>, shape, s,
                                   (const T *)logits->data, (int)logits->cols, stride_of(logits), teach, temperature, loss,
                                   shape.map_bytes, shape.bit_bytes, t->status);
            });
        }
        const size_t slot_bytes = ((size_t)teach.K * SLOT_BYTES * 2 + 15) / 16 * 16;
        Shape shape = twice_shape(logits->rows, logits->cols, Vec<T>::E, room_of(t->device, t->sms), slot_bytes, teach.K);
        if (shape.clusters < 1) return PDB_ECUDA;
        const auto run = [&](auto n) {
            constexpr int N = decltype(n)::value;
            shape.threads = N + 32;     // and the warp that brings the rows
            return launch_rows(teacher_lse ? k_distill_grad<T, true, N> : k_distill_grad<T, false, N>, shape, s,
                               (const T *)logits->data, logits->rows, (int)logits->cols, stride_of(logits), teach,
                               temperature, loss, weight, (T *)dlogits->data, stride_of(dlogits), shape.slots, shape.hold,
                               shape.map_bytes, shape.bit_bytes, t->tries, t->status);
        };
        return shape.threads == 64 ? run(Num<64>()) : shape.threads == 128 ? run(Num<128>()) : run(Num<256>());
    });
}
