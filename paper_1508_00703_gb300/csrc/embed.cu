// Rows of a table by token id, and the table's gradient by sorted ids
// (pdb_embed, pdb_embed_grad), and the handle of the token operators.
#include <algorithm>
#include <mutex>
#include <new>
#include <set>
#include <utility>

#include "tokens.cuh"

using namespace pdb;

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
template <>
struct Raw<16> { using type = uint4; };
template <>
struct Raw<32> { struct type { uint4 a, b; }; };

template <typename T, int E>
struct alignas(E * sizeof(T) < 16 ? E * sizeof(T) : 16) Pack {
    T e[E];
};

template <typename T, int E>
__device__ __forceinline__ Pack<T, E> load_pack(const T *p)
{
    Pack<T, E> v;
    if constexpr (E * sizeof(T) == 32) {
        reinterpret_cast<uint4 *>(&v)[0] = reinterpret_cast<const uint4 *>(p)[0];
        reinterpret_cast<uint4 *>(&v)[1] = reinterpret_cast<const uint4 *>(p)[1];
    } else {
        using R = typename Raw<E * sizeof(T)>::type;
        *reinterpret_cast<R *>(&v) = *reinterpret_cast<const R *>(p);
    }
    return v;
}
template <typename T, int E>
__device__ __forceinline__ void store_pack(T *p, const Pack<T, E> &v)
{
    if constexpr (E * sizeof(T) == 32) {
        __stcs(reinterpret_cast<uint4 *>(p), reinterpret_cast<const uint4 *>(&v)[0]);
        __stcs(reinterpret_cast<uint4 *>(p) + 1, reinterpret_cast<const uint4 *>(&v)[1]);
    } else if constexpr (E * sizeof(T) == 16) {
        __stcs(reinterpret_cast<uint4 *>(p), *reinterpret_cast<const uint4 *>(&v));
    } else {
        using R = typename Raw<E * sizeof(T)>::type;
        *reinterpret_cast<R *>(p) = *reinterpret_cast<const R *>(&v);
    }
}

// whether E elements of each row can be moved as one piece of up to 16 bytes
inline bool fits(const pdb_mat *m, int E)
{
    const int bytes = std::min(16, E * type_bytes(m->type));
    return m->cols % E == 0 && (uintptr_t)m->data % bytes == 0 &&
           (m->rows < 2 || m->stride * type_bytes(m->type) % bytes == 0);
}

// ------------------------------------------------------------------ lookup
// A warp moves one piece of LOOKUP_UNROLL * 32 packs of one row: all its loads are issued before the
// first store.  Bound by memory; the id's and the row's latency are covered by the other warps.
constexpr int LOOKUP_UNROLL = 4;

template <typename T, typename O, int E>
__global__ __launch_bounds__(256) void k_embed(const T *__restrict__ table, int64_t vocab, int64_t stride, Ids ids,
                                               int64_t n, int dim, int pieces, float scale, int64_t pad,
                                               O *__restrict__ out, int64_t out_stride, int *status)
{
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
__device__ __forceinline__ uint32_t embed_key(Ids ids, int64_t i, int64_t vocab, int64_t pad, int *status)
{
    const int64_t v = load_id(ids, i);
    const bool there = v != pad && v >= 0 && v < vocab;
    if (!there && v != pad) set_status(status, PDB_ERANGE);
    return there ? (uint32_t)v : (uint32_t)vocab;
}

__global__ void k_embed_keys(Ids ids, int64_t n, int64_t vocab, int64_t pad, uint32_t *__restrict__ key, int *status)
{
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) key[i] = embed_key(ids, i, vocab, pad, status);
}

// Up to RANK_MAX ids: each id's place is the number of smaller ids and of equal ones before it,
// counted against all of them in shared memory, in one launch.  A block places RANK_IDS ids, its
// threads in RANK_SLICES slices of the others.
constexpr int RANK_MAX = 8192, RANK_IDS = 64, RANK_SLICES = 8, RANK_THREADS = RANK_IDS * RANK_SLICES;

__global__ __launch_bounds__(RANK_THREADS) void k_embed_rank(Ids ids, int n, int64_t vocab, int64_t pad,
                                                             uint32_t *__restrict__ skey, int32_t *__restrict__ spos,
                                                             int *status)
{
    extern __shared__ __align__(16) uint32_t s_key[];       // n, rounded up to 4 * RANK_SLICES
    __shared__ int count[RANK_IDS];
    const int padded = (n + 4 * RANK_SLICES - 1) / (4 * RANK_SLICES) * (4 * RANK_SLICES);
    for (int i = threadIdx.x; i < padded; i += RANK_THREADS)
        s_key[i] = i < n ? embed_key(ids, i, vocab, pad, status) : 0xffffffffu;   // the fill counts for nobody
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

// ------------------------------------------------------------------ sums of runs
// The sorted positions are cut into pieces of 32.  A warp sums one piece of 32 * E columns:
// its rows are loaded SUM_UNROLL at a time, a run of equal ids that lies in the piece is written at once, and
// what belongs to a run that crosses the piece's bounds is left in `part`: row 2b for the run that comes
// into piece b from before, row 2b + 1 for one that starts in b and goes on.  k_embed_join
// adds those in order.  So the work is even whatever the ids: a hot id of 6000 rows is 190 pieces.
// Bound by memory: each row is read once, each result written once, and `part` is at most
// 1/8 (fp32 rows) or 1/4 (16-bit rows) of the rows' bytes again, for runs that cross only.
constexpr int PIECE = 32, SUM_UNROLL = 8, SUM_WARPS = 8;

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
__device__ __forceinline__ int64_t keys_below(const uint32_t *__restrict__ key, int64_t n, uint32_t v)
{
    const int lane = threadIdx.x & 31;
    int64_t lo = 0, hi = n;              // the answer lies in [lo, hi]
    while (lo < hi) {
        const int64_t step = (hi - lo + 31) / 32, at = lo + lane * step;
        const int below = __popc(__ballot_sync(FULL, at < hi && key[at] < v));
        // probes 0 .. below - 1 are below v
        hi = min64(hi, lo + below * step);
        if (below) lo = lo + (below - 1) * step + 1;
    }
    return lo;
}

// zeros in the rows of 32 ids from v0 on that do not occur
template <typename O, int E>
__device__ __forceinline__ void zero_rows(const uint32_t *__restrict__ key, int64_t n, int64_t vocab, int64_t v0,
                                          O *__restrict__ dtable, int64_t stride, int dim)
{
    const int lane = threadIdx.x & 31;
    const int64_t v = v0 + lane;
    int64_t lo = keys_below(key, n, (uint32_t)v0), hi = keys_below(key, n, (uint32_t)min64(vocab, v0 + 32));
    const int64_t end = hi;
    while (lo < hi) {                    // each lane its own id, between the two
        const int64_t mid = (lo + hi) >> 1;
        if (key[mid] < (uint32_t)v) lo = mid + 1;
        else hi = mid;
    }
    unsigned absent = __ballot_sync(FULL, v < vocab && !(lo < end && key[lo] == (uint32_t)v));
    Pack<O, E> zero;
#pragma unroll
    for (int e = 0; e < E; ++e) zero.e[e] = from_float<O>(0.0f);
    while (absent) {
        O *row = dtable + (v0 + __ffs(absent) - 1) * stride;
        absent &= absent - 1;
        for (int j = lane * E; j < dim; j += 32 * E) store_pack<O, E>(row + j, zero);
    }
}

template <typename T, typename O, int E, bool ACC>
__global__ __launch_bounds__(SUM_WARPS * 32) void k_embed_sum(const uint32_t *__restrict__ key,
                                                              const int32_t *__restrict__ pos, int64_t n, int64_t vocab,
                                                              const T *__restrict__ dout, int64_t stride, int dim,
                                                              int tiles, int64_t sum_blocks, float scale,
                                                              O *__restrict__ dtable, int64_t out_stride,
                                                              float *__restrict__ part)
{
    const int lane = threadIdx.x & 31;
    if (blockIdx.x >= sum_blocks) {      // without ACC: the rows of ids that do not occur
        const int64_t group = (blockIdx.x - sum_blocks) * SUM_WARPS + (threadIdx.x >> 5);
        if (group * 32 < vocab) zero_rows<O, E>(key, n, vocab, group * 32, dtable, out_stride, dim);
        return;
    }
    const int64_t w = (int64_t)blockIdx.x * SUM_WARPS + (threadIdx.x >> 5);
    const int64_t piece = w / tiles;
    const int64_t p0 = piece * PIECE;
    if (p0 >= n) return;
    const int col = (int)(w - piece * tiles) * 32 * E + lane * E;
    const bool on = col < dim;
    const int count = (int)min64(PIECE, n - p0);
    const uint32_t k = lane < count ? key[p0 + lane] : 0xffffffffu;
    const int32_t p = lane < count ? pos[p0 + lane] : 0;
    const uint32_t before = p0 > 0 ? key[p0 - 1] : 0xffffffffu, after = p0 + count < n ? key[p0 + count] : 0xffffffffu;
    const uint32_t left = __shfl_up_sync(FULL, k, 1);
    // positions that start a run; positions that end one within the piece or at its end
    const unsigned heads = __ballot_sync(FULL, lane < count && k != (lane == 0 ? before : left));
    const unsigned ends = (heads >> 1) | (1u << (count - 1));
    const uint32_t last = __shfl_sync(FULL, k, count - 1);
    const bool goes_on = last == after;
    int seen = count;                    // positions in front of the ids left out
    {
        const unsigned out = __ballot_sync(FULL, lane < count && k >= (uint32_t)vocab);
        if (out) seen = __ffs(out) - 1;
    }
    float sum[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = 0.0f;
    bool inside = heads & 1;             // the current run starts in this piece
    for (int i0 = 0; i0 < seen; i0 += SUM_UNROLL) {
        Pack<T, E> x[SUM_UNROLL];
        Pack<O, E> old[ACC ? SUM_UNROLL : 1];
        uint32_t id[SUM_UNROLL];
#pragma unroll
        for (int u = 0; u < SUM_UNROLL; ++u) {
            const int i = i0 + u;
            id[u] = __shfl_sync(FULL, k, i & 31);
            const int32_t row = __shfl_sync(FULL, p, i & 31);
            if (i < seen && on) {
                x[u] = load_pack<T, E>(dout + row * stride + col);
                if (ACC && (ends >> i & 1)) old[u] = load_pack<O, E>(dtable + (int64_t)id[u] * out_stride + col);
            }
        }
#pragma unroll
        for (int u = 0; u < SUM_UNROLL; ++u) {
            const int i = i0 + u;
            if (i >= seen) break;
            if (i > 0 && (heads >> i & 1)) {
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] = 0.0f;
                inside = true;
            }
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] = __fadd_rn(sum[e], to_float(x[u].e[e]));
            if ((ends >> i & 1) && on) {
                const bool crosses = !inside || (i == count - 1 && goes_on);
                if (crosses) {
                    Pack<float, E> y;
#pragma unroll
                    for (int e = 0; e < E; ++e) y.e[e] = sum[e];
                    float *at = part + (2 * piece + (inside ? 1 : 0)) * dim + col;
#pragma unroll
                    for (int e = 0; e < E; ++e) at[e] = y.e[e];
                } else {
                    write_sum<O, E, ACC>(dtable + (int64_t)id[u] * out_stride + col, sum, old[ACC ? u : 0], scale);
                }
            }
        }
    }
}

// runs that cross pieces: the block of the piece in which one starts adds its parts, in order
template <typename O, bool ACC>
__global__ __launch_bounds__(256) void k_embed_join(const uint32_t *__restrict__ key, int64_t n, int64_t vocab, int dim,
                                                    int tiles, float scale, O *__restrict__ dtable, int64_t out_stride,
                                                    const float *__restrict__ part)
{
    const int64_t piece = blockIdx.x / tiles;
    const int col = (int)(blockIdx.x - piece * tiles) * 256 + threadIdx.x;
    const int64_t next = (piece + 1) * PIECE;
    const uint32_t v = key[next - 1];
    // starts here and goes on
    if (v >= (uint32_t)vocab || key[next] != v || (piece > 0 && key[piece * PIECE] == v && key[piece * PIECE - 1] == v)) return;
    if (col >= dim) return;
    float sum[1] = {part[(2 * piece + 1) * dim + col]};
    for (int64_t b = piece + 1; b * PIECE < n && key[b * PIECE] == v; ++b)
        sum[0] = __fadd_rn(sum[0], part[2 * b * dim + col]);
    O *at = dtable + (int64_t)v * out_stride + col;
    Pack<O, 1> old;
    if (ACC) old.e[0] = *at;
    write_sum<O, 1, ACC>(at, sum, old, scale);
}

}  // namespace

namespace pdb {

bool allow_smem(const void *kernel)
{
    static std::mutex lock;
    static std::set<std::pair<const void *, int>> done;
    int device = 0, most = 0;
    cudaGetDevice(&device);
    std::lock_guard<std::mutex> guard(lock);
    if (done.count({kernel, device})) return true;
    cudaFuncAttributes at;
    const bool ok = cudaDeviceGetAttribute(&most, cudaDevAttrMaxSharedMemoryPerBlockOptin, device) == cudaSuccess &&
                    cudaFuncGetAttributes(&at, kernel) == cudaSuccess &&
                    cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         most - (int)at.sharedSizeBytes) == cudaSuccess;
    if (!ok) cudaGetLastError();
    else done.insert({kernel, device});
    return ok;
}

}  // namespace pdb

extern "C" {

void pdb_tokens_free(pdb_tokens *t)
{
    if (!t) return;
    if (t->ev_use) cudaEventSynchronize(t->ev_use);
    cudaStream_t s = own_stream();
    for (void *p : {(void *)t->status, (void *)t->key, (void *)t->skey, (void *)t->tkey, (void *)t->spos,
                    (void *)t->tpos, (void *)t->part})
        release(p, s);
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
    int rc = cudaEventCreateWithFlags(&t->ev_use, cudaEventDisableTiming) == cudaSuccess ? PDB_OK : PDB_ECUDA;
    rc = rc ? rc : alloc((void **)&t->status, 2 * sizeof(int), s);
    for (uint32_t **p : {&t->key, &t->skey, &t->tkey, (uint32_t **)&t->spos, (uint32_t **)&t->tpos})
        rc = rc ? rc : alloc((void **)p, sizeof(uint32_t) * max_tokens, s);
    // two rows of columns in fp32 for each piece of 32 ids
    rc = rc ? rc : alloc((void **)&t->part, sizeof(float) * 2 * ((max_tokens + PIECE - 1) / PIECE) * max_dim, s);
    rc = rc ? rc : fill_words(t->status, 0u, 2 * sizeof(int), s);
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
    int st = 0;
    if (read_words(&st, t->status, sizeof(int), (cudaStream_t)stream) != PDB_OK) return PDB_ECUDA;
    return st;
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
    cudaStream_t s = (cudaStream_t)stream;
    TokensUse use{t, s};
    const auto run = [&](auto *a, auto *b, auto e) {
        using T = std::remove_pointer_t<decltype(a)>;
        using O = std::remove_pointer_t<decltype(b)>;
        constexpr int E = decltype(e)::value;
        const int dim = (int)out->cols, pieces = (dim + LOOKUP_UNROLL * 32 * E - 1) / (LOOKUP_UNROLL * 32 * E);
        const int64_t blocks = std::min<int64_t>((out->rows * pieces + 7) / 8, (int64_t)1 << 24);
        k_embed<T, O, E><<<(unsigned)blocks, 256, 0, s>>>((const T *)table->data, table->rows, stride_of(table),
                                                          ids_of(ids), out->rows, dim, pieces, scale, pad,
                                                          (O *)out->data, stride_of(out), t->status);
        note_launch();
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
    return cudaPeekAtLastError() == cudaSuccess ? PDB_OK : PDB_ECUDA;
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
    cudaStream_t s = (cudaStream_t)stream;
    TokensUse use{t, s};
    const bool nothing = dim == 0 || vocab == 0;            // the ids are looked at all the same
    if (n > 0 && n <= RANK_MAX) {
        const size_t smem = sizeof(uint32_t) * ((n + 4 * RANK_SLICES - 1) / (4 * RANK_SLICES) * (4 * RANK_SLICES));
        k_embed_rank<<<(unsigned)((n + RANK_IDS - 1) / RANK_IDS), RANK_THREADS, smem, s>>>(ids_of(ids), (int)n, vocab, pad,
                                                                                          t->skey, t->spos, t->status);
        note_launch();
    } else if (n > 0) {
        k_embed_keys<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(ids_of(ids), n, vocab, pad, t->key, t->status);
        note_launch();
        if (!nothing)
            rc = radix_sort(t->key, nullptr, t->skey, t->spos, t->tkey, t->tpos, n, bits_for(vocab), t->status + 1, s);
    }
    if (rc != PDB_OK) return rc;
    if (nothing) return cudaPeekAtLastError() == cudaSuccess ? PDB_OK : PDB_ECUDA;
    const auto run = [&](auto *a, auto *b, auto e) {
        using T = std::remove_pointer_t<decltype(a)>;
        using O = std::remove_pointer_t<decltype(b)>;
        constexpr int E = decltype(e)::value;
        const int64_t pieces = (n + PIECE - 1) / PIECE;
        const int tiles = (dim + 32 * E - 1) / (32 * E);
        const int64_t sum_blocks = (pieces * tiles + SUM_WARPS - 1) / SUM_WARPS;
        const int64_t zero_blocks = accumulate ? 0 : ((vocab + 31) / 32 + SUM_WARPS - 1) / SUM_WARPS;
        if (sum_blocks + zero_blocks > 0) {
            const auto kernel = accumulate ? k_embed_sum<T, O, E, true> : k_embed_sum<T, O, E, false>;
            kernel<<<(unsigned)(sum_blocks + zero_blocks), SUM_WARPS * 32, 0, s>>>(
                t->skey, t->spos, n, vocab, (const T *)dout->data, stride_of(dout), dim, tiles, sum_blocks, scale,
                (O *)dtable->data, stride_of(dtable), t->part);
            note_launch();
        }
        if (pieces > 1) {
            const auto kernel = accumulate ? k_embed_join<O, true> : k_embed_join<O, false>;
            const int tiles = (dim + 255) / 256;
            kernel<<<(unsigned)((pieces - 1) * tiles), 256, 0, s>>>(t->skey, n, vocab, dim, tiles, scale,
                                                                    (O *)dtable->data, stride_of(dtable), t->part);
            note_launch();
        }
    };
    with_type(dout->type, [&](auto *a) {
        with_type(dtable->type, [&](auto *b) {
            constexpr int E = 16 / sizeof(*a);
            if (fits(dout, E) && fits(dtable, E)) run(a, b, Num<E>());
            else if (fits(dout, 2) && fits(dtable, 2)) run(a, b, Num<2>());
            else run(a, b, Num<1>());
        });
    });
    return cudaPeekAtLastError() == cudaSuccess ? PDB_OK : PDB_ECUDA;
}

}  // extern "C"
