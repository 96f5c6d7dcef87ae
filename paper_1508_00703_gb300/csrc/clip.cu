// The norm over many gradients, and their step clipped to it (pdb_clip_plan_build, pdb_clip).
//
//   N = sqrt(sum over all gradients of g^2),  f = N > max_norm ? max_norm / N : 1,  out = [out +] scale f g
//
// Two launches: the sum, then the step.  A plan cuts the matrices into pieces, which the blocks take in turn, so that one launch
// covers any number of gradients of any sizes, types and strides.  Bound by memory: 484 million bf16 gradients in 59 matrices, the step on fp32
// weights, 138 us for the sum (967 MB at 7.0 TB/s) and 705 us for the step (4.8 GB at 6.9 TB/s).  The second read of the gradients cannot be
// saved (none is scaled before all are summed) but for what L2 still holds, which the step therefore takes first: 102 million fp32 gradients
// into bf16, 61 and 99 us, where 615 MB read and written take 91 and 410 MB more 61.
#include <algorithm>
#include <climits>
#include <cmath>
#include <new>
#include <vector>

#include "pack.cuh"
#include "rows.cuh"

using namespace pdb;

namespace {

constexpr int CLIP_THREADS = 256, NORM_BLOCKS_PER_SM = 4, STEP_BLOCKS_PER_SM = 8;
constexpr int64_t MOST_ELEMENTS = (int64_t)1 << 40;           // more than the memory holds
constexpr int WIDE = 8;                 // elements moved at a time, where the alignment allows it

// rows x cols elements; of each row `head` elements, then whole packs of WIDE, then the rest (head = cols: all one by one)
struct ClipPiece {
    const void *g;
    void *out;
    int64_t g_stride, out_stride;
    int32_t rows, cols, head;
    int16_t g_type, out_type;
};

}  // namespace

struct pdb_clip_plan {
    int device, blocks, step_blocks;    // of the two launches
    int64_t n_pieces;
    ClipPiece *pieces;                  // device
    double *partial;                    // device: the blocks' sums
    pdb::Block arrays;                  // holds the device arrays
    cudaEvent_t ev_use;                 // recorded after the last work any call enqueued on the plan
};

namespace {

// pack(row, column) for a thread's packs of a piece, one(row, column) for its single elements
template <typename F, typename G>
__device__ __forceinline__ void each_of_piece(const ClipPiece &p, G pack, F one)
{
    const int packs = (p.cols - p.head) / WIDE, singles = p.cols - packs * WIDE;
    if (p.rows == 1) {
        for (int v = threadIdx.x; v < packs; v += CLIP_THREADS) pack(0, p.head + v * WIDE);
        for (int x = threadIdx.x; x < singles; x += CLIP_THREADS) one(0, x < p.head ? x : x + packs * WIDE);
    } else {
        for (int v = threadIdx.x; v < p.rows * packs; v += CLIP_THREADS) {
            const int r = v / packs;
            pack(r, p.head + (v - r * packs) * WIDE);
        }
        for (int v = threadIdx.x; v < p.rows * singles; v += CLIP_THREADS) {
            const int r = v / singles, x = v - r * singles;
            one(r, x < p.head ? x : x + packs * WIDE);
        }
    }
}

// vec(16 bytes of a thread's part of a gradient's piece), one(its single elements): the same part whatever they do with it
template <typename T, int U, typename F, typename G>
__device__ __forceinline__ void vectors_of_piece(const ClipPiece &p, F vec, G one)
{
    constexpr int E = Vec<T>::E;
    const T *g = (const T *)p.g;
    const int packs = (p.cols - p.head) / WIDE, singles = p.cols - packs * WIDE, row = packs * (WIDE / E);
    if (p.rows == 1) {
        const uint4 *body = reinterpret_cast<const uint4 *>(g + p.head);
        int i = threadIdx.x;
        if (U > 1)
            for (; i + (U - 1) * CLIP_THREADS < row; i += U * CLIP_THREADS) {
                uint4 v[U];
#pragma unroll
                for (int u = 0; u < U; ++u) v[u] = ld_keep(body + i + u * CLIP_THREADS);
#pragma unroll
                for (int u = 0; u < U; ++u) vec(v[u]);
            }
        for (; i < row; i += CLIP_THREADS) vec(ld_keep(body + i));
    } else {
        for (int i = threadIdx.x; i < p.rows * row; i += CLIP_THREADS) {
            const int r = i / row;
            vec(ld_keep(reinterpret_cast<const uint4 *>(g + r * p.g_stride + p.head) + (i - r * row)));
        }
    }
    for (int i = threadIdx.x; i < p.rows * singles; i += CLIP_THREADS) {
        const int r = i / singles, x = i - r * singles;
        one(to_float(g[r * p.g_stride + (x < p.head ? x : x + packs * WIDE)]));
    }
}

// A thread's sum of squares of a piece.  In 32 bits while that loses nothing: a sum that left fp32's range, or is so small that
// squares may have been lost below it, is formed again in 64.
template <typename T>
__device__ __forceinline__ double piece_squares(const ClipPiece &p)
{
    constexpr int E = Vec<T>::E;
    uint64_t pairs[2] = {0, 0};
    float more = 0.0f, lo, hi;
    uint32_t any = 0;                                 // bits of the magnitudes
    vectors_of_piece<T, 4>(
        p,
        [&](const uint4 &v) {
            float f[E];
            Vec<T>::unpack(v, f);
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const uint64_t x = pair(f[e], f[e + 1]);
                pairs[e >> 1 & 1] = fma2(x, x, pairs[e >> 1 & 1]);
            }
            any |= (v.x | v.y | v.z | v.w) & (sizeof(T) == 2 ? 0x7fff7fffu : 0x7fffffffu);
        },
        [&](float f) {
            more = __fmaf_rn(f, f, more);
            any |= __float_as_uint(f) & 0x7fffffffu;
        });
    unpair(add2(pairs[0], pairs[1]), lo, hi);
    const float sum = __fadd_rn(__fadd_rn(lo, hi), more);
    if ((sum >= 0x1p-90f && sum < INFINITY) || any == 0) return sum;
    double wide = 0.0;
    const auto square = [&](float f) { wide = __fma_rn((double)f, (double)f, wide); };
    vectors_of_piece<T, 1>(
        p,
        [&](const uint4 &v) {
            float f[E];
            Vec<T>::unpack(v, f);
#pragma unroll
            for (int e = 0; e < E; ++e) square(f[e]);
        },
        square);
    return wide;
}

// the threads' numbers added up in a fixed order, on every thread
__device__ __forceinline__ double block_sum(double x, double *part)
{
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) x = __dadd_rn(x, __shfl_xor_sync(FULL, x, off));
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
    __syncthreads();
    x = part[0];
#pragma unroll
    for (int w = 1; w < CLIP_THREADS / 32; ++w) x = __dadd_rn(x, part[w]);
    return x;
}

__global__ __launch_bounds__(CLIP_THREADS) void k_clip_norm(const ClipPiece *pieces, int64_t n, double *__restrict__ partial)
{
    after_previous();
    __shared__ double part[CLIP_THREADS / 32];
    double sum = 0.0;
    ClipPiece next;
    if (blockIdx.x < n) next = pieces[blockIdx.x];
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const ClipPiece p = next;
        if (i + gridDim.x < n) next = pieces[i + gridDim.x];
        const double x = p.g_type == PDB_TYPE_FLOAT    ? piece_squares<float>(p)
                         : p.g_type == PDB_TYPE_BFLOAT ? piece_squares<__nv_bfloat16>(p)
                                                       : piece_squares<__half>(p);
        sum = __dadd_rn(sum, x);
    }
    sum = block_sum(sum, part);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

template <typename T, typename O, bool ACC>
__device__ __forceinline__ void piece_step(const ClipPiece &p, float factor)
{
    const T *g = (const T *)p.g;
    O *out = (O *)p.out;
    const auto step = [&](float x, float old) {
        const float v = __fmul_rn(factor, x);
        return ACC ? __fadd_rn(old, v) : v;
    };
    each_of_piece(
        p,
        [&](int r, int c) {
            O *at = out + r * p.out_stride + c;
            const Pack<T, WIDE> v = load_pack<T, WIDE>(g + r * p.g_stride + c);
            float f[WIDE], old[WIDE];
            if (ACC) to_floats(load_pack<O, WIDE>(at), old);
            to_floats(v, f);
#pragma unroll
            for (int e = 0; e < WIDE; ++e) f[e] = step(f[e], ACC ? old[e] : 0.0f);
            store_pack<O, WIDE>(at, of_floats<O>(f));
        },
        [&](int r, int c) {
            O *at = out + r * p.out_stride + c;
            *at = from_float<O>(step(to_float(g[r * p.g_stride + c]), ACC ? to_float(*at) : 0.0f));
        });
}

template <typename T, bool ACC>
__device__ __forceinline__ void piece_step_to(const ClipPiece &p, float factor)
{
    if (p.out_type == PDB_TYPE_FLOAT) piece_step<T, float, ACC>(p, factor);
    else if (p.out_type == PDB_TYPE_BFLOAT) piece_step<T, __nv_bfloat16, ACC>(p, factor);
    else piece_step<T, __half, ACC>(p, factor);
}

// Every block forms the norm from the blocks' sums, in one order, and then steps its pieces.
template <bool ACC>
__global__ __launch_bounds__(CLIP_THREADS) void k_clip_step(const ClipPiece *pieces, int64_t n, const double *partial, int blocks,
                                                            float max_norm, float scale, float *__restrict__ norm)
{
    after_previous();
    __shared__ double part[CLIP_THREADS / 32];
    double sum = 0.0;
    for (int b = threadIdx.x; b < blocks; b += CLIP_THREADS) sum = __dadd_rn(sum, partial[b]);
    const double all = __dsqrt_rn(block_sum(sum, part));
    if (blockIdx.x == 0 && threadIdx.x == 0 && norm) *norm = (float)all;
    if (!(all < INFINITY)) return;                        // a gradient that is not finite: no step
    const bool clips = all > (double)max_norm;
    const float factor = clips ? (float)((double)scale * ((double)max_norm / all)) : scale;
    // the last pieces first: L2 still holds what the norm's launch read last
    int64_t i = (n - 1 - blockIdx.x) / gridDim.x * gridDim.x + blockIdx.x;
    ClipPiece next;
    if (i >= 0 && i < n) next = pieces[i];
    for (; i >= 0 && i < n; i -= gridDim.x) {
        const ClipPiece p = next;
        if (i >= gridDim.x) next = pieces[i - gridDim.x];
        if (!ACC && factor == 1.0f && p.out == p.g) continue;
        if (p.g_type == PDB_TYPE_FLOAT) piece_step_to<float, ACC>(p, factor);
        else if (p.g_type == PDB_TYPE_BFLOAT) piece_step_to<__nv_bfloat16, ACC>(p, factor);
        else piece_step_to<__half, ACC>(p, factor);
    }
}

// PDB_OK where the results are apart from one another and from the gradients, but for a gradient's own result
int check_apart(const pdb_mat *grads, const pdb_mat *outs, int64_t n)
{
    struct Range {
        const char *from, *to;
        int64_t i;
        bool out;
    };
    std::vector<Range> at;
    at.reserve(2 * n);
    for (int64_t i = 0; i < n; ++i)
        for (const pdb_mat *m : {grads + i, outs + i}) {
            if (m->rows == 0 || m->cols == 0) continue;
            const char *from = (const char *)m->data;
            at.push_back({from, from + ((m->rows - 1) * stride_of(m) + m->cols) * type_bytes(m->type), i, m == outs + i});
        }
    std::sort(at.begin(), at.end(), [](const Range &a, const Range &b) { return a.from < b.from; });
    for (size_t a = 0; a < at.size(); ++a)
        for (size_t b = a + 1; b < at.size() && at[b].from < at[a].to; ++b) {
            if (!at[a].out && !at[b].out) continue;
            const pdb_mat *x = (at[a].out ? outs : grads) + at[a].i, *y = (at[b].out ? outs : grads) + at[b].i;
            const bool own = at[a].i == at[b].i && at[a].out != at[b].out;
            if (own ? !same_or_apart(x, y) : overlap(x, y)) return PDB_EINVAL;
        }
    return PDB_OK;
}

// the matrices' pieces of at most `most` elements
void cut(const pdb_mat *g, const pdb_mat *o, int64_t most, std::vector<ClipPiece> &pieces)
{
    if (g->rows == 0 || g->cols == 0) return;
    int64_t rows = g->rows, cols = g->cols;
    if (stride_of(g) == cols && stride_of(o) == cols) cols *= rows, rows = 1;           // one row
    const int gb = type_bytes(g->type), ob = type_bytes(o->type);
    const int64_t gs = rows > 1 ? g->stride : 0, os = rows > 1 ? o->stride : 0;
    // elements before the first pack, the same in both matrices and in every row, or packs cannot be moved
    const auto before = [](const void *p, int bytes) { return (int)((WIDE - (uintptr_t)p / bytes % WIDE) % WIDE); };
    const bool packs = before(g->data, gb) == before(o->data, ob) && gs % WIDE == 0 && os % WIDE == 0;
    const int64_t head = before(g->data, gb);
    // pieces but a row's first start at a pack (`most` is a multiple of WIDE)
    for (int64_t c = 0; c < cols;) {
        const int64_t to = std::min(cols, c + most + (c == 0 && packs ? head : 0));
        const int64_t high = std::max<int64_t>(1, most / (to - c));
        for (int64_t r = 0; r < rows; r += high) {
            ClipPiece p = {};
            p.g = (const char *)g->data + (r * gs + c) * gb;
            p.out = (char *)o->data + (r * os + c) * ob;
            p.g_stride = gs, p.out_stride = os;
            p.rows = (int32_t)std::min(high, rows - r);
            p.cols = (int32_t)(to - c);
            p.head = packs ? (int32_t)std::min(c == 0 ? head : 0, to - c) : p.cols;
            p.g_type = (int16_t)g->type, p.out_type = (int16_t)o->type;
            pieces.push_back(p);
        }
        c = to;
    }
}

}  // namespace

extern "C" {

void pdb_clip_plan_free(pdb_clip_plan *p)
{
    if (!p) return;
    if (p->ev_use) cudaEventSynchronize(p->ev_use);
    release(p->arrays, own_stream());
    if (p->ev_use) cudaEventDestroy(p->ev_use);
    delete p;
}

int pdb_clip_plan_build(const pdb_mat *grads, const pdb_mat *outs, int64_t n, pdb_clip_plan **out, void *stream)
{
    ApiScope scope("pdb_clip_plan_build", nullptr, nullptr, nullptr, nullptr, false);
    if (!out) return PDB_EINVAL;
    *out = nullptr;
    if (n < 0 || (n > 0 && (!grads || !outs))) return PDB_EINVAL;
    int64_t total = 0;
    for (int64_t i = 0; i < n; ++i) {
        int rc = check_mat(grads + i, MOST_ELEMENTS, MOST_ELEMENTS);
        rc = rc ? rc : check_mat(outs + i, MOST_ELEMENTS, MOST_ELEMENTS);
        if (rc != PDB_OK) return rc;
        if (grads[i].rows != outs[i].rows || grads[i].cols != outs[i].cols) return PDB_EINVAL;
        if (grads[i].rows > MOST_ELEMENTS / std::max<int64_t>(1, grads[i].cols)) return PDB_ETOOBIG;
        if ((total += grads[i].rows * grads[i].cols) > MOST_ELEMENTS) return PDB_ETOOBIG;
    }
    pdb_clip_plan *p = nullptr;
    std::vector<ClipPiece> pieces;
    const Launch l = launch_info();
    try {
        if (const int rc = check_apart(grads, outs, n)) return rc;
        const int64_t shares = (int64_t)l.sms * NORM_BLOCKS_PER_SM * 2;
        const int64_t most = std::min<int64_t>(16384, std::max<int64_t>(2048, (total / shares + WIDE - 1) / WIDE * WIDE));
        for (int64_t i = 0; i < n; ++i) cut(grads + i, outs + i, most, pieces);
        p = new pdb_clip_plan();
    } catch (const std::bad_alloc &) {
        return PDB_ENOMEM;
    }
    cudaStream_t s = (cudaStream_t)stream;
    p->device = l.device;
    p->n_pieces = (int64_t)pieces.size();
    p->blocks = (int)std::max<int64_t>(1, std::min<int64_t>(p->n_pieces, (int64_t)l.sms * NORM_BLOCKS_PER_SM));
    p->step_blocks = (int)std::max<int64_t>(1, std::min<int64_t>(p->n_pieces, (int64_t)l.sms * STEP_BLOCKS_PER_SM));
    int rc = cudaEventCreateWithFlags(&p->ev_use, cudaEventDisableTiming) == cudaSuccess ? PDB_OK : PDB_ECUDA;
    rc = rc ? rc : alloc_block(p->arrays, {{(void **)&p->partial, sizeof(double) * p->blocks},
                                           {(void **)&p->pieces, sizeof(ClipPiece) * p->n_pieces}}, s);
    if (rc == PDB_OK && p->n_pieces > 0 &&
        cudaMemcpyAsync(p->pieces, pieces.data(), sizeof(ClipPiece) * p->n_pieces, cudaMemcpyHostToDevice, s) != cudaSuccess)
        rc = PDB_ECUDA;
    if (rc == PDB_OK && cudaStreamSynchronize(s) != cudaSuccess) rc = PDB_ECUDA;
    if (rc != PDB_OK) {
        cudaGetLastError();
        cudaStreamSynchronize(s);
        pdb_clip_plan_free(p);
        return rc;
    }
    cudaEventRecord(p->ev_use, s);
    *out = p;
    return PDB_OK;
}

int pdb_clip(const pdb_clip_plan *p, float max_norm, float scale, int accumulate, float *norm, void *stream)
{
    ApiScope scope("pdb_clip", nullptr, nullptr, nullptr, nullptr, false);
    if (!p || !(max_norm >= 0.0f) || !std::isfinite(scale) || (uintptr_t)norm % 4 != 0) return PDB_EINVAL;
    int device = -1;
    if (cudaGetDevice(&device) != cudaSuccess) return PDB_ECUDA;
    if (device != p->device) return PDB_EINVAL;
    cudaStream_t s = (cudaStream_t)stream;
    HandleUse use{p->ev_use, s};
    int rc = launch(k_clip_norm, p->blocks, CLIP_THREADS, 0, 1, s, p->pieces, p->n_pieces, p->partial);
    if (rc == PDB_OK)
        rc = launch(accumulate ? k_clip_step<true> : k_clip_step<false>, p->step_blocks, CLIP_THREADS, 0, 1, s, p->pieces,
                    p->n_pieces, p->partial, p->blocks, max_norm, scale, norm);
    return rc;
}

}  // extern "C"
