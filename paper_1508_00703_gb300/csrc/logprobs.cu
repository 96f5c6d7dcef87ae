// Log probabilities of given tokens with entropy and the most probable
// alternatives, and their gradient (pdb_logprobs, pdb_logprobs_grad).
#include <algorithm>
#include <cmath>

#include "tokens.cuh"

using namespace pdb;

namespace {

constexpr int MAX_TOP = 64;

// a logit and its token as one word that orders like (logit descending, token ascending): NaN above all, -0 = +0
__device__ __forceinline__ uint64_t top_key(float z, int j)
{
    uint32_t b = __float_as_uint(z);
    b = z != z ? 0xfffffffeu : z == 0.0f ? 0x80000000u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
    return (uint64_t)b << 32 | (uint32_t)~j;
}

template <typename T>
__global__ __launch_bounds__(ROW_THREADS) void k_logprobs(const T *__restrict__ logits, int64_t rows, int cols,
                                                          int64_t stride, Ids ids,
                                                          float scale, int64_t ignore, float *logp, float *lse,
                                                          float *entropy, int k, float *top_logp, int32_t *top_ids,
                                                          int *status)
{
    __shared__ float s_red[32];
    __shared__ uint64_t s_key[32];
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *z = logits + r * stride;
        float m = -INFINITY;
        for (int j = threadIdx.x; j < cols; j += blockDim.x) m = fmaxf(m, to_float(z[j]));
        m = block_max(m, s_red);
        const float ref = m == -INFINITY ? 0.0f : m;
        float s = 0.0f, w = 0.0f;
        for (int j = threadIdx.x; j < cols; j += blockDim.x) {
            const float d = __fmul_rn(__fsub_rn(to_float(z[j]), ref), scale);
            const float e = expf(d);
            s = __fadd_rn(s, e);
            w = __fadd_rn(w, e == 0.0f ? 0.0f : __fmul_rn(e, d));
        }
        s = block_sum(s, s_red);
        w = block_sum(w, s_red);
        const float logs = logf(s);
        const bool none = s == 0.0f;
        if (threadIdx.x == 0) {
            if (lse) lse[r] = __fmaf_rn(ref, scale, logs);
            if (entropy) entropy[r] = none ? 0.0f : __fsub_rn(logs, __fdiv_rn(w, s));
            if (logp) {
                const int64_t t = load_id(ids, r);
                const bool there = t != ignore && t >= 0 && t < cols;
                if (!there && t != ignore) set_status(status, PDB_ERANGE);
                logp[r] = !there ? 0.0f
                          : none ? -INFINITY
                                 : __fsub_rn(__fmul_rn(__fsub_rn(to_float(z[t]), ref), scale), logs);
            }
        }
        uint64_t below = ~(uint64_t)0;
        for (int i = 0; i < k; ++i) {
            uint64_t best = 0;
            for (int j = threadIdx.x; j < cols; j += blockDim.x) {
                const uint64_t key = top_key(to_float(z[j]), j);
                if (key < below && key > best) best = key;
            }
            for (int off = 16; off >= 1; off >>= 1) best = max(best, __shfl_xor_sync(FULL, best, off));
            __syncthreads();
            if ((threadIdx.x & 31) == 0) s_key[threadIdx.x >> 5] = best;
            __syncthreads();
            for (int q = 0; q < ROW_THREADS / 32; ++q) best = max(best, s_key[q]);
            below = best;
            if (threadIdx.x == 0) {
                const int j = (int)~(uint32_t)best;
                if (top_ids) top_ids[r * k + i] = j;
                if (top_logp)
                    top_logp[r * k + i] =
                        none ? -INFINITY : __fsub_rn(__fmul_rn(__fsub_rn(to_float(z[j]), ref), scale), logs);
            }
        }
        __syncthreads();
    }
}

template <typename T>
__global__ __launch_bounds__(ROW_THREADS) void k_logprobs_grad(const T *logits, int64_t rows, int cols, int64_t stride,
                                                               Ids ids, float scale,
                                                               int64_t ignore, const float *__restrict__ lse,
                                                               const float *__restrict__ entropy,
                                                               const float *__restrict__ dlogp,
                                                               const float *__restrict__ dentropy, T *dlogits,
                                                               int64_t out_stride, int *status)
{
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *z = logits + r * stride;
        T *d = dlogits + r * out_stride;
        float g = dlogp ? dlogp[r] : 0.0f;
        const float h = dentropy ? dentropy[r] : 0.0f;
        int64_t t = -1;
        if (dlogp) {
            t = load_id(ids, r);
            const bool there = t != ignore && t >= 0 && t < cols;
            if (!there && t != ignore && threadIdx.x == 0) set_status(status, PDB_ERANGE);
            if (!there) g = 0.0f, t = -1;
        }
        const float l = lse[r], H = h != 0.0f ? entropy[r] : 0.0f;
        const bool zero = (g == 0.0f && h == 0.0f) || l == -INFINITY;
        for (int j = threadIdx.x; j < cols; j += blockDim.x) {
            float v = 0.0f;
            if (!zero) {
                const float x = __fsub_rn(__fmul_rn(to_float(z[j]), scale), l);
                const float p = expf(x);
                v = __fsub_rn(j == t ? g : 0.0f, __fmul_rn(p, g));
                if (h != 0.0f && p != 0.0f) v = __fsub_rn(v, __fmul_rn(__fmul_rn(h, p), __fadd_rn(x, H)));
                v = __fmul_rn(v, scale);
            }
            d[j] = from_float<T>(v);
        }
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
    if (!(scale > 0.0f) || std::isinf(scale) || k < 0 || k > logits->cols) return PDB_EINVAL;
    if (k > MAX_TOP) return PDB_ETOOBIG;
    if (logits->rows == 0) return PDB_OK;
    cudaStream_t s = (cudaStream_t)stream;
    TokensUse use{t, s};
    with_type(logits->type, [&](auto *a) {
        using T = std::remove_pointer_t<decltype(a)>;
        k_logprobs<T><<<(unsigned)std::min<int64_t>(logits->rows, 1 << 20), ROW_THREADS, 0, s>>>(
            (const T *)logits->data, logits->rows, (int)logits->cols, stride_of(logits), ids_of(ids, logp),
             scale, ignore, logp, lse, entropy, (int)k, top_logp, top_ids, t->status);
        note_launch();
    });
    return cudaPeekAtLastError() == cudaSuccess ? PDB_OK : PDB_ECUDA;
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
    if (!(scale > 0.0f) || std::isinf(scale)) return PDB_EINVAL;
    if (dlogits->rows != logits->rows || dlogits->cols != logits->cols || dlogits->type != logits->type ||
        !same_or_apart(logits, dlogits))
        return PDB_EINVAL;
    if (logits->rows == 0 || logits->cols == 0) return PDB_OK;
    if (!lse || (dentropy && !entropy)) return PDB_EINVAL;
    cudaStream_t s = (cudaStream_t)stream;
    TokensUse use{t, s};
    with_type(logits->type, [&](auto *a) {
        using T = std::remove_pointer_t<decltype(a)>;
        k_logprobs_grad<T><<<(unsigned)std::min<int64_t>(logits->rows, 1 << 20), ROW_THREADS, 0, s>>>(
            (const T *)logits->data, logits->rows, (int)logits->cols, stride_of(logits), ids_of(ids, dlogp),
             scale, ignore, lse, entropy, dlogp, dentropy, (T *)dlogits->data,
            stride_of(dlogits), t->status);
        note_launch();
    });
    return cudaPeekAtLastError() == cudaSuccess ? PDB_OK : PDB_ECUDA;
}

}  // extern "C"
