// Distillation from a teacher's top logits: loss and gradient (pdb_distill).
#include <algorithm>
#include <cmath>

#include "tokens.cuh"

using namespace pdb;

namespace {

constexpr int MAX_SLOTS = 1024;
constexpr float LEAST_REST = 1e-6f;   // a teacher's rest below this is the rounding of its lse

__device__ __forceinline__ float load_float(const void *p, int type, int64_t i)
{
    return type == PDB_TYPE_FLOAT    ? ((const float *)p)[i]
           : type == PDB_TYPE_BFLOAT ? __bfloat162float(((const __nv_bfloat16 *)p)[i])
                                     : __half2float(((const __half *)p)[i]);
}

template <typename T>
__global__ __launch_bounds__(ROW_THREADS) void k_distill(const T *logits, int64_t rows, int cols, int64_t stride,
                                                         Ids top_ids,
                                                         const void *__restrict__ top, int top_type, int64_t top_stride,
                                                         int K, const float *__restrict__ teacher_lse, float temperature,
                                                         float *loss, const float *__restrict__ weight, T *dlogits,
                                                         int64_t out_stride, int *status)
{
    __shared__ float s_red[32];
    __shared__ int s_id[MAX_SLOTS];
    __shared__ float s_q[MAX_SLOTS], s_lq[MAX_SLOTS];
    const float inv = 1.0f / temperature;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *z = logits + r * stride;
        __syncthreads();
        float peak = -INFINITY;
        for (int k = threadIdx.x; k < K; k += blockDim.x) {
            int64_t v = load_id(top_ids, r, k);
            if (v >= cols) set_status(status, PDB_ERANGE), v = -1;
            s_id[k] = v < 0 ? -1 : (int)v;
            const float t = v < 0 ? -INFINITY : __fmul_rn(load_float(top, top_type, r * top_stride + k), inv);
            s_lq[k] = t;
            peak = t != t ? NAN : peak != peak ? peak : fmaxf(peak, t);
        }
        const bool bad = __syncthreads_or(peak != peak);
        peak = block_max(peak, s_red);
        const bool live = bad || peak != -INFINITY;
        float total = 0.0f;
        const float base = teacher_lse ? teacher_lse[r] : peak;
        for (int k = threadIdx.x; k < K; k += blockDim.x) {
            s_lq[k] = __fsub_rn(s_lq[k], base);
            s_q[k] = s_id[k] < 0 || s_lq[k] == -INFINITY ? 0.0f : expf(s_lq[k]);
            total = __fadd_rn(total, s_q[k]);
        }
        total = block_sum(total, s_red);
        float rest = 0.0f;
        if (!teacher_lse) {
            const float logt = logf(total);
            for (int k = threadIdx.x; k < K; k += blockDim.x) {
                s_lq[k] = __fsub_rn(s_lq[k], logt);
                s_q[k] = __fdiv_rn(s_q[k], total);
            }
        } else {
            rest = __fsub_rn(1.0f, total);
            if (rest <= LEAST_REST) rest = 0.0f;
        }
        __syncthreads();
        // the student's statistics: over the tokens in no slot, and over all
        float m = -INFINITY, mo = -INFINITY;
        for (int j = threadIdx.x; j < cols; j += blockDim.x) {
            const float x = to_float(z[j]);
            m = fmaxf(m, x);
            bool in = false;
            if (teacher_lse)
                for (int k = 0; k < K; ++k) in |= s_id[k] == j;
            if (!in) mo = fmaxf(mo, x);
        }
        m = block_max(m, s_red);
        mo = block_max(mo, s_red);
        const float ref = m == -INFINITY ? 0.0f : m, refo = mo == -INFINITY ? 0.0f : mo;
        float out = 0.0f, all = 0.0f;
        for (int j = threadIdx.x; j < cols; j += blockDim.x) {
            const float e = expf(__fmul_rn(__fsub_rn(to_float(z[j]), ref), inv));
            all = __fadd_rn(all, e);
            bool in = false;
            if (teacher_lse)
                for (int k = 0; k < K; ++k) in |= s_id[k] == j;
            if (!in) out = __fadd_rn(out, expf(__fmul_rn(__fsub_rn(to_float(z[j]), refo), inv)));
        }
        all = block_sum(all, s_red);
        out = block_sum(out, s_red);
        const float logs = logf(all);
        float sum = 0.0f;
        for (int k = threadIdx.x; k < K; k += blockDim.x)
            if (s_q[k] != 0.0f) {
                const float x = __fsub_rn(__fmul_rn(__fsub_rn(to_float(z[s_id[k]]), ref), inv), logs);
                sum = __fadd_rn(sum, __fmul_rn(s_q[k], __fsub_rn(s_lq[k], x)));
            }
        sum = block_sum(sum, s_red);
        const float logout = __fadd_rn(__fsub_rn(logf(out), logs), __fmul_rn(__fsub_rn(refo, ref), inv));
        if (rest > 0.0f) sum = __fadd_rn(sum, __fmul_rn(rest, __fsub_rn(logf(rest), logout)));
        if (threadIdx.x == 0 && loss)
            loss[r] = !live ? 0.0f : all == 0.0f ? INFINITY : __fmul_rn(__fmul_rn(temperature, temperature), sum);
        if (!dlogits) continue;
        const float w = weight ? weight[r] : 1.0f;
        const bool zero = w == 0.0f || !live || all == 0.0f;
        const float wt = __fmul_rn(w, temperature);
        // outside of the slots p_j - q_t p_j / p_t = e_j * part with e_j relative to the outside's own maximum, so that
        // neither p_t nor p_j need be representable
        const float refd = teacher_lse ? refo : ref;
        const float part = !teacher_lse ? __fdiv_rn(1.0f, all)
                           : out == 0.0f ? 0.0f
                                         : __fsub_rn(__fdiv_rn(expf(__fmul_rn(__fsub_rn(refo, ref), inv)), all),
                                                     __fdiv_rn(rest, out));
        T *d = dlogits + r * out_stride;
        for (int j = threadIdx.x; j < cols; j += blockDim.x) {
            float v = 0.0f;
            if (!zero) {
                const float x = to_float(z[j]);
                float q = 0.0f;
                bool in = false;
                for (int k = 0; k < K; ++k)
                    if (s_id[k] == j) in = true, q = __fadd_rn(q, s_q[k]);
                v = in ? __fsub_rn(__fdiv_rn(expf(__fmul_rn(__fsub_rn(x, ref), inv)), all), q)
                       : __fmul_rn(expf(__fmul_rn(__fsub_rn(x, refd), inv)), part);
                v = __fmul_rn(wt, v);
            }
            d[j] = from_float<T>(v);
        }
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
    with_type(logits->type, [&](auto *a) {
        using T = std::remove_pointer_t<decltype(a)>;
        k_distill<T><<<(unsigned)std::min<int64_t>(logits->rows, 1 << 20), ROW_THREADS, 0, s>>>(
            (const T *)logits->data, logits->rows, (int)logits->cols, stride_of(logits), ids_of(top_ids),
            top_logits->data, top_logits->type, stride_of(top_logits), (int)top_logits->cols, teacher_lse, temperature,
            loss, weight, dlogits ? (T *)dlogits->data : nullptr, dlogits ? stride_of(dlogits) : 0, t->status);
        note_launch();
    });
    return cudaPeekAtLastError() == cudaSuccess ? PDB_OK : PDB_ECUDA;
}
