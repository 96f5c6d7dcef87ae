// Rows of a table by token id, and the table's gradient by sorted ids
// (pdb_embed, pdb_embed_grad), and the handle of the token operators.
#include <algorithm>
#include <new>

#include "tokens.cuh"

using namespace pdb;

namespace {

// out[i, :] = scale * table[ids[i], :]
template <typename T, typename O>
__global__ void k_embed(const T *__restrict__ table, int64_t vocab, int64_t stride, Ids ids,
                        int64_t n, int dim, float scale, int64_t pad, O *__restrict__ out,
                        int64_t out_stride, int *status)
{
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const int64_t v = load_id(ids, i);
        const bool there = v != pad && v >= 0 && v < vocab;
        if (!there && v != pad && threadIdx.x == 0) set_status(status, PDB_ERANGE);
        for (int j = threadIdx.x; j < dim; j += blockDim.x)
            out[i * out_stride + j] = from_float<O>(there ? __fmul_rn(scale, to_float(table[v * stride + j])) : 0.0f);
    }
}

// ids as sort keys; those left out (pad, out of range) sort last
__global__ void k_embed_keys(Ids ids, int64_t n, int64_t vocab, int64_t pad,
                             uint32_t *__restrict__ key, int *status)
{
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= n) return;
    const int64_t v = load_id(ids, i);
    const bool there = v != pad && v >= 0 && v < vocab;
    if (!there && v != pad) set_status(status, PDB_ERANGE);
    key[i] = there ? (uint32_t)v : (uint32_t)vocab;
}

// one block per sorted position that starts a run: the run's sum
template <typename T, typename O>
__global__ void k_embed_runs(const uint32_t *__restrict__ key, const int32_t *__restrict__ pos, int64_t n,
                             int64_t vocab, const T *__restrict__ dout, int64_t stride, int dim, float scale,
                             int accumulate, O *__restrict__ dtable, int64_t out_stride)
{
    const int64_t i = blockIdx.x;
    const uint32_t v = key[i];
    if (v >= vocab || (i > 0 && key[i - 1] == v)) return;
    for (int j = threadIdx.x; j < dim; j += blockDim.x) {
        float total = 0.0f;
        for (int64_t a = i; a < n && key[a] == v; a += 32) {
            float piece = 0.0f;
            for (int64_t b = a; b < n && b < a + 32 && key[b] == v; ++b)
                piece = __fadd_rn(piece, to_float(dout[(int64_t)pos[b] * stride + j]));
            total = __fadd_rn(total, piece);
        }
        O *at = dtable + (int64_t)v * out_stride + j;
        const float sum = __fmul_rn(scale, total);
        *at = from_float<O>(accumulate ? __fadd_rn(to_float(*at), sum) : sum);
    }
}

template <typename O>
__global__ void k_embed_zero(O *__restrict__ dtable, int64_t vocab, int64_t stride, int dim)
{
    for (int64_t v = blockIdx.x; v < vocab; v += gridDim.x)
        for (int j = threadIdx.x; j < dim; j += blockDim.x) dtable[v * stride + j] = from_float<O>(0.0f);
}

}  // namespace

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
    with_type(table->type, [&](auto *a) {
        with_type(out->type, [&](auto *b) {
            using T = std::remove_pointer_t<decltype(a)>;
            using O = std::remove_pointer_t<decltype(b)>;
            k_embed<T, O><<<(unsigned)std::min<int64_t>(out->rows, 1 << 20), 256, 0, s>>>(
                (const T *)table->data, table->rows, stride_of(table), ids_of(ids), out->rows,
                (int)out->cols, scale, pad, (O *)out->data, stride_of(out), t->status);
            note_launch();
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
    if (n > 0) {
        k_embed_keys<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(ids_of(ids), n, vocab, pad, t->key, t->status);
        note_launch();
    }
    if (dim == 0 || vocab == 0) return cudaPeekAtLastError() == cudaSuccess ? PDB_OK : PDB_ECUDA;
    if (n > 0)
        rc = radix_sort(t->key, nullptr, t->skey, t->spos, t->tkey, t->tpos, n, bits_for(vocab), t->status + 1, s);
    if (rc != PDB_OK) return rc;
    with_type(dtable->type, [&](auto *b) {
        using O = std::remove_pointer_t<decltype(b)>;
        if (!accumulate) {
            k_embed_zero<O><<<(unsigned)std::min<int64_t>(vocab, 152 * 32), 256, 0, s>>>((O *)dtable->data, vocab,
                                                                                        stride_of(dtable), dim);
            note_launch();
        }
        if (n > 0)
            with_type(dout->type, [&](auto *a) {
                using T = std::remove_pointer_t<decltype(a)>;
                k_embed_runs<T, O><<<(unsigned)n, 256, 0, s>>>(t->skey, t->spos, n, vocab, (const T *)dout->data,
                                                               stride_of(dout), dim, scale, accumulate,
                                                               (O *)dtable->data, stride_of(dtable));
                note_launch();
            });
    });
    return cudaPeekAtLastError() == cudaSuccess ? PDB_OK : PDB_ECUDA;
}

}  // extern "C"
