// C entries between token ids and rows: lapsum_sample, lapsum_embed_*.  Argument checks, buffer layout and launches; nothing is allocated
// and the host never waits.
#include <cmath>
#include <cstring>

#include "../../include/lapsum.h"
#include "api.h"
#include "embed.cuh"
#include "host.h"
#include "sample.cuh"

using namespace lapsum;

namespace {

// ------------------------------------------------------------------ sample ----
// Every weight is off by half a unit of 2^-S at most, the sums by vocab times that, and a long tail of small weights all to one side: 2^-28 of the largest weight at 2^18 tokens,
// where S is 45, four times more for each doubling.  Up to here, 2^-22, that is of the size of what u and logprob resolve.
constexpr int64_t SAMPLE_VOCAB = (int64_t)1 << 21;
constexpr int SAMPLE_BLOCK_BYTES = 64 << 10, SMEM_MOST = 226 << 10;

template <typename T, int THREADS, bool RESIDENT, bool TOP_P>
int sample_launch(const SampleArgs &A, int64_t rows, cudaStream_t st)
{
    const auto kernel = sample_kernel<T, THREADS, RESIDENT, TOP_P>;
    const size_t smem = sizeof(SampleShared<THREADS, TOP_P>) + (RESIDENT ? (size_t)A.chunk * sizeof(T) : 0);
    static thread_local int dev_ready = -1;  // the attribute belongs to the device's context
    int dev = 0;
    CU_OK(cudaGetDevice(&dev));
    if (dev != dev_ready) {
        CU_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_MOST));
        dev_ready = dev;
    }
    return launch_clusters((unsigned)A.cluster, kernel, (unsigned)(rows * A.cluster), THREADS, smem, st, A);
}
// Few rows, or a top-p that may have to look far: blocks as many as keep a block's run at 64 KB (two blocks per SM), and more, down to runs of 4096 tokens,
// while all of them find a place at once.  Rows for two thirds of the SMs, long and without top-p: a block of 1024 threads each.  Measured, a block each / clusters, us, no
// filter and top-k 40:
//   fp32   74 x 128000 40 / 41, 26 / 34     99 x 32768 17 / 17, 15 / 16     148 x 50257 27 / 36, 24 / 36    256 x 128000 90 / 121, 63 / 111   600 x 128000 226 / 268, 139 / 235
//          48 x 128000 39 / 29, 25 / 25     99 x 16384 13 / 13, 14 / 15     296 x 16384 25 / 16, 25 / 17    600 x 24000 70 / 59, 69 / 67
//   bf16   99 x 128000 36 / 37, 25 / 32     148 x 65536 23 / 25, 19 / 20    296 x 128000 72 / 98, 45 / 78   but 600 x 32768 73 / 53, 67 / 49
// With top-p clusters win: 0.9 over some 3000 tokens 366 / 424 of 256 x 128000, but rows of all kinds 324 / 193 (a single row of the last kind takes 200 on one SM).  The
// host sees no values of settings per row, so a given top-p counts as one.
template <typename T>
int sample_t(SampleArgs A, int64_t rows, cudaStream_t st)
{
    int sms = 0;
    RUN(sm_count(&sms));
    const bool many = 3 * rows >= 2 * sms && A.vocab >= 32768 && !A.top_p_row && A.top_p >= 1;
    int cluster = 1;
    while (!many && cluster < 8 && ((int64_t)A.vocab * (int)sizeof(T) > (int64_t)cluster * SAMPLE_BLOCK_BYTES ||
                           (rows * cluster * 2 <= 2 * sms && A.vocab >= 2 * 4096 * cluster)))
        cluster *= 2;
    A.cluster = cluster;
    A.chunk = (int)(ceil_div(ceil_div(A.vocab, cluster), 128) * 128);
    if (many) return sample_launch<T, 1024, false, false>(A, rows, st);
    if ((size_t)A.chunk * sizeof(T) + sizeof(SampleShared<512, true>) <= SMEM_MOST) return sample_launch<T, 512, true, true>(A, rows, st);
    return sample_launch<T, 512, false, true>(A, rows, st);
}

// ------------------------------------------------------------------- embed ----
int embed_check(const void *ids, int32_t id_bytes, int64_t tokens, int64_t vocab, int64_t d, double scale, int32_t io_dtype)
{
    if (tokens < 0 || tokens > (int64_t)1 << 30 || vocab < 1 || vocab > (int64_t)1 << 30 || d < 1 || d > (int64_t)1 << 20) return LAPSUM_ERR_SHAPE;
    if ((id_bytes != 4 && id_bytes != 8) || !std::isfinite(scale) || !std::isfinite((float)scale)) return LAPSUM_ERR_PARAM;
    if (io_dtype < LAPSUM_IO_F32 || io_dtype > LAPSUM_IO_BF16) return LAPSUM_ERR_UNSUPPORTED;
    if (tokens > 0 && !ids) return LAPSUM_ERR_NULL;
    return LAPSUM_OK;
}
struct EmbedLayout {
    size_t off_start, off_order, off_long, off_partial, bytes;
};
// Every block of the sort reads all ids, once per range of the table: 1.2e12 products of ids and ranges a second (2^20 ids into 2^20 rows 2.1 ms, 2^22 into 2^24 117).  Sizes
// whose sort would hold the GPU for more than a quarter of a second are refused.
constexpr int64_t EMBED_PRODUCTS = (int64_t)1 << 38;
bool embed_sorts(int64_t tokens, int64_t vocab) { return tokens == 0 || ceil_div(vocab, EMBED_RANGE) <= EMBED_PRODUCTS / tokens; }
EmbedLayout embed_layout(int64_t tokens, int64_t vocab, int64_t d)
{
    EmbedLayout X;
    size_t at = 256;  // the long rows' counter
    X.off_start = at, at += align_up((size_t)(vocab + 1) * 4);
    X.off_order = at, at += align_up((size_t)tokens * 4);
    X.off_long = at, at += align_up((size_t)(tokens / EMBED_LONG + 1) * 4);
    X.off_partial = at, at += align_up((size_t)ceil_div(tokens, EMBED_LONG) * 2 * (size_t)(ceil_div(d, 4) * 4) * 4);
    X.bytes = at;
    return X;
}
template <typename T, bool VEC>
int64_t embed_parts(int64_t d) { return ceil_div(d, EmbedShape<T, VEC>::SPAN); }

template <typename T>
int embed_forward_t(const EmbedArgs &A, cudaStream_t st)
{
    constexpr int V = Io<T>::V;
    const bool vec = A.d % V == 0 && A.table_stride % V == 0 && A.out_stride % V == 0 && aligned(A.table, 16) && aligned(A.out, 16);
    const int64_t units = A.tokens * (vec ? embed_parts<T, true>(A.d) : embed_parts<T, false>(A.d));
    if (ceil_div(units, 8) >= (int64_t)1 << 31) return LAPSUM_ERR_SHAPE;  // a grid ends at 2^31 - 1 blocks
    return launch_pdl(vec ? embed_forward_kernel<T, true> : embed_forward_kernel<T, false>, (unsigned)ceil_div(units, 8), 256, 0, st, A);
}

template <typename T>
int embed_backward_t(EmbedArgs A, cudaStream_t st)
{
    constexpr int V = Io<T>::V, smem = EMBED_WARPS * EMBED_RANGE * 4;
    const bool vec = A.d % V == 0 && A.grad_stride % V == 0 && aligned(A.grad_out, 16) && aligned(A.grad, 16);
    const int64_t parts = vec ? embed_parts<T, true>(A.d) : embed_parts<T, false>(A.d);
    A.chunk_blocks = ceil_div(ceil_div(A.tokens, EMBED_LONG) * parts, 8);
    const int64_t blocks = A.chunk_blocks + ceil_div(ceil_div(A.vocab, EMBED_ROWS) * parts, 8);
    if (blocks >= (int64_t)1 << 31) return LAPSUM_ERR_SHAPE;
    int sms = 0, dev = 0;
    RUN(sm_count(&sms));
    static thread_local int dev_ready = -1;  // the attribute belongs to the device's context
    CU_OK(cudaGetDevice(&dev));
    if (dev != dev_ready) {
        CU_OK(cudaFuncSetAttribute(embed_sort_kernel<int32_t>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        CU_OK(cudaFuncSetAttribute(embed_sort_kernel<int64_t>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        dev_ready = dev;
    }
    RUN(launch_pdl(A.wide_ids ? embed_sort_kernel<int64_t> : embed_sort_kernel<int32_t>, (unsigned)ceil_div(A.vocab, EMBED_RANGE), 32 * EMBED_WARPS,
                   smem, st, A));
    RUN(launch_pdl(vec ? embed_grad_kernel<T, true> : embed_grad_kernel<T, false>, (unsigned)blocks, 256, 0, st, A));
    if (A.tokens <= EMBED_LONG) return LAPSUM_OK;  // no row can be long
    return launch_pdl(embed_join_kernel<T>, (unsigned)(4 * sms), 256, 0, st, A);
}


}  // namespace

extern "C" {

void lapsum_sample_default_params(lapsum_sample_params *p)
{
    if (!p) return;
    std::memset(p, 0, sizeof(*p));
    p->temperature = p->top_p = 1.0;
    p->io_dtype = LAPSUM_IO_F32;
}

int lapsum_sample(const void *logits, int64_t rows, int64_t vocab, int64_t stride, const float *u, const lapsum_sample_params *prm,
                  const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p, int32_t *token, float *logprob,
                  int32_t *kept, void *stream)
{
    if (!prm) return LAPSUM_ERR_NULL;
    if (rows < 0 || rows > (int64_t)1 << 27 || vocab < 1 || vocab > SAMPLE_VOCAB || stride < vocab) return LAPSUM_ERR_SHAPE;
    // a setting for all rows has to be in range (one per row voids its row instead)
    if (prm->io_dtype < LAPSUM_IO_F32 || prm->io_dtype > LAPSUM_IO_BF16 || (!temperature && !(prm->temperature >= 0 && std::isfinite(prm->temperature))) ||
        (!top_p && !(prm->top_p > 0)) || (!min_p && !(prm->min_p >= 0 && prm->min_p <= 1)))
        return LAPSUM_ERR_PARAM;
    if (rows == 0) return LAPSUM_OK;
    if (!logits || !u || !token) return LAPSUM_ERR_NULL;
    SampleArgs A;
    std::memset(&A, 0, sizeof(A));
    A.logits = logits, A.stride = stride, A.u = u;
    A.temperature_row = temperature, A.top_k_row = top_k, A.top_p_row = top_p, A.min_p_row = min_p;
    A.temperature = prm->temperature, A.top_p = prm->top_p, A.min_p = prm->min_p, A.top_k = prm->top_k;
    A.token = token, A.logprob = logprob, A.kept = kept;
    A.vocab = (int)vocab;
    A.bits = 45;
    while (vocab > (int64_t)1 << (63 - A.bits)) --A.bits;  // sums of up to vocab 2^S fit 64 bits
    return BY_TYPE(sample_t, prm->io_dtype, A, rows, static_cast<cudaStream_t>(stream));
}

int lapsum_embed_forward(const void *ids, int32_t id_bytes, int64_t tokens, const void *table, int64_t table_stride, int64_t vocab, int64_t d,
                         double scale, int32_t io_dtype, void *out, int64_t out_stride, void *stream)
{
    RUN(embed_check(ids, id_bytes, tokens, vocab, d, scale, io_dtype));
    if (table_stride < d || out_stride < d) return LAPSUM_ERR_SHAPE;
    if (tokens == 0) return LAPSUM_OK;
    if (!table || !out) return LAPSUM_ERR_NULL;
    EmbedArgs A;
    std::memset(&A, 0, sizeof(A));
    A.ids = ids, A.wide_ids = id_bytes == 8, A.tokens = tokens, A.vocab = vocab, A.d = d, A.skip = -1, A.scale = (float)scale;
    A.table = table, A.table_stride = table_stride, A.out = out, A.out_stride = out_stride;
    return BY_TYPE(embed_forward_t, io_dtype, A, static_cast<cudaStream_t>(stream));
}

int lapsum_embed_workspace_bytes(int64_t tokens, int64_t vocab, int64_t d, size_t *bytes)
{
    if (!bytes) return LAPSUM_ERR_NULL;
    if (tokens < 0 || tokens > (int64_t)1 << 30 || vocab < 1 || vocab > (int64_t)1 << 30 || d < 1 || d > (int64_t)1 << 20 || !embed_sorts(tokens, vocab))
        return LAPSUM_ERR_SHAPE;
    *bytes = embed_layout(tokens, vocab, d).bytes;
    return LAPSUM_OK;
}

int lapsum_embed_backward(const void *grad_out, int64_t grad_stride, const void *ids, int32_t id_bytes, int64_t tokens, int64_t vocab, int64_t d,
                          double scale, int64_t skip, int32_t io_dtype, int32_t grad_dtype, void *grad_table, void *ws, size_t ws_bytes, void *stream)
{
    RUN(embed_check(ids, id_bytes, tokens, vocab, d, scale, io_dtype));
    if (grad_stride < d || !embed_sorts(tokens, vocab)) return LAPSUM_ERR_SHAPE;
    if (grad_dtype != io_dtype && grad_dtype != LAPSUM_IO_F32) return LAPSUM_ERR_UNSUPPORTED;
    if (!grad_table || !ws || (tokens > 0 && !grad_out)) return LAPSUM_ERR_NULL;
    const EmbedLayout X = embed_layout(tokens, vocab, d);
    if (!aligned(ws, 256) || ws_bytes < X.bytes) return LAPSUM_ERR_WORKSPACE;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (tokens == 0) {
        CU_OK(cudaMemsetAsync(grad_table, 0, (size_t)vocab * (size_t)d * (grad_dtype == LAPSUM_IO_F32 ? 4 : 2), st));
        return LAPSUM_OK;
    }
    uint8_t *const at = static_cast<uint8_t *>(ws);
    EmbedArgs A;
    std::memset(&A, 0, sizeof(A));
    A.ids = ids, A.wide_ids = id_bytes == 8, A.tokens = tokens, A.vocab = vocab, A.d = d, A.skip = skip, A.scale = (float)scale;
    A.grad_out = grad_out, A.grad_stride = grad_stride, A.grad = grad_table, A.grad_f32 = grad_dtype == LAPSUM_IO_F32;
    A.long_count = reinterpret_cast<uint32_t *>(at);
    A.row_start = reinterpret_cast<int32_t *>(at + X.off_start), A.order = reinterpret_cast<int32_t *>(at + X.off_order);
    A.long_rows = reinterpret_cast<int32_t *>(at + X.off_long), A.partial = reinterpret_cast<float *>(at + X.off_partial);
    A.partial_stride = ceil_div(d, 4) * 4;
    return BY_TYPE(embed_backward_t, io_dtype, A, st);
}

}  // extern "C"
