// Attention over the 4-bit key/value cache: entry points, argument checks, choice of kernel.

#include <math.h>

#include <algorithm>

#include "kv_attention.h"

namespace qllm {
namespace {

using namespace kv;

int check_attention(const qllm_kv_cache_t* cache, int q_heads, int dtype, const qllm_kv_batch_t* batch) {
    if (!dtype_ok(dtype)) return QLLM_ERR_DTYPE;
    const int rc = check_cache_batch(cache, batch);
    if (rc != QLLM_OK) return rc;
    if (q_heads <= 0 || q_heads % cache->kv_heads) return QLLM_ERR_SHAPE;
    if (q_heads > 65535 || batch->rows * q_heads > 0x7fffffff) return QLLM_ERR_UNSUPPORTED;   // query rows are counted in 31 bits
    return QLLM_OK;
}

// Which kernels a call launches.  The streaming kernel reads a sequence's keys once per 8 or 16 query rows, the tensor-core kernel
// once per 256 and unpacks them for 256 whether there are that many or not: kPromptRows is where they meet (us, streaming against
// tensor-core kernel, heads of 128 in bf16, at 64 / 96 / 128 rows: 4 sequences of 4096 tokens on 8 heads 37 : 43, 49 : 45,
// 60 : 48; 1 of 32768 on 8 heads 53 : 88, 73 : 89, 92 : 90; 4 of 2048 on 32 heads 64 : 76, 88 : 65, 111 : 68; with a flushed L2 50 : 38,
// 63 : 40, 77 : 42; 69 : 93, 93 : 93, 116 : 93; 83 : 52, 112 : 52, 138 : 54, and heads of 64 then 36 : 34, 44 : 34, 52 : 34; 48 : 77,
// 63 : 77, 77 : 77; 56 : 44, 73 : 44, 87 : 44: the border could lie lower for batches, and would have to lie higher for one long
// context).  Either serves any count, so what the batch's hint says wrongly costs time only.  A batch with the same number of new tokens in every
// sequence, as far as the hint goes, needs one of them; others get both, each taking its sequences.
constexpr int kPromptRows = 96;
struct Choice {
    bool split, prompt;
    int hint, most_rows;                                   // query rows per key head of the largest sequence; the border
};
Choice choose(const qllm_kv_cache_t* cache, int q_heads, int dtype, const qllm_kv_batch_t* batch) {
    Choice c;
    c.hint = int(std::min<int64_t>(int64_t(batch->max_new) * (q_heads / cache->kv_heads), 0x7fffffff));
    c.prompt = kv::prompt_serves(cache->head_dim, dtype) && c.hint > kPromptRows;
    c.split = !c.prompt || (batch->seqs > 1 && batch->rows != int64_t(batch->seqs) * batch->max_new);
    c.most_rows = !c.prompt ? 0x7fffffff : c.split ? kPromptRows : 0;
    return c;
}

}  // namespace
}  // namespace qllm

extern "C" int64_t qllm_kv_attention_workspace(const qllm_kv_cache_t* cache, int q_heads, int dtype, const qllm_kv_batch_t* batch) {
    const int rc = qllm::check_attention(cache, q_heads, dtype, batch);
    if (rc != QLLM_OK) return rc;
    if (batch->rows == 0 || batch->seqs == 0) return 0;
    const qllm::Choice ch = qllm::choose(cache, q_heads, dtype, batch);
    const int64_t split = ch.split ? qllm::kv::split_workspace(cache->head_dim, dtype, ch.prompt ? qllm::kPromptRows : ch.hint) : 0;
    const int64_t prompt = ch.prompt ? qllm::kv::prompt_workspace(qllm::kv::view(batch, cache), cache->kv_heads, cache->head_dim, q_heads / cache->kv_heads, batch->max_new) : 0;
    return std::max(split, prompt);                        // one after the other on the stream
}

extern "C" int qllm_kv_attention(const qllm_kv_cache_t* cache, int layer, const void* q, int64_t q_stride, void* out,
                                 int64_t out_stride, int dtype, int q_heads, float scale, int causal, float* lse,
                                 const qllm_kv_batch_t* batch, void* workspace, int64_t workspace_bytes, void* stream) {
    using namespace qllm;
    int rc = check_attention(cache, q_heads, dtype, batch);
    if (rc != QLLM_OK) return rc;
    if (layer < 0 || layer >= cache->layers || !isfinite(scale)) return QLLM_ERR_SHAPE;
    if (batch->rows == 0 || batch->seqs == 0) return QLLM_OK;
    rc = check_packed(q, q_stride, q_heads, cache->head_dim, dtype);
    if (rc == QLLM_OK) rc = check_packed(out, out_stride, q_heads, cache->head_dim, dtype);
    if (rc != QLLM_OK) return rc;
    const int64_t need = qllm_kv_attention_workspace(cache, q_heads, dtype, batch);
    if (need > 0 && !workspace) return QLLM_ERR_NULL;
    if (workspace_bytes < need) return QLLM_ERR_SHAPE;
    if (need > 0 && !aligned16(workspace)) return QLLM_ERR_ALIGN;
    int* status = device_status_word();
    if (!status) return QLLM_ERR_CUDA;
    const kv::Cache c = kv::view(cache, layer);
    const kv::Batch b = kv::view(batch, cache);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    kv::AttnArgs a;
    a.q = q;
    a.out = out;
    a.lse = lse;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.dtype = dtype;
    a.q_heads = q_heads;
    a.group = q_heads / cache->kv_heads;
    a.causal = causal;
    a.scale = scale;
    const Choice ch = choose(cache, q_heads, dtype, batch);
    a.most_rows = ch.most_rows;
    if (ch.prompt) rc = kv::launch_attention_prompt(c, b, cache->head_dim, a, batch->max_new, workspace, status, st);
    if (rc == QLLM_OK && ch.split) rc = kv::launch_attention_split(c, b, cache->head_dim, a, ch.prompt ? kPromptRows : ch.hint, workspace, status, st);
    return rc;
}
