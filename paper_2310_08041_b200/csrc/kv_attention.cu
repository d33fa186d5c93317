// Attention over the 4-bit key/value cache: entry points and the plain kernel.
//
// s_j = scale q . k_j with k_j = ks_j (ck_j - kz_j), softmax with a running maximum and sum, out = sum p_j v_j / sum p_j
// with v_j = vs_j (cv_j - vz_j).  One warp per (row, query head) walks the row's keys; every statistic is float32.

#include <math.h>

#include "device_utils.cuh"
#include "kv_cache.cuh"

namespace qllm {
namespace {

using namespace kv;

template <typename T, int D>
__global__ void __launch_bounds__(128)
kv_attention_plain(const T* __restrict__ q, int64_t q_stride, T* __restrict__ out, int64_t out_stride, Cache c, Batch b,
                   int q_heads, float scale, int causal, float* __restrict__ lse, int* status) {
    constexpr int N = D / 32;
    if (blockIdx.x == 0) b.report(status);
    const int lane = threadIdx.x & 31;
    const int64_t unit = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 5);
    const int64_t t = unit / q_heads;
    const int h = int(unit - t * q_heads), g = h / (q_heads / c.heads);
    if (t >= b.rows) return;
    const int s = b.seq_of(t);
    if (s < 0) return;
    const int len = b.len(s), n = b.count(s);
    const int64_t own = int64_t(len) - n + (t - b.row(s));
    const int keys = causal ? int(own < 0 ? 0 : own + 1) : len;
    float qf[N], acc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        qf[i] = float(q[t * q_stride + int64_t(h) * D + lane * N + i]);
        acc[i] = 0.f;
    }
    float m = -INFINITY, l = 0.f;
    for (int j = 0; j < keys; ++j) {
        const int page = b.table[int64_t(s) * b.width + (j >> b.page_log2)];
        if (page < 0 || page >= c.pages) { if (lane == 0) raise_page(status); continue; }
        const int64_t row = c.row(page, g, j & ((1 << b.page_log2) - 1));
        const float2 kp = c.kp[row], vp = c.vp[row];
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int ch = lane * N + i;
            dot += qf[i] * (float((c.kc[row * (D / 2) + ch / 2] >> (4 * (ch & 1))) & 15) - kp.y);
        }
        const float sc = warp_sum(dot) * kp.x * scale;
        const float m2 = fmaxf(m, sc), at = m2 == -INFINITY ? 0.f : m2;     // a NaN score passes the maximum by and makes l NaN
        const float fix = expf(m - at), p = expf(sc - at);
        l = l * fix + p;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int ch = lane * N + i;
            acc[i] = acc[i] * fix + p * vp.x * (float((c.vc[row * (D / 2) + ch / 2] >> (4 * (ch & 1))) & 15) - vp.y);
        }
        m = m2;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) out[t * out_stride + int64_t(h) * D + lane * N + i] = T(l > 0.f ? acc[i] / l : (l == 0.f ? 0.f : l));
    if (lse && lane == 0) lse[t * q_heads + h] = l > 0.f ? m + logf(l) : (l == 0.f ? -INFINITY : l);
}

int check_attention(const qllm_kv_cache_t* cache, int q_heads, int dtype, const qllm_kv_batch_t* batch) {
    if (!dtype_ok(dtype)) return QLLM_ERR_DTYPE;
    int rc = check_cache(cache);
    if (rc == QLLM_OK) rc = check_batch(batch);
    if (rc != QLLM_OK) return rc;
    if (q_heads <= 0 || q_heads % cache->kv_heads) return QLLM_ERR_SHAPE;
    if (q_heads > 65535) return QLLM_ERR_UNSUPPORTED;
    return QLLM_OK;
}

}  // namespace
}  // namespace qllm

extern "C" int64_t qllm_kv_attention_workspace(const qllm_kv_cache_t* cache, int q_heads, int dtype, const qllm_kv_batch_t* batch) {
    const int rc = qllm::check_attention(cache, q_heads, dtype, batch);
    return rc != QLLM_OK ? rc : 0;
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
    const int64_t grid = (b.rows * q_heads + 3) / 4;
    if (grid > 0x7fffffff) return QLLM_ERR_UNSUPPORTED;
#define QLLM_KV_D(T, D)                                                                                                 \
    if (cache->head_dim == D) {                                                                                         \
        kv_attention_plain<T, D><<<unsigned(grid), 128, 0, st>>>(static_cast<const T*>(q), q_stride, static_cast<T*>(out), \
                                                                 out_stride, c, b, q_heads, scale, causal, lse, status); \
        return after_launch();                                                                                          \
    }
    if (dtype == QLLM_BF16) { QLLM_KV_D(__nv_bfloat16, 64); QLLM_KV_D(__nv_bfloat16, 128); QLLM_KV_D(__nv_bfloat16, 256); }
    else { QLLM_KV_D(float, 64); QLLM_KV_D(float, 128); QLLM_KV_D(float, 256); }
#undef QLLM_KV_D
    return QLLM_ERR_UNSUPPORTED;
}
