// Storing keys and values in the 4-bit cache and reading them back.
//
// qllm_kv_append is the per-token quantizer of Eq. 2 on rows of one head, written to the row's place in its page:
// alpha = (max - min) / 15, zero = -round(min / alpha), code = clamp(round(x / alpha) + zero, 0, 15), with the float32
// arithmetic of qllm_quantize_rows (the same operations in the same order: the codes are the same).  Both directions
// move bytes: head_dim values of 2 or 4 bytes on one side, head_dim / 2 + 8 bytes on the other.  head_dim / 8 lanes own
// a row, 8 channels each: one or two 16-byte accesses of the values, one 32-bit word of codes, the range by shuffles
// inside the group, whole 32-byte sectors on both sides.  A group takes U rows of keys or values at once (their loads
// are in flight together, and the search for a row's sequence and page runs under them).

#include "kv_cache.cuh"
#include "reassemble_quant_common.cuh"

namespace qllm {
namespace {

using namespace kv;

// Place of packed row t: true and (page, place) when the token has a position and its page exists.
__device__ __forceinline__ bool find_place(const Cache& c, const Batch& b, int64_t t, int& s, int& page, int& place, int* status) {
    s = b.seq_of(t);
    if (s < 0) return false;
    const int64_t pos = int64_t(b.len(s)) - b.count(s) + (t - b.row(s));
    if (pos < 0) return false;
    page = b.table[int64_t(s) * b.width + (pos >> b.page_log2)];
    place = int(pos) & ((1 << b.page_log2) - 1);
    if (page < 0 || page >= c.pages) { raise_page(status); return false; }
    return true;
}

// Eq. 2 on 8 channels of a row whose range is known (quantize_rows.cu has the derivation of the rounding).
__device__ __forceinline__ uint32_t codes8(const float (&f)[8], float lo, float hi, float inv, float zero) {
    int n[8];
    if (fmaxf(fabsf(lo), fabsf(hi)) * inv < 2097152.f && fabsf(zero) < 2097152.f) {
        const int zadd = int(zero) - kMagicBits;
#pragma unroll
        for (int j = 0; j < 8; ++j) n[j] = __float_as_int(fmaf(f[j], inv, kMagic)) + zadd;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) n[j] = int(fminf(fmaxf(rintf(f[j] * inv) + zero, 0.f), 15.f));
    }
    uint32_t p = 0;
#pragma unroll
    for (int k = 3; k >= 0; --k) p = pack_sat_u4(n[2 * k + 1], n[2 * k], p);
    return p;
}

// Row units are ordered [packed row][keys, values][head].
template <typename T, int D, int U>
__global__ void __launch_bounds__(256)
kv_append_kernel(const T* __restrict__ k, int64_t k_stride, const T* __restrict__ v, int64_t v_stride, Cache c, Batch b, int* status) {
    constexpr int L = D / 8, G = 256 / L;                  // lanes of a row, rows of a CTA and step
    if (blockIdx.x == 0) b.report(status);
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    const int64_t units = b.rows * 2 * c.heads, first = int64_t(blockIdx.x) * (G * U) + group;
    float f[U][8];
    bool live[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t r = first + u * G;
        live[u] = r < units;
        const int64_t t = live[u] ? r / (2 * c.heads) : 0;
        const int w = live[u] ? int(r - t * (2 * c.heads)) : 0;
        const T* p = w < c.heads ? k + t * k_stride + int64_t(w) * D : v + t * v_stride + int64_t(w - c.heads) * D;
        if (live[u]) load8<T>(p + lane * 8, f[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float lo = INFINITY, hi = -INFINITY;
        if (live[u]) {
#pragma unroll
            for (int j = 0; j < 8; ++j) { lo = fminf(lo, f[u][j]); hi = fmaxf(hi, f[u][j]); }
        }
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) {
            lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
            hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        }
        if (!live[u]) continue;
        const int64_t r = first + u * G, t = r / (2 * c.heads);
        const int w = int(r - t * (2 * c.heads));
        int s, page, place;
        if (!find_place(c, b, t, s, page, place, status)) continue;
        float alpha = (hi - lo) / 15.f;
        if (!(hi > lo)) alpha = lo != 0.f ? fabsf(lo) : 1.f;
        const float inv = __frcp_rn(alpha), zero = -rintf(lo * inv);
        const bool keys = w < c.heads;
        const int64_t row = c.row(page, keys ? w : w - c.heads, place);
        reinterpret_cast<uint32_t*>((keys ? c.kc : c.vc) + row * (D / 2))[lane] = codes8(f[u], lo, hi, inv, zero);
        if (lane == 0) (keys ? c.kp : c.vp)[row] = make_float2(alpha, zero);
    }
}

template <typename T, int D, int U>
__global__ void __launch_bounds__(256)
kv_read_kernel(T* __restrict__ k, int64_t k_stride, T* __restrict__ v, int64_t v_stride, Cache c, Batch b, int* status) {
    constexpr int L = D / 8, G = 256 / L;
    if (blockIdx.x == 0) b.report(status);
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    const int64_t units = b.rows * 2 * c.heads, first = int64_t(blockIdx.x) * (G * U) + group;
    uint32_t word[U];
    float2 prm[U];
    bool live[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t r = first + u * G, t = r / (2 * c.heads);
        const int w = int(r - t * (2 * c.heads));
        int s = -1, page, place;
        word[u] = 0;
        prm[u] = make_float2(0.f, 0.f);
        if (r < units && find_place(c, b, t, s, page, place, status)) {
            const bool keys = w < c.heads;
            const int64_t row = c.row(page, keys ? w : w - c.heads, place);
            word[u] = reinterpret_cast<const uint32_t*>((keys ? c.kc : c.vc) + row * (D / 2))[lane];
            prm[u] = (keys ? c.kp : c.vp)[row];
        }
        live[u] = s >= 0;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (!live[u]) continue;
        const int64_t r = first + u * G, t = r / (2 * c.heads);
        const int w = int(r - t * (2 * c.heads));
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = (float((word[u] >> (4 * j)) & 15u) - prm[u].y) * prm[u].x;
        store8((w < c.heads ? k + t * k_stride + int64_t(w) * D : v + t * v_stride + int64_t(w - c.heads) * D) + lane * 8, f);
    }
}

// Four rows per group once that still gives every SM two CTAs; single rows below (more CTAs, shorter latency).
inline bool four_rows(int64_t units, int rows_per_step) {
    return units >= int64_t(device_sm_count()) * 2 * 4 * rows_per_step;
}

template <typename T, int D>
int launch_append(const void* k, int64_t ks, const void* v, int64_t vs, const Cache& c, const Batch& b, int* status, cudaStream_t st) {
    constexpr int G = 256 / (D / 8);
    const int64_t units = b.rows * 2 * c.heads;
    const T *kp = static_cast<const T*>(k), *vp = static_cast<const T*>(v);
    if (four_rows(units, G)) {
        const int64_t grid = (units + 4 * G - 1) / (4 * G);
        if (grid > 0x7fffffff) return QLLM_ERR_UNSUPPORTED;
        kv_append_kernel<T, D, 4><<<unsigned(grid), 256, 0, st>>>(kp, ks, vp, vs, c, b, status);
    } else {
        kv_append_kernel<T, D, 1><<<unsigned((units + G - 1) / G), 256, 0, st>>>(kp, ks, vp, vs, c, b, status);
    }
    return after_launch();
}
template <typename T, int D>
int launch_read(void* k, int64_t ks, void* v, int64_t vs, const Cache& c, const Batch& b, int* status, cudaStream_t st) {
    constexpr int G = 256 / (D / 8);
    const int64_t units = b.rows * 2 * c.heads;
    T *kp = static_cast<T*>(k), *vp = static_cast<T*>(v);
    if (four_rows(units, G)) {
        const int64_t grid = (units + 4 * G - 1) / (4 * G);
        if (grid > 0x7fffffff) return QLLM_ERR_UNSUPPORTED;
        kv_read_kernel<T, D, 4><<<unsigned(grid), 256, 0, st>>>(kp, ks, vp, vs, c, b, status);
    } else {
        kv_read_kernel<T, D, 1><<<unsigned((units + G - 1) / G), 256, 0, st>>>(kp, ks, vp, vs, c, b, status);
    }
    return after_launch();
}

int check_tokens(const qllm_kv_cache_t* cache, int layer, const void* k, int64_t ks, const void* v, int64_t vs, int dtype,
                 const qllm_kv_batch_t* batch) {
    if (!dtype_ok(dtype)) return QLLM_ERR_DTYPE;
    int rc = check_cache(cache);
    if (rc == QLLM_OK) rc = check_batch(batch);
    if (rc != QLLM_OK) return rc;
    if (layer < 0 || layer >= cache->layers) return QLLM_ERR_SHAPE;
    if (batch->rows == 0 || batch->seqs == 0) return QLLM_OK;
    rc = check_packed(k, ks, cache->kv_heads, cache->head_dim, dtype);
    return rc != QLLM_OK ? rc : check_packed(v, vs, cache->kv_heads, cache->head_dim, dtype);
}

}  // namespace
}  // namespace qllm

extern "C" int qllm_kv_append(const qllm_kv_cache_t* cache, int layer, const void* k, int64_t k_stride, const void* v,
                              int64_t v_stride, int dtype, const qllm_kv_batch_t* batch, void* stream) {
    using namespace qllm;
    const int rc = check_tokens(cache, layer, k, k_stride, v, v_stride, dtype, batch);
    if (rc != QLLM_OK || batch->rows == 0 || batch->seqs == 0) return rc;
    int* status = device_status_word();
    if (!status) return QLLM_ERR_CUDA;
    const kv::Cache c = kv::view(cache, layer);
    const kv::Batch b = kv::view(batch, cache);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
#define QLLM_KV_D(T, D) if (cache->head_dim == D) return launch_append<T, D>(k, k_stride, v, v_stride, c, b, status, st)
    if (dtype == QLLM_BF16) { QLLM_KV_D(__nv_bfloat16, 64); QLLM_KV_D(__nv_bfloat16, 128); QLLM_KV_D(__nv_bfloat16, 256); }
    else { QLLM_KV_D(float, 64); QLLM_KV_D(float, 128); QLLM_KV_D(float, 256); }
#undef QLLM_KV_D
    return QLLM_ERR_UNSUPPORTED;
}

extern "C" int qllm_kv_read(const qllm_kv_cache_t* cache, int layer, void* k, int64_t k_stride, void* v, int64_t v_stride,
                            int dtype, const qllm_kv_batch_t* batch, void* stream) {
    using namespace qllm;
    const int rc = check_tokens(cache, layer, k, k_stride, v, v_stride, dtype, batch);
    if (rc != QLLM_OK || batch->rows == 0 || batch->seqs == 0) return rc;
    int* status = device_status_word();
    if (!status) return QLLM_ERR_CUDA;
    const kv::Cache c = kv::view(cache, layer);
    const kv::Batch b = kv::view(batch, cache);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
#define QLLM_KV_D(T, D) if (cache->head_dim == D) return launch_read<T, D>(k, k_stride, v, v_stride, c, b, status, st)
    if (dtype == QLLM_BF16) { QLLM_KV_D(__nv_bfloat16, 64); QLLM_KV_D(__nv_bfloat16, 128); QLLM_KV_D(__nv_bfloat16, 256); }
    else { QLLM_KV_D(float, 64); QLLM_KV_D(float, 128); QLLM_KV_D(float, 256); }
#undef QLLM_KV_D
    return QLLM_ERR_UNSUPPORTED;
}
