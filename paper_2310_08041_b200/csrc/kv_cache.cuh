// What the kernels of the 4-bit key/value cache share: views of the caller's structures, the way from a packed row to
// its place in the cache, host-side argument checks.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.h"

namespace qllm {
namespace kv {

// Raises the library's status word for an index that is out of range (a wait that expired is not overwritten).
__device__ __forceinline__ void raise_page(int* status) { atomicCAS(status, QLLM_OK, QLLM_ERR_PAGE); }

// One layer of the cache.  Row r of it = ((page * heads + head) << page_log2) + place in the page.
struct Cache {
    uint8_t *kc, *vc;
    float2 *kp, *vp;                                       // (scale, zero-point)
    int pages, heads, page_log2;
    __device__ __forceinline__ int64_t row(int page, int head, int place) const {
        return ((int64_t(page) * heads + head) << page_log2) + place;
    }
};

struct Batch {
    const int32_t *table, *lens, *start;
    int seqs, width, page_log2;
    int64_t rows;
    // length of sequence s, cut to what its table row can hold
    __device__ __forceinline__ int len(int s) const {
        const int64_t top = int64_t(width) << page_log2;
        const int l = lens[s];
        return l < 0 ? 0 : (l > top ? int(top) : l);
    }
    __device__ __forceinline__ int64_t row(int s) const {
        const int64_t r = start[s];
        return r < 0 ? 0 : (r > rows ? rows : r);
    }
    // new tokens of sequence s (none where q_start decreases)
    __device__ __forceinline__ int count(int s) const {
        const int64_t n = row(s + 1) - row(s);
        return n < 0 ? 0 : int(n);
    }
    // The sequence that packed row t belongs to, or -1: the last one whose first row is not behind t.
    __device__ __forceinline__ int seq_of(int64_t t) const {
        int lo = 0, hi = seqs;                             // rows of sequences < lo begin at or before t, of >= hi behind it
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (start[mid] <= t) lo = mid + 1; else hi = mid;
        }
        return lo > 0 && t >= row(lo - 1) && t - row(lo - 1) < count(lo - 1) ? lo - 1 : -1;
    }
    // Raises the status word for lengths and row ranges that had to be cut: `n` threads of one CTA, this is number `i`.
    __device__ __forceinline__ void report(int* status, int i, int n) const {
        for (int s = i; s < seqs; s += n) {
            const int a = start[s], b = start[s + 1];
            if (lens[s] != len(s) || a < 0 || b < a || b > rows) raise_page(status);
        }
    }
};

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&f)[8]);
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&f)[8]) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
template <>
__device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16* p, float (&f)[8]) {
    const uint4 r = __ldg(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        f[2 * k] = __uint_as_float(w[k] << 16);
        f[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void store8(float* p, const float (&f)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * k], f[2 * k + 1]);
        w[k] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// ---- host side: argument checks, in the order of the error codes' documentation --------------------------------
inline int page_log2(int page_size) {
    switch (page_size) {
        case 16: return 4; case 32: return 5; case 64: return 6; case 128: return 7; case 256: return 8;
        default: return -1;
    }
}
inline bool head_dim_ok(int d) { return d == 64 || d == 128 || d == 256; }

inline int check_cache(const qllm_kv_cache_t* c) {
    if (!c) return QLLM_ERR_NULL;
    if (c->layers <= 0 || c->pages <= 0 || c->kv_heads <= 0 || c->page_size <= 0 || c->head_dim <= 0) return QLLM_ERR_SHAPE;
    if (page_log2(c->page_size) < 0 || !head_dim_ok(c->head_dim) || c->kv_heads > 1024) return QLLM_ERR_UNSUPPORTED;
    if (!c->k_codes || !c->k_param || !c->v_codes || !c->v_param) return QLLM_ERR_NULL;
    if (!aligned16(c->k_codes) || !aligned16(c->k_param) || !aligned16(c->v_codes) || !aligned16(c->v_param)) return QLLM_ERR_ALIGN;
    return QLLM_OK;
}
// rows of packed tensors and sequences are counted in 31 bits
inline int check_batch(const qllm_kv_batch_t* b) {
    if (!b) return QLLM_ERR_NULL;
    if (b->seqs < 0 || b->table_width <= 0 || b->rows < 0 || b->max_new < 0) return QLLM_ERR_SHAPE;
    if (b->rows > (int64_t(1) << 30) || b->seqs > (1 << 20) || b->table_width > (1 << 23)) return QLLM_ERR_UNSUPPORTED;
    if (b->seqs > 0 && b->rows > 0 && (!b->table || !b->seq_lens || !b->q_start)) return QLLM_ERR_NULL;
    return QLLM_OK;
}
// Both at once; positions are counted in 30 bits.
inline int check_cache_batch(const qllm_kv_cache_t* c, const qllm_kv_batch_t* b) {
    int rc = check_cache(c);
    if (rc == QLLM_OK) rc = check_batch(b);
    if (rc != QLLM_OK) return rc;
    return int64_t(b->table_width) * c->page_size > (int64_t(1) << 30) ? QLLM_ERR_UNSUPPORTED : QLLM_OK;
}
// A packed tensor of `heads` heads; dtype has been checked.
inline int check_packed(const void* p, int64_t stride, int heads, int head_dim, int dtype) {
    if (!p) return QLLM_ERR_NULL;
    if (stride < int64_t(heads) * head_dim) return QLLM_ERR_SHAPE;
    if (!aligned16(p) || (stride * (dtype == QLLM_BF16 ? 2 : 4)) % 16) return QLLM_ERR_ALIGN;
    return QLLM_OK;
}
inline Cache view(const qllm_kv_cache_t* c, int layer) {
    Cache v;
    const int64_t rows = int64_t(c->pages) * c->kv_heads * c->page_size * layer;   // rows of the layers in front
    v.kc = c->k_codes + rows * (c->head_dim / 2);
    v.vc = c->v_codes + rows * (c->head_dim / 2);
    v.kp = reinterpret_cast<float2*>(c->k_param) + rows;
    v.vp = reinterpret_cast<float2*>(c->v_param) + rows;
    v.pages = c->pages;
    v.heads = c->kv_heads;
    v.page_log2 = page_log2(c->page_size);
    return v;
}
inline Batch view(const qllm_kv_batch_t* b, const qllm_kv_cache_t* c) {
    return Batch{b->table, b->seq_lens, b->q_start, b->seqs, b->table_width, page_log2(c->page_size), b->rows};
}

}  // namespace kv
}  // namespace qllm
