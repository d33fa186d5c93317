// Storing keys and values in the 4-bit cache and reading them back.
//
// qllm_kv_append is the per-token quantizer of Eq. 2 on rows of one head, written to the row's place in its page:
// alpha = (max - min) / 15, zero = -round(min / alpha), code = clamp(round(x / alpha) + zero, 0, 15), with the float32
// arithmetic of qllm_quantize_rows' one-pass kernels (the same operations: the codes are the same).  Both directions move
// bytes: head_dim values of 2 or 4 bytes on one side, head_dim / 2 + 8 bytes on the other.  head_dim / 16 lanes own a row, 16
// channels each: 16-byte accesses of the values, 8 bytes of codes, the range by shuffles inside the group.  (With 8 channels a
// lane, the instructions that a row costs whatever its length were most of them: 94 us instead of 64 to store 9708 bf16 tokens
// of 2 x 32 rows of 128, 50 instead of 46 to read them; 31 is what the bytes take at the copy rate.  What is left is latency:
// storing keeps DRAM a third and the issue slots 60 % busy, and its warps, 32 to an SM of 64 registers, wait for their loads.)
// A CTA takes a run of tokens: where each belongs (sequence, page, place) is found once per token by one thread, for all of its
// 2 kv_heads rows, and two rows of a group are in flight together.

#include <algorithm>

#include "kv_cache.cuh"
#include "reassemble_quant_common.cuh"

namespace qllm {
namespace {

using namespace kv;

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

// The smaller one, NaN if either is: a row's NaN reaches its scale and zero-point through its minimum, and the row reads back as NaN.
__device__ __forceinline__ float min_nan(float a, float b) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// The least scale: its reciprocal is still a float32 number, that of 2^-128 is infinite.
constexpr float kLeastScale = 0x1p-127f;

constexpr int kMostTokens = 32;                            // of a CTA

// A CTA's run of tokens.  Its row units are ordered [token][keys, values][head].
struct Run {
    int tokens;                                            // per CTA
    uint32_t inverse;                                      // ceil(2^32 / (2 heads)): unit -> token, units < 2^16
};

// (page, place) of the CTA's tokens in shared memory: page < 0 where the token has none (-1: nobody's row, -2: absent).  Lane i of
// the first warp has token i.  A token's sequence is found by counting the row ranges that begin at or in front of it, 32 at a time
// in one load, up to 128 sequences; a search by halves, whose loads wait for one another, made a small call a microsecond longer.
__device__ __forceinline__ void find_places(const Cache& c, const Batch& b, int64_t t0, int n, int2* s_place, int* status) {
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x;
        const int64_t t = t0 + lane;
        int s = -1;
        if (b.seqs <= 128) {
            int first[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) first[i] = 32 * i + lane < b.seqs ? b.start[32 * i + lane] : 0x7fffffff;
            for (int k = 0; k < n; ++k) {
                int before = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (32 * i < b.seqs) before += __popc(__ballot_sync(0xffffffffu, first[i] <= t0 + k));
                if (lane == k) s = before - 1;
            }
            if (lane < n && s >= 0 && !(t >= b.row(s) && t - b.row(s) < b.count(s))) s = -1;
        } else if (lane < n) {
            s = b.seq_of(t);
        }
        if (lane < n) {
            int2 at = make_int2(-1, 0);
            if (s >= 0) {
                const int64_t pos = int64_t(b.len(s)) - b.count(s) + (t - b.row(s));
                at.x = -2;
                if (pos >= 0) {
                    const int page = b.table[int64_t(s) * b.width + (pos >> b.page_log2)];
                    if (page >= 0 && page < c.pages) at = make_int2(page, int(pos) & ((1 << b.page_log2) - 1));
                    else raise_page(status);
                }
            }
            s_place[lane] = at;
        }
    }
    __syncthreads();
}

// x / 15 correctly rounded: the product with 1/15 corrected by its exact residual (Markstein), where nothing underflows
__device__ __forceinline__ float fifteenth(float x) {
    const float q = x * (1.f / 15.f);
    return x > 1e-30f && x < 1e38f ? fmaf(fmaf(-15.f, q, x), 1.f / 15.f, q) : x / 15.f;
}

// A finite row with values near the end of its type: where a rounded zero-point would put the row's first or last value beyond the type,
// the zero-point is the quotient itself, both ends a little inside the row's (2^-20: float32 roundings cannot take them out again).
// The row is moved by the zero-point's fraction instead, at half its size, so that its codes follow as from a rounded one.
__device__ __forceinline__ void fit_range(float (&f)[2][8], float lo, float hi, float& alpha, float& inv, float& zero) {
    if (alpha == INFINITY || fmaxf(zero, rintf(hi * inv)) * alpha <= 3.38953139e38f) return;     // bf16's largest number
    alpha *= 1.f - 0x1p-20f;
    inv = __frcp_rn(alpha);
    zero = -lo * inv * (1.f - 0x1p-21f);
    const float by = 0.5f * (zero - truncf(zero)) * alpha;
#pragma unroll
    for (int j = 0; j < 16; ++j) f[j >> 3][j & 7] = fmaf(0.5f, f[j >> 3][j & 7], by);
    inv *= 2.f;
}

template <typename T, int D>
__global__ void __launch_bounds__(256)
kv_append_kernel(const T* __restrict__ k, int64_t k_stride, const T* __restrict__ v, int64_t v_stride, Cache c, Batch b, Run run, int* status) {
    constexpr int L = D / 16, G = 256 / L, U = 2;          // lanes of a row, rows of a CTA and step, steps in flight
    __shared__ int2 s_place[kMostTokens];
    const int lane = threadIdx.x % L, group = threadIdx.x / L, per_token = 2 * c.heads;
    const int64_t t0 = int64_t(blockIdx.x) * run.tokens;
    const int tokens = int(min(int64_t(run.tokens), b.rows - t0)), units = tokens * per_token;
    for (int base = 0; base < units; base += G * U) {
        float f[U][2][8];
        int tok[U], w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = base + u * G + group;
            tok[u] = int(__umulhi(uint32_t(r), run.inverse));
            w[u] = r - tok[u] * per_token;
            if (r < units) {
                const int64_t t = t0 + tok[u];
                const T* p = (w[u] < c.heads ? k + t * k_stride + w[u] * D : v + t * v_stride + (w[u] - c.heads) * D) + lane * 16;
                load8<T>(p, f[u][0]);
                load8<T>(p + 8, f[u][1]);
            } else {
                tok[u] = -1;
#pragma unroll
                for (int j = 0; j < 16; ++j) f[u][j >> 3][j & 7] = 0.f;
            }
        }
        if (base == 0) {                                   // under the first loads
            find_places(c, b, t0, tokens, s_place, status);
            if (blockIdx.x == 0) b.report(status, threadIdx.x, 256);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (base + u * G >= units) break;              // the whole CTA is done
            float lo = f[u][0][0], hi = lo;
#pragma unroll
            for (int j = 1; j < 16; ++j) { lo = min_nan(lo, f[u][j >> 3][j & 7]); hi = fmaxf(hi, f[u][j >> 3][j & 7]); }
#pragma unroll
            for (int o = L / 2; o > 0; o >>= 1) {
                lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
                hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
            }
            const int2 at = tok[u] < 0 ? make_int2(-1, 0) : s_place[tok[u]];
            if (at.x >= 0) {
                const bool wide = hi - lo == INFINITY;     // a finite row's scale is finite all the same
                float alpha = fifteenth(wide ? 0.5f * hi - 0.5f * lo : hi - lo) * (wide ? 2.f : 1.f);
                if (!(hi > lo)) alpha = lo != 0.f ? fabsf(lo) : 1.f;
                if (alpha < kLeastScale) alpha = kLeastScale;                // (not for NaN)
                float inv = __frcp_rn(alpha), zero = -rintf(lo * inv);
                if (alpha > 0x1p120f) fit_range(f[u], lo, hi, alpha, inv, zero);
                const bool keys = w[u] < c.heads;
                const int64_t row = c.row(at.x, keys ? w[u] : w[u] - c.heads, at.y);
                reinterpret_cast<uint2*>((keys ? c.kc : c.vc) + row * (D / 2))[lane] =
                    make_uint2(codes8(f[u][0], lo, hi, inv, zero), codes8(f[u][1], lo, hi, inv, zero));
                if (lane == 0) (keys ? c.kp : c.vp)[row] = make_float2(alpha, zero);
            }
        }
    }
}

// 8 codes of a word -> (code - zero) scale.  Integer zero-points below 2^22: 2^23 + code is made by a byte permutation, and the
// difference to 2^23 + zero is exact; others by conversion.
__device__ __forceinline__ void values8(uint32_t w, float zero, float scale, bool plain, float (&f)[8]) {
    const uint32_t even = w & 0x0F0F0F0Fu, odd = (w >> 4) & 0x0F0F0F0Fu;
    const float sub = 8388608.f + zero;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t e = __byte_perm(even, 0x4B000000u, 0x7440u + j), o = __byte_perm(odd, 0x4B000000u, 0x7440u + j);
        f[2 * j] = (plain ? __uint_as_float(e) - sub : float(e & 15u) - zero) * scale;
        f[2 * j + 1] = (plain ? __uint_as_float(o) - sub : float(o & 15u) - zero) * scale;
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(256)
kv_read_kernel(T* __restrict__ k, int64_t k_stride, T* __restrict__ v, int64_t v_stride, Cache c, Batch b, Run run, int* status) {
    constexpr int L = D / 16, G = 256 / L, U = 2;
    __shared__ int2 s_place[kMostTokens];
    const int lane = threadIdx.x % L, group = threadIdx.x / L, per_token = 2 * c.heads;
    const int64_t t0 = int64_t(blockIdx.x) * run.tokens;
    const int tokens = int(min(int64_t(run.tokens), b.rows - t0)), units = tokens * per_token;
    find_places(c, b, t0, tokens, s_place, status);
    if (blockIdx.x == 0) b.report(status, threadIdx.x, 256);
    for (int base = 0; base < units; base += G * U) {
        uint2 word[U];
        float2 prm[U];
        int tok[U], w[U], page[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = base + u * G + group;
            tok[u] = int(__umulhi(uint32_t(r), run.inverse));
            w[u] = r - tok[u] * per_token;
            const int2 at = r < units ? s_place[tok[u]] : make_int2(-1, 0);
            page[u] = at.x;
            word[u] = make_uint2(0, 0);
            prm[u] = make_float2(0.f, 0.f);
            if (at.x >= 0) {
                const bool keys = w[u] < c.heads;
                const int64_t row = c.row(at.x, keys ? w[u] : w[u] - c.heads, at.y);
                word[u] = reinterpret_cast<const uint2*>((keys ? c.kc : c.vc) + row * (D / 2))[lane];
                prm[u] = (keys ? c.kp : c.vp)[row];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (page[u] == -1) continue;
            const int64_t t = t0 + tok[u];
            T* p = (w[u] < c.heads ? k + t * k_stride + w[u] * D : v + t * v_stride + (w[u] - c.heads) * D) + lane * 16;
            const bool plain = fabsf(prm[u].y) < 4194304.f && prm[u].y == rintf(prm[u].y);
            float f[8];
            values8(word[u].x, prm[u].y, prm[u].x, plain, f);
            store8(p, f);
            values8(word[u].y, prm[u].y, prm[u].x, plain, f);
            store8(p + 8, f);
        }
    }
}

// Tokens of a CTA: as many as keep eight CTAs on every SM, at most 1024 rows' worth (unit numbers stay below 2^16) and at least
// one step's worth where a token has few rows.
inline Run run_of(const Batch& b, int heads, int rows_per_step) {
    const int per_token = 2 * heads;
    int64_t n = b.rows / (int64_t(device_sm_count()) * 8);
    n = std::min<int64_t>(n, std::max(1, 16 * rows_per_step / per_token));
    n = std::max<int64_t>(n, std::min(rows_per_step / per_token, 8));
    n = std::min<int64_t>(std::max<int64_t>(n, 1), kMostTokens);
    return Run{int(n), uint32_t(((uint64_t(1) << 32) + per_token - 1) / per_token)};
}

template <typename T, int D>
int launch_append(const void* k, int64_t ks, const void* v, int64_t vs, const Cache& c, const Batch& b, int* status, cudaStream_t st) {
    const Run run = run_of(b, c.heads, 256 / (D / 16));
    kv_append_kernel<T, D><<<unsigned((b.rows + run.tokens - 1) / run.tokens), 256, 0, st>>>(
        static_cast<const T*>(k), ks, static_cast<const T*>(v), vs, c, b, run, status);
    return after_launch();
}
template <typename T, int D>
int launch_read(void* k, int64_t ks, void* v, int64_t vs, const Cache& c, const Batch& b, int* status, cudaStream_t st) {
    const Run run = run_of(b, c.heads, 256 / (D / 16));
    kv_read_kernel<T, D><<<unsigned((b.rows + run.tokens - 1) / run.tokens), 256, 0, st>>>(
        static_cast<T*>(k), ks, static_cast<T*>(v), vs, c, b, run, status);
    return after_launch();
}

int check_tokens(const qllm_kv_cache_t* cache, int layer, const void* k, int64_t ks, const void* v, int64_t vs, int dtype,
                 const qllm_kv_batch_t* batch) {
    if (!dtype_ok(dtype)) return QLLM_ERR_DTYPE;
    int rc = check_cache_batch(cache, batch);
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
