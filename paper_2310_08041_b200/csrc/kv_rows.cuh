// What the kernels that store rows in the 4-bit cache share: a row's codes and parameters (Eq. 2 with the exceptions that finite
// rows need), and the way from a CTA's run of packed tokens to their places.
#pragma once

#include "kv_cache.cuh"
#include "reassemble_quant_common.cuh"

namespace qllm {
namespace kv {

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

// Scale, its reciprocal and zero-point of a row with this range (NaN in lo: a row with a NaN).  f: the lane's channels, which
// fit_range may move.
__device__ __forceinline__ void row_params(float (&f)[2][8], float lo, float hi, float& alpha, float& inv, float& zero) {
    const bool wide = hi - lo == INFINITY;                 // a finite row's scale is finite all the same
    alpha = fifteenth(wide ? 0.5f * hi - 0.5f * lo : hi - lo) * (wide ? 2.f : 1.f);
    if (!(hi > lo)) alpha = lo != 0.f ? fabsf(lo) : 1.f;
    if (alpha < kLeastScale) alpha = kLeastScale;          // (not for NaN)
    inv = __frcp_rn(alpha);
    zero = -rintf(lo * inv);
    if (alpha > 0x1p120f) fit_range(f, lo, hi, alpha, inv, zero);
}

constexpr int kMostTokens = 32;                            // of a CTA

// The sequence of token t0 + i of a CTA's run, or -1, for lane i of a warp (i < n).  It is found by counting the row ranges that
// begin at or in front of the token, 32 at a time in one load, up to 128 sequences; a search by halves, whose loads wait for one
// another, made a small call a microsecond longer.
__device__ __forceinline__ int seq_of_lane(const Batch& b, int64_t t0, int n, int lane) {
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
    return s;
}

// (page, place) of the CTA's tokens in shared memory: page < 0 where the token has none (-1: nobody's row, -2: absent).  Lane i of
// the first warp has token i.
__device__ __forceinline__ void find_places(const Cache& c, const Batch& b, int64_t t0, int n, int2* s_place, int* status) {
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x;
        const int64_t t = t0 + lane;
        const int s = seq_of_lane(b, t0, n, lane);
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

}  // namespace kv
}  // namespace qllm
