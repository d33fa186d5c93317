// qllm_rmsnorm_quant: residual addition, root-mean-square norm, reassembly map (optional) and the per-token quantizer of Eq. 2;
// qllm_dequantize_rows: the values that a row's codes stand for.
//
//   h = x + residual,   r = 1 / sqrt(mean h^2 + eps),   y = gamma h r,   x'_c = sum_j coef_j y[src_j],   Eq. 2 on x'.
//
// r is one number per row and positive, and everything behind it is linear up to Eq. 2's rounding: with u = gamma h and u' the map's
// sums of u, min, max and alpha of x' are r times those of u', and round(x' / alpha) is round(u' / alpha_u).  So the codes and the
// zero-point are made from u', a_scale = r alpha_u, and ONE exchange between the threads of a row serves both the sum of squares and
// the range (normalising first takes two, one after the other).  It also makes the codes independent of the order in which squares
// are added: they are decided by h (one float32 addition), u (one product), u' (rounded once to float32, members are summed in 64
// bits) and Eq. 2 in float32.  Sums of squares are float32 sums of float32 products: at most 8 NV terms per lane in order, then
// trees; C terms of one sign are off by at most (8 NV + 12) 2^-24.
//
// What bounds it: HBM.  A row is read once, kept in registers, and written once.  The CTAs stay and walk the rows (gamma stays in
// registers, the next row is requested before the present one's exchange); the code sum of a row leaves with the next row's exchange.

#include <cuda_bf16.h>

#include <algorithm>

#include "common.h"
#include "device_utils.cuh"
#include "eq2_rows.cuh"

namespace qllm {
namespace {

struct NormArgs {
    const void *x, *residual;
    int64_t M;
    int C;
    const float* gamma;
    float eps;
    const int32_t *ptr, *src;                              // the map (may be null), see qllm_reassemble_quant
    const float* coef;
    int bits;
    void *h, *y;                                           // may be null
    uint8_t* codes;                                        // may be null: only h and y
    float *a_scale, *a_zero;
    int32_t* a_rowsum;                                     // may be null
};

// 8 channels as they lie in memory.  Loads are plain ones: h may be the residual or x in place.
template <typename XT>
struct Raw;
template <>
struct Raw<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            f[2 * k] = __uint_as_float(w[k] << 16);
            f[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&f)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * k], f[2 * k + 1]);
            w[k] = *reinterpret_cast<const uint32_t*>(&b);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <>
struct Raw<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = reinterpret_cast<const float4*>(p)[0];
        b = reinterpret_cast<const float4*>(p)[1];
    }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
    static __device__ __forceinline__ void store(float* p, const float (&f)[8]) {
        reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
    }
};

// Eq. 2's parameters of u' and the row's factor.  ok = false: the row's numbers are too large or too small for float32 squares or
// for a reciprocal of the scale (2^-120: its reciprocal and the products with it stay finite).
struct RowStats {
    float alpha, inv, zero, r;
    bool ok;
    __device__ __forceinline__ RowStats(float ssq, float lo, float hi, int C, float eps, float qmax) {
        const float ms = ssq / float(C) + eps;
        eq2_params(lo, hi, qmax, alpha, inv, zero);
        r = 1.f / sqrtf(ms);
        ok = ms < INFINITY && ms >= 0x1p-80f && hi - lo < INFINITY && (alpha >= 0x1p-120f);
    }
};
// The factor of a row whose channels have been multiplied by `by` (a power of two), in 64 bits.  0 for a row of zeros with eps = 0 and
// for one with an infinity, NaN for one with a NaN.
__device__ __forceinline__ double scaled_factor(float ssq, int C, float eps, float by) {
    const double ms = double(ssq) / double(C) + double(eps) * double(by) * double(by);
    return ms == 0.0 ? 0.0 : 1.0 / sqrt(ms);
}
// The power of two that brings a row's largest magnitude (finite, not 0) to 1 .. 2, as far as float32 holds it.
__device__ __forceinline__ float scale_of(float top) {
    const int e = int(__float_as_uint(top) >> 23) - 127;   // subnormal: -127
    return exp2f(float(-min(max(e, -126), 126)));
}

// MAP: a thread's 8 output channels beside its 8 source channels; u goes through shared memory at word (k % 8) C / 8 + k / 8, where
// neighbouring threads' neighbouring channels lie side by side.  Rows of the map with one entry (all but the merged ones) are held
// in registers for the whole launch: word and coefficient; merged rows are walked in the caller's arrays.
template <typename XT, int NV, int R, bool MAP, int MAXT>
__global__ void __launch_bounds__(MAXT)
rmsnorm_quant_kernel(const NormArgs a) {
    extern __shared__ float s_u[];                         // MAP: R rows of u
    __shared__ float s_red[2][3 * R][32];
    __shared__ int s_sum[2][R][32];
    __shared__ float s_top[R][32];
    const int t = threadIdx.x, T = blockDim.x, lane = t & 31, warp = t >> 5, nw = T >> 5, C = a.C, nvec = C / 8;
    const XT* x = static_cast<const XT*>(a.x);
    const XT* res = static_cast<const XT*>(a.residual);
    XT* h = static_cast<XT*>(a.h);
    XT* y = static_cast<XT*>(a.y);
    const float qmax = float((1 << a.bits) - 1);
    const bool quant = a.codes != nullptr;
    const int64_t step = int64_t(gridDim.x) * R;
    asm volatile("griddepcontrol.wait;" ::: "memory");     // launched as a dependent

    Raw<XT> rx[R][NV], rr[R][NV];
    const auto request = [&](int64_t m0) {
#pragma unroll
        for (int q = 0; q < R; ++q)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int g = t + i * T;
                if (m0 + q < a.M && g < nvec) {
                    const int64_t at = (m0 + q) * C + 8 * g;
                    rx[q][i].load(x + at);
                    if (res) rr[q][i].load(res + at);
                }
            }
    };
    const auto flush = [&](const int (&part)[R][32], int64_t first) {      // by the first warp
        if (!a.a_rowsum) return;
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const int s = warp_sum_int(lane < nw ? part[q][lane] : 0);
            if (lane == 0 && first + q < a.M) a.a_rowsum[first + q] = s;
        }
    };
    int64_t m0 = int64_t(blockIdx.x) * R;
    request(m0);
    float gamma[NV][8];
    uint32_t word[MAP ? NV : 1][8];
    float coef[MAP ? NV : 1][8];
    uint32_t merged[MAP ? NV : 1];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int g = t + i * T;
#pragma unroll
        for (int j = 0; j < 8; ++j) gamma[i][j] = g < nvec ? a.gamma[8 * g + j] : 0.f;
        if (MAP) {
            merged[i] = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                word[i][j] = 0;
                coef[i][j] = 0.f;
                if (g < nvec) {
                    const int b = a.ptr[8 * g + j], e = a.ptr[8 * g + j + 1];
                    if (e - b == 1) {
                        const uint32_t k = uint32_t(a.src[b]);
                        word[i][j] = (k & 7u) * uint32_t(nvec) + (k >> 3);
                        coef[i][j] = a.coef[b];
                    } else {
                        merged[i] |= 1u << j;
                    }
                }
            }
        }
    }

    int parity = 0, turn = 0;
    int64_t before = -1;                                   // first row of the pass whose code sums wait in s_sum[turn ^ 1]
    for (; m0 < a.M; m0 += step) {
        const int live = int(min(int64_t(R), a.M - m0));
        float f[R][NV][8], v[MAP ? R : 1][MAP ? NV : 1][8], by[R];
#pragma unroll
        for (int q = 0; q < R; ++q) {
            by[q] = 1.f;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int g = t + i * T;
                if (q < live && g < nvec) {
                    rx[q][i].get(f[q][i]);
                    if (res) {
                        float o[8];
                        rr[q][i].get(o);
#pragma unroll
                        for (int j = 0; j < 8; ++j) f[q][i][j] += o[j];
                    }
                    if (h) Raw<XT>::store(h + (m0 + q) * C + 8 * g, f[q][i]);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[q][i][j] = 0.f;
                }
            }
        }
        request(m0 + step);

        float ssq[R], lo[R], hi[R];
        for (int pass = 0;; ++pass) {
#pragma unroll
            for (int q = 0; q < R; ++q) {
                ssq[q] = 0.f;
                lo[q] = INFINITY;
                hi[q] = -INFINITY;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int g = t + i * T;
#pragma unroll
                    for (int j = 0; j < 8; ++j) ssq[q] = fmaf(f[q][i][j], f[q][i][j], ssq[q]);
                    if (g < nvec) {
#pragma unroll
                        for (int j = 0; j < 8; j += 2) {
                            const float u0 = f[q][i][j] * gamma[i][j], u1 = f[q][i][j + 1] * gamma[i][j + 1];
                            if (MAP) {
                                s_u[q * C + j * nvec + g] = u0;
                                s_u[q * C + (j + 1) * nvec + g] = u1;
                            } else {
                                lo[q] = min3(lo[q], u0, u1);
                                hi[q] = max3(hi[q], u0, u1);
                            }
                        }
                    }
                }
            }
            if (MAP) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int g = t + i * T;
                    if (g < nvec) {
#pragma unroll
                        for (int j = 0; j < 8; ++j)
#pragma unroll
                            for (int q = 0; q < R; ++q) v[q][i][j] = coef[i][j] * s_u[q * C + word[i][j]];
                        if (merged[i]) {
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                if (merged[i] >> j & 1) {
                                    const int e = a.ptr[8 * g + j + 1];
                                    double s[R];
#pragma unroll
                                    for (int q = 0; q < R; ++q) s[q] = 0.0;
                                    for (int k = a.ptr[8 * g + j]; k < e; ++k) {
                                        const uint32_t from = uint32_t(a.src[k]), w = (from & 7u) * uint32_t(nvec) + (from >> 3);
                                        const double c = double(a.coef[k]);
#pragma unroll
                                        for (int q = 0; q < R; ++q) s[q] = fma(c, double(s_u[q * C + w]), s[q]);
                                    }
#pragma unroll
                                    for (int q = 0; q < R; ++q) v[q][i][j] = float(s[q]);
                                }
                        }
#pragma unroll
                        for (int q = 0; q < R; ++q)
#pragma unroll
                            for (int j = 0; j < 8; j += 2) {
                                lo[q] = min3(lo[q], v[q][i][j], v[q][i][j + 1]);
                                hi[q] = max3(hi[q], v[q][i][j], v[q][i][j + 1]);
                            }
                    }
                }
            }
            parity ^= 1;
#pragma unroll
            for (int q = 0; q < R; ++q) {
                const float s = warp_sum(ssq[q]), l = redux_min(lo[q]), u = redux_max(hi[q]);
                if (lane == 0) {
                    s_red[parity][3 * q][warp] = s;
                    s_red[parity][3 * q + 1][warp] = l;
                    s_red[parity][3 * q + 2][warp] = u;
                }
            }
            __syncthreads();
            bool good = true;
#pragma unroll
            for (int q = 0; q < R; ++q) {
                ssq[q] = warp_sum(lane < nw ? s_red[parity][3 * q][lane] : 0.f);
                lo[q] = redux_min(lane < nw ? s_red[parity][3 * q + 1][lane] : INFINITY);
                hi[q] = redux_max(lane < nw ? s_red[parity][3 * q + 2][lane] : -INFINITY);
                if (q < live) good = good && RowStats(ssq[q], lo[q], hi[q], C, a.eps, qmax).ok;
            }
            if (good || pass) break;                       // the same in every thread
            // a row with very large or very small numbers: all of it by a power of two, exactly, and once more
#pragma unroll
            for (int q = 0; q < R; ++q) {
                float top = 0.f;
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(f[q][i][j]));
                top = redux_max(top);
                if (lane == 0) s_top[q][warp] = top;
            }
            __syncthreads();
#pragma unroll
            for (int q = 0; q < R; ++q) {
                const float top = redux_max(lane < nw ? s_top[q][lane] : 0.f);
                if (q < live && !RowStats(ssq[q], lo[q], hi[q], C, a.eps, qmax).ok && top > 0.f && top < INFINITY) {
                    by[q] = scale_of(top);
#pragma unroll
                    for (int i = 0; i < NV; ++i)
#pragma unroll
                        for (int j = 0; j < 8; ++j) f[q][i][j] *= by[q];
                }
            }
        }
        // code sums of the rows before: their warps' parts were written in front of this exchange
        if (quant && before >= 0 && warp == 0) flush(s_sum[turn ^ 1], before);
#pragma unroll
        for (int q = 0; q < R; ++q) {
            if (q >= live) break;
            const RowStats st(ssq[q], lo[q], hi[q], C, a.eps, qmax);
            float r = st.r, scale = st.alpha * st.r;
            if (!st.ok || by[q] != 1.f) {
                const double wide = scaled_factor(ssq[q], C, a.eps, by[q]);
                r = float(wide);
                scale = float(wide * double(st.alpha));
            }
            if (lo[q] == 0.f && hi[q] == 0.f) scale = 1.f; // Eq. 2's choice for a row of zeros
            if (y) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int g = t + i * T;
                    if (g < nvec) {
                        float o[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) o[j] = f[q][i][j] * gamma[i][j] * r;
                        Raw<XT>::store(y + (m0 + q) * C + 8 * g, o);
                    }
                }
            }
            if (quant) {
                const RowQuant rq(lo[q], hi[q], st.inv, st.zero, qmax);
                uint8_t* row = a.codes + (m0 + q) * (a.bits == 4 ? C / 2 : C);
                int sum = 0;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int g = t + i * T;
                    if (g < nvec) {
                        if (MAP) {
                            sum += store_codes8(v[q][i], rq, a.bits, row, g);
                        } else {
                            float u[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) u[j] = f[q][i][j] * gamma[i][j];
                            sum += store_codes8(u, rq, a.bits, row, g);
                        }
                    }
                }
                if (a.a_rowsum) {
                    sum = warp_sum_int(sum);
                    if (lane == 0) s_sum[turn][q][warp] = sum;
                }
                if (t == 0) {
                    a.a_scale[m0 + q] = scale;
                    a.a_zero[m0 + q] = st.zero;
                }
            }
        }
        before = m0;
        turn ^= 1;
    }
    if (quant && before >= 0) {
        __syncthreads();
        if (warp == 0) flush(s_sum[turn ^ 1], before);
    }
}

// Any channel count: a CTA per row, h in shared memory, the map through L2.  The same decisions as above.
template <typename XT>
__global__ void __launch_bounds__(512)
rmsnorm_quant_any(const NormArgs a) {
    extern __shared__ float s_u[];                         // h of the row
    __shared__ float red[64];
    const int t = threadIdx.x, T = blockDim.x, C = a.C;
    const XT* x = static_cast<const XT*>(a.x);
    const XT* res = static_cast<const XT*>(a.residual);
    const float qmax = float((1 << a.bits) - 1);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x) {
        float top = 0.f, by = 1.f, ssq, lo, hi;
        for (int k = t; k < C; k += T) {
            float f = float(x[m * C + k]);
            if (res) f += float(res[m * C + k]);
            s_u[k] = f;
            if (a.h) static_cast<XT*>(a.h)[m * C + k] = XT(f);
            top = fmaxf(top, fabsf(f));
        }
        __syncthreads();
        const auto value = [&](int c) {                    // u' of output channel c
            if (!a.ptr) return s_u[c] * by * a.gamma[c];
            const int b = a.ptr[c], e = a.ptr[c + 1];
            if (e - b == 1) return a.coef[b] * (s_u[a.src[b]] * by * a.gamma[a.src[b]]);
            double s = 0.0;
            for (int k = b; k < e; ++k) s = fma(double(a.coef[k]), double(s_u[a.src[k]] * by * a.gamma[a.src[k]]), s);
            return float(s);
        };
        for (int pass = 0;; ++pass) {
            ssq = 0.f;
            lo = INFINITY;
            hi = -INFINITY;
            for (int k = t; k < C; k += T) {
                const float f = s_u[k] * by, u = a.codes ? value(k) : f * a.gamma[k];
                ssq = fmaf(f, f, ssq);
                lo = fminf(lo, u);
                hi = fmaxf(hi, u);
            }
            ssq = block_sum(ssq, red);
            block_minmax(lo, hi, red);
            if (pass || RowStats(ssq, lo, hi, C, a.eps, qmax).ok) break;
            float none = 0.f;
            block_minmax(none, top, red);
            if (top > 0.f && top < INFINITY) by = scale_of(top);
        }
        const RowStats st(ssq, lo, hi, C, a.eps, qmax);
        float r = st.r, scale = st.alpha * st.r;
        if (!st.ok || by != 1.f) {
            const double wide = scaled_factor(ssq, C, a.eps, by);
            r = float(wide);
            scale = float(wide * double(st.alpha));
        }
        if (lo == 0.f && hi == 0.f) scale = 1.f;
        if (a.y)
            for (int k = t; k < C; k += T) static_cast<XT*>(a.y)[m * C + k] = XT(s_u[k] * by * a.gamma[k] * r);
        if (a.codes) {
            const RowQuant rq(lo, hi, st.inv, st.zero, qmax);
            int sum = 0;
            if (a.bits == 4) {
                for (int p = t; p < C / 2; p += T) {
                    const int q0 = rq.code(value(2 * p)), q1 = rq.code(value(2 * p + 1));
                    a.codes[m * (C / 2) + p] = uint8_t(q0 | q1 << 4);
                    sum += q0 + q1;
                }
            } else {
                for (int k = t; k < C; k += T) {
                    const int q = rq.code(value(k));
                    a.codes[m * C + k] = uint8_t(q);
                    sum += q;
                }
            }
            sum = block_sum_int(sum, reinterpret_cast<int*>(red));
            if (t == 0) {
                a.a_scale[m] = scale;
                a.a_zero[m] = st.zero;
                if (a.a_rowsum) a.a_rowsum[m] = sum;
            }
        }
        __syncthreads();                                   // h is overwritten by the next row's
    }
}

template <typename XT, int NV, int R, bool MAP, int MAXT>
int launch_norm_rows(const NormArgs& a, cudaStream_t st) {
    const int nvec = a.C / 8, T = ((nvec + NV - 1) / NV + 31) / 32 * 32;
    const int64_t grid = std::min((a.M + R - 1) / R, int64_t(device_sm_count()) * std::max(1, 1024 / T));
    QLLM_CUDA_TRY(launch_dependent(rmsnorm_quant_kernel<XT, NV, R, MAP, MAXT>, dim3(unsigned(grid)), dim3(unsigned(T)),
                                   MAP ? size_t(R) * a.C * 4 : 0, st, a));
    return after_launch();
}

template <typename XT>
int launch_norm(const NormArgs& a, cudaStream_t st) {
    const int64_t sms = device_sm_count();
    if (a.C % 8 == 0) {
        if (a.ptr) {
            if (a.C <= 4096) return a.M > 2 * sms ? launch_norm_rows<XT, 1, 2, true, 512>(a, st) : launch_norm_rows<XT, 1, 1, true, 512>(a, st);
            if (a.C <= 8192) return launch_norm_rows<XT, 2, 1, true, 512>(a, st);
        } else {
            if (a.C <= 8192 && a.M <= 2 * sms) return launch_norm_rows<XT, 1, 1, false, 1024>(a, st);
            if (a.C <= 8192) return launch_norm_rows<XT, 2, 1, false, 512>(a, st);
            if (a.C <= 16384) return launch_norm_rows<XT, 4, 1, false, 512>(a, st);
        }
    }
    const auto kern = rmsnorm_quant_any<XT>;
    if (a.C * 4 > 40 * 1024) QLLM_CUDA_TRY(allow_smem<rmsnorm_quant_any<XT>>(49152 * 4));
    QLLM_CUDA_TRY(launch_dependent(kern, dim3(unsigned(std::min<int64_t>(a.M, 4 * sms))), dim3(512), size_t(a.C) * 4, st, a));
    return after_launch();
}

// ---- the values that codes stand for -------------------------------------------------------------------------------------
// out = a_scale (code - a_zero), one rounding for the difference (none for codes of zero-points below 2^22), one for the product and
// one to the output's type.  16 codes a thread: 8 or 16 bytes in, 32 or 64 out; two rows of a CTA in flight.
template <typename T>
__global__ void __launch_bounds__(256)
dequantize_rows_kernel(const uint8_t* codes, const float* a_scale, const float* a_zero, int64_t M, int C, int bits, T* out) {
    const int nvec = C / 16, per = (nvec + blockDim.x - 1) / blockDim.x;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int64_t i = blockIdx.x; i < M * per; i += gridDim.x) {
        const int64_t m = i / per;
        const int g = int(i - m * per) * blockDim.x + threadIdx.x;
        if (g >= nvec) continue;
        uint32_t w[4];
        if (bits == 4) {
            const uint2 p = *reinterpret_cast<const uint2*>(codes + m * (C / 2) + 8 * g);
            w[0] = p.x; w[1] = p.y;
        } else {
            const uint4 p = *reinterpret_cast<const uint4*>(codes + m * C + 16 * g);
            w[0] = p.x; w[1] = p.y; w[2] = p.z; w[3] = p.w;
        }
        const float scale = a_scale[m], zero = a_zero[m];
        float f[2][8];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const uint32_t q = bits == 4 ? w[j >> 3] >> (4 * (j & 7)) & 15u : w[j >> 2] >> (8 * (j & 3)) & 255u;
            f[j >> 3][j & 7] = (float(q) - zero) * scale;
        }
        Raw<T>::store(out + m * C + 16 * g, f[0]);
        Raw<T>::store(out + m * C + 16 * g + 8, f[1]);
    }
}

template <typename T>
__global__ void __launch_bounds__(256)
dequantize_rows_any(const uint8_t* codes, const float* a_scale, const float* a_zero, int64_t M, int C, int bits, T* out) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int64_t m = blockIdx.x; m < M; m += gridDim.x)
        for (int k = threadIdx.x; k < C; k += blockDim.x) {
            const int q = bits == 4 ? codes[m * (C / 2) + k / 2] >> (k & 1 ? 4 : 0) & 15 : codes[m * C + k];
            out[m * C + k] = T((float(q) - a_zero[m]) * a_scale[m]);
        }
}

template <typename T>
int launch_dequantize(const uint8_t* codes, const float* a_scale, const float* a_zero, int64_t M, int C, int bits, void* out, cudaStream_t st) {
    const int64_t sms = device_sm_count();
    T* o = static_cast<T*>(out);
    if (C % 16 == 0) {
        const int nvec = C / 16, threads = std::min(256, (nvec + 31) / 32 * 32);
        const int64_t blocks = M * ((nvec + threads - 1) / threads);
        QLLM_CUDA_TRY(launch_dependent(dequantize_rows_kernel<T>, dim3(unsigned(std::min<int64_t>(blocks, 1 << 30))), dim3(unsigned(threads)), 0, st,
                                       codes, a_scale, a_zero, M, C, bits, o));
    } else {
        QLLM_CUDA_TRY(launch_dependent(dequantize_rows_any<T>, dim3(unsigned(std::min<int64_t>(M, 16 * sms))), dim3(256), 0, st, codes, a_scale, a_zero,
                                       M, C, bits, o));
    }
    return after_launch();
}

}  // namespace
}  // namespace qllm

extern "C" int qllm_rmsnorm_quant(const void* x, const void* residual, int x_dtype, int64_t M, int C, const float* gamma, float eps,
                                  const int32_t* map_ptr, const int32_t* map_src, const float* map_coef, int bits, void* h, void* y,
                                  uint8_t* codes, float* a_scale, float* a_zero, int32_t* a_rowsum, void* stream) {
    using namespace qllm;
    if (codes && !bits_ok(bits)) return QLLM_ERR_BITS;
    if (!dtype_ok(x_dtype)) return QLLM_ERR_DTYPE;
    if (M < 0 || C <= 0 || (codes && bits == 4 && (C & 1)) || !(eps >= 0.f) || eps > 3e38f) return QLLM_ERR_SHAPE;
    if (C > 49152) return QLLM_ERR_UNSUPPORTED;
    if (M == 0) return QLLM_OK;
    if (!x || !gamma || (!codes && !y && !h) || (codes && (!a_scale || !a_zero))) return QLLM_ERR_NULL;
    if ((map_ptr || map_src || map_coef) && (!map_ptr || !map_src || !map_coef || !codes)) return QLLM_ERR_NULL;
    if (!aligned16(x) || !aligned16(residual) || !aligned16(h) || !aligned16(y) || !aligned16(codes)) return QLLM_ERR_ALIGN;
    const NormArgs a{x, residual, M, C, gamma, eps, map_ptr, map_src, map_coef, codes ? bits : 8, h, y, codes, a_scale, a_zero, a_rowsum};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return x_dtype == QLLM_BF16 ? launch_norm<__nv_bfloat16>(a, st) : launch_norm<float>(a, st);
}

extern "C" int qllm_dequantize_rows(const uint8_t* codes, const float* a_scale, const float* a_zero, int64_t M, int C, int bits, void* out,
                                    int out_dtype, void* stream) {
    using namespace qllm;
    if (!bits_ok(bits)) return QLLM_ERR_BITS;
    if (!dtype_ok(out_dtype)) return QLLM_ERR_DTYPE;
    if (M < 0 || C <= 0 || (bits == 4 && (C & 1))) return QLLM_ERR_SHAPE;
    if (M == 0) return QLLM_OK;
    if (!codes || !a_scale || !a_zero || !out) return QLLM_ERR_NULL;
    if (!aligned16(codes) || !aligned16(out)) return QLLM_ERR_ALIGN;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return out_dtype == QLLM_BF16 ? launch_dequantize<__nv_bfloat16>(codes, a_scale, a_zero, M, C, bits, out, st)
                                  : launch_dequantize<float>(codes, a_scale, a_zero, M, C, bits, out, st);
}
