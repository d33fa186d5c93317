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
// What bounds it.  A row is read once and written once.  The CTAs stay and walk the rows (gamma stays in registers, the next rows are on their way
// into shared memory); the code sum of a row leaves with the next row's exchange.  2048 rows of 8192 in bf16 with residual, h, y and 8-bit codes:
// 31 us for 151 MB, 4.9 TB/s of a copy's 6.6; two thirds of the issue slots.  With the map, 6011 rows of 4096: 61.5 us for 172 MB, instructions: 35.6 M, half of the issue
// slots at 16 warps an SM; the exchange, the merged outputs and Eq. 2 cost a warp 300 to 390 of its 740 a row.  gamma from L1 instead of registers
// took 79 us there (L1 is what shared memory leaves), one vector a thread and 512 threads 72.  A few rows: one vector a thread, one row a CTA, 2.7 us for a
// row of 4096, 7.3 with a map of 8192 (reading it).
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>

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
    float inv_c, inv_levels;                               // 1 / C, 1 / (2^bits - 1)
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

// Eq. 2's parameters of u' and the row's factor.  ok = false: the row's numbers are too large or too small for float32 squares, or for
// the short ways here; `plain` takes the long ones.  x / (2^bits - 1) is the product with the reciprocal corrected by its exact residual (Markstein),
// correctly rounded for 15, 63 and 255 (checked for every mantissa).  The scale is 2^-100 at least, whose reciprocal and the products with it are finite.
struct RowStats {
    float alpha, inv, zero, r;
    bool ok;
    RowStats() = default;
    __device__ __forceinline__ RowStats(float ssq, float lo, float hi, const NormArgs& a, float qmax) {
        const float ms = fmaf(ssq, a.inv_c, a.eps), range = hi - lo, q = range * a.inv_levels;
        alpha = range > 0.f ? fmaf(fmaf(-qmax, q, range), a.inv_levels, q) : fabsf(lo);
        inv = __frcp_rn(alpha);
        zero = -rintf(lo * inv);
        asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(ms));
        r = fmaf(0.5f * r, fmaf(-ms * r, r, 1.f), r);      // two steps of float32 off at most before
        ok = ms < 0x1p100f && ms >= 0x1p-80f && alpha < 0x1p100f && alpha >= 0x1p-100f;
    }
    __device__ __forceinline__ void plain(float lo, float hi, float qmax) { eq2_params(lo, hi, qmax, alpha, inv, zero); }
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

// Shared memory of the kernel below: S rows as they arrive, each thread's pieces side by side; with a map u (8 words for each of the
// CTA's vector places), behind it the values of merged outputs, then two 16-byte records for each merged output (words of its first four
// entries, coefficients, where further entries begin and end) and the further entries as (word, coefficient).
constexpr int merged_cap(int places) { return places * 3 / 2; }             // of 8 * places outputs
constexpr int entry_cap(int places) { return 2 * places; }
constexpr int map_smem(int places) { return (8 * places + merged_cap(places)) * 4 + merged_cap(places) * 32 + entry_cap(places) * 8; }

// A thread's NV vectors of 8 channels: its own pieces of the next S - 1 rows are on their way into shared memory (asynchronous copies of
// 16 bytes that only the thread itself reads again: no barrier) while it works on the present one.
//
// MAP: a thread also owns 8 NV output channels.  u goes through shared memory at word (k % 8) P + k / 8 (P = NV MAXT places), where
// neighbouring threads' neighbouring channels lie side by side.  An output with one entry (all but the merged ones) is an address and a
// coefficient, held in registers for the whole launch.  Merged outputs are dealt out evenly: thread i sums the i-th one and leaves it behind
// u, from where its owner takes it like any other word.  What a map has beyond the room for these lists is summed by its owner from the
// caller's arrays.
template <typename XT, int NV, bool MAP, int MAXT, int MINB, int S>
__global__ void __launch_bounds__(MAXT, MINB)
rmsnorm_quant_kernel(const NormArgs a) {
    constexpr int VB = 8 * int(sizeof(XT)), VQ = VB / 16;  // bytes and 16-byte pieces of a vector
    constexpr int P = NV * MAXT;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ float s_red[2][3][32];
    __shared__ int s_sum[2][32], s_count[2];
    __shared__ float s_top[32];
    const int t = threadIdx.x, T = blockDim.x, lane = t & 31, warp = t >> 5, nw = T >> 5, C = a.C, nvec = C / 8;
    const XT* x = static_cast<const XT*>(a.x);
    const XT* res = static_cast<const XT*>(a.residual);
    const float qmax = float((1 << a.bits) - 1);
    const bool quant = a.codes != nullptr;
    const int stage = (res ? 2 : 1) * NV * T * VB;
    const int64_t step = gridDim.x;
    asm volatile("griddepcontrol.wait;" ::: "memory");     // launched as a dependent

    // piece q of vector i of x (or, n = 1, the residual) in a stage
    const auto piece = [&](int st, int n, int i, int q) { return smem + st * stage + (((n * NV + i) * VQ + q) * T + t) * 16; };
    const auto request = [&](int st, int64_t m) {
        if (m < a.M) {
            const uint8_t* px = reinterpret_cast<const uint8_t*>(x + m * C + 8 * t);
            const uint8_t* pr = reinterpret_cast<const uint8_t*>(res + m * C + 8 * t);
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (t + i * T < nvec) {
#pragma unroll
                    for (int q = 0; q < VQ; ++q) {
                        cp_async16(piece(st, 0, i, q), px + i * T * VB + 16 * q);
                        if (res) cp_async16(piece(st, 1, i, q), pr + i * T * VB + 16 * q);
                    }
                }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    const auto arrived = [&](int st, int n, int i, float (&f)[8]) {
        Raw<XT> r;
        if constexpr (VQ == 1) {
            r.v = *reinterpret_cast<const uint4*>(piece(st, n, i, 0));
        } else {
            r.a = *reinterpret_cast<const float4*>(piece(st, n, i, 0));
            r.b = *reinterpret_cast<const float4*>(piece(st, n, i, 1));
        }
        r.get(f);
    };
    // h of the thread's i-th vector, times a power of two
    const auto sum_at = [&](int st, int i, float by, float (&f)[8]) {
        arrived(st, 0, i, f);
        if (res) {
            float o[8];
            arrived(st, 1, i, o);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] += o[j];
        }
        if (by != 1.f) {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] *= by;
        }
    };
    int64_t m = blockIdx.x;
#pragma unroll
    for (int i = 0; i < (S > 1 ? S - 1 : 1); ++i) request(i, m + i * step);

    float gamma[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) gamma[i][j] = t + i * T < nvec ? __ldg(a.gamma + 8 * (t + i * T) + j) : 0.f;

    float* s_u = reinterpret_cast<float*>(smem + S * stage);
    uint4* s_first = reinterpret_cast<uint4*>(s_u + 8 * P + merged_cap(P));        // words 0 | 1 << 16, 2 | 3 << 16, coefficients 0, 1
    uint4* s_second = s_first + merged_cap(P);             // coefficients 2, 3, further entries
    uint2* s_entry = reinterpret_cast<uint2*>(s_second + merged_cap(P));
    const auto shared_at = [&](uint32_t bytes) { return *reinterpret_cast<const float*>(reinterpret_cast<const uint8_t*>(s_u) + bytes); };
    uint32_t addr[MAP ? NV : 1][8], walked[MAP ? NV : 1];
    float coef[MAP ? NV : 1][8];
    const auto word_of = [&](int k) { return (uint32_t(k) & 7u) * P + (uint32_t(k) >> 3); };
    const auto addr_of = [&](int k) { return 4u * word_of(k); };
    int merged = 0;
    if (MAP) {
        if (t < 2) s_count[t] = 0;
        __syncthreads();
        uint32_t several[NV];                              // outputs with several entries
        int rows = 0, entries = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int g = t + i * T;
            int from[9];
#pragma unroll
            for (int j = 0; j < 9; ++j) from[j] = g < nvec ? __ldg(a.ptr + 8 * g + j) : j;
            several[i] = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                addr[i][j] = g < nvec ? addr_of(__ldg(a.src + from[j])) : 0;
                coef[i][j] = g < nvec ? __ldg(a.coef + from[j]) : 0.f;
                const int n = from[j + 1] - from[j];
                if (n > 1) {
                    several[i] |= 1u << j;
                    ++rows;
                    entries += min(max(n - 4, 0), entry_cap(P) + 1);
                }
            }
            walked[i] = 0;
        }
        int slot = merged_cap(P), at = 0;
        if (rows) {
            slot = atomicAdd(s_count, rows);
            at = atomicAdd(s_count + 1, min(entries, entry_cap(P) + 1));
        }
        const bool room = slot + rows <= merged_cap(P) && at + entries <= entry_cap(P);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            walked[i] = room ? 0 : several[i];
            const uint32_t own = room ? several[i] : 0;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (own >> j & 1) {
                    addr[i][j] = 4u * uint32_t(8 * P + slot + __popc(own & ((1u << j) - 1)));
                    coef[i][j] = 1.f;
                }
#pragma unroll 1
            for (uint32_t left = own; left; left &= left - 1) {
                const int c = 8 * (t + i * T) + __ffs(left) - 1, b = __ldg(a.ptr + c), e = __ldg(a.ptr + c + 1);
                uint32_t w[4];
                float f[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {              // (a missing entry is the first one times 0)
                    const bool is = b + k < e;
                    w[k] = word_of(__ldg(a.src + (is ? b + k : b)));
                    f[k] = is ? __ldg(a.coef + b + k) : 0.f;
                }
                s_first[slot] = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, __float_as_uint(f[0]), __float_as_uint(f[1]));
                s_second[slot++] = make_uint4(__float_as_uint(f[2]), __float_as_uint(f[3]), at, at + max(e - b - 4, 0));
#pragma unroll 1
                for (int k = b + 4; k < e; ++k) s_entry[at++] = make_uint2(addr_of(__ldg(a.src + k)), __float_as_uint(__ldg(a.coef + k)));
            }
        }
        if (!room)
            for (int k = 0; k < rows; ++k)
                if (slot + k < merged_cap(P)) s_first[slot + k] = s_second[slot + k] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        merged = min(s_count[0], merged_cap(P));
    }
    const auto flush = [&](const int (&part)[32], int64_t row) {           // by the first warp
        const int s = warp_sum_int(lane < nw ? part[lane] : 0);
        if (lane == 0 && a.a_rowsum) a.a_rowsum[row] = s;
    };

    int parity = 0, turn = 0, st = 0;
    int64_t before = -1;                                   // the row whose code sums wait in s_sum[turn ^ 1]
    for (; m < a.M; m += step) {
        if (S > 1) request(st == 0 ? S - 1 : st - 1, m + (S - 1) * step);  // into what the last row was taken from
        asm volatile("cp.async.wait_group %0;" ::"n"(S - 1) : "memory");
        float f[MAP ? 1 : NV][8], v[MAP ? NV : 1][8], by = 1.f;
        float ssq, lo, hi;
        RowStats rs;
        for (int pass = 0;; ++pass) {
            ssq = 0.f;
            lo = INFINITY;
            hi = -INFINITY;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int g = t + i * T;
                float (&e)[8] = f[MAP ? 0 : i];
                if (g < nvec) {
                    sum_at(st, i, by, e);
                    if (a.h && pass == 0) Raw<XT>::store(static_cast<XT*>(a.h) + m * C + 8 * g, e);
#pragma unroll
                    for (int j = 0; j < 8; ++j) ssq = fmaf(e[j], e[j], ssq);
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        const float u0 = e[j] * gamma[i][j], u1 = e[j + 1] * gamma[i][j + 1];
                        if (MAP) {
                            s_u[j * P + g] = u0;
                            s_u[(j + 1) * P + g] = u1;
                        } else {
                            lo = min3(lo, u0, u1);
                            hi = max3(hi, u0, u1);
                        }
                    }
                }
            }
            if (MAP) {
                uint4 one = make_uint4(0, 0, 0, 0), two = one;             // the thread's first record, in front of the barrier
                if (t < merged) { one = s_first[t]; two = s_second[t]; }
                __syncthreads();
                for (int i = t; i < merged; i += T) {
                    const float u0 = shared_at(4u * (one.x & 0xFFFFu)), u1 = shared_at(4u * (one.x >> 16));
                    const float u2 = shared_at(4u * (one.y & 0xFFFFu)), u3 = shared_at(4u * (one.y >> 16));
                    double s = fma(double(__uint_as_float(one.w)), double(u1), double(__uint_as_float(one.z)) * double(u0));
                    if (two.x) s = fma(double(__uint_as_float(two.x)), double(u2), s);
                    if (two.y) s = fma(double(__uint_as_float(two.y)), double(u3), s);
                    for (uint32_t k = two.z; k < two.w; ++k) {
                        const uint2 e = s_entry[k];
                        s = fma(double(__uint_as_float(e.y)), double(shared_at(e.x)), s);
                    }
                    s_u[8 * P + i] = float(s);
                    if (i + T < merged) { one = s_first[i + T]; two = s_second[i + T]; }
                }
                __syncthreads();
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int g = t + i * T;
                    if (g < nvec) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[i][j] = coef[i][j] * shared_at(addr[i][j]);
                        if (walked[i]) {
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                if (walked[i] >> j & 1) {
                                    const int e = a.ptr[8 * g + j + 1];
                                    double s = 0.0;
#pragma unroll 1
                                    for (int k = a.ptr[8 * g + j]; k < e; ++k) s = fma(double(a.coef[k]), double(shared_at(addr_of(a.src[k]))), s);
                                    v[i][j] = float(s);
                                }
                        }
#pragma unroll
                        for (int j = 0; j < 8; j += 2) {
                            lo = min3(lo, v[i][j], v[i][j + 1]);
                            hi = max3(hi, v[i][j], v[i][j + 1]);
                        }
                    }
                }
            }
            parity ^= 1;
            const float s = warp_sum(ssq), l = redux_min(lo), u = redux_max(hi);
            if (lane == 0) {
                s_red[parity][0][warp] = s;
                s_red[parity][1][warp] = l;
                s_red[parity][2][warp] = u;
            }
            __syncthreads();
            ssq = warp_sum(lane < nw ? s_red[parity][0][lane] : 0.f);
            lo = redux_min(lane < nw ? s_red[parity][1][lane] : INFINITY);
            hi = redux_max(lane < nw ? s_red[parity][2][lane] : -INFINITY);
            rs = RowStats(ssq, lo, hi, a, qmax);
            if (pass || rs.ok) break;                      // the same in every thread
            // a row with very large or very small numbers: all of it by a power of two, exactly, and once more
            float top = 0.f;
#pragma unroll 1
            for (int i = 0; i < NV; ++i)
                if (t + i * T < nvec) {
                    float e[8];
                    sum_at(st, i, 1.f, e);
#pragma unroll
                    for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(e[j]));
                }
            top = redux_max(top);
            if (lane == 0) s_top[warp] = top;
            __syncthreads();
            top = redux_max(lane < nw ? s_top[lane] : 0.f);
            if (top > 0.f && top < INFINITY) by = scale_of(top);
        }
        // the code sum of the row before: its warps' parts were written in front of this exchange
        if (quant && before >= 0 && warp == 0) flush(s_sum[turn ^ 1], before);
        float r = rs.r, scale = rs.alpha * rs.r;
        if (!rs.ok || by != 1.f) {
            if (!rs.ok) rs.plain(lo, hi, qmax);
            double wide = scaled_factor(ssq, C, a.eps, by);
            r = float(wide);
            // a row of zeros, which is never ok: Eq. 2's alpha of 1 itself (lo and hi know no NaN, ssq does)
            if (lo == 0.f && hi == 0.f && ssq < INFINITY) wide = 1.0;
            scale = float(wide * double(rs.alpha));
        }
        const RowQuant rq(lo, hi, rs.inv, rs.zero, qmax);
        uint8_t* row = a.codes + m * (a.bits == 4 ? C / 2 : C);
        int sum = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int g = t + i * T;
            if (g < nvec) {
                if (!MAP || a.y) {
                    float e[8];
                    if constexpr (MAP) {
                        sum_at(st, i, by, e);
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) e[j] = f[i][j];
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) e[j] *= gamma[i][j];
                    if (!MAP && quant) sum += store_codes8(e, rq, a.bits, row, g);
                    if (a.y) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) e[j] *= r;
                        Raw<XT>::store(static_cast<XT*>(a.y) + m * C + 8 * g, e);
                    }
                }
                if (MAP) sum += store_codes8(v[i], rq, a.bits, row, g);
            }
        }
        if (quant) {
            sum = warp_sum_int(sum);
            if (lane == 0) s_sum[turn][warp] = sum;
            if (t == 0) {
                a.a_scale[m] = scale;
                a.a_zero[m] = rs.zero;
            }
        }
        before = m;
        turn ^= 1;
        st = st + 1 == S ? 0 : st + 1;
        if (S == 1) request(0, m + step);
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
            if (pass || RowStats(ssq, lo, hi, a, qmax).ok) break;
            float none = 0.f;
            block_minmax(none, top, red);
            if (top > 0.f && top < INFINITY) by = scale_of(top);
        }
        RowStats st(ssq, lo, hi, a, qmax);
        float r = st.r, scale = st.alpha * st.r;
        if (!st.ok || by != 1.f) {
            if (!st.ok) st.plain(lo, hi, qmax);
            double wide = scaled_factor(ssq, C, a.eps, by);
            r = float(wide);
            if (lo == 0.f && hi == 0.f && ssq < INFINITY) wide = 1.0;
            scale = float(wide * double(st.alpha));
        }
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

template <typename XT, int NV, bool MAP, int MAXT, int MINB, int S>
int launch_norm_rows(const NormArgs& a, cudaStream_t st) {
    constexpr auto kern = rmsnorm_quant_kernel<XT, NV, MAP, MAXT, MINB, S>;
    const int nvec = a.C / 8, T = ((nvec + NV - 1) / NV + 31) / 32 * 32;
    const int smem = S * (a.residual ? 2 : 1) * NV * T * 8 * int(sizeof(XT)) + (MAP ? map_smem(NV * MAXT) : 0);
    QLLM_CUDA_TRY(allow_smem<kern>(kSmemBudget - 2048));
    static std::atomic<int> known{0};
    int regs = known.load(std::memory_order_relaxed);
    if (!regs) {
        cudaFuncAttributes fa;
        QLLM_CUDA_TRY(cudaFuncGetAttributes(&fa, kern));
        known.store(regs = (fa.numRegs + 7) / 8 * 8, std::memory_order_relaxed);
    }
    // the CTAs that an SM holds at once: they stay and walk the rows
    const int per_sm = std::max(1, std::min({32, 2048 / T, 65536 / (regs * T), kSmemBudget / (smem + 2048)}));
    const int64_t grid = std::min(a.M, int64_t(device_sm_count()) * per_sm);
    QLLM_CUDA_TRY(launch_dependent(kern, dim3(unsigned(grid)), dim3(unsigned(T)), size_t(smem), st, a));
    return after_launch();
}

template <typename XT>
int launch_norm(const NormArgs& a, cudaStream_t st) {
    const int64_t sms = device_sm_count();
    if (a.C % 8 == 0) {
        constexpr bool half = sizeof(XT) == 2;
        if (a.ptr) {
            if (a.C <= 8192 && a.M <= 2 * sms) return launch_norm_rows<XT, 1, true, 1024, 1, 1>(a, st);
            if (a.C <= 4096) return launch_norm_rows<XT, 2, true, 256, 2, 3>(a, st);
            if (a.C <= 8192) return launch_norm_rows<XT, 2, true, 512, 1, half ? 2 : 1>(a, st);
        } else {
            if (a.C <= 8192 && a.M <= 2 * sms) return launch_norm_rows<XT, 1, false, 1024, 1, 1>(a, st);
            if (a.C <= 8192) return launch_norm_rows<XT, 2, false, 512, 2, 3>(a, st);
            if (a.C <= 16384) return launch_norm_rows<XT, 4, false, 512, 1, half ? 3 : 1>(a, st);
        }
    }
    const auto kern = rmsnorm_quant_any<XT>;
    if (a.C * 4 > 40 * 1024) QLLM_CUDA_TRY(allow_smem<rmsnorm_quant_any<XT>>(49152 * 4));
    QLLM_CUDA_TRY(launch_dependent(kern, dim3(unsigned(std::min<int64_t>(a.M, 4 * sms))), dim3(512), size_t(a.C) * 4, st, a));
    return after_launch();
}

// ---- the values that codes stand for -------------------------------------------------------------------------------------
// out = a_scale (code - a_zero), one rounding for the difference (none for codes of zero-points below 2^22), one for the product and
// one to the output's type.  16 codes a thread: 8 or 16 bytes in, 32 or 64 out.  2048 rows of 8192 in 8 bits to bf16: 10.4 us, 4.8 TB/s.
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
    const int b = codes ? bits : 8;
    const NormArgs a{x, residual, M, C, gamma, eps, map_ptr, map_src, map_coef, b, h, y, codes, a_scale, a_zero, a_rowsum, 1.f / float(C), 1.f / float((1 << b) - 1)};
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
