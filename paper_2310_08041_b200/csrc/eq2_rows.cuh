// Eq. 2 on a row whose range is known: parameters and codes, as the one-pass kernels of qllm_quantize_rows and
// qllm_rmsnorm_quant make them.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "reassemble_quant_common.cuh"

namespace qllm {

// Eq. 2 from the row's range: alpha, 1 / alpha, zero-point (a constant row takes alpha = |value|, 1 if it is 0)
__device__ __forceinline__ void eq2_params(float lo, float hi, float qmax, float& alpha, float& inv, float& zero) {
    alpha = (hi - lo) / qmax;
    if (!(hi > lo)) alpha = lo != 0.f ? fabsf(lo) : 1.f;
    inv = __frcp_rn(alpha);
    zero = -rintf(lo * inv);
}

// How a row's codes are made from its Eq. 2 parameters.  round(f / alpha) + zero is taken as the low bits of
// fma(f, 1 / alpha, 1.5 * 2^23) plus an integer constant (one rounding, to nearest even, no conversion
// instruction: those run at a sixteenth of the arithmetic rate and would bound the kernel); quotients or
// zero-points too large for that constant take the plain form.
struct RowQuant {
    float inv, zero, qmax;
    int zadd, top;
    bool big;
    __device__ __forceinline__ RowQuant(float lo, float hi, float inv_, float zero_, float qmax_)
        : inv(inv_), zero(zero_), qmax(qmax_), zadd(int(zero_) - kMagicBits), top(int(qmax_)),
          big(fmaxf(fabsf(lo), fabsf(hi)) * inv_ >= 2097152.f || fabsf(zero_) >= 2097152.f) {}
    // the code of one value
    __device__ __forceinline__ int code(float f) const {
        if (!big) return min(max(__float_as_int(fmaf(f, inv, kMagic)) + zadd, 0), top);
        return int(fminf(fmaxf(rintf(f * inv) + zero, 0.f), qmax));
    }
};

// 8 codes of consecutive channels -> stored (4 bit: one 32-bit word, else two); returns their sum
__device__ __forceinline__ int store_codes8(const float (&f)[8], const RowQuant& q, int bits, uint8_t* out_row, int g) {
    int n[8];
    if (!q.big) {
#pragma unroll
        for (int j = 0; j < 8; ++j) n[j] = __float_as_int(fmaf(f[j], q.inv, kMagic)) + q.zadd;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) n[j] = int(fminf(fmaxf(rintf(f[j] * q.inv) + q.zero, 0.f), q.qmax));
    }
    if (bits == 4) {
        uint32_t p = 0;                                    // saturating packs clamp to 0 .. 15
#pragma unroll
        for (int k = 3; k >= 0; --k) p = pack_sat_u4(n[2 * k + 1], n[2 * k], p);
        reinterpret_cast<uint32_t*>(out_row)[g] = p;
        const uint32_t nib = (p & 0x0F0F0F0Fu) + ((p >> 4) & 0x0F0F0F0Fu);
        return int(__dp4a(nib, 0x01010101u, 0u));
    }
    // saturating packs clamp to 0 .. 255; 6-bit codes are cut at 63 first
    if (bits == 6) {
#pragma unroll
        for (int j = 0; j < 8; ++j) n[j] = min(n[j], q.top);
    }
    const uint32_t p0 = pack_sat_u8(n[1], n[0], pack_sat_u8(n[3], n[2], 0u)), p1 = pack_sat_u8(n[5], n[4], pack_sat_u8(n[7], n[6], 0u));
    reinterpret_cast<uint2*>(out_row)[g] = make_uint2(p0, p1);
    return int(__dp4a(p1, 0x01010101u, __dp4a(p0, 0x01010101u, 0u)));
}

}  // namespace qllm
