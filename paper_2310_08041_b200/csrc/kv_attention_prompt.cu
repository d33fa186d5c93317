// Attention over the 4-bit cache for many query rows per key head (prompts, chunks of prompts): tcgen05 tensor cores.
//
// A CTA owns 256 query rows of one key head (query tokens x the heads of the group, two tiles of 128) and walks the keys in
// tiles of 128 tokens.  Both products run as 128 x 128 tcgen05 MMAs in fp16: S_t = Q_t K^T into tensor memory, softmax by two
// threads per row (64 columns each), P_t back into tensor memory over S_t, O_t += P_t V.  While one tile's rows are in the
// softmax, the tensor core works for the other.  The tensor pipe's 4 * 256 * 128 * head_dim operations a step and the softmax's
// issue slots are about equal; each key tile is unpacked once for 256 rows.
//
// Roles (24 warps): 0-7 and 8-15 the softmax of tiles 0 and 1, 16-19 unpack codes (a thread per token), 20 fetches codes and
// parameters with bulk copies, 21 issues the MMAs, 22 turns a tile's parameters into what the others need.  Registers are
// shifted to the softmax warps.
//
// Operands.  A nibble under the exponent of 1024 is the fp16 number 1024 + c (1024 + 16 c from the upper half of a byte), one
// packed fp16 operation makes it the exact integer c - zero, another the operand (c - zero) scale 2^-E, E the exponent of the
// tile's largest key or value: rounded to fp16 in the scale and in the product, 11 bits each, where keys and values of 16 bits
// would carry 8.  So nothing acts per score and token: a score's factor is the row's times 2^E, a weight is p 2^E.  Queries are
// scaled per row by a power of two into fp16 (a bf16 query's 8 bits are kept); the scale's mantissa goes to the
// keys (split_scale).  Tiles whose value scales differ by more than
// 2^10, or pass 2^80, keep the values' bare codes and multiply the weights by vs instead, since a weight of a small value must
// not lose its bits to a large value that the row hardly looks at.  So do tiles in which some scale 2^-E is no normal fp16 number (values
// far from zero have scales far below them): a key or value must not lose its bits to a louder one that the row does not see, or turns
// away from.  There each key's own power of two acts on its score.  Rows far from zero (|zero| > 900) are made in float32.
// Channels lie in the order 0 4 1 5 2 6 3 7 of each eight, as the masks leave them: the queries are stored alike and the output
// is put right at the end.

// Measured: a prompt of 2048 tokens, 32 heads of 128, causal: 66 us, 0.52 PFLOP/s; 1024 and 17 new tokens behind up to 8191, 64 query
// on 8 key heads: 320 us, 0.81 PFLOP/s = 0.49 of the measured cuBLAS bf16 rate.  A step of two tiles takes about 5300 cycles where
// its MMAs need 2048 and its exponentials as many: what is left is the chain through one tile (maximum, exchange, weights,
// store, product, next scores), which two tiles in flight do not fill.  Tried and dropped, besides what stands at the functions
// below: waiting warps asleep in their barriers or polling in four instructions (both 2 % slower).

#include <cuda_fp16.h>

#include <algorithm>

#include "kv_attention.h"
#include "ptx_sm100.cuh"
#include "qgemm_tc_common.cuh"

namespace qllm {
namespace {

using namespace kv;
using tc::Abort;
using tc::wait_bounded;

constexpr int BM = 128, BN = 128;                          // query rows of a tile, tokens of a key tile
constexpr int kThreads = 768;
constexpr int kSlots = 4;                                  // key tiles whose parameters are held
constexpr float kPlace = 6.f, kSlack = 8.f;                // as in kv_attention_split.cu

template <int D>
struct Shape {
    static constexpr int ATOM = BN * 128;                  // 128 rows of 64 fp16 in the 128-byte swizzle
    static constexpr int OP = D / 64 * ATOM;               // one operand tile
    static constexpr int OPS = 4;                          // operand buffers: keys 0 and 2, values 1 and 3
    static constexpr int RAW = BN * (D / 2);               // codes as they come
    static constexpr int RAWS = 3;
    static constexpr int RAWP = 2 * BN * 8;                // both parameter arrays, fetched with the keys: two of them
    static constexpr int PRM = BN * 6;                     // per token: a value scale, the upper half of a power of two
    static constexpr int SMEM = 1024 + 2 * OP + OPS * OP + RAWS * RAW + 2 * RAWP + kSlots * PRM;
    static constexpr uint32_t TMEM_S = 0, TMEM_O = 256;    // columns: S_0, S_1, O_0, O_1
};

// ---- instructions ---------------------------------------------------------------------------------------------------------
// kind::f16: fp16 x fp16, fp32 accumulate; A K-major, B K-major or (b_mn) N-major
__host__ __device__ constexpr uint32_t idesc_f16(int m, int n, bool b_mn) {
    return (1u << 4) | (0u << 7) | (0u << 10) | (uint32_t(b_mn) << 16) | (uint32_t(n >> 3) << 17) | (uint32_t(m >> 4) << 24);
}
// Shared-memory operands are given by the low words of their descriptors (the high word is the same for all): a step along an
// operand is one addition, and the issuing warp, whose every instruction waits for its turn among 15 others, is not what the
// tensor core waits for.
constexpr uint32_t kDescHigh = uint32_t((uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61) >> 32);
__device__ __forceinline__ void mma_f16_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 x, {%1, %5};\n\tmov.b64 y, {%2, %5};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "n"(kDescHigh)
                 : "memory");
}
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 y;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 y, {%2, %5};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "n"(kDescHigh)
                 : "memory");
}
__device__ __forceinline__ uint32_t elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r;
}
// Low word of a descriptor in the 128-byte swizzle: address, and (N-major operands: rows of 64 elements along K, groups of 8 rows
// 1024 bytes apart) the distance between blocks of 64 N-elements.
__device__ __forceinline__ uint32_t desc_low(uint32_t addr, uint32_t block) { return (addr & 0x3FFFFu) >> 4 | (block >> 4) << 16; }
__device__ __forceinline__ void tmem_st_x32(uint32_t addr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
        "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_st_x16(uint32_t addr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
// two floats at a time
struct F2 {
    uint64_t v;
    __device__ __forceinline__ F2() {}
    __device__ __forceinline__ F2(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ __forceinline__ F2(uint32_t a, uint32_t b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(a), "r"(b)); }
    __device__ __forceinline__ void get(float& a, float& b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
};
__device__ __forceinline__ F2 add2(F2 a, F2 b) { F2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) { F2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return r; }
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float lg2(float x) {
    float r;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float pow2i(int e) { return __int_as_float((e + 127) << 23); }     // -126 <= e <= 127
__device__ __forceinline__ uint32_t bits(__half2 h) { return *reinterpret_cast<const uint32_t*>(&h); }
__device__ __forceinline__ __half2 halves(uint32_t v) { return *reinterpret_cast<const __half2*>(&v); }
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(ptx::smem_addr(dst)),
                 "l"(src), "r"(bytes), "r"(ptx::smem_addr(bar))
                 : "memory");
}

// Shared memory by 32-bit address: what is reached through pointers handed to functions would be generic accesses.
__device__ __forceinline__ uint32_t lds1(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ uint4 lds4u(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}
__device__ __forceinline__ void sts4(uint32_t a, uint4 v) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// ---- work -----------------------------------------------------------------------------------------------------------------
struct Args {
    Cache c;
    Batch b;
    const __nv_bfloat16* q;
    __nv_bfloat16* out;
    float* lse;                                            // may be null
    int64_t q_stride, out_stride;
    int group, q_heads, causal, most_rows, splits;         // sequences with at most most_rows query rows are another kernel's
    float scale;
    float* part_o;                                         // [splits][rows][q_heads][D], unnormalised
    float2* part_ml;                                       // [splits][rows][q_heads]: reference exponent, sum
    int* status;
};

// 256-row blocks of a sequence
__device__ __forceinline__ unsigned blocks_of(const Args& a, int s) {
    const unsigned rows = unsigned(a.b.count(s)) * unsigned(a.group);
    return rows <= unsigned(a.most_rows) ? 0 : (rows + 2 * BM - 1) / (2 * BM);
}

// One word of codes -> 8 fp16 of (code - zero) mul.
__device__ __forceinline__ uint4 unpack8(uint32_t w, __half2 sub, __half2 sub16, __half2 mul) {
    const uint32_t u = w >> 8;
    const __half2 sixteenth = __floats2half2_rn(0.0625f, 0.0625f);
    const __half2 h0 = __hadd2(halves((w & 0x000F000Fu) | 0x64006400u), sub), h1 = __hfma2(halves((w & 0x00F000F0u) | 0x64006400u), sixteenth, sub16);
    const __half2 h2 = __hadd2(halves((u & 0x000F000Fu) | 0x64006400u), sub), h3 = __hfma2(halves((u & 0x00F000F0u) | 0x64006400u), sixteenth, sub16);
    return make_uint4(bits(__hmul2(h0, mul)), bits(__hmul2(h1, mul)), bits(__hmul2(h2, mul)), bits(__hmul2(h3, mul)));
}
// the same for any zero: (code - zero) factor in float32, rounded once
__device__ __forceinline__ uint4 unpack8_far(uint32_t w, float zero, float factor) {
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        h[i] = bits(__floats2half2_rn((float((w >> (4 * i)) & 15u) - zero) * factor, (float((w >> (4 * i + 16)) & 15u) - zero) * factor));
    return make_uint4(h[0], h[1], h[2], h[3]);
}

// Zero-points for which 1024 + zero, or code - zero, is no exact fp16 integer.
__device__ __forceinline__ bool is_far(float zero) { return fabsf(zero) > 900.f || zero != rintf(zero); }

// A thread's token: 64 / 32 bytes of codes -> its row of an operand tile (shared addresses).
template <int D>
__device__ __forceinline__ void unpack_row(uint32_t raw, uint32_t op, int tok, float zero, float factor, bool far) {
    constexpr int CH = D / 32;                             // 16-byte chunks of a row
    const uint32_t src = raw + tok * (D / 2), dst = op + tok * 128;
    auto unit = [&](int u) { return dst + (u >> 3) * Shape<D>::ATOM + (((u & 7) ^ (tok & 7)) << 4); };      // 8 channels
    if (far) {
#pragma unroll 1
        for (int u = 0; u < D / 8; ++u) sts4(unit(u), unpack8_far(lds1(src + 4 * u), zero, factor));
        return;
    }
    const __half2 sub = __float2half2_rn(-(1024.f + zero)), sub16 = __float2half2_rn(-(64.f + zero)), mul = __float2half2_rn(factor);
#pragma unroll 1
    for (int i = 0; i < CH; ++i) {
        const int ch = (i + (CH == 4 ? tok >> 1 : tok >> 2)) & (CH - 1);     // neighbours read different banks
        const uint4 w = lds4u(src + 16 * ch);
        sts4(unit(4 * ch), unpack8(w.x, sub, sub16, mul));
        sts4(unit(4 * ch + 1), unpack8(w.y, sub, sub16, mul));
        sts4(unit(4 * ch + 2), unpack8(w.z, sub, sub16, mul));
        sts4(unit(4 * ch + 3), unpack8(w.w, sub, sub16, mul));
    }
}

// Half a row's scores as they lie in tensor memory (64 columns from `addr`) become its weights in their place (16 columns for
// 32: a chunk overwrites what has been read).  vs, kx, there: shared addresses of the half's value scales, of its keys' powers of two
// and of the bits of the tokens that exist.  MASKED: some token of the tile is hidden from some row; BARE: the scores take the keys'
// powers of two, the weights the value scales.
//
// Two passes over tensor memory, maximum and weights, of 32 columns at a time.  Holding the half row in registers between them
// spills; with one thread per row, where it did not, the code of all roles together outran the instruction cache (chunks of 1024
// tokens behind up to 8191, 64/8 heads: 453 us instead of 417), as unrolled unpacking does.  Taking every second, third or
// fourth exponential by a polynomial, off the special-function unit, gained nothing (357, 341, 343 us against 330).
constexpr int kCols = 64;
template <bool MASKED>
__device__ __forceinline__ void hide(uint32_t (&r)[32], int first, int limit, uint32_t there) {
    if (!MASKED) return;
    const int n = limit - first;                           // tokens of the 32 in front of the limit
    const uint32_t seen = lds1(there) & (n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1);
#pragma unroll
    for (int k = 0; k < 32; ++k) r[k] = seen >> k & 1 ? r[k] : 0xFF800000u;
}
// (in front of the masks: a hidden key's power of two would turn their infinity into NaN if it were no number)
template <bool BARE>
__device__ __forceinline__ void scale_keys(uint32_t (&r)[32], uint32_t kx) {
    if (!BARE) return;
#pragma unroll
    for (int k = 0; k < 32; k += 2) {
        const uint32_t x = lds1(kx + 2 * k);
        r[k] = __float_as_uint(__uint_as_float(r[k]) * __uint_as_float(x << 16));
        r[k + 1] = __float_as_uint(__uint_as_float(r[k + 1]) * __uint_as_float(x & 0xFFFF0000u));
    }
}
__device__ __forceinline__ float log_scale(uint32_t v) { return fminf(fmaxf(lg2(fabsf(__uint_as_float(v))), -80.f), 80.f); }
template <bool MASKED, bool BARE>
__device__ __forceinline__ float half_max(uint32_t addr, uint32_t vs, uint32_t kx, int first, int limit, uint32_t there, float qn) {
    float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int c = 0; c < kCols / 32; ++c) {
        uint32_t r[32];
        ptx::tmem_ld_32x32b_x32(addr + 32 * c, r);
        ptx::tmem_ld_wait();
        scale_keys<BARE>(r, kx + 64 * c);
        hide<MASKED>(r, first + 32 * c, limit, there + 4 * c);
#pragma unroll
        for (int k = 0; k < 32; k += 2) {
            float a = __uint_as_float(r[k]), b = __uint_as_float(r[k + 1]);
            if (BARE) {                                    // s_j + log2 vs_j, cut to +-80
                a = fmaf(a, qn, log_scale(lds1(vs + 128 * c + 4 * k)));
                b = fmaf(b, qn, log_scale(lds1(vs + 128 * c + 4 * k + 4)));
            }
            m[k >> 1 & 3] = fmaxf(m[k >> 1 & 3], fmaxf(a, b));
        }
    }
    return fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
}
template <bool MASKED, bool BARE>
__device__ __forceinline__ float half_weights(uint32_t addr, uint32_t vs, uint32_t kx, int first, int limit, uint32_t there, float qn, float sub) {
    const F2 q2(qn, qn), s2(sub, sub);
    F2 l[4] = {F2(0.f, 0.f), F2(0.f, 0.f), F2(0.f, 0.f), F2(0.f, 0.f)};
#pragma unroll
    for (int c = 0; c < kCols / 32; ++c) {
        uint32_t r[32], p[16];
        ptx::tmem_ld_32x32b_x32(addr + 32 * c, r);
        ptx::tmem_ld_wait();
        scale_keys<BARE>(r, kx + 64 * c);
        hide<MASKED>(r, first + 32 * c, limit, there + 4 * c);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            float a, b;
            fma2(F2(r[2 * k], r[2 * k + 1]), q2, s2).get(a, b);
            a = ex2(a);
            b = ex2(b);
            l[k & 3] = add2(l[k & 3], F2(a, b));
            if (BARE) {                                    // (a hidden key's value scale may be anything)
                a = a == 0.f ? 0.f : a * __uint_as_float(lds1(vs + 128 * c + 8 * k));
                b = b == 0.f ? 0.f : b * __uint_as_float(lds1(vs + 128 * c + 8 * k + 4));
            }
            p[k] = bits(__floats2half2_rn(a, b));
        }
        tmem_st_x16(addr + 16 * c, p);
    }
    float a, b;
    add2(add2(l[0], l[1]), add2(l[2], l[3])).get(a, b);
    return a + b;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) kv_prompt_kernel(const Args a) {
    using S = Shape<D>;
    extern __shared__ uint8_t smem_dyn[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~uintptr_t(1023));
    uint8_t* s_q = smem;                                   // [2] tiles
    uint8_t* s_op = s_q + 2 * S::OP;                       // [OPS]
    uint8_t* s_raw = s_op + S::OPS * S::OP;                // [RAWS]
    uint8_t* s_rawp = s_raw + S::RAWS * S::RAW;            // [2] (a third tile's keys wait for the first one's values to be unpacked)
    float* s_vs = reinterpret_cast<float*>(s_rawp + 2 * S::RAWP);            // [kSlots][BN] value scales, for tiles of bare codes
    uint16_t* s_kx = reinterpret_cast<uint16_t*>(s_vs + kSlots * BN);        // [kSlots][BN] powers of two (upper halves of floats), likewise
    __shared__ uint64_t s_bar[32];
    __shared__ uint32_t s_tmem, s_pieces[S::RAWS];
    __shared__ int s_abort, s_find[2];
    __shared__ float s_ek[kSlots], s_e[kSlots];            // 2^exponent of a tile's keys, exponent of its values
    __shared__ float s_half[2][2][BM];                     // what the two threads of a row tell each other
    __shared__ uint32_t s_flags[kSlots], s_there[kSlots][4];                 // 1: bare codes, 2: some tokens are not there (bits)
    uint64_t* raw_full = s_bar;                            // [RAWS]
    uint64_t* raw_empty = raw_full + S::RAWS;              // [RAWS]
    uint64_t* op_full = raw_empty + S::RAWS;               // [OPS]
    uint64_t* op_empty = op_full + S::OPS;                 // [OPS]
    uint64_t* prm_full = op_empty + S::OPS;                // [kSlots]
    uint64_t* s_full = prm_full + kSlots;                  // [2]
    uint64_t* p_full = s_full + 2;                         // [2]
    uint64_t* o_full = p_full + 2;                         // [2]
    uint64_t* q_full = o_full + 2;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int i = 0; i < S::RAWS; ++i) { ptx::mbar_init(&raw_full[i], 1); ptx::mbar_init(&raw_empty[i], 4); }
        for (int i = 0; i < S::OPS; ++i) { ptx::mbar_init(&op_full[i], 4); ptx::mbar_init(&op_empty[i], 1); }
        for (int i = 0; i < kSlots; ++i) ptx::mbar_init(&prm_full[i], 1);
        for (int i = 0; i < 2; ++i) { ptx::mbar_init(&s_full[i], 1); ptx::mbar_init(&p_full[i], 8); ptx::mbar_init(&o_full[i], 1); }
        ptx::mbar_init(q_full, 16);
        s_abort = 0;
        ptx::fence_barrier_init();
        ptx::fence_proxy_async_smem();
    }
    if (warp == 1 && blockIdx.x == 0 && blockIdx.y == 0) a.b.report(a.status, lane, 32);
    if (warp == 0) {                                       // which sequence, which block of it
        unsigned x = blockIdx.x / a.c.heads;               // heads vary fastest: all of them start with their longest blocks
        int found = -1;
        for (int base = 0; base < a.b.seqs; base += 32) {
            const int s = base + lane;
            const unsigned n = s < a.b.seqs ? blocks_of(a, s) : 0;
            unsigned incl = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const unsigned y = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += y;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, x < incl);
            if (hit) {
                const int l = __ffs(hit) - 1;
                const unsigned cnt = __shfl_sync(0xffffffffu, n, l), end = __shfl_sync(0xffffffffu, incl, l);
                found = base + l;
                x = cnt - 1 - (x - (end - cnt));           // the last block, which sees the most keys, first
                break;
            }
            x -= __shfl_sync(0xffffffffu, incl, 31);
        }
        if (lane == 0) { s_find[0] = found; s_find[1] = int(x); }
    }
    __syncthreads();
    const int seq = s_find[0];
    if (seq < 0) return;
    const int blk = s_find[1], g = blockIdx.x % a.c.heads, n = a.b.count(seq), len = a.b.len(seq);
    const int64_t row0 = a.b.row(seq);
    const unsigned rows = unsigned(n) * unsigned(a.group);
    // key tiles of the two query tiles, and those of this split
    int nt[2], j0, j1;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const unsigned first = (2 * unsigned(blk) + t) * BM, last = min(first + BM, rows) - 1;
        const int keys = !a.causal ? len : max(len - n + int(last / unsigned(a.group)) + 1, 0);
        nt[t] = first >= rows ? 0 : int((unsigned(keys) + BN - 1) / BN);
    }
    {
        const int all = max(nt[0], nt[1]);
        j0 = int(int64_t(all) * blockIdx.y / a.splits);
        j1 = int(int64_t(all) * (blockIdx.y + 1) / a.splits);
    }
    int scale_e;
    const float scale_m = split_scale(a.scale, scale_e);
    const Abort ab{&s_abort, a.status};
    if (warp == 21) {
        ptx::tmem_alloc(&s_tmem, 512);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = s_tmem;

    if (warp < 16) {
        // ------------------------------------------------------------------------------------------------ softmax
        asm volatile("setmaxnreg.inc.sync.aligned.u32 96;");                 // 512 * 96 + 256 * 48 = 768 * 80
        const int t = warp >> 3, half = warp >> 2 & 1, local = threadIdx.x & 127;            // tile, half of the columns, row
        const int pair = 1 + (t * 4 + (warp & 3));         // barrier of the two warps that share 32 rows
        const unsigned rr = (2 * unsigned(blk) + t) * BM + local, i = rr / unsigned(a.group);
        const bool real = rr < rows;
        const int head = g * a.group + int(rr - i * a.group);
        const int limit = !real ? 0x7fffffff : !a.causal ? len : max(len - n + int(i) + 1, 0);
        float* mine = &s_half[t][half][local];
        const float* other = &s_half[t][half ^ 1][local];
        // ---- the queries into their operand tiles: D / 8 lanes to a row, all of a warp's loads in flight together
        {
            constexpr int L = D / 8, PER = 32 / L, IT = 2 * BM / (16 * PER);
            const int c = lane % L;
            uint4 raw[IT];
#pragma unroll
            for (int x = 0; x < IT; ++x) {
                const unsigned r = 2 * unsigned(blk) * BM + (x * 16 + warp) * PER + lane / L, ri = r / unsigned(a.group);
                raw[x] = make_uint4(0, 0, 0, 0);
                if (r < rows) raw[x] = __ldg(reinterpret_cast<const uint4*>(a.q + (row0 + ri) * a.q_stride + int64_t(g * a.group + int(r - ri * a.group)) * D) + c);
            }
#pragma unroll
            for (int x = 0; x < IT; ++x) {
                const int r = (x * 16 + warp) * PER + lane / L;              // row of the block
                const uint32_t w[4] = {raw[x].x, raw[x].y, raw[x].z, raw[x].w};
                float f[8], m = 0.f;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    f[2 * k] = __uint_as_float(w[k] << 16);
                    f[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
                    m = fmaxf(m, fmaxf(fabsf(f[2 * k]), fabsf(f[2 * k + 1])));
                }
#pragma unroll
                for (int o = L / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
                const int e = max(int(__float_as_uint(m) >> 23) - 127, -100);
                const float up = pow2i(13 - e) * (scale_m < 0.f ? -1.f : 1.f);
                uint32_t h[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) h[k] = bits(__floats2half2_rn(f[k] * up, f[k + 4] * up));
                const int rl = r & (BM - 1);
                sts4(ptx::smem_addr(s_q) + (r / BM) * S::OP + rl * 128 + (c >> 3) * S::ATOM + (((c & 7) ^ (rl & 7)) << 4), make_uint4(h[0], h[1], h[2], h[3]));
                if (c == 0) s_half[r / BM][0][rl] = pow2i(min(max(e - 13 + scale_e, -122), 127));          // not 0: it meets the -infinity of masks
            }
            ptx::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(q_full);
        }
        ptx::named_bar_sync(9, 512);
        const float qn = s_half[t][0][local];              // factor of the row's sums, into base 2
        ptx::named_bar_sync(9, 512);
        const int low = __reduce_min_sync(0xffffffffu, limit);               // fewest keys of this warp's rows
        const uint32_t lanes = uint32_t(warp & 3) << 21;                     // TMEM lane offset of this warp's rows
        const uint32_t t_s = tmem + S::TMEM_S + t * BN + half * kCols + lanes, t_o = tmem + S::TMEM_O + t * D + half * (D / 2) + lanes;
        const int stop = min(nt[t], j1);
        float top = -INFINITY, over = -INFINITY, l = 0.f;                    // the reference, what a score may reach under it, the weights' sum
        bool ok = true, larges = false;                    // some row's reference is a large score
        for (int j = j0; j < stop; ++j) {
            const int slot = (j - j0) % kSlots;
            if (ok && (!wait_bounded(&prm_full[slot], ((j - j0) / kSlots) & 1, ab) || !wait_bounded(&s_full[t], (j - j0) & 1, ab))) ok = false;
            // (after a wait ran out the loop goes on without waiting: the two warps of a row still meet)
            ptx::tc_fence_after_sync();
            const uint32_t flags = s_flags[slot];
            const int first = j * BN + half * kCols;
            const bool masked = j * BN + BN > low || (flags & 2), bare = flags & 1;
            const float e = s_e[slot], qk = fminf(fmaxf(qn * s_ek[slot], 0x1p-122f), 0x1p127f);
            const uint32_t vs = ptx::smem_addr(s_vs + slot * BN + half * kCols), kx = ptx::smem_addr(s_kx + slot * BN + half * kCols), there = ptx::smem_addr(&s_there[slot][2 * half]);
            float m = bare     ? half_max<true, true>(t_s, vs, kx, first, limit, there, qk)
                      : masked ? half_max<true, false>(t_s, vs, kx, first, limit, there, qk)
                               : half_max<false, false>(t_s, vs, kx, first, limit, there, qk);
            *mine = m;
            ptx::named_bar_sync(pair, 64);
            m = fmaxf(m, *other);
            if (!bare) m = fmaf(m, qk, e);
            // the reference moves only when a weight would pass 2^(kPlace + kSlack)
            if (__any_sync(0xffffffffu, m > over)) {
                const float to = m > over ? m - kPlace : top, fix = to == top ? 1.f : ex2(top - to);
                top = to;
                over = to + (fabsf(to) < kLargeScore ? kPlace + kSlack : kPlace);
                larges = __any_sync(0xffffffffu, fabsf(to) >= kLargeScore && to != -INFINITY);
                l *= fix;
                if (j > j0) {
#pragma unroll 1
                    for (int c = 0; c < D / 64; ++c) {
                        uint32_t r[32];
                        ptx::tmem_ld_32x32b_x32(t_o + 32 * c, r);
                        ptx::tmem_ld_wait();
#pragma unroll
                        for (int k = 0; k < 32; ++k) r[k] = __float_as_uint(__uint_as_float(r[k]) * fix);
                        tmem_st_x32(t_o + 32 * c, r);
                    }
                    tmem_st_wait();
                }
            }
            const float at = top == -INFINITY ? 0.f : top;
            float factor = qk, sub = e - at;
            if (larges && e != 0.f) {
                const bool large = fabsf(at) >= kLargeScore;
                // large scores swallow an e that is added to the reference, and with it what tiles differ in: there it comes last, in
                // a pass of its own (in the loops of all scores it cost 4 to 8 %)
#pragma unroll 1
                for (int c = 0; c < kCols / 32; ++c) {
                    uint32_t r[32];
                    ptx::tmem_ld_32x32b_x32(t_s + 32 * c, r);
                    ptx::tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < 32; ++k) r[k] = large ? __float_as_uint(fmaf(__uint_as_float(r[k]), qk, -at) + e) : r[k];
                    tmem_st_x32(t_s + 32 * c, r);
                }
                tmem_st_wait();
                if (large) factor = 1.f, sub = 0.f;
            }
            if (bare) l += half_weights<true, true>(t_s, vs, kx, first, limit, there, factor, sub);
            else l = fmaf(masked ? half_weights<true, false>(t_s, vs, kx, first, limit, there, factor, sub)
                                 : half_weights<false, false>(t_s, vs, kx, first, limit, there, factor, sub), pow2i(-int(e)), l);
            tmem_st_wait();
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&p_full[t]);
        }
        // ---- the row's output, half of the channels each
        ptx::named_bar_sync(pair, 64);                     // `mine` has been read
        *mine = l;
        ptx::named_bar_sync(pair, 64);
        l += *other;
        const int64_t row = row0 + i;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const bool some = stop > j0;
        if (ok && some) {
            ok = wait_bounded(&o_full[t], 0, ab);
            ptx::tc_fence_after_sync();
        }
        if (ok) {
            const int64_t at = (int64_t(blockIdx.y) * a.b.rows + row) * a.q_heads + head;
#pragma unroll 1
            for (int c = 0; c < D / 64; ++c) {
                const int ch = half * (D / 2) + 32 * c;
                uint32_t r[32];
                if (some) {
                    ptx::tmem_ld_32x32b_x32(t_o + 32 * c, r);
                    ptx::tmem_ld_wait();
                } else {
#pragma unroll
                    for (int k = 0; k < 32; ++k) r[k] = 0;
                }
                if (real) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        float f[8];
#pragma unroll
                        for (int x = 0; x < 8; ++x) f[x] = __uint_as_float(r[8 * k + 2 * (x & 3) + (x >> 2)]);   // 0 4 1 5 2 6 3 7
                        if (a.splits > 1) {
                            store8(a.part_o + at * D + ch + 8 * k, f);
                        } else {
#pragma unroll
                            for (int x = 0; x < 8; ++x) f[x] *= inv;
                            store8(a.out + row * a.out_stride + int64_t(head) * D + ch + 8 * k, f);
                        }
                    }
                }
                __syncwarp();
            }
            if (real && half == 0) {
                if (a.splits > 1) a.part_ml[at] = make_float2(top, l);
                else if (a.lse) a.lse[row * a.q_heads + head] = l == 0.f ? -INFINITY : ((top == -INFINITY ? 0.f : top) + log2f(l)) * 0.6931471805599453f;
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
        const int piece_log2 = min(a.b.page_log2, 7), per_tile = BN >> piece_log2;
        if (warp < 20) {
            // -------------------------------------------------------------------------------------------- unpack
            const int tok = threadIdx.x - 512;
            bool ok = true;
            uint32_t step = 0;                             // 2 * tile + (0 keys, 1 values)
            for (int j = j0; ok && j < j1; ++j) {
                const int slot = (j - j0) % kSlots;
                const uint32_t prm = ptx::smem_addr(s_rawp + ((j - j0) & 1) * S::RAWP) + 8 * tok;
                if (!wait_bounded(&prm_full[slot], ((j - j0) / kSlots) & 1, ab)) { ok = false; break; }
#pragma unroll 1
                for (int v = 0; v < 2; ++v, ++step) {      // keys, values
                    const int rs = step % S::RAWS, ob = step % S::OPS;
                    const uint32_t raw = ptx::smem_addr(s_raw + rs * S::RAW), op = ptx::smem_addr(s_op + ob * S::OP);
                    if (!wait_bounded(&raw_full[rs], (step / S::RAWS) & 1, ab)) { ok = false; break; }
                    const float zero = __uint_as_float(lds1(prm + v * (BN * 8))), factor = __uint_as_float(lds1(prm + v * (BN * 8) + 4));
                    const bool far = is_far(zero);
                    if (!wait_bounded(&op_empty[ob], ((step / S::OPS) & 1) ^ 1, ab)) { ok = false; break; }
                    unpack_row<D>(raw, op, tok, zero, factor, far);
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) { ptx::mbar_arrive(&op_full[ob]); ptx::mbar_arrive(&raw_empty[rs]); }
                }
            }
        } else if (warp == 22) {
            // -------------------------------------------------------------------------------------------- parameters
            // Lane l has tokens l, l + 32, ..  The (zero, factor) that unpacking needs takes the place of (scale, zero).
            const int top_keys = !a.causal ? len : max(len - n + int((min((2 * unsigned(blk) + 2) * BM, rows) - 1) / unsigned(a.group)) + 1, 0);
            for (int j = j0; j < j1; ++j) {
                const int slot = (j - j0) % kSlots, step = 2 * (j - j0), rs = step % S::RAWS;
                if (!wait_bounded(&raw_full[rs], (step / S::RAWS) & 1, ab)) break;
                const uint32_t pieces = s_pieces[rs];
                float2* prm = reinterpret_cast<float2*>(s_rawp + ((j - j0) & 1) * S::RAWP);
                float2 kp[4], vp[4];
                int hi = -1000, lo = 1000, vlo = 1000, khi = -1000, klo = 1000;
                float kround[4];                           // what of a key is rounded to fp16: its scale, or (far from zero) its values
                uint32_t goods = 0, everywhere = 0xffffffffu;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int tok = 32 * i + lane;
                    const bool good = j * BN + tok < top_keys && ((pieces >> (tok >> piece_log2)) & 1u);
                    kp[i] = prm[tok];
                    kp[i].x *= fabsf(scale_m);                   // (its sign is the queries')
                    vp[i] = prm[BN + tok];
                    if (!good) kp[i] = vp[i] = make_float2(0.f, 0.f);
                    goods |= uint32_t(good) << i;
                    // parameters that are no numbers: the values stay finite, a row that sees the token gets it from the score
                    if (!(fabsf(vp[i].x) <= 3e38f && fabsf(vp[i].y) <= 3e38f)) { kp[i].x = NAN; vp[i] = make_float2(0.f, 0.f); }
                    if (!(fabsf(kp[i].y) <= 3e38f)) { kp[i].x = NAN; kp[i].y = 0.f; }
                    const float klargest = fabsf(kp[i].x) * fmaxf(fabsf(kp[i].y), fabsf(15.f - kp[i].y));
                    kround[i] = klargest > 0.f && klargest <= 3e38f ? (is_far(kp[i].y) ? klargest : fabsf(kp[i].x)) : 0.f;
                    if (kround[i] != 0.f) {
                        khi = max(khi, int(__float_as_uint(klargest) >> 23) - 127);
                        klo = min(klo, int(__float_as_uint(kround[i]) >> 23) - 127);
                    }
                    const float largest = fabsf(vp[i].x) * fmaxf(fabsf(vp[i].y), fabsf(15.f - vp[i].y));
                    if (largest != 0.f) {
                        const int ex = largest < 1.2e24f ? max(int(__float_as_uint(largest) >> 23) - 127, -80) : 1000;   // 2^80: the logarithm's cut
                        hi = max(hi, ex);
                        lo = min(lo, ex);
                        if (ex > -80 && !is_far(vp[i].y)) vlo = min(vlo, int(__float_as_uint(fabsf(vp[i].x)) >> 23) - 127);
                    }
                    const uint32_t there = __ballot_sync(0xffffffffu, good);
                    everywhere &= there;
                    if (lane == 0) s_there[slot][i] = there;
                }
                hi = __reduce_max_sync(0xffffffffu, hi);
                lo = __reduce_min_sync(0xffffffffu, lo);
                vlo = __reduce_min_sync(0xffffffffu, vlo);
                khi = __reduce_max_sync(0xffffffffu, khi);
                klo = __reduce_min_sync(0xffffffffu, klo);
                const int ek = khi < -900 ? 0 : min(max(khi, -120), 120);
                const bool bare = hi > 900 || hi - lo > 10 || vlo < hi - 14 || klo < ek - 14;      // (none at all: -1000 and 1000)
                const int e = bare || hi < -900 ? 0 : hi;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float vf = 1.f, kf = kp[i].x * pow2i(-ek);
                    if (bare) {
                        int x = ek;                        // (a scale that is 0 or no number stays what it is)
                        if (kround[i] != 0.f) {
                            x = int(__float_as_uint(kround[i]) >> 23) - 127;
                            kf = kp[i].x * pow2i(-x);
                        }
                        s_kx[slot * BN + 32 * i + lane] = uint16_t(__float_as_uint(pow2i(max(x - ek, -126))) >> 16);
                        if (is_far(vp[i].y)) {
                            const int k = min(max(int((__float_as_uint(vp[i].y) >> 23) & 255u) - 127 - 9, 0), 120);
                            vf = pow2i(-k);
                            vp[i].x *= pow2i(k);
                        }
                        s_vs[slot * BN + 32 * i + lane] = vp[i].x;
                    } else {
                        vf = vp[i].x * pow2i(-e);
                    }
                    prm[32 * i + lane] = make_float2(kp[i].y, kf);
                    prm[BN + 32 * i + lane] = make_float2(vp[i].y, goods >> i & 1 ? vf : 0.f);
                }
                if (lane == 0) {
                    s_ek[slot] = pow2i(ek);
                    s_e[slot] = float(e);
                    s_flags[slot] = (bare ? 1 : 0) | (everywhere != 0xffffffffu ? 2 : 0);
                }
                ptx::fence_proxy_async_smem();             // the next bulk copy into prm comes after these writes
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&prm_full[slot]);
            }
        } else if (warp == 20) {
            // -------------------------------------------------------------------------------------------- codes in
            // lane = 4 * piece + array (keys' codes, their parameters, the values' parameters, the values' codes)
            const int piece = lane >> 2, array = lane & 3, log2p = a.b.page_log2;
            const int keys = min(len, j1 * BN), pieces = int((unsigned(keys) + (1u << piece_log2) - 1) >> piece_log2);
            const int32_t* table = a.b.table + int64_t(seq) * a.b.width;
            auto page_of = [&](int q) { return q < pieces ? table[(int64_t(q) << piece_log2) >> log2p] : 0; };
            const uint32_t bytes = uint32_t(array == 0 || array == 3 ? D / 2 : 8) << piece_log2;
            const int offset = (array == 2 ? BN * 8 : 0) + min(piece, per_tile - 1) * int(bytes);
            const uint8_t* source = array == 0 ? a.c.kc : array == 3 ? a.c.vc : reinterpret_cast<const uint8_t*>(array == 1 ? a.c.kp : a.c.vp);
            const int row_bytes = array == 0 || array == 3 ? D / 2 : 8;
            bool ok = true;
            uint32_t step = 0;
            int q0 = j0 * per_tile, held = page_of(q0 + lane), ahead = page_of(q0 + 32 + lane);
            for (int j = j0; ok && j < j1; ++j) {
                const int q = j * per_tile + piece;
                if (j * per_tile - q0 >= 32) {
                    q0 += 32;
                    held = ahead;
                    ahead = page_of(q0 + 32 + lane);
                }
                const int page = __shfl_sync(0xffffffffu, held, q - q0);
                const bool mine = piece < per_tile && q < pieces, good = mine && page >= 0 && page < a.c.pages;
                if (mine && !good) raise_page(a.status);
                const int64_t r = a.c.row(page, g, (q << piece_log2) & ((1 << log2p) - 1));
                const uint32_t got = __ballot_sync(0xffffffffu, good && array == 0);
                uint32_t mask = 0;
#pragma unroll
                for (int x = 0; x < 8; ++x) mask |= ((got >> (4 * x)) & 1u) << x;
#pragma unroll
                for (int v = 0; v < 2; ++v, ++step) {
                    const bool now = good && (array == 3) == (v == 1);
                    const uint32_t total = __reduce_add_sync(0xffffffffu, now ? bytes : 0);
                    const int rs = step % S::RAWS;
                    if (!wait_bounded(&raw_empty[rs], ((step / S::RAWS) & 1) ^ 1, ab)) { ok = false; break; }
                    if (lane == 0) {
                        s_pieces[rs] = mask;
                        ptx::mbar_arrive_expect_tx(&raw_full[rs], total);
                    }
                    __syncwarp();
                    uint8_t* target = array == 0 || array == 3 ? s_raw + rs * S::RAW : s_rawp + ((j - j0) & 1) * S::RAWP;
                    if (now) bulk_load(target + offset, source + r * row_bytes, bytes, &raw_full[rs]);
                }
            }
            if (!ok) {                                     // give copies still in flight a bounded chance to land
                for (uint32_t k = 0; k < uint32_t(S::RAWS) && k < step; ++k) {
                    const uint32_t x = step - 1 - k;
                    const long long t0 = clock64();
                    while (!ptx::mbar_try_wait(&raw_full[x % S::RAWS], (x / S::RAWS) & 1) && clock64() - t0 < (1ll << 24)) {}
                }
            }
        } else if (warp == 21) {
            // -------------------------------------------------------------------------------------------- MMAs
            constexpr uint32_t id_s = idesc_f16(BM, BN, false), id_o = idesc_f16(BM, D, true);
            const uint32_t leader = elect_one();
            const uint32_t q_low = desc_low(ptx::smem_addr(s_q), 16), k_low = desc_low(ptx::smem_addr(s_op), 16), v_low = desc_low(ptx::smem_addr(s_op), S::ATOM);
            auto score = [&](int t, int ob) {
                const uint32_t q = q_low + t * (S::OP >> 4), k = k_low + ob * (S::OP >> 4);
                if (leader) {
#pragma unroll
                    for (int x = 0; x < D / 16; ++x) {
                        const uint32_t at = ((x >> 2) * S::ATOM + (x & 3) * 32) >> 4;
                        mma_f16_ss(tmem + S::TMEM_S + t * BN, q + at, k + at, id_s, x != 0);
                    }
                    ptx::mma_commit(&s_full[t]);
                }
                __syncwarp();
            };
            auto commit = [&](uint64_t* bar) {
                if (leader) ptx::mma_commit(bar);
                __syncwarp();
            };
            bool ok = wait_bounded(q_full, 0, ab);
            if (ok && j0 < j1) {
                ok = wait_bounded(&op_full[0], 0, ab);
                if (ok) {
                    ptx::tc_fence_after_sync();
                    if (j0 < nt[0]) score(0, 0);
                    if (j0 < nt[1]) score(1, 0);
                    commit(&op_empty[0]);
                }
            }
            for (int j = j0; ok && j < j1; ++j) {
                const uint32_t sv = 2 * (j - j0) + 1, sk = sv + 1;           // steps of V_j and K_j+1
                const bool more = j + 1 < j1;
                if (!wait_bounded(&op_full[sv % S::OPS], (sv / S::OPS) & 1, ab)) break;
                if (more && !wait_bounded(&op_full[sk % S::OPS], (sk / S::OPS) & 1, ab)) break;
                const uint32_t v = v_low + (sv % S::OPS) * (S::OP >> 4);
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if (j >= nt[t]) continue;
                    if (!wait_bounded(&p_full[t], (j - j0) & 1, ab)) { ok = false; break; }
                    ptx::tc_fence_after_sync();
                    if (leader) {
#pragma unroll
                        for (int x = 0; x < BN / 16; ++x)
                            mma_f16_ts(tmem + S::TMEM_O + t * D, tmem + S::TMEM_S + t * BN + (x >> 2) * kCols + 8 * (x & 3), v + x * (2048 >> 4), id_o, x > 0 ? 1u : uint32_t(j > j0));
                    }
                    __syncwarp();
                    if (more && j + 1 < nt[t]) score(t, sk % S::OPS);
                    else commit(&o_full[t]);
                }
                commit(&op_empty[sv % S::OPS]);
                if (more) commit(&op_empty[sk % S::OPS]);
            }
        }
    }
    __syncwarp();
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == 21) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem, 512);
    }
}

// Joins the splits of a row: a CTA per (packed row, 4 query heads), a warp per head.
template <int D>
__global__ void __launch_bounds__(128) kv_prompt_join_kernel(const Args a) {
    constexpr int V = D / 32;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const int64_t unit = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 5), row = unit / a.q_heads;
    if (row >= a.b.rows) return;
    const int s = a.b.seq_of(row);
    if (s < 0 || blocks_of(a, s) == 0) return;
    const int64_t step = a.b.rows * a.q_heads;
    float m = -INFINITY;
    for (int z = 0; z < a.splits; ++z) m = fmaxf(m, a.part_ml[z * step + unit].x);
    const float ref = m == -INFINITY ? 0.f : m;
    float l = 0.f, o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = 0.f;
    for (int z = 0; z < a.splits; ++z) {
        const float2 ml = a.part_ml[z * step + unit];
        const float f = ml.y == 0.f ? 0.f : ml.x == -INFINITY ? 1.f : ex2(ml.x - ref);       // (a NaN sum goes through)
        if (f == 0.f) continue;
        l = fmaf(f, ml.y, l);
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] = fmaf(f, a.part_o[(z * step + unit) * D + lane * V + i], o[i]);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int head = int(unit - row * a.q_heads);
#pragma unroll
    for (int i = 0; i < V; ++i) a.out[row * a.out_stride + int64_t(head) * D + lane * V + i] = __float2bfloat16(o[i] * inv);
    if (a.lse && lane == 0) a.lse[unit] = l == 0.f ? -INFINITY : (ref + log2f(l)) * 0.6931471805599453f;
}

// CTAs of a call at most, per split: every sequence rounds its rows up once.
inline int64_t blocks_bound(const Batch& b, int group) { return (b.rows * group + 2 * BM - 1) / (2 * BM) + std::min<int64_t>(b.seqs, b.rows); }

// Keys are cut into as many parts as fill the SMs once with the blocks that there are likely to be: all new tokens in sequences
// of max_new.
inline int splits_of(const Batch& b, int heads, int group, int max_new) {
    const int64_t seqs = (b.rows + max_new - 1) / max_new, ctas = seqs * ((int64_t(max_new) * group + 2 * BM - 1) / (2 * BM)) * heads;
    return int(std::max<int64_t>(1, std::min<int64_t>(8, device_sm_count() / ctas)));
}

template <int D>
int launch(const Args& a, cudaStream_t st) {
    constexpr auto kern = &kv_prompt_kernel<D>;
    QLLM_CUDA_TRY(allow_smem<kern>(Shape<D>::SMEM));
    const int64_t ctas = blocks_bound(a.b, a.group) * a.c.heads;
    if (ctas > 0x7fffffff) return QLLM_ERR_UNSUPPORTED;
    kern<<<dim3(unsigned(ctas), a.splits), kThreads, Shape<D>::SMEM, st>>>(a);
    int rc = after_launch();
    if (rc != QLLM_OK || a.splits == 1) return rc;
    QLLM_CUDA_TRY(launch_dependent(kv_prompt_join_kernel<D>, dim3(unsigned((a.b.rows * a.q_heads + 3) / 4)), dim3(128), 0, st, a));
    return after_launch();
}

}  // namespace

namespace kv {

bool prompt_serves(int head_dim, int dtype) { return dtype == QLLM_BF16 && (head_dim == 64 || head_dim == 128); }

int64_t prompt_workspace(const Batch& b, int heads, int head_dim, int group, int max_new) {
    const int splits = splits_of(b, heads, group, max_new);
    return splits == 1 ? 0 : int64_t(splits) * b.rows * heads * group * (head_dim + 2) * 4;
}

int launch_attention_prompt(const Cache& c, const Batch& b, int head_dim, const AttnArgs& x, int max_new, void* workspace, int* status,
                            cudaStream_t st) {
    Args a;
    a.c = c;
    a.b = b;
    a.q = static_cast<const __nv_bfloat16*>(x.q);
    a.out = static_cast<__nv_bfloat16*>(x.out);
    a.lse = x.lse;
    a.q_stride = x.q_stride;
    a.out_stride = x.out_stride;
    a.group = x.group;
    a.q_heads = x.q_heads;
    a.causal = x.causal;
    a.most_rows = x.most_rows;
    a.scale = x.scale;
    a.splits = splits_of(b, c.heads, x.group, max_new);
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float2*>(a.part_o + int64_t(a.splits) * b.rows * x.q_heads * head_dim);
    a.status = status;
    return head_dim == 64 ? launch<64>(a, st) : launch<128>(a, st);
}

}  // namespace kv
}  // namespace qllm
