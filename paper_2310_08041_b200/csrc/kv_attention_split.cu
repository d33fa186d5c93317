// Attention over the 4-bit cache for few query rows per key head: decode steps, drafted tokens, odd shapes.
//
// s_j = scale q . k_j, k_j = ks_j (ck_j - kz_j), so s_j = ks_j (scale q . ck_j - kz_j scale sum q): the keys enter the
// tensor cores as bare codes, scale and zero-point act on finished sums.  Likewise sum_j p_j v_j = sum_j (p_j vs_j) cv_j -
// sum_j (p_j vs_j) vz_j.  A token's keys and values are D + 16 bytes a head, read once per 8 NT query rows; in the middle of a long
// call they come at the copy rate, at its ends latency is what bounds it (measured below).
//
// Work split: an item is (sequence, key head, tile of 8 NT query rows); its keys are tiles of T tokens.  All items' tiles form
// one line, which the CTAs of one resident wave cut into equal shares, each working out its own from the lengths on the
// device: a batch of any lengths keeps every SM busy, and a captured graph follows them.  An item that lies in several shares
// leaves one piece per share (sum, running maximum, weights) in the workspace, which a second kernel joins by the records that the
// CTAs leave; at most two pieces per CTA.  No CTA waits for another, and the order of all additions is fixed by the shapes and lengths.
//
// In a CTA: one warp fetches a tile's codes and parameters with bulk copies, one per page and array, several tiles ahead; four
// warps own 32 of its tokens each, with a softmax state of their own that meets at the item's end.  Both products run
// transposed (S^T = K Q^T, O^T = V^T P^T) so that 16 tokens or channels fill the 16 rows of the warp-level MMA and the 8
// query rows its 8 columns: a decode step's few rows waste nothing.  A nibble masked in place is a denormal fp16 number (c 2^-24,
// or c 2^-20 from the upper half of a byte), which the MMA takes: five logical instructions turn 8 key codes into operands, and as
// many and four packed subtractions the value codes of 16-bit units that a transposing load has paired.  Channel order inside an
// operand is free as long as both sides agree, so the key codes of one 16-byte read are used where they lie, and the factor 16 of
// the upper nibbles is taken out of the queries.
//
// Precision: queries are scaled by a power of two per row into fp16's range (a bf16 query's 8 bits stay exact) and float32
// queries are split in two; weights p_j vs_j are rounded to fp16, 11 bits, for bf16 results (which carry 8) and split in two
// for float32 ones, whose keys also enter as normal numbers and whose sums over more than 16 or 32 terms are float32 additions.
// So that no weight leaves fp16's range whatever the value scales are, the running maximum is that of s_j + log2 vs_j (the
// logarithm cut to +-80; its integer part for float32), with the largest weight placed at 2^6; it moves only when a weight would
// pass 2^14, which spares most steps the reduction over lanes and the rescaling.  Sums, maxima and zero-point corrections are
// float32.  A row's factor of its scores is a power of two (split_scale).

// Measured (us a call, both kernels; the bytes of the cache at the measured copy rate in brackets): one sequence of 131071
// tokens, 64 query on 8 key heads of 128, bf16: 44 (23), of which the main kernel streams 24 at that rate, starts for 6 (plan, table,
// first tiles) and spreads over 8 at the end, and joining takes 5; 32 sequences of 176 to 9001 tokens: 37 (16); 6 sequences, up to
// 5 new tokens, 40 heads, float32: 23 (4).  By events with a flushed L2: 16 sequences of 8192 tokens, 32 query on 8 key heads of 256,
// 85 (43), in float32 157.  Prompts of float32 calls and of heads of 256 come here too, whose keys are read and decoded again for
// every 8 rows: 1024 tokens, the same heads, 343 in bf16 and 652 in float32, 269 in float32 at heads of 128 (where the tensor-core
// kernel takes 38 in bf16).  Without its arithmetic the kernel took 2 us less: latency at both ends, not the instruction rate, is
// what is left.  Tried and dropped: four CTAs per SM in 96 registers (spills, 60 instead of 48), two or three times as many shares as
// CTAs that fit (60, 80), reading page ids tile by tile (no difference).

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

constexpr int T = 128;                                     // tokens of a tile
constexpr int kWarps = 4;                                  // consumer warps, 32 tokens each
constexpr int kThreads = 32 * (kWarps + 1);
constexpr int kCombineThreads = 128;
constexpr float kPlace = 6.f, kSlack = 8.f;                // where the largest weight is placed (powers of two), how far it may grow

template <int D, int NT, bool F32>
struct Shape {
    static constexpr int R = 8 * NT;                       // query rows of an item
    static constexpr int MT = D / 16;
    static constexpr int STAGE = T * (D + 16);
    static constexpr int STAGES = D == 256 ? 2 : 3;
    static constexpr int OROW = D + 4;                     // floats of a merged row (padded)
    static constexpr int MERGE = kWarps * R * (OROW + 4) * 4;
    static constexpr int SMEM = STAGES * STAGE + MERGE + 256;
    static constexpr int CTAS = SMEM <= 75 * 1024 && NT * D * (F32 ? 3 : 2) <= 256 ? 3 : 2;
};

// ---- the line of work ----------------------------------------------------------------------------------------------------
// An item costs kItemCost tiles for its queries, its first loads and its end, then one for each tile of keys: a share that
// ends in front of the first tile takes none of the item.  (Counting tiles alone gave the CTAs that got the short sequences of
// a ragged batch half as much work again: 46 us instead of 40 for 32 sequences of 176 to 9001 tokens.  2, 3 and 5 tiles: 36.6,
// 36.6, 38.0 us there, 22.7, 24.2, 25.5 for 6 sequences of up to 1999 tokens, 40 heads, float32.)
constexpr int kItemCost = 2;

struct Plan {
    Batch b;
    int heads, group, row_log2, rows;                      // key heads, query heads per key head, rows of an item
    unsigned most_rows;                                    // sequences with more query rows are another kernel's
    // (query rows of a call fit 31 bits: checked before the launch)
    __device__ __forceinline__ unsigned qrows(int n) const { return unsigned(n) * unsigned(group); }
    __device__ __forceinline__ unsigned qtiles(int n) const { return (qrows(n) + rows - 1) >> row_log2; }
    __device__ __forceinline__ int ktiles(int len) const { return len <= T ? 1 : int((unsigned(len) + T - 1) / T); }
    __device__ __forceinline__ int64_t work(int s) const {
        const int n = b.count(s);
        return n == 0 || qrows(n) > most_rows ? 0 : int64_t(heads) * qtiles(n) * (ktiles(b.len(s)) + kItemCost);
    }
};

// quotient and rest, in 32 bits where they suffice
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b, int64_t& rest) {
    if (((a | b) >> 32) == 0) {
        const unsigned q = unsigned(a) / unsigned(b);
        rest = unsigned(a) - q * unsigned(b);
        return q;
    }
    const int64_t q = a / b;
    rest = a - q * b;
    return q;
}

// `total` cut into `ctas` shares that differ by one at most.
struct Shares {
    int64_t each, more;                                    // the first `more` shares have each + 1
    __device__ __forceinline__ Shares(int64_t total, int ctas) { each = divide(total, ctas, more); }
    __device__ __forceinline__ int64_t begin(int64_t c) const { return c * each + min(c, more); }
    __device__ __forceinline__ int owner(int64_t x) const {
        int64_t rest;
        return x < more * (each + 1) ? int(divide(x, each + 1, rest)) : int(more + divide(x - more * (each + 1), each, rest));
    }
};

// Called by a whole CTA of kThreads threads: total work, and (in every thread) the sequence whose range of the line holds
// the beginning of share c, with the work in front of it.
__device__ __forceinline__ int64_t locate(const Plan& p, int64_t* s_mem, int c, int ctas, int& seq, int64_t& before) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (p.b.seqs + kThreads - 1) / kThreads, first = min(tid * per, p.b.seqs), last = min(first + per, p.b.seqs);
    int64_t mine = 0;
    for (int s = first; s < last; ++s) mine += p.work(s);
    int64_t incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) s_mem[warp] = incl;
    __syncthreads();
    int64_t base = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) base += s_mem[w];
        total += s_mem[w];
    }
    const int64_t pre = base + incl - mine, x = Shares(total, ctas).begin(c);
    if (x >= pre && x < pre + mine) {
        int64_t at = pre;
        int s = first;
        for (; s < last - 1; ++s) {
            const int64_t w = p.work(s);
            if (x < at + w) break;
            at += w;
        }
        s_mem[kThreads / 32] = s;
        s_mem[kThreads / 32 + 1] = at;
    }
    __syncthreads();
    seq = int(s_mem[kThreads / 32]);
    before = s_mem[kThreads / 32 + 1];
    return total;
}

// The part of an item that lies in a share.
struct Part {
    int s, g, qt, n, len, tile, tiles, count;              // sequence .., first tile, tiles of the item, tiles of the part
    int64_t row0, first;                                   // first packed row of the sequence, the item's place in the line
    int keys;                                              // keys that the item's last row sees
};
// Walks the parts of [x, end).  Every role of the CTA walks for itself.
struct Walk {
    const Plan& p;
    int64_t x, end, before;
    int s;
    bool causal;
    __device__ __forceinline__ bool next(Part& o) {
        while (x < end) {
            int64_t w;
            while ((w = p.work(s)) <= x - before) { before += w; ++s; }  // x < total: a sequence with work follows
            o.s = s;
            o.n = p.b.count(s);
            o.len = p.b.len(s);
            o.row0 = p.b.row(s);
            o.tiles = p.ktiles(o.len);
            int64_t in_item, qt;
            const int64_t item = divide(x - before, o.tiles + kItemCost, in_item);
            o.g = int(divide(item, p.qtiles(o.n), qt));
            o.qt = int(qt);
            o.first = x - in_item;
            o.tile = max(int(in_item) - kItemCost, 0);
            const int64_t stop = min(int64_t(o.tiles + kItemCost), end - o.first);
            o.count = int(stop) - kItemCost - o.tile;
            x = o.first + stop;
            if (o.count <= 0) continue;                    // the share ends in front of the item's first tile
            const unsigned last = min(unsigned(o.qt + 1) << p.row_log2, p.qrows(o.n)) - 1;
            const int own = o.len - o.n + int(last / unsigned(p.group)) + 1;
            o.keys = !causal ? o.len : max(own, 0);
            return true;
        }
        return false;
    }
};

// What a CTA leaves for the joining kernel: the item that begins in its share and goes on behind it (rows = 0: none).
struct __align__(16) Record {
    int64_t row0;                                          // first packed row of the sequence
    int first_row, rows;                                   // query rows first_row .. first_row + rows - 1 of the key head
    int head;                                              // first query head of the group
    int last;                                              // the share that holds its end
};

// ---- warp-level pieces ---------------------------------------------------------------------------------------------------
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
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
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack2(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
__device__ __forceinline__ float pow2i(int e) { return __int_as_float((e + 127) << 23); }     // -126 <= e <= 127
// 2^e for any e
__device__ __forceinline__ float pow2(int e) { return pow2i(min(max(e, -126), 127)) * (e < -126 ? pow2i(max(e + 126, -126)) : 1.f); }
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(ptx::smem_addr(dst)),
                 "l"(src), "r"(bytes), "r"(ptx::smem_addr(bar))
                 : "memory");
}
// Four 8 x 8 matrices of 16-bit units, transposed: lane (r, t) receives unit r of rows 2t and 2t + 1 of each.
__device__ __forceinline__ void load_units(const uint8_t* p, uint32_t (&x)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(ptx::smem_addr(p)) : "memory");
}

// Codes as A operands: two nibbles of a word (`upper`: those of bits 4-7 and 20-23, else 0-3 and 16-19).  The keys of a bf16 call
// are taken as they are masked, denormal numbers c 2^-24 and 16 c 2^-24.  The MMA aligns its sums to the operands' nominal
// exponents, which for denormals lie up to 10 bits above their values, and cuts what falls off: 2^-16 of a score's terms is lost.
// NORMAL (values, whose sums run over the whole context, and everything in float32): c - 8 as normal numbers; 1024 + c and
// 1024 + 16 c are fp16 numbers, one packed operation makes the difference.
template <bool NORMAL>
__device__ __forceinline__ uint32_t codes2(uint32_t w, bool upper) {
    if constexpr (!NORMAL) return w & (upper ? 0x00F000F0u : 0x000F000Fu);
    const uint32_t h = (w & (upper ? 0x00F000F0u : 0x000F000Fu)) | 0x64006400u;
    const __half2 v = *reinterpret_cast<const __half2*>(&h);
    const __half2 r = upper ? __hfma2(v, __float2half2_rn(0.0625f), __float2half2_rn(-72.f)) : __hadd2(v, __float2half2_rn(-1032.f));
    return *reinterpret_cast<const uint32_t*>(&r);
}

// The query row of column `r` as B operands.  2^(e + kUnit) is what a unit of the sums made with them stands for, `ratio` the row's sum
// in those units (NaN for a row that is not finite).
template <bool F32>
constexpr int kUnit = F32 ? -13 : 11;                      // 2^(e - 13), times 2^24 for the codes of a bf16 call
template <typename QT, int D, bool F32>
__device__ __forceinline__ void load_queries(const QT* row, int t, uint32_t (&hi)[D / 8], uint32_t (&lo)[F32 ? D / 8 : 1], int& e, float& ratio) {
    constexpr int N = D / 4;                               // channels of this lane: N t .. N t + N - 1
    float top = 0.f, sum = 0.f;
    if (row) {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            float f[8];
            load8<QT>(row + t * N + 8 * i, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(f[j]));
        }
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    e = max(int(__float_as_uint(top) >> 23) - 127, -100);                // 2^e <= top < 2^(e+1); infinities: 128
    const float up = pow2i(13 - e);
#pragma unroll
    for (int i = 0; i < N / 8; ++i) {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = 0.f;
        if (row) load8<QT>(row + t * N + 8 * i, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            f[j] *= up;                                    // (summed at this size: the sum of large queries may pass float32)
            sum += f[j];
            if ((j & 1) && !F32) f[j] *= 0.0625f;
        }
        // word 8i of the codes gives the pairs (0, 4), (1, 5) x 16, (2, 6), (3, 7) x 16
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t h = pack2(f[j], f[j + 4]);
            hi[4 * i + j] = h;
            if (F32) {
                const float2 b = unpack2(h);
                lo[4 * i + j] = pack2(f[j] - b.x, f[j + 4] - b.y);
            }
        }
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    ratio = e > 127 ? NAN : sum * pow2i(-13 - kUnit<F32>);
}

template <int W>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[W]) {
    if constexpr (W == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        w[0] = v.x; w[1] = v.y;
    } else {
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
            const uint4 v = reinterpret_cast<const uint4*>(p)[i];
            w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
    }
}

// What a warp keeps of an item: lane (r, t) holds columns 2t, 2t + 1 of every column group.
template <int D, int NT, bool F32>
struct State {
    uint32_t qh[NT][D / 8], ql[NT][F32 ? D / 8 : 1];       // queries of column r as B operands
    float qn[NT][2], qr[NT][2];                            // factor of the scores (into base 2; a power of two), sum of the query in the units of its key sums
    int limit[NT][2];                                      // keys that the column sees
    float o[NT][D / 16][4], top[NT][2], l[NT][2], zs[NT][2];
    float room;                                            // how far scores may lie above `top`: no slack once some were large
};

// 32 tokens, from `first` on.  key_unit: what the key scales are multiplied by, the mantissa of the scale and the part of the columns'
// factors that float32 would not hold in qn.  MASKED: some tokens are hidden from some column, or not there.
template <int D, int NT, bool F32, bool MASKED>
__device__ __forceinline__ void step(State<D, NT, F32>& st, const uint8_t* kc, const uint8_t* vc, const float2* kp, float key_unit,
                                     int first, int len, uint32_t there, int r, int t) {
    constexpr int KW = D / 32, MT = D / 16;
    constexpr float kCentre = F32 ? 8.f : 0.f;             // what the operands have taken off the keys' codes
    float s[NT][2][4], s2[NT][2][4];                       // two chains of MMAs each: their latency bounds a warp
    // ---- S^T = K Q^T, 16 tokens at a time
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        uint32_t w0[KW], w1[KW];
        load_words<KW>(kc + (b * 16 + r) * (D / 2) + t * (D / 8), w0);
        load_words<KW>(kc + (b * 16 + 8 + r) * (D / 2) + t * (D / 8), w1);
#pragma unroll
        for (int a = 0; a < NT; ++a)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[a][b][e] = s2[a][b][e] = 0.f;
#pragma unroll
        for (int i = 0; i < KW; ++i) {
            const uint32_t u0 = w0[i] >> 8, u1 = w1[i] >> 8;
            const uint32_t a0 = codes2<F32>(w0[i], false), a1 = codes2<F32>(w1[i], false), a2 = codes2<F32>(w0[i], true), a3 = codes2<F32>(w1[i], true);
            const uint32_t c0 = codes2<F32>(u0, false), c1 = codes2<F32>(u1, false), c2 = codes2<F32>(u0, true), c3 = codes2<F32>(u1, true);
#pragma unroll
            for (int a = 0; a < NT; ++a) {
                if constexpr (F32) {
                    // the MMA cuts its sums instead of rounding them: 16 channels at a time, joined by additions that round
                    float d[4] = {0.f, 0.f, 0.f, 0.f};
                    mma_f16(d, a0, a1, a2, a3, st.ql[a][4 * i], st.ql[a][4 * i + 1]);
                    mma_f16(d, a0, a1, a2, a3, st.qh[a][4 * i], st.qh[a][4 * i + 1]);
                    float d2[4] = {0.f, 0.f, 0.f, 0.f};
                    mma_f16(d2, c0, c1, c2, c3, st.ql[a][4 * i + 2], st.ql[a][4 * i + 3]);
                    mma_f16(d2, c0, c1, c2, c3, st.qh[a][4 * i + 2], st.qh[a][4 * i + 3]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) { s[a][b][e] += d[e]; s2[a][b][e] += d2[e]; }
                } else {
                    mma_f16(s[a][b], a0, a1, a2, a3, st.qh[a][4 * i], st.qh[a][4 * i + 1]);
                    mma_f16(s2[a][b], c0, c1, c2, c3, st.qh[a][4 * i + 2], st.qh[a][4 * i + 3]);
                }
            }
        }
    }
    // ---- s becomes y, score = qn y in base 2, of tokens (block b, half h) and columns 2t, 2t + 1
    float vs[2][2], vz[2][2], ve[2][2], down[2][2];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int tok = b * 16 + h * 8 + r;
            float2 kk = kp[tok];
            const float2 vv = kp[T + tok];
            kk.x *= key_unit;
            vs[b][h] = vv.x;
            vz[b][h] = vv.y - 8.f;
            if constexpr (F32) {
                // the exponent alone, taken out of the weight exactly: the difference that enters the exponential is small
                // wherever the weight counts, and loses nothing to the size of the logarithm
                const int eb = min(max(int((__float_as_uint(vv.x) >> 23) & 255u), 127 - 80), 127 + 80);
                ve[b][h] = __int_as_float(0x4B000000 | eb) - 8388735.f;
                down[b][h] = __int_as_float((254 - eb) << 23);
                vs[b][h] = vv.x * down[b][h];
            } else {
                ve[b][h] = fminf(fmaxf(lg2(fabsf(vv.x)), -80.f), 80.f);
            }
            if (MASKED && (first + tok >= len || !((there >> (2 * b + h)) & 1u))) vs[b][h] = vz[b][h] = 0.f;
#pragma unroll
            for (int a = 0; a < NT; ++a)
#pragma unroll
                for (int e = 0; e < 2; ++e) s[a][b][2 * h + e] = kk.x * fmaf(kCentre - kk.y, st.qr[a][e], s[a][b][2 * h + e] + s2[a][b][2 * h + e]);
        }
    auto hidden = [&](int b, int h, int a, int e) {
        const int tok = first + b * 16 + h * 8 + r;
        return MASKED && (tok >= len || tok >= st.limit[a][e] || !((there >> (2 * b + h)) & 1u));
    };
    uint32_t ph[NT][4], pl[NT][F32 ? 4 : 1];               // weights as B operands of the second product
#pragma unroll
    for (int a = 0; a < NT; ++a) {
        float m[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            m[e] = -INFINITY;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float x = fmaf(s[a][b][2 * h + e], st.qn[a][e], ve[b][h]);
                    m[e] = fmaxf(m[e], hidden(b, h, a, e) ? -INFINITY : x);
                }
        }
        // the reference moves only when a weight would pass 2^kSlack times its place
        if (__any_sync(0xffffffffu, m[0] > st.top[a][0] + st.room || m[1] > st.top[a][1] + st.room)) {
            float fix[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float x = m[e];
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                x = fmaxf(x - kPlace, st.top[a][e]);
                fix[e] = x == -INFINITY ? 1.f : ex2(st.top[a][e] - x);
                st.top[a][e] = x;
                st.l[a][e] *= fix[e];
                st.zs[a][e] *= fix[e];
            }
            auto large = [](float x) { return fabsf(x) >= kLargeScore && x != -INFINITY; };
            if (__any_sync(0xffffffffu, large(st.top[a][0]) || large(st.top[a][1]))) st.room = kPlace;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) st.o[a][i][e] *= fix[e & 1];
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float at = MASKED && st.top[a][e] == -INFINITY ? 0.f : st.top[a][e];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // a hidden key's parameters may be anything
                    const bool gone = hidden(b, h, a, e);
                    const float x = fmaf(s[a][b][2 * h + e], st.qn[a][e], -at);
                    const float pw = gone ? 0.f : ex2(F32 ? x + ve[b][h] : x);       // (large scores would swallow ve beside the reference)
                    const float w = gone ? 0.f : pw * vs[b][h];
                    st.l[a][e] = F32 ? fmaf(pw, down[b][h], st.l[a][e]) : st.l[a][e] + pw;
                    st.zs[a][e] = gone ? st.zs[a][e] : fmaf(w, vz[b][h], st.zs[a][e]);
                    s[a][b][2 * h + e] = w;
                }
        }
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float w0 = s[a][b][2 * h], w1 = s[a][b][2 * h + 1];
                const uint32_t hi = pack2(w0, w1);
                ph[a][2 * b + h] = transpose8(hi);
                if (F32) {
                    const float2 f = unpack2(hi);
                    pl[a][2 * b + h] = transpose8(pack2(w0 - f.x, w1 - f.y));
                }
            }
    }
    // ---- O^T += V^T P^T.  The transposing load pairs a 16-bit unit (4 channels) of two tokens in a register: lane (r, t)
    // gets channels 32 g + 4 r .. + 3 of tokens 2t, 2t + 1; two of them make an m16 tile's rows r and r + 8
    const int lane = 4 * r + t;
    const uint8_t* mine = vc + ((lane >> 3 & 1) * 8 + (lane & 7)) * (D / 2) + (lane >> 4) * 16;
#pragma unroll
    for (int g = 0; g < D / 32; g += 2) {
        uint32_t x[2][4];
        load_units(mine + g * 16, x[0]);
        load_units(mine + 16 * (D / 2) + g * 16, x[1]);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                const int m = 2 * (g + i) + z;
                float sum[NT][4];                          // float32: the step's share by itself, added to the rest with rounding
                if (F32)
#pragma unroll
                    for (int a = 0; a < NT; ++a)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum[a][e] = 0.f;
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const uint32_t y0 = z ? x[b][2 * i] >> 8 : x[b][2 * i], y1 = z ? x[b][2 * i + 1] >> 8 : x[b][2 * i + 1];
                    const uint32_t v0 = codes2<true>(y0, false), v1 = codes2<true>(y0, true), v2 = codes2<true>(y1, false), v3 = codes2<true>(y1, true);
#pragma unroll
                    for (int a = 0; a < NT; ++a) {
                        if constexpr (F32) {
                            mma_f16(sum[a], v0, v1, v2, v3, pl[a][2 * b], pl[a][2 * b + 1]);
                            mma_f16(sum[a], v0, v1, v2, v3, ph[a][2 * b], ph[a][2 * b + 1]);
                        } else {
                            mma_f16(st.o[a][m], v0, v1, v2, v3, ph[a][2 * b], ph[a][2 * b + 1]);
                        }
                    }
                }
                if (F32)
#pragma unroll
                    for (int a = 0; a < NT; ++a)
#pragma unroll
                        for (int e = 0; e < 4; ++e) st.o[a][m][e] += sum[a][e];
            }
    }
}

template <typename QT, int D, int NT>
__global__ void __launch_bounds__(kThreads, Shape<D, NT, sizeof(QT) == 4>::CTAS)
kv_split_kernel(Cache c, Plan p, const QT* __restrict__ q, int64_t q_stride, QT* __restrict__ out, int64_t out_stride, float scale,
                int causal, float* __restrict__ lse, float* __restrict__ part_o, float2* __restrict__ part_ml, Record* __restrict__ record,
                int* status) {
    constexpr bool F32 = sizeof(QT) == 4;
    using S = Shape<D, NT, F32>;
    constexpr int R = S::R, HALF = T * (D / 2);
    extern __shared__ __align__(128) uint8_t smem[];
    uint8_t* merge = smem + S::STAGES * S::STAGE;
    __shared__ uint64_t s_full[S::STAGES], s_empty[S::STAGES];
    __shared__ uint32_t s_pieces[S::STAGES];
    __shared__ int64_t s_plan[kThreads / 32 + 2];
    __shared__ int s_abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::STAGES; ++i) {
            ptx::mbar_init(&s_full[i], 1);
            ptx::mbar_init(&s_empty[i], kWarps);
        }
        s_abort = 0;
        ptx::fence_barrier_init();
        ptx::fence_proxy_async_smem();
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");     // launched as a dependent: nothing above touched global memory
    int seq;
    int64_t before;
    const int64_t total = locate(p, s_plan, blockIdx.x, gridDim.x, seq, before);
    const Shares shares(total, gridDim.x);
    const int64_t begin = shares.begin(blockIdx.x), end = shares.begin(blockIdx.x + 1);
    const int piece_log2 = min(p.b.page_log2, 7);
    const uint32_t all_pieces = piece_log2 == 4 ? 0xffffffffu : (1u << (4 * (T >> piece_log2))) - 1;
    if (threadIdx.x == 0) record[blockIdx.x].rows = 0;
    if (begin >= end) return;
    const Abort ab{&s_abort, status};
    Walk walk{p, begin, end, before, seq, causal != 0};
    Part it;
    int sg = 0;                                            // pipeline stage and the parity of its turn
    uint32_t turn = 0;
    auto advance = [&]() {
        if (++sg == S::STAGES) { sg = 0; turn ^= 1; }
    };

    if (warp == kWarps) {
        // ---------------------------------------------------------------- producer: lane = 4 * piece + array
        // The page ids of 32 pieces ahead are held across the lanes, and the 32 behind those are on their way: a load from
        // the table in front of every tile's copies would cost the tile its latency.
        const int piece = lane >> 2, array = lane & 3, log2p = p.b.page_log2, per_tile = T >> piece_log2;
        const uint32_t bytes = uint32_t(array & 1 ? 8 : D / 2) << piece_log2;
        uint8_t* place = smem + (array == 0 ? 0 : array == 2 ? HALF : array == 1 ? 2 * HALF : 2 * HALF + T * 8) + min(piece, per_tile - 1) * bytes;
        const uint8_t* source = array == 0 ? c.kc : array == 2 ? c.vc : reinterpret_cast<const uint8_t*>(array == 1 ? c.kp : c.vp);
        const int row_bytes = array & 1 ? 8 : D / 2;
        int issued = 0;
        bool ok = true;
        while (ok && walk.next(it)) {
            const int32_t* row = p.b.table + int64_t(it.s) * p.b.width;
            const int pieces = int((unsigned(it.keys) + (1u << piece_log2) - 1) >> piece_log2), stop = min(it.tile + it.count, (pieces + per_tile - 1) / per_tile);
            auto page_of = [&](int q) { return q < pieces ? row[(int64_t(q) << piece_log2) >> log2p] : 0; };
            int q0 = it.tile * per_tile, held = page_of(q0 + lane), ahead = page_of(q0 + 32 + lane);
            for (int j = it.tile; j < stop; ++j) {         // tiles that a row of this item sees
                const int q = j * per_tile + piece;
                if (j * per_tile - q0 >= 32) {
                    q0 += 32;
                    held = ahead;
                    ahead = page_of(q0 + 32 + lane);
                }
                const int page = __shfl_sync(0xffffffffu, held, q - q0);
                const bool mine = piece < per_tile && q < pieces, good = mine && page >= 0 && page < c.pages;
                if (mine && !good) raise_page(status);
                const uint32_t got = __ballot_sync(0xffffffffu, good), total_bytes = __reduce_add_sync(0xffffffffu, good ? bytes : 0);
                const int64_t r = c.row(page, it.g, (q << piece_log2) & ((1 << log2p) - 1));
                if (!wait_bounded(&s_empty[sg], turn ^ 1, ab)) { ok = false; break; }
                if (lane == 0) {
                    s_pieces[sg] = got;
                    ptx::mbar_arrive_expect_tx(&s_full[sg], total_bytes);
                }
                __syncwarp();
                if (good) bulk_load(place + sg * S::STAGE, source + r * row_bytes, bytes, &s_full[sg]);
                advance();
                ++issued;
            }
        }
        if (!ok) {                                         // give copies still in flight a bounded chance to land
            for (int j = 0; j < S::STAGES && j < issued; ++j) {
                if (--sg < 0) { sg = S::STAGES - 1; turn ^= 1; }
                const long long t0 = clock64();
                while (!ptx::mbar_try_wait(&s_full[sg], turn) && clock64() - t0 < (1ll << 24)) {}
            }
        }
        return;
    }

    // -------------------------------------------------------------------- consumers
    const int r = lane >> 2, t = lane & 3;
    int scale_e;
    const float scale_m = split_scale(scale, scale_e);
    bool ok = true;                                        // false: a wait ran out; go through the motions without waiting
    while (walk.next(it)) {
        State<D, NT, F32> st;
        int low = 0x7fffffff, top_e = -100, e[NT];         // the fewest keys that a column sees, the largest query's exponent
#pragma unroll
        for (int a = 0; a < NT; ++a) {
            const unsigned rr = unsigned(it.qt) * R + a * 8 + r, i = rr / unsigned(p.group);
            const bool real = int(i) < it.n;
            const QT* row = real ? q + (it.row0 + i) * q_stride + (int64_t(it.g) * p.group + (rr - i * p.group)) * D : nullptr;
            float ratio;
            load_queries<QT, D, F32>(row, t, st.qh[a], st.ql[a], e[a], ratio);
            if (e[a] <= 127) top_e = max(top_e, e[a]);
            const int lim = !real ? 0x7fffffff : !causal ? it.len : max(it.len - it.n + int(i) + 1, 0);
            low = min(low, lim);
#pragma unroll
            for (int e = 0; e < 2; ++e) {                  // column 2t + e is lane group 2t + e
                st.qr[a][e] = __shfl_sync(0xffffffffu, ratio, (2 * t + e) * 4);
                st.limit[a][e] = __shfl_sync(0xffffffffu, lim, (2 * t + e) * 4);
            }
        }
        low = __reduce_min_sync(0xffffffffu, low);
        st.room = kPlace + kSlack;
        // the largest query's factor stays below 2^65, what is above goes to the keys (nothing but for queries of 2^50 and more): left
        // in qn it would pass float32 for the largest queries, and the keys that such queries can have would make subnormal scores
        const int lift = min(max(__reduce_max_sync(0xffffffffu, top_e) + kUnit<F32> + scale_e - 64, 0), 126);
        const float key_unit = scale_m * pow2i(lift);
#pragma unroll
        for (int a = 0; a < NT; ++a) {
            const float unit = pow2(e[a] + kUnit<F32> + scale_e - lift);
#pragma unroll
            for (int x = 0; x < 2; ++x) st.qn[a][x] = __shfl_sync(0xffffffffu, unit, (2 * t + x) * 4);
        }
#pragma unroll
        for (int a = 0; a < NT; ++a) {
#pragma unroll
            for (int e = 0; e < 2; ++e) { st.top[a][e] = -INFINITY; st.l[a][e] = 0.f; st.zs[a][e] = 0.f; }
#pragma unroll
            for (int m = 0; m < S::MT; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) st.o[a][m][e] = 0.f;
        }
        for (int j = it.tile; j < it.tile + it.count; ++j) {
            if (j * T >= it.keys) break;
            if (ok && !wait_bounded(&s_full[sg], turn, ab)) ok = false;
            if (!ok) continue;
            const uint8_t* base = smem + sg * S::STAGE;
            const uint8_t* kc = base + (warp * 32) * (D / 2);
            const uint8_t* vc = kc + HALF;
            const float2* kp = reinterpret_cast<const float2*>(base + 2 * HALF) + warp * 32;
            const int first = j * T + warp * 32;           // token of this warp's row 0
            const uint32_t pieces = s_pieces[sg];
            if (first + 32 <= low && pieces == all_pieces) {
                step<D, NT, F32, false>(st, kc, vc, kp, key_unit, first, it.len, 15u, r, t);
            } else if (first < it.keys) {
                uint32_t there = 0;                        // which 8-token blocks of the 32 tokens lie in pages that exist
#pragma unroll
                for (int b8 = 0; b8 < 4; ++b8) there |= ((pieces >> (4 * ((warp * 32 + b8 * 8) >> piece_log2))) & 1u) << b8;
                step<D, NT, F32, true>(st, kc, vc, kp, key_unit, first, it.len, there, r, t);
            }
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&s_empty[sg]);
            advance();
        }
        // ---- the four warps' states meet
        float* m_top = reinterpret_cast<float*>(merge);    // [warps][R], then [warps][R] sums, [warps][R][OROW] outputs
        float* m_l = m_top + kWarps * R;
        float* m_o = m_l + kWarps * R;
#pragma unroll
        for (int a = 0; a < NT; ++a)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) {
                    st.l[a][e] += __shfl_xor_sync(0xffffffffu, st.l[a][e], x);
                    st.zs[a][e] += __shfl_xor_sync(0xffffffffu, st.zs[a][e], x);
                }
                if (r == 0) {
                    m_top[warp * R + a * 8 + 2 * t + e] = st.top[a][e];
                    m_l[warp * R + a * 8 + 2 * t + e] = st.l[a][e];
                }
                float* row = m_o + (warp * R + a * 8 + 2 * t + e) * S::OROW + 4 * r;
#pragma unroll
                for (int m = 0; m < S::MT; m += 2)
                    *reinterpret_cast<float4*>(row + 16 * m) =
                        make_float4(st.o[a][m][e] - st.zs[a][e], st.o[a][m][2 + e] - st.zs[a][e], st.o[a][m + 1][e] - st.zs[a][e],
                                    st.o[a][m + 1][2 + e] - st.zs[a][e]);
            }
        ptx::named_bar_sync(1, 32 * kWarps);
        const bool whole = it.count == it.tiles;
        if (threadIdx.x == 0 && !whole && it.tile == 0) {
            const int first_row = it.qt * R;
            record[blockIdx.x] = Record{it.row0, first_row, min(R, int(p.qrows(it.n)) - first_row), it.g * p.group,
                                        shares.owner(it.first + kItemCost + it.tiles - 1)};
        }
        const int64_t slot = 2 * int64_t(blockIdx.x) + (it.tile > 0 ? 0 : 1);
        constexpr int PER = D / 4;                         // threads of a row: 4 channels each
        for (int u = threadIdx.x; u < R * PER; u += 32 * kWarps) {
            const int col = u / PER, d4 = (u % PER) * 4;
            const unsigned rr = unsigned(it.qt) * R + col, i = rr / unsigned(p.group);
            if (int(i) >= it.n) continue;
            float m = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) m = fmaxf(m, m_top[w * R + col]);
            const float at = m == -INFINITY ? 0.f : m;
            float sum = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = ex2(m_top[w * R + col] - at);
                sum += f * m_l[w * R + col];
                const float4 x = *reinterpret_cast<const float4*>(m_o + (w * R + col) * S::OROW + d4);
                v[0] += f * x.x; v[1] += f * x.y; v[2] += f * x.z; v[3] += f * x.w;
            }
            if (whole) {
                const int64_t row = it.row0 + i;
                const int head = it.g * p.group + int(rr - i * p.group);
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                QT* dst = out + row * out_stride + int64_t(head) * D + d4;
                if constexpr (F32) {
                    *reinterpret_cast<float4*>(dst) = make_float4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
                } else {
                    const __nv_bfloat162 x = __floats2bfloat162_rn(v[0] * inv, v[1] * inv), y = __floats2bfloat162_rn(v[2] * inv, v[3] * inv);
                    *reinterpret_cast<uint2*>(dst) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
                }
                if (lse && d4 == 0) lse[row * (int64_t(c.heads) * p.group) + head] = sum == 0.f ? -INFINITY : (at + log2f(sum)) * 0.6931471805599453f;
            } else {
                *reinterpret_cast<float4*>(part_o + (slot * R + col) * D + d4) = make_float4(v[0], v[1], v[2], v[3]);
                if (d4 == 0) part_ml[slot * R + col] = make_float2(m, sum);
            }
        }
        ptx::named_bar_sync(1, 32 * kWarps);               // the merge area is free again
    }
}

// Joins the pieces of the items that lay in several shares: CTA (c, row) the given row of the item that began in share c, by
// the record that share's CTA left.  Its four warps take 8 pieces at a time: a lane looks each up, then all loads are in flight.
template <typename QT, int D, int R>
__global__ void __launch_bounds__(kCombineThreads)
kv_combine_kernel(Batch b, int* status, int group, QT* __restrict__ out, int64_t out_stride, float* __restrict__ lse, int q_heads, const float* __restrict__ part_o,
                  const float2* __restrict__ part_ml, const Record* __restrict__ record) {
    constexpr int V = D / 32, W = kCombineThreads / 32;
    __shared__ float s_ml[W][2], s_o[W][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c0 = blockIdx.x, col = blockIdx.y;
    asm volatile("griddepcontrol.wait;" ::: "memory");     // in every CTA: this kernel is not over before the one it depends on
    if (blockIdx.x == gridDim.x - 1 && blockIdx.y == gridDim.y - 1) b.report(status, threadIdx.x, kCombineThreads);
    const Record rec = record[c0];
    if (col >= rec.rows) return;
    float m = -INFINITY, l = 0.f, o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = 0.f;
    for (int base = c0 + warp * 8; base <= rec.last; base += 8 * W) {
        const int cc = base + (lane & 7);
        // the first piece is the last one its CTA left, the others are the first of theirs
        const int64_t at = (2 * int64_t(min(cc, rec.last)) + (cc == c0 ? 1 : 0)) * R + col;
        float2 ml = part_ml[at];
        if (cc > rec.last) ml = make_float2(-INFINITY, 0.f);
        float m2 = ml.x;
        m2 = fmaxf(m2, __shfl_xor_sync(0xffffffffu, m2, 1));
        m2 = fmaxf(m2, __shfl_xor_sync(0xffffffffu, m2, 2));
        m2 = fmaxf(m2, __shfl_xor_sync(0xffffffffu, m2, 4));
        m2 = fmaxf(m2, m);
        const float ref = m2 == -INFINITY ? 0.f : m2, f0 = ex2(m - ref);
        const float f1 = ml.y == 0.f ? 0.f : ml.x == -INFINITY ? 1.f : ex2(ml.x - ref);       // (a NaN sum goes through)
        float v[8][V], f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t a = __shfl_sync(0xffffffffu, at, j);
            f[j] = __shfl_sync(0xffffffffu, f1, j);
#pragma unroll
            for (int i = 0; i < V; ++i) v[j][i] = f[j] != 0.f ? part_o[a * D + lane * V + i] : 0.f;
        }
        l *= f0;
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] *= f0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            l = f[j] != 0.f ? fmaf(f[j], __shfl_sync(0xffffffffu, ml.y, j), l) : l;
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = fmaf(f[j], v[j][i], o[i]);
        }
        m = m2;
    }
    if (lane == 0) { s_ml[warp][0] = m; s_ml[warp][1] = l; }
#pragma unroll
    for (int i = 0; i < V; ++i) s_o[warp][lane * V + i] = o[i];
    __syncthreads();
    m = -INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) m = fmaxf(m, s_ml[w][0]);
    const float ref = m == -INFINITY ? 0.f : m;
    l = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) l += ex2(s_ml[w][0] - ref) * s_ml[w][1];
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int rr = rec.first_row + col, i = rr / group, head = rec.head + (rr - i * group);
    const int64_t row = rec.row0 + i;
    for (int d = threadIdx.x; d < D; d += kCombineThreads) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) v += ex2(s_ml[w][0] - ref) * s_o[w][d];
        out[row * out_stride + int64_t(head) * D + d] = QT(v * inv);
    }
    if (lse && threadIdx.x == 0) lse[row * q_heads + head] = l == 0.f ? -INFINITY : (ref + log2f(l)) * 0.6931471805599453f;
}

// Query rows of an item: 16 when a key head has more than 8 of them, which halves the passes over its keys; float32 and
// 256-channel items of 16 would leave most of their accumulators in local memory.  As it is, bytes spilled and read back per thread: 248 / 364
// and 168 / 280 with 16 rows (heads of 128, 64), 32 / 48 with 8 at heads of 128, 92 / 152 at 256; float32 8 / 12, 12 / 16 and 768 / 852 at
// heads of 64, 128, 256.  The fifth warp of a CTA is what caps the registers at 168 and 128.
inline int rows_of_item(int head_dim, int dtype, int rows_hint) { return rows_hint > 8 && head_dim <= 128 && dtype == QLLM_BF16 ? 16 : 8; }

template <typename QT, int D, int NT>
int launch(const Cache& c, const Batch& b, const AttnArgs& a, void* workspace, int* status, cudaStream_t st) {
    using S = Shape<D, NT, sizeof(QT) == 4>;
    const int ctas = device_sm_count() * S::CTAS;
    const Plan p{b, c.heads, a.group, NT == 2 ? 4 : 3, S::R, unsigned(a.most_rows)};
    float* part_o = static_cast<float*>(workspace);
    float2* part_ml = reinterpret_cast<float2*>(part_o + size_t(2) * ctas * S::R * D);
    Record* record = reinterpret_cast<Record*>(part_ml + size_t(2) * ctas * S::R);
    constexpr auto kern = &kv_split_kernel<QT, D, NT>;
    QLLM_CUDA_TRY(allow_smem<kern>(S::SMEM));
    QLLM_CUDA_TRY(launch_dependent(kern, dim3(ctas), dim3(kThreads), S::SMEM, st, c, p, static_cast<const QT*>(a.q), a.q_stride,
                                   static_cast<QT*>(a.out), a.out_stride, a.scale, a.causal, a.lse, part_o, part_ml, record, status));
    const int rc = after_launch();
    if (rc != QLLM_OK) return rc;
    const int live = int(std::min<int64_t>(S::R, b.rows * a.group));     // rows that an item can have
    QLLM_CUDA_TRY(launch_dependent(kv_combine_kernel<QT, D, S::R>, dim3(ctas, live), dim3(kCombineThreads), 0, st, b, status, a.group,
                                   static_cast<QT*>(a.out), a.out_stride, a.lse, a.q_heads, static_cast<const float*>(part_o),
                                   static_cast<const float2*>(part_ml), static_cast<const Record*>(record)));
    return after_launch();
}

}  // namespace

namespace kv {

int64_t split_workspace(int head_dim, int dtype, int rows_hint) {
    // three CTAs on every SM at most, two pieces each
    const int64_t ctas = int64_t(3) * device_sm_count();
    return 2 * ctas * rows_of_item(head_dim, dtype, rows_hint) * (head_dim + 2) * 4 + ctas * int64_t(sizeof(Record));
}

int launch_attention_split(const Cache& c, const Batch& b, int head_dim, const AttnArgs& a, int rows_hint, void* workspace, int* status,
                           cudaStream_t st) {
    const int rows = rows_of_item(head_dim, a.dtype, rows_hint);
#define QLLM_KV_SPLIT(QT, D, NT) return launch<QT, D, NT>(c, b, a, workspace, status, st)
    if (a.dtype == QLLM_BF16) {
        if (head_dim == 64) { if (rows == 16) QLLM_KV_SPLIT(__nv_bfloat16, 64, 2); QLLM_KV_SPLIT(__nv_bfloat16, 64, 1); }
        if (head_dim == 128) { if (rows == 16) QLLM_KV_SPLIT(__nv_bfloat16, 128, 2); QLLM_KV_SPLIT(__nv_bfloat16, 128, 1); }
        if (head_dim == 256) QLLM_KV_SPLIT(__nv_bfloat16, 256, 1);
    } else {
        if (head_dim == 64) QLLM_KV_SPLIT(float, 64, 1);
        if (head_dim == 128) QLLM_KV_SPLIT(float, 128, 1);
        if (head_dim == 256) QLLM_KV_SPLIT(float, 256, 1);
    }
#undef QLLM_KV_SPLIT
    return QLLM_ERR_UNSUPPORTED;
}

}  // namespace kv
}  // namespace qllm
