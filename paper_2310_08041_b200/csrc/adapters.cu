// qllm_adapters_add: low-rank adapters of many requests beside a shared projection,
//
//   out[m] = base[m] + scale[a] B_a (A_a x[m])     for every row m of sequence s, a = adapter[s],
//
// A_a [rank][K], B_a [N][rank] in bf16, all sequences of a packed batch in one launch.
//
// Rows are grouped by adapter: every CTA counts the rows of each adapter (as many integers as there are sequences, from L2) and finds
// its tile, up to T rows of one adapter, wherever in the batch they lie.  So an adapter's weights are read once per T rows, not once per
// sequence, and nothing is sorted or kept between calls.  A cluster of CTAs owns a tile: each takes a part of K in the first
// product, the parts are added over distributed shared memory (in a fixed order), each takes a part of N in the second.
//
// Both products run on the warp-level MMA (m16n8k16: rows x ranks and rows x columns) with operands straight from global memory to
// registers: the order of the summed index is free as long as both operands agree, so a lane's 16 bytes, 8 neighbouring k, serve as the
// two k pairs of two MMAs, and every load is a full sector.  No element is loaded twice by a CTA: in the first product the warps
// split K, in the second N.  The columns of an MMA's 8-wide tile are dealt out so that a lane ends up with 8 neighbouring columns of out.
//
// Precision: sums in float32.  x and the weights are exact operands (float32 x as three bf16 parts of 8 bits each); the sums over K
// are split into two bf16 parts (16 bits) for bf16 outputs, three (24 bits) for float32 ones, before they multiply B.
#include <cuda_bf16.h>

#include <algorithm>

#include "common.h"
#include "kv_cache.cuh"
#include "ptx_sm100.cuh"

namespace qllm {
namespace {

struct AdapterArgs {
    const __nv_bfloat16 *A, *B;
    const float* scale;
    const int32_t* rank;                                   // null: max_rank
    int slots, max_rank, K, N;
    const int32_t *start, *adapter;
    int seqs, cluster;
    int64_t rows;
    const void *x, *base;
    void* out;
    int64_t x_stride, base_stride, out_stride;
    int* status;
    // row ranges, cut to what exists
    __device__ __forceinline__ int first(int s) const { return int(min(max(int64_t(start[s]), int64_t(0)), rows)); }
    __device__ __forceinline__ int count(int s) const { return max(first(s + 1) - first(s), 0); }
    // the group a sequence's rows belong to: its adapter, `slots` for none, -1 for rows that stay as they are
    __device__ __forceinline__ int group(int s) const {
        const int a = adapter[s];
        return a >= 0 && a < slots ? a : base == out ? -1 : slots;
    }
    __device__ __forceinline__ int rank_of(int a) const { return a >= slots ? 0 : rank ? min(max(rank[a], 0), max_rank) : max_rank; }
};

constexpr int kThreads = 256, kWarps = 8;

// exclusive prefix sum over the CTA's threads; total for everyone.  red: 8 ints
__device__ __forceinline__ int block_scan(int v, int* red, int& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int p = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int n = __shfl_up_sync(0xffffffffu, p, o);
        if (lane >= o) p += n;
    }
    __syncthreads();                                       // red may still be read from the last call
    if (lane == 31) red[warp] = p;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += red[w];
        total += red[w];
    }
    return before + p - v;
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// the upper halves of two floats as a bf16 pair (low element first): truncation, 8 bits of each
__device__ __forceinline__ uint32_t upper(float lo, float hi) { return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632); }
__device__ __forceinline__ uint32_t rounded(float lo, float hi) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&b);
}
__device__ __forceinline__ float rest(float f) { return f - __uint_as_float(__float_as_uint(f) & 0xFFFF0000u); }

// 8 neighbouring values of a row as MMA operand words: P parts
template <typename XT>
struct Operand;
template <>
struct Operand<__nv_bfloat16> {
    static constexpr int kParts = 1;
    uint4 v;
    __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = __ldg(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void split(uint32_t (&w)[1][4]) const { w[0][0] = v.x; w[0][1] = v.y; w[0][2] = v.z; w[0][3] = v.w; }
};
template <>
struct Operand<float> {
    static constexpr int kParts = 3;                       // 8 + 8 + 8 bits: all of a float32
    float4 a, b;
    __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void load(const float* p) {
        a = __ldg(reinterpret_cast<const float4*>(p));
        b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    }
    __device__ __forceinline__ void split(uint32_t (&w)[3][4]) const {
        float f[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int p = 0; p < 3; ++p)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                w[p][k] = upper(f[2 * k], f[2 * k + 1]);
                f[2 * k] = rest(f[2 * k]);
                f[2 * k + 1] = rest(f[2 * k + 1]);
            }
    }
};

// 8 neighbouring values of base / out (plain loads: out may be base)
template <typename T>
struct Cells;
template <>
struct Cells<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void add_store(__nv_bfloat16* p, const float (&d)[8]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        uint32_t o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(__uint_as_float(w[k] << 16) + d[2 * k], __uint_as_float(w[k] & 0xFFFF0000u) + d[2 * k + 1]);
            o[k] = *reinterpret_cast<const uint32_t*>(&b);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(o[0], o[1], o[2], o[3]);
    }
};
template <>
struct Cells<float> {
    float4 a, b;
    __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void load(const float* p) { a = reinterpret_cast<const float4*>(p)[0]; b = reinterpret_cast<const float4*>(p)[1]; }
    __device__ __forceinline__ void add_store(float* p, const float (&d)[8]) const {
        reinterpret_cast<float4*>(p)[0] = make_float4(a.x + d[0], a.y + d[1], a.z + d[2], a.w + d[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(b.x + d[4], b.y + d[5], b.z + d[6], b.w + d[7]);
    }
};

__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void st_cluster2(uint32_t addr, uint32_t a, uint32_t b) {
    asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(a), "r"(b) : "memory");
}

template <typename T, int MT, int RN>
struct Layout {
    static constexpr int kTokens = 16 * MT, kRank = 8 * RN;
    static constexpr int kStride = kRank + 8;              // floats / bf16 of a row: rows of a fragment in different banks
    static constexpr int kParts = sizeof(T) == 2 ? 2 : 3;  // of the sums over K
    static constexpr int kPart = kTokens * kStride * 4;    // one warp's sums; the first is reused for the CTA's
    static constexpr int kInner = kTokens * kStride * 2;   // one part of the tile's sums
    // the counts of all adapters, later the warps' sums
    static __host__ __device__ constexpr int first_area(int slots) { return kWarps * kPart > (slots + 4) / 4 * 16 ? kWarps * kPart : (slots + 4) / 4 * 16; }
    static constexpr int bytes(int slots) { return first_area(slots) + kPart + kParts * kInner; }
};

template <typename T, int MT, int RN>
__global__ void __launch_bounds__(kThreads)
adapters_add_kernel(const AdapterArgs p) {
    using Lay = Layout<T, MT, RN>;
    constexpr int kT = Lay::kTokens, kR = Lay::kRank, kS = Lay::kStride, kParts = Lay::kParts;
    constexpr int kQ = kR >= 32 ? 4 : 2;                   // words of a lane's piece of k in the second product
    constexpr int kSteps = kR >= 32 ? kR / 32 : 1;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int s_red[kWarps], s_item[3], s_rows[kT];
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5, g = lane >> 2, q = lane & 3;
    const int cl = p.cluster, part = int(blockIdx.x) % cl, tile = int(blockIdx.x) / cl;
    asm volatile("griddepcontrol.wait;" ::: "memory");     // launched as a dependent

    // ---- the tile's adapter and rows
    int* counts = reinterpret_cast<int*>(smem);
    for (int i = t; i <= p.slots; i += kThreads) counts[i] = 0;
    if (t < kT) s_rows[t] = -1;
    __syncthreads();
    for (int s = t; s < p.seqs; s += kThreads) {
        const int n = p.count(s), a = p.group(s);
        if (n > 0 && a >= 0) atomicAdd(counts + a, n);
        if (blockIdx.x == 0) {
            const int b0 = p.start[s], b1 = p.start[s + 1], ad = p.adapter[s];
            if (b0 < 0 || b1 < b0 || b1 > p.rows || ad >= p.slots || (ad >= 0 && p.rank && (p.rank[ad] < 0 || p.rank[ad] > p.max_rank)))
                kv::raise_page(p.status);
        }
    }
    __syncthreads();
    int total;
    {
        const int per = (p.slots + kThreads) / kThreads, g0 = t * per, g1 = min(g0 + per, p.slots + 1);
        int tiles = 0;
        for (int i = g0; i < g1; ++i) tiles += (counts[i] + kT - 1) / kT;
        int at = block_scan(tiles, s_red, total);
        if (tile >= at && tile < at + tiles)
            for (int i = g0; i < g1; ++i) {
                const int n = (counts[i] + kT - 1) / kT;
                if (tile >= at && tile < at + n) { s_item[0] = i; s_item[1] = (tile - at) * kT; s_item[2] = counts[i]; }
                at += n;
            }
    }
    __syncthreads();
    if (tile >= total) return;                             // the same in all CTAs of a cluster
    const int slot = s_item[0], from = s_item[1], cnt = min(s_item[2] - from, kT);
    {
        const int per = (p.seqs + kThreads - 1) / kThreads, s0 = min(t * per, p.seqs), s1 = min(s0 + per, p.seqs);
        int mine = 0, all;
        for (int s = s0; s < s1; ++s) mine += p.group(s) == slot ? p.count(s) : 0;
        int at = block_scan(mine, s_red, all) - from;      // of the tile's first row
        if (mine > 0 && at < kT && at + mine > 0)
            for (int s = s0; s < s1; ++s) {
                if (p.group(s) != slot) continue;
                const int n = p.count(s), f = p.first(s);
                for (int i = max(0, -at); i < n && at + i < kT; ++i) s_rows[at + i] = f + i;
                at += n;
            }
    }
    __syncthreads();
    const int rank = p.rank_of(slot), mtiles = (cnt + 15) / 16, rtiles = (rank + 7) / 8;

    float* s_part = reinterpret_cast<float*>(smem);
    float* s_sum = reinterpret_cast<float*>(smem + Lay::first_area(p.slots));
    __nv_bfloat16* s_inner = reinterpret_cast<__nv_bfloat16*>(s_sum + kT * kS);

    if (rank > 0) {
        // ---- first product: sums over this CTA's part of K, the warps taking 32 columns in turn
        float acc[MT][RN][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < RN; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][j][i] = 0.f;
        const T* xp[MT][2];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = s_rows[16 * m + 8 * h + g];
                xp[m][h] = static_cast<const T*>(p.x) + (row < 0 ? int64_t(max(s_rows[0], 0)) : int64_t(row)) * p.x_stride + 8 * q;
            }
        const __nv_bfloat16* ap = p.A + (int64_t(slot) * p.max_rank + g) * p.K + 8 * q;
        const int units = (p.K + 31) / 32, u1 = int(int64_t(units) * (part + 1) / cl);
        constexpr int kP = Operand<T>::kParts;
#pragma unroll 2
        for (int u = int(int64_t(units) * part / cl) + warp; u < u1; u += kWarps) {
            const bool in = 32 * u + 8 * q < p.K;
            Operand<T> xv[MT][2];
            uint4 av[RN];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    xv[m][h].zero();
                    if (in && m < mtiles) xv[m][h].load(xp[m][h] + 32 * u);
                }
#pragma unroll
            for (int j = 0; j < RN; ++j) {
                av[j] = make_uint4(0, 0, 0, 0);
                if (in && 8 * j + g < rank) av[j] = __ldg(reinterpret_cast<const uint4*>(ap + int64_t(8 * j) * p.K + 32 * u));
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                if (m >= mtiles) break;
                uint32_t w0[kP][4], w1[kP][4];
                xv[m][0].split(w0);
                xv[m][1].split(w1);
#pragma unroll
                for (int j = 0; j < RN; ++j) {
                    if (j >= rtiles) break;
#pragma unroll
                    for (int k = 0; k < kP; ++k) {
                        mma_bf16(acc[m][j], w0[k][0], w1[k][0], w0[k][1], w1[k][1], av[j].x, av[j].y);
                        mma_bf16(acc[m][j], w0[k][2], w1[k][2], w0[k][3], w1[k][3], av[j].z, av[j].w);
                    }
                }
            }
        }
        // ---- the warps' sums, then the cluster's: CTA `part` adds every cl-th group of four and hands it to all
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            if (m >= mtiles) break;
#pragma unroll
            for (int j = 0; j < RN; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    *reinterpret_cast<float2*>(s_part + warp * kT * kS + (16 * m + 8 * h + g) * kS + 8 * j + 2 * q) = make_float2(acc[m][j][2 * h], acc[m][j][2 * h + 1]);
        }
        __syncthreads();
        for (int e = t; e < cnt * (kR / 4); e += kThreads) {
            const int at = e / (kR / 4) * kS + e % (kR / 4) * 4;
            float4 s = *reinterpret_cast<const float4*>(s_part + at);
#pragma unroll
            for (int w = 1; w < kWarps; ++w) {
                const float4 o = *reinterpret_cast<const float4*>(s_part + w * kT * kS + at);
                s.x += o.x; s.y += o.y; s.z += o.z; s.w += o.w;
            }
            *reinterpret_cast<float4*>(s_sum + at) = s;
        }
        __syncwarp();
        if (cl > 1) ptx::cluster_sync(); else __syncthreads();
        const float scale = p.scale[slot];
        const uint32_t sum_addr = ptx::smem_addr(s_sum), inner_addr = ptx::smem_addr(s_inner);
        for (int e = part + cl * t; e < cnt * (kR / 4); e += cl * kThreads) {
            const int at = e / (kR / 4) * kS + e % (kR / 4) * 4;
            float f[4] = {0.f, 0.f, 0.f, 0.f};
            for (int c = 0; c < cl; ++c) {
                const float4 o = ld_cluster4(ptx::map_to_cta(sum_addr + at * 4, c));
                f[0] += o.x; f[1] += o.y; f[2] += o.z; f[3] += o.w;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] *= scale;
            uint32_t w[kParts][2];
#pragma unroll
            for (int k = 0; k < kParts; ++k) {
                w[k][0] = k + 1 < kParts ? upper(f[0], f[1]) : rounded(f[0], f[1]);
                w[k][1] = k + 1 < kParts ? upper(f[2], f[3]) : rounded(f[2], f[3]);
#pragma unroll
                for (int i = 0; i < 4; ++i) f[i] = rest(f[i]);
            }
            for (int c = 0; c < cl; ++c)
#pragma unroll
                for (int k = 0; k < kParts; ++k) st_cluster2(ptx::map_to_cta(inner_addr + (k * kT * kS + at) * 2, c), w[k][0], w[k][1]);
        }
        __syncwarp();
        if (cl > 1) ptx::cluster_sync(); else __syncthreads();
    }

    // ---- second product: this CTA's part of N, 32 columns a warp
    uint32_t mask[kSteps][kQ];                             // entries of B beyond the rank count for nothing, whatever they are
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int i = 0; i < kQ; ++i) {
            const int k = 32 * s + 2 * kQ * q + 2 * i;
            mask[s][i] = (k < rank ? 0xFFFFu : 0u) | (k + 1 < rank ? 0xFFFF0000u : 0u);
        }
    const T* base = static_cast<const T*>(p.base);
    T* out = static_cast<T*>(p.out);
    const int units = (p.N + 31) / 32, v1 = int(int64_t(units) * (part + 1) / cl);
    for (int v = int(int64_t(units) * part / cl) + warp; v < v1; v += kWarps) {
        const int col = 32 * v + 8 * q;
        uint32_t bw[4][kSteps][kQ];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int n = 32 * v + 8 * (g >> 1) + 2 * j + (g & 1);
            const __nv_bfloat16* bp = p.B + (int64_t(slot) * p.N + n) * p.max_rank + 2 * kQ * q;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                if constexpr (kQ == 4) {
                    uint4 w = make_uint4(0, 0, 0, 0);
                    if (n < p.N && 32 * s + 8 * q < rank) w = __ldg(reinterpret_cast<const uint4*>(bp + 32 * s));
                    bw[j][s][0] = w.x & mask[s][0]; bw[j][s][1] = w.y & mask[s][1];
                    bw[j][s][2] = w.z & mask[s][2]; bw[j][s][3] = w.w & mask[s][3];
                } else {
                    uint2 w = make_uint2(0, 0);
                    if (n < p.N && 4 * q < rank) w = __ldg(reinterpret_cast<const uint2*>(bp));
                    bw[j][s][0] = w.x & mask[s][0]; bw[j][s][1] = w.y & mask[s][1];
                }
            }
        }
        Cells<T> cell[MT][2];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int i = 16 * m + 8 * h + g, row = s_rows[i];
                cell[m][h].zero();
                if (base && i < cnt && row >= 0 && col < p.N) cell[m][h].load(base + int64_t(row) * p.base_stride + col);
            }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            if (m >= mtiles) break;
            float acc[4][4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
            if (rank > 0) {
#pragma unroll
                for (int k = 0; k < kParts; ++k)
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) {
                        if (32 * s >= rank) break;
                        const __nv_bfloat16* hp = s_inner + k * kT * kS + (16 * m + g) * kS + 32 * s + 2 * kQ * q;
                        uint32_t w0[kQ], w1[kQ];
                        if constexpr (kQ == 4) {
                            const uint4 a = *reinterpret_cast<const uint4*>(hp), b = *reinterpret_cast<const uint4*>(hp + 8 * kS);
                            w0[0] = a.x; w0[1] = a.y; w0[2] = a.z; w0[3] = a.w;
                            w1[0] = b.x; w1[1] = b.y; w1[2] = b.z; w1[3] = b.w;
                        } else {
                            const uint2 a = *reinterpret_cast<const uint2*>(hp), b = *reinterpret_cast<const uint2*>(hp + 8 * kS);
                            w0[0] = a.x; w0[1] = a.y;
                            w1[0] = b.x; w1[1] = b.y;
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int i = 0; i < kQ; i += 2) mma_bf16(acc[j], w0[i], w1[i], w0[i + 1], w1[i + 1], bw[j][s][i], bw[j][s][i + 1]);
                    }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int i = 16 * m + 8 * h + g, row = s_rows[i];
                const float d[8] = {acc[0][2 * h], acc[0][2 * h + 1], acc[1][2 * h], acc[1][2 * h + 1],
                                    acc[2][2 * h], acc[2][2 * h + 1], acc[3][2 * h], acc[3][2 * h + 1]};
                if (i < cnt && row >= 0 && col < p.N) cell[m][h].add_store(out + int64_t(row) * p.out_stride + col, d);
            }
        }
    }
}

template <typename T, int MT, int RN>
int launch_tiles(AdapterArgs p, cudaStream_t st) {
    using Lay = Layout<T, MT, RN>;
    const int64_t tiles = p.rows / Lay::kTokens + std::min(p.seqs, p.slots + 1);
    const int bytes = Lay::bytes(p.slots), sms = device_sm_count();
    // as many CTAs to a tile as keep the launch near two CTAs on every SM
    p.cluster = 8;
    while (p.cluster > 1 && tiles * p.cluster > 2 * sms) p.cluster /= 2;
    const cudaError_t e = allow_smem<adapters_add_kernel<T, MT, RN>>(Lay::bytes(8192));
    if (e != cudaSuccess) return cuda_fail(e);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(tiles * p.cluster));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = size_t(bytes);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = unsigned(p.cluster);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const cudaError_t r = cudaLaunchKernelEx(&cfg, adapters_add_kernel<T, MT, RN>, p);
    return r == cudaSuccess ? after_launch() : cuda_fail(r);
}

template <typename T>
int launch_adapters(const AdapterArgs& p, cudaStream_t st) {
    // tiles of 16 rows while groups are that small on average
    const bool few = p.rows <= int64_t(16) * std::min(p.seqs, p.slots + 1);
    if (p.max_rank <= 16) return few ? launch_tiles<T, 1, 2>(p, st) : launch_tiles<T, 4, 2>(p, st);
    if (p.max_rank <= 32) return few ? launch_tiles<T, 1, 4>(p, st) : launch_tiles<T, 4, 4>(p, st);
    if (p.max_rank <= 64) return few ? launch_tiles<T, 1, 8>(p, st) : launch_tiles<T, 4, 8>(p, st);
    return few ? launch_tiles<T, 1, 16>(p, st) : launch_tiles<T, 2, 16>(p, st);
}

int check_rows(const void* p, int64_t stride, int width, int dtype) {
    if (stride < width) return QLLM_ERR_SHAPE;
    return aligned16(p) && stride * (dtype == QLLM_BF16 ? 2 : 4) % 16 == 0 ? QLLM_OK : QLLM_ERR_ALIGN;
}

}  // namespace
}  // namespace qllm

extern "C" int qllm_adapters_add(const qllm_adapters_t* ad, const void* x, int64_t x_stride, const void* base, int64_t base_stride, void* out,
                                 int64_t out_stride, int dtype, const int32_t* q_start, const int32_t* adapter, int seqs, int64_t rows, void* stream) {
    using namespace qllm;
    if (!dtype_ok(dtype)) return QLLM_ERR_DTYPE;
    if (!ad) return QLLM_ERR_NULL;
    if (ad->slots <= 0 || ad->max_rank <= 0 || ad->K <= 0 || ad->N <= 0 || seqs < 0 || rows < 0) return QLLM_ERR_SHAPE;
    if (ad->slots > 8192 || ad->max_rank > 128 || ad->max_rank % 8 || ad->K % 8 || ad->N % 8 || seqs > (1 << 20) || rows > (int64_t(1) << 30))
        return QLLM_ERR_UNSUPPORTED;
    if (rows == 0 || seqs == 0) return QLLM_OK;
    if (!ad->A || !ad->B || !ad->scale || !x || !out || !q_start || !adapter) return QLLM_ERR_NULL;
    if (!aligned16(ad->A) || !aligned16(ad->B)) return QLLM_ERR_ALIGN;
    int rc = check_rows(x, x_stride, ad->K, dtype);
    if (rc == QLLM_OK && base) rc = check_rows(base, base_stride, ad->N, dtype);
    if (rc == QLLM_OK) rc = check_rows(out, out_stride, ad->N, dtype);
    if (rc != QLLM_OK) return rc;
    if (base == out && base_stride != out_stride) return QLLM_ERR_SHAPE;
    int* status = device_status_word();
    if (!status) return QLLM_ERR_CUDA;
    const AdapterArgs p{static_cast<const __nv_bfloat16*>(ad->A), static_cast<const __nv_bfloat16*>(ad->B), ad->scale, ad->rank, ad->slots, ad->max_rank,
                        ad->K, ad->N, q_start, adapter, seqs, 1, rows, x, base, out, x_stride, base_stride, out_stride, status};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dtype == QLLM_BF16 ? launch_adapters<__nv_bfloat16>(p, st) : launch_adapters<float>(p, st);
}
