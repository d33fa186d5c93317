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
// This kernel serves float32 and what is small in bf16; tensor_cores() below says which, with both sides measured.  What bounds it: latency (one
// token of 4096 -> 12288, rank 16: 5.8 us, of which a launch is 3; 35 rows of float32, 5120 x 5120, rank 32: 9.2 us), and, for larger calls, the
// operand registers, which hold too few loads to keep memory busy (48 to 72 words a lane: kLoadK, kLoadN).
//
// Precision: sums in float32.  x and the weights are exact operands (float32 x as three bf16 parts of 8 bits each); so are the sums over K
// when they multiply B, as three parts.
#include <cuda_bf16.h>

#include <algorithm>

#include "adapters.cuh"

namespace qllm {
namespace {

using namespace lora;

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

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

__device__ __forceinline__ void prefetch_line(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
// Eight groups of warps split K in the first product and N in the second; HM warps of a group take MT tiles of 16 rows each.
constexpr int kGroups = 8;

template <typename T, int MT, int HM, int RN>
struct Shape {
    static constexpr int kThreads = 32 * kGroups * HM, kTokens = 16 * MT * HM, kRank = 8 * RN;
    static constexpr int kStride = kRank + 8;              // floats / bf16 of a row: rows of a fragment in different banks
    static constexpr int kParts = kSumParts;               // of the sums over K
    static constexpr int kPart = kTokens * kStride * 4;    // one group's sums; the CTA's
    static constexpr int kInner = kTokens * kStride * 2;   // one part of the tile's sums
    // the counts and ranks of all adapters, later the groups' sums
    static __host__ __device__ constexpr int first_area(int slots) { return kGroups * kPart > find_bytes(slots, kThreads) ? kGroups * kPart : find_bytes(slots, kThreads); }
    static constexpr bool kAll = MT * HM == 1;             // every CTA adds up all parts of the sums
    static constexpr int kMostLog2 = kAll && RN <= 4 ? 4 : 3;          // CTAs of a cluster: what shared memory holds twice over
    static constexpr int kSum = kPart * (kAll ? 1 << kMostLog2 : 1);
    static constexpr int bytes(int slots) { return first_area(slots) + kSum + kParts * kInner; }
    // pieces of 32 columns that a warp loads before it multiplies: what its registers hold
    static constexpr int kWide = sizeof(T) / 2;
    static constexpr int fit(int regs, int each) { return regs / each >= 4 ? 4 : regs / each >= 1 ? regs / each : 1; }
    static constexpr int kLoadK = fit(RN >= 8 && MT * HM > 1 ? 48 : 72, 8 * MT * kWide + 4 * RN);
    static constexpr int kLoadN = fit(72, 8 * MT * kWide + (RN >= 4 ? 4 * RN : 8));
};

template <typename T, int MT, int HM, int RN>
__global__ void __launch_bounds__(32 * kGroups * HM, HM == 1 && RN <= 8 ? 2 : 1)
adapters_add_kernel(const AdapterArgs p) {
    using S = Shape<T, MT, HM, RN>;
    constexpr int kThreads = S::kThreads, kT = S::kTokens, kR = S::kRank, kS = S::kStride, kParts = S::kParts;
    constexpr int kQ = kR >= 32 ? 4 : 2;                   // words of a lane's piece of k in the second product
    constexpr int kSteps = kR >= 32 ? kR / 32 : 1;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int s_red[kThreads / 32], s_item[4], s_rows[kT];
    const int t = threadIdx.x, lane = t & 31, group = (t >> 5) / HM, m0 = (t >> 5) % HM * MT, g = lane >> 2, q = lane & 3;
    const int cl = p.cluster, tile = int(blockIdx.x) / cl, part = int(blockIdx.x) - tile * cl;
    if (cl > 1) cluster_arrive();                          // waited for before the first write to another CTA's memory: all have started

    // ---- the tile's adapter and rows
    Item item;
    if (!find_item<kThreads, kT>(p, tile, kT, smem, s_red, s_item, s_rows, item)) return;   // the same in all CTAs of a cluster
    const int slot = item.slot, cnt = item.cnt, rank = item.rank;
    const int mtiles = (cnt + 15) / 16 - m0, rtiles = (rank + 7) / 8;      // tiles of rows of this warp, of ranks

    float* s_part = reinterpret_cast<float*>(smem);
    float* s_sum = reinterpret_cast<float*>(smem + S::first_area(p.slots));
    __nv_bfloat16* s_inner = reinterpret_cast<__nv_bfloat16*>(s_sum + S::kSum / 4);
    const __nv_bfloat16* weights = p.B + int64_t(slot) * p.N * p.max_rank;
    const T* base = static_cast<const T*>(p.base);
    T* out = static_cast<T*>(p.out);
    const int nunits = (p.N + 31) / 32, v0 = nunits * part / cl, v1 = nunits * (part + 1) / cl;     // K, N <= 2^20

    // the second product's operands start on their way to L2 under the first one
    const int units = (p.K + 31) / 32, u0 = units * part / cl, u1 = units * (part + 1) / cl;
    if (rank > 0) {
        const int n0 = 32 * v0, n1 = min(32 * v1, p.N);
        if (2 * rank > p.max_rank) {
            const char* from = reinterpret_cast<const char*>(weights + int64_t(n0) * p.max_rank);
            for (int i = 128 * t; i < (n1 - n0) * p.max_rank * 2; i += 128 * kThreads) prefetch_line(from + i);
        } else {
            for (int n = n0 + t; n < n1; n += kThreads) prefetch_line(weights + int64_t(n) * p.max_rank);
        }
    }

    // ---- what the second product reads: this CTA's part of N, the groups taking kLoadN x 32 columns in turn
    constexpr int kLN = S::kLoadN;
    uint32_t bw[kLN][4][kSteps][kQ];
    Cells<T> cell[kLN][MT][2];
    // (every lane loads, as above; entries of B beyond the rank count for nothing, whatever they are: the masks below)
    int brow[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) brow[s] = kQ == 4 ? min(32 * s + 8 * q, max(rank - 1, 0) & ~7) : min(4 * q, max(rank - 1, 0) & ~3);
    const T* bp[MT][2];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = s_rows[16 * (m0 + m) + 8 * h + g];
            bp[m][h] = base + int64_t(row < 0 ? max(s_rows[0], 0) : row) * p.base_stride;
        }
    const auto load_columns = [&](int v) {
#pragma unroll
        for (int l = 0; l < kLN; ++l) {
            if (v + l >= v1) break;
            if (rank > 0) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const __nv_bfloat16* wp = weights + int64_t(min(32 * (v + l) + 8 * (g >> 1) + 2 * j + (g & 1), p.N - 1)) * p.max_rank;
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) {
                        if (s > 0 && 32 * s >= rank) break;
                        if constexpr (kQ == 4) {
                            const uint4 w = __ldg(reinterpret_cast<const uint4*>(wp + brow[s]));
                            bw[l][j][s][0] = w.x; bw[l][j][s][1] = w.y; bw[l][j][s][2] = w.z; bw[l][j][s][3] = w.w;
                        } else {
                            const uint2 w = __ldg(reinterpret_cast<const uint2*>(wp + brow[s]));
                            bw[l][j][s][0] = w.x; bw[l][j][s][1] = w.y;
                        }
                    }
                }
            }
            if (base) {
                const int col = min(32 * (v + l) + 8 * q, p.N - 8);
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (m > 0 && m >= mtiles) break;
                        cell[l][m][h].load(bp[m][h] + col);
                    }
            } else {
#pragma unroll
                for (int m = 0; m < MT; ++m) { cell[l][m][0].zero(); cell[l][m][1].zero(); }
            }
        }
    };

    if (rank > 0) {
        // ---- first product: sums over this CTA's part of K, the groups taking kLoadK x 32 columns in turn
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
                const int row = s_rows[16 * (m0 + m) + 8 * h + g];
                xp[m][h] = static_cast<const T*>(p.x) + int64_t(row < 0 ? max(s_rows[0], 0) : row) * p.x_stride;
            }
        // Every lane loads: where there is no such rank, the last one's row again (those sums are dropped below), behind the last
        // column the last 8 again (zeroed).
        const __nv_bfloat16* ap[RN];
#pragma unroll
        for (int j = 0; j < RN; ++j) ap[j] = p.A + (int64_t(slot) * p.max_rank + min(8 * j + g, rank - 1)) * p.K;
        constexpr int kP = Operand<T>::kParts, kL = S::kLoadK;
        if (mtiles > 0)
            for (int u = u0 + group * kL; u < u1; u += kGroups * kL) {
                Operand<T> xv[kL][MT][2];
                uint4 av[kL][RN];
#pragma unroll
                for (int l = 0; l < kL; ++l) {
                    if (l > 0 && u + l >= u1) break;
                    const int k = min(32 * (u + l) + 8 * q, p.K - 8);
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if (m > 0 && m >= mtiles) break;
                            xv[l][m][h].load(xp[m][h] + k);
                        }
#pragma unroll
                    for (int j = 0; j < RN; ++j) {
                        if (j > 0 && j >= rtiles) break;
                        av[l][j] = __ldg(reinterpret_cast<const uint4*>(ap[j] + k));
                    }
                }
#pragma unroll
                for (int l = 0; l < kL; ++l) {
                    if (l > 0 && u + l >= u1) break;
                    if (32 * (u + l) + 32 > p.K && 32 * (u + l) + 8 * q >= p.K) {
#pragma unroll
                        for (int m = 0; m < MT; ++m) { xv[l][m][0].zero(); xv[l][m][1].zero(); }
#pragma unroll
                        for (int j = 0; j < RN; ++j) av[l][j] = make_uint4(0, 0, 0, 0);
                    }
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        if (m > 0 && m >= mtiles) break;
                        uint32_t w0[kP][4], w1[kP][4];
                        xv[l][m][0].split(w0);
                        xv[l][m][1].split(w1);
#pragma unroll
                        for (int j = 0; j < RN; ++j) {
                            if (j > 0 && j >= rtiles) break;
#pragma unroll
                            for (int k = 0; k < kP; ++k) {
                                mma_bf16(acc[m][j], w0[k][0], w1[k][0], w0[k][1], w1[k][1], av[l][j].x, av[l][j].y);
                                mma_bf16(acc[m][j], w0[k][2], w1[k][2], w0[k][3], w1[k][3], av[l][j].z, av[l][j].w);
                            }
                        }
                    }
                }
            }
        // ---- the groups' sums, then the cluster's: CTA `part` adds every cl-th group of four and hands it to all
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            if (m >= mtiles) break;
#pragma unroll
            for (int j = 0; j < RN; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    *reinterpret_cast<float2*>(s_part + group * kT * kS + (16 * (m0 + m) + 8 * h + g) * kS + 8 * j + 2 * q) = make_float2(acc[m][j][2 * h], acc[m][j][2 * h + 1]);
        }
        load_columns(v0 + group * kLN);                    // under the exchange
        __syncthreads();
        if (cl > 1) cluster_wait();
        // Each CTA adds its groups' sums, in fours.  Small tiles: every CTA hands all of its sums to all CTAs, which add them up, each for
        // itself.  Others: the e-th four goes to CTA e % cl, which adds the cl parts and hands the result to all; one more barrier,
        // a cl-th of the traffic.
        const int fours = cnt * (kR / 4);
        const uint32_t sum_addr = ptx::smem_addr(s_sum), inner_addr = ptx::smem_addr(s_inner);
        const float scale = p.scale[slot];
        for (int e = t; e < fours; e += kThreads) {
            const int at = e / (kR / 4) * kS + e % (kR / 4) * 4;
            float4 s = *reinterpret_cast<const float4*>(s_part + at);
#pragma unroll
            for (int w = 1; w < kGroups; ++w) {
                const float4 o = *reinterpret_cast<const float4*>(s_part + w * kT * kS + at);
                s.x += o.x; s.y += o.y; s.z += o.z; s.w += o.w;
            }
            if constexpr (S::kAll) {
                for (int c = 0; c < cl; ++c) st_cluster4(ptx::map_to_cta(sum_addr + (e * cl + part) * 16, c), s);
            } else {
                st_cluster4(ptx::map_to_cta(sum_addr + ((e & -cl) + part) * 16, e & (cl - 1)), s);
            }
        }
        __syncwarp();
        if (cl > 1) ptx::cluster_sync(); else __syncthreads();
        for (int k = t; S::kAll ? k < fours : part + k * cl < fours; k += kThreads) {
            const int e = S::kAll ? k : part + k * cl, at = e / (kR / 4) * kS + e % (kR / 4) * 4;
            float f[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int c = 0; c < cl; ++c) {
                const float4 o = *reinterpret_cast<const float4*>(s_sum + (k * cl + c) * 4);
                f[0] += o.x; f[1] += o.y; f[2] += o.z; f[3] += o.w;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = e % (kR / 4) * 4 + i < rank ? f[i] * scale : 0.f;
            uint32_t w[kParts][2];
#pragma unroll
            for (int i = 0; i < kParts; ++i) {
                w[i][0] = i + 1 < kParts ? upper(f[0], f[1]) : rounded(f[0], f[1]);
                w[i][1] = i + 1 < kParts ? upper(f[2], f[3]) : rounded(f[2], f[3]);
#pragma unroll
                for (int j = 0; j < 4; ++j) f[j] = rest_of_sum(f[j]);
                if constexpr (S::kAll) {
                    *reinterpret_cast<uint2*>(s_inner + i * kT * kS + at) = make_uint2(w[i][0], w[i][1]);
                } else {
                    for (int c = 0; c < cl; ++c) st_cluster2(ptx::map_to_cta(inner_addr + (i * kT * kS + at) * 2, c), w[i][0], w[i][1]);
                }
            }
        }
        if constexpr (S::kAll) {
            __syncthreads();
        } else {
            __syncwarp();
            if (cl > 1) ptx::cluster_sync(); else __syncthreads();
        }
    } else {
        load_columns(v0 + group * kLN);
    }
    if (mtiles <= 0) return;

    // ---- second product
    uint32_t mask[kSteps][kQ];
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int i = 0; i < kQ; ++i) {
            const int k = 32 * s + 2 * kQ * q + 2 * i;
            mask[s][i] = (k < rank ? 0xFFFFu : 0u) | (k + 1 < rank ? 0xFFFF0000u : 0u);
        }
    for (int v = v0 + group * kLN; v < v1; v += kGroups * kLN) {
        if (v != v0 + group * kLN) load_columns(v);
#pragma unroll
        for (int l = 0; l < kLN; ++l) {
            if (v + l >= v1) break;
            const int col = 32 * (v + l) + 8 * q;
            if (rank > 0) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) {
                        if (s > 0 && 32 * s >= rank) break;
#pragma unroll
                        for (int i = 0; i < kQ; ++i) bw[l][j][s][i] &= mask[s][i];
                    }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                if (m > 0 && m >= mtiles) break;
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
                            if (s > 0 && 32 * s >= rank) break;
                            const __nv_bfloat16* hp = s_inner + k * kT * kS + (16 * (m0 + m) + g) * kS + 32 * s + 2 * kQ * q;
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
                                for (int i = 0; i < kQ; i += 2) mma_bf16(acc[j], w0[i], w1[i], w0[i + 1], w1[i + 1], bw[l][j][s][i], bw[l][j][s][i + 1]);
                        }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int i = 16 * (m0 + m) + 8 * h + g, row = s_rows[i];
                    const float d[8] = {acc[0][2 * h], acc[0][2 * h + 1], acc[1][2 * h], acc[1][2 * h + 1],
                                        acc[2][2 * h], acc[2][2 * h + 1], acc[3][2 * h], acc[3][2 * h + 1]};
                    if (i < cnt && row >= 0 && col < p.N) cell[l][m][h].add_store(out + int64_t(row) * p.out_stride + col, d);
                }
            }
        }
    }
}

template <typename T, int MT, int HM, int RN>
int launch_tiles(AdapterArgs p, cudaStream_t st) {
    using S = Shape<T, MT, HM, RN>;
    constexpr auto kern = adapters_add_kernel<T, MT, HM, RN>;
    const int64_t groups = std::min<int64_t>({p.seqs, p.slots + 1, p.rows}), tiles = groups + (p.rows - groups) / S::kTokens;
    const int bytes = S::bytes(p.slots), sms = device_sm_count();
    // as many CTAs to a tile as keep the launch near two CTAs on every SM
    p.cluster = 1 << S::kMostLog2;
    while (p.cluster > 1 && tiles * p.cluster > (p.cluster == 16 ? sms / 2 : 2 * sms)) p.cluster /= 2;
    QLLM_CUDA_TRY(allow_smem<kern>(S::bytes(8192)));
    if (p.cluster > 8) QLLM_CUDA_TRY(allow_large_clusters<kern>());
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(tiles * p.cluster));
    cfg.blockDim = dim3(S::kThreads);
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
    QLLM_CUDA_TRY(cudaLaunchKernelEx(&cfg, kern, p));
    return after_launch();
}

// Which kernel serves a bf16 call: this file's warp-level MMA with operands straight from memory, or the tensor cores' (adapters_tile.cu), which
// have the longer way to their first byte and stream faster behind it.  Measured with random adapters, us here / there:
//   tiles of many rows  rank 16, 4096 x 4096, rows of one adapter: 256 11.1 / 13.5, 768 11.5 / 14.5, 1024 (16 of this kernel's tiles, of whose clusters
//                       15 fit at once) 21.8 / 15.0; 4 adapters of 300 23 / 16.5, 24 of 20 19.6 / 18.2; 4096 rows, 1024 x 1000: 19.1 / 13.1
//                       rank 32, 8192 x 10240: 24 rows 18.2 / 18.4, 64 22.2 / 18.5, 1024 51 / 25, 24 adapters of 40 38.2 / 36.1, 12 of 100 51 / 34;
//                       5120 x 5120: 64 rows 16.0 / 14.1, 768 18.1 / 16.8
//   few rows each       rank 32, 8192 x 10240: one token 7.3 / 17.7, 96 tokens on 24 adapters 17.3 / 25.8; 4096 x 4096: 6.7 / 12.4, 9.7 / 17.4
//                       rank 64, 8192 x 10240: 13.8 / 11.8, 27 / 18.8; 4096 x 4096: 8.5 / 8.8, 13.9 / 12.7
// (Larger ranks were farther apart: rank 64, 8192 x 10240, 1024 rows 87 / 28; rank 128, 4096 x 4096, 96 tokens 33 / 18, with two parts of the sums.)
bool tensor_cores(const AdapterArgs& p, bool few) {
    const int64_t groups = std::min(p.seqs, p.slots + 1), sides = int64_t(p.K) + p.N;
    if (!few) return p.max_rank > 32 || groups + p.rows / 64 > 15 || (p.max_rank > 16 && p.rows >= 48);
    return p.max_rank > 64 || (p.max_rank > 32 && (sides >= 16384 || groups * sides * p.max_rank >= 8000000));
}

template <typename T>
int launch_adapters(const AdapterArgs& p, cudaStream_t st) {
    // tiles of 16 rows while groups are that small on average
    const bool few = p.rows <= int64_t(16) * std::min(p.seqs, p.slots + 1);
    constexpr bool half = sizeof(T) == 2;                  // (whose larger ranks are the other kernel's)
    if (half && tensor_cores(p, few)) return launch_tiles_tc(p, few, st);
    if (few) {
        if (p.max_rank <= 16) return launch_tiles<T, 1, 1, 2>(p, st);
        if (p.max_rank <= 32) return launch_tiles<T, 1, 1, 4>(p, st);
        if (half || p.max_rank <= 64) return launch_tiles<T, 1, 1, 8>(p, st);
        if constexpr (!half) return launch_tiles<T, 1, 1, 16>(p, st);
    }
    if (p.max_rank <= 16) return launch_tiles<T, 2, 2, 2>(p, st);
    if (half || p.max_rank <= 32) return launch_tiles<T, 2, 2, 4>(p, st);
    if constexpr (!half) return p.max_rank <= 64 ? launch_tiles<T, 2, 2, 8>(p, st) : launch_tiles<T, 2, 1, 16>(p, st);
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
    if (ad->slots > 8192 || ad->max_rank > 128 || ad->max_rank % 8 || ad->K % 8 || ad->N % 8 || ad->K > (1 << 20) || ad->N > (1 << 20) ||
        seqs > (1 << 20) || rows > (int64_t(1) << 30))
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
                        ad->K, ad->N, q_start, adapter, seqs, 1, 0, 0, 0, 0, rows, x, base, out, x_stride, base_stride, out_stride, status};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dtype == QLLM_BF16 ? launch_adapters<__nv_bfloat16>(p, st) : launch_adapters<float>(p, st);
}
