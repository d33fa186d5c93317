// What the kernels of qllm_adapters_add share: the call's arguments, the way from a CTA's number to its rows, the splitting of float32
// numbers into bf16 parts, writes to other CTAs of the cluster.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "common.h"
#include "kv_cache.cuh"
#include "ptx_sm100.cuh"

namespace qllm {
namespace lora {

struct AdapterArgs {
    const __nv_bfloat16 *A, *B;
    const float* scale;
    const int32_t* rank;                                   // null: max_rank
    int slots, max_rank, K, N;
    const int32_t *start, *adapter;
    int seqs, cluster;                                     // CTAs of a tile
    int tile_rows, ring, stage, stages;                    // adapters_tile.cu: rows of a tile, bytes of the ring, of a stage, stages
    int64_t rows;
    const void *x, *base;
    void* out;
    int64_t x_stride, base_stride, out_stride;
    int* status;
    // row ranges, cut to what exists
    __device__ __forceinline__ int first(int s) const { return int(min(max(int64_t(start[s]), int64_t(0)), rows)); }
    __device__ __forceinline__ int count(int s) const { return max(first(s + 1) - first(s), 0); }
    // the group that rows with adapter[s] = a belong to: the adapter, `slots` for none, -1 for rows that stay as they are
    __device__ __forceinline__ int group_of(int a) const { return a >= 0 && a < slots ? a : base == out ? -1 : slots; }
    __device__ __forceinline__ int raw_rank(int a) const { return rank ? rank[a] : max_rank; }
    __device__ __forceinline__ int cut_rank(int r) const { return min(max(r, 0), max_rank); }
};

// Parts of 8 bits in which the sums over K enter the second product: all of a float32.  With two (16 bits) outputs were off by up to 1.4e-5 of
// the adapter's product beside their own rounding (2e-7 with three), which shows where base takes most of that product away, and 0.32 % of the
// outputs of ordinary prompts were not the bf16 number next to the formula's (0.08 %, the order of float32 sums).
constexpr int kSumParts = 3;

// exclusive prefix sum over the CTA's threads; total for everyone.  red: an int for each warp
template <int THREADS>
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
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) before += red[w];
        total += red[w];
    }
    return before + p - v;
}

// the upper halves of two floats as a bf16 pair (low element first): truncation, 8 bits of each
__device__ __forceinline__ uint32_t upper(float lo, float hi) { return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632); }
__device__ __forceinline__ uint32_t rounded(float lo, float hi) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&b);
}
__device__ __forceinline__ float rest(float f) { return f - __uint_as_float(__float_as_uint(f) & 0xFFFF0000u); }

// of a sum over K: an infinity is its first part, whose product with B is the formula's
__device__ __forceinline__ float rest_of_sum(float f) { return fabsf(f) == INFINITY ? 0.f : rest(f); }

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void st_cluster4(uint32_t addr, float4 v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void st_cluster2(uint32_t addr, uint32_t a, uint32_t b) {
    asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(a), "r"(b) : "memory");
}

// bytes of shared memory that find_item uses
__host__ __device__ constexpr int find_bytes(int slots, int threads) { return (slots + 2) / 2 * 16 + 3 * threads * 4; }

// Rows f .. f + n - 1 at place `to` of the tile's list, as far as they fall into it: by one thread.
__device__ __forceinline__ void list_rows(int* s_rows, int T, int to, int n, int f) {
    for (int i = max(0, -to); i < n && to + i < T; ++i) s_rows[to + i] = f + i;
}
// The same by a warp, a run of rows for each lane (n = 0: none): short runs by their lanes, long ones by all lanes one after the other.
__device__ __forceinline__ void list_rows_warp(int* s_rows, int T, int to, int n, int f, int lane) {
    const int first = max(0, -to), last = min(n, T - to);
    if (last - first <= 8)
        for (int i = first; i < last; ++i) s_rows[to + i] = f + i;
    for (uint32_t left = __ballot_sync(0xffffffffu, last - first > 8); left; left &= left - 1) {
        const int who = __ffs(left) - 1, t = __shfl_sync(0xffffffffu, to, who), g = __shfl_sync(0xffffffffu, f, who), e = __shfl_sync(0xffffffffu, last, who);
        for (int i = __shfl_sync(0xffffffffu, first, who) + lane; i < e; i += 32) s_rows[t + i] = g + i;
    }
}

struct Item {
    int slot, cnt, rank;                                   // adapter, rows of the tile, the adapter's rank
};
// The tile's item and its rows (packed row numbers in s_rows, -1 behind the last; T rows to a tile, MOST places).  false: there is no such tile.  Ends with the CTA
// synchronised.  Groups of rows are ordered by adapter, the rows of one by sequence.  As many sequences and adapters as threads take one round of
// loads, after which every warp finds the item for itself from the counts and the first one lists the rows.
// Ranges that increase hold `rows` rows at most.  Others overlap and could sum up to more than an int holds: where rows x seqs allows that,
// a batch with a decreasing range has no tiles.
template <int THREADS, int MOST>
__device__ __forceinline__ bool find_item(const AdapterArgs& p, int tile, int T, uint8_t* area, int* s_red, int* s_item, int* s_rows, Item& item) {
    const int t = threadIdx.x, lane = t & 31, groups = p.slots + 1;
    int* counts = reinterpret_cast<int*>(area);
    int* ranks = counts + groups;
    int* seq_first = reinterpret_cast<int*>(area + (p.slots + 2) / 2 * 16);
    int* seq_rows = seq_first + THREADS;
    int* seq_group = seq_rows + THREADS;
    for (int i = t; i < groups; i += THREADS) counts[i] = 0;
    for (int i = t; i < MOST; i += THREADS) s_rows[i] = -1;
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");     // launched as a dependent: nothing above touched global memory
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const bool vast = p.rows * p.seqs > (int64_t(1) << 30);
    if (p.seqs <= THREADS && groups <= THREADS) {
        const bool on = t < p.seqs;
        const int s = on ? t : 0;
        const int b0 = p.start[s], b1 = p.start[s + 1], ad = p.adapter[s], raw = t < p.slots ? p.raw_rank(t) : 0;
        if (vast && __syncthreads_or(on && b1 < b0)) {
            if (blockIdx.x == 0 && t == 0) kv::raise_page(p.status);
            return false;
        }
        const int f = int(min(max(int64_t(b0), int64_t(0)), p.rows)), n = on ? max(int(min(max(int64_t(b1), int64_t(0)), p.rows)) - f, 0) : 0;
        const int a = n > 0 ? p.group_of(ad) : -1;
        if (a >= 0) atomicAdd(counts + a, n);
        if (t < groups) ranks[t] = p.cut_rank(raw);
        if (blockIdx.x == 0 && on && (b0 < 0 || b1 < b0 || b1 > p.rows || ad >= p.slots)) kv::raise_page(p.status);
        seq_first[t] = f;
        seq_rows[t] = n;
        seq_group[t] = a;
        __syncthreads();
        if (blockIdx.x == 0 && t < p.slots && counts[t] > 0 && raw != ranks[t]) kv::raise_page(p.status);
        const int eachg = (groups + 31) / 32, eachs = (p.seqs + 31) / 32;       // of a lane
        int tiles = 0;
        for (int k = lane * eachg; k < min((lane + 1) * eachg, groups); ++k) tiles += (counts[k] + T - 1) / T;
        int at = tiles;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, at, o);
            if (lane >= o) at += v;
        }
        if (tile >= __shfl_sync(0xffffffffu, at, 31)) return false;
        at -= tiles;
        const bool mine = tile >= at && tile < at + tiles;
        int slot = 0, from = 0;
        if (mine)
            for (int k = lane * eachg; k < min((lane + 1) * eachg, groups); ++k) {
                const int c = (counts[k] + T - 1) / T;
                if (tile >= at && tile < at + c) { slot = k; from = (tile - at) * T; }
                at += c;
            }
        const int who = __ffs(__ballot_sync(0xffffffffu, mine)) - 1;
        slot = __shfl_sync(0xffffffffu, slot, who);
        from = __shfl_sync(0xffffffffu, from, who);
        item.slot = slot;
        item.cnt = min(counts[slot] - from, T);
        item.rank = ranks[slot];
        if (t < 32) {
            const int k0 = lane * eachs, k1 = min(k0 + eachs, p.seqs);
            int have = 0;
            for (int k = k0; k < k1; ++k) have += seq_group[k] == slot ? seq_rows[k] : 0;
            int to = have;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, to, o);
                if (lane >= o) to += v;
            }
            to -= have + from;                             // of the tile's first row
            for (int i = 0; i < eachs; ++i) {
                const int k = k0 + i;
                const bool in = k < k1 && seq_group[k] == slot;
                const int n = in ? seq_rows[k] : 0;
                list_rows_warp(s_rows, T, to, n, in ? seq_first[k] : 0, lane);
                to += n;
            }
        }
    } else {
        // a thread's run of sequences, and of adapters
        const int per = (p.seqs + THREADS - 1) / THREADS, s0 = min(t * per, p.seqs), s1 = min(s0 + per, p.seqs);
        if (vast) {
            bool down = false;
            for (int s = t; s < p.seqs; s += THREADS) down |= p.start[s + 1] < p.start[s];
            if (__syncthreads_or(down)) {
                if (blockIdx.x == 0 && t == 0) kv::raise_page(p.status);
                return false;
            }
        }
        for (int i = t; i < groups; i += THREADS) ranks[i] = i < p.slots ? p.cut_rank(p.raw_rank(i)) : 0;
        for (int s = s0; s < s1; ++s) {
            const int n = p.count(s), b0 = p.start[s], b1 = p.start[s + 1], ad = p.adapter[s], a = p.group_of(ad);
            if (n > 0 && a >= 0) atomicAdd(counts + a, n);
            if (blockIdx.x == 0 && (b0 < 0 || b1 < b0 || b1 > p.rows || ad >= p.slots)) kv::raise_page(p.status);
        }
        __syncthreads();
        if (blockIdx.x == 0)
            for (int i = t; i < p.slots; i += THREADS)
                if (counts[i] > 0 && p.raw_rank(i) != ranks[i]) kv::raise_page(p.status);
        const int each = (groups + THREADS - 1) / THREADS, g0 = min(t * each, groups), g1 = min(g0 + each, groups);
        int tiles = 0, total, have = 0, all;
        for (int i = g0; i < g1; ++i) tiles += (counts[i] + T - 1) / T;
        int at = block_scan<THREADS>(tiles, s_red, total);
        if (tile >= total) return false;
        if (tile >= at && tile < at + tiles)
            for (int i = g0; i < g1; ++i) {
                const int n = (counts[i] + T - 1) / T;
                if (tile >= at && tile < at + n) { s_item[0] = i; s_item[1] = (tile - at) * T; }
                at += n;
            }
        __syncthreads();
        const int slot = s_item[0], from = s_item[1];
        item.slot = slot;
        item.cnt = min(counts[slot] - from, T);
        item.rank = ranks[slot];
        for (int s = s0; s < s1; ++s) have += p.group_of(p.adapter[s]) == slot ? p.count(s) : 0;
        int to = block_scan<THREADS>(have, s_red, all) - from;
        if (have > 0 && to < T && to + have > 0)
            for (int s = s0; s < s1; ++s) {
                if (p.group_of(p.adapter[s]) != slot) continue;
                const int n = p.count(s);
                list_rows(s_rows, T, to, n, p.first(s));
                to += n;
            }
    }
    __syncthreads();
    return true;
}

// Allows a kernel clusters of 16, once per kernel and device.
template <auto Kern>
cudaError_t allow_large_clusters() {
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 64 && (done.load(std::memory_order_relaxed) >> dev & 1)) return cudaSuccess;
    const cudaError_t r = cudaFuncSetAttribute(Kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (r == cudaSuccess && dev < 64) done.fetch_or(uint64_t(1) << dev, std::memory_order_relaxed);
    return r;
}

// bf16 calls on the tensor cores (adapters_tile.cu); few: 16 rows of an adapter or fewer on average
int launch_tiles_tc(const AdapterArgs& p, bool few, cudaStream_t st);

}  // namespace lora
}  // namespace qllm
