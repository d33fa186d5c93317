// qllm_adapters_add for bf16 on the tensor cores (tcgen05): up to 128 rows of one adapter are the M side of both products,
//
//   D1[rows x ranks] = X A^T over this CTA's part of K,  H = scale * (sum of the cluster's D1),  D2[rows x 128] = H B^T, out = base + D2.
//
// A cluster owns a tile (adapters.cuh finds its rows); each CTA takes a part of K in the first product and a part of N in the second, the
// sums over K are exchanged over distributed shared memory.  Eight warps feed a ring of stages by asynchronous copies of 16 bytes a thread,
// swizzled as the tensor core reads operands (rows of 128 bytes, 16-byte pieces at piece ^ (row & 7)): first 128 columns of A and of the
// tile's rows of x a stage, then, without waiting for the sums, 128 rows of B and 128 columns of base.  Copies fill with zeros what lies behind
// K and, in B, behind the rank, so operands need no masks; rows behind the tile and the rank are whatever is there: they only reach
// sums that are dropped.  Three threads issue the MMAs, each for the places of the ring that are its own; in the second product each of them has a
// team of four warps, a thread for each row of the tile, that reads the sums back from tensor memory, adds them to base where it lies
// and stores the rows of out (a warp's rows are its own: no barrier among warps).  H enters the second product as three bf16 parts, all of its bits.
//
// The rows of a tile and the CTAs of a cluster are chosen together (launch_shape); fewer rows leave the ring more stages.
//
// ROWS: rows of the tile that there is room for.  With 16 (a step's single tokens) the products are transposed, D1[ranks x rows] and
// D2[128 columns x rows]: the weights are the M side, the rows an N of 16.  An MMA's time is that of its operands' bytes from shared memory, and
// 128 rows of which 16 are real would be most of them (96 tokens on 24 adapters of rank 64, 8192 x 10240: 21.2 us so, 19.4 now).
//
// What bounds it.  3792 rows on 9 adapters of rank <= 32, 8192 x 8192 (53 us, 192 MB: 3.6 TB/s; the floor is 29): 0.4 us for 128 columns of the
// first product, the ring's bytes in flight, and up to 1.3 of the second, the instructions of the teams (3900 for 128 x 128 numbers of out), on
// three quarters of the SMs; finding the tile 2.5, first data 2, the exchange 3.7.  The third part of the sums is 1.3 us of the 53 (its MMAs and
// stores); where MMAs are more of the time it is more: 1024 rows of rank 64, 8192 x 10240, 28.2 -> 30.4, of rank 128, 4096 x 4096, 24.8 -> 28.3.  With two
// parts, when they came to 52: two teams with barriers among their warps took 57.3 us; four teams, or the teams' loop unrolled, were slower
// (instruction fetch); the warp-level MMA (adapters.cu) took 63 (some 20 cycles for each m16n8k16 and quarter of an SM).  A step of 96 tokens: the chain
// search, first data, exchange, and 125 SMs for 25 adapters of 5 CTAs.
#include <algorithm>

#include "adapters.cuh"
#include "qgemm_tc_common.cuh"

namespace qllm {
namespace lora {
namespace {

using tc::Abort;
using tc::wait_bounded;

constexpr int kFeeders = 256, kTeam = 128, kTeams = 3, kWorkers = kTeams * kTeam, kIssuers = kTeams, kThreads = kWorkers + 32 * kIssuers + kFeeders, kCols = 128;

template <int R, int ROWS>
struct Shape {
    static constexpr int kBlocks = (R + 63) / 64;          // operand blocks (64 elements of 128 bytes) of a row of B
    static constexpr bool kFew = ROWS == 16;               // transposed products; every CTA adds up all parts of the sums
    // H: the elements of its parts side by side (R of each), few rows: the rows of its parts below one another
    static constexpr int kHBlocks = kFew ? kBlocks : (kSumParts * R + 63) / 64;
    static constexpr int kABlock = R * 128, kBBlock = kCols * 128, kPart = kFew ? ROWS * R * 4 : 0;
    static constexpr int kPitch = kCols * 2 + 16;          // bytes between rows of base: 16-byte accesses of 8 rows in different banks
    static constexpr int kBytes = 223 * 1024, kMostStages = 8;
    // What tiles of `rows` rows leave the ring, and the ring's stages: the fewer rows, the more of them
    static __host__ __device__ constexpr int h_block(int rows) { return (kFew ? kSumParts * ROWS : rows) * 128; }
    static __host__ __device__ constexpr int sum_bytes(int rows) { return kFew ? 8 * ROWS * R * 4 : rows * R * 4 + 8 * 16; }
    static __host__ __device__ constexpr int ring_bytes(int rows) {
        const int deep = kFew ? 0 : (128 - rows) * 128 - sum_bytes(rows);      // H as an operand is read 128 rows deep
        return (kBytes - kHBlocks * h_block(rows) - kPart - sum_bytes(rows) - (deep > 0 ? deep : 0) - 1024) / 1024 * 1024;
    }
    static __host__ __device__ constexpr int stage_bytes(int rows) {
        const int k = 2 * (kABlock + rows * 128), n = kBlocks * kBBlock + rows * kPitch;
        return ((k > n ? k : n) + 1023) / 1024 * 1024;
    }
    static __host__ __device__ constexpr int stages(int rows) {
        const int n = ring_bytes(rows) / stage_bytes(rows);
        return n > kMostStages ? kMostStages : n;
    }
    // rows of a tile at most: with 128 of rank 64 the ring would have two stages instead of three (8 adapters of 128 rows, 8192 x 10240: 42.6 us
    // with tiles of 128, 35.4 with two of 64 each)
    static constexpr int kMostRows = ROWS == 128 && stages(128) < 3 ? 120 : ROWS;
    static_assert(stages(kMostRows) >= 2, "two stages at least");
};

// kind::f16: bf16 x bf16, both K-major, float32 sums
__host__ __device__ constexpr uint32_t idesc_bf16(int m, int n) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (uint32_t(n >> 3) << 17) | (uint32_t(m >> 4) << 24);
}
// Operands by the low words of their descriptors (128-byte swizzle, K-major, groups of 8 rows 1024 bytes apart; the high word is the same for
// all): a step along an operand is one addition for the one thread that issues.
constexpr uint32_t kDescHigh = uint32_t((uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61) >> 32);
__device__ __forceinline__ uint32_t desc_low(uint32_t addr) { return (addr & 0x3FFFFu) >> 4 | 1u << 16; }
__device__ __forceinline__ void mma_bf16_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 x, {%1, %5};\n\tmov.b64 y, {%2, %5};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "n"(kDescHigh)
                 : "memory");
}
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
__device__ __forceinline__ void tmem_ld_x16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}
// 16 bytes, of which the first `bytes` are copied and the others become zeros
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// This thread's arrival on `bar`, once all copies that it has asked for have landed.
__device__ __forceinline__ void arrive_with_copies(uint64_t* bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(ptx::smem_addr(bar)) : "memory");
}
// wait_bounded for a barrier's first phase that CTAs of the cluster arrive on: what they wrote before is seen behind it
__device__ __forceinline__ bool wait_cluster(uint64_t* bar, const Abort& ab) {
    const bool ok = wait_bounded(bar, 0, ab);
    asm volatile("fence.acq_rel.cluster;" ::: "memory");
    return ok;
}
// a bf16 pair plus two floats, rounded (the sums as one packed addition)
__device__ __forceinline__ uint32_t add_rounded(uint32_t pair, uint32_t d0, uint32_t d1) {
    uint32_t s0, s1;
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=r"(s0), "=r"(s1) : "r"(pair << 16), "r"(pair & 0xFFFF0000u), "r"(d0), "r"(d1));
    return rounded(__uint_as_float(s0), __uint_as_float(s1));
}
// shared memory by 32-bit address
__device__ __forceinline__ uint4 lds4(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}
__device__ __forceinline__ uint32_t lds_half(uint32_t a) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ void sts4(uint32_t a, uint4 v) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ bool all(bool ok) { return __all_sync(0xffffffffu, ok); }

template <int R, int ROWS>
__global__ void __launch_bounds__(kThreads, 1)
adapters_tile_kernel(const AdapterArgs p) {
    using S = Shape<R, ROWS>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t s_full[S::kMostStages], s_empty[S::kMostStages], s_ready[2], s_d1, s_h, s_d2[kTeams], s_d2_free[kTeams];
    __shared__ uint32_t s_tmem;
    __shared__ int s_red[kThreads / 32], s_item[2], s_rows[ROWS], s_abort;
    __shared__ int64_t s_off[ROWS];                        // bytes from out to the tile's rows, -1 behind the last
    uint8_t* smem = smem_raw + (1024 - (ptx::smem_addr(smem_raw) & 1023)) % 1024;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const int cl = p.cluster, tile = int(blockIdx.x) / cl, part = int(blockIdx.x) - tile * cl;
    const int tile_rows = S::kFew ? ROWS : p.tile_rows, x_block = tile_rows * 128;
    const int stage = S::kFew ? S::stage_bytes(ROWS) : p.stage, stages = S::kFew ? S::stages(ROWS) : p.stages;
    const int ring = S::kFew ? S::ring_bytes(ROWS) : p.ring, h_block = S::h_block(tile_rows);
    if (t == 0) {
        for (int i = 0; i < stages; ++i) {
            ptx::mbar_init(&s_full[i], kFeeders);
            ptx::mbar_init(&s_empty[i], kTeam / 32);       // a team's warps; in the first product the MMAs, for all of them
        }
        for (int i = 0; i < 2; ++i) ptx::mbar_init(&s_ready[i], cl);
        for (int i = 0; i < kTeams; ++i) {
            ptx::mbar_init(&s_d2[i], 1);
            ptx::mbar_init(&s_d2_free[i], kTeam / 32);
        }
        ptx::mbar_init(&s_d1, kIssuers);
        ptx::mbar_init(&s_h, kWorkers);
        ptx::fence_barrier_init();
        s_abort = 0;
    }
    __syncwarp();
    if (cl > 1) cluster_arrive();                          // waited for below: all CTAs have started, their barriers are set
    Item item;
    if (!find_item<kThreads, ROWS>(p, tile, tile_rows, smem, s_red, s_item, s_rows, item)) return;  // the same in all CTAs of a cluster
    if (cl > 1) cluster_wait();
    if (t < ROWS) s_off[t] = s_rows[t] < 0 ? -1 : s_rows[t] * p.out_stride * 2;
    if (warp == 0) {
        ptx::tmem_alloc(&s_tmem, 512);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    // Tensor memory: D1, one of each issuer; D2, one of each team, over D1 once it has been read
    const uint32_t tmem = s_tmem;
    const int slot = item.slot, cnt = item.cnt, rank = item.rank;
    // this CTA's parts of K and N, in units of 64 and 128
    const int ku = (p.K + 63) / 64, nu = (p.N + kCols - 1) / kCols;
    const int k0 = 64 * (ku * part / cl), k1 = rank > 0 ? min(64 * (ku * (part + 1) / cl), p.K) : k0;
    const int n0 = kCols * (nu * part / cl), n1 = min(kCols * (nu * (part + 1) / cl), p.N);
    uint8_t* s_hop = smem + ring;                          // H as operand
    float* s_part = reinterpret_cast<float*>(s_hop + S::kHBlocks * h_block);
    float* s_sum = s_part + S::kPart / 4;
    const Abort ab{&s_abort, p.status};
    int sg = 0, owner = 0;                                 // place in the ring, its team
    uint32_t turn = 0;
    const auto leave = [&](bool ok) { tc::leave_cluster(ok, 2, kThreads, cl); };
    const auto advance = [&] {
        if (++owner == kTeams) owner = 0;
        if (++sg == stages) { sg = owner = 0; turn ^= 1; }
    };

    if (warp >= kWorkers / 32 + kIssuers) {
        // ---------------------------------------------------------------- feeders: a thread has the same 16 bytes of its rows in all stages
        const int me = t - kWorkers - 32 * kIssuers, piece = me & 15, row0 = me >> 4;              // 16 rows of 256 bytes at a time
        constexpr int kX = ROWS / 16, kA = R / 16;
        const uint8_t* src[kX];
        const auto set_rows = [&](const void* m, int64_t stride, int at) {
#pragma unroll
            for (int i = 0; i < kX; ++i)
                src[i] = static_cast<const uint8_t*>(m) + (int64_t(max(s_rows[min(row0 + 16 * i, cnt - 1)], 0)) * stride + at + 8 * piece) * 2;
        };
        // place in an operand block of the row and 16-byte piece that this thread copies
        const uint32_t swz = uint32_t(row0 * 128 + (((piece & 7) ^ (row0 & 7)) << 4)), base_addr = ptx::smem_addr(smem);
        bool ok = true;
        set_rows(p.x, p.x_stride, k0);
        const uint8_t* a = reinterpret_cast<const uint8_t*>(p.A + (int64_t(slot) * p.max_rank + row0) * p.K + k0 + 8 * piece);
        const int64_t a_step = int64_t(16) * p.K * 2;
        for (int k = k0; k < k1; k += kCols) {
            if (!(ok = all(wait_bounded(&s_empty[sg], turn ^ 1, ab)))) break;
            const uint32_t to = base_addr + sg * stage + swz;
            const int bytes = k + 8 * piece < k1 ? 16 : 0;             // behind the last column: zeros
            const int64_t back = bytes ? 0 : int64_t(k1 - 8 - k - 8 * piece) * 2;       // (from an address that exists)
            const uint32_t block = piece >> 3;
#pragma unroll
            for (int i = 0; i < kA; ++i)
                if (row0 + 16 * i < rank) cp_async16(to + block * S::kABlock + i * 2048, a + i * a_step + back, bytes);
#pragma unroll
            for (int i = 0; i < kX; ++i) {
                if (row0 + 16 * i < cnt) cp_async16(to + 2 * S::kABlock + block * x_block + i * 2048, src[i] + back, bytes);
                src[i] += kCols * 2;
            }
            a += kCols * 2;
            arrive_with_copies(&s_full[sg]);
            advance();
        }
        // rows of B: R / 8 pieces of each, side by side; what lies behind the rank in the last 16 that are used becomes zero
        constexpr int kP = R / 8, kRows = kFeeders / kP, kTimes = kCols / kRows;
        const int bp = me % kP, br = me / kP, bytes = min(max(rank - 8 * bp, 0), 8) * 2;
        const bool used = 8 * bp < (rank + 15) / 16 * 16;
        const uint8_t* w = reinterpret_cast<const uint8_t*>(p.B + (int64_t(slot) * p.N + n0 + br) * p.max_rank) + (bytes ? 16 * bp : 0);
        const int64_t w_step = int64_t(kRows) * p.max_rank * 2, w_stage = int64_t(kCols) * p.max_rank * 2;
        if (p.base) set_rows(p.base, p.base_stride, n0);
        for (int n = n0; ok && n < n1; n += kCols) {
            if (!(ok = all(wait_bounded(&s_empty[sg], turn ^ 1, ab)))) break;
            const uint32_t to = base_addr + sg * stage;
            if (used) {
#pragma unroll
                for (int i = 0; i < kTimes; ++i) {
                    const int r = br + i * kRows;
                    if (n + r < n1) cp_async16(to + (bp >> 3) * S::kBBlock + r * 128 + (((bp & 7) ^ (r & 7)) << 4), w + i * w_step, bytes);
                }
            }
            w += w_stage;
            if (p.base) {
                const uint32_t cell = to + S::kBlocks * S::kBBlock + row0 * S::kPitch + piece * 16;
#pragma unroll
                for (int i = 0; i < kX; ++i) {
                    if (row0 + 16 * i < cnt && n + 8 * piece < n1) cp_async16(cell + 16 * i * S::kPitch, src[i], 16);
                    src[i] += kCols * 2;
                }
            }
            arrive_with_copies(&s_full[sg]);
            advance();
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        leave(ok);
        return;
    }

    if (warp >= kWorkers / 32) {
        // ---------------------------------------------------------------- one thread of each of three warps issues the MMAs of every third place
        // of the ring, to sums of its own (all lanes walk along, so that operands are the warp's, not a thread's).  A place has the same issuer and
        // team for good: who waits for its next phase has seen the last one end, which a bit of parity alone would not tell.
        const int me = warp - kWorkers / 32;
        bool ok = true;
        if (rank > 0) {
            constexpr uint32_t id1 = idesc_bf16(128, S::kFew ? ROWS : R), id2 = idesc_bf16(128, S::kFew ? kSumParts * ROWS : kCols);
            const uint32_t base_addr = ptx::smem_addr(smem), h_low = desc_low(ptx::smem_addr(s_hop)), d = __shfl_sync(0xffffffffu, tmem, 0);
            const uint32_t d1 = d + me * R, d2 = d + me * kCols;
            const auto issue = [&](uint32_t to, uint32_t rows, uint32_t weights, uint32_t id, uint32_t more) {
                if constexpr (S::kFew) mma_bf16_ss(to, weights, rows, id, more);
                else mma_bf16_ss(to, rows, weights, id, more);
            };
            const bool lead = elect_one();
            uint32_t more = 0;
            for (int k = k0; k < k1; k += kCols, advance()) {
                if (owner != me) continue;
                if (!(ok = all(wait_bounded(&s_full[sg], turn, ab)))) break;
                ptx::fence_proxy_async_smem();             // copies of the generic proxy, read by the tensor core
                ptx::tc_fence_after_sync();
                const uint32_t ranks = desc_low(base_addr + sg * stage), rows = ranks + (2 * S::kABlock >> 4);
                if (lead) {
#pragma unroll
                    for (int s = 0; s < 8; ++s)
                        issue(d1, rows + (((s >> 2) * x_block + (s & 3) * 32) >> 4), ranks + (((s >> 2) * S::kABlock + (s & 3) * 32) >> 4), id1,
                              s > 0 ? 1u : more);
                    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(ptx::smem_addr(&s_empty[sg])), "n"(kTeam / 32 - 1) : "memory");
                    ptx::mma_commit(&s_empty[sg]);
                }
                __syncwarp();
                more = 1;
            }
            if (ok && lead) ptx::mma_commit(&s_d1);
            if (ok) ok = all(wait_bounded(&s_h, 0, ab));
            ptx::fence_proxy_async_smem();
            ptx::tc_fence_after_sync();
            const int steps = (rank + 15) / 16;
            uint32_t uses = 0;                             // the phase of the team's D2
            for (int n = n0; ok && n < n1; n += kCols, advance()) {
                if (owner != me) continue;
                ok = all(wait_bounded(&s_full[sg], turn, ab) && wait_bounded(&s_d2_free[me], uses ^ 1, ab));
                if (!ok) break;
                uses ^= 1;
                ptx::fence_proxy_async_smem();
                ptx::tc_fence_after_sync();
                const uint32_t columns = desc_low(base_addr + sg * stage);
                if (lead) {
#pragma unroll
                    for (int i = 0; i < (S::kFew ? 1 : kSumParts); ++i)        // (few rows: all parts are N of one MMA)
#pragma unroll
                        for (int s = 0; s < R / 16; ++s) {
                            if (s > 0 && s >= steps) break;
                            const int at = i * R + 16 * s;                     // element of a row of H
                            issue(d2, h_low + (((at >> 6) * h_block + (at & 63) * 2) >> 4), columns + (((s >> 2) * S::kBBlock + (s & 3) * 32) >> 4), id2,
                                  i > 0 || s > 0);
                        }
                    ptx::mma_commit(&s_d2[me]);
                }
                __syncwarp();
            }
        }
        leave(ok);
        return;
    }

    // -------------------------------------------------------------------- workers: three teams, thread `row` of a team has that row of the tile
    const int team = t / kTeam, row = t % kTeam, quarter = warp & 3;
    const uint32_t my_tmem = tmem + (uint32_t(quarter * 32) << 16);
    bool ok = true;                                        // false: a wait ran out; go through the motions without waiting
    for (int k = k0; k < k1; k += kCols) advance();        // the stages of the first product are the MMAs'
    if (rank > 0) {
        ok = all(wait_bounded(&s_d1, 0, ab));
        ptx::tc_fence_after_sync();
        const int parts = min((k1 - k0 + kCols - 1) / kCols, min(kIssuers, stages));     // issuers that had a stage
        // Sums in fours.  Small tiles: every CTA hands all of its sums to all CTAs, which add them up, each for itself.  Others: the e-th four
        // goes to CTA e % cl, which adds the cl parts and hands the result to all; a cl-th of the traffic, one more exchange.
        const int fours = cnt * (R / 4);
        const uint32_t sum_addr = ptx::smem_addr(s_sum), h_addr = ptx::smem_addr(s_hop);
        const float scale = p.scale[slot];
        const auto sums = [&](int c, float (&d)[16]) {     // 16 columns of this thread's row of D1
#pragma unroll
            for (int i = 0; i < 16; ++i) d[i] = 0.f;
            for (int i = 0; i < parts; ++i) {
                uint32_t w[16];
                tmem_ld_x16(my_tmem + i * R + c, w);
                ptx::tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 16; ++j) d[j] += __uint_as_float(w[j]);
            }
        };
        if constexpr (S::kFew) {
            if (team == 0 && quarter * 32 < R) {           // thread `row` has rank `row`
                float d[16];
                sums(0, d);
                if (row < R) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (i < cnt) s_part[i * R + row] = d[i];
                }
            }
        } else if (quarter * 32 < cnt) {
#pragma unroll 1
            for (int c = 16 * team; c < R; c += 16 * kTeams) {
                float d[16];
                sums(c, d);
                if (row < cnt) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int e = row * (R / 4) + c / 4 + i;
                        st_cluster4(ptx::map_to_cta(sum_addr + (e / cl * cl + part) * 16, e % cl), make_float4(d[4 * i], d[4 * i + 1], d[4 * i + 2], d[4 * i + 3]));
                    }
                }
            }
        }
        ptx::named_bar_sync(1, kWorkers);
        if constexpr (S::kFew) {
            for (int i = t; i < fours * cl; i += kWorkers) {
                const int e = i / cl, to = i - e * cl;
                st_cluster4(ptx::map_to_cta(sum_addr + (e * cl + part) * 16, to), reinterpret_cast<const float4*>(s_part)[e]);
            }
            ptx::named_bar_sync(1, kWorkers);
        }
        if (t < cl) ptx::mbar_arrive_cluster(ptx::map_to_cta(ptx::smem_addr(&s_ready[0]), t));
        ok = all(ok && wait_cluster(&s_ready[0], ab));
        for (int k = t; S::kFew ? k < fours : part + k * cl < fours; k += kWorkers) {
            const int e = S::kFew ? k : part + k * cl, at_row = e / (R / 4), col = e % (R / 4) * 4;
            float f[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int c = 0; c < cl; ++c) {
                const float4 o = *reinterpret_cast<const float4*>(s_sum + (k * cl + c) * 4);
                f[0] += o.x; f[1] += o.y; f[2] += o.z; f[3] += o.w;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = col + i < rank ? f[i] * scale : 0.f;
#pragma unroll
            for (int i = 0; i < kSumParts; ++i) {
                const bool last = i + 1 == kSumParts;
                const uint32_t w0 = last ? rounded(f[0], f[1]) : upper(f[0], f[1]), w1 = last ? rounded(f[2], f[3]) : upper(f[2], f[3]);
#pragma unroll
                for (int j = 0; j < 4; ++j) f[j] = rest_of_sum(f[j]);
                const int element = (S::kFew ? 0 : i * R) + col, byte = 2 * (element & 63), line = at_row + (S::kFew ? ROWS * i : 0);
                const uint32_t at = h_addr + (element >> 6) * h_block + line * 128 + (((byte >> 4) ^ (line & 7)) << 4) + (byte & 15);
                if constexpr (S::kFew) {
                    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(w0), "r"(w1) : "memory");
                } else {
                    for (int c = 0; c < cl; ++c) st_cluster2(ptx::map_to_cta(at, c), w0, w1);
                }
            }
        }
        if constexpr (!S::kFew) {
            ptx::named_bar_sync(1, kWorkers);
            if (t < cl) ptx::mbar_arrive_cluster(ptx::map_to_cta(ptx::smem_addr(&s_ready[1]), t));
            ok = all(ok && wait_cluster(&s_ready[1], ab));
        }
        ptx::fence_proxy_async_smem();                     // H is read by the tensor core
        ptx::tc_fence_before_sync();                       // D1 is written over
        ptx::mbar_arrive(&s_h);
    }
    uint8_t* out = static_cast<uint8_t*>(p.out);
    const bool has_base = p.base != nullptr;
    const uint32_t smem_base = ptx::smem_addr(smem);
    const int first_row = 32 * quarter + (lane >> 4);
    uint32_t uses = 0;
    for (int n = n0; n < n1; n += kCols, advance()) {
        if (owner != team) continue;                 // another team's
        const uint32_t d2 = my_tmem + team * kCols;
        ok = all(ok && wait_bounded(&s_full[sg], turn, ab) && (rank == 0 || wait_bounded(&s_d2[team], uses, ab)));
        ptx::tc_fence_after_sync();
        const uint32_t cells = smem_base + sg * stage + S::kBlocks * S::kBBlock;
        const auto release = [&] {                         // D2 has been read: the team's next MMAs run under the rest
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&s_d2_free[team]);
        };
        if constexpr (S::kFew) {
            float d[16];                                   // the parts' products, the smallest first
#pragma unroll
            for (int i = 0; i < 16; ++i) d[i] = 0.f;
            if (rank > 0) {
                uint32_t w[kSumParts][16];
#pragma unroll
                for (int i = 0; i < kSumParts; ++i) tmem_ld_x16(d2 + 16 * i, w[i]);
                ptx::tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i) d[i] = __uint_as_float(w[0][i]) + (__uint_as_float(w[1][i]) + __uint_as_float(w[2][i]));
            }
            release();
            uint8_t* to = out + (n + row) * 2;
            if (ok && n + row < n1) {
#pragma unroll
                for (int i0 = 0; i0 < 16; i0 += 4) {       // four rows at a time, as many as there are
                    if (i0 >= cnt) break;
                    uint32_t o[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[i] = has_base ? lds_half(cells + (i0 + i) * S::kPitch + row * 2) : 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int64_t at = s_off[i0 + i];
                        if (at >= 0)
                            *reinterpret_cast<__nv_bfloat16*>(to + at) =
                                __float2bfloat16_rn(__uint_as_float(o[i] << 16) + d[i0 + i]);
                    }
                }
            }
        } else if (ok && quarter * 32 < cnt) {             // a warp's rows are its own from the sums to the stores
            const uint32_t cell = cells + row * S::kPitch;
#pragma unroll 1
            for (int c = 0; c < kCols; c += 32) {
                uint32_t d[32];
                if (rank > 0) {
                    ptx::tmem_ld_32x32b_x32(d2 + c, d);
                    ptx::tmem_ld_wait();
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) d[i] = 0;
                }
                if (row < cnt) {
                    uint4 o[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[i] = has_base ? lds4(cell + c * 2 + 16 * i) : make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t w[4] = {o[i].x, o[i].y, o[i].z, o[i].w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) w[j] = add_rounded(w[j], d[8 * i + 2 * j], d[8 * i + 2 * j + 1]);
                        sts4(cell + c * 2 + 16 * i, make_uint4(w[0], w[1], w[2], w[3]));
                    }
                }
            }
            release();
            // 16 threads a row, 2 rows at a time
            if (n + 8 * (lane & 15) < n1) {
                const uint32_t from = cells + first_row * S::kPitch + (lane & 15) * 16;
                uint8_t* to = out + (n + 8 * (lane & 15)) * 2;
#pragma unroll
                for (int i0 = 0; i0 < 16; i0 += 4) {
                    if (32 * quarter + 2 * i0 >= cnt) break;
                    uint4 o[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[i] = lds4(from + (i0 + i) * 2 * S::kPitch);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int64_t at = s_off[(first_row + 2 * (i0 + i)) % ROWS];
                        if (at >= 0) *reinterpret_cast<uint4*>(to + at) = o[i];
                    }
                }
            }
        } else {
            release();
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&s_empty[sg]);
        uses ^= 1;
    }
    ptx::tc_fence_before_sync();
    leave(ok);
    ptx::tc_fence_after_sync();
    if (warp == 0) ptx::tmem_dealloc(tmem, 512);
}

template <int R, int ROWS>
int launch_shape(AdapterArgs p, cudaStream_t st) {
    using S = Shape<R, ROWS>;
    constexpr auto kern = adapters_tile_kernel<R, ROWS>;
    static_assert(find_bytes(8192, kThreads) <= S::ring_bytes(S::kMostRows), "the counts of 8192 adapters lie where the stages will be, in front of what other CTAs write");
    QLLM_CUDA_TRY(allow_smem<kern>(S::kBytes));
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = S::kBytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    // For each size of a cluster: the rounds that the fewest tiles take, the fewest rows to a tile with which they do, be the groups random (their
    // last tiles are half full, some more) or alike; of these the shortest launch: 128 columns of both products together take a CTA
    // (180 + rows) 5.6 ns (rank 32; 100 + rows transposed), and a round has 8 us of its own.  3792 rows on 9 adapters, 8192 x 8192: 3 CTAs to 104 rows 56.1 us (timed
    // like the following), 3 to 112 57.5, 3 to 128 59.6, 2 to 64 56.2, 4 to 128 (two rounds) 65.4.  1024 rows of one, 8192 x 10240: 8 to 72 25.6; 8 to 128 33.8,
    // 6 to 48 27.4, 2 to 16 48.7; rank 64: 8 to 72 30.5, 8 to 120 38.7, 6 to 48 30.9.  20000 rows of one, 4096 x 4096, rank 16: 3 rounds of 2 CTAs to 96 rows 116,
    // 2 rounds of single CTAs to 128 148.
    // (Clusters of 4: 33 of 148 SMs' possible 37, whatever their parts of the chip.)
    const int64_t groups = std::min<int64_t>({p.seqs, p.slots + 1, p.rows});
    static std::atomic<int> known[64][9];
    int dev = 0;
    QLLM_CUDA_TRY(cudaGetDevice(&dev));
    const int64_t each = (p.rows + groups - 1) / groups;
    double least = 1e30;
    for (int cl = 8; cl >= 1; --cl) {
        int most = dev < 64 ? known[dev][cl].load(std::memory_order_relaxed) : 0;
        if (!most) {
            attr[0].val.clusterDim.x = unsigned(cl);
            cfg.gridDim = dim3(unsigned(cl));
            cfg.numAttrs = 1;
            QLLM_CUDA_TRY(cudaOccupancyMaxActiveClusters(&most, kern, &cfg));
            most = std::max(most, 1);
            if (dev < 64) known[dev][cl].store(most, std::memory_order_relaxed);
        }
        const int64_t fewest = std::max(p.rows / S::kMostRows + 3 * groups / 4, groups * ((each + S::kMostRows - 1) / S::kMostRows)), rounds = (fewest + most - 1) / most;
        const int64_t room = 4 * most * rounds - 3 * groups;               // fours of tiles beside the groups' last ones
        const int64_t rows = std::max(4 * p.rows / room + 1, (each + most * rounds / groups - 1) / (most * rounds / groups));
        const int tile_rows = S::kFew ? ROWS : int(std::min<int64_t>((rows + 7) / 8 * 8, S::kMostRows));
        const double time = double(rounds) * (double(tile_rows + (S::kFew ? 100 : 180)) / cl + 366e3 / (double(p.K) + p.N));
        if (time < least) {
            least = time;
            p.cluster = cl;
            p.tile_rows = tile_rows;
        }
    }
    p.ring = S::ring_bytes(p.tile_rows);
    p.stage = S::stage_bytes(p.tile_rows);
    p.stages = S::stages(p.tile_rows);
    const int64_t tiles = groups + (p.rows - groups) / p.tile_rows;        // at most
    attr[0].val.clusterDim.x = unsigned(p.cluster);
    cfg.gridDim = dim3(unsigned(tiles * p.cluster));
    cfg.numAttrs = 2;
    QLLM_CUDA_TRY(cudaLaunchKernelEx(&cfg, kern, p));
    return after_launch();
}

}  // namespace

int launch_tiles_tc(const AdapterArgs& p, bool few, cudaStream_t st) {
    if (p.max_rank <= 16) return launch_shape<16, 128>(p, st);
    if (p.max_rank <= 32) return launch_shape<32, 128>(p, st);
    if (p.max_rank <= 64) return few ? launch_shape<64, 16>(p, st) : launch_shape<64, 128>(p, st);
    return few ? launch_shape<128, 16>(p, st) : launch_shape<128, 64>(p, st);
}

}  // namespace lora
}  // namespace qllm
