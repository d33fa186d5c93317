// qllm_kv_rotate_append: queries and keys turned by their tokens' angles, keys and values stored in the 4-bit cache, in one launch;
// qllm_rotary_table: the table of cosines and sines.
//
// A pair (a, b) of channels becomes (a cos - b sin, b cos + a sin), products and sums rounded to float32 one by one (no fused
// multiply-add: stored codes then follow from the formula as it stands, whatever computes it), queries rounded once to their type.
// Keys go into Eq. 2 unrounded.  Codes and parameters of keys and values are those of qllm_kv_append on the turned rows.
//
// It moves bytes: queries in and out, keys and values in, (head_dim / 2 + 8) bytes a row out, 4 rot_dim bytes of table a token.
// head_dim / 16 lanes own a row, 16 channels each in two runs of 8, so chosen that both channels of a pair lie in one lane: for pairs
// (p, p + rot_dim / 2) lane l < rot_dim / 16 has the runs l and l + rot_dim / 16, for pairs (2p, 2p + 1) two neighbouring runs; either way its
// pairs are 8l .. 8l + 7, one 64-byte piece of the table.  A unit of work is a few rows of one token and one kind (queries, keys or values):
// their loads are in flight together, before the token's place has been found, and share the cosines and sines in registers.

#include <algorithm>

#include "kv_rows.cuh"

namespace qllm {
namespace {

using namespace kv;

struct Angles {
    const float4* table;                                   // [positions][rot_dim / 2] pairs (cos, sin), two to a float4
    int positions, rot_dim, interleaved;
};

struct Turn {
    const void *q, *k, *v;
    void* q_out;
    int64_t q_stride, q_out_stride, k_stride, v_stride;
    int q_heads;
};

// 8 channels as they lie in memory; plain loads (queries may be turned in place)
template <typename T>
struct Run8;
template <>
struct Run8<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            f[2 * k] = __uint_as_float(w[k] << 16);
            f[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
        }
    }
};
template <>
struct Run8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) { a = reinterpret_cast<const float4*>(p)[0]; b = reinterpret_cast<const float4*>(p)[1]; }
    __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
};

// the least of three, NaN if one is
__device__ __forceinline__ float min3_nan(float a, float b, float c) {
    float r;
    asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// The lane's pairs (a, b) by cosine and sine, one rounding an operation.  (The packed operations on two floats would be half as many
// instructions, but a packed product and sum come out fused, whatever rounding they name.)
struct Sines {
    float4 w[4];                                           // cos, sin of two pairs
    __device__ __forceinline__ void load(const float4* p) {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = __ldg(p + j);
    }
    __device__ __forceinline__ void turn(float c, float s, float& a, float& b) const {
        const float x = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
        b = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
        a = x;
    }
    __device__ __forceinline__ void turn_row(float (&f)[2][8], bool interleaved) const {
        if (interleaved) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                turn(w[j].x, w[j].y, f[j >> 1][4 * (j & 1)], f[j >> 1][4 * (j & 1) + 1]);
                turn(w[j].z, w[j].w, f[j >> 1][4 * (j & 1) + 2], f[j >> 1][4 * (j & 1) + 3]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                turn(w[j].x, w[j].y, f[0][2 * j], f[1][2 * j]);
                turn(w[j].z, w[j].w, f[0][2 * j + 1], f[1][2 * j + 1]);
            }
        }
    }
};

// A CTA's tokens and units: U rows of one kind each, ordered [token][queries, keys, values].
struct Work {
    int tokens, q_blocks, kv_blocks;
    uint32_t inverse;                                      // ceil(2^32 / blocks): unit -> token, units < 2^16
};

template <typename T, int D, int U>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 4 : 2)
kv_rotate_append_kernel(const Turn a, const Cache c, const Batch b, const Angles ang, const Work work, int* status) {
    constexpr int L = D / 16, G = 256 / L;                 // lanes of a row, units of a CTA in flight
    __shared__ int4 s_place[kMostTokens];                  // page (or -1: nobody's row, -2: no place), place in it, position or -1
    const int lane = threadIdx.x % L, group = threadIdx.x / L, blocks = work.q_blocks + 2 * work.kv_blocks;
    const int64_t t0 = int64_t(blockIdx.x) * work.tokens;
    const int tokens = int(min(int64_t(work.tokens), b.rows - t0)), units = tokens * blocks;
    const int turned = ang.rot_dim / 16;                   // lanes that turn
    int ra = 2 * lane, rb = 2 * lane + 1;                  // the lane's runs of 8 channels
    if (!ang.interleaved && lane < turned) { ra = lane; rb = lane + turned; }
    asm volatile("griddepcontrol.wait;" ::: "memory");     // launched as a dependent: nothing above touched global memory
    for (int base = 0; base < units; base += G) {
        const int unit = min(base + group, units - 1), tok = int(__umulhi(uint32_t(unit), work.inverse)), block = unit - tok * blocks;
        const int64_t t = t0 + tok;
        const int kind = block < work.q_blocks ? 0 : block < work.q_blocks + work.kv_blocks ? 1 : 2;       // query, key, value
        const int head = (kind == 0 ? block : kind == 1 ? block - work.q_blocks : block - work.q_blocks - work.kv_blocks) * U;
        const int rows = base + group < units ? min(U, (kind == 0 ? a.q_heads : c.heads) - head) : 0;
        const T* p = (kind == 0 ? static_cast<const T*>(a.q) + t * a.q_stride
                    : kind == 1 ? static_cast<const T*>(a.k) + t * a.k_stride : static_cast<const T*>(a.v) + t * a.v_stride) + head * D;
        Run8<T> x[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u < rows) {
                x[u][0].load(p + u * D + 8 * ra);
                x[u][1].load(p + u * D + 8 * rb);
            } else {
                x[u][0].zero();
                x[u][1].zero();
            }
        }
        if (base == 0) {                                   // under the first loads
            if (threadIdx.x < 32) {
                const int i = threadIdx.x;
                const int s = seq_of_lane(b, t0, tokens, i);
                if (i < tokens) {
                    int4 at = make_int4(-1, 0, -1, 0);
                    if (s >= 0) {
                        const int64_t pos = int64_t(b.len(s)) - b.count(s) + (t0 + i - b.row(s));
                        at.x = -2;
                        if (pos >= ang.positions) {
                            raise_page(status);
                        } else if (pos >= 0) {
                            at.z = int(pos);
                            const int page = b.table[int64_t(s) * b.width + (pos >> b.page_log2)];
                            if (page >= 0 && page < c.pages) { at.x = page; at.y = int(pos) & ((1 << b.page_log2) - 1); }
                            else raise_page(status);
                        }
                    }
                    s_place[i] = at;
                }
            }
            if (blockIdx.x == 0) b.report(status, threadIdx.x, 256);
            __syncthreads();
        }
        const int4 at = s_place[tok];
        const bool turns = kind < 2 && at.z >= 0 && lane < turned;
        Sines sc;
        if (turns) sc.load(ang.table + int64_t(at.z) * (ang.rot_dim / 4) + 4 * lane);
        if (kind == 0 && at.x != -1) {
            T* to = static_cast<T*>(a.q_out) + t * a.q_out_stride + head * D;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u >= rows) break;
                if (at.z < 0) { x[u][0].zero(); x[u][1].zero(); }
                float f[2][8];
                x[u][0].get(f[0]);
                x[u][1].get(f[1]);
                if (turns) sc.turn_row(f, ang.interleaved);
                store8(to + u * D + 8 * ra, f[0]);
                store8(to + u * D + 8 * rb, f[1]);
            }
        }
        const bool stores = kind > 0 && at.x >= 0 && rows > 0;
        if (!__any_sync(0xffffffffu, stores)) continue;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[2][8];
            x[u][0].get(f[0]);
            x[u][1].get(f[1]);
            if (turns && kind == 1) sc.turn_row(f, ang.interleaved);
            float lo = f[0][0], hi = lo;
#pragma unroll
            for (int j = 1; j < 15; j += 2) {
                lo = min3_nan(lo, f[j >> 3][j & 7], f[(j + 1) >> 3][(j + 1) & 7]);
                hi = max3(hi, f[j >> 3][j & 7], f[(j + 1) >> 3][(j + 1) & 7]);
            }
            lo = min_nan(lo, f[1][7]);
            hi = fmaxf(hi, f[1][7]);
#pragma unroll
            for (int o = L / 2; o > 0; o >>= 1) {
                lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
                hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
            }
            if (stores && u < rows) {
                float alpha, inv, zero;
                row_params(f, lo, hi, alpha, inv, zero);
                const int64_t row = c.row(at.x, head + u, at.y);
                uint32_t* to = reinterpret_cast<uint32_t*>((kind == 1 ? c.kc : c.vc) + row * (D / 2));
                to[ra] = codes8(f[0], lo, hi, inv, zero);
                to[rb] = codes8(f[1], lo, hi, inv, zero);
                if (lane == 0) (kind == 1 ? c.kp : c.vp)[row] = make_float2(alpha, zero);
            }
        }
    }
}

// Tokens of a CTA: as many as give every SM sixteen CTAs, at least one step's worth where a token has few rows.  U: rows of a unit; two and
// four CTAs on an SM (64 registers, bf16) were better than 4 and 3, or 1 and 5: 79, 104, 112 us for 9708 tokens of 32 + 2 x 32 heads of 128.  Small
// calls have units of one row, on as many SMs as there are.
template <typename T, int D, int U>
int launch_units(const Turn& a, const Cache& c, const Batch& b, const Angles& ang, int* status, cudaStream_t st) {
    const int qb = (a.q_heads + U - 1) / U, kb = (c.heads + U - 1) / U, blocks = qb + 2 * kb, group = 256 / (D / 16);
    int64_t n = b.rows / (int64_t(device_sm_count()) * 16);
    n = std::min<int64_t>(n, std::max(1, 8 * group / blocks));
    n = std::max<int64_t>(n, std::min(group / blocks, 8));
    n = std::min<int64_t>(std::max<int64_t>(n, 1), std::min(kMostTokens, 65535 / blocks));
    const Work work{int(n), qb, kb, uint32_t(((uint64_t(1) << 32) + blocks - 1) / blocks)};
    QLLM_CUDA_TRY(launch_dependent(kv_rotate_append_kernel<T, D, U>, dim3(unsigned((b.rows + n - 1) / n)), dim3(256), 0, st, a, c, b, ang, work, status));
    return after_launch();
}
template <typename T, int D>
int launch_rotate(const Turn& a, const Cache& c, const Batch& b, const Angles& ang, int* status, cudaStream_t st) {
    constexpr int U = 2;
    const int64_t rows = b.rows * (a.q_heads + 2 * c.heads);
    if (rows * (D / 16) <= int64_t(device_sm_count()) * 256) return launch_units<T, D, 1>(a, c, b, ang, status, st);
    return launch_units<T, D, U>(a, c, b, ang, status, st);
}

// cos and sin of position / divisor * base^(-2 p / rot_dim), the angle in 64 bits
__global__ void __launch_bounds__(256)
rotary_table_kernel(float2* table, int64_t n, int half, double base, double divisor) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) {
        const int64_t pos = i / half;
        const int p = int(i - pos * half);
        double s, co;
        sincos(double(pos) / divisor * pow(base, -double(p) / double(half)), &s, &co);
        table[i] = make_float2(float(co), float(s));
    }
}

int check_rotary(const void* table, int positions, int rot_dim) {
    if (positions <= 0 || rot_dim <= 0) return QLLM_ERR_SHAPE;
    if (rot_dim % 16 || rot_dim > 256 || positions > (1 << 30)) return QLLM_ERR_UNSUPPORTED;
    if (!table) return QLLM_ERR_NULL;
    return aligned16(table) ? QLLM_OK : QLLM_ERR_ALIGN;
}

}  // namespace
}  // namespace qllm

extern "C" int qllm_rotary_table(float* table, int positions, int rot_dim, double base, double divisor, void* stream) {
    using namespace qllm;
    if (!(base > 0.0) || !(base < 1e300) || !(divisor > 0.0) || !(divisor < 1e300)) return QLLM_ERR_SHAPE;
    const int rc = check_rotary(table, positions, rot_dim);
    if (rc != QLLM_OK) return rc;
    const int64_t n = int64_t(positions) * (rot_dim / 2);
    QLLM_CUDA_TRY(launch_dependent(rotary_table_kernel, dim3(unsigned(std::min<int64_t>((n + 255) / 256, int64_t(device_sm_count()) * 8))), dim3(256), 0,
                                   static_cast<cudaStream_t>(stream), reinterpret_cast<float2*>(table), n, rot_dim / 2, base, divisor));
    return after_launch();
}

extern "C" int qllm_kv_rotate_append(const qllm_kv_cache_t* cache, int layer, const void* q, int64_t q_stride, void* q_out, int64_t q_out_stride,
                                     int q_heads, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int dtype,
                                     const qllm_rotary_t* rotary, const qllm_kv_batch_t* batch, void* stream) {
    using namespace qllm;
    if (!dtype_ok(dtype)) return QLLM_ERR_DTYPE;
    int rc = kv::check_cache_batch(cache, batch);
    if (rc != QLLM_OK) return rc;
    if (!rotary) return QLLM_ERR_NULL;
    if (layer < 0 || layer >= cache->layers || q_heads < 0 || rotary->rot_dim > cache->head_dim) return QLLM_ERR_SHAPE;
    if (q_heads > 8192) return QLLM_ERR_UNSUPPORTED;
    rc = check_rotary(rotary->table, rotary->positions, rotary->rot_dim);
    if (rc != QLLM_OK || batch->rows == 0 || batch->seqs == 0) return rc;
    if (q_heads > 0) {
        rc = kv::check_packed(q, q_stride, q_heads, cache->head_dim, dtype);
        if (rc == QLLM_OK) rc = kv::check_packed(q_out, q_out_stride, q_heads, cache->head_dim, dtype);
        if (rc != QLLM_OK) return rc;
        if (q == q_out && q_stride != q_out_stride) return QLLM_ERR_SHAPE;
    }
    rc = kv::check_packed(k, k_stride, cache->kv_heads, cache->head_dim, dtype);
    if (rc == QLLM_OK) rc = kv::check_packed(v, v_stride, cache->kv_heads, cache->head_dim, dtype);
    if (rc != QLLM_OK) return rc;
    int* status = device_status_word();
    if (!status) return QLLM_ERR_CUDA;
    const kv::Cache c = kv::view(cache, layer);
    const kv::Batch b = kv::view(batch, cache);
    const Turn a{q, k, v, q_out, q_stride, q_out_stride, k_stride, v_stride, q_heads};
    const Angles ang{reinterpret_cast<const float4*>(rotary->table), rotary->positions, rotary->rot_dim, rotary->interleaved != 0};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
#define QLLM_KV_D(T, D) if (cache->head_dim == D) return launch_rotate<T, D>(a, c, b, ang, status, st)
    if (dtype == QLLM_BF16) { QLLM_KV_D(__nv_bfloat16, 64); QLLM_KV_D(__nv_bfloat16, 128); QLLM_KV_D(__nv_bfloat16, 256); }
    else { QLLM_KV_D(float, 64); QLLM_KV_D(float, 128); QLLM_KV_D(float, 256); }
#undef QLLM_KV_D
    return QLLM_ERR_UNSUPPORTED;
}
