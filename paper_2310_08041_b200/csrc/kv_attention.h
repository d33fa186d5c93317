// What the attention kernels over the 4-bit cache share on the host side.
#pragma once

#include "kv_cache.cuh"

namespace qllm {
namespace kv {

struct AttnArgs {
    const void* q;
    void* out;
    float* lse;                     // may be null
    int64_t q_stride, out_stride;   // elements
    int dtype, q_heads, group, causal;
    float scale;
    // Sequences with more than this many (new token, grouped query head) rows per key head are the prompt kernel's, the others
    // the streaming kernel's.
    int most_rows;
};

// scale log2 e = the result 2^e: a row's factor of its scores takes the power of two, the keys the rest (1 to 2 in size; 0, and less for subnormal scales).  A
// product with the factor is then exact, and the score that is compared with a maximum is the very one that enters the exponential.
// (A factor that rounds leaves in the fused difference what the compared product lost, 2^-24 of the score: from scores of 10^8 on
// weights became infinite.)
__device__ __forceinline__ float split_scale(float scale, int& e) {
    const float x = fminf(fmaxf(scale * 1.4426950408889634f, -3e38f), 3e38f);
    const uint32_t bits = __float_as_uint(x);
    e = max(int(bits >> 23 & 255u) - 127, -126);
    return fabsf(x) >= 0x1p-126f ? __uint_as_float((bits & 0x807FFFFFu) | 0x3F800000u) : x * 0x1p126f;
}
// Scores from here on: the exponent of a weight is off by the roundings of the reference, none of the slack is left to later tiles.
constexpr float kLargeScore = 0x1p20f;

// Streaming kernel (kv_attention_split.cu): any shape.  Bytes of workspace it takes, and the launch.
int64_t split_workspace(int head_dim, int dtype, int rows_hint);
int launch_attention_split(const Cache& c, const Batch& b, int head_dim, const AttnArgs& a, int rows_hint, void* workspace,
                           int* status, cudaStream_t st);

// Tensor-core kernel (kv_attention_prompt.cu): sequences with more than most_rows query rows per key head.
bool prompt_serves(int head_dim, int dtype);
int64_t prompt_workspace(const Batch& b, int heads, int head_dim, int group, int max_new);
int launch_attention_prompt(const Cache& c, const Batch& b, int head_dim, const AttnArgs& a, int max_new, void* workspace, int* status,
                            cudaStream_t st);

}  // namespace kv
}  // namespace qllm
