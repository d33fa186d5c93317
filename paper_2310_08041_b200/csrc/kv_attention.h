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
