// Attention of packed prompts: what its kernels share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "bv_cache.cuh"

namespace bv {

struct PromptArgs {
    const void *q, *k, *v;
    void* out;
    long long qs[2], ks[2], vs[2], os[2];      // elements between tokens, heads
    const int32_t* offsets;                    // [B + 1]
    int B, tokens, Hkv, group, D;
    Divider by_group;
    float kf;                                  // scale log2(e)
    int window, sinks;
    int* status;                               // set if a bounded wait gave up
    unsigned wait_limit;
    int never_signal;
};

// A sequence: its first row and how many there are; none where its offsets are out of order or out of range.
struct Prompt {
    int first, length;
};
__device__ __forceinline__ Prompt prompt_of(const PromptArgs& a, int b) {
    const int first = __ldg(a.offsets + b), end = __ldg(a.offsets + b + 1);
    return first >= 0 && end > first && end <= a.tokens ? Prompt{first, end - first} : Prompt{0, 0};
}
// The lowest position that a token at `pos` sees through its window.
__device__ __forceinline__ int low_of(const PromptArgs& a, int pos) { return a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0; }

cudaError_t launch_prompt_rows(const PromptArgs& a, int dtype, bool aligned, int sms, cudaStream_t stream);
bool prompt_tiles_takes(const PromptArgs& a);
// (`taken` is false if no map of the tensors could be had)
cudaError_t launch_prompt_tiles(const PromptArgs& a, bool out_vec, cudaStream_t stream, bool* taken);
int prompt_tiles_launches(int B);

}  // namespace bv
