// Internal definitions of prompt attention (rlkv_prompt_*): shared by its host side and its kernels.
#pragma once

#include "rlkv_internal.cuh"

namespace rlkv {

// One call.  Documents d: queries q_starts[d] .. q_starts[d+1]-1, keys k_starts[d] .. k_starts[d+1]-1; query i of a
// document with qn queries and kn keys stands at position i + kn - qn, key j at position j.
struct PromptArgs {
    const __nv_bfloat16 *q, *k, *v;      // tokens *_stride elements apart
    long long q_stride, k_stride, v_stride;
    int q_tokens, k_tokens;
    const int *q_starts, *k_starts;      // device, [n_docs + 1]
    const int* prefix;                   // device, [n_docs], or null
    int n_docs, group, q_heads, kv_heads, sink, window;
    float scale, softcap;                // 1 / sqrt(head_dim); 0: no cap
    const float* slopes;                 // device, [q_heads], or null
    __nv_bfloat16* out;                  // [q_tokens][q_heads][head_dim]
    float* lse;                          // [q_tokens][q_heads], may be null in the forward pass
    const __nv_bfloat16* dout;
    __nv_bfloat16 *dq, *dk, *dv;
    float* delta;                        // scratch, [q_tokens][q_heads]: sum over head_dim of dout * out
    int* status;
    unsigned char full[kMaxKvHeads];     // 1: the KV head sees every key, 0: sink and window only
};

// The part of the packed tokens that belongs to document d.  Starts come from device memory: whatever they
// hold, the range stays inside the tensors.
struct DocRange {
    int q0, qn, k0, kn, prefix;
};
__device__ __forceinline__ DocRange doc_range(const PromptArgs& a, int d)
{
    DocRange r;
    r.q0 = min(max(a.q_starts[d], 0), a.q_tokens);
    r.qn = min(max(a.q_starts[d + 1], r.q0), a.q_tokens) - r.q0;
    r.k0 = min(max(a.k_starts[d], 0), a.k_tokens);
    r.kn = min(max(a.k_starts[d + 1], r.k0), a.k_tokens) - r.k0;
    r.prefix = a.prefix ? min(max(a.prefix[d], 0), r.kn) : 0;
    return r;
}

cudaError_t launch_prompt_forward(const PromptArgs& a, int head_dim, cudaStream_t stream);
cudaError_t launch_prompt_backward(const PromptArgs& a, int head_dim, cudaStream_t stream);

}  // namespace rlkv
