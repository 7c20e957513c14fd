// Attention over packed prompts, forward and backward.
//
// s_ij = cap(q_i.k_j / sqrt(D)) - slope |pos_i - pos_j| over the visible keys, p = softmax(s), o_i = sum p_ij v_j,
// lse_i = log sum exp s_ij; backward with D_i = do_i.o_i: ds = p (do.v - D) (1 - tanh^2), dq = ds k / sqrt(D),
// dk = ds^T q / sqrt(D), dv = p^T do.
#include "rlkv_prompt.cuh"

namespace rlkv {
namespace {

__device__ __forceinline__ bool visible(const PromptArgs& a, bool full, int prefix, int pos, int j)
{
    return j < max(pos + 1, prefix) && (full || j < a.sink || j > pos - a.window);
}

// The document that holds packed token i (starts ascend): the last one that starts at or before it.
__device__ __forceinline__ int doc_of(const int* starts, int n_docs, int i)
{
    int lo = 0, hi = n_docs - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (starts[mid] <= i) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <int D>
__device__ __forceinline__ float dot(const __nv_bfloat16* x, const __nv_bfloat16* y)
{
    float s = 0.f;
    for (int d = 0; d < D; d += 2) {
        const float2 u = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(x + d));
        const float2 w = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(y + d));
        s = fmaf(u.x, w.x, s);
        s = fmaf(u.y, w.y, s);
    }
    return s;
}

// The score of a product, and its derivative by q.k / sqrt(D).
__device__ __forceinline__ float score(const PromptArgs& a, float x, float slope, int dist, float& dx)
{
    dx = 1.f;
    if (a.softcap != 0.f) {
        const float t = tanhf(x / a.softcap);
        dx = 1.f - t * t;
        x = a.softcap * t;
    }
    return x - slope * (float)abs(dist);
}

// One warp per (query, head): 32 keys at a time, a lane per key for the scores, a lane per D / 32 elements for p.V
// (forward) or ds.K (backward).
template <int D, bool BACKWARD>
__global__ void __launch_bounds__(256) prompt_rows_kernel(const __grid_constant__ PromptArgs a)
{
    constexpr int E = D / 32;
    const int lane = threadIdx.x & 31, h = blockIdx.y, kvh = h / a.group;
    const int i = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (i >= a.q_tokens) return;
    const DocRange r = doc_range(a, doc_of(a.q_starts, a.n_docs, i));
    if (i < r.q0 || i >= r.q0 + r.qn) return;
    const int pos = i - r.q0 + r.kn - r.qn;
    const bool full = a.full[kvh];
    const float slope = a.slopes ? a.slopes[h] : 0.f;
    const __nv_bfloat16* q = a.q + i * a.q_stride + h * D;
    const long long row = ((long long)i * a.q_heads + h);
    const int end = min(max(pos + 1, r.prefix), r.kn);
    float m = -INFINITY, l = 0.f, acc[E], delta = 0.f, lse = 0.f;
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    if (BACKWARD) {
        for (int e = 0; e < E; ++e)
            delta += __bfloat162float(a.out[row * D + lane * E + e]) * __bfloat162float(a.dout[row * D + lane * E + e]);
        for (int o = 16; o > 0; o >>= 1) delta += __shfl_xor_sync(0xffffffffu, delta, o);
        if (lane == 0) a.delta[row] = delta;
        lse = a.lse[row];
    }
    for (int j0 = 0; j0 < end; j0 += 32) {
        const int j = j0 + lane;
        float s = -INFINITY, dx = 1.f, p, w;
        if (j < end && visible(a, full, r.prefix, pos, j))
            s = score(a, dot<D>(q, a.k + (r.k0 + j) * a.k_stride + kvh * D) * a.scale, slope, pos - j, dx);
        if (BACKWARD) {
            w = 0.f;
            if (s != -INFINITY)
                w = expf(s - lse) * (dot<D>(a.dout + row * D, a.v + (r.k0 + j) * a.v_stride + kvh * D) - delta) * dx * a.scale;
        } else {
            float mx = s;
            for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const float mn = fmaxf(m, mx);
            if (mn == -INFINITY) continue;
            p = s == -INFINITY ? 0.f : expf(s - mn);
            const float corr = m == -INFINITY ? 0.f : expf(m - mn);
            float sum = p;
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            l = l * corr + sum;
            m = mn;
            for (int e = 0; e < E; ++e) acc[e] *= corr;
            w = p;
        }
        for (int t = 0; t < min(32, end - j0); ++t) {
            const float wt = __shfl_sync(0xffffffffu, w, t);
            if (wt == 0.f) continue;  // (uniform)
            const __nv_bfloat16* x = BACKWARD ? a.k + (r.k0 + j0 + t) * a.k_stride + kvh * D : a.v + (r.k0 + j0 + t) * a.v_stride + kvh * D;
            for (int e = 0; e < E; ++e) acc[e] = fmaf(wt, __bfloat162float(x[lane * E + e]), acc[e]);
        }
    }
    __nv_bfloat16* dst = BACKWARD ? a.dq : a.out;
    const float inv = BACKWARD ? 1.f : l > 0.f ? 1.f / l : 0.f;
    for (int e = 0; e < E; ++e) dst[row * D + lane * E + e] = __float2bfloat16_rn(acc[e] * inv);
    if (!BACKWARD && lane == 0 && a.lse) a.lse[row] = l > 0.f ? m + logf(l) : -INFINITY;
}

// One warp per (key, KV head): 32 queries at a time of every head of the group.
template <int D>
__global__ void __launch_bounds__(256) prompt_keys_kernel(const __grid_constant__ PromptArgs a)
{
    constexpr int E = D / 32;
    const int lane = threadIdx.x & 31, kvh = blockIdx.y;
    const int kj = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (kj >= a.k_tokens) return;
    const DocRange r = doc_range(a, doc_of(a.k_starts, a.n_docs, kj));
    if (kj < r.k0 || kj >= r.k0 + r.kn) return;
    const int j = kj - r.k0;
    const bool full = a.full[kvh];
    const __nv_bfloat16* k = a.k + kj * a.k_stride + kvh * D;
    const __nv_bfloat16* v = a.v + kj * a.v_stride + kvh * D;
    float dk[E], dv[E];
    for (int e = 0; e < E; ++e) dk[e] = dv[e] = 0.f;
    for (int g = 0; g < a.group; ++g) {
        const int h = kvh * a.group + g;
        const float slope = a.slopes ? a.slopes[h] : 0.f;
        for (int i0 = 0; i0 < r.qn; i0 += 32) {
            const int i = i0 + lane, pos = i + r.kn - r.qn;
            float p = 0.f, w = 0.f;
            if (i < r.qn && visible(a, full, r.prefix, pos, j)) {
                const long long row = (long long)(r.q0 + i) * a.q_heads + h;
                float dx;
                const float s = score(a, dot<D>(a.q + (r.q0 + i) * a.q_stride + h * D, k) * a.scale, slope, pos - j, dx);
                p = expf(s - a.lse[row]);
                w = p * (dot<D>(a.dout + row * D, v) - a.delta[row]) * dx * a.scale;
            }
            if (!__any_sync(0xffffffffu, p != 0.f)) continue;
            for (int t = 0; t < min(32, r.qn - i0); ++t) {
                const float pt = __shfl_sync(0xffffffffu, p, t), wt = __shfl_sync(0xffffffffu, w, t);
                const long long x = (long long)(r.q0 + i0 + t);
                if (pt == 0.f) continue;
                for (int e = 0; e < E; ++e) {
                    dv[e] = fmaf(pt, __bfloat162float(a.dout[(x * a.q_heads + h) * D + lane * E + e]), dv[e]);
                    dk[e] = fmaf(wt, __bfloat162float(a.q[x * a.q_stride + h * D + lane * E + e]), dk[e]);
                }
            }
        }
    }
    for (int e = 0; e < E; ++e) {
        const long long at = ((long long)kj * a.kv_heads + kvh) * D + lane * E + e;
        a.dk[at] = __float2bfloat16_rn(dk[e]);
        a.dv[at] = __float2bfloat16_rn(dv[e]);
    }
}

}  // namespace

cudaError_t launch_prompt_backward(const PromptArgs& a, int head_dim, cudaStream_t stream)
{
    const dim3 rows((a.q_tokens + 7) / 8, a.q_heads), keys((a.k_tokens + 7) / 8, a.kv_heads);
    if (head_dim == 128) {
        prompt_rows_kernel<128, true><<<rows, 256, 0, stream>>>(a);
        prompt_keys_kernel<128><<<keys, 256, 0, stream>>>(a);
    } else {
        prompt_rows_kernel<64, true><<<rows, 256, 0, stream>>>(a);
        prompt_keys_kernel<64><<<keys, 256, 0, stream>>>(a);
    }
    return cudaGetLastError();
}

}  // namespace rlkv
