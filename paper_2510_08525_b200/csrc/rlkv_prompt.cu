// Host side of prompt attention (rlkv_prompt_* in include/rlkv.h): the handle keeps what a model fixes once
// (heads, masks, scores) and the scratch of the backward pass; every call names its tensors.
#include <math.h>
#include <string.h>

#include <new>
#include <vector>

#include "rlkv_chunk.cuh"
#include "rlkv_host.cuh"
#include "rlkv_prompt.cuh"

using namespace rlkv;

constexpr int kNormArrivals = 16;  // counters of the norms' gradients in the status area

struct rlkv_prompt {
    int layers, kv_heads, q_heads, head_dim, max_tokens, sink, window, device;
    float softcap;
    bool biased;
    std::vector<uint8_t> is_full;  // [layers*kv_heads]
    uint8_t* dev_base;             // status, then slopes [layers][q_heads], then stats (float2) [q_heads][max_tokens], then the norms' sums
    size_t off_slopes, off_stats, off_norms;
    const float* rotary;           // rlkv_prompt_set_rotary: the caller's table of angles (device), null: none set
    int rotary_rows, rotary_dim, rotary_interleaved;
    const float *q_norm, *k_norm;  // rlkv_prompt_set_norms: the caller's weights (device), null: none set
    float norm_eps;
};

namespace {

constexpr int kMaxPromptTokens = 1 << 24;
constexpr int kMaxDocs = 65535;

int fill_prompt_args(const rlkv_prompt* p, int layer, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                     int64_t v_stride, int q_tokens, int k_tokens, const int* q_starts, const int* k_starts, int n_docs,
                     const int* prefix, const void* out, const float* lse, PromptArgs& a)
{
    if (!p || layer < 0 || layer >= p->layers || !q || !k || !v || !out || !q_starts) return RLKV_EINVAL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out)) return RLKV_EINVAL;
    if (q_tokens < 1 || q_tokens > p->max_tokens || k_tokens < 1 || k_tokens > kMaxPromptTokens || n_docs < 1 || n_docs > kMaxDocs)
        return RLKV_EINVAL;
    const uintptr_t words = reinterpret_cast<uintptr_t>(q_starts) | reinterpret_cast<uintptr_t>(k_starts) |
                            reinterpret_cast<uintptr_t>(prefix) | reinterpret_cast<uintptr_t>(lse);
    if (words & 3) return RLKV_EINVAL;
    const int64_t q_row = (int64_t)p->q_heads * p->head_dim, kv_row = (int64_t)p->kv_heads * p->head_dim;
    if (!q_stride) q_stride = q_row;
    if (!k_stride) k_stride = kv_row;
    if (!v_stride) v_stride = kv_row;
    const int64_t most = (int64_t)1 << 30;  // a tensor map's strides end at 2^40 bytes
    if (q_stride < q_row || k_stride < kv_row || v_stride < kv_row || q_stride % 8 || k_stride % 8 || v_stride % 8 ||
        q_stride > most || k_stride > most || v_stride > most)
        return RLKV_EINVAL;
    memset(&a, 0, sizeof a);
    a.q = static_cast<const __nv_bfloat16*>(q);
    a.k = static_cast<const __nv_bfloat16*>(k);
    a.v = static_cast<const __nv_bfloat16*>(v);
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.q_tokens = q_tokens;
    a.k_tokens = k_tokens;
    a.q_starts = q_starts;
    a.k_starts = k_starts ? k_starts : q_starts;
    a.prefix = prefix;
    a.n_docs = n_docs;
    a.group = p->q_heads / p->kv_heads;
    a.q_heads = p->q_heads;
    a.kv_heads = p->kv_heads;
    a.sink = p->sink;
    a.window = p->window;
    a.scale = 1.f / sqrtf((float)p->head_dim);
    a.softcap = p->softcap;
    a.slopes = p->biased ? reinterpret_cast<const float*>(p->dev_base + p->off_slopes) + (size_t)layer * p->q_heads : nullptr;
    a.out = static_cast<__nv_bfloat16*>(const_cast<void*>(out));
    a.lse = const_cast<float*>(lse);
    a.stats = reinterpret_cast<float2*>(p->dev_base + p->off_stats);
    a.status = reinterpret_cast<int*>(p->dev_base);
    for (int h = 0; h < p->kv_heads; ++h) a.full[h] = p->is_full[(size_t)layer * p->kv_heads + h] ? 1 : 0;
    return RLKV_OK;
}

}  // namespace

int rlkv::encode_heads_map(CUtensorMap* map, const void* base, long long tokens, int heads, int head_dim, int64_t stride, int box_heads,
                           int box_tokens)
{
    typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                      const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                      CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static void* volatile fn = nullptr;  // (two threads that look it up at once find the same)
    if (!fn) {
        void* found = nullptr;
        cudaDriverEntryPointQueryResult q;
        RLKV_CUDA(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &found, cudaEnableDefault, &q));
        if (!found || q != cudaDriverEntryPointSuccess) return cuda_fail(cudaErrorNotSupported, "cuTensorMapEncodeTiled lookup");
        fn = found;
    }
    const cuuint64_t dims[3] = {(cuuint64_t)head_dim, (cuuint64_t)heads, (cuuint64_t)tokens};
    const cuuint64_t strides[2] = {(cuuint64_t)head_dim * 2, (cuuint64_t)stride * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_tokens};
    const cuuint32_t one[3] = {1, 1, 1};
    const CUresult r = reinterpret_cast<EncodeTiledFn>(fn)(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides,
                                                           box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                                           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        snprintf(g_cuda_text, sizeof g_cuda_text, "cuTensorMapEncodeTiled (heads) failed with CUresult %d", (int)r);
        return RLKV_ECUDA;
    }
    return RLKV_OK;
}

extern "C" {

int rlkv_prompt_create(rlkv_prompt** out, int layers, int kv_heads, int q_heads, int head_dim, int max_tokens,
                       const uint8_t* head_is_full, int sink, int window, float softcap, const float* slopes)
{
    if (!out) return RLKV_EINVAL;
    *out = nullptr;
    if (!head_is_full || layers < 1 || layers > 65535 || kv_heads < 1 || kv_heads > kMaxKvHeads || q_heads < 1 ||
        q_heads % kv_heads != 0 || q_heads / kv_heads > kMaxGroup || (head_dim != 64 && head_dim != 128) || max_tokens < 1 ||
        max_tokens > kMaxPromptTokens || sink < 0 || window < 1 || (long long)sink + window > (1 << 24))
        return RLKV_EINVAL;
    if (!(softcap >= 0.f) || (softcap != 0.f && (softcap < 1e-3f || softcap > 1e3f))) return RLKV_EINVAL;
    const size_t count = (size_t)layers * q_heads;
    bool biased = false;
    if (slopes)
        for (size_t i = 0; i < count; ++i) {
            if (!(fabsf(slopes[i]) <= 1e6f)) return RLKV_EINVAL;
            if (slopes[i] != 0.f) biased = true;
        }
    rlkv_prompt* p = new (std::nothrow) rlkv_prompt();
    if (!p) return RLKV_ENOMEM;
    p->layers = layers; p->kv_heads = kv_heads; p->q_heads = q_heads; p->head_dim = head_dim; p->max_tokens = max_tokens;
    p->sink = sink; p->window = window; p->softcap = softcap; p->biased = biased; p->dev_base = nullptr;
    p->rotary = p->q_norm = p->k_norm = nullptr; p->rotary_rows = p->rotary_dim = p->rotary_interleaved = 0; p->norm_eps = 0.f;
    try {
        p->is_full.assign(head_is_full, head_is_full + (size_t)layers * kv_heads);
    } catch (const std::bad_alloc&) {
        delete p;
        return RLKV_ENOMEM;
    }
    p->off_slopes = 1024;
    p->off_stats = align_up(p->off_slopes + count * sizeof(float), 1024);
    p->off_norms = align_up(p->off_stats + (size_t)max_tokens * q_heads * sizeof(float2), 1024);
    const size_t total = p->off_norms + (size_t)kMaxNormBlocks * head_dim * sizeof(float);
    cudaError_t e = cudaGetDevice(&p->device);
    if (e != cudaSuccess) { delete p; return cuda_fail(e, "device query"); }
    void* mem = nullptr;
    e = cudaMalloc(&mem, total);
    if (e != cudaSuccess) { cudaGetLastError(); delete p; return RLKV_ENOMEM; }
    p->dev_base = static_cast<uint8_t*>(mem);
    e = cudaMemset(mem, 0, p->off_stats);
    if (e == cudaSuccess && biased) e = cudaMemcpy(p->dev_base + p->off_slopes, slopes, count * sizeof(float), cudaMemcpyHostToDevice);
    if (e == cudaSuccess) e = prepare_prompt_kernels(head_dim);
    if (e == cudaSuccess) e = prepare_prompt_backward(head_dim);
    if (e == cudaSuccess) e = prepare_norm_backward();
    if (e == cudaSuccess) e = cudaDeviceSynchronize();  // the memset is done before a call on any stream
    if (e != cudaSuccess) {
        cudaFree(mem);
        delete p;
        return cuda_fail(e, "rlkv_prompt_create");
    }
    *out = p;
    return RLKV_OK;
}

int rlkv_prompt_destroy(rlkv_prompt* p)
{
    if (!p) return RLKV_EINVAL;
    DeviceGuard g(p->device);
    cudaDeviceSynchronize();
    cudaFree(p->dev_base);
    delete p;
    return RLKV_OK;
}

int rlkv_prompt_attention(rlkv_prompt* p, int layer, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                          const void* v, int64_t v_stride, int q_tokens, int k_tokens, const int* q_starts,
                          const int* k_starts, int n_docs, const int* prefix, void* out, float* lse, void* stream)
{
    PromptArgs a;
    const int rc = fill_prompt_args(p, layer, q, q_stride, k, k_stride, v, v_stride, q_tokens, k_tokens, q_starts, k_starts, n_docs,
                                    prefix, out, lse, a);
    if (rc) return rc;
    DeviceGuard g(p->device);
    if (!g.ok) return RLKV_ECUDA;
    CUtensorMap map_q, map_k, map_v;
    int e = encode_heads_map(&map_q, q, q_tokens, p->q_heads, p->head_dim, a.q_stride, 1, 128);
    if (!e) e = encode_heads_map(&map_k, k, k_tokens, p->kv_heads, p->head_dim, a.k_stride, 1, 128);
    if (!e) e = encode_heads_map(&map_v, v, k_tokens, p->kv_heads, p->head_dim, a.v_stride, 1, 128);
    if (e) return e;
    RLKV_CUDA(launch_prompt_forward(a, map_q, map_k, map_v, p->head_dim, static_cast<cudaStream_t>(stream)));
    return RLKV_OK;
}

int rlkv_prompt_attention_backward(rlkv_prompt* p, int layer, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                   const void* v, int64_t v_stride, int q_tokens, int k_tokens, const int* q_starts,
                                   const int* k_starts, int n_docs, const int* prefix, const void* out, const float* lse,
                                   const void* dout, void* dq, void* dk, void* dv, void* stream)
{
    if (!lse || !dout || !dq || !dk || !dv || !aligned16(dout) || !aligned16(dq) || !aligned16(dk) || !aligned16(dv)) return RLKV_EINVAL;
    PromptArgs a;
    const int rc = fill_prompt_args(p, layer, q, q_stride, k, k_stride, v, v_stride, q_tokens, k_tokens, q_starts, k_starts, n_docs,
                                    prefix, out, lse, a);
    if (rc) return rc;
    a.dout = static_cast<const __nv_bfloat16*>(dout);
    a.dq = static_cast<__nv_bfloat16*>(dq);
    a.dk = static_cast<__nv_bfloat16*>(dk);
    a.dv = static_cast<__nv_bfloat16*>(dv);
    DeviceGuard g(p->device);
    if (!g.ok) return RLKV_ECUDA;
    CUtensorMap map_q, map_k, map_v, map_do;
    int e = encode_heads_map(&map_q, q, q_tokens, p->q_heads, p->head_dim, a.q_stride, 1, 128);
    if (!e) e = encode_heads_map(&map_k, k, k_tokens, p->kv_heads, p->head_dim, a.k_stride, 1, 128);
    if (!e) e = encode_heads_map(&map_v, v, k_tokens, p->kv_heads, p->head_dim, a.v_stride, 1, 128);
    if (!e) e = encode_heads_map(&map_do, dout, q_tokens, p->q_heads, p->head_dim, (int64_t)p->q_heads * p->head_dim, 1, 128);
    if (e) return e;
    RLKV_CUDA(launch_prompt_backward(a, map_q, map_k, map_v, map_do, p->head_dim, static_cast<cudaStream_t>(stream)));
    return RLKV_OK;
}

int rlkv_prompt_set_rotary(rlkv_prompt* p, const void* table, int positions, int rot_dim, int interleaved)
{
    if (!p) return RLKV_EINVAL;
    if (table && (positions < 1 || rot_dim < 16 || rot_dim % 16 || rot_dim > p->head_dim || !on_device(table, p->device))) return RLKV_EINVAL;
    p->rotary = static_cast<const float*>(table);
    p->rotary_rows = table ? positions : 0;
    p->rotary_dim = rot_dim;
    p->rotary_interleaved = interleaved ? 1 : 0;
    return RLKV_OK;
}

int rlkv_prompt_set_norms(rlkv_prompt* p, const float* q_weight, const float* k_weight, float eps)
{
    if (!p) return RLKV_EINVAL;
    if (q_weight || k_weight) {
        if (!(eps > 0.f) || !(eps <= 1.f)) return RLKV_EINVAL;
        for (const float* w : {q_weight, k_weight})
            if (w && !on_device(w, p->device)) return RLKV_EINVAL;
    }
    p->q_norm = q_weight;
    p->k_norm = k_weight;
    p->norm_eps = eps;
    return RLKV_OK;
}

// Strides of rows of queries and keys: 0 stands for contiguous tokens, 2^30 elements are the most, so that no token's offset leaves 64 bits.
static bool row_strides(const rlkv_prompt* p, int64_t& q_stride, int64_t& k_stride)
{
    const int64_t q_row = (int64_t)p->q_heads * p->head_dim, kv_row = (int64_t)p->kv_heads * p->head_dim, most = (int64_t)1 << 30;
    if (!q_stride) q_stride = q_row;
    if (!k_stride) k_stride = kv_row;
    return q_stride >= q_row && k_stride >= kv_row && q_stride % 8 == 0 && k_stride % 8 == 0 && q_stride <= most && k_stride <= most;
}

// What the two directions share.
static int norm_rotary_args(const rlkv_prompt* p, int layer, const void* q, int64_t q_stride, const void* k, int64_t k_stride, int tokens,
                            const int* positions, NormRotaryArgs& a)
{
    if (!p || layer < 0 || layer >= p->layers || !q || !k || !aligned16(q) || !aligned16(k) || tokens < 1 || tokens > p->max_tokens ||
        (reinterpret_cast<uintptr_t>(positions) & 3))
        return RLKV_EINVAL;
    if (!p->rotary && !p->q_norm && !p->k_norm) return RLKV_EINVAL;
    if (!row_strides(p, q_stride, k_stride)) return RLKV_EINVAL;
    memset(&a, 0, sizeof a);
    a.q = static_cast<const __nv_bfloat16*>(q);
    a.k = static_cast<const __nv_bfloat16*>(k);
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.table = p->rotary;
    a.positions = p->rotary ? p->rotary_rows : INT_MAX;
    a.rot = p->rotary_dim;
    a.interleaved = p->rotary_interleaved;
    a.q_weight = p->q_norm ? p->q_norm + (size_t)layer * p->head_dim : nullptr;
    a.k_weight = p->k_norm ? p->k_norm + (size_t)layer * p->head_dim : nullptr;
    a.eps = p->norm_eps;
    a.position = positions;
    a.n = tokens;
    a.q_heads = p->q_heads;
    a.kv_heads = p->kv_heads;
    a.head_dim = p->head_dim;
    return RLKV_OK;
}

int rlkv_prompt_rotate(rlkv_prompt* p, int layer, const void* q, int64_t q_stride, const void* k, int64_t k_stride, int tokens,
                       const int* positions, void* q_out, void* k_out, void* stream)
{
    NormRotaryArgs a;
    const int rc = norm_rotary_args(p, layer, q, q_stride, k, k_stride, tokens, positions, a);
    if (rc) return rc;
    if (!q_out || !k_out || !aligned16(q_out) || !aligned16(k_out)) return RLKV_EINVAL;
    a.q_out = static_cast<__nv_bfloat16*>(q_out);
    a.k_out = static_cast<__nv_bfloat16*>(k_out);
    DeviceGuard g(p->device);
    if (!g.ok) return RLKV_ECUDA;
    RLKV_CUDA(launch_norm_rotary(a, static_cast<cudaStream_t>(stream)));
    return RLKV_OK;
}

int rlkv_prompt_rotate_backward(rlkv_prompt* p, int layer, const void* q, int64_t q_stride, const void* k, int64_t k_stride, int tokens,
                                const int* positions, const void* dq_out, const void* dk_out, void* dq, int64_t dq_stride, void* dk,
                                int64_t dk_stride, float* dq_weight, float* dk_weight, void* stream)
{
    NormRotaryArgs a;
    const int rc = norm_rotary_args(p, layer, q, q_stride, k, k_stride, tokens, positions, a);
    if (rc) return rc;
    if (!dq_out || !dk_out || !dq || !dk || !aligned16(dq_out) || !aligned16(dk_out) || !aligned16(dq) || !aligned16(dk)) return RLKV_EINVAL;
    if ((reinterpret_cast<uintptr_t>(dq_weight) | reinterpret_cast<uintptr_t>(dk_weight)) & 3) return RLKV_EINVAL;
    if ((dq_weight && !p->q_norm) || (dk_weight && !p->k_norm)) return RLKV_EINVAL;
    if (!row_strides(p, dq_stride, dk_stride)) return RLKV_EINVAL;
    a.dq_out = static_cast<const __nv_bfloat16*>(dq_out);
    a.dk_out = static_cast<const __nv_bfloat16*>(dk_out);
    a.dq = static_cast<__nv_bfloat16*>(dq);
    a.dk = static_cast<__nv_bfloat16*>(dk);
    a.dq_stride = dq_stride;
    a.dk_stride = dk_stride;
    a.dq_weight = dq_weight;
    a.dk_weight = dk_weight;
    a.partials = reinterpret_cast<float*>(p->dev_base + p->off_norms);
    a.arrived = reinterpret_cast<int*>(p->dev_base) + kNormArrivals;
    DeviceGuard g(p->device);
    if (!g.ok) return RLKV_ECUDA;
    RLKV_CUDA(launch_norm_rotary_backward(a, static_cast<cudaStream_t>(stream)));
    return RLKV_OK;
}

int rlkv_prompt_kernel_status(rlkv_prompt* p, int* status_out)
{
    if (!p || !status_out) return RLKV_EINVAL;
    DeviceGuard g(p->device);
    if (!g.ok) return RLKV_ECUDA;
    RLKV_CUDA(cudaDeviceSynchronize());
    RLKV_CUDA(cudaMemcpy(status_out, p->dev_base, sizeof(int), cudaMemcpyDeviceToHost));
    return RLKV_OK;
}

}  // extern "C"
