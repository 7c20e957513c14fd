// Internal definitions of prompt attention (rlkv_prompt_*): shared by its host side and its kernels.
#pragma once

#include <limits.h>

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
    float2* stats;                       // scratch, [q_heads][q_tokens]: lse * log2(e), sum over head_dim of dout * out
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

// Status codes of prompt attention (device error word): which wait ran out.
enum : int { kPromptWaitLoad = 101, kPromptWaitProduct = 102, kPromptWaitSoftmax = 103, kPromptWaitStage = 104, kPromptWaitDrain = 105,
             kPromptSmemMisaligned = 106 };

// Tiles of `rows` queries (or keys), numbered from the LAST tile of the last document backwards (a causal document's last
// tiles are its longest, and the longest are best started first).  Called by one whole warp; returns false where there
// are no more than `index` tiles, else tile `tile` of the document in `range`.
__device__ __forceinline__ bool find_tile(const PromptArgs& a, bool keys, int rows, int index, DocRange& range, int& tile)
{
    const int lane = threadIdx.x & 31;
    auto tiles_of = [&](const DocRange& r) { return ((keys ? r.kn : r.qn) + rows - 1) / rows; };
    if (a.n_docs == 1) {
        range = doc_range(a, 0);
        tile = tiles_of(range) - 1 - index;
        return tile >= 0;
    }
    auto scan = [&](int x) {  // inclusive, over the lanes
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        return x;
    };
    int left = index;
    if (a.n_docs <= 64) {  // a document per lane: one trip to memory, the range comes from its lane
        for (int top = a.n_docs; top > 0; top -= 32) {
            const int d = top - 1 - lane;
            const DocRange r = d >= 0 ? doc_range(a, d) : DocRange{0, 0, 0, 0, 0};
            const int n = tiles_of(r), upto = scan(n);
            const unsigned hit = __ballot_sync(0xffffffffu, upto > left);
            if (hit) {
                const int owner = __ffs(hit) - 1;
                range.q0 = __shfl_sync(0xffffffffu, r.q0, owner);
                range.qn = __shfl_sync(0xffffffffu, r.qn, owner);
                range.k0 = __shfl_sync(0xffffffffu, r.k0, owner);
                range.kn = __shfl_sync(0xffffffffu, r.kn, owner);
                range.prefix = __shfl_sync(0xffffffffu, r.prefix, owner);
                tile = __shfl_sync(0xffffffffu, upto, owner) - 1 - left;
                return true;
            }
            left -= __shfl_sync(0xffffffffu, upto, 31);
        }
        return false;
    }
    for (int top = a.n_docs; top > 0; top -= 256) {  // eight neighbouring documents per lane
        int n[8], sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int d = top - 1 - lane * 8 - i;
            n[i] = d >= 0 ? tiles_of(doc_range(a, d)) : 0;
            sum += n[i];
        }
        const int upto = scan(sum);
        const unsigned hit = __ballot_sync(0xffffffffu, upto > left);
        if (hit) {
            const int owner = __ffs(hit) - 1;
            int d = 0, t = 0;
            if (lane == owner) {
                int rest = left - (upto - sum), i = 0;
                while (rest >= n[i]) rest -= n[i++];
                d = top - 1 - lane * 8 - i;
                t = n[i] - 1 - rest;
            }
            range = doc_range(a, __shfl_sync(0xffffffffu, d, owner));
            tile = __shfl_sync(0xffffffffu, t, owner);
            return true;
        }
        left -= __shfl_sync(0xffffffffu, upto, 31);
    }
    return false;
}

// The queries of a CTA of the forward or rows kernel: two sub-tiles of up to 128, and the key tiles they see.  Where the
// query heads of a KV head pair up, the sub-tiles are the same 128 queries of two heads (both read the same keys to
// the last one, and short documents waste less of a tile); else 256 queries of one head.
struct RowTile {
    int valid, kv_head, n_sub;
    int head[2], q0[2], rows[2], pos0[2];  // per sub-tile: head, first packed query, how many, position of the first
    int k0, kn, prefix;                    // the document's keys
    int a_end, b0, n_tiles;                // key tiles of the CTA: 0 .. a_end-1, then from b0 on
    int sub_a[2], sub_b[2], sub_e[2];      // those a sub-tile needs: 0 .. a-1 and b .. e-1
};
__host__ __device__ inline bool heads_pair(int group) { return group % 2 == 0; }
inline long long row_tile_blocks(const PromptArgs& a)
{
    const bool pair = heads_pair(a.group);
    return ((long long)a.q_tokens / (pair ? 128 : 256) + (a.n_docs < a.q_tokens ? a.n_docs : a.q_tokens)) * (pair ? a.q_heads / 2 : a.q_heads);
}
// One whole warp; `keys`: keys of a tile.
__device__ __forceinline__ void find_row_tile(const PromptArgs& a, int keys, RowTile& t)
{
    const bool pair = heads_pair(a.group);
    const int units = pair ? a.q_heads / 2 : a.q_heads, span = pair ? 128 : 256;
    int tile = 0;
    DocRange r;
    const bool valid = find_tile(a, false, span, blockIdx.x / units, r, tile);
    if ((threadIdx.x & 31) != 0) return;
    t.valid = valid;
    if (!valid) return;
    const int unit = blockIdx.x % units, first = tile * span;
    t.k0 = r.k0;
    t.kn = r.kn;
    t.prefix = r.prefix;
    t.n_sub = pair || r.qn - first > 128 ? 2 : 1;
    t.kv_head = (pair ? 2 * unit : unit) / a.group;
    const bool full = a.full[t.kv_head] != 0;
    int hi = 0;
    for (int w = 0; w < 2; ++w) {
        const int from = first + (pair ? 0 : w * 128);
        t.head[w] = pair ? 2 * unit + w : unit;
        t.q0[w] = r.q0 + from;
        t.rows[w] = max(0, min(128, r.qn - from));
        t.pos0[w] = from + r.kn - r.qn;
        const int seen = t.rows[w] > 0 ? max(0, min(r.kn, max(t.pos0[w] + t.rows[w], r.prefix))) : 0;
        const int e = (seen + keys - 1) / keys;
        t.sub_a[w] = full ? e : min(e, (a.sink + keys - 1) / keys);
        t.sub_b[w] = max(t.sub_a[w], max(0, t.pos0[w] - a.window + 1) / keys);
        t.sub_e[w] = max(e, t.sub_b[w]);
        hi = max(hi, e);
    }
    t.a_end = full ? hi : min(hi, (a.sink + keys - 1) / keys);
    t.b0 = full ? hi : max(t.a_end, max(0, t.pos0[0] - a.window + 1) / keys);
    t.n_tiles = t.a_end + max(0, hi - t.b0);
}

// Bits c of 32 with lo <= c < hi.
__device__ __forceinline__ uint32_t range_bits(int lo, int hi)
{
    const uint32_t below_hi = hi >= 32 ? ~0u : hi <= 0 ? 0u : (1u << hi) - 1u;
    const uint32_t below_lo = lo >= 32 ? ~0u : lo <= 0 ? 0u : (1u << lo) - 1u;
    return below_hi & ~below_lo;
}

cudaError_t launch_prompt_forward(const PromptArgs& a, const CUtensorMap& map_q, const CUtensorMap& map_k, const CUtensorMap& map_v,
                                  int head_dim, cudaStream_t stream);
cudaError_t prepare_prompt_kernels(int head_dim);
cudaError_t launch_prompt_backward(const PromptArgs& a, const CUtensorMap& map_q, const CUtensorMap& map_k, const CUtensorMap& map_v,
                                   const CUtensorMap& map_do, int head_dim, cudaStream_t stream);
cudaError_t prepare_prompt_backward(int head_dim);

}  // namespace rlkv
