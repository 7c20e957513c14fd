// Norms of query and key heads and their rotation in one pass, on their own: for packed tokens of training samples, with the
// gradients behind it, and for the chunks of several sequences before they are attended.
//
//   y = R(t) (u * w),   u = x r,   r = 1 / sqrt(mean(x^2) + eps)     per head, x a head's row, R the rotation by position t
// and, with h = R(t)^T dy and g = h * w,
//   dx = r (g - u mean(g u)),   dw = sum over tokens and heads of h * u.
// Either of norm and rotation may be left out.  Everything is computed in fp32 from the bf16 rows and rounded once; nothing of
// the forward pass is kept for the backward pass, which finds r again from the row it reads anyway.
#include "rotary.cuh"
#include "rlkv_chunk.cuh"

namespace rlkv {
namespace {

struct DevicePositions {
    const int* at;  // null: token i stands at position i
    __device__ __forceinline__ int operator()(int token) const { return at ? __ldg(at + token) : token; }
};
struct ChunkPositions {
    ChunkSeqs seqs;
    __device__ __forceinline__ int operator()(int token) const
    {
        const int i = entry_of_token(seqs, token);
        return seqs.len[i] + token - seqs.start[i];
    }
};

// A lane holds eight neighbouring elements of a row, D / 8 lanes a row; where pairs are the halves of the rotated part, the other
// element of each pair is another lane's, and comes by a shuffle.  What a lane multiplies with -- cos, sin, the weights -- stays in
// registers over a token's heads, whose loads are issued several at a time.  Bound by memory (8192 tokens of 32 / 8 heads of 128):
// see the kernels.  (Sixteen elements a thread, pairs in one thread, took 117 and 151 registers and had too few loads in flight:
// 43 us forward and 79 backward.)
template <int D>
struct Lane {
    static constexpr int kLanes = D / 8, kRows = 32 / kLanes;  // of a row, rows of a warp
    int row, column, partner;  // row of the warp, first element, lane with the pairs' other elements
    bool turned, inside;       // rotated at all; pairs lie inside a lane
    float sign;                // of the other element's term in this one's
    __device__ __forceinline__ Lane(const NormRotaryArgs& a)
    {
        const int lane = threadIdx.x & 31, piece = lane % kLanes, half = a.rot / 16;  // lanes of half the rotated part
        row = lane / kLanes;
        column = piece * 8;
        turned = a.table && column < a.rot;
        inside = a.interleaved;  // (the same for the whole warp, whose lanes all take part in the shuffles otherwise)
        const bool low = piece < half;
        partner = turned && !inside ? lane + (low ? half : -half) : lane;
        sign = !turned ? 0.f : low ? -1.f : 1.f;
    }
    // cos and sin of the lane's elements, sin with the sign of the other element's term
    __device__ __forceinline__ void angles(const NormRotaryArgs& a, int t, float (&c)[8], float (&s)[8]) const
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            c[j] = 1.f;
            s[j] = 0.f;
        }
        if (!turned) return;
        const float* row_of = a.table + (long long)t * a.rot;
        if (inside) {  // four pairs
            const float4* p = reinterpret_cast<const float4*>(row_of + column);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float4 v = __ldg(p + j);
                c[4 * j] = c[4 * j + 1] = v.x;
                c[4 * j + 2] = c[4 * j + 3] = v.z;
                s[4 * j] = -v.y;
                s[4 * j + 1] = v.y;
                s[4 * j + 2] = -v.w;
                s[4 * j + 3] = v.w;
            }
        } else {  // eight
            const float4* p = reinterpret_cast<const float4*>(row_of + (sign < 0.f ? column : column - a.rot / 2) * 2);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 v = __ldg(p + j);
                c[2 * j] = v.x;
                c[2 * j + 1] = v.z;
                s[2 * j] = sign * v.y;
                s[2 * j + 1] = sign * v.w;
            }
        }
    }
    // the other elements of the pairs of the lane's eight
    __device__ __forceinline__ void others(const uint4& own, float (&x)[8]) const
    {
        if (inside) {
            float y[8];
            unpack8(own, y);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = y[j ^ 1];
            return;
        }
        uint4 p;
        p.x = __shfl_sync(0xffffffffu, own.x, partner);
        p.y = __shfl_sync(0xffffffffu, own.y, partner);
        p.z = __shfl_sync(0xffffffffu, own.z, partner);
        p.w = __shfl_sync(0xffffffffu, own.w, partner);
        unpack8(p, x);
    }
};

__device__ __forceinline__ float lanes_sum(float x, int lanes)
{
    for (int o = 1; o < lanes; o <<= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// A lane's way to its rows: copies to shared memory that run kAhead steps before it reads them (its own pieces only: nothing to
// wait for but its own copies).  A step is kRows heads of a token; steps go through a warp's heads and then to its next token.
__device__ __forceinline__ void copy16(void* dst, const void* src, bool take)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(dst))), "l"(src), "r"(take ? 16 : 0)
                 : "memory");
}
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_landed() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

struct Steps {
    int e, h;  // token and first head of the next step
    __device__ __forceinline__ void next(int rows, int head0, int head1, int stride)
    {
        h += rows;
        if (h >= head1) {
            h = head0;
            e += stride;
        }
    }
};

// blockIdx.y: `heads` query heads, or KV heads; the block's warps take tokens blockIdx.x * 8 + warp and so on.
template <int D, class Positions>
__global__ void __launch_bounds__(256, 4) norm_rotary_kernel(const __grid_constant__ NormRotaryArgs a, const __grid_constant__ Positions positions, const int heads,
                                                             const int q_groups)
{
    constexpr int kAhead = 4, kRows = Lane<D>::kRows;
    __shared__ uint4 ring[kAhead][256];
    const bool is_q = (int)blockIdx.y < q_groups;
    const int of = is_q ? a.q_heads : a.kv_heads;
    const int head0 = ((int)blockIdx.y - (is_q ? 0 : q_groups)) * heads, head1 = min(of, head0 + heads);
    const __nv_bfloat16* rows = is_q ? a.q : a.k;
    const long long row_stride = is_q ? a.q_stride : a.k_stride;
    __nv_bfloat16* out = is_q ? a.q_out : a.k_out;
    const float* weight = is_q ? a.q_weight : a.k_weight;
    const Lane<D> lane(a);
    const int stride = gridDim.x * 8;
    Steps ahead{(int)(blockIdx.x * 8 + (threadIdx.x >> 5)), head0}, at = ahead;
    auto issue = [&](int slot) {
        const int h = ahead.h + lane.row;
        if (ahead.e < a.n) copy16(&ring[slot][threadIdx.x], rows + ahead.e * row_stride + min(h, head1 - 1) * D + lane.column, h < head1);
        copies_issued();
        ahead.next(kRows, head0, head1, stride);
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) issue(i);
    float w[8], wo[8], c[8], s[8];
    if (weight) {
        load8(weight + lane.column, w);
        load8(weight + (lane.partner % Lane<D>::kLanes) * 8, wo);
    }
    int t = -1;
    for (int slot = 0; at.e < a.n; slot = slot + 1 == kAhead ? 0 : slot + 1) {
        const int h = at.h + lane.row;
        if (at.h == head0) {
            t = positions(at.e);
            if (t >= a.positions) t = -1;  // of no document: the token's rows stay as they are
            if (t >= 0) {
                lane.angles(a, t, c, s);
                if (weight) {  // y = r (x c w + x' s w')
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        c[j] *= w[j];
                        s[j] *= lane.inside ? wo[j ^ 1] : wo[j];
                    }
                }
            }
        }
        copies_landed<kAhead - 1>();
        const uint4 x = ring[slot][threadIdx.x];
        issue(slot);
        if (t >= 0) {
            float y[8], z[8], sum = 0.f;
            unpack8(x, y);
            lane.others(x, z);
            float r = 1.f;
            if (weight) {
#pragma unroll
                for (int j = 0; j < 8; ++j) sum = fmaf(y[j], y[j], sum);
                r = rsqrtf(lanes_sum(sum, Lane<D>::kLanes) * (1.f / D) + a.eps);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = r * fmaf(z[j], s[j], y[j] * c[j]);
            if (h < head1) *reinterpret_cast<uint4*>(out + ((long long)at.e * of + h) * D + lane.column) = pack8(y);
        }
        at.next(kRows, head0, head1, stride);
    }
}

// The same walk.  A lane adds up its eight columns of dw over all steps, and the block's sums go to `partials`, whose order the
// launch fixes.
template <int D>
__global__ void __launch_bounds__(256, 3) norm_rotary_backward_kernel(const __grid_constant__ NormRotaryArgs a, const int heads, const int q_groups)
{
    constexpr int kAhead = 5, kRows = Lane<D>::kRows, kLanes = Lane<D>::kLanes;
    __shared__ uint4 ring[kAhead][2][256];
    const bool is_q = (int)blockIdx.y < q_groups;
    const int of = is_q ? a.q_heads : a.kv_heads;
    const int head0 = ((int)blockIdx.y - (is_q ? 0 : q_groups)) * heads, head1 = min(of, head0 + heads);
    const __nv_bfloat16 *rows = is_q ? a.q : a.k, *grads = is_q ? a.dq_out : a.dk_out;
    const long long row_stride = is_q ? a.q_stride : a.k_stride, to_stride = is_q ? a.dq_stride : a.dk_stride;
    __nv_bfloat16* to = is_q ? a.dq : a.dk;
    const float* weight = is_q ? a.q_weight : a.k_weight;
    const Lane<D> lane(a);
    const int stride = gridDim.x * 8;
    Steps ahead{(int)(blockIdx.x * 8 + (threadIdx.x >> 5)), head0}, at = ahead;
    auto issue = [&](int slot) {
        const int h = ahead.h + lane.row, hc = min(h, head1 - 1);
        if (ahead.e < a.n) {
            copy16(&ring[slot][0][threadIdx.x], grads + ((long long)ahead.e * of + hc) * D + lane.column, h < head1);
            if (weight) copy16(&ring[slot][1][threadIdx.x], rows + ahead.e * row_stride + hc * D + lane.column, h < head1);
        }
        copies_issued();
        ahead.next(kRows, head0, head1, stride);
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) issue(i);
    float w[8], d[8], c[8], s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        w[j] = 1.f;
        d[j] = 0.f;
    }
    if (weight) load8(weight + lane.column, w);
    int t = -1;
    for (int slot = 0; at.e < a.n; slot = slot + 1 == kAhead ? 0 : slot + 1) {
        const int h = at.h + lane.row;
        if (at.h == head0) {
            t = a.position ? __ldg(a.position + at.e) : at.e;
            if (t >= a.positions) t = -1;
            if (t >= 0) lane.angles(a, t, c, s);  // (turned back: sin with the other sign)
        }
        copies_landed<kAhead - 1>();
        const uint4 g = ring[slot][0][threadIdx.x], x = ring[slot][1][threadIdx.x];
        issue(slot);
        if (t >= 0) {
            float y[8], z[8];
            unpack8(g, y);
            lane.others(g, z);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = fmaf(-s[j], z[j], y[j] * c[j]);  // h
            if (weight) {
                unpack8(x, z);
                float square = 0.f, dot = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    square = fmaf(z[j], z[j], square);
                    dot = fmaf(y[j] * w[j], z[j], dot);
                }
                square = lanes_sum(square, kLanes);
                dot = lanes_sum(dot, kLanes);
                const float r = rsqrtf(square * (1.f / D) + a.eps), back = dot * r * r * (1.f / D);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    d[j] = fmaf(y[j] * r, z[j], d[j]);
                    y[j] = r * fmaf(-z[j], back, y[j] * w[j]);
                }
            }
            if (h < head1) *reinterpret_cast<uint4*>(to + at.e * to_stride + h * D + lane.column) = pack8(y);
        }
        at.next(kRows, head0, head1, stride);
    }
    if (!a.partials) return;
    grid_dep_launch();
    float(*sums)[D] = reinterpret_cast<float(*)[D]>(ring);
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int o = kLanes; o < 32; o <<= 1) d[j] += __shfl_xor_sync(0xffffffffu, d[j], o);
    __syncthreads();  // (no copy is on its way any more: each wait above leaves only those behind the last step, which copy nothing)
    if (lane.row == 0)
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[threadIdx.x >> 5][lane.column + j] = d[j];
    __syncthreads();
    if (threadIdx.x < D) {
        float all = 0.f;
#pragma unroll
        for (int x = 0; x < 8; ++x) all += sums[x][threadIdx.x];
        a.partials[((long long)blockIdx.y * gridDim.x + blockIdx.x) * D + threadIdx.x] = all;
    }
}

// dw of the queries' norm (blockIdx.y 0) and the keys' (1): eight columns a block, the blocks' sums added up in a fixed order.
__global__ void __launch_bounds__(256) norm_weights_kernel(const float* partials, int q_blocks, int k_blocks, int head_dim, float* dq_weight, float* dk_weight)
{
    __shared__ float sums[32][9];
    grid_dep_wait();
    const bool is_q = blockIdx.y == 0;
    float* to = is_q ? dq_weight : dk_weight;
    if (!to) return;
    const int n = is_q ? q_blocks : k_blocks, c = threadIdx.x & 7, r = threadIdx.x >> 3;
    const float* p = partials + (is_q ? 0 : (long long)q_blocks * head_dim) + blockIdx.x * 8 + c;
    float s = 0.f;
#pragma unroll 8
    for (int b = r; b < n; b += 32) s += p[(long long)b * head_dim];
    sums[r][c] = s;
    __syncthreads();
    if (threadIdx.x < 8) {
        float all = 0.f;
#pragma unroll
        for (int x = 0; x < 32; ++x) all += sums[x][c];
        to[blockIdx.x * 8 + c] = all;
    }
}

// How a launch is cut: as many heads to a block's walk as leave the GPU filled (they share the angles), at most `most` blocks.
struct Cut {
    int heads, q_groups, groups, columns;
};
Cut cut_heads(const NormRotaryArgs& a, int most)
{
    const int rows = a.head_dim == 128 ? 2 : 4, tiles = (a.n + 7) / 8;
    Cut c;
    auto groups = [&](int h) { return (a.q_heads + h - 1) / h + (a.kv_heads + h - 1) / h; };
    c.heads = rows;
    while (c.heads < 16 && ((long long)tiles * groups(2 * c.heads) >= most || groups(c.heads) > most)) c.heads *= 2;
    c.q_groups = (a.q_heads + c.heads - 1) / c.heads;
    c.groups = groups(c.heads);
    c.columns = most / c.groups < tiles ? most / c.groups : tiles;
    return c;
}

template <class Positions>
cudaError_t launch_forward(const NormRotaryArgs& a, const Positions& positions, cudaStream_t stream)
{
    const Cut c = cut_heads(a, kMaxNormBlocks);
    const dim3 grid(c.columns, c.groups);
    if (a.head_dim == 128) norm_rotary_kernel<128, Positions><<<grid, 256, 0, stream>>>(a, positions, c.heads, c.q_groups);
    else norm_rotary_kernel<64, Positions><<<grid, 256, 0, stream>>>(a, positions, c.heads, c.q_groups);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_norm_rotary(const NormRotaryArgs& a, cudaStream_t stream) { return launch_forward(a, DevicePositions{a.position}, stream); }

cudaError_t launch_norm_rotary_chunks(const NormRotaryArgs& a, const ChunkSeqs& seqs, cudaStream_t stream)
{
    return launch_forward(a, ChunkPositions{seqs}, stream);
}

cudaError_t launch_norm_rotary_backward(const NormRotaryArgs& args, cudaStream_t stream)
{
    NormRotaryArgs a = args;
    const Cut c = cut_heads(a, 148 * 3);
    if (!a.dq_weight && !a.dk_weight) a.partials = nullptr;
    const dim3 grid(c.columns, c.groups);
    if (a.head_dim == 128) norm_rotary_backward_kernel<128><<<grid, 256, 0, stream>>>(a, c.heads, c.q_groups);
    else norm_rotary_backward_kernel<64><<<grid, 256, 0, stream>>>(a, c.heads, c.q_groups);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || !a.partials) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(a.head_dim / 8, 2);
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, norm_weights_kernel, (const float*)a.partials, c.columns * c.q_groups, c.columns * (c.groups - c.q_groups), a.head_dim, a.dq_weight, a.dk_weight);
}

}  // namespace rlkv
