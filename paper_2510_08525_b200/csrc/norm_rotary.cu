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
#include "tcgen05.cuh"

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

using tc::add2;
using tc::fma2;
using tc::mul2;

// Eight elements as four pairs, for the instructions that take two fp32 numbers at a time.
struct Eight {
    float2 p[4];
};
__device__ __forceinline__ Eight unpack(const uint4& x)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    Eight e;
#pragma unroll
    for (int j = 0; j < 4; ++j) e.p[j] = make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
    return e;
}
__device__ __forceinline__ uint4 pack(const Eight& e)
{
    return make_uint4(tc::bf16x2(e.p[0].x, e.p[0].y), tc::bf16x2(e.p[1].x, e.p[1].y), tc::bf16x2(e.p[2].x, e.p[2].y), tc::bf16x2(e.p[3].x, e.p[3].y));
}

// A lane holds eight neighbouring elements of a row, D / 8 lanes a row; where pairs are the halves of the rotated part, the other
// element of each pair is another lane's, and comes by a shuffle.  What a lane multiplies with -- cos, sin, the weights -- stays in
// registers over a token's heads.
//
// Bound by memory at large sizes, and next to it by the instructions a row takes, so that both kernels count them: pairs of fp32
// operations, running pointers, and copies to shared memory that go out several steps ahead in place of loads whose registers
// wait.  8192 tokens of 32 / 8 heads of 128: sixteen elements a thread, loads four heads at a time, took 43 us forward and 79
// backward (117 and 151 registers: too few loads in flight); this form with single operations and addresses computed for every row 42
// and 68 (72 % of the issue slots).
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
    // cos and sin of the lane's elements, sin with the sign of the other element's term, from the token's row of the table
    __device__ __forceinline__ void angles(const float* row_of, int rot, Eight& c, Eight& s) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            c.p[j] = make_float2(1.f, 1.f);
            s.p[j] = make_float2(0.f, 0.f);
        }
        if (!turned) return;
        if (inside) {  // four pairs
            const float4* p = reinterpret_cast<const float4*>(row_of + column);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float4 v = p[j];
                c.p[2 * j] = make_float2(v.x, v.x);
                c.p[2 * j + 1] = make_float2(v.z, v.z);
                s.p[2 * j] = make_float2(-v.y, v.y);
                s.p[2 * j + 1] = make_float2(-v.w, v.w);
            }
        } else {  // eight
            const float4* p = reinterpret_cast<const float4*>(row_of + (sign < 0.f ? column : column - rot / 2) * 2);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 v = p[j];
                c.p[j] = make_float2(v.x, v.z);
                s.p[j] = make_float2(sign * v.y, sign * v.w);
            }
        }
    }
    // the other elements of the pairs of the lane's eight
    __device__ __forceinline__ Eight others(const uint4& own, const Eight& mine) const
    {
        if (inside) {
            Eight e;
#pragma unroll
            for (int j = 0; j < 4; ++j) e.p[j] = make_float2(mine.p[j].y, mine.p[j].x);
            return e;
        }
        uint4 p;
        p.x = __shfl_sync(0xffffffffu, own.x, partner);
        p.y = __shfl_sync(0xffffffffu, own.y, partner);
        p.z = __shfl_sync(0xffffffffu, own.z, partner);
        p.w = __shfl_sync(0xffffffffu, own.w, partner);
        return unpack(p);
    }
};

// Sum over a row's lanes of x.x + x.y.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float2 x)
{
    float s = x.x + x.y;
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
}

// Copies of 16 bytes to shared memory (zeros unless `take`).
__device__ __forceinline__ void copy16(void* dst, const void* src, bool take)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(dst))), "l"(src), "r"(take ? 16 : 0)
                 : "memory");
}
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_landed() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// What a warp keeps of the two tokens it has copies on the way for: STEPS times kRows heads of ROWS tensors, a piece to each lane,
// and the token's row of the table.
template <int STEPS, int ROWS>
struct Ring {
    uint4 piece[2][STEPS][ROWS][256];
    float angles[2][8][128];
};

// blockIdx.y: STEPS * kRows query heads, or KV heads; the block's warps take tokens blockIdx.x * 8 + warp and so on.  A token's rows
// and angles are copied while those of the token before are worked on.
template <int D, int STEPS, class Positions>
__global__ void __launch_bounds__(256, 3) norm_rotary_kernel(const __grid_constant__ NormRotaryArgs a, const __grid_constant__ Positions positions, const int q_groups)
{
    constexpr int kRows = Lane<D>::kRows;
    extern __shared__ __align__(16) unsigned char memory[];
    Ring<STEPS, 1>& ring = *reinterpret_cast<Ring<STEPS, 1>*>(memory);
    const bool is_q = (int)blockIdx.y < q_groups;
    const int of = is_q ? a.q_heads : a.kv_heads, warp = threadIdx.x >> 5, stride = gridDim.x * 8;
    const Lane<D> lane(a);
    const int head0 = ((int)blockIdx.y - (is_q ? 0 : q_groups)) * STEPS * kRows + lane.row;  // the lane's first
    const float* weight = is_q ? a.q_weight : a.k_weight;
    const long long row_stride = is_q ? a.q_stride : a.k_stride;
    int e = blockIdx.x * 8 + warp;
    const __nv_bfloat16* src = (is_q ? a.q : a.k) + e * row_stride + lane.column;
    __nv_bfloat16* dst = (is_q ? a.q_out : a.k_out) + ((long long)e * of + head0) * D + lane.column;
    auto place = [&](int token) {  // (-1: of no document, the token's rows stay as they are)
        const int t = token < a.n ? positions(token) : -1;
        return t < a.positions ? t : -1;
    };
    auto issue = [&](int buffer, int token, int t) {
        if (token < a.n) {
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const int h = head0 + i * kRows;
                copy16(&ring.piece[buffer][i][0][threadIdx.x], src + (h < of ? h : 0) * D, h < of);
            }
            if (a.table && t >= 0 && (threadIdx.x & 31) * 4 < a.rot)
                copy16(&ring.angles[buffer][warp][(threadIdx.x & 31) * 4], a.table + (long long)t * a.rot + (threadIdx.x & 31) * 4, true);
        }
        copies_issued();
        src += stride * row_stride;
    };
    int t = place(e), after = place(e + stride), then = place(e + 2 * stride);
    issue(0, e, t);
    issue(1, e + stride, after);
    float w[8], wo[8];
    if (weight) {
        load8(weight + lane.column, w);
        load8(weight + (lane.partner % Lane<D>::kLanes) * 8, wo);
    }
    for (int buffer = 0; e < a.n; e += stride, buffer ^= 1) {
        copies_landed<1>();
        __syncwarp();
        const int further = place(e + 3 * stride);
        if (t >= 0) {
            Eight c, s;
            lane.angles(ring.angles[buffer][warp], a.rot, c, s);
            if (weight) {  // y = r (x c w + x' s w')
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    c.p[j] = mul2(c.p[j], make_float2(w[2 * j], w[2 * j + 1]));
                    s.p[j] = mul2(s.p[j], lane.inside ? make_float2(wo[2 * j + 1], wo[2 * j]) : make_float2(wo[2 * j], wo[2 * j + 1]));
                }
            }
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const uint4 x = ring.piece[buffer][i][0][threadIdx.x];
                Eight y = unpack(x);
                const Eight z = lane.others(x, y);
                float2 r = make_float2(1.f, 1.f);
                if (weight) {
                    float2 sum = mul2(y.p[0], y.p[0]);
#pragma unroll
                    for (int j = 1; j < 4; ++j) sum = fma2(y.p[j], y.p[j], sum);
                    r.x = r.y = rsqrtf(lanes_sum<Lane<D>::kLanes>(sum) * (1.f / D) + a.eps);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) y.p[j] = mul2(r, fma2(z.p[j], s.p[j], mul2(y.p[j], c.p[j])));
                if (head0 + i * kRows < of) *reinterpret_cast<uint4*>(dst + i * kRows * D) = pack(y);
            }
        }
        __syncwarp();  // every lane has read the angles
        issue(buffer, e + 2 * stride, then);
        dst += (long long)stride * of * D;
        t = after;
        after = then;
        then = further;
    }
}

// The same walk.  A lane adds up its eight columns of dw over all steps, and the block's sums go to `partials`, whose order the
// launch fixes.
template <int D, int STEPS>
__global__ void __launch_bounds__(256, 3) norm_rotary_backward_kernel(const __grid_constant__ NormRotaryArgs a, const int q_groups)
{
    constexpr int kRows = Lane<D>::kRows, kLanes = Lane<D>::kLanes;
    extern __shared__ __align__(16) unsigned char memory[];
    Ring<STEPS, 2>& ring = *reinterpret_cast<Ring<STEPS, 2>*>(memory);
    const bool is_q = (int)blockIdx.y < q_groups;
    const int of = is_q ? a.q_heads : a.kv_heads, warp = threadIdx.x >> 5, stride = gridDim.x * 8;
    const Lane<D> lane(a);
    const int head0 = ((int)blockIdx.y - (is_q ? 0 : q_groups)) * STEPS * kRows + lane.row;
    const float* weight = is_q ? a.q_weight : a.k_weight;
    const long long row_stride = is_q ? a.q_stride : a.k_stride, to_stride = is_q ? a.dq_stride : a.dk_stride;
    int e = blockIdx.x * 8 + warp;
    const __nv_bfloat16* src = (is_q ? a.q : a.k) + e * row_stride + lane.column;
    const __nv_bfloat16* grad = (is_q ? a.dq_out : a.dk_out) + (long long)e * of * D + lane.column;
    __nv_bfloat16* dst = (is_q ? a.dq : a.dk) + e * to_stride + head0 * D + lane.column;
    auto place = [&](int token) {
        const int t = token >= a.n ? -1 : a.position ? __ldg(a.position + token) : token;
        return t < a.positions ? t : -1;
    };
    auto issue = [&](int buffer, int token, int t) {
        if (token < a.n) {
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const int h = head0 + i * kRows, at = (h < of ? h : 0) * D;
                copy16(&ring.piece[buffer][i][0][threadIdx.x], grad + at, h < of);
                if (weight) copy16(&ring.piece[buffer][i][1][threadIdx.x], src + at, h < of);
            }
            if (a.table && t >= 0 && (threadIdx.x & 31) * 4 < a.rot)
                copy16(&ring.angles[buffer][warp][(threadIdx.x & 31) * 4], a.table + (long long)t * a.rot + (threadIdx.x & 31) * 4, true);
        }
        copies_issued();
        src += stride * row_stride;
        grad += (long long)stride * of * D;
    };
    int t = place(e), after = place(e + stride), then = place(e + 2 * stride);
    issue(0, e, t);
    issue(1, e + stride, after);
    Eight w, d;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        w.p[j] = make_float2(1.f, 1.f);
        d.p[j] = make_float2(0.f, 0.f);
    }
    if (weight) {
        float x[8];
        load8(weight + lane.column, x);
#pragma unroll
        for (int j = 0; j < 4; ++j) w.p[j] = make_float2(x[2 * j], x[2 * j + 1]);
    }
    for (int buffer = 0; e < a.n; e += stride, buffer ^= 1) {
        copies_landed<1>();
        __syncwarp();
        const int further = place(e + 3 * stride);
        if (t >= 0) {
            Eight c, s;
            lane.angles(ring.angles[buffer][warp], a.rot, c, s);
#pragma unroll
            for (int j = 0; j < 4; ++j) s.p[j] = make_float2(-s.p[j].x, -s.p[j].y);  // turned back
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const uint4 g = ring.piece[buffer][i][0][threadIdx.x], x = ring.piece[buffer][i][1][threadIdx.x];
                Eight h = unpack(g);
                {
                    const Eight o = lane.others(g, h);
#pragma unroll
                    for (int j = 0; j < 4; ++j) h.p[j] = fma2(s.p[j], o.p[j], mul2(h.p[j], c.p[j]));
                }
                if (weight) {
                    const Eight z = unpack(x);
                    Eight hw;
                    float2 square = make_float2(0.f, 0.f), dot = square;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        hw.p[j] = mul2(h.p[j], w.p[j]);
                        square = fma2(z.p[j], z.p[j], square);
                        dot = fma2(hw.p[j], z.p[j], dot);
                    }
                    const float r = rsqrtf(lanes_sum<kLanes>(square) * (1.f / D) + a.eps), back = -lanes_sum<kLanes>(dot) * r * r * (1.f / D);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        d.p[j] = fma2(mul2(h.p[j], make_float2(r, r)), z.p[j], d.p[j]);
                        h.p[j] = mul2(make_float2(r, r), fma2(z.p[j], make_float2(back, back), hw.p[j]));
                    }
                }
                if (head0 + i * kRows < of) *reinterpret_cast<uint4*>(dst + i * kRows * D) = pack(h);
            }
        }
        __syncwarp();
        issue(buffer, e + 2 * stride, then);
        dst += stride * to_stride;
        t = after;
        after = then;
        then = further;
    }
    if (!a.partials) return;
    grid_dep_launch();
    float(*sums)[D] = reinterpret_cast<float(*)[D]>(memory);
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int o = kLanes; o < 32; o <<= 1)
            d.p[j] = add2(d.p[j], make_float2(__shfl_xor_sync(0xffffffffu, d.p[j].x, o), __shfl_xor_sync(0xffffffffu, d.p[j].y, o)));
    __syncthreads();  // (no copy is on its way any more: those behind the last token copy nothing)
    if (lane.row == 0)
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<float2*>(&sums[warp][lane.column + 2 * j]) = d.p[j];
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

// How a launch is cut: four steps of heads to a token where that leaves the GPU filled (they share the angles and what a token
// costs beside its rows), else one; at most three blocks on every SM.
struct Cut {
    int steps, q_groups, groups, columns;
};
Cut cut_heads(const NormRotaryArgs& a)
{
    const int rows = a.head_dim == 128 ? 2 : 4, tiles = (a.n + 7) / 8, most = 148 * 3;
    Cut c;
    auto groups = [&](int heads) { return (a.q_heads + heads - 1) / heads + (a.kv_heads + heads - 1) / heads; };
    c.steps = (long long)tiles * groups(4 * rows) >= most || groups(rows) > most ? 4 : 1;
    c.q_groups = (a.q_heads + c.steps * rows - 1) / (c.steps * rows);
    c.groups = groups(c.steps * rows);
    c.columns = most / c.groups < tiles ? most / c.groups : tiles;
    return c;
}

template <int D, int STEPS, class Positions>
cudaError_t launch_forward_steps(const NormRotaryArgs& a, const Positions& positions, const Cut& c, cudaStream_t stream)
{
    norm_rotary_kernel<D, STEPS, Positions><<<dim3(c.columns, c.groups), 256, sizeof(Ring<STEPS, 1>), stream>>>(a, positions, c.q_groups);
    return cudaGetLastError();
}

template <class Positions>
cudaError_t launch_forward(const NormRotaryArgs& a, const Positions& positions, cudaStream_t stream)
{
    const Cut c = cut_heads(a);
    if (a.head_dim == 128) return c.steps == 4 ? launch_forward_steps<128, 4>(a, positions, c, stream) : launch_forward_steps<128, 1>(a, positions, c, stream);
    return c.steps == 4 ? launch_forward_steps<64, 4>(a, positions, c, stream) : launch_forward_steps<64, 1>(a, positions, c, stream);
}

template <int D, int STEPS>
cudaError_t launch_backward_steps(const NormRotaryArgs& a, const Cut& c, cudaStream_t stream)
{
    norm_rotary_backward_kernel<D, STEPS><<<dim3(c.columns, c.groups), 256, sizeof(Ring<STEPS, 2>), stream>>>(a, c.q_groups);
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
    const Cut c = cut_heads(a);
    if (!a.dq_weight && !a.dk_weight) a.partials = nullptr;
    cudaError_t e = a.head_dim == 128 ? (c.steps == 4 ? launch_backward_steps<128, 4>(a, c, stream) : launch_backward_steps<128, 1>(a, c, stream))
                                      : (c.steps == 4 ? launch_backward_steps<64, 4>(a, c, stream) : launch_backward_steps<64, 1>(a, c, stream));
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

cudaError_t prepare_norm_backward()
{
    cudaError_t e = cudaFuncSetAttribute(norm_rotary_backward_kernel<128, 4>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Ring<4, 2>));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(norm_rotary_backward_kernel<64, 4>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Ring<4, 2>));
    return e;
}

}  // namespace rlkv
