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

// Eight numbers as four pairs, for the instructions that take two fp32 numbers at a time.
struct Eight {
    float2 p[4];
};

// A lane holds sixteen elements of a row, the eight pairs that it turns: u the first elements of the pairs, v the second; D / 16 lanes
// a row.  Two runs of eight in memory, which are u and v where pairs are the halves of the rotated part, and whose even and odd
// elements are u and v where pairs are neighbours (or where nothing is rotated).
//
// Bound by memory at large sizes, and next to it by the instructions a row takes, so that both kernels count them: pairs of fp32
// operations, both elements of a pair in one lane, running pointers, and copies to shared memory that go out while the token before
// is worked on in place of loads whose registers wait.  8192 tokens of 32 / 8 heads of 128: loads of four heads at a time took 43 us
// forward and 79 backward (117 and 151 registers: too few loads in flight); eight elements a lane, the pairs' others by shuffles, 36
// and 65 (250 and then 190 instructions for 512 bytes; half of the issue slots); this, 31.6 and 45.5 (168 and 252 MB: 5.3 and 5.5 TB/s,
// 81 and 84 % of a copy's rate; half of the issue slots still).
template <int D>
struct Lane {
    static constexpr int kLanes = D / 16, kRows = 32 / kLanes;  // of a row, rows of a warp
    int row, piece, first, second;  // row of the warp, piece of the row, where its runs begin
    bool turned, halves;
    __device__ __forceinline__ Lane(const NormRotaryArgs& a)
    {
        const int lane = threadIdx.x & 31;
        row = lane / kLanes;
        piece = lane % kLanes;
        turned = a.table && piece * kPiece < a.rot;
        halves = turned && !a.interleaved;
        first = halves ? piece * 8 : piece * kPiece;
        second = halves ? first + a.rot / 2 : first + 8;
    }
    __device__ __forceinline__ void unpack(const uint4& x, const uint4& y, Eight& u, Eight& v) const
    {
        const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        auto lo = [&](int i) { return __uint_as_float(w[i] << 16); };
        auto hi = [&](int i) { return __uint_as_float(w[i] & 0xffff0000u); };
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u.p[i] = halves ? make_float2(lo(i), hi(i)) : make_float2(lo(2 * i), lo(2 * i + 1));
            v.p[i] = halves ? make_float2(lo(4 + i), hi(4 + i)) : make_float2(hi(2 * i), hi(2 * i + 1));
        }
    }
    __device__ __forceinline__ void store(__nv_bfloat16* row_at, const Eight& u, const Eight& v) const
    {
        uint32_t w[8];
        if (halves) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = tc::bf16x2(u.p[i].x, u.p[i].y);
                w[4 + i] = tc::bf16x2(v.p[i].x, v.p[i].y);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[2 * i] = tc::bf16x2(u.p[i].x, v.p[i].x);
                w[2 * i + 1] = tc::bf16x2(u.p[i].y, v.p[i].y);
            }
        }
        *reinterpret_cast<uint4*>(row_at + first) = make_uint4(w[0], w[1], w[2], w[3]);
        *reinterpret_cast<uint4*>(row_at + second) = make_uint4(w[4], w[5], w[6], w[7]);
    }
    // A row of fp32 numbers (a norm's weights) in the lane's order, and back.
    __device__ __forceinline__ void load(const float* from, Eight& u, Eight& v) const
    {
        float x[8], y[8];
        load8(from + first, x);
        load8(from + second, y);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u.p[i] = halves ? make_float2(x[2 * i], x[2 * i + 1]) : i < 2 ? make_float2(x[4 * i], x[4 * i + 2]) : make_float2(y[4 * i - 8], y[4 * i - 6]);
            v.p[i] = halves ? make_float2(y[2 * i], y[2 * i + 1]) : i < 2 ? make_float2(x[4 * i + 1], x[4 * i + 3]) : make_float2(y[4 * i - 7], y[4 * i - 5]);
        }
    }
    __device__ __forceinline__ void store(float* to, const Eight& u, const Eight& v) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float* at = to + (i < 2 ? first + 4 * i : second + 4 * i - 8);  // (neighbours)
            *reinterpret_cast<float2*>(halves ? to + first + 2 * i : at) = halves ? u.p[i] : make_float2(u.p[i].x, v.p[i].x);
            *reinterpret_cast<float2*>(halves ? to + second + 2 * i : at + 2) = halves ? v.p[i] : make_float2(u.p[i].y, v.p[i].y);
        }
    }
    // cos and sin of the lane's pairs, from the token's row of the table
    __device__ __forceinline__ void angles(const float* row_of, Eight& c, Eight& s) const
    {
        const float4* p = reinterpret_cast<const float4*>(row_of + piece * kPiece);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float4 x = turned ? p[j] : make_float4(1.f, 0.f, 1.f, 0.f);
            c.p[j] = make_float2(x.x, x.z);
            s.p[j] = make_float2(x.y, x.w);
        }
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

// What a warp keeps of the two tokens it has copies on the way for: STEPS times kRows heads of ROWS tensors, a piece of two runs to each lane,
// and the token's row of the table.
template <int STEPS, int ROWS>
struct Ring {
    uint4 piece[2][STEPS][ROWS][2][256];
    float angles[2][8][128];
};

// blockIdx.y: STEPS * kRows query heads, or KV heads; the block's warps take tokens blockIdx.x * 8 + warp and so on.  A token's rows
// and angles are copied while those of the token before are worked on.
template <int D, int STEPS, class Positions>
__global__ void __launch_bounds__(256, 2) norm_rotary_kernel(const __grid_constant__ NormRotaryArgs a, const __grid_constant__ Positions positions, const int q_groups)
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
    const __nv_bfloat16* src = (is_q ? a.q : a.k) + e * row_stride;
    __nv_bfloat16* dst = (is_q ? a.q_out : a.k_out) + ((long long)e * of + head0) * D;
    auto place = [&](int token) {  // (-1: of no document, the token's rows stay as they are)
        const int t = token < a.n ? positions(token) : -1;
        return t < a.positions ? t : -1;
    };
    auto issue = [&](int buffer, int token, int t) {
        if (token < a.n) {
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const int h = head0 + i * kRows;
                const __nv_bfloat16* at = src + (h < of ? h : 0) * D;
                copy16(&ring.piece[buffer][i][0][0][threadIdx.x], at + lane.first, h < of);
                copy16(&ring.piece[buffer][i][0][1][threadIdx.x], at + lane.second, h < of);
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
    Eight wu, wv;
    if (weight) lane.load(weight, wu, wv);
    for (int buffer = 0; e < a.n; e += stride, buffer ^= 1) {
        copies_landed<1>();
        __syncwarp();
        const int further = place(e + 3 * stride);
        if (t >= 0) {
            Eight c, s;
            lane.angles(ring.angles[buffer][warp], c, s);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                Eight u, v;
                lane.unpack(ring.piece[buffer][i][0][0][threadIdx.x], ring.piece[buffer][i][0][1][threadIdx.x], u, v);
                if (weight) {
                    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum = fma2(v.p[j], v.p[j], fma2(u.p[j], u.p[j], sum));
                    const float x = rsqrtf(lanes_sum<Lane<D>::kLanes>(sum) * (1.f / D) + a.eps);
                    const float2 r = make_float2(x, x);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        u.p[j] = mul2(mul2(u.p[j], r), wu.p[j]);
                        v.p[j] = mul2(mul2(v.p[j], r), wv.p[j]);
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 x = u.p[j], minus = make_float2(-v.p[j].x, -v.p[j].y);
                    u.p[j] = fma2(x, c.p[j], mul2(minus, s.p[j]));
                    v.p[j] = fma2(v.p[j], c.p[j], mul2(x, s.p[j]));
                }
                if (head0 + i * kRows < of) lane.store(dst + i * kRows * D, u, v);
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

// The same walk.  A lane adds up its columns of dw over all steps, and the block's sums go to `partials`; the last block of the
// queries' and of the keys' to arrive adds them up, in the order of the blocks whichever it is.  (A kernel of its own behind this one, with
// its launch: 1777 tokens of 8 / 2 heads of 64, forward and backward, 21.4 us a pass, so 19.2; 8192 of 32 / 8 of 128 84.0 and 82.6.)
template <int D, int STEPS>
__global__ void __launch_bounds__(256, 2) norm_rotary_backward_kernel(const __grid_constant__ NormRotaryArgs a, const int q_groups)
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
    const __nv_bfloat16* src = (is_q ? a.q : a.k) + e * row_stride;
    const __nv_bfloat16* grad = (is_q ? a.dq_out : a.dk_out) + (long long)e * of * D;
    __nv_bfloat16* dst = (is_q ? a.dq : a.dk) + e * to_stride + head0 * D;
    auto place = [&](int token) {
        const int t = token >= a.n ? -1 : a.position ? __ldg(a.position + token) : token;
        return t < a.positions ? t : -1;
    };
    auto issue = [&](int buffer, int token, int t) {
        if (token < a.n) {
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const int h = head0 + i * kRows, at = (h < of ? h : 0) * D;
                copy16(&ring.piece[buffer][i][0][0][threadIdx.x], grad + at + lane.first, h < of);
                copy16(&ring.piece[buffer][i][0][1][threadIdx.x], grad + at + lane.second, h < of);
                if (weight) {
                    copy16(&ring.piece[buffer][i][1][0][threadIdx.x], src + at + lane.first, h < of);
                    copy16(&ring.piece[buffer][i][1][1][threadIdx.x], src + at + lane.second, h < of);
                }
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
    Eight wu, wv, du, dv;
#pragma unroll
    for (int j = 0; j < 4; ++j) du.p[j] = dv.p[j] = make_float2(0.f, 0.f);
    if (weight) lane.load(weight, wu, wv);
    for (int buffer = 0; e < a.n; e += stride, buffer ^= 1) {
        copies_landed<1>();
        __syncwarp();
        const int further = place(e + 3 * stride);
        if (t >= 0) {
            Eight c, s;
            lane.angles(ring.angles[buffer][warp], c, s);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                Eight u, v;  // h, the gradient turned back
                lane.unpack(ring.piece[buffer][i][0][0][threadIdx.x], ring.piece[buffer][i][0][1][threadIdx.x], u, v);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 x = u.p[j], minus = make_float2(-x.x, -x.y);
                    u.p[j] = fma2(x, c.p[j], mul2(v.p[j], s.p[j]));
                    v.p[j] = fma2(v.p[j], c.p[j], mul2(minus, s.p[j]));
                }
                if (weight) {
                    Eight xu, xv;
                    lane.unpack(ring.piece[buffer][i][1][0][threadIdx.x], ring.piece[buffer][i][1][1][threadIdx.x], xu, xv);
                    float2 square = make_float2(0.f, 0.f), dot = square;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        square = fma2(xv.p[j], xv.p[j], fma2(xu.p[j], xu.p[j], square));
                        dot = fma2(mul2(v.p[j], wv.p[j]), xv.p[j], fma2(mul2(u.p[j], wu.p[j]), xu.p[j], dot));
                    }
                    const float x = rsqrtf(lanes_sum<kLanes>(square) * (1.f / D) + a.eps), y = -lanes_sum<kLanes>(dot) * x * x * (1.f / D);
                    const float2 r = make_float2(x, x), back = make_float2(y, y);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        u.p[j] = mul2(u.p[j], r);
                        v.p[j] = mul2(v.p[j], r);
                        du.p[j] = fma2(u.p[j], xu.p[j], du.p[j]);
                        dv.p[j] = fma2(v.p[j], xv.p[j], dv.p[j]);
                        u.p[j] = fma2(mul2(xu.p[j], back), r, mul2(u.p[j], wu.p[j]));
                        v.p[j] = fma2(mul2(xv.p[j], back), r, mul2(v.p[j], wv.p[j]));
                    }
                }
                if (head0 + i * kRows < of) lane.store(dst + i * kRows * D, u, v);
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
    float(*sums)[D] = reinterpret_cast<float(*)[D]>(memory);
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int o = kLanes; o < 32; o <<= 1) {
            du.p[j] = add2(du.p[j], make_float2(__shfl_xor_sync(0xffffffffu, du.p[j].x, o), __shfl_xor_sync(0xffffffffu, du.p[j].y, o)));
            dv.p[j] = add2(dv.p[j], make_float2(__shfl_xor_sync(0xffffffffu, dv.p[j].x, o), __shfl_xor_sync(0xffffffffu, dv.p[j].y, o)));
        }
    __syncthreads();  // (no copy is on its way any more: those behind the last token copy nothing)
    if (lane.row == 0) lane.store(sums[warp], du, dv);
    __syncthreads();
    float* to = is_q ? a.dq_weight : a.dk_weight;
    if (!to) return;
    if (threadIdx.x < D) {
        float all = 0.f;
#pragma unroll
        for (int x = 0; x < 8; ++x) all += sums[x][threadIdx.x];
        a.partials[((long long)blockIdx.y * gridDim.x + blockIdx.x) * D + threadIdx.x] = all;
    }
    const int blocks = (is_q ? q_groups : (int)gridDim.y - q_groups) * gridDim.x;
    __threadfence();
    __syncthreads();  // (every thread's sum is out before the block counts as arrived)
    if (__syncthreads_or(threadIdx.x == 0 && atomicAdd(a.arrived + (is_q ? 0 : 1), 1) == blocks - 1) == 0) return;
    __threadfence();
    if (threadIdx.x == 0) a.arrived[is_q ? 0 : 1] = 0;  // for the next launch
    constexpr int kPer = D / 4, kSlices = 256 / kPer;     // threads of a block's sums, blocks at a time
    const int c = threadIdx.x % kPer, slice = threadIdx.x / kPer;
    const float4* from = reinterpret_cast<const float4*>(a.partials + (is_q ? 0 : (long long)q_groups * gridDim.x * D)) + c;
    float4 all = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = slice; i0 < blocks; i0 += 16 * kSlices) {  // sixteen loads on the way
        float4 x[16];
#pragma unroll
        for (int j = 0; j < 16; ++j)
            x[j] = i0 + j * kSlices < blocks ? __ldcg(from + (long long)(i0 + j * kSlices) * kPer) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int j = 0; j < 16; ++j) all = make_float4(all.x + x[j].x, all.y + x[j].y, all.z + x[j].z, all.w + x[j].w);
    }
    float4* meet = reinterpret_cast<float4*>(memory);
    meet[slice * kPer + c] = all;  // (the block's own sums have been read)
    __syncthreads();
    if (threadIdx.x < D) {
        float w = 0.f;
#pragma unroll
        for (int x = 0; x < kSlices; ++x) w += reinterpret_cast<const float*>(meet)[x * D + threadIdx.x];
        to[threadIdx.x] = w;
    }
}

// How a launch is cut: two steps of heads to a token where there are so many and that leaves the GPU filled (they share the angles and
// what a token costs beside its rows), else one (8 / 2 heads of 64, a step half empty: 13.9 us on the GPU, so 12.0); at most two
// blocks on every SM.
struct Cut {
    int steps, q_groups, groups, columns;
};
Cut cut_heads(const NormRotaryArgs& a)
{
    const int rows = a.head_dim == 128 ? 4 : 8, tiles = (a.n + 7) / 8, most = 148 * 2;
    Cut c;
    auto groups = [&](int heads) { return (a.q_heads + heads - 1) / heads + (a.kv_heads + heads - 1) / heads; };
    c.steps = a.q_heads > rows && ((long long)tiles * groups(2 * rows) >= most || groups(rows) > most) ? 2 : 1;
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
    if (a.head_dim == 128) return c.steps == 2 ? launch_forward_steps<128, 2>(a, positions, c, stream) : launch_forward_steps<128, 1>(a, positions, c, stream);
    return c.steps == 2 ? launch_forward_steps<64, 2>(a, positions, c, stream) : launch_forward_steps<64, 1>(a, positions, c, stream);
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
    return a.head_dim == 128 ? (c.steps == 2 ? launch_backward_steps<128, 2>(a, c, stream) : launch_backward_steps<128, 1>(a, c, stream))
                             : (c.steps == 2 ? launch_backward_steps<64, 2>(a, c, stream) : launch_backward_steps<64, 1>(a, c, stream));
}

cudaError_t prepare_norm_backward()
{
    cudaError_t e = cudaFuncSetAttribute(norm_rotary_backward_kernel<128, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Ring<2, 2>));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(norm_rotary_backward_kernel<64, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Ring<2, 2>));
    return e;
}

}  // namespace rlkv
