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

// The columns of a piece's two runs.
__device__ __forceinline__ void piece_columns(const NormRotaryArgs& a, int piece, int& c0, int& c1, bool& turned)
{
    turned = a.table && piece * kPiece < a.rot;
    const bool halves = turned && !a.interleaved;
    c0 = halves ? piece * 8 : piece * kPiece;
    c1 = halves ? c0 + a.rot / 2 : c0 + 8;
}

// A block takes 256 / PIECES tokens and `heads` of the heads (q heads, then K heads).  A thread keeps one piece of one token:
// its angles stay in registers over the heads, whose loads are issued four at a time.
template <int PIECES, class Positions>
__global__ void __launch_bounds__(256) norm_rotary_kernel(const __grid_constant__ NormRotaryArgs a, const __grid_constant__ Positions positions, const int heads)
{
    constexpr int kTokens = 256 / PIECES, kBatch = 4, D = PIECES * kPiece;
    const int piece = threadIdx.x % PIECES, e = blockIdx.x * kTokens + threadIdx.x / PIECES;
    const int head0 = blockIdx.y * heads, head1 = min(a.q_heads + a.kv_heads, head0 + heads);
    if (e >= a.n) return;
    const int t = positions(e);
    if (t < 0 || t >= a.positions) return;  // of no document: the token's rows stay as they are
    int c0, c1;
    bool turned;
    piece_columns(a, piece, c0, c1, turned);
    float2 f[8];
    if (turned) load_angles(a.table, t, a.rot, piece, f);
    for (int base = head0; base < head1; base += kBatch) {
        uint4 b[kBatch][2];
#pragma unroll
        for (int x = 0; x < kBatch; ++x) {
            const int hh = base + x;
            if (hh < head1) {
                const bool is_q = hh < a.q_heads;
                const __nv_bfloat16* src = is_q ? a.q + e * a.q_stride + hh * D : a.k + e * a.k_stride + (hh - a.q_heads) * D;
                b[x][0] = *reinterpret_cast<const uint4*>(src + c0);
                b[x][1] = *reinterpret_cast<const uint4*>(src + c1);
            }
        }
#pragma unroll
        for (int x = 0; x < kBatch; ++x) {
            const int hh = base + x;
            if (hh >= head1) break;
            const bool is_q = hh < a.q_heads;
            float x0[8], x1[8];
            unpack8(b[x][0], x0);
            unpack8(b[x][1], x1);
            const float* weight = is_q ? a.q_weight : a.k_weight;
            if (weight) {
                const float rms = row_rsqrt<PIECES>(x0, x1, a.eps);
                float w0[8], w1[8];
                load8(weight + c0, w0);
                load8(weight + c1, w1);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x0[j] = x0[j] * rms * w0[j];
                    x1[j] = x1[j] * rms * w1[j];
                }
            }
            if (turned) rotate_piece(x0, x1, f, a.interleaved);
            __nv_bfloat16* dst = is_q ? a.q_out + ((long long)e * a.q_heads + hh) * D : a.k_out + ((long long)e * a.kv_heads + hh - a.q_heads) * D;
            *reinterpret_cast<uint4*>(dst + c0) = pack8(x0);
            *reinterpret_cast<uint4*>(dst + c1) = pack8(x1);
        }
    }
}

// A block takes `heads` heads of one kind and every gridDim.x-th tile of tokens; a thread adds up its sixteen columns of dw
// over all of them, and the block's sums go to `partials`, whose order the launch fixes.
template <int PIECES>
__global__ void __launch_bounds__(256) norm_rotary_backward_kernel(const __grid_constant__ NormRotaryArgs a, const int heads, const int q_groups)
{
    constexpr int kTokens = 256 / PIECES, kBatch = 2, D = PIECES * kPiece;
    __shared__ float sums[8][D];
    const int piece = threadIdx.x % PIECES;
    const bool is_q = (int)blockIdx.y < q_groups;
    const int of = is_q ? a.q_heads : a.kv_heads;
    const int head0 = ((int)blockIdx.y - (is_q ? 0 : q_groups)) * heads, head1 = min(of, head0 + heads);
    const __nv_bfloat16 *rows = is_q ? a.q : a.k, *grads = is_q ? a.dq_out : a.dk_out;
    const long long stride = is_q ? a.q_stride : a.k_stride, to_stride = is_q ? a.dq_stride : a.dk_stride;
    __nv_bfloat16* to = is_q ? a.dq : a.dk;
    const float* weight = is_q ? a.q_weight : a.k_weight;
    int c0, c1;
    bool turned;
    piece_columns(a, piece, c0, c1, turned);
    float w0[8], w1[8], d0[8], d1[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        w0[j] = w1[j] = 1.f;
        d0[j] = d1[j] = 0.f;
    }
    if (weight) {
        load8(weight + c0, w0);
        load8(weight + c1, w1);
    }
    for (int tile = blockIdx.x; tile * kTokens < a.n; tile += gridDim.x) {
        const int e = tile * kTokens + threadIdx.x / PIECES;
        if (e >= a.n) break;
        const int t = a.position ? __ldg(a.position + e) : e;
        if (t < 0 || t >= a.positions) continue;
        float2 f[8];
        if (turned) {
            load_angles(a.table, t, a.rot, piece, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j].y = -f[j].y;  // turned back
        }
        for (int base = head0; base < head1; base += kBatch) {
            uint4 b[kBatch][2], g[kBatch][2];
#pragma unroll
            for (int x = 0; x < kBatch; ++x) {
                const int h = base + x;
                if (h < head1) {
                    const __nv_bfloat16 *src = rows + e * stride + h * D, *grad = grads + ((long long)e * of + h) * D;
                    g[x][0] = *reinterpret_cast<const uint4*>(grad + c0);
                    g[x][1] = *reinterpret_cast<const uint4*>(grad + c1);
                    if (weight) {
                        b[x][0] = *reinterpret_cast<const uint4*>(src + c0);
                        b[x][1] = *reinterpret_cast<const uint4*>(src + c1);
                    }
                }
            }
#pragma unroll
            for (int x = 0; x < kBatch; ++x) {
                const int h = base + x;
                if (h >= head1) break;
                float h0[8], h1[8];
                unpack8(g[x][0], h0);
                unpack8(g[x][1], h1);
                if (turned) rotate_piece(h0, h1, f, a.interleaved);
                if (weight) {
                    float x0[8], x1[8];
                    unpack8(b[x][0], x0);
                    unpack8(b[x][1], x1);
                    const float rms = row_rsqrt<PIECES>(x0, x1, a.eps);
                    float dot = 0.f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        x0[j] *= rms;
                        x1[j] *= rms;
                        d0[j] = fmaf(h0[j], x0[j], d0[j]);
                        d1[j] = fmaf(h1[j], x1[j], d1[j]);
                        h0[j] *= w0[j];
                        h1[j] *= w1[j];
                        dot = fmaf(h0[j], x0[j], fmaf(h1[j], x1[j], dot));
                    }
                    const float mean = row_sum<PIECES>(dot) * (1.f / D);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        h0[j] = rms * fmaf(-x0[j], mean, h0[j]);
                        h1[j] = rms * fmaf(-x1[j], mean, h1[j]);
                    }
                }
                __nv_bfloat16* dst = to + e * to_stride + h * D;
                *reinterpret_cast<uint4*>(dst + c0) = pack8(h0);
                *reinterpret_cast<uint4*>(dst + c1) = pack8(h1);
            }
        }
    }
    if (!a.partials) return;
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int o = PIECES; o < 32; o <<= 1) {
            d0[j] += __shfl_xor_sync(0xffffffffu, d0[j], o);
            d1[j] += __shfl_xor_sync(0xffffffffu, d1[j], o);
        }
    if ((threadIdx.x & 31) < PIECES)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            sums[threadIdx.x >> 5][c0 + j] = d0[j];
            sums[threadIdx.x >> 5][c1 + j] = d1[j];
        }
    __syncthreads();
    grid_dep_launch();
    if (threadIdx.x < D) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += sums[w][threadIdx.x];
        a.partials[((long long)blockIdx.y * gridDim.x + blockIdx.x) * D + threadIdx.x] = s;
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

template <class Positions>
cudaError_t launch_forward(const NormRotaryArgs& a, const Positions& positions, cudaStream_t stream)
{
    const int pieces = a.head_dim / kPiece, tokens = 256 / pieces, tiles = (a.n + tokens - 1) / tokens, rows = a.q_heads + a.kv_heads;
    // as for the rotated append: enough blocks to fill the GPU first, then as many heads as share one load of the angles
    int heads = 1;
    while (heads < 8 && (long long)tiles * ((rows + 2 * heads - 1) / (2 * heads)) >= 148 * 8) heads *= 2;
    const dim3 grid(tiles, (rows + heads - 1) / heads);
    if (pieces == 8) norm_rotary_kernel<8, Positions><<<grid, 256, 0, stream>>>(a, positions, heads);
    else norm_rotary_kernel<4, Positions><<<grid, 256, 0, stream>>>(a, positions, heads);
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
    const int pieces = a.head_dim / kPiece, tokens = 256 / pieces, tiles = (a.n + tokens - 1) / tokens;
    int heads = 1;
    auto groups = [&](int h) { return (a.q_heads + h - 1) / h + (a.kv_heads + h - 1) / h; };
    while (heads < 8 && ((long long)tiles * groups(2 * heads) >= kMaxNormBlocks || groups(heads) > kMaxNormBlocks)) heads *= 2;
    const int q_groups = (a.q_heads + heads - 1) / heads, all = groups(heads);
    int columns = kMaxNormBlocks / all;
    if (columns > tiles) columns = tiles;
    if (!a.dq_weight && !a.dk_weight) a.partials = nullptr;
    if (pieces == 8) norm_rotary_backward_kernel<8><<<dim3(columns, all), 256, 0, stream>>>(a, heads, q_groups);
    else norm_rotary_backward_kernel<4><<<dim3(columns, all), 256, 0, stream>>>(a, heads, q_groups);
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
    return cudaLaunchKernelEx(&cfg, norm_weights_kernel, (const float*)a.partials, columns * q_groups, columns * (all - q_groups), a.head_dim, a.dq_weight, a.dk_weight);
}

}  // namespace rlkv
