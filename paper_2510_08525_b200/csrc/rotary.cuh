// What the kernels that turn queries and keys by their position share: a thread's piece of a head, its products, its norm.
#pragma once

#include <cuda_fp8.h>

#include "rlkv_internal.cuh"

namespace rlkv {

constexpr int kPiece = 16;  // elements one thread turns: eight pairs, so two 16-byte loads and one 64-byte table read

__device__ __forceinline__ void rotate(float& u, float& v, float2 cs)
{
    const float x = u, y = v;
    u = fmaf(x, cs.x, -__fmul_rn(y, cs.y));
    v = fmaf(y, cs.x, __fmul_rn(x, cs.y));
}

__device__ __forceinline__ void unpack8(const uint4& bits, float (&x)[8])
{
    const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&bits);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 f = __bfloat1622float2(p[j]);
        x[2 * j] = f.x;
        x[2 * j + 1] = f.y;
    }
}

__device__ __forceinline__ uint4 pack8(const float (&x)[8])
{
    uint4 bits;
    __nv_bfloat162* p = reinterpret_cast<__nv_bfloat162*>(&bits);
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = __floats2bfloat162_rn(x[2 * j], x[2 * j + 1]);
    return bits;
}

__device__ __forceinline__ uint2 codes8(const float (&x)[8], float inv)
{
    uint2 bits;
    unsigned char* c = reinterpret_cast<unsigned char*>(&bits);
#pragma unroll
    for (int j = 0; j < 8; ++j) c[j] = (unsigned char)__nv_cvt_float_to_fp8(x[j] * inv, __NV_SATFINITE, __NV_E4M3);
    return bits;
}

// The angles of piece `piece` of a token at position t: cos and sin of eight pairs.
__device__ __forceinline__ void load_angles(const float* table, long long t, int rot, int piece, float2 (&f)[8])
{
    const float4* cs = reinterpret_cast<const float4*>(table + t * rot + piece * kPiece);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float4 v = __ldg(cs + j);
        f[2 * j] = make_float2(v.x, v.y);
        f[2 * j + 1] = make_float2(v.z, v.w);
    }
}

// Turns a piece's two runs of eight elements: the halves of eight pairs, or sixteen in a row.
__device__ __forceinline__ void rotate_piece(float (&x0)[8], float (&x1)[8], const float2 (&f)[8], bool interleaved)
{
    if (interleaved) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            rotate(x0[2 * j], x0[2 * j + 1], f[j]);
            rotate(x1[2 * j], x1[2 * j + 1], f[4 + j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) rotate(x0[j], x1[j], f[j]);
    }
}

// Sum of x over the PIECES neighbouring lanes that hold a head's row.
template <int PIECES>
__device__ __forceinline__ float row_sum(float x)
{
    const unsigned lanes = ((1u << PIECES) - 1u) << ((threadIdx.x & 31) & ~(PIECES - 1));
#pragma unroll
    for (int o = 1; o < PIECES; o <<= 1) x += __shfl_xor_sync(lanes, x, o);
    return x;
}

__device__ __forceinline__ void load8(const float* p, float (&w)[8])
{
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
    w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
}

// 1 / sqrt(mean square + eps) of the row whose pieces the lanes hold.
template <int PIECES>
__device__ __forceinline__ float row_rsqrt(const float (&x0)[8], const float (&x1)[8], float eps)
{
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(x0[j], x0[j], fmaf(x1[j], x1[j], s));
    return rsqrtf(row_sum<PIECES>(s) * (1.f / (PIECES * kPiece)) + eps);
}

}  // namespace rlkv
