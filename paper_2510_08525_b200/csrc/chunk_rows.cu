// Rows of chunks of several sequences into the paged cache and back out of it, one launch for all of them.
//
// Both kernels go tile by tile: a block takes the 64 rows of one page (or ring tile, or of the tokens read back) of one head, K
// and V.  Written tiles are driven by their destination: every row of a touched page or ring tile asks which new token, if
// any, ends up in it, so that a ring row is written once, by the last token that belongs there, and the result is that of
// single appends bit for bit.  V codes of an 8-bit page lie transposed ([128][64 tokens]): they turn in shared memory and move as
// sixteen tokens at a time.
#include <cuda_fp8.h>

#include "rlkv_chunk.cuh"

namespace rlkv {
namespace {

constexpr int kPageBytes8 = 2 * kTile * 128;
constexpr int kColumn = kTile + 4;  // bytes of a column of transposed codes in shared memory


__device__ __forceinline__ uint2 codes8(const uint4& bits, float inv)
{
    const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&bits);
    uint2 out;
    __nv_fp8x2_storage_t* c = reinterpret_cast<__nv_fp8x2_storage_t*>(&out);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float2 f = __bfloat1622float2(p[j]);
        f.x *= inv;
        f.y *= inv;
        c[j] = __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3);
    }
    return out;
}

// Eight codes times a scale, rounded to bf16.
__device__ __forceinline__ uint4 values8(uint2 codes, float scale)
{
    const __nv_fp8x2_storage_t* c = reinterpret_cast<const __nv_fp8x2_storage_t*>(&codes);
    uint4 out;
    __nv_bfloat162* p = reinterpret_cast<__nv_bfloat162*>(&out);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(c[j], __NV_E4M3);
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
        p[j] = __floats2bfloat162_rn(f.x * scale, f.y * scale);
    }
    return out;
}

// The entry whose tasks hold block b; first_task: [n + 1], ascending.
__device__ __forceinline__ int entry_of_task(const int* first_task, int n, int b)
{
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (first_task[mid + 1] > b) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

__global__ void __launch_bounds__(256) write_chunks_kernel(const __grid_constant__ ChunkRowsArgs a, const __grid_constant__ ChunkPages pages)
{
    __shared__ int source[kTile];  // new token (inside the chunk) that each row takes, -1: the row stays as it is
    __shared__ __align__(16) unsigned char turned[128 * kColumn];
    const int i = entry_of_task(pages.first_task, a.seqs.n, blockIdx.x);
    int task = blockIdx.x - pages.first_task[i];
    const int t0 = a.seqs.len[i], m = a.seqs.start[i + 1] - a.seqs.start[i], seq = a.seqs.slot[i];
    const int first_page = t0 / kTile, n_pages = (t0 + m - 1) / kTile - first_page + 1;
    const bool full = task < n_pages * a.n_full;
    int tile, slot;
    if (full) {
        tile = task / a.n_full;  // page of the sequence, from first_page on
        slot = task % a.n_full;
    } else {
        task -= n_pages * a.n_full;
        tile = task / a.n_comp;
        slot = task % a.n_comp;
    }
    const int head = a.head_of_slot[full ? slot : a.n_full + slot];
    const int page = full ? pages.page[pages.page0[i] + tile] : 0;
    if (threadIdx.x < kTile) {
        int j = -1;
        if (full) {
            j = (first_page + tile) * kTile + threadIdx.x - t0;
            if (j >= m) j = -1;
        } else {
            const int row = tile * kTile + threadIdx.x, newest = t0 + m - 1;
            int t = -1;
            if (row < a.sink) {
                t = row <= newest ? row : -1;
            } else if (row < a.sink + a.window && newest >= a.sink) {
                const int back = ((newest - a.sink) % a.window - (row - a.sink) + a.window) % a.window;
                t = newest - back >= a.sink ? newest - back : -1;
            }
            j = t >= t0 ? t - t0 : -1;
        }
        source[threadIdx.x] = max(j, -1);
    }
    if (full && slot == 0 && threadIdx.x == 0) a.page_table[(size_t)seq * a.table_stride + first_page + tile] = page;
    if (!__syncthreads_or(threadIdx.x < kTile && source[threadIdx.x] >= 0)) return;
    const int chunks = a.head_dim / 8;
    const long long token0 = a.seqs.start[i];
    const __nv_bfloat16 *k = a.k + token0 * a.k_stride + head * a.head_dim, *v = a.v + token0 * a.v_stride + head * a.head_dim;
    if (!a.pool8) {
        const long long row0 = full ? a.full_row0 + ((long long)slot * a.n_pages + page) * 2 * kTile
                                    : a.comp_row0 + ((long long)seq * a.n_comp + slot) * 2 * a.rows_comp + tile * kTile;
        const int to_v = full ? kTile : a.rows_comp;
#pragma unroll 4
        for (int x = threadIdx.x; x < 2 * kTile * chunks; x += 256) {
            const int c = x % chunks, r = x / chunks % kTile, kv = x / (chunks * kTile), j = source[r];
            if (j < 0) continue;
            const uint4 bits = *(reinterpret_cast<const uint4*>(kv ? v + j * a.v_stride : k + j * a.k_stride) + c);
            *(reinterpret_cast<uint4*>(a.pool + (row0 + (kv ? to_v : 0) + r) * a.head_dim) + c) = bits;
        }
        return;
    }
    const long long index = full ? a.page0_8 + (long long)slot * a.n_pages + page
                                 : a.ring0_8 + ((long long)seq * a.n_comp + slot) * a.ring_tiles + tile;
    unsigned char* to = a.pool8 + index * kPageBytes8;
    const float k_inv = a.k_inv[head], v_inv = a.v_inv[head];
#pragma unroll
    for (int x = 0; x < 2; ++x) {  // K: sixteen elements of a row
        const int piece = x * 256 + threadIdx.x, r = piece >> 3, c = piece & 7, j = source[r];
        if (j < 0) continue;
        const uint4* src = reinterpret_cast<const uint4*>(k + j * a.k_stride) + c * 2;
        const uint4 lo = src[0], hi = src[1];
        const uint2 p = codes8(lo, k_inv), q = codes8(hi, k_inv);
        reinterpret_cast<uint4*>(to)[piece] = make_uint4(p.x, p.y, q.x, q.y);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {  // V: neighbouring lanes take neighbouring rows, so that a column's bytes are stored together
        const int r = threadIdx.x & 63, c = x * 4 + (threadIdx.x >> 6), j = source[r];
        if (j < 0) continue;
        const uint4* src = reinterpret_cast<const uint4*>(v + j * a.v_stride) + c * 2;
        const uint4 lo = src[0], hi = src[1];
        const uint2 p = codes8(lo, v_inv), q = codes8(hi, v_inv);
        const uint4 codes = make_uint4(p.x, p.y, q.x, q.y);
        const unsigned char* u = reinterpret_cast<const unsigned char*>(&codes);
#pragma unroll
        for (int y = 0; y < 16; ++y) turned[(c * 16 + y) * kColumn + r] = u[y];
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int piece = x * 256 + threadIdx.x, d = piece >> 2, r0 = (piece & 3) * 16;
        unsigned valid = 0;
#pragma unroll
        for (int y = 0; y < 16; ++y) valid |= (unsigned)(source[r0 + y] >= 0) << y;
        const unsigned char* src = turned + d * kColumn + r0;
        unsigned char* dst = to + kTile * 128 + d * kTile + r0;
        if (valid == 0xffffu) {
            const uint32_t* w = reinterpret_cast<const uint32_t*>(src);
            *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
        } else if (valid) {
            for (int y = 0; y < 16; ++y)
                if (valid >> y & 1) dst[y] = src[y];
        }
    }
}

__global__ void __launch_bounds__(256) read_rows_kernel(const __grid_constant__ ChunkRowsArgs a, const __grid_constant__ ChunkPages pages)
{
    __shared__ int place[kTile];  // row of the page or ring that holds each of the tile's tokens; -1: none does any more, -2: not asked for
    __shared__ __align__(16) unsigned char turned[128 * kColumn];
    const int i = entry_of_task(pages.first_task, a.seqs.n, blockIdx.x);
    const int task = blockIdx.x - pages.first_task[i], tile = task / a.kv_heads, head = task % a.kv_heads;
    const int first = a.seqs.len[i], count = a.seqs.start[i + 1] - a.seqs.start[i], seq = a.seqs.slot[i], held = a.length[i];
    const int slot = a.slot_of_head[head];
    const bool full = slot >= 0;
    const int page_of = first / kTile + tile;
    if (threadIdx.x < kTile) {
        const int t = page_of * kTile + threadIdx.x;
        int p = -2;
        if (t >= first && t < first + count) {
            if (full) p = threadIdx.x;
            else if (t < a.sink) p = t;
            else p = t >= held - a.window ? a.sink + (t - a.sink) % a.window : -1;
        }
        place[threadIdx.x] = p;
    }
    const bool any = __syncthreads_or(threadIdx.x < kTile && place[threadIdx.x] >= 0);
    const int page = full ? min(max(a.page_table[(size_t)seq * a.table_stride + page_of], 0), a.n_pages - 1) : 0;
    const int chunks = a.head_dim / 8;
    const long long row = (long long)a.kv_heads * a.head_dim;  // elements from token to token of the result
    const long long out0 = ((long long)a.seqs.start[i] + page_of * kTile - first) * row + head * a.head_dim;
    if (!a.pool8 || !any) {
        const long long row0 = full ? a.full_row0 + ((long long)slot * a.n_pages + page) * 2 * kTile
                                    : a.comp_row0 + ((long long)seq * a.n_comp + (-slot - 1)) * 2 * a.rows_comp;
        const int to_v = full ? kTile : a.rows_comp;
#pragma unroll 4
        for (int x = threadIdx.x; x < 2 * kTile * chunks; x += 256) {
            const int c = x % chunks, r = x / chunks % kTile, kv = x / (chunks * kTile), p = place[r];
            if (p == -2) continue;
            uint4 bits = make_uint4(0, 0, 0, 0);
            if (p >= 0) bits = *(reinterpret_cast<const uint4*>(a.pool + (row0 + (kv ? to_v : 0) + p) * a.head_dim) + c);
            *(reinterpret_cast<uint4*>((kv ? a.v_out : a.k_out) + out0 + r * row) + c) = bits;
        }
        return;
    }
    const long long index = full ? a.page0_8 + (long long)slot * a.n_pages + page
                                 : a.ring0_8 + ((long long)seq * a.n_comp + (-slot - 1)) * a.ring_tiles;
    const unsigned char* from = a.pool8 + index * kPageBytes8;
    const float k_scale = a.k_scale[head], v_scale = a.v_scale[head];
    if (full) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {  // V codes, sixteen tokens of an element
            const int piece = x * 256 + threadIdx.x, d = piece >> 2, r0 = (piece & 3) * 16;
            const uint4 bits = reinterpret_cast<const uint4*>(from + kTile * 128)[piece];
            uint32_t* w = reinterpret_cast<uint32_t*>(turned + d * kColumn + r0);
            w[0] = bits.x;
            w[1] = bits.y;
            w[2] = bits.z;
            w[3] = bits.w;
        }
    } else {
        for (int x = threadIdx.x; x < 128 * kTile; x += 256) {  // (a ring's rows wrap wherever the window ends)
            const int r = x & 63, d = x >> 6, p = place[r];
            if (p >= 0) turned[d * kColumn + r] = from[(long long)(p / kTile) * kPageBytes8 + kTile * 128 + d * kTile + p % kTile];
        }
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < 2; ++x) {  // K: sixteen elements of a row
        const int piece = x * 256 + threadIdx.x, r = piece >> 3, c = piece & 7, p = place[r];
        if (p == -2) continue;
        uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
        if (p >= 0) {
            const uint4 bits = *(reinterpret_cast<const uint4*>(from + (long long)(p / kTile) * kPageBytes8 + p % kTile * 128) + c);
            lo = values8(make_uint2(bits.x, bits.y), k_scale);
            hi = values8(make_uint2(bits.z, bits.w), k_scale);
        }
        uint4* dst = reinterpret_cast<uint4*>(a.k_out + out0 + r * row) + c * 2;
        dst[0] = lo;
        dst[1] = hi;
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int r = threadIdx.x & 63, c = x * 4 + (threadIdx.x >> 6), p = place[r];
        if (p == -2) continue;
        uint4 codes;
        unsigned char* u = reinterpret_cast<unsigned char*>(&codes);
#pragma unroll
        for (int y = 0; y < 16; ++y) u[y] = turned[(c * 16 + y) * kColumn + r];
        uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
        if (p >= 0) {
            lo = values8(make_uint2(codes.x, codes.y), v_scale);
            hi = values8(make_uint2(codes.z, codes.w), v_scale);
        }
        uint4* dst = reinterpret_cast<uint4*>(a.v_out + out0 + r * row) + c * 2;
        dst[0] = lo;
        dst[1] = hi;
    }
}

}  // namespace

cudaError_t launch_write_chunks(const ChunkRowsArgs& a, const ChunkPages& pages, cudaStream_t stream)
{
    write_chunks_kernel<<<(unsigned)pages.first_task[a.seqs.n], 256, 0, stream>>>(a, pages);
    return cudaGetLastError();
}

cudaError_t launch_read_rows(const ChunkRowsArgs& a, const ChunkPages& pages, cudaStream_t stream)
{
    read_rows_kernel<<<(unsigned)pages.first_task[a.seqs.n], 256, 0, stream>>>(a, pages);
    return cudaGetLastError();
}

}  // namespace rlkv
