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

// Four words of four bytes each, transposed: byte i of word j becomes byte j of word i.
__device__ __forceinline__ void transpose4(uint32_t (&w)[4])
{
    const uint32_t a = __byte_perm(w[0], w[1], 0x5140), b = __byte_perm(w[2], w[3], 0x5140);  // bytes 0 and 1 of both
    const uint32_t c = __byte_perm(w[0], w[1], 0x7362), d = __byte_perm(w[2], w[3], 0x7362);
    w[0] = __byte_perm(a, b, 0x5410);
    w[1] = __byte_perm(a, b, 0x7632);
    w[2] = __byte_perm(c, d, 0x5410);
    w[3] = __byte_perm(c, d, 0x7632);
}

// Bound by memory where the rows are many, else by the launch.  A thread's loads all go out before its first store, and V codes are
// turned four tokens by four elements in registers.  Measured (us on the GPU; 8 heads of 128, 4 full): 24 requests of 843 tokens on
// average into an 8-bit cache 15.9 (10.9 at a copy's rate; with V codes stored byte by byte 17.2); 16384 tokens of one request (6 full)
// in 16 bits 12.7 (101 MB, some of which stay in the L2; with one row at a time 19.9).
template <int D, bool FP8>
__global__ void __launch_bounds__(256) write_chunks_kernel(const __grid_constant__ ChunkRowsArgs a, const __grid_constant__ ChunkPages pages)
{
    __shared__ __align__(16) int source[kTile];  // new token (inside the chunk) that each row takes, -1: the row stays as it is
    __shared__ __align__(16) unsigned char turned[FP8 ? 128 * kColumn : 16];
    const int i = entry_of_task(pages.first_task, a.seqs.n, blockIdx.x);
    int task = blockIdx.x - pages.first_task[i];
    const int t0 = a.seqs.len[i], m = a.seqs.start[i + 1] - a.seqs.start[i], seq = a.seqs.slot[i];
    const int first_page = t0 / kTile, n_pages = (t0 + m - 1) / kTile - first_page + 1;
    const bool full = task < n_pages * a.n_full;
    int tile, slot;
    if (full) {
        tile = task / a.n_full;  // page of the sequence, from first_page on
        slot = task - tile * a.n_full;
    } else {
        task -= n_pages * a.n_full;
        tile = task / a.n_comp;
        slot = task - tile * a.n_comp;
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
    const long long token0 = a.seqs.start[i];
    const __nv_bfloat16 *k = a.k + token0 * a.k_stride + head * D, *v = a.v + token0 * a.v_stride + head * D;
    if (!FP8) {
        constexpr int kChunks = D / 8, kStep = 256 / kChunks, kPasses = kTile / kStep;  // 16-byte pieces of a row, rows of a pass
        const long long row0 = full ? a.full_row0 + ((long long)slot * a.n_pages + page) * 2 * kTile
                                    : a.comp_row0 + ((long long)seq * a.n_comp + slot) * 2 * a.rows_comp + tile * kTile;
        const int c = threadIdx.x % kChunks, r0 = threadIdx.x / kChunks;
        uint4 x[kPasses], y[kPasses];
        int j[kPasses];
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            j[p] = source[r0 + p * kStep];
            if (j[p] < 0) continue;
            x[p] = *(reinterpret_cast<const uint4*>(k + j[p] * a.k_stride) + c);
            y[p] = *(reinterpret_cast<const uint4*>(v + j[p] * a.v_stride) + c);
        }
        uint4* to = reinterpret_cast<uint4*>(a.pool + (row0 + r0) * D) + c;
        const long long to_v = (long long)(full ? kTile : a.rows_comp) * kChunks;
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            if (j[p] < 0) continue;
            to[p * kStep * kChunks] = x[p];
            to[p * kStep * kChunks + to_v] = y[p];
        }
        return;
    }
    const long long index = full ? a.page0_8 + (long long)slot * a.n_pages + page
                                 : a.ring0_8 + ((long long)seq * a.n_comp + slot) * a.ring_tiles + tile;
    unsigned char* to = a.pool8 + index * kPageBytes8;
    const float k_inv = a.k_inv[head], v_inv = a.v_inv[head];
    // V: eight elements of four neighbouring rows a thread, as words of four tokens of an element to shared memory
    const int r4 = (threadIdx.x & 15) * 4, c8 = threadIdx.x >> 4;
    const int4 rows = *reinterpret_cast<const int4*>(source + r4);
    const int from[4] = {rows.x, rows.y, rows.z, rows.w};
    uint4 bits[4], lo[2], hi[2];
#pragma unroll
    for (int y = 0; y < 4; ++y)
        if (from[y] >= 0) bits[y] = *(reinterpret_cast<const uint4*>(v + from[y] * a.v_stride) + c8);
    int kj[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {  // K: sixteen elements of a row
        const int piece = x * 256 + threadIdx.x;
        kj[x] = source[piece >> 3];
        if (kj[x] < 0) continue;
        const uint4* src = reinterpret_cast<const uint4*>(k + kj[x] * a.k_stride) + (piece & 7) * 2;
        lo[x] = src[0];
        hi[x] = src[1];
    }
    uint2 codes[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) codes[y] = from[y] >= 0 ? codes8(bits[y], v_inv) : make_uint2(0, 0);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        uint32_t w[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) w[y] = half ? codes[y].y : codes[y].x;
        transpose4(w);
#pragma unroll
        for (int y = 0; y < 4; ++y) *reinterpret_cast<uint32_t*>(turned + (c8 * 8 + half * 4 + y) * kColumn + r4) = w[y];
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        if (kj[x] < 0) continue;
        const uint2 p = codes8(lo[x], k_inv), q = codes8(hi[x], k_inv);
        reinterpret_cast<uint4*>(to)[x * 256 + threadIdx.x] = make_uint4(p.x, p.y, q.x, q.y);
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int piece = x * 256 + threadIdx.x, d = piece >> 2, r0 = (piece & 3) * 16;
        unsigned valid = 0;
#pragma unroll
        for (int y = 0; y < 16; y += 4) {
            const int4 s = *reinterpret_cast<const int4*>(source + r0 + y);
            valid |= ((unsigned)(s.x >= 0) | (unsigned)(s.y >= 0) << 1 | (unsigned)(s.z >= 0) << 2 | (unsigned)(s.w >= 0) << 3) << y;
        }
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

// As above, the other way round.  Measured (us on the GPU): the 24 requests above 24.5 (16.3 at a copy's rate; with V codes gathered
// byte by byte 28.2), the second half of the 16384 tokens 7.5 (59 MB, read out of the L2; one row at a time 11.4).
template <int D, bool FP8>
__global__ void __launch_bounds__(256) read_rows_kernel(const __grid_constant__ ChunkRowsArgs a, const __grid_constant__ ChunkPages pages)
{
    __shared__ __align__(16) int place[kTile];  // row of the page or ring that holds each of the tile's tokens; -1: none does any more, -2: not asked for
    __shared__ __align__(16) unsigned char turned[FP8 ? 128 * kColumn : 16];
    const int i = entry_of_task(pages.first_task, a.seqs.n, blockIdx.x);
    const int task = blockIdx.x - pages.first_task[i], tile = task / a.kv_heads, head = task - tile * a.kv_heads;
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
    const int page = full ? min(max(a.page_table[(size_t)seq * a.table_stride + page_of], 0), a.n_pages - 1) : 0;
    const bool any = __syncthreads_or(threadIdx.x < kTile && place[threadIdx.x] >= 0);
    const long long row = (long long)a.kv_heads * D;  // elements from token to token of the result
    const long long out0 = ((long long)a.seqs.start[i] + page_of * kTile - first) * row + head * D;
    if (!FP8 || !any) {
        constexpr int kChunks = D / 8, kStep = 256 / kChunks, kPasses = kTile / kStep;
        const long long row0 = full ? a.full_row0 + ((long long)slot * a.n_pages + page) * 2 * kTile
                                    : a.comp_row0 + ((long long)seq * a.n_comp + (-slot - 1)) * 2 * a.rows_comp;
        const long long to_v = (long long)(full ? kTile : a.rows_comp) * kChunks;
        const int c = threadIdx.x % kChunks, r0 = threadIdx.x / kChunks;
        const uint4* from = reinterpret_cast<const uint4*>(a.pool + row0 * D) + c;
        uint4 x[kPasses], y[kPasses];
        int at[kPasses];
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            at[p] = place[r0 + p * kStep];
            x[p] = y[p] = make_uint4(0, 0, 0, 0);
            if (!FP8 && at[p] >= 0) {
                x[p] = from[at[p] * kChunks];
                y[p] = from[at[p] * kChunks + to_v];
            }
        }
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            if (at[p] == -2) continue;
            const long long to = out0 + (r0 + p * kStep) * row + c * 8;
            *reinterpret_cast<uint4*>(a.k_out + to) = x[p];
            *reinterpret_cast<uint4*>(a.v_out + to) = y[p];
        }
        return;
    }
    const long long index = full ? a.page0_8 + (long long)slot * a.n_pages + page
                                 : a.ring0_8 + ((long long)seq * a.n_comp + (-slot - 1)) * a.ring_tiles;
    const unsigned char* from = a.pool8 + index * kPageBytes8;
    const float k_scale = a.k_scale[head], v_scale = a.v_scale[head];
    uint4 k_bits[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {  // K: sixteen elements of a row
        const int piece = x * 256 + threadIdx.x, p = place[piece >> 3];
        k_bits[x] = make_uint4(0, 0, 0, 0);
        if (p >= 0) k_bits[x] = *(reinterpret_cast<const uint4*>(from + (long long)(p / kTile) * kPageBytes8 + p % kTile * 128) + (piece & 7));
    }
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
            turned[d * kColumn + r] = p >= 0 ? from[(long long)(p / kTile) * kPageBytes8 + kTile * 128 + d * kTile + p % kTile] : 0;
        }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int piece = x * 256 + threadIdx.x, r = piece >> 3;
        if (place[r] == -2) continue;
        uint4* dst = reinterpret_cast<uint4*>(a.k_out + out0 + r * row) + (piece & 7) * 2;
        dst[0] = values8(make_uint2(k_bits[x].x, k_bits[x].y), k_scale);
        dst[1] = values8(make_uint2(k_bits[x].z, k_bits[x].w), k_scale);
    }
    __syncthreads();
    // V: eight elements of four neighbouring tokens a thread
    const int r4 = (threadIdx.x & 15) * 4, c8 = threadIdx.x >> 4;
    uint2 codes[4];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        uint32_t w[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) w[y] = *reinterpret_cast<const uint32_t*>(turned + (c8 * 8 + half * 4 + y) * kColumn + r4);
        transpose4(w);
#pragma unroll
        for (int y = 0; y < 4; ++y) (half ? codes[y].y : codes[y].x) = w[y];
    }
    const int4 p = *reinterpret_cast<const int4*>(place + r4);
    const int at[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
    for (int y = 0; y < 4; ++y) {
        if (at[y] == -2) continue;
        *(reinterpret_cast<uint4*>(a.v_out + out0 + (r4 + y) * row) + c8) = at[y] >= 0 ? values8(codes[y], v_scale) : make_uint4(0, 0, 0, 0);
    }
}

}  // namespace

cudaError_t launch_write_chunks(const ChunkRowsArgs& a, const ChunkPages& pages, cudaStream_t stream)
{
    const unsigned blocks = (unsigned)pages.first_task[a.seqs.n];
    if (a.pool8) write_chunks_kernel<128, true><<<blocks, 256, 0, stream>>>(a, pages);
    else if (a.head_dim == 128) write_chunks_kernel<128, false><<<blocks, 256, 0, stream>>>(a, pages);
    else write_chunks_kernel<64, false><<<blocks, 256, 0, stream>>>(a, pages);
    return cudaGetLastError();
}

cudaError_t launch_read_rows(const ChunkRowsArgs& a, const ChunkPages& pages, cudaStream_t stream)
{
    const unsigned blocks = (unsigned)pages.first_task[a.seqs.n];
    if (a.pool8) read_rows_kernel<128, true><<<blocks, 256, 0, stream>>>(a, pages);
    else if (a.head_dim == 128) read_rows_kernel<128, false><<<blocks, 256, 0, stream>>>(a, pages);
    else read_rows_kernel<64, false><<<blocks, 256, 0, stream>>>(a, pages);
    return cudaGetLastError();
}

}  // namespace rlkv
