// Chunks of new tokens of several sequences of the paged cache: what the host side (rlkv_paged_chunks.cu) and the
// kernels (chunk_attention.cu, chunk_rows.cu, norm_rotary.cu) share.
#pragma once

#include "rlkv_internal.cuh"

namespace rlkv {

// The sequences of a call, in the caller's order: entry i holds packed tokens start[i] .. start[i+1]-1, which stand at
// positions len[i], len[i]+1, ... of request slot slot[i].
struct ChunkSeqs {
    int n;
    int start[kMaxPagedBatch + 1];
    int len[kMaxPagedBatch];
    unsigned short slot[kMaxPagedBatch];
};
// The entry that holds packed token t (0 <= t < start[n]).
__device__ __forceinline__ int entry_of_token(const ChunkSeqs& s, int t)
{
    int lo = 0, hi = s.n - 1;  // the first entry whose end lies behind t
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (s.start[mid + 1] > t) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// ---- attention ----------------------------------------------------------------------------------------
// A UNIT is one KV head of one sequence and a row tile of its chunk: the queries of `tokens` consecutive tokens, all the
// query heads of the KV head packed into one tile of rows (token-major).  Its keys come in tiles of `kt`: first the chunk's own
// tokens, then the rows the cache holds (pages of a full head, the ring of a compressed one).
struct ChunkUnit {
    int tok0;        // first token of the row tile, inside the chunk
    int rows;        // cached rows that any of its queries may see
    int cached;      // tiles of them
    int a_end, b0;   // key tiles of the chunk: 0 .. a_end-1, then from b0 on (they come first)
    int tiles;       // in all
};
__host__ __device__ inline ChunkUnit chunk_unit(int len, int m, int row_tile, int tokens, int kt, bool full, int sink, int window)
{
    ChunkUnit u;
    u.tok0 = row_tile * tokens;
    const int last = u.tok0 + tokens < m ? u.tok0 + tokens : m, e = (last + kt - 1) / kt;
    if (full) {
        u.rows = len;
        u.a_end = u.b0 = e;
    } else {
        // the newest cached token is at len - 1; the tile's first query sees back to len + tok0 - window + 1
        const int cap = sink + window, held = len < cap ? len : cap, sunk = len < sink ? len : sink;
        u.rows = u.tok0 < window - 1 ? held : sunk;
        const int to_come = sink > len ? sink - len : 0;  // sink tokens that the chunk itself brings
        const int near = u.tok0 - window + 1 > 0 ? (u.tok0 - window + 1) / kt : 0;
        u.a_end = (to_come + kt - 1) / kt < e ? (to_come + kt - 1) / kt : e;
        u.b0 = u.a_end > near ? u.a_end : near;
    }
    u.cached = (u.rows + kt - 1) / kt;
    u.tiles = u.cached + u.a_end + (e - u.b0);
    return u;
}

// The units' key tiles form one flat sequence: sequence by sequence, row tile by row tile, the full heads and then the
// compressed ones.  It is cut into one contiguous range per CTA (all of them run at once), each of the same number of
// tiles, so that CTAs end together whatever the batch looks like.  A unit that a boundary cuts leaves a RECORD in every
// piece -- the rows' running maximum, sum and unscaled output -- which a second kernel adds up, in the order of the pieces.
// The CTA whose range begins in a unit keeps its record in 2 * cta, one whose range ends in it in 2 * cta + 1.
struct ChunkPos {
    unsigned short seq, head;  // entry; slot among the full heads, then among the compressed ones
    int row_tile, tile;
};
__host__ __device__ inline bool same_unit(const ChunkPos& a, const ChunkPos& b)
{
    return a.seq == b.seq && a.head == b.head && a.row_tile == b.row_tile;
}
constexpr int kMaxChunkCtas = 2 * 148;

// The chunks of a launch: entry i's `count[i]` tokens lie from packed token start[i] on.
struct ChunkList {
    int n;
    int start[kMaxPagedBatch], count[kMaxPagedBatch], len[kMaxPagedBatch];
    unsigned short slot[kMaxPagedBatch];
};

struct ChunkArgs {
    ChunkList seqs;
    const int* page_table;
    int table_stride, n_pages;
    long long full_row0, comp_row0;  // 16-bit pool: first rows of the layer's regions, as in PagedArgs
    int rows_comp;
    const unsigned char* pool8;      // 8-bit pool (null: 16-bit rows)
    long long page0_8, ring0_8;
    int ring_tiles;
    int n_full, n_comp, group, q_heads, sink, window;
    float scale, softcap;            // 1 / sqrt(head_dim); 0: no cap
    const float* slopes;             // device, [q_heads], or null
    __nv_bfloat16* out;              // [tokens][q_heads][head_dim]
    float* lse;                      // [tokens][q_heads], or null
    float* records;
    int* status;
    int ctas;
    ChunkPos at[kMaxChunkCtas + 1];  // where each CTA's range begins; the last entry: the end
    unsigned char head_of_slot[kMaxKvHeads];
    float k_scale[kMaxKvHeads], v_scale[kMaxKvHeads];  // by head
};
// The kernel's shapes: query rows of a unit's row tile, keys of a tile.  0: 32 rows, 64 keys; 1: 128 rows, 64 keys (both two
// CTAs on an SM); 2: two times 128 rows, 128 keys.
__host__ __device__ constexpr int chunk_keys(int shape) { return shape == 2 ? 128 : 64; }
__host__ __device__ constexpr int chunk_tokens(int shape, int group) { return shape == 2 ? 2 * (128 / group) : (shape == 1 ? 128 : 32) / group; }
// Floats of one record: of each sub-tile of R rows (32 or 128) [head_dim / 4][R] float4, then [2][R] maximum and sum.
__host__ __device__ constexpr long long chunk_record_floats(int head_dim, int shape) { return (shape == 2 ? 256ll : shape == 1 ? 128 : 32) * (head_dim + 2); }
// Two records a CTA, of the largest launches: kMaxChunkCtas of 128 rows, or half as many of 256.
inline size_t chunk_record_bytes(int head_dim) { return (size_t)2 * kMaxChunkCtas * chunk_record_floats(head_dim, 1) * sizeof(float); }
static_assert(chunk_record_floats(128, 2) == 2 * chunk_record_floats(128, 1) && chunk_record_floats(128, 0) <= chunk_record_floats(128, 1), "records");

// Status codes (device error word of the cache): which wait of the chunk kernel ran out.
enum : int { kChunkWaitLoad = 201, kChunkWaitProduct = 202, kChunkWaitSoftmax = 203, kChunkWaitStage = 204, kChunkWaitDrain = 205,
             kChunkWaitDecoded = 206, kChunkWaitQueries = 207, kChunkSmemMisaligned = 208 };

struct ChunkMaps {
    CUtensorMap q, k, v, pool;  // pool: 64 elements x 64 rows of the 16-bit pool, or whole pages of the 8-bit one
};
// pieces: most ranges that a unit lies in (1: none is cut)
cudaError_t launch_chunk_attention(const ChunkArgs& a, const ChunkMaps& m, int head_dim, int shape, int pieces, cudaStream_t stream);
cudaError_t prepare_chunk_kernels(int head_dim, bool fp8);

// ---- rows in and out of the cache -----------------------------------------------------------------------

struct ChunkRowsArgs {
    ChunkSeqs seqs;
    int* page_table;
    int table_stride, n_pages;
    __nv_bfloat16* pool;
    long long full_row0, comp_row0;
    int rows_comp;
    unsigned char* pool8;            // null: 16-bit rows
    long long page0_8, ring0_8;
    int ring_tiles, n_full, n_comp, kv_heads, head_dim, sink, window;
    const int* slot_of_head;         // device, [kv_heads]: >= 0 full slot, < 0: -(comp slot + 1)
    unsigned char head_of_slot[kMaxKvHeads];
    const float *k_inv, *v_inv;      // 1 / scale per KV head (written rows)
    const float *k_scale, *v_scale;  // scale per KV head (rows read back)
    const __nv_bfloat16 *k, *v;      // written: tokens *_stride elements apart
    long long k_stride, v_stride;
    __nv_bfloat16 *k_out, *v_out;    // read back: contiguous [tokens][kv_heads][head_dim]
    int length[kMaxPagedBatch];      // read back: tokens the sequence holds
};
// Blocks first_task[i] .. first_task[i+1]-1 serve entry i.  Rows written: the physical pages that they touch, entry by entry;
// entry i's begin at page0[i].
constexpr int kMaxChunkPages = 1024;
struct ChunkPages {
    int first_task[kMaxPagedBatch + 1];
    int page0[kMaxPagedBatch];
    int page[kMaxChunkPages];
};

cudaError_t launch_write_chunks(const ChunkRowsArgs& a, const ChunkPages& pages, cudaStream_t stream);
cudaError_t launch_read_rows(const ChunkRowsArgs& a, const ChunkPages& pages, cudaStream_t stream);

// ---- norms and rotation --------------------------------------------------------------------------------

struct NormRotaryArgs {
    const __nv_bfloat16 *q, *k;          // [n][heads][head_dim], tokens *_stride elements apart
    long long q_stride, k_stride;
    __nv_bfloat16 *q_out, *k_out;        // contiguous
    const __nv_bfloat16 *dq_out, *dk_out;  // contiguous
    __nv_bfloat16 *dq, *dk;
    long long dq_stride, dk_stride;
    const float* table;                  // [positions][rot / 2] (cos, sin), or null: no rotation
    int positions, rot, interleaved;     // (no table: any position that is not negative)
    const float *q_weight, *k_weight;    // [head_dim], or null: no norm
    float eps;
    const int* position;                 // device, [n], or null: token i at position i
    int n, q_heads, kv_heads, head_dim;
    float* partials;                     // [kMaxNormBlocks][head_dim]
    int* arrived;                        // [2], 0 between launches: blocks of the queries and of the keys that are done
    float *dq_weight, *dk_weight;
};
constexpr int kMaxNormBlocks = 148 * 2;
cudaError_t launch_norm_rotary(const NormRotaryArgs& a, cudaStream_t stream);
cudaError_t launch_norm_rotary_chunks(const NormRotaryArgs& a, const ChunkSeqs& seqs, cudaStream_t stream);
cudaError_t launch_norm_rotary_backward(const NormRotaryArgs& a, cudaStream_t stream);
cudaError_t prepare_norm_backward();

}  // namespace rlkv
