// Appending keys and values to the paged cache with the position rotation applied on the way, and the
// table of rotation angles.
//
// Token t's query and key heads are turned pairwise: (a, b) -> (a cos - b sin, b cos + a sin) with the
// angle t * inv_freq[j] of pair j (pairs (j, j + rot/2) or, interleaved, (2j, 2j + 1)); elements past
// `rot` pass through.  The products are computed in fp32 on the bf16 inputs and rounded ONCE: to bf16 for
// the rotated queries, the prompt's rotated keys and 16-bit rows, to the E4M3 code for 8-bit pages (from
// the fp32 value, not from its bf16 rounding).  With norms set, a query or key head is first divided by the root of its mean
// square and multiplied by the norm's weight, in fp32 as well: the lanes that hold a row's pieces add up its squares.  Where a row goes is the rule of append_kernel.cu.
#include "rotary.cuh"

namespace rlkv {
namespace {

// Where the K (kv = 0) or V (kv = 1) row of a token lands; `slot`: the head's place among the heads of its class.
struct RowPlace {
    bool stored;           // false: the prompt evicts the token before it ends
    __nv_bfloat16* row;    // 16-bit row
    unsigned char* page8;  // 8-bit page and the row inside it
    int prow;
};

__device__ __forceinline__ RowPlace place_of(const PagedAppendArgs& a, int slot, int kv, int seq, int t, int page)
{
    RowPlace p{true, nullptr, nullptr, 0};
    int phys = 0;
    if (slot < 0) {
        if (a.prefill && !(t < a.sink || t >= a.t0 + a.n - a.window)) {
            p.stored = false;
            return p;
        }
        phys = t < a.sink ? t : a.sink + (t - a.sink) % a.window;
    }
    if (a.pool8) {
        const long long index = slot >= 0 ? a.page0_8 + (long long)slot * a.n_pages + page
                                          : a.ring0_8 + ((long long)seq * a.n_comp + (-slot - 1)) * a.ring_tiles + phys / kTile;
        p.page8 = a.pool8 + index * (2 * kTile * 128);
        p.prow = slot >= 0 ? t % kTile : phys % kTile;
    } else {
        const long long row = slot >= 0 ? a.full_row0 + (((long long)slot * a.n_pages + page) * 2 + kv) * kTile + t % kTile
                                        : a.comp_row0 + (((long long)seq * a.n_comp + (-slot - 1)) * 2 + kv) * a.rows_comp + phys;
        p.row = a.pool + row * a.head_dim;
    }
    return p;
}

// Bound by memory: 8192 tokens of 32 / 8 heads of 128 read and write 210 MB in 41 us, 5.1 TB/s (78 % of a copy's rate).  One
// thread per piece and head, its angles read again for every head, took 57 us; two or eight heads' loads at a time 49 and 60
// (fewer in flight; fewer threads), more threads with spilled registers 62.  Few tokens are launch latency: 2.5 us.
// An 8-bit cache takes 44.7 us for the same prompt, which moves 197 MB, and 7.7 for a token each of 64 sequences (2.6 in 16 bits):
// a V thread writes its sixteen transposed codes one byte at a time.
// A block takes 256 / PIECES tokens and `heads` of the heads (numbered q heads, K heads, V heads).  A thread keeps
// one piece of one token: its eight angles stay in registers over the heads, whose loads are issued four at a time.
template <int PIECES, bool NORM>
__global__ void __launch_bounds__(256) rotated_append_kernel(const __grid_constant__ RotatedAppendArgs r, const int heads)
{
    constexpr int kTokens = 256 / PIECES, kBatch = 4;
    const PagedAppendArgs& a = r.rows;
    const int q_heads = r.q ? r.q_heads : 0, rows = q_heads + 2 * a.kv_heads;
    const int head0 = blockIdx.y * heads, head1 = min(rows, head0 + heads);
    // pieces of one row in neighbouring lanes; the transposed V codes of an 8-bit page the other way round: tokens in
    // neighbouring lanes write neighbouring bytes
    const int v_turned = a.pool8 ? max(head0, q_heads + a.kv_heads) : head1;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
        const int from = pass ? v_turned : head0, to = pass ? head1 : min(head1, v_turned);
        if (from >= to) continue;
        const int piece = pass ? threadIdx.x / kTokens : threadIdx.x % PIECES;
        const int e = blockIdx.x * kTokens + (pass ? threadIdx.x % kTokens : threadIdx.x / PIECES);
        if (e >= a.n) continue;
        const int seq = a.prefill ? a.slot[0] : a.slot[e];
        const int t = a.prefill ? a.t0 + e : a.t[e];
        const int page = a.page[a.prefill ? t / kTile - a.first_page : e];
        // the piece's two runs of eight elements: the two halves of eight pairs, or sixteen in a row
        const bool turned = piece * kPiece < r.rot;
        float2 f[8];
        if (turned && from < q_heads + a.kv_heads) {
            load_angles(r.table, t, r.rot, piece, f);
        }
        for (int base = from; base < to; base += kBatch) {
            uint4 b[kBatch][2];
#pragma unroll
            for (int x = 0; x < kBatch; ++x) {
                const int hh = base + x;
                if (hh < to) {
                    const bool is_q = hh < q_heads, is_v = hh >= q_heads + a.kv_heads;
                    const int h = is_q ? hh : hh - q_heads - (is_v ? a.kv_heads : 0);
                    const bool halves = turned && !is_v && !r.interleaved;
                    const int c0 = halves ? piece * 8 : piece * kPiece, c1 = halves ? c0 + r.rot / 2 : c0 + 8;
                    const __nv_bfloat16* src = (is_q ? r.q + e * r.q_stride : is_v ? a.v + e * r.v_stride : a.k + e * r.k_stride) + h * a.head_dim;
                    b[x][0] = *reinterpret_cast<const uint4*>(src + c0);
                    b[x][1] = *reinterpret_cast<const uint4*>(src + c1);
                }
            }
#pragma unroll
            for (int x = 0; x < kBatch; ++x) {
                const int hh = base + x;
                if (hh >= to) break;
                const bool is_q = hh < q_heads, is_v = hh >= q_heads + a.kv_heads;
                const int h = is_q ? hh : hh - q_heads - (is_v ? a.kv_heads : 0);
                const bool turn = turned && !is_v, halves = turn && !r.interleaved;
                const int c0 = halves ? piece * 8 : piece * kPiece, c1 = halves ? c0 + r.rot / 2 : c0 + 8;
                float x0[8], x1[8];
                unpack8(b[x][0], x0);
                unpack8(b[x][1], x1);
                if (NORM && !is_v) {
                    const float* weight = is_q ? r.q_weight : r.k_weight;
                    if (weight) {
                        const float rms = row_rsqrt<PIECES>(x0, x1, r.eps);
                        float w0[8], w1[8];
                        load8(weight + c0, w0);
                        load8(weight + c1, w1);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            x0[j] = x0[j] * rms * w0[j];
                            x1[j] = x1[j] * rms * w1[j];
                        }
                    }
                }
                if (turn) rotate_piece(x0, x1, f, r.interleaved);
                if (turn || (NORM && !is_v)) {
                    b[x][0] = pack8(x0);
                    b[x][1] = pack8(x1);
                }
                if (is_q || (!is_v && r.k_out)) {
                    __nv_bfloat16* dst = is_q ? r.q_out + ((long long)e * q_heads + h) * a.head_dim
                                              : r.k_out + ((long long)e * a.kv_heads + h) * a.head_dim;
                    *reinterpret_cast<uint4*>(dst + c0) = b[x][0];
                    *reinterpret_cast<uint4*>(dst + c1) = b[x][1];
                    if (is_q) continue;
                }
                const int slot = a.slot_of_head[h];
                if (!is_v && piece == 0 && slot == 0) a.page_table[(size_t)seq * a.table_stride + t / kTile] = page;
                const RowPlace p = place_of(a, slot, is_v, seq, t, page);
                if (!p.stored) continue;
                if (!a.pool8) {
                    *reinterpret_cast<uint4*>(p.row + c0) = b[x][0];
                    *reinterpret_cast<uint4*>(p.row + c1) = b[x][1];
                    continue;
                }
                const float inv = (is_v ? a.v_inv : a.k_inv)[h];
                const uint2 k0 = codes8(x0, inv), k1 = codes8(x1, inv);
                if (!is_v) {
                    *reinterpret_cast<uint2*>(p.page8 + p.prow * 128 + c0) = k0;
                    *reinterpret_cast<uint2*>(p.page8 + p.prow * 128 + c1) = k1;
                } else {  // V codes lie transposed behind the K codes
                    unsigned char* col = p.page8 + kTile * 128 + p.prow;
                    const unsigned char* u0 = reinterpret_cast<const unsigned char*>(&k0);
                    const unsigned char* u1 = reinterpret_cast<const unsigned char*>(&k1);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        col[(c0 + j) * kTile] = u0[j];
                        col[(c1 + j) * kTile] = u1[j];
                    }
                }
            }
        }
    }
}

// cos and sin of position * inv_freq, in 64 bits: an fp32 product is off by half a step of the ANGLE,
// which at position 65535 is 2^-9 of a turn's radian -- as much as a bf16 rounding.
__global__ void __launch_bounds__(256) rotary_table_kernel(const __grid_constant__ RotaryTableArgs a)
{
    const long long total = (long long)a.positions * a.pairs;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (long long)gridDim.x * blockDim.x) {
        const int p = (int)(i / a.pairs), j = (int)(i - (long long)p * a.pairs);
        double s, c;
        sincos((double)p * a.inv_freq[j], &s, &c);
        a.table[i] = make_float2((float)c, (float)s);
    }
}

unsigned blocks_for(long long threads, int most)
{
    long long b = (threads + 255) / 256;
    return (unsigned)(b > most ? most : b < 1 ? 1 : b);
}

}  // namespace

cudaError_t launch_rotated_append(const RotatedAppendArgs& a, cudaStream_t stream)
{
    const int pieces = a.rows.head_dim / kPiece, tokens = 256 / pieces;
    const int rows = (a.q ? a.q_heads : 0) + 2 * a.rows.kv_heads, tiles = (a.rows.n + tokens - 1) / tokens;
    // heads per block: enough blocks to fill the GPU first (few tokens: one head a block, the launch is all latency),
    // then as many heads as share one load of the angles
    int heads = 1;
    while (heads < 8 && (long long)tiles * ((rows + 2 * heads - 1) / (2 * heads)) >= 148 * 8) heads *= 2;
    const dim3 grid(tiles, (rows + heads - 1) / heads);
    if (a.q_weight || a.k_weight) {
        if (pieces == 8) rotated_append_kernel<8, true><<<grid, 256, 0, stream>>>(a, heads);
        else rotated_append_kernel<4, true><<<grid, 256, 0, stream>>>(a, heads);
    } else {
        if (pieces == 8) rotated_append_kernel<8, false><<<grid, 256, 0, stream>>>(a, heads);
        else rotated_append_kernel<4, false><<<grid, 256, 0, stream>>>(a, heads);
    }
    return cudaGetLastError();
}

cudaError_t launch_rotary_table(const RotaryTableArgs& a, cudaStream_t stream)
{
    rotary_table_kernel<<<blocks_for((long long)a.positions * a.pairs, 148 * 32), 256, 0, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace rlkv
