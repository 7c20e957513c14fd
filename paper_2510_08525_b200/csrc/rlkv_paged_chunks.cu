// Host side of the calls that take a chunk of tokens of each of several sequences of the paged cache (rlkv_paged_rotate_chunks,
// rlkv_paged_chunk_attention, rlkv_paged_append_chunks, rlkv_paged_read in include/rlkv.h).
#include <math.h>
#include <string.h>

#include "rlkv_chunk.cuh"
#include "rlkv_paged.cuh"

using namespace rlkv;

namespace {

constexpr int kMaxChunkTokens = 1 << 24;  // of one call
// Keys of a CTA's range, at least: three times 100 tokens on 500, 8 bits, tiles of 128, 30 us with 512, 27 so; tiles of 64: 27 to 28 us
// for 512 on 1000 with 64 to 512, 31 with 768.
constexpr int kMinChunkKeys = 256;

// What a unit's start and end -- its queries' way to shared memory, the first product, its results -- count as in key tiles.  Measured
// over counts from 1 to 14: 32 rows a unit, 16 bits: 48 single tokens on 3400 each 58 us with 3, 52 with 6, 54 with 10, four drafted
// tokens of 32 sequences 130, 131 and 135; 8 bits, whose tiles take half as long: 75, 65 and 59 us, 122, 114 and 108; 128 rows: 512
// tokens beside 47 single ones 105 us with 1, 97 with 4; two times 128 rows: a prompt of 8192 tokens 668 us with 1, 483 with 3.
int unit_tiles(int shape, bool fp8) { return shape == 2 ? 3 : shape == 1 ? 4 : fp8 ? 10 : 5; }

// The sequences of a call: open slots, none twice, `counts` tokens each, from `first` on (null: behind those held).  `to`:
// most tokens a sequence may come to; more are `over`.
int check_chunks(const rlkv_paged* p, int layer, const int* slots, const int* first, const int* counts, int n, bool held, ChunkSeqs& s)
{
    if (!valid_layer(p, layer) || !slots || !counts || n < 1 || n > p->max_batch) return RLKV_EINVAL;
    uint64_t seen[65536 / 64];
    memset(seen, 0, sizeof(uint64_t) * ((size_t)(p->max_seqs + 63) / 64));
    const int* len = len_of(p, layer);
    s.n = n;
    long long at = 0;
    bool over = false;
    for (int i = 0; i < n; ++i) {
        const int slot = slots[i];
        if (!valid_slot(p, slot) || (seen[slot / 64] >> (slot % 64) & 1) || counts[i] < 0) return RLKV_EINVAL;
        seen[slot / 64] |= 1ull << (slot % 64);
        const int from = first ? first[i] : len[slot];
        if (from < 0 || (held && (long long)from + counts[i] > len[slot])) return RLKV_EINVAL;
        if ((long long)from + counts[i] > p->max_seq_len) over = true;
        s.slot[i] = (unsigned short)slot;
        s.len[i] = from;
        s.start[i] = (int)at;
        at += counts[i];
        if (at > kMaxChunkTokens) return RLKV_EINVAL;
    }
    s.start[n] = (int)at;
    return over ? RLKV_EFULL : RLKV_OK;
}

// Strides of rows of `heads` heads: 0 stands for contiguous tokens.
bool check_stride(const rlkv_paged* p, int heads, int64_t& stride)
{
    const int64_t row = (int64_t)heads * p->head_dim;
    if (!stride) stride = row;
    return stride >= row && stride % 8 == 0 && stride <= (int64_t)1 << 30;
}

void fill_rows_args(rlkv_paged* p, int layer, ChunkRowsArgs& a)
{
    a.page_table = dev_at<int>(p, p->off_page_table);
    a.table_stride = p->table_stride;
    a.n_pages = p->n_pages;
    a.pool = dev_at<__nv_bfloat16>(p, p->off_pool);
    a.full_row0 = p->full_row0[layer];
    a.comp_row0 = p->comp_row0[layer];
    a.rows_comp = p->rows_comp;
    a.pool8 = p->fp8 ? p->dev_base + p->off_pool8 : nullptr;
    a.page0_8 = p->page0_8[layer];
    a.ring0_8 = p->ring0_8[layer];
    a.ring_tiles = p->rows_comp / kTile;
    a.n_full = p->n_full[layer];
    a.n_comp = p->n_comp[layer];
    a.kv_heads = p->kv_heads;
    a.head_dim = p->head_dim;
    a.sink = p->sink;
    a.window = p->window;
    a.slot_of_head = dev_at<int>(p, p->off_tables) + (size_t)layer * p->kv_heads;
    const float* scales = dev_at<float>(p, p->off_scales) + (size_t)layer * p->kv_heads;
    const size_t all = (size_t)p->layers * p->kv_heads;
    a.k_inv = scales;
    a.v_inv = scales + all;
    a.k_scale = scales + 2 * all;
    a.v_scale = scales + 3 * all;
    for (int h = 0; h < p->kv_heads; ++h) a.head_of_slot[h] = (unsigned char)p->head_of_slot[(size_t)layer * p->kv_heads + h];
}

// Cuts the flat sequence of the units' key tiles for at most max_ctas CTAs of at least min_tiles tiles; a unit counts `extra`
// tiles more than it has (its queries' load and its results cost about as much).  Returns the most ranges that one unit lies in.
int plan_chunks(ChunkArgs& a, int shape, int max_ctas, int min_tiles, int extra)
{
    const int keys = chunk_keys(shape), tokens = chunk_tokens(shape, a.group);
    const ChunkList& s = a.seqs;
    auto unit = [&](int i, int j, bool full) {
        return chunk_unit(s.len[i], s.count[i], j, tokens, keys, full, a.sink, a.window).tiles + extra;
    };
    auto row_tiles = [&](int i) { return (s.count[i] + tokens - 1) / tokens; };
    long long all = 0;
    for (int i = 0; i < s.n; ++i)
        for (int j = 0; j < row_tiles(i); ++j) {
            if (a.n_full) all += (long long)a.n_full * unit(i, j, true);
            if (a.n_comp) all += (long long)a.n_comp * unit(i, j, false);
        }
    long long ctas = all / (min_tiles + extra);
    if (ctas > max_ctas) ctas = max_ctas;
    if (ctas < 1) ctas = 1;
    a.ctas = (int)ctas;
    int c = 0, pieces = 1, most = 1;
    long long x = 0;  // flat tiles before the units at hand
    auto boundary = [&](int k) { return all * k / ctas; };
    for (int i = 0; i < s.n; ++i)
        for (int j = 0; j < row_tiles(i); ++j)
            for (int comp = 0; comp < 2; ++comp) {
                const int heads = comp ? a.n_comp : a.n_full;
                if (!heads) continue;
                const int each = unit(i, j, !comp);
                while (c < ctas && boundary(c) < x + (long long)heads * each) {
                    const long long y = boundary(c) - x;
                    ChunkPos& at = a.at[c++];
                    at.seq = (unsigned short)i;
                    at.head = (unsigned short)((comp ? a.n_full : 0) + (int)(y / each));
                    at.row_tile = j;
                    at.tile = (int)(y % each) - extra;
                    if (at.tile < 0) at.tile = 0;
                    pieces = at.tile == 0 ? 1 : c > 1 && same_unit(a.at[c - 2], at) ? pieces + 1 : 2;
                    if (pieces > most) most = pieces;
                }
                x += (long long)heads * each;
            }
    for (; c <= ctas; ++c) a.at[c] = ChunkPos{(unsigned short)s.n, 0, 0, 0};
    return most;
}

// The shape of a launch.  32 rows where every chunk's queries of a KV head fit them.  Two sub-tiles of 128 are for launches most of whose
// key tiles belong to chunks that fill more than one: on an 8-bit cache for all of these, since a tile's codes are decoded once for
// both (us with one sub-tile and so: a prompt of 8192 tokens 877 and 651, 512 tokens on 3400 65 and 57, three times 100 on 500 31
// and 30), but few others beside them, whose tiles are as long (512 tokens on 3400 beside 11 single ones 94 and 110); in 16 bits where
// the K and V rows are too many for the L2, in which the other tiles of rows would find them (four times 512 on 8192 300 and 270, 64
// of each of 32 sequences on 8064 341 and 272) and every SM has 32 such tiles of 128 keys (64 tokens on 40000 62 and 65), or where it
// has 100 (2048 on 8192 280 and 282, under the power cap 320 and 315, a prompt of 8192 497 and 490; eight times 512 on 3400, 6 of 8 full,
// 203 and 209: near this line the two are within 3 %, either way); but 512 on 8192 78 and 81, four times 512 on 3400 111 and 117.
constexpr long long kNearL2 = 80ll << 20;
// Key rows that a chunk of m tokens meets over all heads, on average over its tokens: of a ring no more than the sequence has.
long long key_rows(const ChunkArgs& a, int len, int m)
{
    const long long held = (long long)len + m / 2, ring = a.sink + a.window;
    return a.n_full * held + a.n_comp * (held < ring ? held : ring);
}
int choose_shape(const ChunkArgs& a, int sms, int head_dim, bool fp8)
{
    long long small = 0, large = 0, shared = 0;  // key rows times row tiles of 128; rows that several of these read
    bool few = true;
    for (int i = 0; i < a.seqs.n; ++i) {
        const int m = a.seqs.count[i];
        if (m > chunk_tokens(0, a.group)) few = false;
        const long long rows = key_rows(a, a.seqs.len[i], m);
        const int tiles = (int)(((long long)m * a.group + 127) / 128);
        (tiles > 1 ? large : small) += rows * tiles;
        if (tiles > 1) shared += rows;
    }
    if (few) return 0;
    if (large <= (fp8 ? 4 * small : small)) return 1;
    return fp8 || large / 256 >= (shared * head_dim * 4 > kNearL2 ? 32ll : 100ll) * sms ? 2 : 1;
}

// Whether chunks of at most 32 rows and the others go out as two launches, each in its own shape.  In 16 bits one launch is shorter
// (one kind's products run beside the other's stream: 512 tokens on 3400 beside 47 single ones on 1700 71 us, apart 52 and 36); in 8
// bits its one sub-tile is not (139 us, as two 130; on 3400 all 172 and 154; 1024 tokens of a new prompt beside 47 126 and 107), unless
// either kind is little (40 tokens on 100 beside 16 single ones on 2000 46, apart 34 and 15; 300 on 3400 beside 23, all full, 116 and 118).
bool two_launches(const ChunkSeqs& s, const ChunkArgs& a, int sms, bool fp8)
{
    if (!fp8) return false;
    long long few = 0, more = 0;  // key rows times row tiles of 128
    for (int i = 0; i < s.n; ++i) {
        const int m = s.start[i + 1] - s.start[i];
        const long long rows = key_rows(a, s.len[i], m);
        if (m > 0) (m * a.group <= 32 ? few : more) += rows * (((long long)m * a.group + 127) / 128);
    }
    return few / 256 >= 6ll * sms && more / 256 >= 2ll * sms;
}

// The chunks of a launch, 0: all, 1: those of at most 32 rows, 2: the others; empty ones in none.  entries: where each stands in the call
// (or null).
void pick_chunks(const ChunkSeqs& s, int group, int pick, ChunkList& l, int* entries)
{
    l.n = 0;
    for (int i = 0; i < s.n; ++i) {
        const int m = s.start[i + 1] - s.start[i];
        if (m == 0 || (pick && (m * group <= 32) != (pick == 1))) continue;
        if (entries) entries[l.n] = i;
        l.start[l.n] = s.start[i];
        l.count[l.n] = m;
        l.len[l.n] = s.len[i];
        l.slot[l.n++] = s.slot[i];
    }
}

// Launch `which` of a call's (two: the small chunks and the others): its chunks, its shape and its CTAs' ranges, with records in `bytes`.
struct Cut {
    int shape, pieces;
};
Cut cut_launch(const ChunkSeqs& s, ChunkArgs& a, bool two, int which, int sms, int head_dim, bool fp8, size_t bytes, int* entries)
{
    Cut c;
    pick_chunks(s, a.group, two ? 1 + which : 0, a.seqs, entries);
    c.shape = choose_shape(a, sms, head_dim, fp8);
    const long long room = (long long)(bytes / (2 * sizeof(float) * chunk_record_floats(head_dim, c.shape)));  // CTAs there are records for
    int ctas = c.shape == 2 ? sms : 2 * sms;
    if (ctas > room) ctas = room < 1 ? 1 : (int)room;  // (one alone cuts no unit: it leaves no record)
    c.pieces = plan_chunks(a, c.shape, ctas, kMinChunkKeys / chunk_keys(c.shape), unit_tiles(c.shape, fp8));
    return c;
}

// A boundary per CTA and the end, four numbers each; sequences as in the call.
void write_ranges(const ChunkArgs& a, const int* entries, int n, int* at_out)
{
    for (int c = 0; c <= a.ctas; ++c) {
        const int seq = a.at[c].seq;
        at_out[4 * c] = !entries ? seq : seq < a.seqs.n ? entries[seq] : n;
        at_out[4 * c + 1] = a.at[c].row_tile;
        at_out[4 * c + 2] = a.at[c].head;
        at_out[4 * c + 3] = a.at[c].tile;
    }
}

// The arguments that the two below share, checked.
int debug_args(const int* lens, const int* counts, int n, int n_full, int n_comp, int group, int sink, int window, ChunkSeqs& s, ChunkArgs& a)
{
    if (!lens || !counts || n < 1 || n > kMaxPagedBatch || n_full < 0 || n_comp < 0 || n_full + n_comp < 1 || group < 1 || group > kMaxGroup ||
        sink < 0 || window < 1)
        return RLKV_EINVAL;
    s.n = n;
    long long total = 0;
    for (int i = 0; i < n; ++i) {
        if (lens[i] < 0 || counts[i] < 0) return RLKV_EINVAL;
        s.len[i] = lens[i];
        s.start[i] = (int)total;
        s.slot[i] = 0;
        total += counts[i];
        if (total > kMaxChunkTokens) return RLKV_EINVAL;
    }
    if (total < 1) return RLKV_EINVAL;
    s.start[n] = (int)total;
    a.n_full = n_full;
    a.n_comp = n_comp;
    a.group = group;
    a.sink = sink;
    a.window = window;
    return RLKV_OK;
}

// Records for every CTA of a launch, before the first call: memory of the library's own where the decode launches' records, which serve
// calls on the same cache in turn, take less.  (In a captured call, too: the allocation is no part of the graph.)  Where there is
// none left those serve, with fewer CTAs to a launch, from then on.
void settle_scratch(rlkv_paged* p)
{
    if (p->chunk_settled) return;
    p->chunk_settled = true;
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    cudaThreadExchangeStreamCaptureMode(&mode);
    void* mem = nullptr;
    if (cudaMalloc(&mem, chunk_record_bytes(p->head_dim)) == cudaSuccess) {
        p->chunk_records = p->own_records = static_cast<float*>(mem);
        p->chunk_bytes = chunk_record_bytes(p->head_dim);
    } else {
        cudaGetLastError();
    }
    cudaThreadExchangeStreamCaptureMode(&mode);
}

}  // namespace

extern "C" {

int rlkv_paged_chunk_scratch_size(const rlkv_paged* p, size_t* bytes_out)
{
    if (!p || !bytes_out) return RLKV_EINVAL;
    *bytes_out = chunk_record_bytes(p->head_dim);
    return RLKV_OK;
}

int rlkv_paged_set_chunk_scratch(rlkv_paged* p, void* scratch, size_t bytes)
{
    if (!p || (scratch && !on_device(scratch, p->device))) return RLKV_EINVAL;
    const size_t all = chunk_record_bytes(p->head_dim), decode = p->total - p->off_partials;
    p->chunk_settled = scratch || p->own_records || decode >= all;
    p->chunk_records = scratch ? static_cast<float*>(scratch) : p->own_records ? p->own_records : dev_at<float>(p, p->off_partials);
    p->chunk_bytes = scratch ? bytes : p->own_records ? all : decode;
    return RLKV_OK;
}

int rlkv_paged_set_norms(rlkv_paged* p, const float* q_weight, const float* k_weight, float eps)
{
    if (!p) return RLKV_EINVAL;
    if (q_weight || k_weight) {
        if (!(eps > 0.f) || !(eps <= 1.f)) return RLKV_EINVAL;
        for (const float* w : {q_weight, k_weight})
            if (w && !on_device(w, p->device)) return RLKV_EINVAL;
    }
    p->q_norm = q_weight;
    p->k_norm = k_weight;
    p->norm_eps = eps;
    return RLKV_OK;
}

int rlkv_paged_rotate_chunks(rlkv_paged* p, int layer, const int* slots, const int* counts, int n, const void* q, int64_t q_stride,
                             const void* k, int64_t k_stride, void* q_out, void* k_out, void* stream)
{
    ChunkSeqs s;
    const int rc = check_chunks(p, layer, slots, nullptr, counts, n, false, s);
    if (rc) return rc;
    if (!p->rotary && !p->q_norm && !p->k_norm) return RLKV_EINVAL;
    if (!check_stride(p, p->q_heads, q_stride) || !check_stride(p, p->kv_heads, k_stride)) return RLKV_EINVAL;
    for (int i = 0; i < n; ++i)
        if (p->rotary && counts[i] > 0 && (long long)s.len[i] + counts[i] > p->rotary_rows) return RLKV_EINVAL;
    if (s.start[n] == 0) return RLKV_OK;
    if (!q || !k || !q_out || !k_out || !aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out)) return RLKV_EINVAL;
    DeviceGuard g(p->device);
    if (!g.ok) return RLKV_ECUDA;
    NormRotaryArgs a;
    memset(&a, 0, sizeof a);
    a.q = static_cast<const __nv_bfloat16*>(q);
    a.k = static_cast<const __nv_bfloat16*>(k);
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.q_out = static_cast<__nv_bfloat16*>(q_out);
    a.k_out = static_cast<__nv_bfloat16*>(k_out);
    a.table = p->rotary;
    a.positions = p->rotary ? p->rotary_rows : kMaxSeqPages * kTile;
    a.rot = p->rotary_dim;
    a.interleaved = p->rotary_interleaved;
    a.q_weight = p->q_norm ? p->q_norm + (size_t)layer * p->head_dim : nullptr;
    a.k_weight = p->k_norm ? p->k_norm + (size_t)layer * p->head_dim : nullptr;
    a.eps = p->norm_eps;
    a.n = s.start[n];
    a.q_heads = p->q_heads;
    a.kv_heads = p->kv_heads;
    a.head_dim = p->head_dim;
    RLKV_CUDA(launch_norm_rotary_chunks(a, s, static_cast<cudaStream_t>(stream)));
    p->launches++;
    return RLKV_OK;
}

int rlkv_paged_chunk_attention(rlkv_paged* p, int layer, const int* slots, const int* counts, int n, const void* q, int64_t q_stride,
                               const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* out, float* lse, void* stream)
{
    ChunkSeqs s;
    ChunkArgs a;
    const int rc = check_chunks(p, layer, slots, nullptr, counts, n, false, s);
    if (rc) return rc;
    if (!check_stride(p, p->q_heads, q_stride) || !check_stride(p, p->kv_heads, k_stride) || !check_stride(p, p->kv_heads, v_stride))
        return RLKV_EINVAL;
    const int total = s.start[n];
    if (total == 0) return RLKV_OK;
    if (!q || !k || !v || !out || !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || (reinterpret_cast<uintptr_t>(lse) & 3))
        return RLKV_EINVAL;
    DeviceGuard g(p->device);
    if (!g.ok) return RLKV_ECUDA;
    a.page_table = dev_at<int>(p, p->off_page_table);
    a.table_stride = p->table_stride;
    a.n_pages = p->n_pages;
    a.full_row0 = p->full_row0[layer];
    a.comp_row0 = p->comp_row0[layer];
    a.rows_comp = p->rows_comp;
    a.pool8 = p->fp8 ? p->dev_base + p->off_pool8 : nullptr;
    a.page0_8 = p->page0_8[layer];
    a.ring0_8 = p->ring0_8[layer];
    a.ring_tiles = p->rows_comp / kTile;
    a.n_full = p->n_full[layer];
    a.n_comp = p->n_comp[layer];
    a.group = p->q_heads / p->kv_heads;
    a.q_heads = p->q_heads;
    a.sink = p->sink;
    a.window = p->window;
    a.scale = 1.f / sqrtf((float)p->head_dim);
    a.softcap = p->softcap;
    a.slopes = p->biased ? dev_at<float>(p, p->off_slopes) + (size_t)layer * p->q_heads : nullptr;
    a.out = static_cast<__nv_bfloat16*>(out);
    a.lse = lse;
    settle_scratch(p);
    a.records = p->chunk_records;
    a.status = dev_at<int>(p, p->off_status);
    for (int h = 0; h < p->kv_heads; ++h) {
        a.head_of_slot[h] = (unsigned char)p->head_of_slot[(size_t)layer * p->kv_heads + h];
        a.k_scale[h] = p->fp8 ? p->k_scale[(size_t)layer * p->kv_heads + h] : 1.f;
        a.v_scale[h] = p->fp8 ? p->v_scale[(size_t)layer * p->kv_heads + h] : 1.f;
    }
    const int sms = p->sm_count < kMaxChunkCtas / 2 ? p->sm_count : kMaxChunkCtas / 2;
    const bool two = two_launches(s, a, sms, p->fp8);
    for (int which = 0; which < 1 + two; ++which) {
        const Cut cut = cut_launch(s, a, two, which, sms, p->head_dim, p->fp8, p->chunk_bytes, nullptr);
        const int keys = chunk_keys(cut.shape);
        ChunkMaps m;
        int e = encode_heads_map(&m.q, q, total, p->q_heads, p->head_dim, q_stride, a.group, (cut.shape == 0 ? 32 : 128) / a.group);
        if (!e) e = encode_heads_map(&m.k, k, total, p->kv_heads, p->head_dim, k_stride, 1, keys);
        if (!e) e = encode_heads_map(&m.v, v, total, p->kv_heads, p->head_dim, v_stride, 1, keys);
        if (!e && !p->fp8) e = encode_heads_map(&m.pool, dev_at<__nv_bfloat16>(p, p->off_pool), p->pool_rows, 1, p->head_dim, p->head_dim, 1, kTile);
        else if (!e) m.pool = cut.shape == 2 ? p->map_codes : p->map_k;
        if (e) return e;
        RLKV_CUDA(launch_chunk_attention(a, m, p->head_dim, cut.shape, cut.pieces, static_cast<cudaStream_t>(stream)));
        p->launches += cut.pieces > 1 ? 2 : 1;
    }
    return RLKV_OK;
}

int rlkv_paged_append_chunks(rlkv_paged* p, int layer, const int* slots, const int* counts, int n, const void* k, int64_t k_stride,
                             const void* v, int64_t v_stride, void* stream)
{
    ChunkSeqs s;
    int rc = check_chunks(p, layer, slots, nullptr, counts, n, false, s);
    if (rc) return rc;
    if (!check_stride(p, p->kv_heads, k_stride) || !check_stride(p, p->kv_heads, v_stride)) return RLKV_EINVAL;
    if (s.start[n] == 0) return RLKV_OK;
    if (!k || !v || !aligned16(k) || !aligned16(v)) return RLKV_EINVAL;
    auto first_page = [&](int i) { return s.len[i] / kTile; };
    auto end_page = [&](int i) { return counts[i] ? (s.len[i] + counts[i] - 1) / kTile + 1 : first_page(i); };
    // every page there is room for, before anything changes
    long long need = 0;
    for (int i = 0; i < n; ++i)
        for (int j = first_page(i); j < end_page(i); ++j)
            if (p->table[(size_t)slots[i] * p->table_stride + j] < 0) ++need;
    if (need > (long long)p->free_pages.size()) return RLKV_EFULL;
    DeviceGuard g(p->device);
    if (!g.ok) return RLKV_ECUDA;
    for (int i = 0; i < n; ++i)
        for (int j = first_page(i); j < end_page(i); ++j) {
            int& entry = p->table[(size_t)slots[i] * p->table_stride + j];
            if (entry < 0) {
                entry = p->free_pages.back();
                p->free_pages.pop_back();
            }
        }
    // launches of as many sequences as the arguments can name pages for (one sequence's always fit)
    for (int i0 = 0; i0 < n;) {
        ChunkRowsArgs a;
        ChunkPages pages;
        fill_rows_args(p, layer, a);
        a.k = static_cast<const __nv_bfloat16*>(k);
        a.v = static_cast<const __nv_bfloat16*>(v);
        a.k_stride = k_stride;
        a.v_stride = v_stride;
        int named = 0, tasks = 0, i = i0;
        for (; i < n && named + end_page(i) - first_page(i) <= kMaxChunkPages; ++i) {
            const int x = i - i0, count = end_page(i) - first_page(i);
            a.seqs.slot[x] = s.slot[i];
            a.seqs.len[x] = s.len[i];
            a.seqs.start[x] = s.start[i];
            pages.first_task[x] = tasks;
            pages.page0[x] = named;
            for (int j = 0; j < count; ++j) pages.page[named + j] = p->table[(size_t)slots[i] * p->table_stride + first_page(i) + j];
            named += count;
            if (counts[i]) tasks += count * a.n_full + a.ring_tiles * a.n_comp;
        }
        a.seqs.n = i - i0;
        a.seqs.start[i - i0] = s.start[i];
        pages.first_task[i - i0] = tasks;
        if (tasks) {
            RLKV_CUDA(launch_write_chunks(a, pages, static_cast<cudaStream_t>(stream)));
            p->launches++;
        }
        i0 = i;
    }
    int* len = len_of(p, layer);
    for (int i = 0; i < n; ++i) len[slots[i]] += counts[i];
    return RLKV_OK;
}

int rlkv_paged_read(rlkv_paged* p, int layer, const int* slots, const int* first, const int* counts, int n, void* k_out, void* v_out,
                    void* stream)
{
    ChunkRowsArgs a;
    if (!first) return RLKV_EINVAL;
    const int rc = check_chunks(p, layer, slots, first, counts, n, true, a.seqs);
    if (rc) return rc;
    if (a.seqs.start[n] == 0) return RLKV_OK;
    if (!k_out || !v_out || !aligned16(k_out) || !aligned16(v_out)) return RLKV_EINVAL;
    DeviceGuard g(p->device);
    if (!g.ok) return RLKV_ECUDA;
    fill_rows_args(p, layer, a);
    a.k_out = static_cast<__nv_bfloat16*>(k_out);
    a.v_out = static_cast<__nv_bfloat16*>(v_out);
    ChunkPages pages;
    long long tasks = 0;
    for (int i = 0; i < n; ++i) {
        a.length[i] = len_of(p, layer)[slots[i]];
        pages.first_task[i] = (int)tasks;
        if (counts[i]) tasks += (long long)((first[i] + counts[i] - 1) / kTile - first[i] / kTile + 1) * p->kv_heads;
        if (tasks >= 1ll << 31) return RLKV_EINVAL;
    }
    pages.first_task[n] = (int)tasks;
    RLKV_CUDA(launch_read_rows(a, pages, static_cast<cudaStream_t>(stream)));
    p->launches++;
    return RLKV_OK;
}

int rlkv_debug_chunk_plan(const int* lens, const int* counts, int n, int n_full, int n_comp, int group, int sink, int window, int shape,
                          int max_ctas, int* ctas_out, int* at_out)
{
    if (max_ctas < 1 || max_ctas > kMaxChunkCtas || !ctas_out || !at_out) return RLKV_EINVAL;
    ChunkSeqs s;
    ChunkArgs a;
    const int rc = debug_args(lens, counts, n, n_full, n_comp, group, sink, window, s, a);
    if (rc) return rc;
    a.seqs.n = n;
    for (int i = 0; i < n; ++i) {
        a.seqs.len[i] = lens[i];
        a.seqs.start[i] = s.start[i];
        a.seqs.count[i] = counts[i];
    }
    if (shape < 0) shape = choose_shape(a, kMaxChunkCtas / 2, 128, shape == -2);
    if (shape > 2) return RLKV_EINVAL;
    plan_chunks(a, shape, max_ctas, kMinChunkKeys / chunk_keys(shape), unit_tiles(shape, false));
    write_ranges(a, nullptr, n, at_out);
    *ctas_out = a.ctas;
    return RLKV_OK;
}

int rlkv_debug_chunk_launch(const int* lens, const int* counts, int n, int n_full, int n_comp, int group, int sink, int window, int head_dim,
                            int fp8, int which, int* launches_out, int* shape_out, int* ctas_out, int* at_out)
{
    if ((head_dim != 64 && head_dim != 128) || (fp8 && head_dim != 128) || !launches_out || !shape_out || !ctas_out || !at_out) return RLKV_EINVAL;
    ChunkSeqs s;
    ChunkArgs a;
    const int rc = debug_args(lens, counts, n, n_full, n_comp, group, sink, window, s, a);
    if (rc) return rc;
    const int sms = kMaxChunkCtas / 2;
    const bool two = two_launches(s, a, sms, fp8 != 0);
    if (which < 0 || which > (two ? 1 : 0)) return RLKV_EINVAL;
    int entries[kMaxPagedBatch];
    *shape_out = cut_launch(s, a, two, which, sms, head_dim, fp8 != 0, chunk_record_bytes(head_dim), entries).shape;
    write_ranges(a, entries, n, at_out);
    *launches_out = two ? 2 : 1;
    *ctas_out = a.ctas;
    return RLKV_OK;
}

}  // extern "C"
