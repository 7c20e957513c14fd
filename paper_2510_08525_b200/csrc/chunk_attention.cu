// Attention of a chunk of new tokens of each of several sequences over the paged cache and over the chunk itself.
//
// The queries of a KV head's group are packed token by token into tiles of 128 rows, so that a few drafted tokens of eight
// heads fill a tensor-core tile as well as a prompt does, and every K and V row is read once for all of them.  Per key tile:
// S = Q.K^T (both operands in shared memory, fp32 in tensor memory); a warpgroup, one thread per query row, turns S into
// P = exp2(s - m), written as bf16 over S; O += P.V with P read from tensor memory.  Keys come from the cache's 64-row pages
// or rings as they lie (a box of a tensor map; in 8 bits a whole page as one copy, which four warps then decode) and, behind
// them, from the chunk's own rows.
//
// Two shapes of the same kernel:
//   SUBS 1  one tile of 128 rows, keys 64 at a time, two CTAs on an SM: while one waits for memory, sets up or writes results,
//           the other computes.  S alternates between two places, so the next product runs beside the softmax.
//   SUBS 2  two tiles of rows that share their key tiles of 128, one CTA on an SM: one's products run while the other's
//           softmax does, and the K/V rows pass through shared memory half as often.
// Each CTA walks one contiguous range of the units' key tiles (rlkv_chunk.cuh); units that a range's end cuts are added up
// by a second kernel.
//
//   warps 0-3 (0-7)  softmax of sub-tile 0 (1), and its output rows at the end
//   then             TMA: queries, K and V tiles through one ring, raw 8-bit pages through another
//                    the issue of every tcgen05.mma, in order
//                    clearing the V rows that hold no token (0 * NaN of a recycled page would be NaN)
//   last four        8-bit caches: E4M3 codes to bf16 operands (K as rows, V as it lies: transposed, its tokens contiguous)
//
// The running maximum of a row moves only when it would grow by more than 2^8 (its effect cancels in O / l; P <= 256, and O, l
// are fp32).  P is rounded to bf16 for the product, half a step 2^-8 of each weight; l sums the fp32 values.  Scales of an 8-bit
// cache never touch the codes: K's goes into the score's factor; O is kept in units of V's and multiplied by it once, before
// the chunk's first tile or at the end.
#include "rlkv_chunk.cuh"
#include "rlkv_prompt.cuh"
#include "tcgen05.cuh"

namespace rlkv {
namespace {

using namespace tc;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kRows = 128;           // query rows of a sub-tile
constexpr int kQBlock = kRows * 128; // bytes of a [128 rows][64 elements] block
constexpr int kPageBytes = 2 * kTile * 128;  // of an 8-bit page

template <int D, int SUBS, bool FP8>
struct Chunk {
    static constexpr int kKeys = SUBS == 2 ? 128 : 64;  // of a tile
    static constexpr int kPages = kKeys / kTile;
    static constexpr int kQBytes = kRows * D * 2, kTileBytes = kKeys * D * 2;
    static constexpr int kBlock = kKeys * 128;  // bytes of a [kKeys][64 elements] block
    static constexpr int kStages = FP8 ? (SUBS == 2 ? 4 : 3) : D == 128 ? 5 : 10;
    static constexpr int kRaw = FP8 ? 2 : 0;  // pages
    static constexpr int kState = SUBS * kQBytes + kStages * kTileBytes + kRaw * kPageBytes;
    static constexpr int kSmem = kState + 1024 * SUBS;
    static constexpr int kSoftmaxWarps = 4 * SUBS;
    static constexpr int kThreads = 32 * (kSoftmaxWarps + 4 + (FP8 ? 4 : 0));
    static constexpr int kPerSm = SUBS == 2 ? 1 : 2;
    static constexpr int kColumns = SUBS == 2 ? 512 : 256;  // of tensor memory: two S/P places, then O
    static constexpr int kFills = FP8 ? 4 : 1;  // arrivals that fill a stage: the decoding warps', or one copy's
};

// The part of a CTA's range that lies in one unit.
struct Segment {
    ChunkUnit u;
    int len, m, start, slot;  // of the sequence
    int head;                 // KV head
    bool full;
    int index;                // among the heads of its class
    int t0, t1, subs;         // key tiles, sub-tiles that hold rows
    int record;               // -1: the whole unit, whose rows are final
};
// A softmax warp's place in its CTA's range and the segment it is at, kept in shared memory: its threads' registers go to scores.
struct SoftmaxPlace {
    ChunkPos at;
    int first;
    Segment g;
};

struct ChunkShared {
    uint64_t q_full, q_empty[2], full[10], empty[10], dirty[10], clean[10], raw_full[2], raw_empty[2], s_full[2], p_full[2][2], pv_done[2], drain;
    uint32_t tmem;
    int abort;
    SoftmaxPlace place[1];  // (one of each softmax warp)
};

__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}

// `bytes` (a multiple of 16) from 16-byte aligned global to shared memory.
__device__ __forceinline__ void load_bytes(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}

// P = 2^(s factor - base) of a row's scores, as bf16 to tensor memory, and their sums; 64 keys at a time, so that the
// product starts on the first.
template <int N>
__device__ __forceinline__ void exponentials(float (&s)[N], float factor, float base, float2 (&sum)[2], uint32_t P, uint64_t* done, int lane)
{
    const float2 factor2 = make_float2(factor, factor), base2 = make_float2(-base, -base);
#pragma unroll
    for (int c = 0; c < N; c += 32) {
        uint32_t packed[16];
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            const float2 x = fma2(make_float2(s[c + i], s[c + i + 1]), factor2, base2);
            s[c + i] = ex2(x.x);
            s[c + i + 1] = ex2(x.y);
            packed[i / 2] = bf16x2(s[c + i], s[c + i + 1]);
        }
        tmem_st16(P + c / 2, packed);
        if (c % 64 == 32) {
            wait_st();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(done + c / 64));
        }
    }
#pragma unroll
    for (int c = 0; c < N; c += 2) sum[c / 2 & 1] = add2(sum[c / 2 & 1], make_float2(s[c], s[c + 1]));
}

// Two E4M3 codes in the high bytes of a word's halves, as bf16: the exponent and mantissa bits moved to their places read
// as a bf16 number 2^-120 times the value (subnormals too); the product is exact.
__device__ __forceinline__ uint32_t decode2(uint32_t x)
{
    const uint32_t y = (x & 0x80008000u) | ((x >> 4) & 0x07f007f0u), two120 = 0x7b807b80u;
    const __nv_bfloat162 z = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&y), *reinterpret_cast<const __nv_bfloat162*>(&two120));
    return *reinterpret_cast<const uint32_t*>(&z);
}
__device__ __forceinline__ void decode16(const uint4& codes, uint4& lo, uint4& hi)
{
    lo.x = decode2(__byte_perm(codes.x, 0, 0x1404));
    lo.y = decode2(__byte_perm(codes.x, 0, 0x3424));
    lo.z = decode2(__byte_perm(codes.y, 0, 0x1404));
    lo.w = decode2(__byte_perm(codes.y, 0, 0x3424));
    hi.x = decode2(__byte_perm(codes.z, 0, 0x1404));
    hi.y = decode2(__byte_perm(codes.z, 0, 0x3424));
    hi.z = decode2(__byte_perm(codes.w, 0, 0x1404));
    hi.w = decode2(__byte_perm(codes.w, 0, 0x3424));
}

// Walks the segments of CTA `cta` in order.
template <int KEYS, int SUBS>
struct Walk {
    const ChunkArgs& a;
    ChunkPos at, end;
    int tokens, cta;  // tokens of a sub-tile
    bool first = true;
    __device__ __forceinline__ Walk(const ChunkArgs& args) : a(args), at(args.at[blockIdx.x]), end(args.at[blockIdx.x + 1]), tokens(kRows / args.group), cta(blockIdx.x) {}
    __device__ __forceinline__ bool next(Segment& s)
    {
        if (same_unit(at, end) && at.tile >= end.tile) return false;
        s.start = a.seqs.start[at.seq];
        s.m = a.seqs.start[at.seq + 1] - s.start;
        s.len = a.seqs.len[at.seq];
        s.slot = a.seqs.slot[at.seq];
        s.full = at.head < a.n_full;
        s.index = s.full ? at.head : at.head - a.n_full;
        s.head = a.head_of_slot[at.head];
        s.u = chunk_unit(s.len, s.m, at.row_tile, SUBS * tokens, KEYS, s.full, a.sink, a.window);
        s.subs = SUBS == 2 && s.m - s.u.tok0 > tokens ? 2 : 1;
        s.t0 = at.tile;
        const bool last = same_unit(at, end);
        s.t1 = last ? end.tile : s.u.tiles;
        s.record = s.t0 == 0 && s.t1 == s.u.tiles ? -1 : 2 * cta + (first ? 0 : 1);
        first = false;
        if (last) {
            at.tile = end.tile;
        } else {
            at.tile = 0;
            if (++at.head == a.n_full + a.n_comp) {
                at.head = 0;
                if (++at.row_tile * SUBS * tokens >= s.m) {
                    at.row_tile = 0;
                    do ++at.seq;
                    while (at.seq < a.seqs.n && a.seqs.start[at.seq + 1] == a.seqs.start[at.seq]);
                }
            }
        }
        return true;
    }
    // First chunk token of key tile t >= cached.
    static __device__ __forceinline__ int chunk_tile(const volatile ChunkUnit& u, int t)
    {
        const int x = t - u.cached;
        return (x < u.a_end ? x : u.b0 + x - u.a_end) * KEYS;
    }
    // Whether the K (v 0) or V rows of key tile t are to be cleared where they hold no token: V always (0 * NaN), K where what it
    // holds has a say in how a warp computes the cap; decoded rows are finite, and cleared as they are written.
    template <bool FP8, bool CAP>
    static __device__ __forceinline__ bool unclean(const Segment& s, int t, int v)
    {
        return (v || CAP) && (!FP8 || t >= s.u.cached) && valid_rows(s, t) < KEYS;
    }
    // Rows of key tile t that hold a token (KEYS or more: all of them).
    static __device__ __forceinline__ int valid_rows(const Segment& s, int t)
    {
        return t < s.u.cached ? s.u.rows - t * KEYS : s.m - chunk_tile(s.u, t);
    }
};

template <int D, int SUBS, bool FP8, bool CAP, bool BIAS>
__global__ void __launch_bounds__(Chunk<D, SUBS, FP8>::kThreads, Chunk<D, SUBS, FP8>::kPerSm)
chunk_attention_kernel(const __grid_constant__ ChunkArgs a, const __grid_constant__ ChunkMaps maps)
{
    using C = Chunk<D, SUBS, FP8>;
    using W = Walk<C::kKeys, SUBS>;
    constexpr int KEYS = C::kKeys, kHalves = KEYS / 64;
    extern __shared__ __align__(1024) uint8_t smem[];
    static_assert(sizeof(ChunkShared) + (C::kSoftmaxWarps - 1) * sizeof(SoftmaxPlace) <= C::kSmem - C::kState && C::kSmem <= kMaxDynamicSmem, "shared memory");
    static_assert(C::kPerSm * (C::kSmem + 1024) <= 228 * 1024, "shared memory of an SM");
    ChunkShared& sh = *reinterpret_cast<ChunkShared*>(smem + C::kState);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    volatile int* abort_flag = &sh.abort;
    constexpr int kLoad = C::kSoftmaxWarps, kMma = kLoad + 1, kClean = kLoad + 2, kDecode = kLoad + 4;

    grid_dep_launch();
    if ((smem_u32(smem) & 1023u) != 0) {
        if (tid == 0) atomicCAS(a.status, 0, kChunkSmemMisaligned);
        return;
    }
    if (warp == kLoad) {
        if (lane == 0) {
            prefetch_map(&maps.q);
            prefetch_map(&maps.k);
            prefetch_map(&maps.v);
            if (!FP8) prefetch_map(&maps.pool);
            sh.abort = 0;
            mbar_init(smem_u32(&sh.q_full), 1);
            for (int i = 0; i < C::kStages; ++i) {
                mbar_init(smem_u32(&sh.full[i]), C::kFills);
                mbar_init(smem_u32(&sh.empty[i]), 1);
                mbar_init(smem_u32(&sh.dirty[i]), 1);
                mbar_init(smem_u32(&sh.clean[i]), 1);
            }
            for (int w = 0; w < 2; ++w) {
                mbar_init(smem_u32(&sh.q_empty[w]), 4);
                mbar_init(smem_u32(&sh.raw_full[w]), 1);
                mbar_init(smem_u32(&sh.raw_empty[w]), 4);
                mbar_init(smem_u32(&sh.s_full[w]), 1);
                mbar_init(smem_u32(&sh.p_full[w][0]), 4);
                mbar_init(smem_u32(&sh.p_full[w][1]), 4);
                mbar_init(smem_u32(&sh.pv_done[w]), 1);
            }
            mbar_init(smem_u32(&sh.drain), 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
    } else if (warp == kMma) {
        tmem_alloc(smem_u32(&sh.tmem), C::kColumns);
        fence_before();
    }
    __syncthreads();
    fence_after();
    const uint32_t tmem = sh.tmem;
    const uint32_t q_smem = smem_u32(smem), ring = q_smem + SUBS * C::kQBytes, raw = ring + C::kStages * C::kTileBytes;
    const uint32_t o_column = SUBS == 2 ? 256 : 128;
    // Registers: 384 x 168 = 64512 = 256 x 224 + 128 x 56; 512 x 128 = 65536 = 256 x 200 + 256 x 56;
    // 256 x 128 = 32768 = 128 x 184 + 128 x 72; 384 x 80 = 30720 = 128 x 128 + 256 x 56
    if (warp < C::kSoftmaxWarps) more_registers<SUBS == 2 ? (FP8 ? 200 : 224) : FP8 ? 128 : 184>();
    else fewer_registers<SUBS == 1 && !FP8 ? 72 : 56>();
    if (warp < C::kSoftmaxWarps) {
        // ------------------------------------------------------------------ softmax
        const int w = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t O = tmem + lanes + o_column + w * D;
        const int in_tile = row / a.group, member = row - in_tile * a.group;
        const int tokens = kRows / a.group;
        int total = 0;  // tiles of this sub-tile so far
        bool ok = true;
        // SUBS 1: the score product of tile n goes out before the value product of tile n - 1, so that two of the latter may be
        // outstanding: they take turns at two barriers, or a wait could take the end of the one before for its own
        auto product_done = [&](int n) {
            return SUBS == 2 ? wait(smem_u32(&sh.pv_done[w]), n & 1, abort_flag, a.status, kChunkWaitProduct)
                             : wait(smem_u32(&sh.pv_done[n & 1]), n >> 1 & 1, abort_flag, a.status, kChunkWaitProduct);
        };
        SoftmaxPlace* place_of = sh.place + warp;
        const volatile Segment& g = place_of->g;
        if (lane == 0) {
            place_of->at = a.at[blockIdx.x];
            place_of->first = 1;
        }
        while (ok) {
            int more = 0;
            __syncwarp();  // no lane reads the segment before any more
            if (lane == 0) {
                W walk(a);
                walk.at = place_of->at;
                walk.first = place_of->first;
                Segment next;
                more = walk.next(next);
                place_of->at = walk.at;
                place_of->first = walk.first;
                if (more) place_of->g = next;
            }
            if (!__shfl_sync(0xffffffffu, more, 0)) break;
            __syncwarp();
            if (w >= g.subs) continue;
            const int from = g.u.tok0 + w * tokens;     // the sub-tile's first token
            const int i = from + in_tile, head = g.head * a.group + member;
            const bool mine = in_tile < tokens && i < g.m;
            const int upto = min(from + tokens, g.m) - 1;   // its last
            const float slope2 = BIAS && mine ? a.slopes[head] * kLog2e : 0.f;
            // the ring: its sink rows hold tokens 0 .. sink-1, the rows up to w1 the newest, the rows from w1 on those one
            // window older
            const int w1 = g.len > a.sink ? a.sink + (g.len - 1 - a.sink) % a.window + 1 : g.len;
            const float k_scale = FP8 ? a.k_scale[g.head] : 1.f, v_scale = FP8 ? a.v_scale[g.head] : 1.f;
            float scale = a.scale * (FP8 && g.t0 < g.u.cached ? k_scale : 1.f);
            Cap cap(CAP ? a.softcap : 1.f, scale);
            float m = -INFINITY, l = 0.f;
            for (int t = g.t0; t < g.t1; ++t) {
                const int place = SUBS == 2 ? w : total & 1;
                const uint32_t S = tmem + lanes + place * KEYS;
                ok = wait(smem_u32(&sh.s_full[place]), (SUBS == 2 ? total : total >> 1) & 1, abort_flag, a.status, kChunkWaitProduct);
                if (!ok) break;
                fence_after();
                float s[KEYS];
#pragma unroll
                for (int c = 0; c < KEYS; c += 32) tmem_ld32(S + c, s + c);
                wait_ld();
#pragma unroll
                for (int c = 0; c < KEYS; ++c) asm volatile("" : "+f"(s[c]));  // nothing of the above is used before the wait
                const bool cached = t < g.u.cached;
                float corr = 1.f;  // of O
                if (FP8 && t == g.u.cached && t > g.t0) {  // from the cache's codes to the chunk's rows
                    corr = v_scale;
                    scale = a.scale;
                    if (CAP) cap = Cap(a.softcap, scale);
                }
                const int start = cached ? t * KEYS : W::chunk_tile(g.u, t);
                if (CAP) cap.apply(s, mine);
                if (BIAS) {
                    // from the distance itself, a whole number and exact: a sum of terms would round at their size and lose the
                    // scores next to the query where slopes are steep
                    const float sl2 = scale * kLog2e;
                    const float far = (float)(cached ? g.len + i - start : i - start);
                    if (!cached || g.full) {
                        float2 d[4];
#pragma unroll
                        for (int c = 0; c < 8; c += 2) d[c / 2] = make_float2((float)c - far, (float)(c + 1) - far);
#pragma unroll
                        for (int c = 0; c < KEYS; c += 2) {
                            const float2 x = CAP ? make_float2(s[c], s[c + 1]) : mul2(make_float2(s[c], s[c + 1]), make_float2(sl2, sl2));
                            const float2 y = fma2(make_float2(slope2, slope2), d[c / 2 & 3], x);
                            s[c] = y.x;
                            s[c + 1] = y.y;
                            d[c / 2 & 3] = add2(d[c / 2 & 3], make_float2(8.f, 8.f));
                        }
                    } else {
                        const float near = (float)(i + w1 - start), older = (float)(i + w1 + a.window - start);
                        const int b1 = a.sink - start, b2 = w1 - start;
#pragma unroll
                        for (int c = 0; c < KEYS; ++c) {
                            const float from_row = c < b1 ? far : c < b2 ? near : older;
                            s[c] = fmaf(-slope2, from_row - (float)c, CAP ? s[c] : s[c] * sl2);
                        }
                    }
                }
                // what this row sees of the tile: up to three ranges of columns
                bool plain;
                int lo1 = 0, hi1, lo2 = 0, hi2 = 0, hi3 = 0;  // [lo1, hi1), [lo2, hi2), [0, hi3)
                if (cached) {
                    if (g.full) {
                        hi1 = g.len - start;
                        plain = hi1 >= KEYS;
                    } else {
                        hi3 = min(a.sink, g.u.rows) - start;
                        lo1 = max(a.sink, w1 + i + 1 - a.window) - start;
                        hi1 = w1 - start;
                        lo2 = w1 + i + 1 - start;
                        hi2 = g.u.rows - start;
                        plain = false;
                    }
                } else {
                    hi1 = i + 1 - start;
                    plain = start + KEYS <= from + 1;
                    if (!g.full) {
                        lo1 = i - a.window + 1 - start;
                        hi3 = min(a.sink - g.len, i + 1) - start;
                        plain = plain && (start > upto - a.window || start + KEYS <= a.sink - g.len);
                    }
                }
                if (!plain) {
#pragma unroll
                    for (int x = 0; x < KEYS; x += 32) {
                        const uint32_t see = mine ? range_bits(lo1 - x, hi1 - x) | range_bits(lo2 - x, hi2 - x) | range_bits(0, hi3 - x) : 0u;
#pragma unroll
                        for (int c = 0; c < 32; ++c) s[x + c] = see >> c & 1 ? s[x + c] : -INFINITY;
                    }
                }
                const float factor = CAP || BIAS ? 1.f : scale * kLog2e;
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < KEYS; ++c) mx[c & 3] = fmaxf(mx[c & 3], s[c]);
                const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * factor;
                if (top > m + 8.f) {  // (m may still be -infinity: then there is nothing to correct)
                    const float x = m == -INFINITY ? 1.f : ex2(m - top);
                    m = top;
                    l *= x;
                    corr *= x;
                }
                if (t > g.t0 && __any_sync(0xffffffffu, corr != 1.f)) {
                    ok = product_done(total - 1);
                    if (!ok) break;
                    fence_after();
#pragma unroll
                    for (int c = 0; c < D; c += 32) {
                        float o[32];
                        tmem_read32(O + c, o);
#pragma unroll
                        for (int x = 0; x < 32; ++x) o[x] *= corr;
                        tmem_st32(O + c, o);
                    }
                }
                const float base = m == -INFINITY ? 0.f : m;
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                exponentials(s, factor, base, sum, S, sh.p_full[place], lane);
                l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                ++total;
            }
            if (!ok) break;
            ok = product_done(total - 1);
            if (!ok) break;
            fence_after();
            const float unit = FP8 && g.t1 <= g.u.cached ? v_scale : 1.f;
            const long long at_head = ((long long)(g.start + i) * a.q_heads + head);
            if (g.record < 0) {
                const float inv = l > 0.f ? unit / l : 0.f;
                if (mine && a.lse) a.lse[at_head] = l > 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
                // through shared memory (the sub-tile's queries are not needed any more), so that whole rows go out
                uint8_t* stage = smem + w * C::kQBytes + (warp & 3) * 32 * D * 2;
                constexpr int kChunks = D / 8, kPerStore = 32 / kChunks;  // 16-byte pieces of a row, rows per store instruction
#pragma unroll
                for (int c = 0; c < D; c += 32) {
                    float o[32];
                    tmem_read32(O + c, o);
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        *reinterpret_cast<uint4*>(stage + lane * D * 2 + (((c / 8 + x) ^ (lane & 7)) << 4)) =
                            make_uint4(bf16x2(o[8 * x] * inv, o[8 * x + 1] * inv), bf16x2(o[8 * x + 2] * inv, o[8 * x + 3] * inv),
                                       bf16x2(o[8 * x + 4] * inv, o[8 * x + 5] * inv), bf16x2(o[8 * x + 6] * inv, o[8 * x + 7] * inv));
                }
                __syncwarp();
                const long long to = mine ? at_head * D : -1;
#pragma unroll 4
                for (int x = 0; x < 32; x += kPerStore) {
                    const int r = x + lane / kChunks;
                    const long long dst = __shfl_sync(0xffffffffu, to, r);
                    if (dst >= 0)
                        *reinterpret_cast<uint4*>(a.out + dst + lane % kChunks * 8) =
                            *reinterpret_cast<const uint4*>(stage + r * D * 2 + (((lane % kChunks) ^ (r & 7)) << 4));
                }
            } else {
                float* rec = a.records + (long long)g.record * chunk_record_floats(D, SUBS) + (long long)w * kRows * (D + 2);
#pragma unroll
                for (int c = 0; c < D; c += 32) {
                    float o[32];
                    tmem_read32(O + c, o);
                    if (mine)
#pragma unroll
                        for (int x = 0; x < 8; ++x)
                            reinterpret_cast<float4*>(rec)[(c / 4 + x) * kRows + row] =
                                make_float4(o[4 * x] * unit, o[4 * x + 1] * unit, o[4 * x + 2] * unit, o[4 * x + 3] * unit);
                }
                rec[D * kRows + row] = m;
                rec[(D + 1) * kRows + row] = l;
            }
            fence_before();
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.q_empty[w]));
        }
    } else if (warp == kLoad) {
        // ------------------------------------------------------------------ tile loads
        W walk(a);
        Segment g;
        int issued = 0, pages = 0, segs[2] = {0, 0};  // stages and raw pages so far; segments of each sub-tile
        uint32_t copied = 0;  // stages whose last fill was a copy of this warp's
        bool ok = true, q_out = false;
        while (ok && walk.next(g)) {
            const int row0 = g.start + g.u.tok0;
            bool q_waits = true;
            auto queries = [&]() {  // once the sub-tiles' rows of the segment before have been written
                for (int w = 0; w < g.subs; ++w) {
                    ok = ok && wait_warp(smem_u32(&sh.q_empty[w]), (segs[w] & 1) ^ 1, abort_flag, a.status, kChunkWaitQueries);
                    ++segs[w];
                }
                if (!ok) return;
                if (lane == 0) {
                    mbar_expect_tx(smem_u32(&sh.q_full), g.subs * (D / 64) * walk.tokens * a.group * 128);
                    for (int w = 0; w < g.subs; ++w)
                        for (int b = 0; b < D / 64; ++b)
                            load_box(q_smem + w * C::kQBytes + b * kQBlock, &maps.q, b * 64, g.head * a.group, row0 + w * walk.tokens,
                                     smem_u32(&sh.q_full));
                }
                q_waits = false;
                q_out = true;
            };
            auto free_queries = [&]() {
                bool yes = true;
                for (int w = 0; w < g.subs; ++w) yes = yes && mbar_test(smem_u32(&sh.q_empty[w]), (segs[w] & 1) ^ 1);
                return __all_sync(0xffffffffu, yes);
            };
            // waits for a stage (or raw page) to be free; K and V tiles of a segment come in ahead of its queries while those
            // of the segment before are still in use, but never wait for a stage that only their product would free
            auto free_stage = [&](uint64_t* bar, uint32_t parity) {
                if (q_waits && (free_queries() || !__all_sync(0xffffffffu, mbar_test(smem_u32(bar), parity)))) queries();
                ok = ok && wait_warp(smem_u32(bar), parity, abort_flag, a.status, kChunkWaitStage);
                return ok;
            };
            const int* table = a.page_table + (long long)g.slot * a.table_stride;
            const int n_pages = (g.u.rows + kTile - 1) / kTile;
            int batch = g.t0 * C::kPages, entry = 0;  // page-table entries batch .. batch+31, one per lane
            auto fetch = [&](int first) {
                batch = first;
                entry = g.full && first + lane < n_pages ? min(max(table[first + lane], 0), a.n_pages - 1) : 0;
            };
            if (g.t0 < g.u.cached) fetch(batch);
            for (int t = g.t0; ok && t < g.t1; ++t) {
                if (t < g.u.cached) {
                    const int page = t * C::kPages;
                    if (page >= batch + 32) fetch(page);
                    const int have = min(C::kPages, n_pages - page);  // pages of this tile
                    if constexpr (FP8) {
                        for (int p = 0; p < have; ++p) {
                            const int phys = __shfl_sync(0xffffffffu, entry, (page + p - batch) & 31);
                            const long long index = g.full ? a.page0_8 + (long long)g.index * a.n_pages + phys
                                                           : a.ring0_8 + ((long long)g.slot * a.n_comp + g.index) * a.ring_tiles + page + p;
                            const int rs = pages & 1;
                            if (!free_stage(&sh.raw_empty[rs], (pages >> 1 & 1) ^ 1)) break;
                            if (lane == 0) {
                                mbar_expect_tx(smem_u32(&sh.raw_full[rs]), kPageBytes);
                                load_bytes(raw + rs * kPageBytes, a.pool8 + index * kPageBytes, kPageBytes, smem_u32(&sh.raw_full[rs]));
                            }
                            ++pages;
                        }
                        copied &= ~(1u << issued % C::kStages | 1u << (issued + 1) % C::kStages);
                        issued += 2;
                    } else {
                    int phys[C::kPages];
#pragma unroll
                    for (int p = 0; p < C::kPages; ++p) phys[p] = __shfl_sync(0xffffffffu, entry, (page + p - batch) & 31);
                    for (int kv = 0; kv < 2; ++kv) {
                        const int slot = issued % C::kStages;
                        if (!free_stage(&sh.empty[slot], (issued / C::kStages & 1) ^ 1)) break;
                        if (lane == 0) {
                            mbar_expect_tx(smem_u32(&sh.full[slot]), have * kTile * D * 2);
#pragma unroll
                            for (int p = 0; p < C::kPages; ++p) {
                                if (p >= have) break;
                                const long long r = g.full ? a.full_row0 + (((long long)g.index * a.n_pages + phys[p]) * 2 + kv) * kTile
                                                           : a.comp_row0 + (((long long)g.slot * a.n_comp + g.index) * 2 + kv) * a.rows_comp +
                                                                 (page + p) * kTile;
                                for (int b = 0; b < D / 64; ++b)
                                    load_box(ring + slot * C::kTileBytes + b * C::kBlock + p * kTile * 128, &maps.pool, b * 64, 0, (int)r,
                                             smem_u32(&sh.full[slot]));
                            }
                            if (W::template unclean<FP8, CAP>(g, t, kv)) mbar_arrive(smem_u32(&sh.dirty[slot]));
                        }
                        copied |= 1u << slot;
                        ++issued;
                    }
                    }
                } else {
                    // (a stage's earlier contents may be the decoding warps': those have all been written once the last raw
                    // page has been read, so that the wait below cannot take an earlier use of the stage for its last)
                    if (FP8 && pages > 0) {
                        if (q_waits) queries();
                        ok = ok && wait_warp(smem_u32(&sh.raw_empty[(pages - 1) & 1]), (pages - 1) >> 1 & 1, abort_flag, a.status, kChunkWaitRaw);
                    }
                    const int token = g.start + W::chunk_tile(g.u, t);
                    for (int kv = 0; ok && kv < 2; ++kv) {
                        const int slot = issued % C::kStages;
                        if (!free_stage(&sh.empty[slot], (issued / C::kStages & 1) ^ 1)) break;
                        if (lane == 0) {
                            mbar_expect_tx(smem_u32(&sh.full[slot]), C::kTileBytes);
                            for (int x = 1; x < C::kFills; ++x) mbar_arrive(smem_u32(&sh.full[slot]));
                            for (int b = 0; b < D / 64; ++b)
                                load_box(ring + slot * C::kTileBytes + b * C::kBlock, kv ? &maps.v : &maps.k, b * 64, g.head, token,
                                         smem_u32(&sh.full[slot]));
                            if (W::template unclean<FP8, CAP>(g, t, kv)) mbar_arrive(smem_u32(&sh.dirty[slot]));
                        }
                        copied |= 1u << slot;
                        ++issued;
                    }
                }
            }
            if (ok && q_waits) queries();
        }
        if (!ok || *abort_flag) {  // nothing of this CTA's copies may be in flight when it ends
            if (q_out) wait_warp(smem_u32(&sh.q_full), (max(segs[0], 1) - 1) & 1, nullptr, a.status, kChunkWaitDrain);
            for (int i = max(0, issued - C::kStages); i < issued; ++i)
                if (copied >> i % C::kStages & 1) wait_warp(smem_u32(&sh.full[i % C::kStages]), i / C::kStages & 1, nullptr, a.status, kChunkWaitDrain);
            for (int i = max(0, pages - 2); i < pages; ++i)
                wait_warp(smem_u32(&sh.raw_full[i & 1]), i >> 1 & 1, nullptr, a.status, kChunkWaitDrain);
        }
    } else if (warp == kMma) {
        // ------------------------------------------------------------------ matrix products
        W walk(a);
        Segment g;
        constexpr uint32_t kQK = instr_desc(kRows, KEYS, false), kPV = instr_desc(kRows, D, true), kPVt = instr_desc(kRows, D, false);
        int used[2] = {0, 0};    // P tiles multiplied so far (SUBS 1: used[0])
        int base = 0, seg = 0;   // stages and segments so far
        uint32_t cleaned = 0;    // phase of each stage's `clean`
        bool ok = true;
        while (ok && walk.next(g)) {
            const int n = g.t1 - g.t0;
            auto stage = [&](int i) { return ring + (base + i) % C::kStages * C::kTileBytes; };
            // K (even) and V tiles in turn
            auto loaded = [&](int i) {
                const int slot = (base + i) % C::kStages, t = g.t0 + (i >> 1);
                if (!wait_warp(smem_u32(&sh.full[slot]), (base + i) / C::kStages & 1, abort_flag, a.status, kChunkWaitLoad)) return false;
                if (W::template unclean<FP8, CAP>(g, t, i & 1)) {
                    if (!wait_warp(smem_u32(&sh.clean[slot]), cleaned >> slot & 1, abort_flag, a.status, kChunkWaitLoad)) return false;
                    cleaned ^= 1u << slot;
                }
                return true;
            };
            auto signal = [&](uint64_t* bar) {
                if (elect_one()) commit(smem_u32(bar));
            };
            auto scores = [&](int w, int place, int j) {
                const uint64_t q = smem_desc(q_smem + w * C::kQBytes), k = smem_desc(stage(2 * j));
                fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int x = 0; x < D / 16; ++x)
                        mma_ss(tmem + place * KEYS, q + ((x / 4 * kQBlock + x % 4 * 32) >> 4), k + ((x / 4 * C::kBlock + x % 4 * 32) >> 4), kQK, x > 0);
                    commit(smem_u32(&sh.s_full[place]));
                }
            };
            // the products of one half (64 keys) of tile j's P
            auto values = [&](int w, int place, int j, int half) {
                fence_after();
                const uint32_t d = tmem + o_column + w * D, p = tmem + place * KEYS + half * 32;
                if (FP8 && g.t0 + j < g.u.cached) {  // V^T: rows of 64 tokens
                    const uint64_t v = smem_desc(stage(2 * j + 1) + half * (D * 128));
                    if (elect_one()) {
#pragma unroll
                        for (int x = 0; x < 4; ++x) mma_ts(d, p + x * 8, v + (x * 32 >> 4), kPVt, j > 0 || half > 0 || x > 0);
                    }
                } else {
                    const uint64_t v = smem_desc(stage(2 * j + 1) + half * (64 * 128), C::kBlock);
                    if (elect_one()) {
#pragma unroll
                        for (int x = 0; x < 4; ++x) mma_ts(d, p + x * 8, v + (x * 2048 >> 4), kPV, j > 0 || half > 0 || x > 0);
                    }
                }
            };
            ok = wait_warp(smem_u32(&sh.q_full), seg & 1, abort_flag, a.status, kChunkWaitQueries) && loaded(0);
            if (!ok) break;
            if (SUBS == 1) {
                scores(0, used[0] & 1, 0);
                signal(&sh.empty[base % C::kStages]);
                for (int j = 0; ok && j < n; ++j) {
                    const int place = used[0] & 1;
                    if (j + 1 < n) {
                        ok = loaded(2 * j + 2);
                        if (!ok) break;
                        scores(0, place ^ 1, j + 1);
                        signal(&sh.empty[(base + 2 * j + 2) % C::kStages]);
                    }
                    ok = wait_warp(smem_u32(&sh.p_full[place][0]), used[0] >> 1 & 1, abort_flag, a.status, kChunkWaitSoftmax) && loaded(2 * j + 1);
                    if (!ok) break;
                    values(0, place, j, 0);
                    signal(&sh.pv_done[place]);
                    signal(&sh.empty[(base + 2 * j + 1) % C::kStages]);
                    ++used[0];
                }
            } else {
                for (int w = 0; w < g.subs; ++w) scores(w, w, 0);
                signal(&sh.empty[base % C::kStages]);
                for (int j = 0; ok && j < n; ++j) {
                    ok = loaded(2 * j + 1);
                    if (ok && j + 1 < n) ok = loaded(2 * j + 2);
#pragma unroll
                    for (int w = 0; w < SUBS; ++w) {
                        if (!ok) break;
                        if (w < g.subs) {
                            for (int half = 0; half < kHalves; ++half) {
                                ok = wait_warp(smem_u32(&sh.p_full[w][half]), used[w] & 1, abort_flag, a.status, kChunkWaitSoftmax);
                                if (!ok) break;
                                values(w, w, j, half);
                            }
                            if (!ok) break;
                            signal(&sh.pv_done[w]);
                            ++used[w];
                        }
                        if (w == SUBS - 1) signal(&sh.empty[(base + 2 * j + 1) % C::kStages]);
                        if (j + 1 < n && w < g.subs) scores(w, w, j + 1);
                    }
                    if (ok && j + 1 < n) signal(&sh.empty[(base + 2 * j + 2) % C::kStages]);
                }
            }
            base += 2 * n;
            ++seg;
        }
        // every product is done before tensor memory is given back
        if (elect_one()) commit(smem_u32(&sh.drain));
        wait_warp(smem_u32(&sh.drain), 0, nullptr, a.status, kChunkWaitDrain);
    } else if (warp == kClean) {
        // ------------------------------------------------------------------ rows that hold no token
        W walk(a);
        Segment g;
        // (told of each such copy by the warp that issued it: a stage's barrier alone would not say which of its uses it is at)
        int base = 0;
        uint32_t told = 0;  // phase of each stage's `dirty`
        bool ok = true;
        while (ok && walk.next(g)) {
            for (int t = g.t0; ok && t < g.t1; ++t)
                for (int v = 0; ok && v < 2; ++v) {
                    if (!W::template unclean<FP8, CAP>(g, t, v)) continue;
                    const int i = base + 2 * (t - g.t0) + v, slot = i % C::kStages;
                    ok = wait_warp(smem_u32(&sh.dirty[slot]), told >> slot & 1, abort_flag, a.status, kChunkWaitLoad) &&
                         wait_warp(smem_u32(&sh.full[slot]), i / C::kStages & 1, abort_flag, a.status, kChunkWaitLoad);
                    if (!ok) break;
                    told ^= 1u << slot;
                    uint8_t* x = smem + SUBS * C::kQBytes + slot * C::kTileBytes;
                    for (int y = W::valid_rows(g, t) * 8 + lane; y < KEYS * 8; y += 32)
                        for (int b = 0; b < D / 64; ++b) *reinterpret_cast<uint4*>(x + b * C::kBlock + y * 16) = make_uint4(0, 0, 0, 0);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&sh.clean[slot]));
                }
            base += 2 * (g.t1 - g.t0);
        }
    } else if (FP8 && warp >= kDecode) {
        // ------------------------------------------------------------------ codes to bf16 operands
        W walk(a);
        Segment g;
        const int ct = (warp - kDecode) * 32 + lane;
        int base = 0, pages = 0;
        bool ok = true;
        while (ok && walk.next(g)) {
            const int n_pages = (g.u.rows + kTile - 1) / kTile;
            for (int t = g.t0; ok && t < min(g.t1, g.u.cached); ++t) {
                const int i = base + 2 * (t - g.t0);
                const int ks = i % C::kStages, vs = (i + 1) % C::kStages;
                // the raw page first: by then the copies before it have been issued, so that the stages' last uses are known
                ok = wait_warp(smem_u32(&sh.raw_full[pages & 1]), pages >> 1 & 1, abort_flag, a.status, kChunkWaitRaw) &&
                     wait_warp(smem_u32(&sh.empty[ks]), (i / C::kStages & 1) ^ 1, abort_flag, a.status, kChunkWaitStage) &&
                     wait_warp(smem_u32(&sh.empty[vs]), ((i + 1) / C::kStages & 1) ^ 1, abort_flag, a.status, kChunkWaitStage);
                if (!ok) break;
                uint8_t *kt = smem + SUBS * C::kQBytes + ks * C::kTileBytes, *vt = smem + SUBS * C::kQBytes + vs * C::kTileBytes;
#pragma unroll 1
                for (int p = 0; p < C::kPages; ++p) {
                    const bool have = t * C::kPages + p < n_pages;
                    const int rs = pages & 1;
                    if (have) {
                        ok = wait_warp(smem_u32(&sh.raw_full[rs]), pages >> 1 & 1, abort_flag, a.status, kChunkWaitRaw);
                        if (!ok) break;
                    }
                    const uint4* src = reinterpret_cast<const uint4*>(smem + SUBS * C::kQBytes + C::kStages * C::kTileBytes + rs * kPageBytes);
                    const int valid = g.u.rows - (t * KEYS + p * kTile);  // rows of the page that hold a token
#pragma unroll
                    for (int x = 0; x < 4; ++x) {  // K: 16 elements of a row
                        const int piece = x * 128 + ct, r = piece >> 3, c = piece & 7;
                        uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
                        if (r < valid) decode16(src[piece], lo, hi);
                        const int y = p * kTile + r, ch = (c & 3) * 2, odd = c >> 2;  // (the two blocks' first stores go to different banks)
                        uint8_t* to = kt + (c >> 2) * C::kBlock + y * 128;
                        *reinterpret_cast<uint4*>(to + (((ch + odd) ^ (y & 7)) << 4)) = odd ? hi : lo;
                        *reinterpret_cast<uint4*>(to + (((ch + 1 - odd) ^ (y & 7)) << 4)) = odd ? lo : hi;
                    }
#pragma unroll
                    for (int x = 0; x < 4; ++x) {  // V^T: 16 tokens of an element
                        const int piece = x * 128 + ct, d = piece >> 2, ch = (piece & 3) * 2;
                        uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
                        if (have) decode16(src[512 + piece], lo, hi);
                        uint8_t* to = vt + p * (128 * 128) + d * 128;
                        *reinterpret_cast<uint4*>(to + ((ch ^ (d & 7)) << 4)) = lo;
                        *reinterpret_cast<uint4*>(to + (((ch + 1) ^ (d & 7)) << 4)) = hi;
                    }
                    if (have) {
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&sh.raw_empty[rs]));
                        ++pages;
                    }
                }
                if (!ok) break;
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(smem_u32(&sh.full[ks]));
                    mbar_arrive(smem_u32(&sh.full[vs]));
                }
            }
            base += 2 * (g.t1 - g.t0);
        }
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == kMma) {
        __syncwarp();
        tmem_free(tmem, C::kColumns);
    }
}

// Adds up the pieces of the units that a boundary cuts.  Block (c - 1, rows, columns): the unit that CTA c's range begins
// inside of, if it is the first to; 32 rows and 32 columns of it.  A lane holds a row's columns of every eighth piece, the
// eight warps' sums meet in shared memory.  The pieces' order is that of the keys, whatever CTA ran first.
template <int D, int SUBS>
__global__ void __launch_bounds__(256) chunk_combine_kernel(const __grid_constant__ ChunkArgs a)
{
    __shared__ float part[8][32][33], top[8][32], sum[8][32];
    const int c = blockIdx.x + 1;
    const ChunkPos b = a.at[c], before = a.at[c - 1];
    if (b.tile == 0 || b.seq >= a.seqs.n || (same_unit(before, b) && before.tile > 0)) return;
    const int tokens = kRows / a.group, w = blockIdx.y / 4, row0 = blockIdx.y % 4 * 32;
    const int start = a.seqs.start[b.seq], m = a.seqs.start[b.seq + 1] - start;
    const int from = b.row_tile * SUBS * tokens + w * tokens;
    if (row0 / a.group >= tokens || from + row0 / a.group >= m) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int last = c;  // the pieces are those of CTAs c - 1 .. last
    while (last + 1 < a.ctas && same_unit(a.at[last + 1], b)) ++last;
    grid_dep_wait();
    float o[32], mx = -INFINITY, l = 0.f;
#pragma unroll
    for (int x = 0; x < 32; ++x) o[x] = 0.f;
    for (int k = c - 1 + warp; k <= last; k += 8) {
        const int slot = k > c - 1 || (same_unit(before, b)) ? 2 * k : 2 * k + 1;
        const float* rec = a.records + (long long)slot * chunk_record_floats(D, SUBS) + (long long)w * kRows * (D + 2);
        const float pm = rec[D * kRows + row0 + lane], pl = rec[(D + 1) * kRows + row0 + lane];
        float4 y[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) y[x] = reinterpret_cast<const float4*>(rec)[(blockIdx.z * 8 + x) * kRows + row0 + lane];
        if (pm == -INFINITY) continue;  // the row sees none of the piece's keys
        const float to = fmaxf(mx, pm), old = mx == -INFINITY ? 0.f : ex2(mx - to), f = ex2(pm - to);
        mx = to;
        l = l * old + pl * f;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            o[4 * x] = o[4 * x] * old + y[x].x * f;
            o[4 * x + 1] = o[4 * x + 1] * old + y[x].y * f;
            o[4 * x + 2] = o[4 * x + 2] * old + y[x].z * f;
            o[4 * x + 3] = o[4 * x + 3] * old + y[x].w * f;
        }
    }
    top[warp][lane] = mx;
    sum[warp][lane] = l;
#pragma unroll
    for (int x = 0; x < 32; ++x) part[warp][lane][x] = o[x];
    __syncthreads();
    // eight threads a row, four columns each
    const int r = threadIdx.x >> 3, x0 = (threadIdx.x & 7) * 4, in_tile = (row0 + r) / a.group, i = from + in_tile;
    if (in_tile >= tokens || i >= m) return;
    float all = -INFINITY;
#pragma unroll
    for (int k = 0; k < 8; ++k) all = fmaxf(all, top[k][r]);
    float total = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if (top[k][r] == -INFINITY) continue;
        const float f = ex2(top[k][r] - all);
        total += sum[k][r] * f;
#pragma unroll
        for (int x = 0; x < 4; ++x) y[x] += part[k][r][x0 + x] * f;
    }
    const float inv = total > 0.f ? 1.f / total : 0.f;
    const int head = a.head_of_slot[b.head] * a.group + (row0 + r) % a.group;
    const long long at_head = (long long)(start + i) * a.q_heads + head;
    *reinterpret_cast<uint2*>(a.out + at_head * D + blockIdx.z * 32 + x0) = make_uint2(bf16x2(y[0] * inv, y[1] * inv), bf16x2(y[2] * inv, y[3] * inv));
    if (a.lse && blockIdx.z == 0 && x0 == 0) a.lse[at_head] = total > 0.f ? (all + log2f(total)) * kLn2 : -INFINITY;
}

template <int D, int SUBS, bool FP8>
cudaError_t launch_shape(const ChunkArgs& a, const ChunkMaps& m, bool split, cudaStream_t stream)
{
    using C = Chunk<D, SUBS, FP8>;
    auto kernel = a.softcap != 0.f ? (a.slopes ? chunk_attention_kernel<D, SUBS, FP8, true, true> : chunk_attention_kernel<D, SUBS, FP8, true, false>)
                                   : (a.slopes ? chunk_attention_kernel<D, SUBS, FP8, false, true> : chunk_attention_kernel<D, SUBS, FP8, false, false>);
    kernel<<<a.ctas, C::kThreads, C::kSmem, stream>>>(a, m);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || !split) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(a.ctas - 1, SUBS * 4, D / 32);
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, chunk_combine_kernel<D, SUBS>, a);
}

template <int D, int SUBS, bool FP8>
cudaError_t prepare_shape()
{
    const void* kernels[] = {(const void*)chunk_attention_kernel<D, SUBS, FP8, false, false>, (const void*)chunk_attention_kernel<D, SUBS, FP8, false, true>,
                             (const void*)chunk_attention_kernel<D, SUBS, FP8, true, false>, (const void*)chunk_attention_kernel<D, SUBS, FP8, true, true>};
    for (const void* k : kernels) {
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, Chunk<D, SUBS, FP8>::kSmem);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_chunk_attention(const ChunkArgs& a, const ChunkMaps& m, int head_dim, int subs, bool split, cudaStream_t stream)
{
    if (a.pool8) return subs == 2 ? launch_shape<128, 2, true>(a, m, split, stream) : launch_shape<128, 1, true>(a, m, split, stream);
    if (head_dim == 128) return subs == 2 ? launch_shape<128, 2, false>(a, m, split, stream) : launch_shape<128, 1, false>(a, m, split, stream);
    return subs == 2 ? launch_shape<64, 2, false>(a, m, split, stream) : launch_shape<64, 1, false>(a, m, split, stream);
}

cudaError_t prepare_chunk_kernels(int head_dim, bool fp8)
{
    cudaError_t e;
    if (fp8) {
        e = prepare_shape<128, 2, true>();
        return e != cudaSuccess ? e : prepare_shape<128, 1, true>();
    }
    e = head_dim == 128 ? prepare_shape<128, 2, false>() : prepare_shape<64, 2, false>();
    return e != cudaSuccess ? e : head_dim == 128 ? prepare_shape<128, 1, false>() : prepare_shape<64, 1, false>();
}

}  // namespace rlkv
