// Attention of a chunk of new tokens of each of several sequences over the paged cache and over the chunk itself.
//
// The queries of a KV head's group are packed token by token into tiles of 128 rows, so that a few drafted tokens of eight
// heads fill a tensor-core tile as well as a prompt does, and every K and V row is read once for all of them.  Per key tile:
// S = Q.K^T (both operands in shared memory, fp32 in tensor memory); a warpgroup turns S into P = exp2(s - m), written over S; O +=
// P.V with P read from tensor memory.  Keys are the chunk's own rows and then what the cache holds, from the newest back: its
// 64-row pages or rings as they lie.
//
// Three shapes of one kernel (rlkv_paged_chunks.cu chooses, with what both sides measured):
//   SHAPE 0  at most 32 rows a unit: they stand four times in the tile, once for each softmax warp, which takes a quarter of the
//            tile's 64 keys for all of them; the warps' maxima, sums and outputs meet when the unit ends.  (One warp with all the
//            keys was the bound: four drafted tokens of 32 sequences, 8 bits, 202 us, so 160.)
//   SHAPE 1  128 rows, 64 keys.  Both of these with two CTAs on an SM: while one waits for memory, sets up or writes results, the
//            other computes.  S alternates between two places, so the next product runs beside the softmax.
//   SHAPE 2  two tiles of rows that share their key tiles of 128, one CTA on an SM: one's products run while the other's softmax does,
//            and the K/V rows pass through shared memory half as often, codes through their decoding.
// Each CTA walks one contiguous range of the units' key tiles (rlkv_chunk.cuh); units that a range's end cuts are added up
// by a second kernel.
//
//   warps 0-3 (0-7)  softmax of sub-tile 0 (1), and its output rows at the end
//   then             TMA: queries, K and V tiles through one ring
//                    the issue of every tcgen05.mma, in order
//                    clearing the V rows that hold no token (0 * NaN of a recycled page would be NaN)
//   last four        8-bit caches: V codes to fp16
//
// The running maximum of a row moves only when it would grow by more than 2^8 (its effect cancels in O / l, which are fp32).
// Every row sees its own token at least, so that l is above 0, unless scores are not finite: those rows become NaN, in one piece or
// in many (a maximum passes over NaN, a sum does not).
// P is rounded to bf16 for the product, half a step 2^-8 of each weight; l sums the fp32 values.
//
// An 8-bit cache.  Scores come from the K codes as they lie, on the products of 8-bit operands: the queries are split into an E4M3
// and an E5M2 number (split_row), which costs the same products as bf16 would.  V codes (they lie transposed, an element's tokens contiguous)
// are decoded by four warps, to fp16, which holds them exactly and which one instruction converts two of; so P is fp16 there, with
// its reference 2^7 below a row's largest score: P from 2^15 down to 2^-14 keeps eleven bits, the step below that is 2^-31 of the
// largest weight.  (Both operands decoded to bf16 by their bits: 250 us for four drafted tokens of 32 sequences; V only 137; V by
// conversions 127.  P in two E4M3 parts would need no decoding, but loses the tail behind a sink token's weight.  Tiles of 128
// keys with a single place for S: 139.)  Scales never touch codes or queries: K's goes into the scores' factor, O is kept in units of
// V's from the first cached tile on.
//
// Measured on one B200 (us on the GPU; 32 / 8 heads of 128, 6 of 8 full, unless said otherwise): five drafted tokens on 8192 14.5
// (latency of one wave and of the join); four of each of 32 sequences of 8064 on average, 16 bits 129 (819 MB: 6.3 TB/s), 8 bits 106
// (410 MB: the products, the decoding and the softmax of a tile share an SM's shared memory and issue slots); 512 beside 47 single
// tokens of 3400 on average (28 / 4 heads, 3 of 4 full, capped) 86 (alone 42 and 55), in 8 bits, as two launches, 135 (68 and 59); 2048 on 8192, all full, 267 in bursts (1.16 PFLOP/s, 69 % of a large
// library product's burst rate), 8 bits 384 (one product per 128 keys; 395 with one per page).
//
// Tried and not taken: units of at most 32 rows four times in the tile of SHAPE 1 too, where they stand beside larger ones (512 beside
// 47 88 -> 116, in 8 bits 144 -> 207: the code of both costs the softmax its registers); the two kinds as two launches at once on two
// streams (70.9 -> 113 and more), and in 16 bits one behind the other (8-bit caches have them so, see two_launches in rlkv_paged_chunks.cu); ranges that weigh tiles of few rows less or more (equal weights are best).
#include <cuda_fp16.h>
#include <float.h>

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

template <int D, int SHAPE, bool FP8>
struct Chunk {
    static constexpr int SUBS = SHAPE == 2 ? 2 : 1;
    static constexpr bool QUAD = SHAPE == 0;
    static constexpr int kKeys = SUBS == 2 ? 128 : 64;  // of a tile
    static constexpr int kPages = kKeys / kTile;
    static constexpr int kQBytes = kRows * D * 2, kTileBytes = kKeys * D * 2;
    static constexpr int kBlock = kKeys * 128;  // bytes of a [kKeys][64 elements] block
    static constexpr int kStages = FP8 ? 3 : D == 128 ? 5 : 10;  // K or V tiles in the ring; of an 8-bit cache, the codes of both
    static constexpr int kDecoded = FP8 ? 2 : 0;                 // decoded V tiles
    static constexpr int kState = SUBS * kQBytes + (kStages + kDecoded) * kTileBytes;
    static constexpr int kSmem = kState + 1024 * SUBS;
    static constexpr int kSoftmaxWarps = 4 * SUBS;
    static constexpr int kThreads = 32 * (kSoftmaxWarps + 4 + (FP8 ? 4 : 0));
    static constexpr int kPerSm = SUBS == 2 ? 1 : 2;
    static constexpr int kColumns = SUBS == 2 ? 512 : 256;  // of tensor memory: two S/P places, then O
    static constexpr int kReleases = FP8 ? 5 : 1;           // arrivals that free a stage: the products' end, and the decoding warps
};

// The part of a CTA's range that lies in one unit.
struct Segment {
    ChunkUnit u;
    int len, m, start, slot;  // of the sequence
    int head;                 // KV head
    bool full;
    int index;                // among the heads of its class
    int fresh;                // the chunk's own key tiles; the cached ones come behind them
    int t0, t1, subs;         // key tiles, sub-tiles that hold rows
    int record;               // -1: the whole unit, whose rows are final
};
// A softmax warp's place in its CTA's range and the segment it is at, kept in shared memory: its threads' registers go to scores.
struct SoftmaxPlace {
    ChunkPos at;
    int first;
    Segment g;
};

template <bool REFER, class A, class B>
struct Choose;
template <class A, class B>
struct Choose<true, A, B> {
    typedef A type;
    static __device__ __forceinline__ A of(const Segment& s) { return s; }
};
template <class A, class B>
struct Choose<false, A, B> {
    typedef B type;
    static __device__ __forceinline__ B of(const Segment& s) { return s; }
};

struct ChunkShared {
    uint64_t q_full[2], q_split[2], q_empty[2], full[10], empty[10], dirty[10], clean[10], decoded[2], decoded_empty[2];
    uint64_t s_full[2], p_full[2][2], pv_done[2], meet, drain;
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

// An 8-bit page, or its K or its V codes: rows of 128 bytes from row `row` on, as many as the map's box has, 128-byte swizzle.
__device__ __forceinline__ void load_page(uint32_t dst, const CUtensorMap* map, int row, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(0),
                 "r"(row), "r"(bar)
                 : "memory");
}

// E4M3 (`wide`: E5M2) x E4M3 -> fp32, 32 elements of the contraction; both operands in shared memory, rows of 128 bytes.
__host__ __device__ constexpr uint32_t instr_desc8(int m, int n, bool wide)
{
    return 1u << 4 | (wide ? 1u << 7 : 0u) | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}
__device__ __forceinline__ void mma_ss8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}

// Sixteen E4M3 codes as fp16.
__device__ __forceinline__ void decode4(uint32_t codes, uint32_t& lo, uint32_t& hi)
{
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=&r"(lo), "=&r"(hi) : "r"(codes));
}
__device__ __forceinline__ void decode16(const uint4& codes, uint4& lo, uint4& hi)
{
    decode4(codes.x, lo.x, lo.y);
    decode4(codes.y, lo.z, lo.w);
    decode4(codes.z, hi.x, hi.y);
    decode4(codes.w, hi.z, hi.w);
}

// The first n bytes of a word (n below 0: none, above 4: all).
__device__ __forceinline__ uint32_t first_bytes(int n) { return n <= 0 ? 0u : n >= 4 ? ~0u : (1u << 8 * n) - 1u; }

// Four numbers to E4M3 (nearest, saturating) and back.
__device__ __forceinline__ uint32_t codes4(float2 f, float2 g)
{
    uint32_t d;
    asm("{\n\t.reg .b16 a, b;\n\tcvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\n\tmov.b32 %0, {a, b};\n\t}"
        : "=r"(d)
        : "f"(f.x), "f"(f.y), "f"(g.x), "f"(g.y));
    return d;
}
// Four numbers to E5M2.
__device__ __forceinline__ uint32_t wide_codes4(float2 f, float2 g)
{
    uint32_t d;
    asm("{\n\t.reg .b16 a, b;\n\tcvt.rn.satfinite.e5m2x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e5m2x2.f32 b, %4, %3;\n\tmov.b32 %0, {a, b};\n\t}"
        : "=r"(d)
        : "f"(f.x), "f"(f.y), "f"(g.x), "f"(g.y));
    return d;
}
__device__ __forceinline__ void values4(uint32_t codes, float2& f, float2& g)
{
    uint32_t a, b;
    decode4(codes, a, b);
    f = __half22float2(*reinterpret_cast<const __half2*>(&a));
    g = __half22float2(*reinterpret_cast<const __half2*>(&b));
}

// A query row of 128 bf16 elements in shared memory (two runs of 128 bytes, swizzled by the row) becomes, in place, two rows of
// 8-bit numbers: x 2^e = a + b, a rounded to E4M3, b what is left, to E5M2.  2^e brings the largest element to 128 .. 256.  A bf16
// number has eight bits; where a is a normal number of four, b has at most three, which E5M2 holds down to 2^-16: a + b is exact down
// to 2^-13 of the largest element.  Below, b is at most 2^-10 and off by 2^-14: 2^-21 of the largest element.  (With b in E4M3 too, whose
// step ends at 2^-9, it was 2^-18, and one channel 1000 or 3000 times the others cost them: out over 4096 keys off by 2.6e-3 and 9.0e-3
// of its norm, so 1.65e-3 with either -- its own rounding; lse of five keys 4.5e-3 and 2.4e-2, so 9e-5 and 6e-4; the same time.)
// Returns 2^-e, and of a row with an infinite element (a code stands for its sign)
// infinity: its scores are infinite, or NaN against keys of zero, as they would be of the queries as given.
__device__ __forceinline__ float split_row(uint8_t* q, int row)
{
    uint4* at[2] = {reinterpret_cast<uint4*>(q + row * 128), reinterpret_cast<uint4*>(q + kQBlock + row * 128)};
    uint4 x[16];
#pragma unroll
    for (int c = 0; c < 16; ++c) x[c] = at[c / 8][(c & 7) ^ (row & 7)];
    __nv_bfloat162 top = __float2bfloat162_rn(0.f);
    const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(x);
#pragma unroll
    for (int i = 0; i < 64; ++i) top = __hmax2(top, __habs2(p[i]));
    const float big = fmaxf(__low2float(top), __high2float(top));
    const int exponent = min(max((__float_as_int(big) >> 23 & 255) - 134, -126), 120);  // of the largest element's distance from 2^7
    const float up = __int_as_float((127 - exponent) << 23), down = big == INFINITY ? INFINITY : __int_as_float((127 + exponent) << 23);
#pragma unroll
    for (int c = 0; c < 8; ++c) {  // sixteen elements: sixteen bytes of a and of b
        uint32_t a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float2 f = __bfloat1622float2(p[c * 8 + 2 * i]), g = __bfloat1622float2(p[c * 8 + 2 * i + 1]), r, t;
            f = mul2(f, make_float2(up, up));
            g = mul2(g, make_float2(up, up));
            a[i] = codes4(f, g);
            values4(a[i], r, t);
            b[i] = wide_codes4(make_float2(f.x - r.x, f.y - r.y), make_float2(g.x - t.x, g.y - t.y));
        }
        at[0][c ^ (row & 7)] = make_uint4(a[0], a[1], a[2], a[3]);
        at[1][c ^ (row & 7)] = make_uint4(b[0], b[1], b[2], b[3]);
    }
    return down;
}

// A row's columns, waited for in the same statement: none of them can be spilled before it has arrived.
__device__ __forceinline__ void read_columns(uint32_t addr, float (&s)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(s[0]), "=f"(s[1]), "=f"(s[2]), "=f"(s[3]), "=f"(s[4]), "=f"(s[5]), "=f"(s[6]), "=f"(s[7]), "=f"(s[8]),
          "=f"(s[9]), "=f"(s[10]), "=f"(s[11]), "=f"(s[12]), "=f"(s[13]), "=f"(s[14]), "=f"(s[15])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void read_columns(uint32_t addr, float (&s)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(s[0]), "=f"(s[1]), "=f"(s[2]), "=f"(s[3]), "=f"(s[4]), "=f"(s[5]), "=f"(s[6]), "=f"(s[7]), "=f"(s[8]), "=f"(s[9]),
          "=f"(s[10]), "=f"(s[11]), "=f"(s[12]), "=f"(s[13]), "=f"(s[14]), "=f"(s[15]), "=f"(s[16]), "=f"(s[17]), "=f"(s[18]),
          "=f"(s[19]), "=f"(s[20]), "=f"(s[21]), "=f"(s[22]), "=f"(s[23]), "=f"(s[24]), "=f"(s[25]), "=f"(s[26]), "=f"(s[27]),
          "=f"(s[28]), "=f"(s[29]), "=f"(s[30]), "=f"(s[31])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void read_columns(uint32_t addr, float (&s)[64])
{
    asm volatile(
        "{\n\t.reg .b32 at;\n\tmov.b32 at, %64;\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [at];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,"
        "%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [at+32];\n\t"
        "tcgen05.wait::ld.sync.aligned;\n\t}"
        : "=f"(s[0]), "=f"(s[1]), "=f"(s[2]), "=f"(s[3]), "=f"(s[4]), "=f"(s[5]), "=f"(s[6]), "=f"(s[7]), "=f"(s[8]), "=f"(s[9]),
          "=f"(s[10]), "=f"(s[11]), "=f"(s[12]), "=f"(s[13]), "=f"(s[14]), "=f"(s[15]), "=f"(s[16]), "=f"(s[17]), "=f"(s[18]),
          "=f"(s[19]), "=f"(s[20]), "=f"(s[21]), "=f"(s[22]), "=f"(s[23]), "=f"(s[24]), "=f"(s[25]), "=f"(s[26]), "=f"(s[27]),
          "=f"(s[28]), "=f"(s[29]), "=f"(s[30]), "=f"(s[31]), "=f"(s[32]), "=f"(s[33]), "=f"(s[34]), "=f"(s[35]), "=f"(s[36]),
          "=f"(s[37]), "=f"(s[38]), "=f"(s[39]), "=f"(s[40]), "=f"(s[41]), "=f"(s[42]), "=f"(s[43]), "=f"(s[44]), "=f"(s[45]),
          "=f"(s[46]), "=f"(s[47]), "=f"(s[48]), "=f"(s[49]), "=f"(s[50]), "=f"(s[51]), "=f"(s[52]), "=f"(s[53]), "=f"(s[54]),
          "=f"(s[55]), "=f"(s[56]), "=f"(s[57]), "=f"(s[58]), "=f"(s[59]), "=f"(s[60]), "=f"(s[61]), "=f"(s[62]), "=f"(s[63])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void read_columns(uint32_t addr, float (&s)[128])
{
    asm volatile(
        "{\n\t.reg .b32 at;\n\tmov.b32 at, %128;\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [at];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,"
        "%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [at+32];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%64,%65,%66,%67,%68,%69,%70,%71,%72,%73,%74,%75,%76,%77,%78,%79,"
        "%80,%81,%82,%83,%84,%85,%86,%87,%88,%89,%90,%91,%92,%93,%94,%95}, [at+64];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%96,%97,%98,%99,%100,%101,%102,%103,%104,%105,%106,%107,%108,%109,%110,%111,"
        "%112,%113,%114,%115,%116,%117,%118,%119,%120,%121,%122,%123,%124,%125,%126,%127}, [at+96];\n\t"
        "tcgen05.wait::ld.sync.aligned;\n\t}"
        : "=f"(s[0]), "=f"(s[1]), "=f"(s[2]), "=f"(s[3]), "=f"(s[4]), "=f"(s[5]), "=f"(s[6]), "=f"(s[7]), "=f"(s[8]), "=f"(s[9]),
          "=f"(s[10]), "=f"(s[11]), "=f"(s[12]), "=f"(s[13]), "=f"(s[14]), "=f"(s[15]), "=f"(s[16]), "=f"(s[17]), "=f"(s[18]),
          "=f"(s[19]), "=f"(s[20]), "=f"(s[21]), "=f"(s[22]), "=f"(s[23]), "=f"(s[24]), "=f"(s[25]), "=f"(s[26]), "=f"(s[27]),
          "=f"(s[28]), "=f"(s[29]), "=f"(s[30]), "=f"(s[31]), "=f"(s[32]), "=f"(s[33]), "=f"(s[34]), "=f"(s[35]), "=f"(s[36]),
          "=f"(s[37]), "=f"(s[38]), "=f"(s[39]), "=f"(s[40]), "=f"(s[41]), "=f"(s[42]), "=f"(s[43]), "=f"(s[44]), "=f"(s[45]),
          "=f"(s[46]), "=f"(s[47]), "=f"(s[48]), "=f"(s[49]), "=f"(s[50]), "=f"(s[51]), "=f"(s[52]), "=f"(s[53]), "=f"(s[54]),
          "=f"(s[55]), "=f"(s[56]), "=f"(s[57]), "=f"(s[58]), "=f"(s[59]), "=f"(s[60]), "=f"(s[61]), "=f"(s[62]), "=f"(s[63]),
          "=f"(s[64]), "=f"(s[65]), "=f"(s[66]), "=f"(s[67]), "=f"(s[68]), "=f"(s[69]), "=f"(s[70]), "=f"(s[71]), "=f"(s[72]),
          "=f"(s[73]), "=f"(s[74]), "=f"(s[75]), "=f"(s[76]), "=f"(s[77]), "=f"(s[78]), "=f"(s[79]), "=f"(s[80]), "=f"(s[81]),
          "=f"(s[82]), "=f"(s[83]), "=f"(s[84]), "=f"(s[85]), "=f"(s[86]), "=f"(s[87]), "=f"(s[88]), "=f"(s[89]), "=f"(s[90]),
          "=f"(s[91]), "=f"(s[92]), "=f"(s[93]), "=f"(s[94]), "=f"(s[95]), "=f"(s[96]), "=f"(s[97]), "=f"(s[98]), "=f"(s[99]),
          "=f"(s[100]), "=f"(s[101]), "=f"(s[102]), "=f"(s[103]), "=f"(s[104]), "=f"(s[105]), "=f"(s[106]), "=f"(s[107]),
          "=f"(s[108]), "=f"(s[109]), "=f"(s[110]), "=f"(s[111]), "=f"(s[112]), "=f"(s[113]), "=f"(s[114]), "=f"(s[115]),
          "=f"(s[116]), "=f"(s[117]), "=f"(s[118]), "=f"(s[119]), "=f"(s[120]), "=f"(s[121]), "=f"(s[122]), "=f"(s[123]),
          "=f"(s[124]), "=f"(s[125]), "=f"(s[126]), "=f"(s[127])
        : "r"(addr)
        : "memory");
}

__device__ __forceinline__ uint32_t f16x2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// P = 2^(s factor - base) of a row's scores, as bf16 (F16 and `half`: as fp16) to tensor memory, and their sums; 64 keys at a
// time, so that the product starts on the first.
template <bool F16, int N>
__device__ __forceinline__ void exponentials(float (&s)[N], float factor, float base, bool half, float2 (&sum)[2], uint32_t P, uint64_t* done, int lane, int)
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
            if (!F16) packed[i / 2] = bf16x2(s[c + i], s[c + i + 1]);
        }
        if (F16) {
            if (half) {
#pragma unroll
                for (int i = 0; i < 16; ++i) packed[i] = f16x2(s[c + 2 * i], s[c + 2 * i + 1]);
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) packed[i] = bf16x2(s[c + 2 * i], s[c + 2 * i + 1]);
            }
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
// The same for a quarter of 64 keys, those of warp `quarter`: P of the other keys is zero in this warp's rows.
template <bool F16>
__device__ __forceinline__ void exponentials(float (&s)[16], float factor, float base, bool half, float2 (&sum)[2], uint32_t P, uint64_t* done, int lane, int quarter)
{
    const float2 factor2 = make_float2(factor, factor), base2 = make_float2(-base, -base);
#pragma unroll
    for (int x = 1; x < 4; ++x)
        asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%1,%1,%1,%1,%1,%1,%1};" ::"r"(P + ((quarter + x) & 3) * 8), "r"(0) : "memory");
    uint32_t packed[8];
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
        const float2 x = fma2(make_float2(s[i], s[i + 1]), factor2, base2);
        s[i] = ex2(x.x);
        s[i + 1] = ex2(x.y);
        if (!F16) packed[i / 2] = bf16x2(s[i], s[i + 1]);
    }
    if (F16) {
        if (half) {
#pragma unroll
            for (int i = 0; i < 8; ++i) packed[i] = f16x2(s[2 * i], s[2 * i + 1]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) packed[i] = bf16x2(s[2 * i], s[2 * i + 1]);
        }
    }
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(P + quarter * 8), "r"(packed[0]), "r"(packed[1]),
                 "r"(packed[2]), "r"(packed[3]), "r"(packed[4]), "r"(packed[5]), "r"(packed[6]), "r"(packed[7])
                 : "memory");
    wait_st();
    fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(done));
#pragma unroll
    for (int c = 0; c < 16; c += 2) sum[c / 2 & 1] = add2(sum[c / 2 & 1], make_float2(s[c], s[c + 1]));
}

// Walks the segments of CTA `cta` in order.
template <int KEYS, int SUBS, int ROWS>
struct Walk {
    const ChunkArgs& a;
    ChunkPos at, end;
    int tokens, cta;  // tokens of a sub-tile
    bool first = true;
    __device__ __forceinline__ Walk(const ChunkArgs& args) : a(args), at(args.at[blockIdx.x]), end(args.at[blockIdx.x + 1]), tokens(ROWS / args.group), cta(blockIdx.x) {}
    __device__ __forceinline__ bool next(Segment& s)
    {
        if (same_unit(at, end) && at.tile >= end.tile) return false;
        s.start = a.seqs.start[at.seq];
        s.m = a.seqs.count[at.seq];
        s.len = a.seqs.len[at.seq];
        s.slot = a.seqs.slot[at.seq];
        s.full = at.head < a.n_full;
        s.index = s.full ? at.head : at.head - a.n_full;
        s.head = a.head_of_slot[at.head];
        s.u = chunk_unit(s.len, s.m, at.row_tile, SUBS * tokens, KEYS, s.full, a.sink, a.window);
        s.subs = SUBS == 2 && s.m - s.u.tok0 > tokens ? 2 : 1;
        s.fresh = s.u.tiles - s.u.cached;
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
                    ++at.seq;
                }
            }
        }
        return true;
    }
    // First key of key tile t: a token of the chunk (t < fresh), or a row of what the cache holds -- from the newest back, so
    // that distance terms are at their largest first and the running maximum stays.
    template <class S>
    static __device__ __forceinline__ int key_tile(const S& s, int t)
    {
        return (t >= s.fresh ? s.u.tiles - 1 - t : t < s.u.a_end ? t : s.u.b0 + t - s.u.a_end) * KEYS;
    }
    // Rows of key tile t that hold a token (KEYS or more: all of them).
    static __device__ __forceinline__ int valid_rows(const Segment& s, int t) { return (t < s.fresh ? s.m : s.u.rows) - key_tile(s, t); }
    // Whether the V rows of key tile t are to be cleared where they hold no token: 0 * NaN of what lies there would be NaN.
    // (Decoded codes are finite.)
    template <bool FP8>
    static __device__ __forceinline__ bool unclean(const Segment& s, int t) { return (!FP8 || t < s.fresh) && valid_rows(s, t) < KEYS; }
};

template <int D, int SHAPE, bool FP8, bool CAP, bool BIAS>
__global__ void __launch_bounds__(Chunk<D, SHAPE, FP8>::kThreads, Chunk<D, SHAPE, FP8>::kPerSm)
chunk_attention_kernel(const __grid_constant__ ChunkArgs a, const __grid_constant__ ChunkMaps maps)
{
    using C = Chunk<D, SHAPE, FP8>;
    constexpr int SUBS = C::SUBS, KEYS = C::kKeys, kHalves = KEYS / 64;
    constexpr bool QUAD = C::QUAD;
    constexpr float kLift = FP8 ? 7.f : 0.f;  // what the running maximum lies below a row's largest score: fp16 P of 2^7, 2^15 at most
    constexpr int kTileRows = QUAD ? 32 : kRows;      // query rows of a sub-tile
    constexpr int kColumnsOf = QUAD ? KEYS / 4 : KEYS;  // scores of a thread
    using W = Walk<KEYS, SUBS, kTileRows>;
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
            prefetch_map(&maps.pool);
            sh.abort = 0;
            for (int i = 0; i < C::kStages; ++i) {
                mbar_init(smem_u32(&sh.full[i]), 1);
                mbar_init(smem_u32(&sh.empty[i]), C::kReleases);
                mbar_init(smem_u32(&sh.dirty[i]), 1);
                mbar_init(smem_u32(&sh.clean[i]), 1);
            }
            for (int w = 0; w < 2; ++w) {
                mbar_init(smem_u32(&sh.q_full[w]), 1);
                mbar_init(smem_u32(&sh.q_empty[w]), 4);
                mbar_init(smem_u32(&sh.q_split[w]), 4);
                mbar_init(smem_u32(&sh.decoded[w]), 4);
                mbar_init(smem_u32(&sh.decoded_empty[w]), 1);
                mbar_init(smem_u32(&sh.s_full[w]), 1);
                mbar_init(smem_u32(&sh.p_full[w][0]), 4);
                mbar_init(smem_u32(&sh.p_full[w][1]), 4);
                mbar_init(smem_u32(&sh.pv_done[w]), 1);
            }
            mbar_init(smem_u32(&sh.meet), 4);
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
    const uint32_t q_smem = smem_u32(smem), ring = q_smem + SUBS * C::kQBytes, decoded = ring + C::kStages * C::kTileBytes;
    const uint32_t o_column = SUBS == 2 ? 256 : 128;
    // Registers of the warpgroups, which together have what the block was launched with.  16 bits: 384 x 168 = 256 x 224 + 128 x 56,
    // 256 x 128 = 128 x 184 + 128 x 72; 8 bits: 512 x 128 = 256 x 208 + 128 x 56 + 128 x 40, 384 x 80 = 128 x (128 + 72 + 40)
    if (warp < C::kSoftmaxWarps) more_registers<SUBS == 2 ? (FP8 ? 208 : 224) : FP8 ? 128 : 184>();
    else if (warp >= kDecode) fewer_registers<40>();
    else fewer_registers<SUBS == 2 ? 56 : 72>();
    if (warp < C::kSoftmaxWarps) {
        // ------------------------------------------------------------------ softmax
        const int w = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t O = tmem + lanes + o_column + w * D;
        const int tile_row = QUAD ? lane : row, in_tile = tile_row / a.group, member = tile_row - in_tile * a.group;
        const int tokens = kTileRows / a.group;
        const int column0 = QUAD ? warp * kColumnsOf : 0;  // the warp's part of a tile's keys
        int total = 0, seg = 0;  // tiles of this sub-tile and segments so far
        bool ok = true;
        // SUBS 1: the score product of tile n goes out before the value product of tile n - 1, so that two of the latter may be
        // outstanding: they take turns at two barriers, or a wait could take the end of the one before for its own
        auto product_done = [&](int n) {
            return SUBS == 2 ? wait_warp(smem_u32(&sh.pv_done[w]), n & 1, abort_flag, a.status, kChunkWaitProduct)
                             : wait_warp(smem_u32(&sh.pv_done[n & 1]), n >> 1 & 1, abort_flag, a.status, kChunkWaitProduct);
        };
        int met = 0;
        auto meet = [&]() {  // the four softmax warps of a CTA wait for one another
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.meet));
            return wait_warp(smem_u32(&sh.meet), met++ & 1, abort_flag, a.status, kChunkWaitSoftmax);
        };
        SoftmaxPlace* place_of = sh.place + warp;
        const volatile Segment& kept = place_of->g;
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
            if (w >= kept.subs) continue;
            // (where scores take all registers, the segment is read where it is needed)
            typedef Choose<SUBS == 2 || (FP8 && !QUAD), const volatile Segment&, const Segment> Kept;
            typename Kept::type g = Kept::of(place_of->g);
            const int from = g.u.tok0 + w * tokens;     // the sub-tile's first token
            const int i = from + in_tile, head = g.head * a.group + member;
            const bool mine = in_tile < tokens && i < g.m;
            const int upto = min(from + tokens, g.m) - 1;   // its last
            const float slope2 = BIAS && mine ? a.slopes[head] * kLog2e : 0.f;
            // the ring: its sink rows hold tokens 0 .. sink-1, the rows up to w1 the newest, the rows from w1 on those one
            // window older
            const int w1 = g.len > a.sink ? a.sink + (g.len - 1 - a.sink) % a.window + 1 : g.len;
            const float k_scale = FP8 ? a.k_scale[g.head] : 1.f, v_scale = FP8 ? a.v_scale[g.head] : 1.f;
            const bool busy = __any_sync(0xffffffffu, mine);  // (a warp none of whose rows is a query only keeps step)
            float scale = a.scale;
            Cap cap(CAP ? a.softcap : 1.f, scale);
            float m = -INFINITY, l = 0.f;
            for (int t = g.t0; t < g.t1; ++t) {
                const int place = SUBS == 2 ? w : total & 1;
                const uint32_t S = tmem + lanes + place * KEYS;
                const bool cached = t >= g.fresh;
                float corr = 1.f;  // of O
                if (FP8 && cached && t == max(g.t0, g.fresh)) {  // from the chunk's rows to the cache's codes
                    // (the score products of the rows have ended: this warp has seen the last one's result)
                    ok = wait_warp(smem_u32(&sh.q_full[w]), seg & 1, abort_flag, a.status, kChunkWaitQueries);
                    if (!ok) break;
                    if (busy) scale = a.scale * k_scale * split_row(smem + w * C::kQBytes, row);
                    if (CAP) cap = Cap(a.softcap, scale);
                    if (t > g.t0) corr = 1.f / v_scale;
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&sh.q_split[w]));
                }
                ok = wait_warp(smem_u32(&sh.s_full[place]), (SUBS == 2 ? total : total >> 1) & 1, abort_flag, a.status, kChunkWaitProduct);
                if (!ok) break;
                ++total;
                if (!busy) {
                    __syncwarp();
                    if (lane < kHalves) mbar_arrive(smem_u32(&sh.p_full[place][lane]));
                    continue;
                }
                fence_after();
                const int start = W::key_tile(g, t) + column0;
                const bool plain = cached ? g.full && start + kColumnsOf <= g.len
                                          : start + kColumnsOf <= from + 1 && (g.full || start > upto - a.window || start + kColumnsOf <= a.sink - g.len);
                uint32_t see[(kColumnsOf + 31) / 32];
                if (!plain) {
                    // what this row sees of the tile: up to three ranges of columns, [lo1, hi1), [lo2, hi2), [0, hi3)
                    int lo1 = 0, hi1, lo2 = 0, hi2 = 0, hi3 = 0;
                    if (cached) {
                        hi1 = g.len - start;
                        if (!g.full) {
                            hi3 = min(a.sink, g.u.rows) - start;
                            lo1 = max(a.sink, w1 + i + 1 - a.window) - start;
                            hi1 = w1 - start;
                            lo2 = w1 + i + 1 - start;
                            hi2 = g.u.rows - start;
                        }
                    } else {
                        hi1 = i + 1 - start;
                        if (!g.full) {
                            lo1 = i - a.window + 1 - start;
                            hi3 = min(a.sink - g.len, i + 1) - start;
                        }
                    }
#pragma unroll
                    for (int x = 0; x < kColumnsOf; x += 32)
                        see[x / 32] = mine ? range_bits(lo1 - x, hi1 - x) | range_bits(lo2 - x, hi2 - x) | range_bits(0, hi3 - x) : 0u;
                }
                float s[kColumnsOf];
                read_columns(S + column0, s);
                if (CAP) {
                    if (!plain) {  // (what lies in rows without a token has no say in how a warp computes the cap)
#pragma unroll
                        for (int c = 0; c < kColumnsOf; ++c) s[c] = see[c / 32] >> (c & 31) & 1 ? s[c] : 0.f;
                    }
                    cap.apply(s, mine);
                }
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
                        for (int c = 0; c < kColumnsOf; c += 2) {
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
                        for (int c = 0; c < kColumnsOf; ++c) {
                            const float from_row = c < b1 ? far : c < b2 ? near : older;
                            s[c] = fmaf(-slope2, from_row - (float)c, CAP ? s[c] : s[c] * sl2);
                        }
                    }
                }
                if (!plain) {
#pragma unroll
                    for (int c = 0; c < kColumnsOf; ++c) s[c] = see[c / 32] >> (c & 31) & 1 ? s[c] : -INFINITY;
                }
                // (a row of zeros on an 8-bit cache has next to no scale; times -infinity it must not be 0)
                const float factor = CAP || BIAS ? 1.f : FP8 ? fmaxf(scale * kLog2e, FLT_MIN) : scale * kLog2e;
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < kColumnsOf; ++c) mx[c & 3] = fmaxf(mx[c & 3], s[c]);
                const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * factor;
                if (top > m + 8.f + kLift) {  // (m may still be -infinity: then there is nothing to correct)
                    const float next = top - kLift, x = m == -INFINITY ? 1.f : ex2(m - next);
                    m = next;
                    l *= x;
                    corr *= x;
                }
                if (t > g.t0 && __any_sync(0xffffffffu, corr != 1.f)) {
                    ok = product_done(total - 2);
                    if (!ok) break;
                    fence_after();
#pragma unroll
                    for (int c = 0; c < D; c += 32) {
                        float o[32];
                        read_columns(O + c, o);
#pragma unroll
                        for (int x = 0; x < 32; ++x) o[x] *= corr;
                        tmem_st32(O + c, o);
                    }
                }
                const float base = m == -INFINITY ? 0.f : m;
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                exponentials<FP8>(s, factor, base, cached, sum, S, sh.p_full[place], lane, warp);
                l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
            }
            if (!ok) break;
            ++seg;
            if (busy) {
                ok = product_done(total - 1);
                if (!ok) break;
                fence_after();
            }
            const float unit = FP8 && g.t1 > g.fresh ? v_scale : 1.f;
            const long long at_head = ((long long)(g.start + i) * a.q_heads + head);
            if (QUAD) {
                // the warps' parts of the keys meet, in the memory of the queries (which are not needed any more): maxima and sums,
                // then half of the output's columns at a time, of which each warp adds up a quarter
                float* at = reinterpret_cast<float*>(smem);
                at[warp * 32 + lane] = m;
                at[128 + warp * 32 + lane] = l;
                ok = meet();
                float all = -INFINITY, total_l = 0.f;
#pragma unroll
                for (int x = 0; x < 4; ++x) all = fmaxf(all, at[x * 32 + lane]);
#pragma unroll
                for (int x = 0; x < 4; ++x) total_l += at[128 + x * 32 + lane] * (at[x * 32 + lane] == -INFINITY ? 0.f : ex2(at[x * 32 + lane] - all));
                const bool whole = g.record < 0;
                const float f = m == -INFINITY ? 0.f : ex2(m - all) * unit, inv = whole ? 1.f / total_l : 1.f;
                float* rec = a.records + (long long)max(g.record, 0) * chunk_record_floats(D, SHAPE);
                if (warp == 0) {
                    if (!whole) {
                        rec[D * 32 + lane] = all;
                        rec[(D + 1) * 32 + lane] = total_l;
                    } else if (mine && a.lse) {
                        a.lse[at_head] = (all + log2f(total_l)) * kLn2;
                    }
                }
                constexpr int kHalf = D / 8, kMine = D / 32;  // groups of four columns in a half, and a warp's of them
                float4* part = reinterpret_cast<float4*>(smem);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    ok = ok && meet();
#pragma unroll
                    for (int c = 0; c < D / 2; c += 32) {
                        float o[32];
                        read_columns(O + half * (D / 2) + c, o);
#pragma unroll
                        for (int x = 0; x < 8; ++x)
                            part[(warp * kHalf + c / 4 + x) * 32 + lane] = make_float4(o[4 * x] * f, o[4 * x + 1] * f, o[4 * x + 2] * f, o[4 * x + 3] * f);
                    }
                    ok = ok && meet();
                    float4 y[kMine];
#pragma unroll
                    for (int c = 0; c < kMine; ++c) {
                        y[c] = part[(warp * kMine + c) * 32 + lane];
#pragma unroll
                        for (int x = 1; x < 4; ++x) {
                            const float4 z = part[(x * kHalf + warp * kMine + c) * 32 + lane];
                            y[c] = make_float4(y[c].x + z.x, y[c].y + z.y, y[c].z + z.z, y[c].w + z.w);
                        }
                        if (!whole) reinterpret_cast<float4*>(rec)[(half * kHalf + warp * kMine + c) * 32 + lane] = y[c];
                    }
                    if (whole && mine)
#pragma unroll
                        for (int c = 0; c < kMine; c += 2)
                            *reinterpret_cast<uint4*>(a.out + at_head * D + half * (D / 2) + (warp * kMine + c) * 4) =
                                make_uint4(bf16x2(y[c].x * inv, y[c].y * inv), bf16x2(y[c].z * inv, y[c].w * inv),
                                           bf16x2(y[c + 1].x * inv, y[c + 1].y * inv), bf16x2(y[c + 1].z * inv, y[c + 1].w * inv));
                }
            } else if (!busy) {
            } else if (g.record < 0) {
                const float inv = unit / l;
                if (mine && a.lse) a.lse[at_head] = (m + log2f(l)) * kLn2;
                // through shared memory (the sub-tile's queries are not needed any more), so that whole rows go out
                uint8_t* stage = smem + w * C::kQBytes + (warp & 3) * 32 * D * 2;
                constexpr int kChunks = D / 8, kPerStore = 32 / kChunks;  // 16-byte pieces of a row, rows per store instruction
#pragma unroll
                for (int c = 0; c < D; c += 32) {
                    float o[32];
                    read_columns(O + c, o);
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
                float* rec = a.records + (long long)g.record * chunk_record_floats(D, SHAPE) + (long long)w * kRows * (D + 2);
#pragma unroll
                for (int c = 0; c < D; c += 32) {
                    float o[32];
                    read_columns(O + c, o);
                    if (mine)
#pragma unroll
                        for (int x = 0; x < 8; ++x)
                            reinterpret_cast<float4*>(rec)[(c / 4 + x) * kRows + row] =
                                make_float4(o[4 * x] * unit, o[4 * x + 1] * unit, o[4 * x + 2] * unit, o[4 * x + 3] * unit);
                }
                rec[D * kRows + row] = m;
                rec[(D + 1) * kRows + row] = l;
            }
            if (!ok) break;
            fence_before();
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.q_empty[w]));
        }
    } else if (warp == kLoad) {
        // ------------------------------------------------------------------ tile loads
        W walk(a);
        Segment g;
        int issued = 0, segs[2] = {0, 0}, loaded[2] = {0, 0};  // stages so far; segments of each sub-tile, those whose queries are on the way
        bool ok = true;
        while (ok && walk.next(g)) {
            const int row0 = g.start + g.u.tok0;
            bool q_waits = true;
            auto queries = [&]() {  // once the sub-tiles' rows of the segment before have been written
                for (int w = 0; w < g.subs; ++w) {
                    ok = ok && wait_warp(smem_u32(&sh.q_empty[w]), (segs[w] & 1) ^ 1, abort_flag, a.status, kChunkWaitQueries);
                    ++segs[w];
                }
                if (!ok) return;
                if (lane == 0)
                    for (int w = 0; w < g.subs; ++w) {
                        constexpr int kCopies = QUAD ? 4 : 1;  // (the quarters' warps each have rows of their own)
                        mbar_expect_tx(smem_u32(&sh.q_full[w]), kCopies * (D / 64) * walk.tokens * a.group * 128);
                        for (int b = 0; b < kCopies * (D / 64); ++b)
                            load_box(q_smem + w * C::kQBytes + b / kCopies * kQBlock + b % kCopies * (32 * 128), &maps.q, b / kCopies * 64,
                                     g.head * a.group, row0 + w * walk.tokens, smem_u32(&sh.q_full[w]));
                    }
                q_waits = false;
                for (int w = 0; w < g.subs; ++w) ++loaded[w];
            };
            auto free_queries = [&]() {
                bool yes = true;
                for (int w = 0; w < g.subs; ++w) yes = yes && mbar_test(smem_u32(&sh.q_empty[w]), (segs[w] & 1) ^ 1);
                return __all_sync(0xffffffffu, yes);
            };
            // waits for a stage to be free; K and V tiles of a segment come in ahead of its queries while those of the segment
            // before are still in use, but never wait for a stage that only their product would free
            auto free_stage = [&](int slot) {
                const uint32_t bar = smem_u32(&sh.empty[slot]), parity = (issued / C::kStages & 1) ^ 1;
                if (q_waits && (free_queries() || !__all_sync(0xffffffffu, mbar_test(bar, parity)))) queries();
                ok = ok && wait_warp(bar, parity, abort_flag, a.status, kChunkWaitStage);
                return ok;
            };
            const int* table = a.page_table + (long long)g.slot * a.table_stride;
            const int n_pages = (g.u.rows + kTile - 1) / kTile;
            int batch = 0, entry = 0;  // page-table entries batch .. batch+31, one per lane; tiles come from the last one back
            auto fetch = [&](int last) {
                batch = max(last - 31, 0);
                entry = g.full && batch + lane < n_pages ? min(max(table[batch + lane], 0), a.n_pages - 1) : 0;
            };
            if (g.t1 > g.fresh) fetch(W::key_tile(g, max(g.t0, g.fresh)) / kTile + C::kPages - 1);
            for (int t = g.t0; ok && t < g.t1; ++t) {
                if (t < g.fresh) {
                    const int token = g.start + W::key_tile(g, t);
                    for (int kv = 0; kv < 2; ++kv) {
                        const int slot = issued % C::kStages;
                        if (!free_stage(slot)) break;
                        if (lane == 0) {
                            mbar_expect_tx(smem_u32(&sh.full[slot]), C::kTileBytes);
                            for (int b = 0; b < D / 64; ++b)
                                load_box(ring + slot * C::kTileBytes + b * C::kBlock, kv ? &maps.v : &maps.k, b * 64, g.head, token,
                                         smem_u32(&sh.full[slot]));
                            if (kv && W::template unclean<FP8>(g, t)) mbar_arrive(smem_u32(&sh.dirty[slot]));
                        }
                        ++issued;
                    }
                    continue;
                }
                const int page = W::key_tile(g, t) / kTile;
                if (page < batch) fetch(page + C::kPages - 1);
                const int have = min(C::kPages, n_pages - page);  // pages of this tile
                int phys[C::kPages];
#pragma unroll
                for (int p = 0; p < C::kPages; ++p) phys[p] = __shfl_sync(0xffffffffu, entry, (page + p - batch) & 31);
                for (int kv = 0; kv < (FP8 ? 1 : 2); ++kv) {
                    const int slot = issued % C::kStages;
                    if (!free_stage(slot)) break;
                    if (lane == 0) {
                        mbar_expect_tx(smem_u32(&sh.full[slot]), have * (FP8 ? kPageBytes : kTile * D * 2));
#pragma unroll
                        for (int p = 0; p < C::kPages; ++p) {
                            if (p >= have) break;
                            if constexpr (FP8 && SUBS == 2) {  // the pages' K codes behind one another, then their V codes
                                const long long index = g.full ? a.page0_8 + (long long)g.index * a.n_pages + phys[p]
                                                               : a.ring0_8 + ((long long)g.slot * a.n_comp + g.index) * a.ring_tiles + page + p;
                                for (int v = 0; v < 2; ++v)
                                    load_page(ring + slot * C::kTileBytes + (2 * v + p) * (kPageBytes / 2), &maps.pool, (int)(index * 128) + v * 64,
                                              smem_u32(&sh.full[slot]));
                            } else if constexpr (FP8) {
                                const long long index = g.full ? a.page0_8 + (long long)g.index * a.n_pages + phys[p]
                                                               : a.ring0_8 + ((long long)g.slot * a.n_comp + g.index) * a.ring_tiles + page + p;
                                load_page(ring + slot * C::kTileBytes + p * kPageBytes, &maps.pool, (int)(index * 128), smem_u32(&sh.full[slot]));
                            } else {
                                const long long r = g.full ? a.full_row0 + (((long long)g.index * a.n_pages + phys[p]) * 2 + kv) * kTile
                                                           : a.comp_row0 + (((long long)g.slot * a.n_comp + g.index) * 2 + kv) * a.rows_comp +
                                                                 (page + p) * kTile;
                                for (int b = 0; b < D / 64; ++b)
                                    load_box(ring + slot * C::kTileBytes + b * C::kBlock + p * kTile * 128, &maps.pool, b * 64, 0, (int)r,
                                             smem_u32(&sh.full[slot]));
                            }
                        }
                        if (kv && W::template unclean<FP8>(g, t)) mbar_arrive(smem_u32(&sh.dirty[slot]));
                    }
                    ++issued;
                }
            }
            if (ok && q_waits) queries();
        }
        if (!ok || *abort_flag) {  // nothing of this CTA's copies may be in flight when it ends
            for (int w = 0; w < SUBS; ++w)
                if (loaded[w] > 0) wait_warp(smem_u32(&sh.q_full[w]), (loaded[w] - 1) & 1, nullptr, a.status, kChunkWaitDrain);
            for (int i = max(0, issued - C::kStages); i < issued; ++i)
                wait_warp(smem_u32(&sh.full[i % C::kStages]), i / C::kStages & 1, nullptr, a.status, kChunkWaitDrain);
        }
    } else if (warp == kMma) {
        // ------------------------------------------------------------------ matrix products
        W walk(a);
        Segment g;
        constexpr uint32_t kQK = instr_desc(kRows, KEYS, false), kPV = instr_desc(kRows, D, true), kPVt = instr_desc(kRows, D, false) & ~(1u << 7 | 1u << 10);  // (fp16)
        constexpr uint32_t kQK8 = instr_desc8(kRows, KEYS, false), kQK8Wide = instr_desc8(kRows, KEYS, true);
        int used[2] = {0, 0};               // P tiles multiplied so far (SUBS 1: used[0])
        int base = 0, dbase = 0;            // stages and decoded tiles so far
        int segs[2] = {0, 0}, split[2] = {0, 0};  // segments of each sub-tile, those whose queries were split
        uint32_t cleaned = 0;               // phase of each stage's `clean`
        bool ok = true;
        while (ok && walk.next(g)) {
            const int n = g.t1 - g.t0, c = FP8 ? max(0, min(g.t1, g.fresh) - g.t0) : n;  // tiles, and those that take two stages
            // the stage of tile j's K rows (of an 8-bit cache, of its codes) and, of the chunk or a 16-bit cache, of its V rows
            auto k_stage = [&](int j) { return base + (j < c ? 2 * j : c + j); };
            auto k_loaded = [&](int j) {
                const int i = k_stage(j);
                return wait_warp(smem_u32(&sh.full[i % C::kStages]), i / C::kStages & 1, abort_flag, a.status, kChunkWaitLoad);
            };
            auto v_loaded = [&](int j) {
                if (FP8 && j >= c) {
                    const int i = dbase + j - c;
                    return wait_warp(smem_u32(&sh.decoded[i & 1]), i >> 1 & 1, abort_flag, a.status, kChunkWaitDecoded);
                }
                const int i = k_stage(j) + 1, slot = i % C::kStages;
                if (!wait_warp(smem_u32(&sh.full[slot]), i / C::kStages & 1, abort_flag, a.status, kChunkWaitLoad)) return false;
                if (W::template unclean<FP8>(g, g.t0 + j)) {
                    if (!wait_warp(smem_u32(&sh.clean[slot]), cleaned >> slot & 1, abort_flag, a.status, kChunkWaitLoad)) return false;
                    cleaned ^= 1u << slot;
                }
                return true;
            };
            auto signal = [&](uint64_t* bar) {
                if (elect_one()) commit(smem_u32(bar));
            };
            auto k_done = [&](int j) { signal(&sh.empty[k_stage(j) % C::kStages]); };
            auto v_done = [&](int j) { signal(FP8 && j >= c ? &sh.decoded_empty[(dbase + j - c) & 1] : &sh.empty[(k_stage(j) + 1) % C::kStages]); };
            // S of tile j; the first cached tile of an 8-bit cache waits for the queries' split
            auto scores = [&](int w, int place, int j) {
                if (FP8 && j == c) {
                    if (!wait_warp(smem_u32(&sh.q_split[w]), split[w] & 1, abort_flag, a.status, kChunkWaitQueries)) return false;
                    ++split[w];
                }
                const uint32_t to = tmem + place * KEYS, at = ring + k_stage(j) % C::kStages * C::kTileBytes;
                const uint64_t q = smem_desc(q_smem + w * C::kQBytes), k = smem_desc(at);
                fence_after();
                if (FP8 && j >= c) {
                    if (elect_one()) {
#pragma unroll
                        for (int x = 0; x < 8; ++x)  // the queries' first and second parts
                            mma_ss8(to, q + ((x / 4 * kQBlock + x % 4 * 32) >> 4), k + (x % 4 * 32 >> 4), x < 4 ? kQK8 : kQK8Wide, x > 0);
                        commit(smem_u32(&sh.s_full[place]));
                    }
                } else if (elect_one()) {
#pragma unroll
                    for (int x = 0; x < D / 16; ++x)
                        mma_ss(to, q + ((x / 4 * kQBlock + x % 4 * 32) >> 4), k + ((x / 4 * C::kBlock + x % 4 * 32) >> 4), kQK, x > 0);
                    commit(smem_u32(&sh.s_full[place]));
                }
                return true;
            };
            // the products of one half (64 keys) of tile j's P
            auto values = [&](int w, int place, int j, int half) {
                fence_after();
                const uint32_t d = tmem + o_column + w * D, p = tmem + place * KEYS + half * 32;
                if (FP8 && j >= c) {  // V^T: rows of 64 tokens
                    const uint64_t v = smem_desc(decoded + ((dbase + j - c) & 1) * C::kTileBytes + half * (D * 128));
                    if (elect_one()) {
#pragma unroll
                        for (int x = 0; x < 4; ++x) mma_ts(d, p + x * 8, v + (x * 32 >> 4), kPVt, j > 0 || half > 0 || x > 0);
                    }
                } else {
                    const uint64_t v = smem_desc(ring + (k_stage(j) + 1) % C::kStages * C::kTileBytes + half * (64 * 128), C::kBlock);
                    if (elect_one()) {
#pragma unroll
                        for (int x = 0; x < 4; ++x) mma_ts(d, p + x * 8, v + (x * 2048 >> 4), kPV, j > 0 || half > 0 || x > 0);
                    }
                }
            };
            for (int w = 0; ok && w < g.subs; ++w)
                ok = wait_warp(smem_u32(&sh.q_full[w]), segs[w]++ & 1, abort_flag, a.status, kChunkWaitQueries);
            ok = ok && k_loaded(0);
            if (!ok) break;
            if (SUBS == 1) {
                ok = scores(0, used[0] & 1, 0);
                if (ok) k_done(0);
                for (int j = 0; ok && j < n; ++j) {
                    const int place = used[0] & 1;
                    if (j + 1 < n) {
                        ok = k_loaded(j + 1) && scores(0, place ^ 1, j + 1);
                        if (!ok) break;
                        k_done(j + 1);
                    }
                    ok = wait_warp(smem_u32(&sh.p_full[place][0]), used[0] >> 1 & 1, abort_flag, a.status, kChunkWaitSoftmax) && v_loaded(j);
                    if (!ok) break;
                    values(0, place, j, 0);
                    signal(&sh.pv_done[place]);
                    v_done(j);
                    ++used[0];
                }
            } else {
                for (int w = 0; ok && w < g.subs; ++w) ok = scores(w, w, 0);
                if (ok) k_done(0);
                for (int j = 0; ok && j < n; ++j) {
                    ok = v_loaded(j);
                    if (ok && j + 1 < n) ok = k_loaded(j + 1);
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
                        if (w == SUBS - 1) v_done(j);
                        if (j + 1 < n && w < g.subs) ok = scores(w, w, j + 1);
                    }
                    if (ok && j + 1 < n) k_done(j + 1);
                }
            }
            base += c + n;
            dbase += n - c;
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
            const int n = g.t1 - g.t0, c = FP8 ? max(0, min(g.t1, g.fresh) - g.t0) : n;
            for (int j = 0; ok && j < c; ++j) {
                if (!W::template unclean<FP8>(g, g.t0 + j)) continue;
                const int i = base + 2 * j + 1, slot = i % C::kStages;
                ok = wait_warp(smem_u32(&sh.dirty[slot]), told >> slot & 1, abort_flag, a.status, kChunkWaitLoad) &&
                     wait_warp(smem_u32(&sh.full[slot]), i / C::kStages & 1, abort_flag, a.status, kChunkWaitLoad);
                if (!ok) break;
                told ^= 1u << slot;
                uint8_t* x = smem + SUBS * C::kQBytes + slot * C::kTileBytes;
                for (int y = W::valid_rows(g, g.t0 + j) * 8 + lane; y < KEYS * 8; y += 32)
                    for (int b = 0; b < D / 64; ++b) *reinterpret_cast<uint4*>(x + b * C::kBlock + y * 16) = make_uint4(0, 0, 0, 0);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh.clean[slot]));
            }
            base += c + n;
        }
    } else if (FP8 && warp >= kDecode) {
        // ------------------------------------------------------------------ V codes to fp16
        W walk(a);
        Segment g;
        const int ct = (warp - kDecode) * 32 + lane;
        // a thread's pieces, sixteen tokens of an element, lie 16 rows of 128 bytes apart, which hold two elements each; decoded, an
        // element's 64 tokens are a row
        const int r = ct >> 3, c = ct & 7, e = r * 2 + (c >> 2), ch = (c & 3) * 2;
        const int piece = r * 128 + ((c ^ (r & 7)) << 4), to_lo = e * 128 + ((ch ^ (e & 7)) << 4), to_hi = e * 128 + (((ch + 1) ^ (e & 7)) << 4);
        int i = 0, d = 0;  // stages and decoded tiles so far
        bool ok = true;
        while (ok && walk.next(g)) {
            for (int t = g.t0; ok && t < g.t1; ++t) {
                if (t < g.fresh) {  // rows of the chunk: nothing to decode (a stage is free when these warps have let it go, too)
                    for (int kv = 0; ok && kv < 2; ++kv, ++i) {
                        ok = wait_warp(smem_u32(&sh.full[i % C::kStages]), i / C::kStages & 1, abort_flag, a.status, kChunkWaitLoad);
                        if (ok && lane == 0) mbar_arrive(smem_u32(&sh.empty[i % C::kStages]));
                    }
                    continue;
                }
                const int slot = i % C::kStages;
                ok = wait_warp(smem_u32(&sh.full[slot]), i / C::kStages & 1, abort_flag, a.status, kChunkWaitLoad) &&
                     wait_warp(smem_u32(&sh.decoded_empty[d & 1]), (d >> 1 & 1) ^ 1, abort_flag, a.status, kChunkWaitDecoded);
                if (!ok) break;
                const uint8_t* from = smem + SUBS * C::kQBytes + slot * C::kTileBytes + C::kPages * (kPageBytes / 2);
                uint8_t* to = smem + SUBS * C::kQBytes + (C::kStages + (d & 1)) * C::kTileBytes;
#pragma unroll 1
                for (int p = 0; p < C::kPages; ++p) {
                    const int left = W::valid_rows(g, t) - p * kTile;  // tokens from here on (64 or more: the page is full)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        uint4 lo, hi, codes = make_uint4(0, 0, 0, 0);
                        if (left > 0) codes = *reinterpret_cast<const uint4*>(from + p * (kPageBytes / 2) + x * (16 * 128) + piece);
                        if (left < kTile) {  // (0 * NaN of what lies behind the last token would be NaN)
                            const int n = left - (c & 3) * 16;
                            codes.x &= first_bytes(n);
                            codes.y &= first_bytes(n - 4);
                            codes.z &= first_bytes(n - 8);
                            codes.w &= first_bytes(n - 12);
                        }
                        decode16(codes, lo, hi);
                        uint8_t* row = to + p * (128 * 128) + x * (32 * 128);
                        *reinterpret_cast<uint4*>(row + to_lo) = lo;
                        *reinterpret_cast<uint4*>(row + to_hi) = hi;
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(smem_u32(&sh.decoded[d & 1]));
                    mbar_arrive(smem_u32(&sh.empty[slot]));
                }
                ++i;
                ++d;
            }
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

// Adds up the pieces of the units that a boundary cuts.  Block (c - 1, 32 rows, columns): the unit that CTA c's range begins
// inside of, if it is the first to.  A warp's lanes hold 32 rows' columns, a run of RUN; a block's eight warps take RUNS such runs,
// and of each run every 8 / RUNS-th piece, and meet in shared memory: all columns where units are cut once or twice, eight columns
// and 32 pieces at a time where few units are cut into many (five drafted tokens on 8192: 49 pieces of 8 units).  The pieces'
// order is that of the keys, whatever CTA ran first.
template <int D, int SHAPE, int RUN, int RUNS>
__global__ void __launch_bounds__(256) chunk_combine_kernel(const __grid_constant__ ChunkArgs a)
{
    constexpr int kPieces = 8 / RUNS, kAtOnce = 32 / RUN, kRecordRows = SHAPE == 0 ? 32 : kRows;
    __shared__ float part[8][32][RUN + 1], top[8][32], sum[8][32];
    const int c = blockIdx.x + 1;
    const ChunkPos b = a.at[c], before = a.at[c - 1];
    if (b.tile == 0 || b.seq >= a.seqs.n || (same_unit(before, b) && before.tile > 0)) return;
    const int tokens = kRecordRows / a.group, w = blockIdx.y / 4, row0 = blockIdx.y % 4 * 32;
    const int start = a.seqs.start[b.seq], m = a.seqs.count[b.seq];
    const int from = (b.row_tile * (SHAPE == 2 ? 2 : 1) + w) * tokens;
    if (row0 / a.group >= tokens || from + row0 / a.group >= m) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int last = c;  // the pieces are those of CTAs c - 1 .. last
    while (last + 1 < a.ctas && same_unit(a.at[last + 1], b)) ++last;
    grid_dep_wait();
    float o[RUN], mx = -INFINITY, l = 0.f;
#pragma unroll
    for (int x = 0; x < RUN; ++x) o[x] = 0.f;
    for (int k0 = c - 1 + warp / RUNS; k0 <= last; k0 += kPieces * kAtOnce) {
        float pm[kAtOnce], pl[kAtOnce];
        float4 y[kAtOnce][RUN / 4];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int k = k0 + u * kPieces;
            pm[u] = -INFINITY;
            pl[u] = 0.f;
            if (k > last) continue;
            const int slot = k > c - 1 || same_unit(before, b) ? 2 * k : 2 * k + 1;
            const float* rec = a.records + (long long)slot * chunk_record_floats(D, SHAPE) + (long long)w * kRows * (D + 2);
            pm[u] = rec[D * kRecordRows + row0 + lane];
            pl[u] = rec[(D + 1) * kRecordRows + row0 + lane];
#pragma unroll
            for (int x = 0; x < RUN / 4; ++x)
                y[u][x] = reinterpret_cast<const float4*>(rec)[((blockIdx.z * RUNS + warp % RUNS) * (RUN / 4) + x) * kRecordRows + row0 + lane];
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (pm[u] == -INFINITY && pl[u] == 0.f) continue;  // the row sees none of the piece's keys (of NaN scores, the sum is NaN)
            const float to = fmaxf(mx, pm[u]), old = mx == -INFINITY ? 0.f : ex2(mx - to), f = ex2(pm[u] - to);
            mx = to;
            l = l * old + pl[u] * f;
#pragma unroll
            for (int x = 0; x < RUN / 4; ++x) {
                o[4 * x] = o[4 * x] * old + y[u][x].x * f;
                o[4 * x + 1] = o[4 * x + 1] * old + y[u][x].y * f;
                o[4 * x + 2] = o[4 * x + 2] * old + y[u][x].z * f;
                o[4 * x + 3] = o[4 * x + 3] * old + y[u][x].w * f;
            }
        }
    }
    top[warp][lane] = mx;
    sum[warp][lane] = l;
#pragma unroll
    for (int x = 0; x < RUN; ++x) part[warp][lane][x] = o[x];
    __syncthreads();
    // RUN / 4 threads a row, four columns of each run
    const int r = threadIdx.x / (RUN / 4), x0 = threadIdx.x % (RUN / 4) * 4, in_tile = (row0 + r) / a.group, i = from + in_tile;
    if (r >= 32 || in_tile >= tokens || i >= m) return;
    float all = -INFINITY, total = 0.f, f[kPieces];
#pragma unroll
    for (int k = 0; k < kPieces; ++k) all = fmaxf(all, top[k * RUNS][r]);
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
        const float t = top[k * RUNS][r];
        f[k] = t == -INFINITY ? 0.f : ex2(t - all);
        total += sum[k * RUNS][r] * f[k];
    }
    const float inv = 1.f / total;
    const int head = a.head_of_slot[b.head] * a.group + (row0 + r) % a.group;
    const long long at_head = (long long)(start + i) * a.q_heads + head;
#pragma unroll
    for (int run = 0; run < RUNS; ++run) {
        float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
#pragma unroll
            for (int x = 0; x < 4; ++x) y[x] += part[k * RUNS + run][r][x0 + x] * f[k];
        *reinterpret_cast<uint2*>(a.out + at_head * D + (blockIdx.z * RUNS + run) * RUN + x0) =
            make_uint2(bf16x2(y[0] * inv, y[1] * inv), bf16x2(y[2] * inv, y[3] * inv));
    }
    if (a.lse && blockIdx.z == 0 && x0 == 0) a.lse[at_head] = (all + log2f(total)) * kLn2;
}

template <int D, int SHAPE, bool FP8>
cudaError_t launch_shape(const ChunkArgs& a, const ChunkMaps& m, int pieces, cudaStream_t stream)
{
    using C = Chunk<D, SHAPE, FP8>;
    auto kernel = a.softcap != 0.f ? (a.slopes ? chunk_attention_kernel<D, SHAPE, FP8, true, true> : chunk_attention_kernel<D, SHAPE, FP8, true, false>)
                                   : (a.slopes ? chunk_attention_kernel<D, SHAPE, FP8, false, true> : chunk_attention_kernel<D, SHAPE, FP8, false, false>);
    kernel<<<a.ctas, C::kThreads, C::kSmem, stream>>>(a, m);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || pieces < 2) return e;
    const bool few = pieces <= (SHAPE == 0 ? 4 : 16);  // (128 rows of a unit are four times the blocks: 512 tokens on 3400, five pieces, 54 -> 36 us)
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(a.ctas - 1, SHAPE == 0 ? 1 : SHAPE * 4, few ? 1 : D / 8);
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return few ? cudaLaunchKernelEx(&cfg, chunk_combine_kernel<D, SHAPE, 32, D / 32>, a)
               : cudaLaunchKernelEx(&cfg, chunk_combine_kernel<D, SHAPE, 8, 1>, a);
}

template <int D, int SHAPE, bool FP8>
cudaError_t prepare_shape()
{
    const void* kernels[] = {(const void*)chunk_attention_kernel<D, SHAPE, FP8, false, false>, (const void*)chunk_attention_kernel<D, SHAPE, FP8, false, true>,
                             (const void*)chunk_attention_kernel<D, SHAPE, FP8, true, false>, (const void*)chunk_attention_kernel<D, SHAPE, FP8, true, true>};
    for (const void* k : kernels) {
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, Chunk<D, SHAPE, FP8>::kSmem);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <int D, bool FP8>
cudaError_t launch_dim(const ChunkArgs& a, const ChunkMaps& m, int shape, int pieces, cudaStream_t stream)
{
    return shape == 2 ? launch_shape<D, 2, FP8>(a, m, pieces, stream)
                      : shape == 1 ? launch_shape<D, 1, FP8>(a, m, pieces, stream) : launch_shape<D, 0, FP8>(a, m, pieces, stream);
}

template <int D, bool FP8>
cudaError_t prepare_dim()
{
    cudaError_t e = prepare_shape<D, 0, FP8>();
    if (e == cudaSuccess) e = prepare_shape<D, 1, FP8>();
    return e == cudaSuccess ? prepare_shape<D, 2, FP8>() : e;
}

}  // namespace

cudaError_t launch_chunk_attention(const ChunkArgs& a, const ChunkMaps& m, int head_dim, int shape, int pieces, cudaStream_t stream)
{
    return a.pool8 ? launch_dim<128, true>(a, m, shape, pieces, stream)
                   : head_dim == 128 ? launch_dim<128, false>(a, m, shape, pieces, stream) : launch_dim<64, false>(a, m, shape, pieces, stream);
}

cudaError_t prepare_chunk_kernels(int head_dim, bool fp8)
{
    return fp8 ? prepare_dim<128, true>() : head_dim == 128 ? prepare_dim<128, false>() : prepare_dim<64, false>();
}

}  // namespace rlkv
