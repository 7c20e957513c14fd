// The backward pass of prompt attention on the tensor cores, in three launches without atomics:
//
//   stats   D_i = sum over head_dim of dout * out, stored with lse (log2 domain) per head and query
//   rows    one CTA per 256 query rows (two heads, or one): over their keys, S = Q.K^T and dP = dO.V^T, then dQ += dS.K.
//           It also corrects D: out was rounded to bf16, and sum_j P (dP - D) is what that changed
//   keys    one CTA (or one per part of the query heads, in a cluster that adds them up) per 128 keys of a KV head: over
//           the queries that see them, S^T = K.Q^T and dP^T = V.dO^T, then dV += P^T.dO and dK += dS^T.Q
//
// S and dP are computed twice, seven products where five would do, and in return every gradient is summed by one CTA
// in a fixed order: no atomics on dQ, no fp32 copy of it in memory, the same bits on every run.  P and dS are written
// to tensor memory as bf16 over S and dP and are the A operand of the second products straight from there.
//
// Measured (32 / 8 heads of 128, causal, 8192 tokens, in bursts): stats 26 us (DRAM), rows 700 us, keys 810 us; 0.9 PFLOP/s of the
// five products, 1.25 of the seven that run.  With the forward pass 1985 us in bursts and 2220 to 2320 over a run of passes, under
// the power cap.  What bounds it: in `keys` the exponential unit (64 scores a thread, eight warps at
// once: 1024 cycles of the 1180 that P takes) in the chain S - P - dV - S of 2900 cycles beside 2048 of products; in `rows`
// the same unit and the hand-overs between threads and products.
#include "rlkv_prompt.cuh"
#include "tcgen05.cuh"

namespace rlkv {
namespace {

using namespace tc;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kTok = 128;            // tokens of a tile, of queries and of keys
constexpr int kBlock = kTok * 128;  // bytes of a block of 64 elements of its rows
constexpr int kThreads = 384;
constexpr int kFewKeys = 1024;

// ---- D and lse ---------------------------------------------------------------------------------------

// One warp per head and eight queries, half a warp per row, all loads at once.  Stored head by head, so that the keys
// kernel reads consecutive queries.  A query that sees nothing gets lse = +infinity: its P is then exp2(s - infinity) = 0.
template <int D>
__global__ void __launch_bounds__(256) prompt_stats_kernel(const __grid_constant__ PromptArgs a)
{
    constexpr int E = D / 16, kTokens = 8;  // elements of a lane, queries of a warp
    const int lane = threadIdx.x & 31, half = lane >> 4, l16 = lane & 15;
    const int h = blockIdx.y * 8 + (threadIdx.x >> 5);
    grid_dep_launch();
    if (h >= a.q_heads) return;
    const int t0 = blockIdx.x * kTokens;
    float sum[kTokens / 2];
#pragma unroll
    for (int i = 0; i < kTokens / 2; ++i) {
        const int t = t0 + 2 * i + half;
        sum[i] = 0.f;
        if (t < a.q_tokens) {
            const long long at = ((long long)t * a.q_heads + h) * D + l16 * E;
            __nv_bfloat162 x[E / 2], y[E / 2];
            if (E == 8) {
                *reinterpret_cast<uint4*>(x) = *reinterpret_cast<const uint4*>(a.out + at);
                *reinterpret_cast<uint4*>(y) = *reinterpret_cast<const uint4*>(a.dout + at);
            } else {
                *reinterpret_cast<uint2*>(x) = *reinterpret_cast<const uint2*>(a.out + at);
                *reinterpret_cast<uint2*>(y) = *reinterpret_cast<const uint2*>(a.dout + at);
            }
#pragma unroll
            for (int e = 0; e < E / 2; ++e) {
                const float2 u = __bfloat1622float2(x[e]), w = __bfloat1622float2(y[e]);
                sum[i] = fmaf(u.x, w.x, sum[i]);
                sum[i] = fmaf(u.y, w.y, sum[i]);
            }
        }
    }
    const int t = t0 + lane;
    const float lse = lane < kTokens && t < a.q_tokens ? a.lse[(long long)t * a.q_heads + h] : 0.f;
    float mine = 0.f;
#pragma unroll
    for (int i = 0; i < kTokens / 2; ++i) {
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
        const float x = __shfl_sync(0xffffffffu, sum[i], lane & 1 ? 16 : 0);
        if (lane / 2 == i) mine = x;
    }
    if (lane < kTokens && t < a.q_tokens)
        a.stats[(long long)h * a.q_tokens + t] = make_float2(lse == -INFINITY ? INFINITY : lse * kLog2e, mine);
}

// ---- what both kernels do with a score ------------------------------------------------------------------

// N products q.k -> scores in the log2 domain over `factor` (with neither cap nor bias the products are left as they
// are, the factor is applied with the exponent), and (CAP) the slopes of the cap, 1 - tanh^2.  `dist0`: distance of the
// first score, `step`: +1 or -1 from one to the next.
template <bool CAP, bool BIAS, int N>
__device__ __forceinline__ void finish_scores(const Cap& cap, float sl2, float slope2, int dist0, int step, bool vote, float (&s)[N], float (&f)[CAP ? N : 1])
{
    if constexpr (CAP) {
        cap.apply(s, vote);
        const float2 k = make_float2(-1.f / (cap.cap2 * cap.cap2), -1.f / (cap.cap2 * cap.cap2));
#pragma unroll
        for (int c = 0; c < N; c += 2) {
            const float2 x = make_float2(s[c], s[c + 1]), y = fma2(mul2(x, x), k, make_float2(1.f, 1.f));
            f[c] = y.x;
            f[c + 1] = y.y;
        }
    }
    if constexpr (BIAS) {
#pragma unroll
        for (int c = 0; c < N; ++c) s[c] = fmaf(-slope2, fabsf((float)dist0 + (float)(step * c)), CAP ? s[c] : s[c] * sl2);
    }
}

// A tile of 128 tokens of one head from token `token` on: D / 64 blocks of [128 rows][128 bytes].
template <int D>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, int head, int token, uint32_t bar)
{
    for (int b = 0; b < D / 64; ++b) load_box(dst + b * kBlock, map, b * 64, head, token, bar);
}

// Zeros over rows `from` .. 127 of BLOCKS blocks; visible to the products of whoever the caller tells afterwards.
template <int BLOCKS>
__device__ __forceinline__ void clear_rows(uint8_t* tile, int from, int lane)
{
    for (int i = from * 8 + lane; i < kTok * 8; i += 32)
        for (int b = 0; b < BLOCKS; ++b) *reinterpret_cast<uint4*>(tile + b * kBlock + i * 16) = make_uint4(0, 0, 0, 0);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

__device__ __forceinline__ void signal(uint64_t* bar)
{
    if (elect_one()) commit(smem_u32(bar));
}
// d (128 x 128) = A.B^T of two tiles, over head_dim; `bar` is told when it is done.
template <int D>
__device__ __forceinline__ void scores(uint32_t d, uint32_t a_smem, uint32_t b_smem, uint64_t* bar)
{
    const uint64_t x = smem_desc(a_smem), y = smem_desc(b_smem);
    if (elect_one()) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            const uint32_t off = (i / 4 * kBlock + i % 4 * 32) >> 4;
            mma_ss(d, x + off, y + off, instr_desc(kTok, kTok, false), i > 0);
        }
        commit(smem_u32(bar));
    }
}
// d (128 x D) += A.B over 64 tokens: two runs of 32, 64 tokens apart in the tile B and `apart` columns in A, which is bf16 in
// tensor memory.
template <int D>
__device__ __forceinline__ void gradient_half(uint32_t d, uint32_t a_tmem, int apart, uint32_t b_smem, bool add)
{
    const uint64_t y = smem_desc(b_smem, kBlock);
    if (elect_one()) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            mma_ts(d, a_tmem + i / 2 * apart + i % 2 * 8, y + ((i / 2 * 64 + i % 2 * 16) * 128 >> 4), instr_desc(kTok, D, true), add || i > 0);
    }
}
// d (128 x D) += A.B over a tile's 128 tokens, A in 32-token blocks 32 columns apart: 16 columns of rounded values and, `in_two`, 16 more of what the
// rounding left.
template <int D>
__device__ __forceinline__ void gradient_blocks(uint32_t d, uint32_t a_tmem, uint32_t b_smem, bool in_two, bool add)
{
    const uint64_t y = smem_desc(b_smem, kBlock);
    if (elect_one()) {
#pragma unroll
        for (int i = 0; i < kTok / 16; ++i)
            mma_ts(d, a_tmem + i / 2 * 32 + i % 2 * 8, y + (i * 2048 >> 4), instr_desc(kTok, D, true), add || i > 0);
        if (in_two) {
#pragma unroll 1  // (unrolled too, the descriptors of both loops would not fit this warp's registers)
            for (int i = 0; i < kTok / 16; ++i) mma_ts(d, a_tmem + i / 2 * 32 + i % 2 * 8 + 16, y + (i * 2048 >> 4), instr_desc(kTok, D, true), true);
        }
    }
}

// ---- dK and dV ------------------------------------------------------------------------------------------
//
// One tile of 128 queries at a time, both warpgroups on it (64 columns each).  The products of a tile are issued as
//   dV(n) += P.dO | S(n+1) | dK(n) += dS.Q | dP(n+1)
// so that one of them always runs beside the arithmetic on P and dS: S(n+1) may overwrite P(n) once dV(n) has read it,
// dP(n+1) overwrites dS(n) after dK(n).  (Tiles of 64 queries, two in flight, left the tensor core waiting for shared
// memory: with N = 64 a product reads 6 KB of operands per 32 cycles, where 128 bytes per cycle is what there is.)

template <int D>
struct Keys {
    static constexpr int kTile = kTok * D * 2;
    static constexpr int kStages = D == 128 ? 2 : 4;  // Q and dO tiles
    static constexpr int kStats = (2 + 2 * kStages) * kTile;
    static constexpr int kSmem = kStats + kStages * kTok * 8 + 1024;
};

struct KeysShared {
    uint64_t kv_full, full[4], empty[4], ready[4], s_full, p_full[2], dp_full, ds_full, done, drain;
    uint32_t tmem;
    int abort, valid;
    int k0, rows, j0, q0, qn, off, prefix, u0, n_u;  // the CTA's keys; first query tile that sees them, and how many
};

template <int D, bool CAP, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1)
prompt_keys_kernel(const __grid_constant__ PromptArgs a, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do, const int split)
{
    using F = Keys<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    float* stats = reinterpret_cast<float*>(smem + F::kStats);  // per stage: -lse of 128 queries, then their -D
    static_assert(sizeof(KeysShared) <= 1024 && F::kSmem <= kMaxDynamicSmem, "shared memory");
    KeysShared& sh = *reinterpret_cast<KeysShared*>(smem + F::kStats + F::kStages * kTok * 8);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    // `split` CTAs, a cluster, share the query heads of a KV head
    const int rank = blockIdx.x % split, block = blockIdx.x / split, kv_head = block % a.kv_heads;
    const int heads = a.group / split, head0 = kv_head * a.group + rank * heads;
    const bool full_head = a.full[kv_head] != 0;
    volatile int* abort_flag = &sh.abort;

    if ((smem_u32(smem) & 1023u) != 0) {
        if (tid == 0) atomicCAS(a.status, 0, kPromptSmemMisaligned);
        return;
    }
    if (warp == 0) {
        int tile = 0;
        DocRange r;
        const bool valid = find_tile(a, true, kTok, block / a.kv_heads, r, tile);
        if (lane == 0) {
            sh.valid = valid;
            if (valid) {
                tile = (r.kn + kTok - 1) / kTok - 1 - tile;  // a document's first keys are seen by the most queries
                const int j0 = tile * kTok, j1 = min(j0 + kTok, r.kn), off = r.kn - r.qn;
                sh.k0 = r.k0 + j0;
                sh.rows = j1 - j0;
                sh.j0 = j0;
                sh.q0 = r.q0;
                sh.qn = r.qn;
                sh.off = off;
                sh.prefix = r.prefix;
                // queries lower .. upper-1 see some key of the tile
                const int lower = j0 < r.prefix ? 0 : max(0, j0 - off);
                const int upper = full_head || j0 < a.sink ? r.qn : min(r.qn, j1 - 1 + a.window - off);
                sh.u0 = lower / kTok;
                sh.n_u = upper > lower ? (upper + kTok - 1) / kTok - sh.u0 : 0;
            }
        }
    } else if (warp == 8) {
        if (lane == 0) {
            prefetch_map(&map_q);
            prefetch_map(&map_k);
            prefetch_map(&map_v);
            prefetch_map(&map_do);
            sh.abort = 0;
            mbar_init(smem_u32(&sh.kv_full), 1);
            for (int i = 0; i < F::kStages; ++i) {
                mbar_init(smem_u32(&sh.full[i]), 1);
                mbar_init(smem_u32(&sh.empty[i]), 1);
                mbar_init(smem_u32(&sh.ready[i]), 1);
            }
            mbar_init(smem_u32(&sh.s_full), 1);
            mbar_init(smem_u32(&sh.p_full[0]), 8);
            mbar_init(smem_u32(&sh.p_full[1]), 8);
            mbar_init(smem_u32(&sh.dp_full), 1);
            mbar_init(smem_u32(&sh.ds_full), 8);
            mbar_init(smem_u32(&sh.done), 1);
            mbar_init(smem_u32(&sh.drain), 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
    } else if (warp == 9) {
        tmem_alloc(smem_u32(&sh.tmem), 512);
        fence_before();
    }
    __syncthreads();
    fence_after();
    const uint32_t tmem = sh.tmem;
    grid_dep_wait();  // the rows kernel's D
    if (!sh.valid) {
        if (warp == 9) tmem_free(tmem, 512);
        return;
    }
    const uint32_t dP = tmem + kTok, dV = tmem + 256, dK = tmem + 256 + D;  // S at column 0
    const uint32_t k_smem = smem_u32(smem), v_smem = k_smem + F::kTile, ring = v_smem + F::kTile;
    const int n_u = sh.n_u, steps = n_u * heads;  // step n: query tile u0 + n % n_u of query head head0 + n / n_u

    if (warp < 8) {
        // ------------------------------------------------------------------ P and dS, one thread per key and 64 queries
        const int w = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, mine_s = tmem + lanes + w * 64, mine_dp = dP + lanes + w * 64;
        const int j = sh.j0 + row, j_last = sh.j0 + sh.rows - 1;
        const bool mine = row < sh.rows;
        // the key is seen from positions lo .. hi-1
        const int lo = j < sh.prefix ? INT_MIN / 2 : j, hi = full_head || j < a.sink ? INT_MAX / 2 : j + a.window;
        const Cap cap(CAP ? a.softcap : 1.f, a.scale);
        const float sl2 = a.scale * kLog2e;
        bool ok = true;
        int g = 0, u = 0;  // of step n
        for (int n = 0; n < steps; ++n) {
            const int st = n % F::kStages;
            ok = wait(smem_u32(&sh.ready[st]), n / F::kStages & 1, abort_flag, a.status, kPromptWaitLoad) &&
                 wait(smem_u32(&sh.s_full), n & 1, abort_flag, a.status, kPromptWaitProduct);
            if (!ok) break;
            fence_after();
            const float4* minus_lse = reinterpret_cast<const float4*>(stats + st * 2 * kTok + w * 64);
            const float4* minus_d = minus_lse + kTok / 4;
            const int p0 = (sh.u0 + u) * kTok + sh.off + w * 64;  // position of this thread's first query
            const bool plain = (p0 >= j_last || j_last < sh.prefix) && (full_head || j_last < a.sink || p0 + 63 < sh.j0 + a.window);
            const float slope2 = BIAS ? a.slopes[head0 + g] * kLog2e : 0.f;
            float s[64], f[CAP ? 64 : 1];
            tmem_ld32(mine_s, s);
            tmem_ld32(mine_s + 32, s + 32);
            wait_ld();
#pragma unroll
            for (int c = 0; c < 64; ++c) asm volatile("" : "+f"(s[c]));  // nothing of it is used before the wait
            finish_scores<CAP, BIAS>(cap, sl2, slope2, p0 - j, 1, mine, s, f);
            const float2 factor = CAP || BIAS ? make_float2(1.f, 1.f) : make_float2(sl2, sl2);
            // 32 queries at a time, so that dV starts on the first
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float* p = s + h * 32;
#pragma unroll
                for (int c = 0; c < 32; c += 4) {
                    const float4 x = minus_lse[h * 8 + c / 4];
                    const float2 y = fma2(make_float2(p[c], p[c + 1]), factor, make_float2(x.x, x.y));
                    const float2 z = fma2(make_float2(p[c + 2], p[c + 3]), factor, make_float2(x.z, x.w));
                    p[c] = ex2(y.x);
                    p[c + 1] = ex2(y.y);
                    p[c + 2] = ex2(z.x);
                    p[c + 3] = ex2(z.y);
                }
                if (!plain) {
                    const uint32_t see = range_bits(lo - p0 - h * 32, hi - p0 - h * 32);
#pragma unroll
                    for (int c = 0; c < 32; ++c) p[c] = see >> c & 1 ? p[c] : 0.f;
                }
                uint32_t packed[16];
#pragma unroll
                for (int c = 0; c < 16; ++c) packed[c] = bf16x2(p[2 * c], p[2 * c + 1]);
                tmem_st16(mine_s + h * 16, packed);  // (over this warpgroup's own columns of S)
                wait_st();
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh.p_full[h]));
            }
            ok = wait(smem_u32(&sh.dp_full), n & 1, abort_flag, a.status, kPromptWaitProduct);
            if (!ok) break;
            fence_after();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float d[32];
                tmem_read32(mine_dp + h * 32, d);
                uint32_t packed[16];
#pragma unroll
                for (int c = 0; c < 32; c += 4) {
                    const float4 x = minus_d[h * 8 + c / 4];
                    const int e = h * 32 + c;
                    float2 y = mul2(make_float2(s[e], s[e + 1]), add2(make_float2(d[c], d[c + 1]), make_float2(x.x, x.y)));
                    float2 z = mul2(make_float2(s[e + 2], s[e + 3]), add2(make_float2(d[c + 2], d[c + 3]), make_float2(x.z, x.w)));
                    if constexpr (CAP) {
                        y = mul2(y, make_float2(f[e], f[e + 1]));
                        z = mul2(z, make_float2(f[e + 2], f[e + 3]));
                    }
                    packed[c / 2] = bf16x2(y.x, y.y);
                    packed[c / 2 + 1] = bf16x2(z.x, z.y);
                }
                tmem_st16(mine_dp + h * 16, packed);
            }
            wait_st();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.ds_full));
            if (++u == n_u) { u = 0; ++g; }
        }
        if (ok && steps > 0) {
            ok = wait(smem_u32(&sh.done), 0, abort_flag, a.status, kPromptWaitProduct);
            fence_after();
        }
        const int part = (warp & 3) * 32;
        if (ok && split == 1) {
            // through shared memory: the keys' tile for dV, the values' for dK (neither is needed any more)
            const long long at = ((long long)(sh.k0 + part) * a.kv_heads + kv_head) * D;
            write_rows<D>(smem + w * F::kTile + part * D * 2, (w == 0 ? dV : dK) + lanes, w == 0 ? 1.f : a.scale, steps > 0,
                          (w == 0 ? a.dv : a.dk) + at, (long long)a.kv_heads * D, sh.rows - part, lane);
        } else if (ok) {
            // this CTA's share of the sums in fp32, for the cluster to add up: dV over the K and V tiles, dK over the ring
            uint8_t* mine_rows = smem + w * 2 * F::kTile + row * D * 4;
#pragma unroll
            for (int c = 0; c < D; c += 32) {
                float o[32];
                if (steps > 0) tmem_read32((w == 0 ? dV : dK) + lanes + c, o);
                else
#pragma unroll
                    for (int x = 0; x < 32; ++x) o[x] = 0.f;
#pragma unroll
                for (int x = 0; x < 8; ++x)
                    *reinterpret_cast<float4*>(mine_rows + (((c / 4 + x) ^ (lane & 7)) << 4)) = make_float4(o[4 * x], o[4 * x + 1], o[4 * x + 2], o[4 * x + 3]);
            }
        }
    } else if (warp == 8) {
        // ------------------------------------------------------------------ tile loads
        if (lane == 0 && steps > 0) {
            mbar_expect_tx(smem_u32(&sh.kv_full), 2 * F::kTile);
            load_tile<D>(k_smem, &map_k, kv_head, sh.k0, smem_u32(&sh.kv_full));
            load_tile<D>(v_smem, &map_v, kv_head, sh.k0, smem_u32(&sh.kv_full));
            int n = 0, g = 0, u = 0;
            bool ok = true;
            for (; n < steps; ++n) {
                const int st = n % F::kStages;
                ok = wait(smem_u32(&sh.empty[st]), (n / F::kStages & 1) ^ 1, abort_flag, a.status, kPromptWaitStage);
                if (!ok) break;
                const uint32_t bar = smem_u32(&sh.full[st]), dst = ring + st * 2 * F::kTile;
                mbar_expect_tx(bar, 2 * F::kTile);
                const int token = sh.q0 + (sh.u0 + u) * kTok;
                load_tile<D>(dst, &map_q, head0 + g, token, bar);
                load_tile<D>(dst + F::kTile, &map_do, head0 + g, token, bar);
                if (++u == n_u) { u = 0; ++g; }
            }
            if (!ok || *abort_flag) {  // nothing of this CTA's copies may be in flight when it ends
                wait(smem_u32(&sh.kv_full), 0, nullptr, a.status, kPromptWaitDrain);
                for (int i = max(0, n - F::kStages); i < n; ++i)
                    wait(smem_u32(&sh.full[i % F::kStages]), i / F::kStages & 1, nullptr, a.status, kPromptWaitDrain);
            }
        }
    } else if (warp == 9) {
        // ------------------------------------------------------------------ matrix products
        if (steps > 0) {
            auto loaded = [&](int n) {
                const int st = n % F::kStages;
                return wait_warp(smem_u32(&sh.full[st]), n / F::kStages & 1, abort_flag, a.status, kPromptWaitLoad) &&
                       wait_warp(smem_u32(&sh.ready[st]), n / F::kStages & 1, abort_flag, a.status, kPromptWaitLoad);
            };
            auto q_at = [&](int n) { return ring + n % F::kStages * 2 * F::kTile; };
            bool ok = wait_warp(smem_u32(&sh.kv_full), 0, abort_flag, a.status, kPromptWaitLoad) && loaded(0);
            if (ok) {
                scores<D>(tmem, k_smem, q_at(0), &sh.s_full);
                scores<D>(dP, v_smem, q_at(0) + F::kTile, &sh.dp_full);
            }
            for (int n = 0; ok && n < steps; ++n) {
                for (int h = 0; h < 2; ++h) {
                    ok = wait_warp(smem_u32(&sh.p_full[h]), n & 1, abort_flag, a.status, kPromptWaitSoftmax);
                    if (!ok) break;
                    fence_after();
                    gradient_half<D>(dV, tmem + h * 16, 64, q_at(n) + F::kTile + h * 32 * 128, n > 0 || h > 0);
                }
                if (!ok) break;
                const bool more = n + 1 < steps;
                if (more) {
                    ok = loaded(n + 1);
                    if (!ok) break;
                    scores<D>(tmem, k_smem, q_at(n + 1), &sh.s_full);
                }
                ok = wait_warp(smem_u32(&sh.ds_full), n & 1, abort_flag, a.status, kPromptWaitSoftmax);
                if (!ok) break;
                fence_after();
                gradient_half<D>(dK, dP, 64, q_at(n), n > 0);
                gradient_half<D>(dK, dP + 16, 64, q_at(n) + 32 * 128, true);
                signal(&sh.empty[n % F::kStages]);
                if (more) scores<D>(dP, v_smem, q_at(n + 1) + F::kTile, &sh.dp_full);
            }
            signal(&sh.done);
            signal(&sh.drain);
            wait_warp(smem_u32(&sh.drain), 0, nullptr, a.status, kPromptWaitDrain);
        }
    } else if (warp == 10) {
        // ------------------------------------------------------------------ lse and D of the query tiles; rows behind the
        // last query: lse +infinity (P = 0), and zeros for what another document or nobody holds there (0 * NaN)
        int g = 0, u = 0;
        auto fetch = [&](float2 (&x)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int q = (sh.u0 + u) * kTok + lane + 32 * i;
                x[i] = q < sh.qn ? a.stats[(long long)(head0 + g) * a.q_tokens + sh.q0 + q] : make_float2(INFINITY, 0.f);
            }
        };
        float2 next[4];
        if (steps > 0) fetch(next);
        for (int n = 0; n < steps; ++n) {
            const int st = n % F::kStages, valid = sh.qn - (sh.u0 + u) * kTok;
            float2 now[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) now[i] = next[i];
            if (++u == n_u) { u = 0; ++g; }
            if (n + 1 < steps) fetch(next);
            if (!wait(smem_u32(&sh.empty[st]), (n / F::kStages & 1) ^ 1, abort_flag, a.status, kPromptWaitStage)) break;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                stats[st * 2 * kTok + lane + 32 * i] = -now[i].x;
                stats[st * 2 * kTok + kTok + lane + 32 * i] = -now[i].y;
            }
            if (!wait(smem_u32(&sh.full[st]), n / F::kStages & 1, abort_flag, a.status, kPromptWaitLoad)) break;
            if (valid < kTok) clear_rows<2 * D / 64>(smem + (2 + 2 * st) * F::kTile, valid, lane);
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.ready[st]));
        }
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == 9) {
        __syncwarp();
        tmem_free(tmem, 512);
    }
    if (split > 1) {
        // every CTA of the cluster adds up every split-th row of dV and dK, over the CTAs in order of their rank
        // (where a wait ran out the sums are as wrong as the status word says)
        cluster_sync();
        if (warp < 8) {
            const int w = warp >> 2;
            for (int row = (warp & 3) * split + rank; row < sh.rows; row += 4 * split) {
                constexpr int kLanes = D / 4;  // four elements a lane
                if (lane < kLanes) {
                    const uint32_t at = smem_u32(smem) + w * 2 * F::kTile + row * D * 4 + ((lane ^ (row & 7)) << 4);
                    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
                    for (int r = 0; r < split; ++r) {
                        const float4 x = load_cluster(at, r);
                        sum.x += x.x;
                        sum.y += x.y;
                        sum.z += x.z;
                        sum.w += x.w;
                    }
                    const float scale = w == 0 ? 1.f : a.scale;
                    __nv_bfloat16* dst = (w == 0 ? a.dv : a.dk) + ((long long)(sh.k0 + row) * a.kv_heads + kv_head) * D + lane * 4;
                    *reinterpret_cast<uint2*>(dst) = make_uint2(bf16x2(sum.x * scale, sum.y * scale), bf16x2(sum.z * scale, sum.w * scale));
                }
            }
        }
        cluster_sync();  // nobody leaves while its rows are read
    }
}

// ---- dQ ----------------------------------------------------------------------------------------------------
//
// Tiles of 128 keys; each of the two sub-tiles has ONE block of 128 columns in tensor memory, which holds S, then dP (once
// the threads have taken S into registers), then dS.  The products of a tile are issued as
//   dQ0(j) | S0(j+1) | dQ1(j) | S1(j+1) | dP0(j+1) | dP1(j+1)
// and each sub-tile's arithmetic runs beside the other's products.

template <int D>
struct RowsK {
    static constexpr int kTile = kTok * D * 2;
    static constexpr int kValues = D == 128 ? 1 : 2;  // V tiles in flight (two K tiles: K is needed again for dQ)
    static constexpr int kSmem = (4 + 2 + kValues) * kTile + 1024;
};

struct RowsShared {
    uint64_t q_full, k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], s_read[2], dp_full[2], ds_full[2], done, clean[2], drain;
    uint32_t tmem;
    int abort;
    RowTile at;
};

template <int D, bool CAP, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1)
prompt_rows_kernel(const __grid_constant__ PromptArgs a, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do)
{
    using F = RowsK<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    static_assert(sizeof(RowsShared) <= 1024 && F::kSmem <= kMaxDynamicSmem, "shared memory");
    RowsShared& sh = *reinterpret_cast<RowsShared*>(smem + (6 + F::kValues) * F::kTile);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    volatile int* abort_flag = &sh.abort;

    if ((smem_u32(smem) & 1023u) != 0) {
        if (tid == 0) atomicCAS(a.status, 0, kPromptSmemMisaligned);
        return;
    }
    if (warp == 0) {
        find_row_tile(a, kTok, sh.at);
    } else if (warp == 8) {
        if (lane == 0) {
            prefetch_map(&map_q);
            prefetch_map(&map_k);
            prefetch_map(&map_v);
            prefetch_map(&map_do);
            sh.abort = 0;
            mbar_init(smem_u32(&sh.q_full), 1);
            for (int i = 0; i < 2; ++i) {
                mbar_init(smem_u32(&sh.k_full[i]), 1);
                mbar_init(smem_u32(&sh.k_empty[i]), 1);
                mbar_init(smem_u32(&sh.v_full[i]), 1);
                mbar_init(smem_u32(&sh.v_empty[i]), 1);
                mbar_init(smem_u32(&sh.s_full[i]), 1);
                mbar_init(smem_u32(&sh.s_read[i]), 4);
                mbar_init(smem_u32(&sh.dp_full[i]), 1);
                mbar_init(smem_u32(&sh.ds_full[i]), 4);
                mbar_init(smem_u32(&sh.clean[i]), 1);
            }
            mbar_init(smem_u32(&sh.done), 1);
            mbar_init(smem_u32(&sh.drain), 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
    } else if (warp == 9) {
        tmem_alloc(smem_u32(&sh.tmem), 512);
        fence_before();
    }
    __syncthreads();
    fence_after();
    const uint32_t tmem = sh.tmem;
    grid_dep_wait();  // the stats kernel's results
    grid_dep_launch();
    if (!sh.at.valid) {
        if (warp == 9) tmem_free(tmem, 512);
        return;
    }
    const int n_tiles = sh.at.n_tiles, a_end = sh.at.a_end, b0 = sh.at.b0, kn = sh.at.kn, prefix = sh.at.prefix;
    const int n_sub = sh.at.n_sub, kv_head = sh.at.kv_head;
    const bool full_head = a.full[kv_head] != 0;
    // Where queries see few keys, or slopes leave them few that matter, the rounding of dS weighs as much in dQ as that of the
    // result: dS then goes into its product in two bf16 parts.  The first queries of a long document, whose gradients are the
    // largest, are such queries, and cheap ones: 8192 tokens 697 -> 700 us (in bursts), dQ off by 1.9e-3 of its norm instead of 2.4e-3 (one
    // rounding of the exact gradient: 1.7e-3).  Up to 2048 keys: 712 us, 1.9e-3; for all, the fourth product would cost a quarter
    // of the kernel's time (857 us).  The usual slopes, 2^(-8 (j + 1) / heads), are steep in this sense for every head, so a sample
    // with a distance term pays that at every length.
    const int seen = full_head ? min(kn, n_tiles * kTok) : min(kn, a.sink + a.window);
    const float steepest = BIAS ? fmaxf(fabsf(a.slopes[sh.at.head[0]]), fabsf(a.slopes[sh.at.head[1]])) : 0.f;
    const bool in_two = seen <= kFewKeys || steepest * kFewKeys >= 1.f;
    const uint32_t q_smem = smem_u32(smem), o_smem = q_smem + 2 * F::kTile, k_smem = q_smem + 4 * F::kTile, v_smem = q_smem + 6 * F::kTile;
    auto tile_at = [&](int j) { return j < a_end ? j : b0 + j - a_end; };
    // (launched with 384 x 168 = 64512 registers: 256 x 232 + 128 x 40)
    if (warp < 8) more_registers<232>();
    else fewer_registers<40>();
    if (warp < 8) {
        // ------------------------------------------------------------------ P and dS, one thread per query
        const int w = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, S = tmem + lanes + w * kTok;
        const int first = sh.at.pos0[w], pos = first + row, last = first + kTok - 1, head = sh.at.head[w];
        const bool mine = row < sh.at.rows[w];
        const int hi = min(kn, max(pos + 1, prefix)), lo = full_head ? 0 : pos - a.window + 1, sink = full_head ? 0 : min(a.sink, hi);
        const Cap cap(CAP ? a.softcap : 1.f, a.scale);
        const float sl2 = a.scale * kLog2e;
        const float slope2 = BIAS ? a.slopes[head] * kLog2e : 0.f;
        float2* stat_at = a.stats + (long long)head * a.q_tokens + sh.at.q0[w] + row;
        const float2 stat = mine ? *stat_at : make_float2(INFINITY, 0.f);
        float2 excess = make_float2(0.f, 0.f);  // sum of P (dP - D): zero but for the rounding of `out` that D comes from
        const int first_seen = full_head || sink > 0 ? 0 : max(lo, 0);
        bool ok = true;
        int done = 0;
        const int sub_a = sh.at.sub_a[w], sub_b = sh.at.sub_b[w], sub_e = sh.at.sub_e[w];
        for (int t = sub_a > 0 ? 0 : sub_b; t < sub_e; t = t + 1 == sub_a ? sub_b : t + 1) {
            const int start = t * kTok;
            ok = wait(smem_u32(&sh.s_full[w]), done & 1, abort_flag, a.status, kPromptWaitProduct);
            if (!ok) break;
            fence_after();
            float s[kTok];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(S + c * 32, s + c * 32);
            wait_ld();
#pragma unroll
            for (int c = 0; c < kTok; ++c) asm volatile("" : "+f"(s[c]));  // nothing of the above is used before the wait
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.s_read[w]));
            const bool plain = start + kTok <= kn && (start + kTok <= first + 1 || start + kTok <= prefix) &&
                               (full_head || start + kTok <= a.sink || start > last - a.window);
            // 32 scores -> P (with CAP after dP is there: its slopes would not fit in registers beside P)
            const float2 factor = CAP || BIAS ? make_float2(1.f, 1.f) : make_float2(sl2, sl2), minus_lse = make_float2(-stat.x, -stat.x);
            auto probabilities = [&](float (&x)[32], float (&f)[CAP ? 32 : 1], int c0) {
                finish_scores<CAP, BIAS>(cap, sl2, slope2, pos - c0, -1, mine, x, f);
#pragma unroll
                for (int c = 0; c < 32; c += 2) {
                    const float2 y = fma2(make_float2(x[c], x[c + 1]), factor, minus_lse);
                    x[c] = ex2(y.x);
                    x[c + 1] = ex2(y.y);
                }
                if (!plain) {
                    const uint32_t see = range_bits(lo - c0, hi - c0) | range_bits(0, sink - c0);
#pragma unroll
                    for (int c = 0; c < 32; ++c) x[c] = see >> c & 1 ? x[c] : 0.f;
                }
            };
            if constexpr (!CAP) {
                float none[1];
#pragma unroll
                for (int c = 0; c < 4; ++c) probabilities(reinterpret_cast<float(&)[32]>(s[c * 32]), none, start + c * 32);
            }
            ok = wait(smem_u32(&sh.dp_full[w]), done & 1, abort_flag, a.status, kPromptWaitProduct);
            if (!ok) break;
            fence_after();
            // A query whose keys all lie in this tile has its D put right before dS is rounded: of few keys (a window of five,
            // say) the rounding of `out` in D would weigh more in dQ than all others (2.6e-3 of its norm; 1.7e-3 so).  Five
            // documents of 355 tokens: 29 -> 31 us.
            float minus_d = -stat.y;
            const bool whole = mine && first_seen >= start && hi <= start + kTok;
            if (__any_sync(0xffffffffu, whole)) {
                float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float p[32], f[CAP ? 32 : 1], d[32];
#pragma unroll
                    for (int c = 0; c < 32; ++c) p[c] = s[q * 32 + c];
                    if constexpr (CAP) probabilities(p, f, start + q * 32);
                    tmem_read32(S + q * 32, d);
#pragma unroll
                    for (int c = 0; c < 32; c += 2)
                        sum = fma2(make_float2(p[c], p[c + 1]), add2(make_float2(d[c], d[c + 1]), make_float2(minus_d, minus_d)), sum);
                }
                if (whole) {
                    excess.x += sum.x + sum.y;
                    minus_d -= sum.x + sum.y;
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float(&p)[32] = reinterpret_cast<float(&)[32]>(s[q * 32]);
                float f[CAP ? 32 : 1], d[32];
                if constexpr (CAP) probabilities(p, f, start + q * 32);
                tmem_read32(S + q * 32, d);
                uint32_t packed[16];
#pragma unroll
                for (int c = 0; c < 32; c += 2) {
                    float2 ds = mul2(make_float2(p[c], p[c + 1]), add2(make_float2(d[c], d[c + 1]), make_float2(minus_d, minus_d)));
                    excess = add2(excess, ds);
                    if constexpr (CAP) ds = mul2(ds, make_float2(f[c], f[c + 1]));
                    packed[c / 2] = bf16x2(ds.x, ds.y);
                    p[c] = ds.x;
                    p[c + 1] = ds.y;
                }
                tmem_st16(S + q * 32, packed);
                if (in_two) {
#pragma unroll
                    for (int c = 0; c < 16; ++c)
                        packed[c] = bf16x2(p[2 * c] - __uint_as_float(packed[c] << 16), p[2 * c + 1] - __uint_as_float(packed[c] & 0xffff0000u));
                    tmem_st16(S + q * 32 + 16, packed);
                }
            }
            wait_st();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.ds_full[w]));
            ++done;
        }
        if (ok && n_tiles > 0) {
            ok = wait(smem_u32(&sh.done), 0, abort_flag, a.status, kPromptWaitProduct);
            fence_after();
        }
        if (ok && mine && w < n_sub) stat_at->y = stat.y + excess.x + excess.y;  // for the keys kernel
        if (ok && w < n_sub) {  // through shared memory: the sub-tile's queries are not needed any more
            const int part = (warp & 3) * 32;
            write_rows<D>(smem + w * F::kTile + part * D * 2, tmem + lanes + 256 + w * D, a.scale, done > 0,
                          a.dq + ((long long)(sh.at.q0[w] + part) * a.q_heads + head) * D, (long long)a.q_heads * D, sh.at.rows[w] - part, lane);
        }
    } else if (warp == 8) {
        // ------------------------------------------------------------------ tile loads
        if (lane == 0 && n_tiles > 0) {
            mbar_expect_tx(smem_u32(&sh.q_full), 2 * n_sub * F::kTile);
            for (int w = 0; w < n_sub; ++w) {
                load_tile<D>(q_smem + w * F::kTile, &map_q, sh.at.head[w], sh.at.q0[w], smem_u32(&sh.q_full));
                load_tile<D>(o_smem + w * F::kTile, &map_do, sh.at.head[w], sh.at.q0[w], smem_u32(&sh.q_full));
            }
            int n_k = 0, n_v = 0;
            bool ok = true;
            for (int j = 0; ok && j < n_tiles; ++j) {
                const int token = sh.at.k0 + tile_at(j) * kTok;
                ok = wait(smem_u32(&sh.k_empty[j % 2]), (j / 2 & 1) ^ 1, abort_flag, a.status, kPromptWaitStage);
                if (!ok) break;
                mbar_expect_tx(smem_u32(&sh.k_full[j % 2]), F::kTile);
                load_tile<D>(k_smem + j % 2 * F::kTile, &map_k, kv_head, token, smem_u32(&sh.k_full[j % 2]));
                ++n_k;
                const int v = j % F::kValues;
                ok = wait(smem_u32(&sh.v_empty[v]), (j / F::kValues & 1) ^ 1, abort_flag, a.status, kPromptWaitStage);
                if (!ok) break;
                mbar_expect_tx(smem_u32(&sh.v_full[v]), F::kTile);
                load_tile<D>(v_smem + v * F::kTile, &map_v, kv_head, token, smem_u32(&sh.v_full[v]));
                ++n_v;
            }
            if (!ok || *abort_flag) {  // nothing of this CTA's copies may be in flight when it ends
                wait(smem_u32(&sh.q_full), 0, nullptr, a.status, kPromptWaitDrain);
                for (int i = max(0, n_k - 2); i < n_k; ++i) wait(smem_u32(&sh.k_full[i % 2]), i / 2 & 1, nullptr, a.status, kPromptWaitDrain);
                for (int i = max(0, n_v - F::kValues); i < n_v; ++i)
                    wait(smem_u32(&sh.v_full[i % F::kValues]), i / F::kValues & 1, nullptr, a.status, kPromptWaitDrain);
            }
        }
        __syncwarp();
        // rows behind the last key: only the last tiles can hold any.  (This warp may wait for them: it has seen their
        // slots' earlier copies consumed)
        const int end = n_tiles - 1, rows = n_tiles > 0 ? kn - tile_at(end) * kTok : kTok;
        if (rows < kTok) {
            if (!*abort_flag && wait(smem_u32(&sh.k_full[end % 2]), end / 2 & 1, abort_flag, a.status, kPromptWaitLoad)) {
                clear_rows<D / 64>(smem + (4 + end % 2) * F::kTile, rows, lane);
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh.clean[0]));
            }
            __syncwarp();
            const int v = end % F::kValues;
            if (!*abort_flag && wait(smem_u32(&sh.v_full[v]), end / F::kValues & 1, abort_flag, a.status, kPromptWaitLoad)) {
                clear_rows<D / 64>(smem + (6 + v) * F::kTile, rows, lane);
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh.clean[1]));
            }
        }
    } else if (warp == 9) {
        // ------------------------------------------------------------------ matrix products
        if (n_tiles > 0) {
            // Each sub-tile goes its own way -- S, dP once its threads hold S, dQ once they have written dS -- and whatever is
            // ready first is issued first: in a fixed order of the two one would wait for the other's arithmetic.
            const int sub_a[2] = {sh.at.sub_a[0], sh.at.sub_a[1]}, sub_b[2] = {sh.at.sub_b[0], sh.at.sub_b[1]}, sub_e[2] = {sh.at.sub_e[0], sh.at.sub_e[1]};
            enum { kNextS, kNextDp, kNextDq, kNothing };  // the product that comes next
            int tile[2], next[2], done[2] = {0, 0}, passed_k[2], passed_v[2], freed_k = 0, freed_v = 0;
            // (the CTA's running number of a tile, which its K and V slots go by)
            auto number = [&](int t) { return t < a_end ? t : a_end + t - b0; };
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                tile[w] = sub_a[w] > 0 ? 0 : sub_b[w];
                next[w] = tile[w] < sub_e[w] ? kNextS : kNothing;
                passed_k[w] = passed_v[w] = next[w] == kNothing ? n_tiles : number(tile[w]);
            }
            auto ready = [&](uint64_t* bar, int parity) { return __all_sync(0xffffffffu, mbar_try_wait(smem_u32(bar), parity & 1)); };
            // rows behind the last key have been cleared
            auto cleaned = [&](int t, int which) { return (t + 1) * kTok <= kn || ready(&sh.clean[which], 0); };
            bool ok = wait_warp(smem_u32(&sh.q_full), 0, abort_flag, a.status, kPromptWaitLoad);
            uint64_t idle_since = 0;
            while (ok && (next[0] != kNothing || next[1] != kNothing)) {
                bool moved = false;
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const int t = tile[w], j = number(t), after = t + 1 == sub_a[w] ? sub_b[w] : t + 1;
                    const int after_j = after < sub_e[w] ? number(after) : n_tiles;
                    if (next[w] == kNextS) {
                        // (a slot's phase says which tile it holds only once the one before it has been given back)
                        if (freed_k < j - 1 || !ready(&sh.k_full[j % 2], j / 2) || !cleaned(t, 0)) continue;
                        scores<D>(tmem + w * kTok, q_smem + w * F::kTile, k_smem + j % 2 * F::kTile, &sh.s_full[w]);
                        next[w] = kNextDp;
                    } else if (next[w] == kNextDp) {
                        const int v = j % F::kValues;
                        if (freed_v < j - F::kValues + 1 || !ready(&sh.s_read[w], done[w]) || !ready(&sh.v_full[v], j / F::kValues) || !cleaned(t, 1)) continue;
                        fence_after();
                        scores<D>(tmem + w * kTok, o_smem + w * F::kTile, v_smem + v * F::kTile, &sh.dp_full[w]);
                        next[w] = kNextDq;
                        passed_v[w] = after_j;
                    } else if (next[w] == kNextDq) {
                        if (!ready(&sh.ds_full[w], done[w])) continue;
                        fence_after();
                        gradient_blocks<D>(tmem + 256 + w * D, tmem + w * kTok, k_smem + j % 2 * F::kTile, in_two, done[w] > 0);
                        ++done[w];
                        passed_k[w] = after_j;
                        tile[w] = after;
                        next[w] = after_j < n_tiles ? kNextS : kNothing;
                        // (the next S at once where its keys are there: the two sub-tiles then stay out of step, and one's
                        // arithmetic runs beside the other's products)
                        if (after_j < n_tiles && freed_k >= after_j - 1 && ready(&sh.k_full[after_j % 2], after_j / 2) && cleaned(after, 0)) {
                            scores<D>(tmem + w * kTok, q_smem + w * F::kTile, k_smem + after_j % 2 * F::kTile, &sh.s_full[w]);
                            next[w] = kNextDp;
                        }
                    } else {
                        continue;
                    }
                    moved = true;
                    // slots that neither sub-tile needs any more
                    for (; freed_k < min(passed_k[0], passed_k[1]); ++freed_k) signal(&sh.k_empty[freed_k % 2]);
                    for (; freed_v < min(passed_v[0], passed_v[1]); ++freed_v) signal(&sh.v_empty[freed_v % F::kValues]);
                }
                if (moved) {
                    idle_since = 0;
                } else {
                    const uint64_t now = __shfl_sync(0xffffffffu, now_ns(), 0);
                    if (idle_since == 0) idle_since = now;
                    if (now - idle_since > kWaitNs) {
                        if (lane == 0) {
                            *abort_flag = 1;
                            atomicCAS(a.status, 0, kPromptWaitSoftmax);
                        }
                        ok = false;
                    }
                    if (__any_sync(0xffffffffu, *abort_flag != 0)) ok = false;
                }
            }
            signal(&sh.done);
            signal(&sh.drain);
            wait_warp(smem_u32(&sh.drain), 0, nullptr, a.status, kPromptWaitDrain);
        }
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == 9) {
        __syncwarp();
        tmem_free(tmem, 512);
    }
}

struct Maps {
    const CUtensorMap &q, &k, &v, &dout;
};

template <int D, bool CAP, bool BIAS>
cudaError_t launch_one(const PromptArgs& a, const Maps& m, cudaStream_t stream)
{
    const dim3 stats((a.q_tokens + 7) / 8, (a.q_heads + 7) / 8);
    prompt_stats_kernel<D><<<stats, 256, 0, stream>>>(a);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    // The other two start while the kernel before them drains, set themselves up and wait for it; what they read until then
    // (documents' starts) is older than the stats kernel, which is launched the ordinary way.  Five documents: 77.2 -> 75.7 us
    // a pass, 4096 tokens 402 -> 397.  Loads and first products before the wait gained no more than 0.7 us.
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3((unsigned)row_tile_blocks(a));
    cfg.dynamicSmemBytes = RowsK<D>::kSmem;
    e = cudaLaunchKernelEx(&cfg, prompt_rows_kernel<D, CAP, BIAS>, a, m.q, m.k, m.v, m.dout);
    if (e != cudaSuccess) return e;
    // Few key tiles: the query heads of a KV head go to several CTAs, as many (a divisor of the group) as leave no more than
    // four per SM.  A causal document's first key tile is seen by all its queries, so this also evens out the CTAs' work.
    const long long tiles = ((long long)a.k_tokens / kTok + (a.n_docs < a.k_tokens ? a.n_docs : a.k_tokens)) * a.kv_heads;
    int split = 1;
    for (int x = 2; x <= a.group; ++x)
        if (a.group % x == 0 && tiles * x <= 4 * 148) split = x;
    cfg.gridDim = dim3((unsigned)(tiles * split));
    cfg.dynamicSmemBytes = Keys<D>::kSmem;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = split;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    if (split > 1) cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, prompt_keys_kernel<D, CAP, BIAS>, a, m.q, m.k, m.v, m.dout, split);
}

template <int D>
cudaError_t launch_dim(const PromptArgs& a, const Maps& m, cudaStream_t stream)
{
    if (a.softcap != 0.f) return a.slopes ? launch_one<D, true, true>(a, m, stream) : launch_one<D, true, false>(a, m, stream);
    return a.slopes ? launch_one<D, false, true>(a, m, stream) : launch_one<D, false, false>(a, m, stream);
}

template <int D, bool CAP, bool BIAS>
cudaError_t prepare_one()
{
    const cudaError_t e = cudaFuncSetAttribute(prompt_keys_kernel<D, CAP, BIAS>, cudaFuncAttributeMaxDynamicSharedMemorySize, Keys<D>::kSmem);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(prompt_rows_kernel<D, CAP, BIAS>, cudaFuncAttributeMaxDynamicSharedMemorySize, RowsK<D>::kSmem);
}

template <int D>
cudaError_t prepare_dim()
{
    cudaError_t e = prepare_one<D, false, false>();
    if (e == cudaSuccess) e = prepare_one<D, false, true>();
    if (e == cudaSuccess) e = prepare_one<D, true, false>();
    return e == cudaSuccess ? prepare_one<D, true, true>() : e;
}

}  // namespace

cudaError_t launch_prompt_backward(const PromptArgs& a, const CUtensorMap& map_q, const CUtensorMap& map_k, const CUtensorMap& map_v,
                                   const CUtensorMap& map_do, int head_dim, cudaStream_t stream)
{
    const Maps m{map_q, map_k, map_v, map_do};
    return head_dim == 128 ? launch_dim<128>(a, m, stream) : launch_dim<64>(a, m, stream);
}

cudaError_t prepare_prompt_backward(int head_dim) { return head_dim == 128 ? prepare_dim<128>() : prepare_dim<64>(); }

}  // namespace rlkv
