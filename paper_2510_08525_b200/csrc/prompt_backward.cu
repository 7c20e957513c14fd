// The backward pass of prompt attention on the tensor cores, in three launches without atomics:
//
//   stats   D_i = sum over head_dim of dout * out, stored with lse (log2 domain) per head and query
//   rows    one CTA per 256 query rows (two heads, or one): over their keys (64 at a time), S = Q.K^T and dP = dO.V^T,
//           then dQ += dS.K.  It also corrects D: out was rounded to bf16, and sum_j P (dP - D) is what that changed
//   keys    one CTA (or one per part of the query heads, in a cluster that adds them up) per 128 keys of a KV head: over
//           the queries that see them (64 at a time), S^T = K.Q^T and dP^T = V.dO^T, then dV += P^T.dO and dK += dS^T.Q
//
// S and dP are computed twice, seven products where five would do, and in return every gradient is summed by one CTA
// in a fixed order: no atomics on dQ, no fp32 copy of it in memory, the same bits on every run.  P and dS are written
// to tensor memory as bf16 over S and dP and are the A operand of the second products straight from there.  Two
// warpgroups alternate -- over query tiles in `keys`, over 128-row sub-tiles in `rows` -- so that one's products run
// beside the other's arithmetic.
#include "rlkv_prompt.cuh"
#include "tcgen05.cuh"

namespace rlkv {
namespace {

using namespace tc;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kRows = 128;  // rows of a product's result: keys (keys kernel) or queries (rows kernel)
constexpr int kCols = 64;   // its columns: queries or keys
constexpr int kRowBlock = kRows * 128, kColBlock = kCols * 128;  // bytes of a block of 64 elements of so many rows
constexpr int kThreads = 384;

// ---- D and lse ---------------------------------------------------------------------------------------

// One warp per head and eight queries, half a warp per row, all loads at once.  Stored head by head, so that the keys
// kernel reads consecutive queries.  A query that sees nothing gets lse = +infinity: its P is then exp2(s - infinity) = 0.
template <int D>
__global__ void __launch_bounds__(256) prompt_stats_kernel(const __grid_constant__ PromptArgs a)
{
    constexpr int E = D / 16, kTokens = 8;  // elements of a lane, queries of a warp
    const int lane = threadIdx.x & 31, half = lane >> 4, l16 = lane & 15;
    const int h = blockIdx.y * 8 + (threadIdx.x >> 5);
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

// 32 products q.k -> scores in the log2 domain, and (CAP) the slopes of the cap, 1 - tanh^2.
template <bool CAP>
__device__ __forceinline__ void capped(const Cap& cap, float sl2, bool vote, float (&s)[32], float (&f)[CAP ? 32 : 1])
{
    if constexpr (!CAP) {
#pragma unroll
        for (int c = 0; c < 32; ++c) s[c] *= sl2;
    } else {
        cap.apply(s, vote);
        const float2 k = make_float2(-1.f / (cap.cap2 * cap.cap2), -1.f / (cap.cap2 * cap.cap2));
#pragma unroll
        for (int c = 0; c < 32; c += 2) {
            const float2 x = make_float2(s[c], s[c + 1]), y = fma2(mul2(x, x), k, make_float2(1.f, 1.f));
            f[c] = y.x;
            f[c + 1] = y.y;
        }
    }
}

// rows x 64 elements of one head from token `token` on: boxes of 64 tokens, D / 64 of them side by side.
template <int D>
__device__ __forceinline__ void load_rows(uint32_t dst, int rows, const CUtensorMap* map, int head, int token, uint32_t bar)
{
    for (int b = 0; b < D / 64; ++b)
        for (int r = 0; r < rows; r += 64) load_box(dst + b * rows * 128 + r * 128, map, b * 64, head, token + r, bar);
}

// ---- dK and dV ------------------------------------------------------------------------------------------

template <int D>
struct Keys {
    static constexpr int kRowTile = kRows * D * 2, kColTile = kCols * D * 2;
    static constexpr int kStages = 4;  // (even: a stage is always used by the same warpgroup)
    static constexpr int kStats = 2 * kRowTile + kStages * 2 * kColTile;
    static constexpr int kSmem = kStats + kStages * kCols * 8 + 1024;
};

struct KeysShared {
    uint64_t kv_full, full[4], empty[4], ready[4], sd_full[2], pds_full[2], done, drain;
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
    float2* stats = reinterpret_cast<float2*>(smem + F::kStats);
    KeysShared& sh = *reinterpret_cast<KeysShared*>(smem + F::kStats + F::kStages * kCols * 8);
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
        int doc = 0, tile = 0;
        const bool valid = find_tile(a, true, kRows, block / a.kv_heads, doc, tile);
        if (lane == 0) {
            sh.valid = valid;
            if (valid) {
                const DocRange r = doc_range(a, doc);
                tile = (r.kn + kRows - 1) / kRows - 1 - tile;  // a document's first keys are seen by the most queries
                const int j0 = tile * kRows, j1 = min(j0 + kRows, r.kn), off = r.kn - r.qn;
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
                sh.u0 = lower / kCols;
                sh.n_u = upper > lower ? (upper + kCols - 1) / kCols - sh.u0 : 0;
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
            for (int w = 0; w < 2; ++w) {
                mbar_init(smem_u32(&sh.sd_full[w]), 1);
                mbar_init(smem_u32(&sh.pds_full[w]), 4);
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
    if (!sh.valid) {
        if (warp == 9) tmem_free(tmem, 512);
        return;
    }
    const uint32_t dV = tmem + 256, dK = tmem + 256 + D;
    const uint32_t k_smem = smem_u32(smem), v_smem = k_smem + F::kRowTile, ring = v_smem + F::kRowTile;
    const int n_u = sh.n_u, steps = n_u * heads;  // step n: query tile u0 + n % n_u of query head head0 + n / n_u

    if (warp < 8) {
        // ------------------------------------------------------------------ P and dS, one thread per key
        const int w = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t S = tmem + lanes + w * 128, dP = S + 64;
        const int j = sh.j0 + row, j_last = sh.j0 + sh.rows - 1;
        const bool mine = row < sh.rows;
        // the key is seen from positions lo .. hi-1
        const int lo = j < sh.prefix ? INT_MIN / 2 : j, hi = full_head || j < a.sink ? INT_MAX / 2 : j + a.window;
        const Cap cap(CAP ? a.softcap : 1.f, a.scale);
        const float sl2 = a.scale * kLog2e;
        bool ok = true;
        int g = 0, u = w;  // of step n
        while (n_u > 0 && u >= n_u) { u -= n_u; ++g; }
        for (int n = w; ok && n < steps; n += 2) {
            const int st = n % F::kStages;
            ok = wait(smem_u32(&sh.ready[st]), n / F::kStages & 1, abort_flag, a.status, kPromptWaitLoad) &&
                 wait(smem_u32(&sh.sd_full[w]), n >> 1 & 1, abort_flag, a.status, kPromptWaitProduct);
            if (!ok) break;
            fence_after();
            const float4* stat = reinterpret_cast<const float4*>(stats + st * kCols);
            const int p0 = (sh.u0 + u) * kCols + sh.off;  // position of column 0
            const bool past = p0 >= j_last;               // every query at or behind every key
            const bool plain = (past || j_last < sh.prefix) && (full_head || j_last < a.sink || p0 + kCols - 1 < sh.j0 + a.window);
            const float slope2 = BIAS ? a.slopes[head0 + g] * kLog2e : 0.f;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float s[32], f[CAP ? 32 : 1];
                tmem_read32(S + half * 32, s);
                capped<CAP>(cap, sl2, mine, s, f);
                const int d0 = p0 + half * 32 - j;  // distance of column 0
                if (BIAS) {
#pragma unroll
                    for (int c = 0; c < 32; ++c) s[c] = fmaf(-slope2, fabsf((float)(d0 + c)), s[c]);
                }
#pragma unroll
                for (int c = 0; c < 32; c += 2) {
                    const float4 x = stat[half * 16 + c / 2];  // (lse, D) of two queries
                    s[c] = ex2(s[c] - x.x);
                    s[c + 1] = ex2(s[c + 1] - x.z);
                }
                if (!plain) {
                    const uint32_t see = range_bits(lo - j - d0, hi - j - d0);
#pragma unroll
                    for (int c = 0; c < 32; ++c) s[c] = see >> c & 1 ? s[c] : 0.f;
                }
                uint32_t packed[16];
#pragma unroll
                for (int c = 0; c < 16; ++c) packed[c] = bf16x2(s[2 * c], s[2 * c + 1]);
                tmem_st16(S + half * 16, packed);
                float d[32];
                tmem_read32(dP + half * 32, d);
#pragma unroll
                for (int c = 0; c < 32; c += 2) {
                    const float4 x = stat[half * 16 + c / 2];
                    d[c] = s[c] * (d[c] - x.y);
                    d[c + 1] = s[c + 1] * (d[c + 1] - x.w);
                    if constexpr (CAP) {
                        d[c] *= f[c];
                        d[c + 1] *= f[c + 1];
                    }
                    packed[c / 2] = bf16x2(d[c], d[c + 1]);
                }
                tmem_st16(dP + half * 16, packed);
            }
            wait_st();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.pds_full[w]));
            u += 2;
            while (u >= n_u) { u -= n_u; ++g; }
        }
        if (ok && steps > 0) {
            ok = wait(smem_u32(&sh.done), 0, abort_flag, a.status, kPromptWaitProduct);
            fence_after();
        }
        const int part = (warp & 3) * 32;
        if (ok && split == 1) {
            // through shared memory: the keys' tile for dV, the values' for dK (neither is needed any more)
            const long long at = ((long long)(sh.k0 + part) * a.kv_heads + kv_head) * D;
            write_rows<D>(smem + w * F::kRowTile + part * D * 2, (w == 0 ? dV : dK) + lanes, w == 0 ? 1.f : a.scale, steps > 0,
                          (w == 0 ? a.dv : a.dk) + at, (long long)a.kv_heads * D, sh.rows - part, lane);
        } else if (ok) {
            // this CTA's share of the sums in fp32, for the cluster to add up: dV over the K and V tiles, dK over the ring
            uint8_t* mine_rows = smem + w * 2 * F::kRowTile + row * D * 4;
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
            mbar_expect_tx(smem_u32(&sh.kv_full), 2 * F::kRowTile);
            load_rows<D>(k_smem, kRows, &map_k, kv_head, sh.k0, smem_u32(&sh.kv_full));
            load_rows<D>(v_smem, kRows, &map_v, kv_head, sh.k0, smem_u32(&sh.kv_full));
            int n = 0, g = 0, u = 0;
            bool ok = true;
            for (; n < steps; ++n) {
                const int st = n % F::kStages;
                ok = wait(smem_u32(&sh.empty[st]), (n / F::kStages & 1) ^ 1, abort_flag, a.status, kPromptWaitStage);
                if (!ok) break;
                const uint32_t bar = smem_u32(&sh.full[st]), dst = ring + st * 2 * F::kColTile;
                mbar_expect_tx(bar, 2 * F::kColTile);
                const int token = sh.q0 + (sh.u0 + u) * kCols;
                load_rows<D>(dst, kCols, &map_q, head0 + g, token, bar);
                load_rows<D>(dst + F::kColTile, kCols, &map_do, head0 + g, token, bar);
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
            constexpr uint32_t kScores = instr_desc(kRows, kCols, false), kGrads = instr_desc(kRows, D, true);
            const uint64_t k_desc = smem_desc(k_smem), v_desc = smem_desc(v_smem);
            auto signal = [&](uint64_t* bar) {
                if (elect_one()) commit(smem_u32(bar));
            };
            auto first_products = [&](int n) {
                const int st = n % F::kStages;
                if (!wait_warp(smem_u32(&sh.full[st]), n / F::kStages & 1, abort_flag, a.status, kPromptWaitLoad) ||
                    !wait_warp(smem_u32(&sh.ready[st]), n / F::kStages & 1, abort_flag, a.status, kPromptWaitLoad))
                    return false;
                const uint64_t q = smem_desc(ring + st * 2 * F::kColTile), o = smem_desc(ring + st * 2 * F::kColTile + F::kColTile);
                const uint32_t d = tmem + (n & 1) * 128;
                if (elect_one()) {
#pragma unroll
                    for (int x = 0; x < D / 16; ++x)
                        mma_ss(d, k_desc + ((x / 4 * kRowBlock + x % 4 * 32) >> 4), q + ((x / 4 * kColBlock + x % 4 * 32) >> 4), kScores, x > 0);
#pragma unroll
                    for (int x = 0; x < D / 16; ++x)
                        mma_ss(d + 64, v_desc + ((x / 4 * kRowBlock + x % 4 * 32) >> 4), o + ((x / 4 * kColBlock + x % 4 * 32) >> 4), kScores, x > 0);
                    commit(smem_u32(&sh.sd_full[n & 1]));
                }
                return true;
            };
            bool ok = wait_warp(smem_u32(&sh.kv_full), 0, abort_flag, a.status, kPromptWaitLoad) && first_products(0);
            if (ok && steps > 1) ok = first_products(1);
            for (int n = 0; ok && n < steps; ++n) {
                const int st = n % F::kStages, w = n & 1;
                ok = wait_warp(smem_u32(&sh.pds_full[w]), n >> 1 & 1, abort_flag, a.status, kPromptWaitSoftmax);
                if (!ok) break;
                fence_after();
                const uint64_t q = smem_desc(ring + st * 2 * F::kColTile, kColBlock), o = smem_desc(ring + st * 2 * F::kColTile + F::kColTile, kColBlock);
                const uint32_t d = tmem + w * 128;
                if (elect_one()) {
#pragma unroll
                    for (int x = 0; x < kCols / 16; ++x) mma_ts(dV, d + x * 8, o + (x * 2048 >> 4), kGrads, n > 0 || x > 0);
#pragma unroll
                    for (int x = 0; x < kCols / 16; ++x) mma_ts(dK, d + 64 + x * 8, q + (x * 2048 >> 4), kGrads, n > 0 || x > 0);
                    commit(smem_u32(&sh.empty[st]));
                }
                if (n + 2 < steps) ok = first_products(n + 2);
            }
            signal(&sh.done);
            signal(&sh.drain);
            wait_warp(smem_u32(&sh.drain), 0, nullptr, a.status, kPromptWaitDrain);
        }
    } else if (warp == 10) {
        // ------------------------------------------------------------------ lse and D of the query tiles; rows behind the
        // last query: lse +infinity (P = 0), and zeros for what another document or nobody holds there (0 * NaN)
        int g = 0, u = 0;
        auto fetch = [&](float2 (&x)[2]) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int q = (sh.u0 + u) * kCols + lane + 32 * i;
                x[i] = q < sh.qn ? a.stats[(long long)(head0 + g) * a.q_tokens + sh.q0 + q] : make_float2(INFINITY, 0.f);
            }
        };
        float2 next[2];
        if (steps > 0) fetch(next);
        for (int n = 0; n < steps; ++n) {
            const int st = n % F::kStages, valid = sh.qn - (sh.u0 + u) * kCols;
            const float2 now[2] = {next[0], next[1]};
            if (++u == n_u) { u = 0; ++g; }
            if (n + 1 < steps) fetch(next);
            if (!wait(smem_u32(&sh.empty[st]), (n / F::kStages & 1) ^ 1, abort_flag, a.status, kPromptWaitStage)) break;
            stats[st * kCols + lane] = now[0];
            stats[st * kCols + lane + 32] = now[1];
            if (!wait(smem_u32(&sh.full[st]), n / F::kStages & 1, abort_flag, a.status, kPromptWaitLoad)) break;
            if (valid < kCols) {
                uint8_t* x = smem + 2 * F::kRowTile + st * 2 * F::kColTile;
                for (int i = valid * 8 + lane; i < kCols * 8; i += 32)
                    for (int b = 0; b < 2 * D / 64; ++b) *reinterpret_cast<uint4*>(x + b * kColBlock + i * 16) = make_uint4(0, 0, 0, 0);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
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
                    const uint32_t at = smem_u32(smem) + w * 2 * F::kRowTile + row * D * 4 + ((lane ^ (row & 7)) << 4);
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

template <int D>
struct RowsK {
    static constexpr int kRowTile = kRows * D * 2, kColTile = kCols * D * 2;
    static constexpr int kStages = D == 128 ? 3 : 6;
    static constexpr int kSmem = 4 * kRowTile + kStages * 2 * kColTile + 1024;
};

struct RowsShared {
    uint64_t q_full, full[6], empty[6], sd_full[2], ds_full[2], done, clean, drain;
    uint32_t tmem;
    int abort;
    RowTile at;  // as in the forward pass, key tiles of 64
};

template <int D, bool CAP, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1)
prompt_rows_kernel(const __grid_constant__ PromptArgs a, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do)
{
    using F = RowsK<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    RowsShared& sh = *reinterpret_cast<RowsShared*>(smem + 4 * F::kRowTile + F::kStages * 2 * F::kColTile);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    volatile int* abort_flag = &sh.abort;

    if ((smem_u32(smem) & 1023u) != 0) {
        if (tid == 0) atomicCAS(a.status, 0, kPromptSmemMisaligned);
        return;
    }
    if (warp == 0) {
        find_row_tile(a, kCols, sh.at);
    } else if (warp == 8) {
        if (lane == 0) {
            prefetch_map(&map_q);
            prefetch_map(&map_k);
            prefetch_map(&map_v);
            prefetch_map(&map_do);
            sh.abort = 0;
            mbar_init(smem_u32(&sh.q_full), 1);
            for (int i = 0; i < F::kStages; ++i) {
                mbar_init(smem_u32(&sh.full[i]), 1);
                mbar_init(smem_u32(&sh.empty[i]), 1);
            }
            for (int w = 0; w < 2; ++w) {
                mbar_init(smem_u32(&sh.sd_full[w]), 1);
                mbar_init(smem_u32(&sh.ds_full[w]), 4);
            }
            mbar_init(smem_u32(&sh.done), 1);
            mbar_init(smem_u32(&sh.clean), 1);
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
    if (!sh.at.valid) {
        if (warp == 9) tmem_free(tmem, 512);
        return;
    }
    const int n_tiles = sh.at.n_tiles, a_end = sh.at.a_end, b0 = sh.at.b0, kn = sh.at.kn, prefix = sh.at.prefix;
    const int n_sub = sh.at.n_sub, kv_head = sh.at.kv_head;
    const bool full_head = a.full[kv_head] != 0;
    const uint32_t q_smem = smem_u32(smem), o_smem = q_smem + 2 * F::kRowTile, ring = q_smem + 4 * F::kRowTile;
    auto tile_at = [&](int j) { return j < a_end ? j : b0 + j - a_end; };

    if (warp < 8) {
        // ------------------------------------------------------------------ P and dS, one thread per query
        const int w = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t S = tmem + lanes + w * 128, dP = S + 64;
        const int first = sh.at.pos0[w], pos = first + row, last = first + kRows - 1, head = sh.at.head[w];
        const bool mine = row < sh.at.rows[w];
        const int hi = min(kn, max(pos + 1, prefix)), lo = full_head ? 0 : pos - a.window + 1, sink = full_head ? 0 : min(a.sink, hi);
        const Cap cap(CAP ? a.softcap : 1.f, a.scale);
        const float sl2 = a.scale * kLog2e;
        const float slope2 = BIAS ? a.slopes[head] * kLog2e : 0.f;
        const int q = sh.at.q0[w] + row;
        float2* stat_at = a.stats + (long long)head * a.q_tokens + q;
        const float2 stat = mine ? *stat_at : make_float2(INFINITY, 0.f);
        float2 excess = make_float2(0.f, 0.f);  // sum of P (dP - D): zero but for the rounding of `out` that D comes from
        bool ok = true;
        int done = 0;
        const int sub_a = sh.at.sub_a[w], sub_b = sh.at.sub_b[w], sub_e = sh.at.sub_e[w];
        for (int t = sub_a > 0 ? 0 : sub_b; t < sub_e; t = t + 1 == sub_a ? sub_b : t + 1) {
            const int start = t * kCols;
            ok = wait(smem_u32(&sh.sd_full[w]), done & 1, abort_flag, a.status, kPromptWaitProduct);
            if (!ok) break;
            fence_after();
            const bool plain = start + kCols <= kn && (start + kCols <= first + 1 || start + kCols <= prefix) &&
                               (full_head || start + kCols <= a.sink || start > last - a.window);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float s[32], f[CAP ? 32 : 1];
                tmem_read32(S + half * 32, s);
                capped<CAP>(cap, sl2, mine, s, f);
                const int c0 = start + half * 32;
                if (BIAS) {
#pragma unroll
                    for (int c = 0; c < 32; ++c) s[c] = fmaf(-slope2, fabsf((float)(pos - c0 - c)), s[c]);
                }
#pragma unroll
                for (int c = 0; c < 32; ++c) s[c] = ex2(s[c] - stat.x);
                if (!plain) {
                    const uint32_t see = range_bits(lo - c0, hi - c0) | range_bits(0, sink - c0);
#pragma unroll
                    for (int c = 0; c < 32; ++c) s[c] = see >> c & 1 ? s[c] : 0.f;
                }
                float d[32];
                tmem_read32(dP + half * 32, d);
                uint32_t packed[16];
#pragma unroll
                for (int c = 0; c < 32; c += 2) {
                    const float2 ds = mul2(make_float2(s[c], s[c + 1]), add2(make_float2(d[c], d[c + 1]), make_float2(-stat.y, -stat.y)));
                    excess = add2(excess, ds);
                    d[c] = ds.x;
                    d[c + 1] = ds.y;
                    if constexpr (CAP) {
                        d[c] *= f[c];
                        d[c + 1] *= f[c + 1];
                    }
                    packed[c / 2] = bf16x2(d[c], d[c + 1]);
                }
                tmem_st16(dP + half * 16, packed);
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
            write_rows<D>(smem + w * F::kRowTile + part * D * 2, tmem + lanes + 256 + w * D, a.scale, done > 0,
                          a.dq + ((long long)(sh.at.q0[w] + part) * a.q_heads + head) * D, (long long)a.q_heads * D, sh.at.rows[w] - part, lane);
        }
    } else if (warp == 8) {
        // ------------------------------------------------------------------ tile loads
        if (lane == 0 && n_tiles > 0) {
            mbar_expect_tx(smem_u32(&sh.q_full), 2 * n_sub * F::kRowTile);
            for (int w = 0; w < n_sub; ++w) {
                load_rows<D>(q_smem + w * F::kRowTile, kRows, &map_q, sh.at.head[w], sh.at.q0[w], smem_u32(&sh.q_full));
                load_rows<D>(o_smem + w * F::kRowTile, kRows, &map_do, sh.at.head[w], sh.at.q0[w], smem_u32(&sh.q_full));
            }
            int j = 0;
            bool ok = true;
            for (; j < n_tiles; ++j) {
                const int st = j % F::kStages;
                ok = wait(smem_u32(&sh.empty[st]), (j / F::kStages & 1) ^ 1, abort_flag, a.status, kPromptWaitStage);
                if (!ok) break;
                const uint32_t bar = smem_u32(&sh.full[st]), dst = ring + st * 2 * F::kColTile;
                mbar_expect_tx(bar, 2 * F::kColTile);
                const int token = sh.at.k0 + tile_at(j) * kCols;
                load_rows<D>(dst, kCols, &map_k, kv_head, token, bar);
                load_rows<D>(dst + F::kColTile, kCols, &map_v, kv_head, token, bar);
            }
            if (!ok || *abort_flag) {  // nothing of this CTA's copies may be in flight when it ends
                wait(smem_u32(&sh.q_full), 0, nullptr, a.status, kPromptWaitDrain);
                for (int i = max(0, j - F::kStages); i < j; ++i)
                    wait(smem_u32(&sh.full[i % F::kStages]), i / F::kStages & 1, nullptr, a.status, kPromptWaitDrain);
            }
        }
        __syncwarp();
        // rows behind the last key: only the last tile can hold any
        const int end = n_tiles - 1, rows = n_tiles > 0 ? kn - tile_at(end) * kCols : kCols;
        if (rows < kCols && !*abort_flag &&
            wait(smem_u32(&sh.full[end % F::kStages]), end / F::kStages & 1, abort_flag, a.status, kPromptWaitLoad)) {
            uint8_t* x = smem + 4 * F::kRowTile + end % F::kStages * 2 * F::kColTile;
            for (int i = rows * 8 + lane; i < kCols * 8; i += 32)
                for (int b = 0; b < 2 * D / 64; ++b) *reinterpret_cast<uint4*>(x + b * kColBlock + i * 16) = make_uint4(0, 0, 0, 0);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.clean));
        }
    } else if (warp == 9) {
        // ------------------------------------------------------------------ matrix products
        if (n_tiles > 0) {
            constexpr uint32_t kScores = instr_desc(kRows, kCols, false), kGrads = instr_desc(kRows, D, true);
            int used[2] = {0, 0};
            const int sub_a[2] = {sh.at.sub_a[0], sh.at.sub_a[1]}, sub_b[2] = {sh.at.sub_b[0], sh.at.sub_b[1]}, sub_e[2] = {sh.at.sub_e[0], sh.at.sub_e[1]};
            auto needed = [&](int w, int t) { return t < sub_a[w] || (t >= sub_b[w] && t < sub_e[w]); };
            auto signal = [&](uint64_t* bar) {
                if (elect_one()) commit(smem_u32(bar));
            };
            auto loaded = [&](int j) {
                return wait_warp(smem_u32(&sh.full[j % F::kStages]), j / F::kStages & 1, abort_flag, a.status, kPromptWaitLoad) &&
                       ((tile_at(j) + 1) * kCols <= kn || wait_warp(smem_u32(&sh.clean), 0, abort_flag, a.status, kPromptWaitLoad));
            };
            auto first_products = [&](int w, int j) {
                const uint64_t k = smem_desc(ring + j % F::kStages * 2 * F::kColTile), v = smem_desc(ring + j % F::kStages * 2 * F::kColTile + F::kColTile);
                const uint64_t q = smem_desc(q_smem + w * F::kRowTile), o = smem_desc(o_smem + w * F::kRowTile);
                const uint32_t d = tmem + w * 128;
                if (elect_one()) {
#pragma unroll
                    for (int x = 0; x < D / 16; ++x)
                        mma_ss(d, q + ((x / 4 * kRowBlock + x % 4 * 32) >> 4), k + ((x / 4 * kColBlock + x % 4 * 32) >> 4), kScores, x > 0);
#pragma unroll
                    for (int x = 0; x < D / 16; ++x)
                        mma_ss(d + 64, o + ((x / 4 * kRowBlock + x % 4 * 32) >> 4), v + ((x / 4 * kColBlock + x % 4 * 32) >> 4), kScores, x > 0);
                    commit(smem_u32(&sh.sd_full[w]));
                }
            };
            bool ok = wait_warp(smem_u32(&sh.q_full), 0, abort_flag, a.status, kPromptWaitLoad) && loaded(0);
            if (ok)
                for (int w = 0; w < 2; ++w)
                    if (needed(w, tile_at(0))) first_products(w, 0);
            for (int j = 0; ok && j < n_tiles; ++j) {
                const int st = j % F::kStages;
                if (j + 1 < n_tiles) ok = loaded(j + 1);
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    if (!ok) break;
                    if (needed(w, tile_at(j))) {
                        ok = wait_warp(smem_u32(&sh.ds_full[w]), used[w] & 1, abort_flag, a.status, kPromptWaitSoftmax);
                        if (!ok) break;
                        fence_after();
                        const uint64_t k = smem_desc(ring + st * 2 * F::kColTile, kColBlock);
                        if (elect_one()) {
#pragma unroll
                            for (int x = 0; x < kCols / 16; ++x)
                                mma_ts(tmem + 256 + w * D, tmem + w * 128 + 64 + x * 8, k + (x * 2048 >> 4), kGrads, used[w] > 0 || x > 0);
                        }
                        ++used[w];
                    }
                    if (w == 1) signal(&sh.empty[st]);
                    if (j + 1 < n_tiles && needed(w, tile_at(j + 1))) first_products(w, j + 1);
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
    prompt_rows_kernel<D, CAP, BIAS><<<(unsigned)row_tile_blocks(a), kThreads, RowsK<D>::kSmem, stream>>>(a, m.q, m.k, m.v, m.dout);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    // Few key tiles: the query heads of a KV head go to several CTAs, as many (a divisor of the group) as leave no more than
    // four per SM.  A causal document's first key tile is seen by all its queries, so this also evens out the CTAs' work.
    const long long tiles = ((long long)a.k_tokens / kRows + (a.n_docs < a.k_tokens ? a.n_docs : a.k_tokens)) * a.kv_heads;
    int split = 1;
    for (int x = 2; x <= a.group; ++x)
        if (a.group % x == 0 && tiles * x <= 4 * 148) split = x;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * split));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Keys<D>::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = split > 1 ? 1 : 0;
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
