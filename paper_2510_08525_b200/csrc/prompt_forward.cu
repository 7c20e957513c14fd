// The forward pass of prompt attention on the tensor cores.
//
// One CTA takes 256 queries of one head of one document -- two sub-tiles of 128 rows -- and walks the 128-key tiles
// that any of them sees.  Per key tile and sub-tile: S = Q.K^T (128 x 128, both operands in shared memory, fp32 in
// tensor memory); a warpgroup, one thread per query row, turns S into P = exp2(s - m) and writes it as bf16 over S;
// O += P.V with P read from tensor memory.  Two sub-tiles so that one's products run while the other's softmax does.
//
//   warps 0-3, 4-7   softmax of sub-tile 0 / 1, and its output rows at the end
//   warp 8           TMA: Q once, then K and V tiles in turn through one ring; clears the V rows behind the document's
//                    last key (0 * NaN of a neighbour would be NaN)
//   warp 9           issues every tcgen05.mma (in order, so S of the next tile may overwrite P of this one)
//
// Tensor memory: S/P of the sub-tiles at columns 0 and 128, O at 256 and 256 + D.
// The running maximum of a row moves only when it would grow by more than 2^8 (its effect cancels in O / l; P <= 256 and
// O, l are fp32), so the correction of O in tensor memory is rare after the first tile.  P is rounded to bf16 for the
// product; l sums the fp32 values.
#include "rlkv_prompt.cuh"
#include "tcgen05.cuh"

namespace rlkv {
namespace {

using namespace tc;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kRows = 128;          // queries of a sub-tile, keys of a tile
constexpr int kPolyPairs = 4;      // the exponential unit alone would need as long as the tensor core
constexpr int kBlock = kRows * 128; // bytes of a [128 rows][64 elements] block

template <int D>
struct Fwd {
    static constexpr int kTileBytes = kRows * D * 2;
    static constexpr int kStages = D == 128 ? 5 : 10;  // K and V tiles in the ring
    static constexpr int kSmem = (2 + kStages) * kTileBytes + 1024;
    static constexpr int kThreads = 384;
};

struct FwdShared {
    uint64_t q_full, full[10], empty[10], s_full[2], p_full[2][2], pv_done[2], clean, drain;
    uint32_t tmem;
    int abort, valid;
    int q0, rows, pos0, k0, kn, prefix;    // the CTA's queries, its document's keys
    int a_end, b0, n_tiles;                // its key tiles: 0 .. a_end-1, then from b0 on
    int sub_a[2], sub_b[2], sub_e[2];      // those a sub-tile needs: 0 .. a-1 and b .. e-1
};

// P = 2^(s factor - base) of a row's 128 scores, as bf16 to tensor memory, and their sums; POLY > 0: one pair in POLY on
// the FMA pipe.  64 keys at a time, so that the product starts on the first.
template <int POLY>
__device__ __forceinline__ void exponentials(float (&s)[kRows], float factor, float base, float2 (&sum)[2], uint32_t P, uint64_t* done, int lane)
{
    const float2 factor2 = make_float2(factor, factor), base2 = make_float2(-base, -base);
#pragma unroll
    for (int c = 0; c < kRows; c += 32) {
        uint32_t packed[16];
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            const float2 x = fma2(make_float2(s[c + i], s[c + i + 1]), factor2, base2);
            s[c + i] = x.x;
            s[c + i + 1] = x.y;
        }
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            float2 p = make_float2(s[c + i], s[c + i + 1]);
            if (POLY > 0 && i / 2 % (POLY > 0 ? POLY : 1) == POLY - 1) p = exp2_fma(p);
            else p = make_float2(ex2(p.x), ex2(p.y));
            s[c + i] = p.x;
            s[c + i + 1] = p.y;
            packed[i / 2] = bf16x2(p.x, p.y);
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
    for (int c = 0; c < kRows; c += 2) sum[c / 2 & 1] = add2(sum[c / 2 & 1], make_float2(s[c], s[c + 1]));
}

template <int D, bool CAP, bool BIAS>
__global__ void __launch_bounds__(Fwd<D>::kThreads, 1)
prompt_forward_kernel(const __grid_constant__ PromptArgs a, const __grid_constant__ CUtensorMap map_q,
                      const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v)
{
    using F = Fwd<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    FwdShared& sh = *reinterpret_cast<FwdShared*>(smem + (2 + F::kStages) * F::kTileBytes);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int head = blockIdx.x % a.q_heads, kv_head = head / a.group;
    const bool full_head = a.full[kv_head] != 0;
    volatile int* abort_flag = &sh.abort;

    if ((smem_u32(smem) & 1023u) != 0) {
        if (tid == 0) atomicCAS(a.status, 0, kPromptSmemMisaligned);
        return;
    }
    if (warp == 0) {
        int doc = 0, tile = 0;
        const bool valid = find_tile(a, false, 2 * kRows, blockIdx.x / a.q_heads, doc, tile);
        if (lane == 0) {
            sh.valid = valid;
            sh.abort = 0;
            if (valid) {
                const DocRange r = doc_range(a, doc);
                sh.q0 = r.q0 + tile * 2 * kRows;
                sh.rows = min(2 * kRows, r.qn - tile * 2 * kRows);
                sh.pos0 = tile * 2 * kRows + r.kn - r.qn;
                sh.k0 = r.k0;
                sh.kn = r.kn;
                sh.prefix = r.prefix;
                const int hi = min(r.kn, max(sh.pos0 + sh.rows, r.prefix));
                const int end = hi > 0 ? (hi + kRows - 1) / kRows : 0;
                int a_end = end, b0 = end;
                if (!full_head) {
                    a_end = min(end, (min(a.sink, max(hi, 0)) + kRows - 1) / kRows);
                    b0 = max(a_end, max(0, sh.pos0 - a.window + 1) / kRows);
                }
                sh.a_end = a_end;
                sh.b0 = b0;
                sh.n_tiles = a_end + max(0, end - b0);
                for (int w = 0; w < 2; ++w) {
                    const int rows = min(kRows, sh.rows - w * kRows), first = sh.pos0 + w * kRows;
                    const int seen = rows > 0 ? max(0, min(r.kn, max(first + rows, r.prefix))) : 0;
                    const int e = (seen + kRows - 1) / kRows;
                    sh.sub_a[w] = full_head ? e : min(e, (a.sink + kRows - 1) / kRows);
                    sh.sub_b[w] = max(sh.sub_a[w], max(0, first - a.window + 1) / kRows);
                    sh.sub_e[w] = max(e, sh.sub_b[w]);
                }
            }
            mbar_init(smem_u32(&sh.q_full), 1);
            for (int i = 0; i < F::kStages; ++i) {
                mbar_init(smem_u32(&sh.full[i]), 1);
                mbar_init(smem_u32(&sh.empty[i]), 1);
            }
            for (int w = 0; w < 2; ++w) {
                mbar_init(smem_u32(&sh.s_full[w]), 1);
                mbar_init(smem_u32(&sh.p_full[w][0]), 4);
                mbar_init(smem_u32(&sh.p_full[w][1]), 4);
                mbar_init(smem_u32(&sh.pv_done[w]), 1);
            }
            mbar_init(smem_u32(&sh.clean), 1);
            mbar_init(smem_u32(&sh.drain), 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
    }
    __syncthreads();
    if (!sh.valid) return;
    if (warp == 9) tmem_alloc(smem_u32(&sh.tmem), 512);
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = sh.tmem;
    const int n_tiles = sh.n_tiles, a_end = sh.a_end, b0 = sh.b0, kn = sh.kn, prefix = sh.prefix;
    const uint32_t q_smem = smem_u32(smem), ring = q_smem + 2 * F::kTileBytes;
    const int n_sub = sh.rows > kRows ? 2 : 1;
    auto tile_at = [&](int j) { return j < a_end ? j : b0 + j - a_end; };
    // (launched with 384 x 168 = 64512 registers: 256 x 216 + 128 x 72)
    if (warp < 8) more_registers<216>();
    else fewer_registers<72>();
    if (warp < 8) {
        // ------------------------------------------------------------------ softmax
        const int w = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t S = tmem + lanes + w * kRows, O = tmem + lanes + 2 * kRows + w * D;
        const int pos = sh.pos0 + w * kRows + row;
        const bool mine = w * kRows + row < sh.rows;  // else the row is another document's, or behind the last one
        const int first = sh.pos0 + w * kRows, last = first + kRows - 1;
        const int hi = min(kn, max(pos + 1, prefix)), lo = full_head ? 0 : pos - a.window + 1, sink = full_head ? 0 : min(a.sink, hi);
        const float sl2 = a.scale * kLog2e, factor = CAP || BIAS ? 1.f : sl2;
        const float slope2 = BIAS ? a.slopes[head] * kLog2e : 0.f;
        const int sub_a = sh.sub_a[w], sub_b = sh.sub_b[w], sub_e = sh.sub_e[w];
        float m = -INFINITY, l = 0.f;
        int done = 0;  // tiles of this sub-tile so far
        bool ok = true;
        if (w < n_sub)
            for (int t = sub_a > 0 ? 0 : sub_b; t < sub_e; t = t + 1 == sub_a ? sub_b : t + 1) {
                const int start = t * kRows;
                ok = wait(smem_u32(&sh.s_full[w]), done & 1, abort_flag, a.status, kPromptWaitProduct);
                if (!ok) break;
                fence_after();
                float s[kRows];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(S + c * 32, s + c * 32);
                wait_ld();
#pragma unroll
                for (int c = 0; c < kRows; ++c) asm volatile("" : "+f"(s[c]));  // nothing of the above is used before the wait
                const bool causal_past = start + kRows <= first + 1;  // every key at or before every query
                const bool plain = start + kRows <= kn && (causal_past || start + kRows <= prefix) &&
                                   (full_head || start + kRows <= a.sink || start > last - a.window);
                uint32_t see[4];  // the keys this row sees, 32 to a word
                if (!plain) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        see[c] = mine ? range_bits(lo - start - c * 32, hi - start - c * 32) | range_bits(0, sink - start - c * 32) : 0u;
                }
                if (CAP) {
                    // what the row does not see has no say in how its warp computes the cap (nothing another document holds
                    // may change a bit of this one's result)
                    if (!plain) {
#pragma unroll
                        for (int c = 0; c < kRows; ++c) s[c] = see[c / 32] >> (c & 31) & 1 ? s[c] : 0.f;
                    }
                    // cap tanh(z) in the log2 domain.  Small z (most scores are far below the cap): the Taylor series,
                    // off by 1e-8 of z at 0.3, on the FMA pipe; else 1 - 2 / (1 + e^2z) with its exp2 and division
                    const float cap2 = a.softcap * kLog2e, zs = a.scale / a.softcap;
                    float big = 0.f;
#pragma unroll
                    for (int c = 0; c < kRows; ++c) big = fmaxf(big, fabsf(s[c]));
                    if (__any_sync(0xffffffffu, mine && big * zs > 0.3f)) {
                        const float e2 = 2.f * kLog2e * zs;
#pragma unroll
                        for (int c = 0; c < kRows; ++c) s[c] = cap2 - __fdividef(2.f * cap2, 1.f + ex2(s[c] * e2));
                    } else {
#pragma unroll
                        for (int c = 0; c < kRows; ++c) {
                            const float z = s[c] * zs, y = z * z;
                            const float f = fmaf(y, fmaf(y, fmaf(y, fmaf(y, 62.f / 2835, -17.f / 315), 2.f / 15), -1.f / 3), 1.f);
                            s[c] = z * cap2 * f;
                        }
                    }
                }
                if (BIAS) {
                    if (causal_past) {  // -slope (pos - start - c): linear in the column
                        const float t0 = slope2 * (float)(start - pos);
#pragma unroll
                        for (int c = 0; c < kRows; ++c) s[c] = fmaf(slope2, (float)c, CAP ? s[c] + t0 : fmaf(s[c], sl2, t0));
                    } else {
#pragma unroll
                        for (int c = 0; c < kRows; ++c) s[c] = fmaf(-slope2, fabsf((float)(pos - start - c)), CAP ? s[c] : s[c] * sl2);
                    }
                }
                if (!plain) {
#pragma unroll
                    for (int c = 0; c < kRows; ++c) s[c] = see[c / 32] >> (c & 31) & 1 ? s[c] : -INFINITY;
                }
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < kRows; ++c) mx[c & 3] = fmaxf(mx[c & 3], s[c]);
                const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * factor;
                float corr = 1.f;
                if (top > m + 8.f) {  // (m may still be -infinity: then there is nothing to correct)
                    corr = m == -INFINITY ? 1.f : ex2(m - top);
                    m = top;
                    l *= corr;
                }
                if (done > 0 && __any_sync(0xffffffffu, corr != 1.f)) {
                    ok = wait(smem_u32(&sh.pv_done[w]), (done - 1) & 1, abort_flag, a.status, kPromptWaitProduct);
                    if (!ok) break;
                    fence_after();
#pragma unroll
                    for (int c = 0; c < D; c += 32) {
                        float o[32];
                        tmem_ld32(O + c, o);
                        wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            asm volatile("" : "+f"(o[i]));
                            o[i] *= corr;
                        }
                        tmem_st32(O + c, o);
                    }
                }
                const float base = m == -INFINITY ? 0.f : m;
                // (where every key is seen: the FMA pipe's exponential wants finite arguments)
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                if (plain) exponentials<kPolyPairs>(s, factor, base, sum, S, sh.p_full[w], lane);
                else exponentials<0>(s, factor, base, sum, S, sh.p_full[w], lane);
                l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                ++done;
            }
        if (ok && w < n_sub) {
            const long long at = (long long)(sh.q0 + w * kRows + row) * a.q_heads + head;
            if (done > 0) {
                ok = wait(smem_u32(&sh.pv_done[w]), (done - 1) & 1, abort_flag, a.status, kPromptWaitProduct);
                fence_after();
            }
            if (ok) {
                const float inv = l > 0.f ? 1.f / l : 0.f;
                if (mine && a.lse) a.lse[at] = l > 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
#pragma unroll
                for (int c = 0; c < D; c += 32) {
                    float o[32];
                    if (done > 0) {
                        tmem_ld32(O + c, o);
                        wait_ld();
                    }
                    uint32_t x[16];
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        asm volatile("" : "+f"(o[i]));
                        if (inv == 0.f) o[i] = 0.f;  // a row that sees nothing
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = bf16x2(o[2 * i] * inv, o[2 * i + 1] * inv);
                    if (mine) {
                        uint4* dst = reinterpret_cast<uint4*>(a.out + at * D + c);
#pragma unroll
                        for (int i = 0; i < 4; ++i) dst[i] = make_uint4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
                    }
                }
            }
        }
    } else if (warp == 8) {
        // ------------------------------------------------------------------ tile loads
        if (lane == 0 && n_tiles > 0) {
            mbar_expect_tx(smem_u32(&sh.q_full), n_sub * F::kTileBytes);
            for (int w = 0; w < n_sub; ++w)
                for (int b = 0; b < D / 64; ++b)
                    load_box(q_smem + w * F::kTileBytes + b * kBlock, &map_q, b * 64, head, sh.q0 + w * kRows, smem_u32(&sh.q_full));
            int issued = 0;
            bool ok = true;
            for (; issued < 2 * n_tiles; ++issued) {
                const int slot = issued % F::kStages;
                ok = wait(smem_u32(&sh.empty[slot]), (issued / F::kStages & 1) ^ 1, abort_flag, a.status, kPromptWaitStage);
                if (!ok) break;
                mbar_expect_tx(smem_u32(&sh.full[slot]), F::kTileBytes);
                const int token = sh.k0 + tile_at(issued >> 1) * kRows;
                for (int b = 0; b < D / 64; ++b)
                    load_box(ring + slot * F::kTileBytes + b * kBlock, issued & 1 ? &map_v : &map_k, b * 64, kv_head, token,
                             smem_u32(&sh.full[slot]));
            }
            if (!ok || *abort_flag) {  // nothing of this CTA's copies may be in flight when it ends
                wait(smem_u32(&sh.q_full), 0, nullptr, a.status, kPromptWaitDrain);
                for (int i = max(0, issued - F::kStages); i < issued; ++i)
                    wait(smem_u32(&sh.full[i % F::kStages]), i / F::kStages & 1, nullptr, a.status, kPromptWaitDrain);
            }
        }
        __syncwarp();
        // the last tile copied is V's last; it is the only one that can reach past the keys.  (This warp may wait for it:
        // it has seen the stage's earlier copies consumed)
        const int last = 2 * n_tiles - 1, rows = n_tiles > 0 ? kn - tile_at(n_tiles - 1) * kRows : kRows;
        if (rows < kRows && !*abort_flag &&
            wait(smem_u32(&sh.full[last % F::kStages]), last / F::kStages & 1, abort_flag, a.status, kPromptWaitLoad)) {
            uint8_t* v = smem + (2 + last % F::kStages) * F::kTileBytes;
            for (int x = rows * 8 + lane; x < kRows * 8; x += 32)
                for (int b = 0; b < D / 64; ++b) *reinterpret_cast<uint4*>(v + b * kBlock + x * 16) = make_uint4(0, 0, 0, 0);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.clean));
        }
    } else if (warp == 9) {
        // ------------------------------------------------------------------ matrix products
        if (n_tiles > 0) {
            constexpr uint32_t kQK = instr_desc(kRows, kRows, false), kPV = instr_desc(kRows, D, true);
            bool ok = true;
            int used[2] = {0, 0};  // P tiles of the sub-tile multiplied so far
            const int sub_a[2] = {sh.sub_a[0], sh.sub_a[1]}, sub_b[2] = {sh.sub_b[0], sh.sub_b[1]}, sub_e[2] = {sh.sub_e[0], sh.sub_e[1]};
            auto needed = [&](int w, int t) { return t < sub_a[w] || (t >= sub_b[w] && t < sub_e[w]); };
            auto stage = [&](int i) { return ring + i % F::kStages * F::kTileBytes; };
            auto loaded = [&](int i) {
                return wait_warp(smem_u32(&sh.full[i % F::kStages]), i / F::kStages & 1, abort_flag, a.status, kPromptWaitLoad);
            };
            auto signal = [&](uint64_t* bar) {
                if (elect_one()) commit(smem_u32(bar));
            };
            auto scores = [&](int w, int j) {
                const uint64_t q = smem_desc(q_smem + w * F::kTileBytes), k = smem_desc(stage(2 * j));
                if (elect_one()) {
#pragma unroll
                    for (int x = 0; x < D / 16; ++x) {
                        const uint32_t off = (x / 4 * kBlock + x % 4 * 32) >> 4;
                        mma_ss(tmem + w * kRows, q + off, k + off, kQK, x > 0);
                    }
                    commit(smem_u32(&sh.s_full[w]));
                }
            };
            ok = wait_warp(smem_u32(&sh.q_full), 0, abort_flag, a.status, kPromptWaitLoad) && loaded(0);
            if (ok) {
                for (int w = 0; w < 2; ++w)
                    if (needed(w, tile_at(0))) scores(w, 0);
                signal(&sh.empty[0]);
            }
            for (int j = 0; ok && j < n_tiles; ++j) {
                const int t = tile_at(j);
                ok = loaded(2 * j + 1);
                if (ok && (t + 1) * kRows > kn) ok = wait_warp(smem_u32(&sh.clean), 0, abort_flag, a.status, kPromptWaitLoad);
                if (ok && j + 1 < n_tiles) ok = loaded(2 * j + 2);
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    if (!ok) break;
                    if (needed(w, t)) {
                        const uint64_t v = smem_desc(stage(2 * j + 1), kBlock);
                        for (int half = 0; half < 2; ++half) {
                            ok = wait_warp(smem_u32(&sh.p_full[w][half]), used[w] & 1, abort_flag, a.status, kPromptWaitSoftmax);
                            if (!ok) break;
                            fence_after();
                            if (elect_one()) {
#pragma unroll
                                for (int x = 0; x < kRows / 32; ++x) {
                                    const int y = half * (kRows / 32) + x;
                                    mma_ts(tmem + 2 * kRows + w * D, tmem + w * kRows + y * 8, v + (y * 2048 >> 4), kPV, used[w] > 0 || y > 0);
                                }
                            }
                        }
                        if (!ok) break;
                        signal(&sh.pv_done[w]);
                        ++used[w];
                    }
                    if (w == 1) signal(&sh.empty[(2 * j + 1) % F::kStages]);
                    if (j + 1 < n_tiles && needed(w, tile_at(j + 1))) scores(w, j + 1);
                }
                if (ok && j + 1 < n_tiles) signal(&sh.empty[(2 * j + 2) % F::kStages]);
            }
            // every product is done before tensor memory is given back
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

template <int D, bool CAP, bool BIAS>
cudaError_t launch_one(const PromptArgs& a, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, cudaStream_t stream)
{
    const long long tiles = (long long)a.q_tokens / (2 * kRows) + (a.n_docs < a.q_tokens ? a.n_docs : a.q_tokens);
    prompt_forward_kernel<D, CAP, BIAS><<<(unsigned)(tiles * a.q_heads), Fwd<D>::kThreads, Fwd<D>::kSmem, stream>>>(a, q, k, v);
    return cudaGetLastError();
}

template <int D>
cudaError_t launch_dim(const PromptArgs& a, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, cudaStream_t stream)
{
    if (a.softcap != 0.f) return a.slopes ? launch_one<D, true, true>(a, q, k, v, stream) : launch_one<D, true, false>(a, q, k, v, stream);
    return a.slopes ? launch_one<D, false, true>(a, q, k, v, stream) : launch_one<D, false, false>(a, q, k, v, stream);
}

template <int D>
cudaError_t prepare_dim()
{
    const void* kernels[] = {(const void*)prompt_forward_kernel<D, false, false>, (const void*)prompt_forward_kernel<D, false, true>,
                             (const void*)prompt_forward_kernel<D, true, false>, (const void*)prompt_forward_kernel<D, true, true>};
    for (const void* k : kernels) {
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, Fwd<D>::kSmem);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_prompt_forward(const PromptArgs& a, const CUtensorMap& map_q, const CUtensorMap& map_k, const CUtensorMap& map_v,
                                  int head_dim, cudaStream_t stream)
{
    return head_dim == 128 ? launch_dim<128>(a, map_q, map_k, map_v, stream) : launch_dim<64>(a, map_q, map_k, map_v, stream);
}

cudaError_t prepare_prompt_kernels(int head_dim) { return head_dim == 128 ? prepare_dim<128>() : prepare_dim<64>(); }

}  // namespace rlkv
