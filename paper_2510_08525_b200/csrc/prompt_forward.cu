// The forward pass of prompt attention on the tensor cores.
//
// One CTA takes two sub-tiles of 128 query rows -- the same queries of two heads of a KV head where the heads pair up,
// else 256 queries of one head -- and walks the 128-key tiles that any of them sees.  Per key tile and sub-tile: S = Q.K^T (128 x 128, both operands in shared memory, fp32 in
// tensor memory); a warpgroup, one thread per query row, turns S into P = exp2(s - m) and writes it as bf16 over S;
// O += P.V with P read from tensor memory.  Two sub-tiles so that one's products run while the other's softmax does.
//
//   warps 0-3, 4-7   softmax of sub-tile 0 / 1, and its output rows at the end
//   warp 8           TMA: Q once, then K and V tiles in turn through one ring; clears the rows behind the document's
//                    last key (0 * NaN of a neighbour would be NaN)
//   warp 9           issues every tcgen05.mma (in order, so S of the next tile may overwrite P of this one)
//
// Tensor memory: S/P of the sub-tiles at columns 0 and 128, O at 256 and 256 + D.
// Measured (32 / 8 heads of 128, causal): 8192 tokens 450 us in bursts, 1.22 PFLOP/s of visible products, 74 % of what a large
// library product reaches in bursts; 510 to 520 us over a run of passes, where the power cap holds the clocks down (1.07 PFLOP/s,
// 76 % of the library's rate over seconds).  Half of a 128 x 128 x 128 score product's time is spent at the full rate of shared
// memory (both operands come from there), and a sub-tile's chain -- products, softmax, hand-overs -- takes 3200 cycles where the
// two sub-tiles' products take 2048: the chain bounds it, and what lengthens it shows (8192 tokens with a distance term 615 us,
// with a cap 630).  24 documents of 333 tokens on average, half of the heads compressed, capped: 117 us, two thirds of it set-up,
// first loads and results of CTAs that see two or three key tiles.
// Tried and dropped: CTAs that stay and claim items, with the next item's loads early (8 % and 19 % slower: results can then not
// go out as whole rows, and the issuing warp runs out of registers); exponentials against the old maximum while the new one is
// looked for (5 % slower); two threads per row in four softmax warpgroups, which halves a thread's work but adds an exchange of
// the maxima to every tile (8192 tokens 481 us against 455 in bursts, 534 against 494 over a run; 24 documents the same).
// The running maximum of a row moves only when it would grow by more than 2^8 (a published idea; its effect cancels in O / l;
// P <= 256 and O, l are fp32), so the correction of O in tensor memory is rare after the first tile.  P is rounded to bf16 for
// the product; l sums the fp32 values.
#include "rlkv_prompt.cuh"
#include "tcgen05.cuh"

namespace rlkv {
namespace {

using namespace tc;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kRows = 128;          // queries of a sub-tile, keys of a tile
constexpr int kBlock = kRows * 128; // bytes of a [128 rows][64 elements] block

template <int D>
struct Fwd {
    static constexpr int kTileBytes = kRows * D * 2;
    static constexpr int kStages = D == 128 ? 5 : 10;  // K and V tiles in the ring
    static constexpr int kSmem = (2 + kStages) * kTileBytes + 1024;
    static constexpr int kThreads = 384;
};

struct FwdShared {
    uint64_t q_full, full[10], empty[10], s_full[2], p_full[2][2], pv_done[2], clean[2], drain;
    uint32_t tmem;
    int abort;
    RowTile at;
};

// P = 2^(s factor - base) of a row's 128 scores, as bf16 to tensor memory, and their sums.  64 keys at a time, so that
// the product starts on the first.  (A polynomial on the FMA pipe for a quarter or half of the exponentials, to spare the
// exponential unit, measured 4 to 8 % slower: with one warp per scheduler and sub-tile it is the instructions that count.)
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
            s[c + i] = ex2(s[c + i]);
            s[c + i + 1] = ex2(s[c + i + 1]);
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
    for (int c = 0; c < kRows; c += 2) sum[c / 2 & 1] = add2(sum[c / 2 & 1], make_float2(s[c], s[c + 1]));
}

template <int D, bool CAP, bool BIAS>
__global__ void __launch_bounds__(Fwd<D>::kThreads, 1)
prompt_forward_kernel(const __grid_constant__ PromptArgs a, const __grid_constant__ CUtensorMap map_q,
                      const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v)
{
    using F = Fwd<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    static_assert(sizeof(FwdShared) <= 1024 && F::kSmem <= kMaxDynamicSmem, "shared memory");
    FwdShared& sh = *reinterpret_cast<FwdShared*>(smem + (2 + F::kStages) * F::kTileBytes);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    volatile int* abort_flag = &sh.abort;

    if ((smem_u32(smem) & 1023u) != 0) {
        if (tid == 0) atomicCAS(a.status, 0, kPromptSmemMisaligned);
        return;
    }
    if (warp == 0) {
        find_row_tile(a, kRows, sh.at);
    } else if (warp == 8) {
        if (lane == 0) {
            prefetch_map(&map_q);
            prefetch_map(&map_k);
            prefetch_map(&map_v);
            sh.abort = 0;
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
            mbar_init(smem_u32(&sh.clean[0]), 1);
            mbar_init(smem_u32(&sh.clean[1]), 1);
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
    const uint32_t q_smem = smem_u32(smem), ring = q_smem + 2 * F::kTileBytes;
    auto tile_at = [&](int j) { return j < a_end ? j : b0 + j - a_end; };
    // (launched with 384 x 168 = 64512 registers: 256 x 232 + 128 x 40)
    if (warp < 8) more_registers<232>();
    else fewer_registers<40>();
    if (warp < 8) {
        // ------------------------------------------------------------------ softmax
        const int w = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t S = tmem + lanes + w * kRows, O = tmem + lanes + 2 * kRows + w * D;
        const int first = sh.at.pos0[w], last = first + kRows - 1, pos = first + row, head = sh.at.head[w];
        const bool mine = row < sh.at.rows[w];  // else the row is another document's, or behind the last one
        const int hi = min(kn, max(pos + 1, prefix)), lo = full_head ? 0 : pos - a.window + 1, sink = full_head ? 0 : min(a.sink, hi);
        const float sl2 = a.scale * kLog2e, factor = CAP || BIAS ? 1.f : sl2;
        const float slope2 = BIAS ? a.slopes[head] * kLog2e : 0.f;
        const int sub_a = sh.at.sub_a[w], sub_b = sh.at.sub_b[w], sub_e = sh.at.sub_e[w];
        const Cap cap(CAP ? a.softcap : 1.f, a.scale);
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
                    // (rows behind the document's last key read as zero, so nothing another document holds has a say in how
                    // the warp computes the cap)
                    cap.apply(s, mine);
                }
                if (BIAS) {
                    // From the distance itself, a whole number and exact: slope * (start - pos) + slope * c would round at the size
                    // of its terms and lose the score of the keys next to the query where slopes are steep.
                    const float far = (float)(pos - start);
                    if (causal_past) {
                        float2 d[4];
#pragma unroll
                        for (int c = 0; c < 8; c += 2) d[c / 2] = make_float2((float)c - far, (float)(c + 1) - far);
#pragma unroll
                        for (int c = 0; c < kRows; c += 2) {
                            const float2 x = CAP ? make_float2(s[c], s[c + 1]) : mul2(make_float2(s[c], s[c + 1]), make_float2(sl2, sl2));
                            const float2 y = fma2(make_float2(slope2, slope2), d[c / 2 & 3], x);
                            s[c] = y.x;
                            s[c + 1] = y.y;
                            d[c / 2 & 3] = add2(d[c / 2 & 3], make_float2(8.f, 8.f));
                        }
                    } else {
#pragma unroll
                        for (int c = 0; c < kRows; ++c) s[c] = fmaf(-slope2, fabsf(far - (float)c), CAP ? s[c] : s[c] * sl2);
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
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                exponentials(s, factor, base, sum, S, sh.p_full[w], lane);
                l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                ++done;
            }
        if (ok && w < n_sub) {
            if (done > 0) {
                ok = wait(smem_u32(&sh.pv_done[w]), (done - 1) & 1, abort_flag, a.status, kPromptWaitProduct);
                fence_after();
            }
            if (ok) {
                const float inv = l > 0.f ? 1.f / l : 0.f;  // (0: a row that sees nothing)
                const long long q0 = sh.at.q0[w];
                if (mine && a.lse) a.lse[(q0 + row) * a.q_heads + head] = l > 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
                // through shared memory (the sub-tile's queries are not needed any more), so that whole rows go out
                write_rows<D>(smem + w * F::kTileBytes + (warp & 3) * 32 * D * 2, O, inv, done > 0, a.out + (q0 + (warp & 3) * 32) * a.q_heads * D + head * D,
                              (long long)a.q_heads * D, sh.at.rows[w] - (warp & 3) * 32, lane);
            }
        }
    } else if (warp == 8) {
        // ------------------------------------------------------------------ tile loads
        if (lane == 0 && n_tiles > 0) {
            // (no queries for a sub-tile that sees no key beside one that does: its threads wait for no product, and the zeros of its
            // rows go out through the memory that the queries would be copied to)
            auto sees = [&](int w) { return sh.at.sub_a[w] > 0 || sh.at.sub_b[w] < sh.at.sub_e[w]; };
            mbar_expect_tx(smem_u32(&sh.q_full), ((int)sees(0) + (int)sees(1)) * F::kTileBytes);
            for (int w = 0; w < 2; ++w)
                for (int b = 0; sees(w) && b < D / 64; ++b)
                    load_box(q_smem + w * F::kTileBytes + b * kBlock, &map_q, b * 64, sh.at.head[w], sh.at.q0[w], smem_u32(&sh.q_full));
            int issued = 0;
            bool ok = true;
            for (; issued < 2 * n_tiles; ++issued) {
                const int slot = issued % F::kStages;
                ok = wait(smem_u32(&sh.empty[slot]), (issued / F::kStages & 1) ^ 1, abort_flag, a.status, kPromptWaitStage);
                if (!ok) break;
                mbar_expect_tx(smem_u32(&sh.full[slot]), F::kTileBytes);
                const int token = sh.at.k0 + tile_at(issued >> 1) * kRows;
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
        // rows behind the document's last key: only the last K and V tiles can hold any.  (This warp may wait for them: it has
        // seen their stages' earlier copies consumed)
        const int rows = n_tiles > 0 ? kn - tile_at(n_tiles - 1) * kRows : kRows;
        if (rows < kRows)
            for (int v = 0; v < 2; ++v) {
                const int last = 2 * n_tiles - 2 + v;
                if (*abort_flag || !wait(smem_u32(&sh.full[last % F::kStages]), last / F::kStages & 1, abort_flag, a.status, kPromptWaitLoad)) break;
                uint8_t* x = smem + (2 + last % F::kStages) * F::kTileBytes;
                for (int i = rows * 8 + lane; i < kRows * 8; i += 32)
                    for (int b = 0; b < D / 64; ++b) *reinterpret_cast<uint4*>(x + b * kBlock + i * 16) = make_uint4(0, 0, 0, 0);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh.clean[v]));
            }
    } else if (warp == 9) {
        // ------------------------------------------------------------------ matrix products
        if (n_tiles > 0) {
            constexpr uint32_t kQK = instr_desc(kRows, kRows, false), kPV = instr_desc(kRows, D, true);
            bool ok = true;
            int used[2] = {0, 0};  // P tiles of the sub-tile multiplied so far
            const int sub_a[2] = {sh.at.sub_a[0], sh.at.sub_a[1]}, sub_b[2] = {sh.at.sub_b[0], sh.at.sub_b[1]}, sub_e[2] = {sh.at.sub_e[0], sh.at.sub_e[1]};
            auto needed = [&](int w, int t) { return t < sub_a[w] || (t >= sub_b[w] && t < sub_e[w]); };
            auto stage = [&](int i) { return ring + i % F::kStages * F::kTileBytes; };
            // K (even) and V tiles in turn; the last two once the rows behind the last key have been cleared
            auto loaded = [&](int i) {
                return wait_warp(smem_u32(&sh.full[i % F::kStages]), i / F::kStages & 1, abort_flag, a.status, kPromptWaitLoad) &&
                       ((tile_at(i >> 1) + 1) * kRows <= kn || wait_warp(smem_u32(&sh.clean[i & 1]), 0, abort_flag, a.status, kPromptWaitLoad));
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
    prompt_forward_kernel<D, CAP, BIAS><<<(unsigned)row_tile_blocks(a), Fwd<D>::kThreads, Fwd<D>::kSmem, stream>>>(a, q, k, v);
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
