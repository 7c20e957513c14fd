// Wrappers of the sm_100a instructions prompt attention is built from: mbarriers with bounded waits, TMA tile
// loads, tcgen05 matrix products and tensor memory.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <stdint.h>

namespace rlkv {
namespace tc {

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ uint64_t now_ns()
{
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

constexpr uint64_t kWaitNs = 1000000000ull;  // a wait gives up after about a second ...

// ... and then records `code` in the device error word and tells the CTA's other warps to stop.  Returns false
// where this or another wait of the CTA gave up.
// (inlined: a call would have the softmax threads' 128 scores go through the stack)
__device__ __forceinline__ bool wait_slow(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status, int code)
{
    const uint64_t t0 = now_ns();
    for (;;) {
#pragma unroll 1
        for (int i = 0; i < 64; ++i)
            if (mbar_try_wait(bar, parity)) return true;
        if (abort_flag && *abort_flag) return false;
        if (now_ns() - t0 > kWaitNs) {
            if (abort_flag) *abort_flag = 1;
            atomicCAS(status, 0, code);
            return false;
        }
    }
}
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status, int code)
{
    if (mbar_try_wait(bar, parity)) return true;
    return wait_slow(bar, parity, abort_flag, status, code);
}

// The whole warp waits; the answer is the same in every lane (control flow after it stays uniform).
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status, int code)
{
    return __all_sync(0xffffffffu, wait(bar, parity, abort_flag, status, code));
}

// One lane of a converged warp, always the same.  Products are issued under it in warp-uniform code, so that their
// descriptors live in uniform registers: issued by `if (lane == 0)` each took about 100 cycles, longer than it ran.
__device__ __forceinline__ bool elect_one()
{
    uint32_t leader;
    asm volatile(
        "{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(leader)
        :
        : "memory");
    return leader != 0;
}

// A box of 64 elements (128 bytes, 128-byte swizzle) x 1 head x some tokens of a [tokens][heads][head_dim] tensor.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int element, int head, int token, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(element), "r"(head), "r"(token), "r"(bar)
        : "memory");
}

// ---- a cluster's CTAs ---------------------------------------------------------------------------------

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// Four floats at the same place of CTA `rank`'s shared memory.
__device__ __forceinline__ float4 load_cluster(uint32_t addr, int rank)
{
    float4 x;
    asm volatile(
        "{\n\t.reg .b32 p;\n\tmapa.shared::cluster.u32 p, %4, %5;\n\tld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [p];\n\t}"
        : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w)
        : "r"(addr), "r"(rank)
        : "memory");
    return x;
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

// Registers of a warpgroup's threads from here on (every warp of it executes this).
template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// ---- tcgen05 ----------------------------------------------------------------------------------------

__device__ __forceinline__ void tmem_alloc(uint32_t slot, uint32_t columns)  // a whole warp
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t columns)  // a whole warp
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns));
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Shared-memory operand, 128-byte swizzle: rows of 128 bytes, eight rows a group of 1024 bytes.  `lbo` matters only
// where the rows are the contraction index (the operand's other index runs along the 128 bytes): bytes from one block
// of 64 elements to the next.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lbo = 16)
{
    return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)((lbo & 0x3ffff) >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 |
           2ull << 61;
}
// bf16 x bf16 -> fp32, M x N; `b_rows`: B's rows in shared memory are the contraction index.
__host__ __device__ constexpr uint32_t instr_desc(int m, int n, bool b_rows)
{
    return 1u << 4 | 1u << 7 | 1u << 10 | (b_rows ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}

// 32 columns of the warp's 32 lanes: lane l of the warp gets lane l's columns.
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float* r)
{
    uint32_t* u = reinterpret_cast<uint32_t*>(r);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]),
          "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]),
          "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]),
          "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t* u)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr), "r"(u[0]),
        "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]), "r"(u[10]), "r"(u[11]),
        "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const float* r)
{
    const uint32_t* u = reinterpret_cast<const uint32_t*>(r);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(
            addr),
        "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]), "r"(u[10]),
        "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]), "r"(u[16]), "r"(u[17]), "r"(u[18]), "r"(u[19]), "r"(u[20]),
        "r"(u[21]), "r"(u[22]), "r"(u[23]), "r"(u[24]), "r"(u[25]), "r"(u[26]), "r"(u[27]), "r"(u[28]), "r"(u[29]), "r"(u[30]),
        "r"(u[31])
        : "memory");
}

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}

// 32 columns, usable at once.
__device__ __forceinline__ void tmem_read32(uint32_t addr, float (&s)[32])
{
    tmem_ld32(addr, s);
    wait_ld();
#pragma unroll
    for (int c = 0; c < 32; ++c) asm volatile("" : "+f"(s[c]));  // nothing of it is used before the wait
}

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}


// A warp's 32 result rows of D columns in tensor memory, times `scale` (each row its own), rounded to bf16, to rows
// `stride` elements apart, the first `valid` of them.  `stage`: the warp's 32 * D * 2 bytes of shared memory: a thread
// holds one row, and storing it as it is would touch 32 rows per instruction.  `any` false: zeros.
template <int D>
__device__ __forceinline__ void write_rows(uint8_t* stage, uint32_t src, float scale, bool any, __nv_bfloat16* dst, long long stride, int valid, int lane)
{
    constexpr int kChunks = D / 8, kPerStore = 32 / kChunks;  // 16-byte pieces of a row, rows per store instruction
#pragma unroll
    for (int c = 0; c < D; c += 32) {
        float o[32];
        if (any) tmem_read32(src + c, o);
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = any && scale != 0.f ? o[i] * scale : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint4*>(stage + lane * D * 2 + (((c / 8 + i) ^ (lane & 7)) << 4)) =
                make_uint4(bf16x2(o[8 * i], o[8 * i + 1]), bf16x2(o[8 * i + 2], o[8 * i + 3]), bf16x2(o[8 * i + 4], o[8 * i + 5]),
                           bf16x2(o[8 * i + 6], o[8 * i + 7]));
    }
    __syncwarp();
#pragma unroll 4
    for (int r = lane / kChunks; r < 32; r += kPerStore)
        if (r < valid)
            *reinterpret_cast<uint4*>(dst + r * stride + lane % kChunks * 8) =
                *reinterpret_cast<const uint4*>(stage + r * D * 2 + (((lane % kChunks) ^ (r & 7)) << 4));
}

// cap * tanh(x * scale / cap), in the log2 domain.  Where every |z| = |x| scale / cap of a warp's scores is at most 0.4
// (most are far below the cap), tanh z = z f(z^2) with a polynomial f of four terms fitted to the smallest largest
// relative error, 1e-7 -- five pairwise instructions for two scores -- ; else 1 - 2 / (1 + e^2z) with its exponential
// and division.
struct Cap {
    float cap2, e2, limit, k0, k1, k2, k3;  // cap * log2(e); 2 log2(e) scale / cap; 0.4 cap / scale; f's coefficients in x
    __device__ __forceinline__ Cap(float cap, float scale)
    {
        const float z = scale / cap;
        cap2 = cap * 1.4426950408889634f;
        e2 = 2.f * 1.4426950408889634f * z;
        limit = 0.4f / z;
        k0 = 0.999999902f * cap2 * z;
        k1 = -0.333313625f * cap2 * z * z * z;
        k2 = 0.132709767f * cap2 * z * z * z * z * z;
        k3 = -0.0475536035f * cap2 * z * z * z * z * z * z * z;
    }
    // N scores of a row in place; `vote`: whether the row has a say in how its warp computes them.
    template <int N>
    __device__ __forceinline__ void apply(float (&s)[N], bool vote) const
    {
        float big = 0.f;
#pragma unroll
        for (int c = 0; c < N; c += 2) big = fmaxf(fmaxf(big, fabsf(s[c])), fabsf(s[c + 1]));
        if (__any_sync(0xffffffffu, vote && big > limit)) {
#pragma unroll
            for (int c = 0; c < N; ++c) s[c] = cap2 - __fdividef(2.f * cap2, 1.f + ex2(s[c] * e2));
        } else {
#pragma unroll
            for (int c = 0; c < N; c += 2) {
                const float2 x = make_float2(s[c], s[c + 1]), y = mul2(x, x);
                float2 f = fma2(make_float2(k3, k3), y, make_float2(k2, k2));
                f = fma2(f, y, make_float2(k1, k1));
                f = fma2(f, y, make_float2(k0, k0));
                f = mul2(f, x);
                s[c] = f.x;
                s[c + 1] = f.y;
            }
        }
    }
};

}  // namespace tc
}  // namespace rlkv
