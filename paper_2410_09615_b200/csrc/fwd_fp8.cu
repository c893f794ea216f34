// The linear layer on 8-bit floating-point operands (include/slim.h, slim_linear_fwd_fp8):
//     Y[m][n] = sum_g xs[m][g] ws[n / 128][g] * (sum over the 128 columns k of group g of xq[m][k] wq[n][k])
//
// The inner sums are tcgen05.mma (kind::f8f6f4, fp32 accumulate) of one group of 128 columns each, into a tensor-memory buffer of its
// own; the outer sum is made in registers: warps read a group's buffer, multiply it with the group's two scales and add it to their
// fp32 accumulators, while the next groups' MMAs run.  (A scale is any binary32 number, so it cannot ride in the MMA, whose block scales are
// powers of two.)
//
// Two kernels, which differ in what the MMA's rows (M) are; fp8_plan.h picks one and its tile:
//   fp8_small_kernel   few tokens.  The weight's 128 rows of a block are the MMA's rows, so that none is empty; the tokens are its columns.
//                      Clusters cut the columns of the layer among their CTAs.  Bound by the weight's stream from the HBM, or by one
//                      launch's chain: first bytes, MMAs, exchange.
//   fp8_tokens_kernel  more tokens, as the MMA's rows: a thread has one token, and a group's scales are one number for it.  Persistent CTA
//                      pairs on tiles of 256 tokens, or single CTAs on 128.  Bound by the hand-over of the two buffers of 256 columns
//                      that tensor memory holds (MMAs 513 cycles, reading 350, and the way between the two), and by the power limit.
//
// A product of scales below 2^-126 is a subnormal number and counts: this file is compiled without flush-to-zero.
//
// What the loops' waits cost decides both, so they are written for it: a warp's lanes stay together (warp_wait), nothing behind a barrier's
// answer is spilled, remote arrivals have no cluster scope (1100 cycles where they had).
#include <atomic>
#include <mutex>
#include "fp8.cuh"
#include "fp8_plan.h"
#include "fp8_ring.h"
#include "tcgen05.cuh"

namespace slim {

namespace f8 {

using namespace pf;

// Instruction descriptor, kind::f8f6f4: fp32 accumulate, both operands K-major.
__host__ __device__ constexpr uint32_t idesc_f8(int m, int n, int a_format, int b_format) {
    return (1u << 4) | ((uint32_t)a_format << 7) | ((uint32_t)b_format << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %3, p;\n\t}"
        :: "r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi) : "memory");
}
__device__ __forceinline__ void mma_f8_pair(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], a, b, %3, p;\n\t}"
        :: "r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi) : "memory");
}

// A warp's bounded wait (tcgen05.cuh's mbar_wait, for lanes that go on together: the vote tells the compiler so, and spares it bringing them
// together again before every instruction of a whole warp).  One that expires raises the CTA's flag, which ends all others and is looked
// at at the end.  False: it gave up; a loader then asks for no more.  (The issuing warp does not look: its MMAs go on over what the stages hold, one
// group in the time that such a wait takes, and a branch on the answer took 100 tokens, 8192 -> 8192 from 20.1 us to 21.8.)
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile uint32_t* abort_flag) {
    for (uint32_t it = 0; it < kPSpinLimit; ++it) {
        if (__all_sync(0xffffffffu, mbar_try(bar, parity, false))) return true;
        if ((it & 63u) == 63u && __any_sync(0xffffffffu, *abort_flag)) return false;
    }
    *abort_flag = 1u;
    return false;
}
__device__ __forceinline__ bool warp_wait2(uint64_t* b0, uint32_t p0, uint64_t* b1, uint32_t p1, volatile uint32_t* abort_flag) {
    for (uint32_t it = 0; it < kPSpinLimit; ++it) {
        if (__all_sync(0xffffffffu, mbar_try(b0, p0, false) & mbar_try(b1, p1, false))) return true;
        if ((it & 63u) == 63u && __any_sync(0xffffffffu, *abort_flag)) return false;
    }
    *abort_flag = 1u;
    return false;
}

// A loader's end: no MMA's completion may arrive in this CTA's shared memory after it has left (fp8_ring.h).
__device__ __forceinline__ void drain(uint64_t* empty, int requested, int places, volatile uint32_t* abort_flag) {
#pragma unroll 1
    for (int i = ring_tail(requested, places); i < requested; ++i)
        if (!warp_wait(&empty[i % places], (i / places) & 1, abort_flag)) break;
}
// The end of a CTA in which a wait gave up: what was started is given a million cycles, where a copy or an MMA takes a few thousand at most, before
// its shared and tensor memory are another's.
__device__ __forceinline__ void settle(volatile uint32_t* abort_flag) {
    if (*abort_flag == 0u) return;
    for (const long long t0 = clock64(); clock64() - t0 < 1000000ll;) {}
    __syncthreads();
}

// 16 rows x 8 A columns of a buffer: four values an eight columns.  The wait names the registers, so nothing that uses them is moved ahead of it.
template <int A> struct Frag { float v[A][4]; };
__device__ __forceinline__ void tmem_ld(uint32_t taddr, Frag<2>& f) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(f.v[0][0]), "=f"(f.v[0][1]), "=f"(f.v[0][2]), "=f"(f.v[0][3]), "=f"(f.v[1][0]), "=f"(f.v[1][1]), "=f"(f.v[1][2]), "=f"(f.v[1][3])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld(uint32_t taddr, Frag<4>& f) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=f"(f.v[0][0]), "=f"(f.v[0][1]), "=f"(f.v[0][2]), "=f"(f.v[0][3]), "=f"(f.v[1][0]), "=f"(f.v[1][1]), "=f"(f.v[1][2]), "=f"(f.v[1][3]),
                   "=f"(f.v[2][0]), "=f"(f.v[2][1]), "=f"(f.v[2][2]), "=f"(f.v[2][3]), "=f"(f.v[3][0]), "=f"(f.v[3][1]), "=f"(f.v[3][2]), "=f"(f.v[3][3])
                 : "r"(taddr) : "memory");
}
template <int A>
__device__ __forceinline__ void tmem_wait(Frag<A>& f, Frag<A>& g) {
#pragma unroll
    for (int i = 0; i < A; ++i) {
        if (i == 0)
            asm volatile("tcgen05.wait::ld.sync.aligned;"
                         : "+f"(f.v[0][0]), "+f"(f.v[0][1]), "+f"(f.v[0][2]), "+f"(f.v[0][3]), "+f"(g.v[0][0]), "+f"(g.v[0][1]), "+f"(g.v[0][2]), "+f"(g.v[0][3]) :: "memory");
        else
            asm volatile("" : "+f"(f.v[i][0]), "+f"(f.v[i][1]), "+f"(f.v[i][2]), "+f"(f.v[i][3]), "+f"(g.v[i][0]), "+f"(g.v[i][1]), "+f"(g.v[i][2]), "+f"(g.v[i][3]));
    }
}

// 32 or 16 columns of this thread's row of a buffer; the wait as above.
__device__ __forceinline__ void tmem_ld_row(uint32_t taddr, float (&r)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]),
                   "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]),
                   "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]),
                   "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_wait_row(float (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7]),
                   "+f"(r[8]), "+f"(r[9]), "+f"(r[10]), "+f"(r[11]), "+f"(r[12]), "+f"(r[13]), "+f"(r[14]), "+f"(r[15]) :: "memory");
    asm volatile("" : "+f"(r[16]), "+f"(r[17]), "+f"(r[18]), "+f"(r[19]), "+f"(r[20]), "+f"(r[21]), "+f"(r[22]), "+f"(r[23]),
                      "+f"(r[24]), "+f"(r[25]), "+f"(r[26]), "+f"(r[27]), "+f"(r[28]), "+f"(r[29]), "+f"(r[30]), "+f"(r[31]));
}

__device__ __forceinline__ void tmem_ld_row(uint32_t taddr, float (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]),
                   "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_wait_row(float (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7]),
                   "+f"(r[8]), "+f"(r[9]), "+f"(r[10]), "+f"(r[11]), "+f"(r[12]), "+f"(r[13]), "+f"(r[14]), "+f"(r[15]) :: "memory");
}

// acc += v * s, for two neighbouring columns.
__device__ __forceinline__ void fma2(unsigned long long& acc, float v0, float v1, unsigned long long s) {
    asm("{\n\t.reg .b64 v;\n\tmov.b64 v, {%1, %2};\n\tfma.rn.f32x2 %0, v, %3, %0;\n\t}" : "+l"(acc) : "f"(v0), "f"(v1), "l"(s));
}
__device__ __forceinline__ unsigned long long pair_of(float a, float b) {
    unsigned long long v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    return v;
}
__device__ __forceinline__ float2 halves(unsigned long long v) {
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
    return f;
}
__device__ __forceinline__ unsigned long long lds64(uint32_t addr) {
    unsigned long long v;
    asm volatile("ld.shared.b64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void sts32(uint32_t addr, float v) { asm volatile("st.shared.f32 [%0], %1;" :: "r"(addr), "f"(v) : "memory"); }
__device__ __forceinline__ float4 lds128(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
// Sixteen bytes into a peer's shared memory; its barrier counts them.
__device__ __forceinline__ void st_peer4(uint32_t addr, float2 a, float2 b, uint32_t bar) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                 :: "r"(addr), "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t peer(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// Rows r, r + 8 of tokens c, c + 1 (what tcgen05.ld 16x256b gives a lane: above fp8_small_kernel) into Y.  Lanes four apart have neighbouring
// rows: they swap, and each stores two rows of one token at once where rows of Y are a whole number of words.
__device__ __forceinline__ void store_frag(__nv_bfloat16* Y, int d_out, int row, int token, int b, float2 lo, float2 hi, int lane) {
    const bool odd = lane & 4;
    const float give_lo = odd ? lo.x : lo.y, give_hi = odd ? hi.x : hi.y;
    const float got_lo = __shfl_xor_sync(0xffffffffu, give_lo, 4), got_hi = __shfl_xor_sync(0xffffffffu, give_hi, 4);
    const __nv_bfloat162 two_lo = odd ? __floats2bfloat162_rn(got_lo, lo.y) : __floats2bfloat162_rn(lo.x, got_lo);
    const __nv_bfloat162 two_hi = odd ? __floats2bfloat162_rn(got_hi, hi.y) : __floats2bfloat162_rn(hi.x, got_hi);
    const int r0 = row & ~1, m = token + (odd ? 1 : 0);
    if (m >= b) return;
    __nv_bfloat16* to = Y + (size_t)m * d_out + r0;
    if ((d_out & 1) == 0) {
        if (r0 < d_out) *reinterpret_cast<__nv_bfloat162*>(to) = two_lo;
        if (r0 + 8 < d_out) *reinterpret_cast<__nv_bfloat162*>(to + 8) = two_hi;
    } else {
        if (r0 < d_out) to[0] = two_lo.x;
        if (r0 + 1 < d_out) to[1] = two_lo.y;
        if (r0 + 8 < d_out) to[8] = two_hi.x;
        if (r0 + 9 < d_out) to[9] = two_hi.y;
    }
}

}  // namespace f8

struct alignas(128) Fp8Params {
    __nv_bfloat16* Y;
    const float* Xs; const float* Ws;
    uint32_t* status;
    int b, d_out, groups;
    uint32_t idesc;
    int ahead;
};

// ---------------------------------------------------------------- a cluster for 128 rows: few tokens
// Registers of a batch's tile: tcgen05.ld 16x256b gives a lane, of every 16 rows x 8 tokens, rows r = lane / 4 and r + 8 and tokens
// c = 2 (lane % 4) and c + 1: four values, two pairs of tokens, so that a lane needs the scales of a quarter of the tokens (as pairs, the
// operand of fma.f32x2) instead of all of them.  The block's scale is one number for the whole CTA.
// The C CTAs of a cluster cut the groups of columns into C ranges; each makes the partial tile of 128 rows x N tokens of its range, and
// they exchange them once at the end: 128 / C rows to each, added up in the CTAs' order.
// A wait, a load and an arrival take longer than a group's few tokens: kBatch groups are handed over at a time, side by side in tensor memory
// (one token, 4096 -> 4096, a CTA a tile: 10.1 us a group at a time, 9.6 so).
// Warps: 0-3 accumulate (32 rows each), 4 and 7 request tiles by TMA, 5 issues MMAs, 6 brings the scales.
// Up to 32 tokens a CTA takes less than half of an SM's shared memory, and two are there at once: while one exchanges, the other streams.
template <int N> struct SmallCfg8 {
    static constexpr int kThreads = 8 * 32;
    static constexpr int kCtasPerSm = N <= 32 ? 2 : 1;
    static constexpr int kStages = N <= 16 ? 5 : N == 32 ? 4 : N == 64 ? 7 : 4;
    static constexpr int kStage = kF8Group * (kF8Group + N);             // the weight's tile, then the tokens'
    static constexpr int kBatch = N <= 16 ? 4 : N <= 64 ? 2 : 1, kCols = kBatch * N;      // groups of a batch; its columns of tensor memory
    static constexpr int kSets = 2, kTmemCols = kSets * kCols;           // batches in tensor memory
    static constexpr int kSlots = 4;                                     // batches whose scales are there
    static constexpr int kChunk = 32;                                    // columns read from tensor memory at once
    static constexpr int kOffRecv = kStages * kStage, kOffScales = kOffRecv + N * 512, kOffBars = kOffScales + kSlots * kCols * 4;
    static constexpr size_t kSmem = 1024 + kOffBars + 256;
    static_assert(kSmem <= (kCtasPerSm == 2 ? 113 : 227) * 1024 && (2 * kStages + 2 * kSets + 2 * kSlots + 1) * 8 + 8 <= 256, "shared memory");
};

template <int N>
__global__ void __launch_bounds__(SmallCfg8<N>::kThreads, SmallCfg8<N>::kCtasPerSm)
fp8_small_kernel(const Fp8Params p, const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX)
{
    using namespace f8;
    using Cfg = SmallCfg8<N>;
    constexpr int kStages = Cfg::kStages, kBatch = Cfg::kBatch, kCols = Cfg::kCols, kSets = Cfg::kSets, kSlots = Cfg::kSlots, kAtoms = N / 8;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + Cfg::kOffBars);      // [kStages] tiles landed
    uint64_t* empty = full + kStages;                // [kStages] the MMAs that read the stage are complete
    uint64_t* acc_full = empty + kStages;            // [kSets] a batch's MMAs are complete
    uint64_t* acc_empty = acc_full + kSets;          // [kSets] four warps have read the batch
    uint64_t* sc_full = acc_empty + kSets;           // [kSlots] a batch's scales are there
    uint64_t* sc_empty = sc_full + kSlots;           // [kSlots] four warps have read them
    uint64_t* recv_full = sc_empty + kSlots;         // the cluster's partial tiles have come
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(recv_full + 1);
    volatile uint32_t* abort_flag = tmem_slot + 1;

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    uint32_t ctas;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
    const uint32_t rank = cluster_rank();
    const int tile = (int)(blockIdx.x / ctas), m0 = tile * kF8Group, n0 = (int)blockIdx.y * N;
    const int g0 = (int)((long long)rank * p.groups / ctas), n_groups = (int)((long long)(rank + 1) * p.groups / ctas) - g0;
    const int atoms = min(kAtoms, ceil_div(p.b - n0, 8));            // eights of tokens that there are
    const int shares = 8 / (int)ctas;                                // 16-row pieces that a CTA of the cluster adds up

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
        for (int i = 0; i < kSets; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], 4); }
        for (int i = 0; i < kSlots; ++i) { mbar_init(&sc_full[i], 1); mbar_init(&sc_empty[i], 4); }
        mbar_init(recv_full, 1);
        *abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        mbar_expect_tx(recv_full, (uint32_t)(8 * atoms * 512));
    }
    if (warp == 4 && elect_one()) { prefetch_map(&tmW); prefetch_map(&tmX); }
    if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(s32(tmem_slot)), "r"(Cfg::kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    if (ctas > 1) cluster_arrive();                  // this CTA's barriers are there; waited for before the first remote store
    // The weight's first tiles are asked into the L2 while the grid before still runs (which reads nothing: what that grid may write to them is
    // seen), where all CTAs have an SM of their own: one token, 4096 -> 4096 6.15 us -> 5.6, but 13824 -> 5120, 160 CTAs, 14.6 -> 16.1.
    if (p.ahead && warp == 4 && elect_one())
        for (int i = 0; i < min(n_groups, kStages); ++i) prefetch_tile(&tmW, (g0 + i) * kF8Group, m0);
    const uint32_t tmem_base = __shfl_sync(0xffffffffu, *reinterpret_cast<volatile uint32_t*>(tmem_slot), 0);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("fence.proxy.async;" ::: "memory");            // what the grid before wrote is read through TMA

    if (warp == 4 || warp == 7) {
        // ============================ tiles ============================
        // The weight's by one warp, the tokens' by another: a request takes its warp about 100 ns.
        const bool weight = warp == 4;
        auto request = [&](int i) {
            const int st = i % kStages;
            unsigned char* at = smem + st * Cfg::kStage;
            if (weight) {
                mbar_expect_tx(&full[st], Cfg::kStage);          // (bytes that land before are counted below zero)
                tma_tile(at, &tmW, (g0 + i) * kF8Group, m0, &full[st]);
            } else tma_tile(at + kF8Group * kF8Group, &tmX, (g0 + i) * kF8Group, n0, &full[st]);
        };
        int i = min(n_groups, kStages);
        if (elect_one())
            for (int k = 0; k < i; ++k) request(k);
        __syncwarp();
        for (; i < n_groups; ++i) {
            if (!warp_wait(&empty[i % kStages], ((i / kStages) & 1) ^ 1, abort_flag)) break;
            if (elect_one()) request(i);
            __syncwarp();
        }
        drain(empty, i, kStages, abort_flag);
    } else if (warp == 5) {
        // ============================ MMA issue ============================
        // Two groups at a time: what the warp spends on a group is barriers' answers and the way in and out of its elected lane (16 tokens,
        // 8192 -> 28672 41.7 us -> 39.4; the requests stay apart: a stage is asked for as soon as it is free).
        for (int i = 0; i < n_groups; i += 2) {
            const bool two = i + 1 < n_groups;
            const int st0 = i % kStages, st1 = (i + 1) % kStages;
            // (batches of one group: the second one's buffer is asked for behind the first one's MMAs)
            auto buffer = [&](int k) {
                const int batch = k / kBatch, set = batch % kSets;
                if (k % kBatch == 0 && batch >= kSets) warp_wait(&acc_empty[set], ((batch / kSets) & 1) ^ 1, abort_flag);
            };
            auto issue = [&](int k, int st) {
                const int set = (k / kBatch) % kSets, u = k % kBatch;
                const uint32_t a = desc_lo(s32(smem + st * Cfg::kStage)), x = a + (kF8Group * kF8Group >> 4), d = tmem_base + set * kCols + u * N;
#pragma unroll
                for (int j = 0; j < 4; ++j) mma_f8(d, a + 2 * j, x + 2 * j, p.idesc, j > 0 ? 1u : 0u);       // 32 columns each
                if (u + 1 == kBatch || k + 1 == n_groups) mma_commit(&acc_full[set]);
                mma_commit(&empty[st]);
            };
            buffer(i);
            if (two) warp_wait2(&full[st0], (i / kStages) & 1, &full[st1], ((i + 1) / kStages) & 1, abort_flag);
            else     warp_wait(&full[st0], (i / kStages) & 1, abort_flag);
            fence_after_sync();
            if (kBatch > 1) {
                if (elect_one()) {
                    issue(i, st0);
                    if (two) issue(i + 1, st1);
                }
            } else {
                if (elect_one()) issue(i, st0);
                if (two) {
                    buffer(i + 1);
                    fence_after_sync();
                    if (elect_one()) issue(i + 1, st1);
                }
            }
            __syncwarp();
        }
    } else if (warp == 6) {
        // ============================ scales: of the tokens times the block's, [group of a batch][token] ============================
        constexpr int kEach = kCols / 32, kAhead = 2;
        const float* ws = p.Ws + (size_t)tile * p.groups + g0;
        const int batches = ceil_div(n_groups, kBatch);
        float v[kAhead][kEach], w[kAhead][kEach];
        auto load = [&](int k0) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    const int at = lane + 32 * e, i = (k0 + k) * kBatch + at / N, n = n0 + at % N;
                    const bool in = i < n_groups && n < p.b;
                    v[k][e] = in ? p.Xs[(size_t)n * p.groups + g0 + i] : 0.f;
                    w[k][e] = in ? ws[i] : 0.f;
                }
        };
        load(0);
        for (int k0 = 0; k0 < batches; k0 += kAhead) {
            float s[kAhead][kEach];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
#pragma unroll
                for (int e = 0; e < kEach; ++e) s[k][e] = v[k][e] * w[k][e];
            load(k0 + kAhead);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int batch = k0 + k, slot = batch % kSlots;
                if (batch >= batches) break;
                if (batch >= kSlots) warp_wait(&sc_empty[slot], ((batch / kSlots) & 1) ^ 1, abort_flag);
#pragma unroll
                for (int e = 0; e < kEach; ++e) sts32(s32(smem + Cfg::kOffScales) + (slot * kCols + lane + 32 * e) * 4, s[k][e]);
                __syncwarp();
                if (lane == 0) mbar_arrive(&sc_full[slot]);
            }
        }
    } else {
        // ============================ accumulation ============================
        constexpr int kA = Cfg::kChunk / 8, kChunks = kCols / Cfg::kChunk;
        unsigned long long acc[2][kAtoms][2] = {};               // 16 rows each: pairs of tokens of rows r and r + 8
        for (int i = 0, batch = 0; i < n_groups; i += kBatch, ++batch) {
            const int set = batch % kSets, slot = batch % kSlots;
            warp_wait2(&acc_full[set], (batch / kSets) & 1, &sc_full[slot], (batch / kSlots) & 1, abort_flag);
            fence_after_sync();
            const uint32_t t = tmem_base + ((uint32_t)(warp * 32) << 16) + set * kCols;
            const uint32_t sc = s32(smem + Cfg::kOffScales) + slot * kCols * 4 + (lane & 3) * 8;
            Frag<kA> f[2][2];
            tmem_ld(t, f[0][0]);
            tmem_ld(t + (16u << 16), f[0][1]);
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                tmem_wait(f[c & 1][0], f[c & 1][1]);
                if (c + 1 < kChunks) {
                    tmem_ld(t + (c + 1) * Cfg::kChunk, f[(c + 1) & 1][0]);
                    tmem_ld(t + (16u << 16) + (c + 1) * Cfg::kChunk, f[(c + 1) & 1][1]);
                } else {
                    fence_before_sync();
                    __syncwarp();
                    if (elect_one()) mbar_arrive(&acc_empty[set]);
                }
#pragma unroll
                for (int a = 0; a < kA; ++a) {
                    const int col = c * Cfg::kChunk + a * 8, at = (col % N) / 8;
                    if (kBatch > 1 && i + col / N >= n_groups) continue;             // no such group: what the columns hold is none of this call's
                    const unsigned long long s = lds64(sc + col * 4);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float* v = f[c & 1][h].v[a];
                        fma2(acc[h][at][0], v[0], v[1], s);
                        fma2(acc[h][at][1], v[2], v[3], s);
                    }
                }
            }
            __syncwarp();
            if (elect_one()) mbar_arrive(&sc_empty[slot]);
        }
        const int row = m0 + (lane >> 2), token = n0 + (lane & 3) * 2;
        if (ctas == 1) {
#pragma unroll
            for (int a = 0; a < kAtoms; ++a)
                if (a < atoms)
#pragma unroll
                    for (int h = 0; h < 2; ++h) store_frag(p.Y, p.d_out, row + (warp * 2 + h) * 16, token + a * 8, p.b, halves(acc[h][a][0]), halves(acc[h][a][1]), lane);
        } else {
            // a CTA's place for source c: [its 16-row pieces][eights of tokens][lane] of four values
            cluster_wait();
            const uint32_t recv = s32(smem + Cfg::kOffRecv), per = (uint32_t)(shares * kAtoms * 512);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int piece = warp * 2 + h;
                const uint32_t to = (uint32_t)(piece / shares), dst = peer(recv + rank * per + (uint32_t)((piece % shares) * kAtoms * 512 + lane * 16), to), bar = peer(s32(recv_full), to);
#pragma unroll
                for (int a = 0; a < kAtoms; ++a)
                    if (a < atoms) st_peer4(dst + a * 512, halves(acc[h][a][0]), halves(acc[h][a][1]), bar);
            }
            // (a CTA that gave up sends what it has and stays for what the others send)
            if (!mbar_wait_all(recv_full, 0, true, nullptr, 0, false, nullptr, 0, false, abort_flag))
                for (uint32_t it = 0; it < kPSpinLimit && !mbar_try(recv_full, 0, true); ++it) {}
            __syncwarp();
            for (int i = warp; i < shares * atoms; i += 4) {
                const int piece = i / atoms, a = i - piece * atoms;
                const uint32_t from = recv + (uint32_t)((piece * kAtoms + a) * 512 + lane * 16);
                float4 s = lds128(from);
                for (uint32_t c = 1; c < ctas; ++c) {
                    const float4 v = lds128(from + c * per);
                    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
                }
                store_frag(p.Y, p.d_out, row + ((int)rank * shares + piece) * 16, token + a * 8, p.b, make_float2(s.x, s.y), make_float2(s.z, s.w), lane);
            }
        }
    }
    if (ctas > 1 && warp >= 4) cluster_wait();

    fence_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && *abort_flag) flag_error(p.status, SLIM_ERR_TIMEOUT);
    settle(abort_flag);
    if (warp == 5) {
        fence_after_sync();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem_base), "r"(Cfg::kTmemCols) : "memory");
    }
}

// ---------------------------------------------------------------- pairs of CTAs: many tokens
// Persistent clusters of two CTAs walk tiles of 256 tokens x N rows (128 or 256) with cta_group::2 MMAs that the even CTA
// issues: each CTA loads its own 128 tokens and half of the tile's rows, and accumulates its 128 tokens.  All rings run on across
// tiles, so the next tile's groups are multiplied while this tile is stored.
// Tokens are the MMA's rows here: a thread has one token, so the product of a group's scales is one number for each 128 rows of the
// weight, and the buffer is read with tcgen05.ld 32x32b, 64 words a cycle and quarter of the SM (16x256b: 16, so that a buffer of
// 128 x 256 took as long to read as to multiply).
// Warps: 0-7 accumulate (32 tokens x half of the rows each), 8 and 11 request tiles by TMA, 9 issues MMAs, 10 brings the scales.
// PAIR false: single CTAs on tiles of 128 tokens x N rows (32, 64 or 128), for layers whose pair tiles would leave most SMs without one; a warp
// then accumulates all rows of its 32 tokens.
template <int N, bool PAIR> struct TokCfg8 {
    static constexpr int kWarps = PAIR ? 8 : 4, kThreads = (kWarps + 4) * 32;            // .. kWarps and + 3 tiles, + 1 MMAs, + 2 scales
    static constexpr int kRegs = 216, kOtherRegs = 72;                                  // pairs: 2 x 216 + 72 = 3 x 168, what the three warpgroups are launched with
    static constexpr int kSides = PAIR ? 2 : 1, kCols = N / kSides;                     // columns of a warp
    // Columns read at once: more give a buffer back earlier (pairs, 256 rows: 660 cycles a group, 680 with 16), where the registers hold them
    // (128 rows a warp and no share of the other warps' registers: 100 tokens, 8192 -> 8192 22.3 us with 16, 27.7 with 32).
    static constexpr int kChunk = !PAIR && N == 128 ? 16 : 32;
    static constexpr int kRowsW = PAIR ? N / 2 : N;                                     // of the weight that a CTA loads
    static constexpr int kOffW = kF8Group * kF8Group, kStage = kOffW + kRowsW * kF8Group, kStages = 163840 / kStage;
    static constexpr int kBufferCols = N <= 128 ? 128 : 256, kBuffers = 512 / kBufferCols;
    static constexpr int kScales = kSides * kF8Group * 32, kSlots = 2;                  // of eight groups: 128 tokens x the sides' blocks
    static constexpr int kOutCols = kCols < 64 ? kCols : 64, kOutSlot = 32 * kOutCols * 2;      // a warp's 32 tokens x 64 (32) rows on their way out
    static constexpr int kOffOut = kStages * kStage, kOffScales = kOffOut + kWarps * kOutSlot, kOffBars = kOffScales + kSlots * kScales;
    static constexpr size_t kSmem = 1024 + kOffBars + 256;
    static_assert(kSmem <= 227 * 1024 && kStage % 1024 == 0 && (2 * kStages + 2 * kBuffers + 2 * kSlots) * 8 + 8 <= 256, "shared memory");
};

struct alignas(128) Fp8TokensParams {
    __nv_bfloat16* Y;
    const float* Xs; const float* Ws;
    uint32_t* status;
    int b, d_out, groups;
    uint32_t idesc;
    int row_tiles, token_tiles, token_group;     // tiles of a group of token tiles follow each other, token tiles first
    int by_tma;             // rows of Y are a multiple of 16 bytes
};

template <int N, bool PAIR>
__global__ void __launch_bounds__(TokCfg8<N, PAIR>::kThreads, 1)
fp8_tokens_kernel(const Fp8TokensParams p, const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmY)
{
    using namespace f8;
    using Cfg = TokCfg8<N, PAIR>;
    constexpr int kStages = Cfg::kStages, kBufferCols = Cfg::kBufferCols, kBuffers = Cfg::kBuffers, kSlots = Cfg::kSlots, kWarps = Cfg::kWarps, kSides = Cfg::kSides, kCols = Cfg::kCols;
    constexpr int kCtas = PAIR ? 2 : 1;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + Cfg::kOffBars);      // [kStages] even CTA: both CTAs' tiles landed
    uint64_t* empty = full + kStages;                // [kStages] the MMAs that read the stage are complete
    uint64_t* acc_full = empty + kStages;            // [kBuffers] a group's MMAs are complete
    uint64_t* acc_empty = acc_full + kBuffers;       // [kBuffers] even CTA: the warps of both CTAs have read the buffer
    uint64_t* sc_full = acc_empty + kBuffers;        // [kSlots] the scales of eight groups are there
    uint64_t* sc_empty = sc_full + kSlots;           // [kSlots] the accumulating warps have read them
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sc_empty + kSlots);
    volatile uint32_t* abort_flag = tmem_slot + 1;

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? cluster_rank() : 0u;
    const int units = gridDim.x / kCtas, first_tile = blockIdx.x / kCtas, tiles = p.row_tiles * p.token_tiles;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
        for (int i = 0; i < kBuffers; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], kCtas * kWarps); }
        for (int i = 0; i < kSlots; ++i) { mbar_init(&sc_full[i], 1); mbar_init(&sc_empty[i], kWarps); }
        *abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kWarps && elect_one()) { prefetch_map(&tmX); prefetch_map(&tmW); prefetch_map(&tmY); }
    if (PAIR) cluster_sync_all();                    // both CTAs' barriers exist before anything crosses
    if (warp == kWarps + 1) {
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(s32(tmem_slot)), "r"(512) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(s32(tmem_slot)), "r"(512) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem_base = __shfl_sync(0xffffffffu, *reinterpret_cast<volatile uint32_t*>(tmem_slot), 0);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("fence.proxy.async;" ::: "memory");            // what the grid before wrote is read through TMA
    // A tile's first token in this CTA and its first row.
    struct Tile { int m0, n0; };
    auto tile_of = [&](int t) {
        const int per = p.token_group * p.row_tiles, group = t / per, in = t - group * per;
        const int here = min(p.token_group, p.token_tiles - group * p.token_group), rt = in / here;
        return Tile{(kCtas * (group * p.token_group + in - rt * here) + (int)rank) * kF8Group, rt * N};
    };

    // (the roles stand inside the branches that set the registers: behind them the compiler would have to reckon with the smaller number)
    if (warp < kWarps) {
        if (PAIR) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(Cfg::kRegs));
        // ============================ accumulation, then a tile's end ============================
        constexpr int kChunk = Cfg::kChunk, kChunks = kCols / kChunk;
        const int side = warp >> 2, quarter = warp & 3;
        const uint32_t t0 = tmem_base + ((uint32_t)(quarter * 32) << 16) + side * kCols;
        const uint32_t out = s32(smem + Cfg::kOffOut) + warp * Cfg::kOutSlot, give = PAIR ? peer_addr(acc_empty, 0) : 0u;
        const uint32_t scales = s32(smem + Cfg::kOffScales) + side * (Cfg::kScales / kSides) + (quarter * 32 + lane) * 32;
        int g = 0, eights = 0;
        for (int t = first_tile; t < tiles; t += units) {
            const Tile ti = tile_of(t);
            const int row0 = ti.n0 + side * kCols, tok0 = ti.m0 + quarter * 32;
            unsigned long long acc[kCols / 2] = {};           // neighbouring rows of the weight
            float4 s4 = make_float4(0.f, 0.f, 0.f, 0.f);     // this token's scales of the next groups, times the block's
#pragma unroll 1
            for (int i = 0; i < p.groups; ++i, ++g) {
                if ((i & 3) == 0) {
                    const int slot = eights % kSlots;
                    if ((i & 7) == 0) warp_wait(&sc_full[slot], (eights / kSlots) & 1, abort_flag);
                    s4 = lds128(scales + slot * Cfg::kScales + (i & 4) * 4);
                    if ((i & 7) == 4 || i + 4 >= p.groups) {
                        __syncwarp();
                        if (elect_one()) mbar_arrive(&sc_empty[slot]);
                        ++eights;
                    }
                }
                const int buf = g % kBuffers;
                const uint32_t ta = t0 + buf * kBufferCols;
                warp_wait(&acc_full[buf], (g / kBuffers) & 1, abort_flag);
                fence_after_sync();
                float f[2][kChunk];
                tmem_ld_row(ta, f[0]);
                const unsigned long long s = pair_of(s4.x, s4.x);
                s4.x = s4.y; s4.y = s4.z; s4.z = s4.w;
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    tmem_wait_row(f[c & 1]);
                    if (c + 1 < kChunks) tmem_ld_row(ta + (c + 1) * kChunk, f[(c + 1) & 1]);
                    else {
                        fence_before_sync();
                        __syncwarp();
                        if (elect_one()) { if (PAIR) mbar_arrive_remote(give + buf * 8); else mbar_arrive(&acc_empty[buf]); }
                    }
#pragma unroll
                    for (int k = 0; k < kChunk / 2; ++k) fma2(acc[c * (kChunk / 2) + k], f[c & 1][2 * k], f[c & 1][2 * k + 1], s);
                }
            }
            // 64 rows of the weight (32) at a time into the warp's place in shared memory, [token][64 rows] bf16, 128-byte (64-byte) swizzle,
            // and out from there
            constexpr int kOut = Cfg::kOutCols;
            auto place_of = [&](int token, int chunk) {      // of eight rows
                return out + token * (kOut * 2) + ((uint32_t)(chunk ^ (kOut == 64 ? token & 7 : (token >> 1) & 3)) << 4);
            };
#pragma unroll
            for (int c = 0; c < kCols / kOut; ++c) {
                if (row0 + c * kOut >= p.d_out || tok0 >= p.b) break;
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                __syncwarp();
#pragma unroll
                for (int k = 0; k < kOut / 8; ++k) {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 v = halves(acc[c * (kOut / 2) + k * 4 + e]);
                        const __nv_bfloat162 two = __floats2bfloat162_rn(v.x, v.y);
                        w[e] = *reinterpret_cast<const uint32_t*>(&two);
                    }
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(place_of(lane, k)), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
                }
                if (p.by_tma) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];"
                                     :: "l"(&tmY), "r"(row0 + c * kOut), "r"(tok0), "r"(out) : "memory");
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                } else {
                    __syncwarp();
                    for (int k = 0; k < 32; ++k) {                  // a token; two rows a lane
                        if (tok0 + k >= p.b) break;
#pragma unroll
                        for (int e = 0; e < kOut / 32; ++e) {
                            const int r = lane + 32 * e;
                            uint16_t v;
                            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(place_of(k, r >> 3) + (r & 7) * 2) : "memory");
                            if (row0 + c * kOut + r < p.d_out) reinterpret_cast<uint16_t*>(p.Y)[(size_t)(tok0 + k) * p.d_out + row0 + c * kOut + r] = v;
                        }
                    }
                    __syncwarp();
                }
            }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    } else {
        if (PAIR) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(Cfg::kOtherRegs));
        if (warp == kWarps || warp == kWarps + 3) {
            // ============================ tiles: the tokens', the weight's ============================
            // A warp each: a request takes its warp about 100 ns, as long as a narrow tile's MMAs.
            const bool tokens = warp == kWarps;
            int g = 0;
            bool ok = true;
            for (int t = first_tile; ok && t < tiles; t += units) {
                const Tile ti = tile_of(t);
                for (int i = 0; i < p.groups; ++i, ++g) {
                    const int st = g % kStages;
                    if (g >= kStages && !(ok = warp_wait(&empty[st], ((g / kStages) & 1) ^ 1, abort_flag))) break;
                    unsigned char* at = smem + st * Cfg::kStage;
                    if (elect_one()) {
                        // (bytes that land before they are announced, the odd CTA's among them, are counted below zero: the phase cannot end
                        // without the announcement)
                        const uint32_t bar = PAIR ? peer_addr(&full[st], 0) : 0u;
                        if (tokens) {
                            if (rank == 0) mbar_expect_tx(&full[st], (uint32_t)(kCtas * Cfg::kStage));
                            if (PAIR) tma_tile_pair(at, &tmX, i * kF8Group, ti.m0, bar);
                            else      tma_tile(at, &tmX, i * kF8Group, ti.m0, &full[st]);
                        } else {
                            if (PAIR) tma_tile_pair(at + Cfg::kOffW, &tmW, i * kF8Group, ti.n0 + (int)rank * Cfg::kRowsW, bar);
                            else      tma_tile(at + Cfg::kOffW, &tmW, i * kF8Group, ti.n0, &full[st]);
                        }
                    }
                }
            }
            __syncwarp();
            drain(empty, g, kStages, abort_flag);
        } else if (warp == kWarps + 1) {
            // ============================ MMA issue: a warp of the even CTA ============================
            if (rank == 0) {
                int g = 0;
                bool there = false;                          // the coming stage was found full by an early question
                const uint32_t first = desc_lo(s32(smem));
                for (int t = first_tile; t < tiles; t += units) {
                    for (int i = 0; i < p.groups; ++i, ++g) {
                        const int st = g % kStages, buf = g % kBuffers, use = g / kBuffers;
                        if (!there) warp_wait(&full[st], (g / kStages) & 1, abort_flag);
                        if (use > 0) warp_wait(&acc_empty[buf], (use & 1) ^ 1, abort_flag);
                        fence_after_sync();
                        const uint32_t x = first + (uint32_t)st * (Cfg::kStage >> 4), w = x + (Cfg::kOffW >> 4), d = tmem_base + (uint32_t)(buf * kBufferCols);
                        if (elect_one()) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                if (PAIR) mma_f8_pair(d, x + 2 * j, w + 2 * j, p.idesc, j > 0 ? 1u : 0u);
                                else      mma_f8(d, x + 2 * j, w + 2 * j, p.idesc, j > 0 ? 1u : 0u);
                            }
                            if (PAIR) { mma_commit2(&acc_full[buf]); mma_commit2(&empty[st]); }
                            else      { mma_commit(&acc_full[buf]); mma_commit(&empty[st]); }
                        }
                        there = __all_sync(0xffffffffu, mbar_test(&full[(g + 1) % kStages], ((g + 1) / kStages) & 1, false));
                    }
                }
            }
        } else if (warp == kWarps + 2) {
            // ============================ scales: of the tokens times the blocks' ============================
            // Eight groups at a time, [block][token][group]: a lane loads group lane % 8 of every fourth token, so that a load touches four
            // lines (a token a lane: 32, and the barriers and loads of the other warps waited behind them: 740 cycles a group instead of 690).
            const int blocks = ceil_div(p.d_out, kF8Group), k = lane & 7;
            int eights = 0;
            for (int t = first_tile; t < tiles; t += units) {
                const Tile ti = tile_of(t);
                const float* w0 = p.Ws + (size_t)min(ti.n0 / kF8Group, blocks - 1) * p.groups;
                const float* w1 = p.Ws + (size_t)min((ti.n0 + N / kSides) / kF8Group, blocks - 1) * p.groups;
                const int tok0 = ti.m0 + (lane >> 3);
                for (int i0 = 0; i0 < p.groups; i0 += 8, ++eights) {
                    const int slot = eights % kSlots, i = min(i0 + k, p.groups - 1);
                    const float wa = w0[i], wb = PAIR ? w1[i] : 0.f;
                    const uint32_t at = s32(smem + Cfg::kOffScales) + slot * Cfg::kScales + lane * 4;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        float v[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) v[e] = p.Xs[(size_t)min(tok0 + half * 64 + e * 4, p.b - 1) * p.groups + i];
                        if (half == 0 && eights >= kSlots) warp_wait(&sc_empty[slot], ((eights / kSlots) & 1) ^ 1, abort_flag);
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            sts32(at + (half * 16 + e) * 128, v[e] * wa);
                            if (PAIR) sts32(at + (half * 16 + e) * 128 + Cfg::kScales / 2, v[e] * wb);
                        }
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sc_full[slot]);
                }
            }
        }
    }

    fence_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && *abort_flag) flag_error(p.status, SLIM_ERR_TIMEOUT);
    settle(abort_flag);
    if (PAIR) cluster_sync_all();                    // neither CTA leaves while the other may still use its shared memory
    if (warp == kWarps + 1) {
        fence_after_sync();
        if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(tmem_base), "r"(512) : "memory");
        else      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem_base), "r"(512) : "memory");
    }
}

// ---------------------------------------------------------------- host side
// 8-bit rows of d_in bytes: boxes of 128 columns x box_rows rows, 128-byte swizzle.
static bool f8_map(CUtensorMap* map, const void* base, int d_in, int rows, int box_rows) {
    return pf_map(map, base, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, (uint64_t)d_in, (uint64_t)rows, kF8Group, box_rows, 128);
}

// Attributes and what is resident at once, per device: set and found once (twice is harmless, both find the same).
struct Fp8Device { int pairs; int clusters[4][4]; };
static Fp8Device g_f8[64];
static std::atomic<bool> g_f8_ready[64];

// Clusters of a kernel that are resident at once (0: the launch would fail).
template <typename K>
static int resident_clusters(K kernel, int ctas, int threads, size_t smem) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas); cfg.blockDim = dim3((unsigned)threads); cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)ctas; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    int n = 0;
    return cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess ? n : 0;
}
template <typename K>
static bool large_smem(K kernel, size_t bytes) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess;
}

template <int N>
static bool prepare_small8(int (&clusters)[4]) {
    using Cfg = SmallCfg8<N>;
    if (!large_smem(fp8_small_kernel<N>, Cfg::kSmem)) return false;
    // (the occupancy query says one CTA an SM for every kernel with tensor memory, however little shared memory it has)
    for (int i = 0; i < 4; ++i)
        if ((clusters[i] = Cfg::kCtasPerSm * resident_clusters(fp8_small_kernel<N>, 1 << i, Cfg::kThreads, Cfg::kSmem)) < 1) return false;
    return true;
}
template <int N, bool PAIR>
static bool prepare_tokens8() { return large_smem(fp8_tokens_kernel<N, PAIR>, TokCfg8<N, PAIR>::kSmem); }

static const Fp8Device* fp8_device(const DeviceInfo* di) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
    if (!g_f8_ready[dev].load(std::memory_order_acquire)) {
        static std::mutex m;
        std::lock_guard<std::mutex> lock(m);
        if (!g_f8_ready[dev].load(std::memory_order_relaxed)) {
            Fp8Device& d = g_f8[dev];
            if (!prepare_small8<16>(d.clusters[0]) || !prepare_small8<32>(d.clusters[1]) || !prepare_small8<64>(d.clusters[2]) || !prepare_small8<128>(d.clusters[3]) ||
                !prepare_tokens8<32, false>() || !prepare_tokens8<64, false>() || !prepare_tokens8<128, false>() || !prepare_tokens8<128, true>() ||
                !prepare_tokens8<256, true>())
                return nullptr;
            const int n = resident_clusters(fp8_tokens_kernel<256, true>, 2, TokCfg8<256, true>::kThreads, TokCfg8<256, true>::kSmem);
            if (n < 1) return nullptr;
            d.pairs = n < di->sm_count / 2 ? n : di->sm_count / 2;
            g_f8_ready[dev].store(true, std::memory_order_release);
        }
    }
    return &g_f8[dev];
}

template <int N>
static slim_status_t launch_small8(Fp8Params p, const void* Xq, int x_format, const void* Wq, int w_format, int d_in, int ctas, int sm_count, cudaStream_t st) {
    using Cfg = SmallCfg8<N>;
    p.idesc = f8::idesc_f8(kF8Group, N, w_format, x_format);
    CUtensorMap tmW, tmX;
    if (!f8_map(&tmW, Wq, d_in, p.d_out, kF8Group) || !f8_map(&tmX, Xq, d_in, p.b, N)) return SLIM_ERR_CUDA;
    const int tiles = ceil_div(p.d_out, kF8Group), token_tiles = ceil_div(p.b, N);
    p.ahead = (long long)tiles * token_tiles * ctas <= sm_count;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * ctas), (unsigned)token_tiles); cfg.blockDim = dim3(Cfg::kThreads); cfg.dynamicSmemBytes = Cfg::kSmem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)ctas; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, fp8_small_kernel<N>, p, tmW, tmX);
    count_launch(1);
    note_token_tile(N);
    return e == cudaSuccess ? SLIM_OK : SLIM_ERR_CUDA;
}

template <int N, bool PAIR>
static slim_status_t launch_tokens8(const Fp8Params& q, const void* Xq, int x_format, const void* Wq, int w_format, int d_in, int units, cudaStream_t st) {
    using Cfg = TokCfg8<N, PAIR>;
    constexpr int kCtas = PAIR ? 2 : 1;
    Fp8TokensParams p = {};
    p.Y = q.Y; p.Xs = q.Xs; p.Ws = q.Ws; p.status = q.status; p.b = q.b; p.d_out = q.d_out; p.groups = q.groups;
    p.token_tiles = ceil_div(q.b, kCtas * kF8Group);
    p.row_tiles = ceil_div(q.d_out, N);
    p.token_group = p.token_tiles < 8 ? p.token_tiles : 8;
    p.idesc = f8::idesc_f8(kCtas * kF8Group, N, x_format, w_format);
    p.by_tma = q.d_out % 8 == 0;
    CUtensorMap tmW, tmX, tmY;
    if (!f8_map(&tmW, Wq, d_in, q.d_out, Cfg::kRowsW) || !f8_map(&tmX, Xq, d_in, q.b, kF8Group)) return SLIM_ERR_CUDA;
    tmY = tmX;                                   // not used where rows of Y are no multiple of 16 bytes
    if (p.by_tma && !pf_map(&tmY, q.Y, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, (uint64_t)q.d_out, (uint64_t)q.b, Cfg::kOutCols, 32, Cfg::kOutCols * 2)) return SLIM_ERR_CUDA;
    const long long tiles = (long long)p.row_tiles * p.token_tiles;
    if (tiles > 0x7FFFFFFFll - 256) return SLIM_ERR_INVALID_ARG;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(kCtas * (tiles < units ? tiles : units))); cfg.blockDim = dim3(Cfg::kThreads); cfg.dynamicSmemBytes = Cfg::kSmem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr + (PAIR ? 0 : 1); cfg.numAttrs = PAIR ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, fp8_tokens_kernel<N, PAIR>, p, tmX, tmW, tmY);
    count_launch(1);
    note_token_tile(kCtas * kF8Group);
    return e == cudaSuccess ? SLIM_OK : SLIM_ERR_CUDA;
}

slim_status_t launch_fp8(const uint8_t* Xq, const float* Xs, int x_format, int b, const uint8_t* Wq, const float* Ws, int w_format, int d_out, int d_in,
                         __nv_bfloat16* Y, uint32_t* status_dev, cudaStream_t st)
{
    slim_status_t err;
    const DeviceInfo* di = device_info(&err);
    if (!di) return err;
    const Fp8Device* dev = fp8_device(di);
    if (!dev) return SLIM_ERR_CUDA;
    Fp8Params p = {};
    p.Y = Y; p.Xs = Xs; p.Ws = Ws; p.status = status_dev; p.b = b; p.d_out = d_out; p.groups = ceil_div(d_in, kF8Group);
    const Fp8Plan plan = fp8_plan(b, d_out, p.groups, di->sm_count, dev->pairs, dev->clusters);
    auto launch = [&]() -> slim_status_t {
        switch (plan.kernel) {
        case FP8_CLUSTER_16:  return launch_small8<16>(p, Xq, x_format, Wq, w_format, d_in, plan.ctas, di->sm_count, st);
        case FP8_CLUSTER_32:  return launch_small8<32>(p, Xq, x_format, Wq, w_format, d_in, plan.ctas, di->sm_count, st);
        case FP8_CLUSTER_64:  return launch_small8<64>(p, Xq, x_format, Wq, w_format, d_in, plan.ctas, di->sm_count, st);
        case FP8_CLUSTER_128: return launch_small8<128>(p, Xq, x_format, Wq, w_format, d_in, plan.ctas, di->sm_count, st);
        case FP8_ROWS_32:     return launch_tokens8<32, false>(p, Xq, x_format, Wq, w_format, d_in, di->sm_count, st);
        case FP8_ROWS_64:     return launch_tokens8<64, false>(p, Xq, x_format, Wq, w_format, d_in, di->sm_count, st);
        case FP8_ROWS_128:    return launch_tokens8<128, false>(p, Xq, x_format, Wq, w_format, d_in, di->sm_count, st);
        case FP8_PAIR_128:    return launch_tokens8<128, true>(p, Xq, x_format, Wq, w_format, d_in, dev->pairs, st);
        case FP8_PAIR_256:    return launch_tokens8<256, true>(p, Xq, x_format, Wq, w_format, d_in, dev->pairs, st);
        }
        return SLIM_ERR_UNSUPPORTED_SHAPE;
    };
    err = launch();
    static_assert(SLIM_FP8_CLUSTER_16 == 1 + (int)FP8_CLUSTER_16 && SLIM_FP8_PAIR_256 == 1 + (int)FP8_PAIR_256, "the plan's kernels in the header's order");
    if (err == SLIM_OK) note_fp8_kernel(static_cast<slim_fp8_kernel_t>(1 + (int)plan.kernel), plan.ctas);
    return err;
}

}  // namespace slim
