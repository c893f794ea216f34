// The linear layer on 8-bit floating-point operands (include/slim.h, slim_linear_fwd_fp8):
//     Y[m][n] = sum_g xs[m][g] ws[n / 128][g] * (sum over the 128 columns k of group g of xq[m][k] wq[n][k])
//
// The inner sums are tcgen05.mma (kind::f8f6f4, fp32 accumulate) of one group of 128 columns each, into a tensor-memory buffer of its
// own; the outer sum is made in registers: warps read a group's buffer, multiply it with the group's two scales and add it to their
// fp32 accumulators, while the next groups' MMAs run.  The weight's 128 rows of a block are the MMA's rows (M), so the block's scale is one
// number for a whole CTA; tokens are its columns (N).
//
// Registers of a group's tile: tcgen05.ld 16x256b gives a lane, of every 16 rows x 8 tokens, rows r = lane / 4 and r + 8 and tokens
// c = 2 (lane % 4) and c + 1: four values, two pairs of tokens, so that a lane needs the scales of a quarter of the tokens (as pairs, the
// operand of fma.f32x2) instead of all of them.
#include <atomic>
#include "fp8.cuh"
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

// acc += v * s, for two neighbouring tokens.
__device__ __forceinline__ void fma2(unsigned long long& acc, float v0, float v1, unsigned long long s) {
    asm("{\n\t.reg .b64 v;\n\tmov.b64 v, {%1, %2};\n\tfma.rn.f32x2 %0, v, %3, %0;\n\t}" : "+l"(acc) : "f"(v0), "f"(v1), "l"(s));
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

// Rows r, r + 8 of tokens c, c + 1 (see the file's header) into Y.  Lanes four apart have neighbouring rows: they swap, and each stores two
// rows of one token at once where rows of Y are a whole number of words.
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
};

// ---------------------------------------------------------------- a cluster for 128 rows: few tokens
// The C CTAs of a cluster cut the groups of columns into C ranges; each makes the partial tile of 128 rows x N tokens of its range, and
// they exchange them once at the end: 128 / C rows to each, added up in the CTAs' order.
// Warps: 0-3 accumulate (32 rows each), 4 requests tiles by TMA, 5 issues MMAs, 6 brings the scales.
template <int N> struct SmallCfg8 {
    static constexpr int kThreads = 7 * 32;
    static constexpr int kCtasPerSm = N <= 32 ? 2 : 1;
    static constexpr int kStages = N <= 16 ? 5 : N == 32 ? 4 : N == 64 ? 6 : 4;
    static constexpr int kStage = kF8Group * (kF8Group + N);             // the weight's tile, then the tokens'
    static constexpr int kBuffers = N <= 64 ? 4 : 2, kTmemCols = kBuffers * N;
    static constexpr int kSlots = N <= 64 ? 8 : 4;                       // groups whose scales are there
    static constexpr int kChunk = N < 32 ? N : 32;                       // tokens read from tensor memory at once
    static constexpr int kOffRecv = kStages * kStage, kOffScales = kOffRecv + N * 512, kOffBars = kOffScales + kSlots * N * 4;
    static constexpr size_t kSmem = 1024 + kOffBars + 256;
    static_assert(kSmem <= (kCtasPerSm == 2 ? 113 : 227) * 1024, "shared memory");
};

template <int N>
__global__ void __launch_bounds__(SmallCfg8<N>::kThreads, SmallCfg8<N>::kCtasPerSm)
fp8_small_kernel(const Fp8Params p, const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX)
{
    using namespace f8;
    using Cfg = SmallCfg8<N>;
    constexpr int kStages = Cfg::kStages, kBuffers = Cfg::kBuffers, kSlots = Cfg::kSlots, kAtoms = N / 8;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + Cfg::kOffBars);      // [kStages] tiles landed
    uint64_t* empty = full + kStages;                // [kStages] the MMAs that read the stage are complete
    uint64_t* acc_full = empty + kStages;            // [kBuffers] a group's MMAs are complete
    uint64_t* acc_empty = acc_full + kBuffers;       // [kBuffers] four warps have read the buffer
    uint64_t* sc_full = acc_empty + kBuffers;        // [kSlots]
    uint64_t* sc_empty = sc_full + kSlots;           // [kSlots]
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
        for (int i = 0; i < kBuffers; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], 4); }
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
    const uint32_t tmem_base = __shfl_sync(0xffffffffu, *reinterpret_cast<volatile uint32_t*>(tmem_slot), 0);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("fence.proxy.async;" ::: "memory");            // what the grid before wrote is read through TMA
    bool ok = true;

    if (warp == 4) {
        // ============================ tiles ============================
        for (int i = 0; i < n_groups; ++i) {
            const int st = i % kStages;
            if (i >= kStages) ok = mbar_wait(&empty[st], ((i / kStages) & 1) ^ 1, abort_flag) && ok;
            unsigned char* at = smem + st * Cfg::kStage;
            if (elect_one()) {
                mbar_expect_tx(&full[st], Cfg::kStage);
                tma_tile(at, &tmW, (g0 + i) * kF8Group, m0, &full[st]);
                tma_tile(at + kF8Group * kF8Group, &tmX, (g0 + i) * kF8Group, n0, &full[st]);
            }
        }
    } else if (warp == 5) {
        // ============================ MMA issue ============================
        for (int i = 0; i < n_groups; ++i) {
            const int st = i % kStages, buf = i % kBuffers;
            ok = mbar_wait_all(&full[st], (i / kStages) & 1, false, i >= kBuffers ? &acc_empty[buf] : nullptr, ((i / kBuffers) & 1) ^ 1, false,
                               nullptr, 0, false, abort_flag) && ok;
            fence_after_sync();
            const uint32_t a = desc_lo(s32(smem + st * Cfg::kStage)), x = a + (kF8Group * kF8Group >> 4), d = tmem_base + buf * N;
            if (elect_one()) {
#pragma unroll
                for (int j = 0; j < 4; ++j) mma_f8(d, a + 2 * j, x + 2 * j, p.idesc, j > 0 ? 1u : 0u);       // 32 columns each
                mma_commit(&empty[st]);
                mma_commit(&acc_full[buf]);
            }
        }
    } else if (warp == 6) {
        // ============================ scales: of the tokens times the block's ============================
        constexpr int kAhead = 4, kEach = (N + 31) / 32;
        const float* ws = p.Ws + (size_t)tile * p.groups + g0;
        float v[kAhead][kEach], w[kAhead];
        auto load = [&](int i0) {
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                w[j] = i0 + j < n_groups ? ws[i0 + j] : 0.f;
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    const int n = lane + 32 * e;
                    v[j][e] = n < N && n0 + n < p.b && i0 + j < n_groups ? p.Xs[(size_t)(n0 + n) * p.groups + g0 + i0 + j] : 0.f;
                }
            }
        };
        load(0);
        for (int i0 = 0; i0 < n_groups; i0 += kAhead) {
            float s[kAhead][kEach];
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
#pragma unroll
                for (int e = 0; e < kEach; ++e) s[j][e] = v[j][e] * w[j];
            load(i0 + kAhead);
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int i = i0 + j, slot = i % kSlots;
                if (i >= n_groups) break;
                if (i >= kSlots) ok = mbar_wait(&sc_empty[slot], ((i / kSlots) & 1) ^ 1, abort_flag) && ok;
#pragma unroll
                for (int e = 0; e < kEach; ++e)
                    if (lane + 32 * e < N) sts32(s32(smem + Cfg::kOffScales) + (slot * N + lane + 32 * e) * 4, s[j][e]);
                __syncwarp();
                if (lane == 0) mbar_arrive(&sc_full[slot]);
            }
        }
    } else {
        // ============================ accumulation ============================
        constexpr int kA = Cfg::kChunk / 8, kChunks = N / Cfg::kChunk;
        unsigned long long acc[2][kAtoms][2] = {};               // 16 rows each: pairs of tokens of rows r and r + 8
        for (int i = 0; i < n_groups; ++i) {
            const int buf = i % kBuffers, slot = i % kSlots;
            ok = mbar_wait_all(&acc_full[buf], (i / kBuffers) & 1, false, &sc_full[slot], (i / kSlots) & 1, false, nullptr, 0, false, abort_flag) && ok;
            fence_after_sync();
            const uint32_t t = tmem_base + ((uint32_t)(warp * 32) << 16) + buf * N;
            const uint32_t sc = s32(smem + Cfg::kOffScales) + slot * N * 4 + (lane & 3) * 8;
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
                    if (lane == 0) mbar_arrive(&acc_empty[buf]);
                }
#pragma unroll
                for (int a = 0; a < kA; ++a) {
                    const unsigned long long s = lds64(sc + (c * kA + a) * 32);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float* v = f[c & 1][h].v[a];
                        fma2(acc[h][c * kA + a][0], v[0], v[1], s);
                        fma2(acc[h][c * kA + a][1], v[2], v[3], s);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sc_empty[slot]);
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
            ok = mbar_wait_all(recv_full, 0, true, nullptr, 0, false, nullptr, 0, false, abort_flag) && ok;
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

    if (!ok && lane == 0) flag_error(p.status, SLIM_ERR_TIMEOUT);
    fence_before_sync();
    __syncthreads();
    if (warp == 5) {
        fence_after_sync();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem_base), "r"(Cfg::kTmemCols) : "memory");
    }
}

// ---------------------------------------------------------------- host side
// 8-bit rows of d_in bytes: boxes of 128 columns x box_rows rows, 128-byte swizzle.
static bool f8_map(CUtensorMap* map, const void* base, int d_in, int rows, int box_rows) {
    return pf_map(map, base, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, (uint64_t)d_in, (uint64_t)rows, kF8Group, box_rows, 128);
}

static std::atomic<bool> g_f8_attr_set[64];        // attributes set once per device (setting them twice is harmless)

template <int N>
static slim_status_t launch_small8(Fp8Params p, const void* Xq, int x_format, const void* Wq, int w_format, int d_in, int sm_count, cudaStream_t st) {
    using Cfg = SmallCfg8<N>;
    p.idesc = f8::idesc_f8(kF8Group, N, w_format, x_format);
    CUtensorMap tmW, tmX;
    if (!f8_map(&tmW, Wq, d_in, p.d_out, kF8Group) || !f8_map(&tmX, Xq, d_in, p.b, N)) return SLIM_ERR_CUDA;
    const int tiles = ceil_div(p.d_out, kF8Group), token_tiles = ceil_div(p.b, N);
    int ctas = 8;
    while (ctas > 1 && ((long long)tiles * token_tiles * ctas > (long long)sm_count * Cfg::kCtasPerSm || p.groups < 2 * ctas)) ctas /= 2;
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

slim_status_t launch_fp8(const uint8_t* Xq, const float* Xs, int x_format, int b, const uint8_t* Wq, const float* Ws, int w_format, int d_out, int d_in,
                         __nv_bfloat16* Y, uint32_t* status_dev, cudaStream_t st)
{
    slim_status_t err;
    const DeviceInfo* di = device_info(&err);
    if (!di) return err;
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64) return SLIM_ERR_CUDA;
    if (!g_f8_attr_set[dev].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(fp8_small_kernel<16>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SmallCfg8<16>::kSmem) != cudaSuccess ||
            cudaFuncSetAttribute(fp8_small_kernel<32>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SmallCfg8<32>::kSmem) != cudaSuccess ||
            cudaFuncSetAttribute(fp8_small_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SmallCfg8<64>::kSmem) != cudaSuccess ||
            cudaFuncSetAttribute(fp8_small_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SmallCfg8<128>::kSmem) != cudaSuccess)
            return SLIM_ERR_CUDA;
        g_f8_attr_set[dev].store(true, std::memory_order_release);
    }
    Fp8Params p = {};
    p.Y = Y; p.Xs = Xs; p.Ws = Ws; p.status = status_dev; p.b = b; p.d_out = d_out; p.groups = ceil_div(d_in, kF8Group);
    return b <= 16   ? launch_small8<16>(p, Xq, x_format, Wq, w_format, d_in, di->sm_count, st)
           : b <= 32 ? launch_small8<32>(p, Xq, x_format, Wq, w_format, d_in, di->sm_count, st)
           : b <= 64 ? launch_small8<64>(p, Xq, x_format, Wq, w_format, d_in, di->sm_count, st)
                     : launch_small8<128>(p, Xq, x_format, Wq, w_format, d_in, di->sm_count, st);
}

}  // namespace slim
