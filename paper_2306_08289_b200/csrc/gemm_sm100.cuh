// Matrix products on the 5th-generation tensor cores: C[b] = A[b] B[b]^T summed in fp32, with an epilogue of the caller's.
//
// A pair of CTAs (a cluster of two, cta_group::2) makes one 256 x 256 tile: each CTA holds 128 rows of A and 128 rows of
// B in shared memory and 128 x 256 sums in its tensor memory. Per K step of 16 a CTA loads 8 KB; alone on a 128 x 256 tile it
// would load 12 KB for the same work, more than L2 gives an SM in that time. Roles inside a CTA: one thread issues the TMA loads (a ring of kStages blocks of 64 along K), one
// thread of the pair's first CTA issues the MMAs, eight warps read the sums back and run the epilogue while the other half
// of the tensor memory (2 x 256 columns) takes the next tile. Persistent: tiles are handed out round robin.
//
// Operands are 16-bit, either fp16 (in words, see below) or bf16, each K-major (K contiguous) or MN-major (the other
// index contiguous); the 128-byte swizzle of TMA is the one the MMA descriptors name. Everything outside a matrix is
// read as zero, so any M, N and K work.
//
// Words: an fp32 operand x is held as two fp16 words, hi = fp16(s x), lo = fp16((s x - hi) 2^11), s a power of two that puts the largest
// element just below 2^15. That keeps 22 bits of every element down to 2^-28 of the largest one, and 2^-50 of the largest one
// below (a low word without its 2^11 would run into fp16's smallest numbers 11 bits earlier). A product is then three passes over K,
// lo*hi + hi*lo + hi*hi: the small terms first, in a stay of their own whose sums are taken times 2^-11 when they are read back.
//
// Sums: the tensor core cuts, rather than rounds, each addition to its fp32 sums, an error that adds up with one sign over
// thousands of steps. With kPromote the sums leave tensor memory every `flush` K blocks and are added up in registers (the passes
// of the small terms, 2^-11 of the others, make one stay). Products of two words are always promoted.
//
// What bounds it, measured: a block of 64 along K takes 610 cycles (560 with the loads left out): the tensor core. Launch by launch (no power cap)
// the products of the loss of 8,192 x 65,536 x 2,048 bf16 run at 1.41 PFLOP/s (statistics, in stays of 16 blocks), 1.29 (P, which is written), 1.38 (head's gradient) and
// 1.22 (hidden's, added to kept sums); the call as a whole, eight of T V H, at 1.13 to 1.15 under the cap. Three-pass products: 1.1 PFLOP/s at
// 2,048 x 32,000 x 512, where reading the sums back takes the accumulators' port for 700 cycles a stay. A launch costs about 8 us beside its blocks (first
// loads 1.6, epilogue 3 to 5, end 1.2, start of the next 1.7), which is what bounds small ones.
//
// Every wait has a limit in time (kWaitNs); a kernel that runs into it sets *gave_up (pinned host memory: the next call sees it without
// waiting for the GPU), waits for its copies, frees its tensor memory and returns.
#pragma once

#include <cuda.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>

#include "lm_ops.h"

namespace a2 {

constexpr int kTileM = 256, kTileN = 256, kBlockK = 64;
constexpr int kStages = 6;
constexpr int kOperandBytes = 128 * kBlockK * 2;           // one CTA's rows of one operand, one stage
constexpr int kStageBytes = 2 * kOperandBytes;             // 32 KB
constexpr int kEpilogueWarps = 8;
constexpr int kGemmThreads = (kEpilogueWarps + 4) * 32;   // loads, products and two idle warps (registers are split by groups of four)
constexpr int kStagePitch = 33;                            // floats; odd, so rows and columns are both free of bank conflicts
constexpr int kWarpStaging = 32 * kStagePitch * 4;         // bytes; a multiple of 128
constexpr int kStagingBytes = kEpilogueWarps * kWarpStaging;
constexpr int kGemmSmem = kStages * kStageBytes + kStagingBytes + 256 + 1024;  // barriers, alignment
static_assert(kGemmSmem <= 227 * 1024, "shared memory of one CTA");
constexpr uint32_t kTryNs = 100000;  // a try sleeps up to this long, so that waiting warps leave the issue slots to the others
constexpr unsigned long long kWaitNs = 4000000000ull;

struct GemmArgs {
    CUtensorMap a[2], b[2];                // word 0 (or the only one) and word 1
    CUtensorMap a_mirror[2], b_mirror[2];  // the same as MN-major operands, where symmetric
    int32_t tiles_m, tiles_n, batch;
    int32_t k_blocks;
    int32_t splits;  // parts of K, summed up by the caller's epilogue and a later kernel
    int32_t passes;  // 1, or 3 for operands of two words
    int32_t flush;   // K blocks of the last pass per stay in tensor memory (kPromote)
    uint32_t idesc;
    uint32_t a_mn, b_mn;    // MN-major operand
    uint32_t a_sym, b_sym;  // symmetric, only tiles on and below the diagonal stored: the others are read from their mirror images
    uint32_t lower;       // only tiles on and below the diagonal (tiles_m == tiles_n)
    int* gave_up;
};

// ---- host side --------------------------------------------------------------------------------
struct Operand {  // a 16-bit matrix, K-major [rows, k] or MN-major [k, rows], `mats` of them
    const void* p;
    const void* lo;        // second word, or NULL
    int64_t rows, k;
    int64_t pitch, stride;  // elements, row to row and matrix to matrix
    bool mn;
    bool symmetric = false;  // rows == k, K-major
};
[[nodiscard]] cudaError_t make_gemm(const Operand& a, const Operand& b, int64_t mats, bool bf16, bool lower, int flush, int splits, GemmArgs* out);
[[nodiscard]] cudaError_t gave_up_flag(int** out);  // where kernels note a wait that ran out on the current device
int gemm_clusters();  // CTA pairs that run at once on the current device

#ifdef __CUDACC__

namespace ptx {

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t cta_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t on_leader(uint32_t addr) {  // the same place in the pair's first CTA
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "r"(kTryNs)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ unsigned long long now_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ bool bar_wait_slow(uint32_t bar, uint32_t parity, int* gave_up) {
    if (bar_try(bar, parity)) return true;  // a try sleeps until the phase ends or kTryNs are over: seldom more than two
    const unsigned long long start = now_ns();
    while (!bar_try(bar, parity))
        if (now_ns() - start > kWaitNs) {
            *static_cast<volatile int*>(gave_up) = 1;
            __threadfence_system();
            return false;
        }
    return true;
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, int* gave_up) {
    return bar_try(bar, parity) || bar_wait_slow(bar, parity, gave_up);
}

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint32_t leader_bar, int x, int y, int z) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
        "l"(map), "r"(leader_bar), "r"(x), "r"(y), "r"(z)
        : "memory");
}
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(add)
        : "memory");
}
__device__ __forceinline__ void commit_both(uint32_t bar) {  // arrives at `bar` in both CTAs once the MMAs issued so far are done
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3)
                 : "memory");
}
__device__ __forceinline__ void mma_one(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {  // a CTA by itself
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(add)
        : "memory");
}
__device__ __forceinline__ void commit_one(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_load32(float (&v)[32], uint32_t addr) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
          "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
          "=r"(r[31])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int k = 0; k < 32; ++k) v[k] = __uint_as_float(r[k]);
}
// The same as pairs of columns, for packed additions.
__device__ __forceinline__ void tmem_load_pairs(uint64_t (&v)[16], uint32_t addr) {
    float f[32];
    tmem_load32(f, addr);
#pragma unroll
    for (int k = 0; k < 16; ++k) asm volatile("mov.b64 %0, {%1, %2};" : "=l"(v[k]) : "f"(f[2 * k]), "f"(f[2 * k + 1]));
}
__device__ __forceinline__ uint64_t pair(float v) {
    uint64_t p;
    asm("mov.b64 %0, {%1, %1};" : "=l"(p) : "f"(v));
    return p;
}
__device__ __forceinline__ void tmem_store_pairs(uint32_t addr, const uint64_t* p) {
    uint32_t v[32];
#pragma unroll
    for (int k = 0; k < 16; ++k) asm volatile("mov.b64 {%0, %1}, %2;" : "=r"(v[2 * k]), "=r"(v[2 * k + 1]) : "l"(p[k]));
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(v[0]),
        "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]),
        "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]),
        "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

}  // namespace ptx

// The fp32-sum instruction descriptor: fp16 (0) or bf16 (1) operands, MN-major bits, N / 8 and M / 16.
__host__ __device__ constexpr uint32_t instruction_desc(bool bf16, bool a_mn, bool b_mn, int m, int n) {
    return 1u << 4 | (bf16 ? 1u : 0u) << 7 | (bf16 ? 1u : 0u) << 10 | (a_mn ? 1u : 0u) << 15 | (b_mn ? 1u : 0u) << 16 | (uint32_t)(n / 8) << 17 |
           (uint32_t)(m / 16) << 24;
}

// Shared-memory descriptor of an operand tile under the 128-byte swizzle. K-major: rows of 128 bytes (64 along K), groups of
// eight rows 1024 bytes apart. MN-major: boxes of 64 along MN by 64 along K, 8 KB each; the leading offset steps from box to
// box along MN, the stride offset over eight steps of K.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, bool mn, uint32_t box_bytes = 8192) {
    const uint64_t leading = mn ? box_bytes >> 4 : 1, stride = 1024 >> 4;
    return (uint64_t)((addr & 0x3ffff) >> 4) | leading << 16 | stride << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

// K blocks of the stay in tensor memory that begins at block `done` of `blocks` (all passes).
template <bool kPromote>
__device__ __forceinline__ int stay_end(const GemmArgs& g, int done, int blocks) {
    if (!kPromote) return blocks;
    const int small = g.passes == 1 ? 0 : blocks / 3 * 2;
    return done < small ? small : min(done + g.flush, blocks);
}

struct Tile {
    int b, m, n;      // matrix, tile row, tile column
    int split, k0, k1;  // part of K, in blocks
};
__device__ __forceinline__ int tiles_of(const GemmArgs& g) {
    return g.batch * g.splits * (g.lower ? g.tiles_m * (g.tiles_m + 1) / 2 : g.tiles_m * g.tiles_n);
}
__device__ __forceinline__ Tile tile_at(const GemmArgs& g, int t) {
    const int per = g.lower ? g.tiles_m * (g.tiles_m + 1) / 2 : g.tiles_m * g.tiles_n;
    Tile r;
    r.split = t / (g.batch * per);  // parts of one tile far apart: they read different blocks
    t -= r.split * g.batch * per;
    r.k0 = (int)((int64_t)g.k_blocks * r.split / g.splits);
    r.k1 = (int)((int64_t)g.k_blocks * (r.split + 1) / g.splits);
    r.b = t / per;
    t -= r.b * per;
    if (g.lower) {
        r.m = (int)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
        while (r.m * (r.m + 1) / 2 > t) --r.m;
        while ((r.m + 1) * (r.m + 2) / 2 <= t) ++r.m;
        r.n = t - r.m * (r.m + 1) / 2;
    } else if (g.tiles_m <= g.tiles_n) {  // along the shorter side first: the larger operand streams once, the other stays in L2
        r.n = t / g.tiles_m;
        r.m = t - r.n * g.tiles_m;
    } else {
        r.m = t / g.tiles_n;
        r.n = t - r.m * g.tiles_n;
    }
    return r;
}

// 32 x 32 16-bit values, a row a lane, to rows of a matrix: through shared memory (2 KB, 16-byte pieces swizzled free of
// bank conflicts), so that an instruction writes 8 rows of 64 bytes and not 32 pieces of 16.
template <class H>
__device__ __forceinline__ void store_rows16(void* staging, const H (&v)[32], H* to, int64_t ld, int rows, int lane) {
    static_assert(sizeof(H) == 2, "16-bit values");
    char* s = static_cast<char*>(staging);
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        Pack<H, 8> p;
#pragma unroll
        for (int k = 0; k < 8; ++k) p.v[k] = v[c * 8 + k];
        *reinterpret_cast<Pack<H, 8>*>(s + lane * 64 + ((c ^ ((lane >> 1) & 3)) * 16)) = p;
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i * 8 + lane / 4, c = lane % 4;
        const Pack<H, 8> p = *reinterpret_cast<const Pack<H, 8>*>(s + r * 64 + ((c ^ ((r >> 1) & 3)) * 16));
        if (r < rows) *reinterpret_cast<Pack<H, 8>*>(to + r * ld + c * 8) = p;
    }
}

// The same from rows of a matrix to a row a lane.
template <class H>
__device__ __forceinline__ void load_rows16(void* staging, H (&v)[32], const H* from, int64_t ld, int rows, int lane) {
    char* s = static_cast<char*>(staging);
    Pack<H, 8> p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i * 8 + lane / 4, c = lane % 4;
        if (r < rows) p[i] = *reinterpret_cast<const Pack<H, 8>*>(from + r * ld + c * 8);
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i * 8 + lane / 4, c = lane % 4;
        *reinterpret_cast<Pack<H, 8>*>(s + r * 64 + ((c ^ ((r >> 1) & 3)) * 16)) = p[i];
    }
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const Pack<H, 8> q = *reinterpret_cast<const Pack<H, 8>*>(s + lane * 64 + ((c ^ ((lane >> 1) & 3)) * 16));
#pragma unroll
        for (int k = 0; k < 8; ++k) v[c * 8 + k] = q.v[k];
    }
}

// 32 x 32 sums, a row a lane, turned in shared memory into a column a lane: v[r] is then row r of the lane's column, so that a
// warp reads and writes 32 columns of a row side by side, whatever the alignment.
__device__ __forceinline__ void turn_columns(float* staging, float (&v)[32], int lane) {
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 32; ++k) staging[lane * kStagePitch + k] = v[k];
    __syncwarp();
#pragma unroll
    for (int r = 0; r < 32; ++r) v[r] = staging[r * kStagePitch + lane];
}

// Parts of K that let `tiles` tiles fill the pairs of CTAs, each part with at least `least` blocks of K.
inline int split_parts(int64_t tiles, int64_t k_blocks, int64_t pairs, int64_t least) {
    const int64_t parts = std::min(pairs / std::max<int64_t>(1, tiles), k_blocks / least);
    return (int)std::max<int64_t>(1, parts);
}

// v * 2^e in two factors, so that no intermediate leaves the range unless the result does.
struct PowerOfTwo {
    float a, b;
    __device__ __forceinline__ explicit PowerOfTwo(int e) {
        e = max(-250, min(250, e));
        a = ldexpf(1.0f, e / 2);
        b = ldexpf(1.0f, e - e / 2);
    }
    __device__ __forceinline__ float operator()(float v) const { return v * a * b; }
};

constexpr int kLowUp = 2048;  // low words are held times this

// x as hi + lo / kUp.
template <int kUp = kLowUp>
__device__ __forceinline__ void split_words(float x, __half& hi, __half& lo) {
    hi = __float2half_rn(x);
    const float back = __half2float(hi);
    lo = __float2half_rn(fabsf(back) <= 65504.0f ? (x - back) * kUp : 0.0f);
}

// A pair of finite values in packed conversions, for the epilogues.
template <int kUp = kLowUp>
__device__ __forceinline__ void split_pair(float x, float y, __half& hx, __half& hy, __half& lx, __half& ly) {
    const __half2 h = __floats2half2_rn(x, y);
    const float2 back = __half22float2(h);
    float2 low{x - back.x, y - back.y};
    if constexpr (kUp != 1) {  // the difference times kUp in two packed instructions; exact, for kUp is a power of two
        uint64_t both, rest;
        asm("mov.b64 %0, {%1, %2};" : "=l"(both) : "f"(x), "f"(y));
        asm("mov.b64 %0, {%1, %2};" : "=l"(rest) : "f"(back.x), "f"(back.y));
        asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(rest) : "l"(ptx::pair(-kUp)));
        asm("fma.rn.f32x2 %0, %0, %1, %2;" : "+l"(both) : "l"(ptx::pair(kUp)), "l"(rest));
        asm("mov.b64 {%0, %1}, %2;" : "=f"(low.x), "=f"(low.y) : "l"(both));
    }
    const __half2 l = __floats2half2_rn(low.x, low.y);
    hx = __low2half(h);
    hy = __high2half(h);
    lx = __low2half(l);
    ly = __high2half(l);
}

// The first block of K that an operand is read MN-major from: all of them, none, or, of a symmetric one, those above the diagonal.
__device__ __forceinline__ int turned_from(uint32_t mn, uint32_t symmetric, int tile, const Tile& t) {
    return mn ? t.k0 : symmetric ? min(t.k1, (tile + 1) * (kTileM / kBlockK)) : t.k1;
}
// The blocks from kb on that both operands read the same way end here.
__device__ __forceinline__ int run_end(int kb, int from_a, int from_b, int k1) {
    int end = k1;
    if (kb < from_a) end = min(end, from_a);
    if (kb < from_b) end = min(end, from_b);
    return end;
}

// A CTA's 128 rows of one block: one box of 64 (along K) x 128 rows, or two of 64 x 64 (along K) side by side. (Boxes of 64 x 64 for
// K-major operands too would do with one map, but cost 20 % of the rate of a long product.)
__device__ __forceinline__ void load_operand(const CUtensorMap* map, bool turned, uint32_t to, uint32_t bar, int row, int k, int mat) {
    if (turned) {
        ptx::tma_load(to, map, bar, row, k, mat);
        ptx::tma_load(to + 8192, map, bar, row + 64, k, mat);
    } else {
        ptx::tma_load(to, map, bar, k, row, mat);
    }
}

// Epilogue: constructed per tile by every thread of the eight warps as
//   Epi(args, tile, row of lane 0 of the warp, first column of the thread's 128, lane, staging of the warp)
// then chunk(c, v) for c = 0 .. 3 with the sums of row (row0 + lane), columns col0 + 32 c .., then finish().
//
// A launch takes one product or two independent ones (kJobs), whose tiles it hands out one after the other: two that would each
// leave CTAs idle fill the GPU together.
template <class Epi, int kJobs>
struct Jobs {
    GemmArgs g[kJobs];
    typename Epi::Args args[kJobs];
};

template <class Epi, bool kPromote, int kJobs>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGemmThreads, 1) k_gemm(const __grid_constant__ Jobs<Epi, kJobs> jobs) {
    extern __shared__ char raw[];
    char* smem = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    float* staging = reinterpret_cast<float*>(smem + kStages * kStageBytes);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kStages * kStageBytes + kStagingBytes);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * kStages + 4);
    const uint32_t full = ptx::smem_addr(bars), empty = full + 8 * kStages, acc_full = empty + 8 * kStages, acc_empty = acc_full + 16;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = ptx::cta_rank();

    if (warp == kEpilogueWarps + 1 && lane == 0)
        for (int w = 0; w < (jobs.g[0].passes == 1 ? 1 : 2); ++w) {
            asm volatile("prefetch.tensormap [%0];" ::"l"(&jobs.g[0].a[w]) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&jobs.g[0].b[w]) : "memory");
        }
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            ptx::bar_init(full + 8 * s, 1);
            ptx::bar_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            ptx::bar_init(acc_full + 8 * s, 1);
            ptx::bar_init(acc_empty + 8 * s, 2 * kEpilogueWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kEpilogueWarps) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(ptx::smem_addr(tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        ptx::fence_before();
    }
    __syncthreads();
    ptx::cluster_sync();
    ptx::fence_after();
    const uint32_t tmem = *tmem_slot;
    ptx::release_next();
    ptx::wait_previous();

    const int first_tiles = tiles_of(jobs.g[0]), n_tiles = first_tiles + (kJobs > 1 ? tiles_of(jobs.g[kJobs - 1]) : 0);
    const int first = blockIdx.x / 2, step = gridDim.x / 2;
    int* const gave_up = jobs.g[0].gave_up;
    auto job_of = [&](int t) { return kJobs > 1 && t >= first_tiles ? 1 : 0; };
    const uint32_t ring = ptx::smem_addr(smem);

    // 384 threads start with 168 registers each (64,512). The sums kept in registers need more than that in the epilogue's eight
    // warps: 256 * 224 + 128 * 56 = 64,512.
    if (warp >= kEpilogueWarps) {
        if constexpr (kPromote) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        // One thread issues the loads and one the products; each must get through a block in the 512 cycles that its products
        // take, at a handful of cycles per instruction: what does not change from block to block stays out of their loops.
        if (warp == kEpilogueWarps && lane == 0) {  // loads
            uint32_t s = 0, parity = 1;  // a fresh barrier counts as one whose phase 1 is over
            bool ok = true;
            const uint32_t leader_full = ptx::on_leader(full);
            for (int t = first; t < n_tiles && ok; t += step) {
                const GemmArgs& g = jobs.g[job_of(t)];
                const Tile at = tile_at(g, t - job_of(t) * first_tiles);
                const int row_a = at.m * kTileM + rank * 128, row_b = at.n * kTileN + rank * 128;
                const int from_a = turned_from(g.a_mn, g.a_sym, at.m, at), from_b = turned_from(g.b_mn, g.b_sym, at.n, at);
                for (int pass = 0; pass < g.passes && ok; ++pass) {
                    const bool one = g.passes == 1;
                    const int wa = one ? 0 : pass == 0, wb = one ? 0 : pass == 1;  // lo hi, hi lo, hi hi
                    for (int kb = at.k0; kb < at.k1 && ok;) {
                        const bool turn_a = kb >= from_a, turn_b = kb >= from_b;
                        const CUtensorMap* ma = turn_a && !g.a_mn ? &g.a_mirror[wa] : &g.a[wa];
                        const CUtensorMap* mb = turn_b && !g.b_mn ? &g.b_mirror[wb] : &g.b[wb];
                        const int end = run_end(kb, from_a, from_b, at.k1);
                        for (; kb < end; ++kb) {
                            if (!(ok = ptx::bar_wait(empty + 8 * s, parity, gave_up))) break;
                            const uint32_t sa = ring + s * kStageBytes;
                            if (rank == 0) ptx::bar_expect(full + 8 * s, 2 * kStageBytes);
                            load_operand(ma, turn_a, sa, leader_full + 8 * s, row_a, kb * kBlockK, at.b);
                            load_operand(mb, turn_b, sa + kOperandBytes, leader_full + 8 * s, row_b, kb * kBlockK, at.b);
                            if (++s == kStages) s = 0, parity ^= 1;
                        }
                    }
                }
            }
            // the last products' signals to this CTA: all of them have arrived once the whole ring is free again
            for (int k = 0; k < kStages && ok; ++k) {
                ok = ptx::bar_wait(empty + 8 * s, parity, gave_up);
                if (++s == kStages) s = 0, parity ^= 1;
            }
            if (!ok) {  // gave up: leave the copies in flight time to land before the CTA goes
                const unsigned long long start = ptx::now_ns();
                while (ptx::now_ns() - start < 10000000ull) {
                }
            }
        }
        if (warp == kEpilogueWarps + 1 && lane == 0 && rank == 0) {  // products
            uint32_t s = 0, parity = 0, buf = 0, acc_parity = 1;
            bool ok = true;
            for (int t = first; t < n_tiles && ok; t += step) {
                const GemmArgs& g = jobs.g[job_of(t)];
                const Tile at = tile_at(g, t - job_of(t) * first_tiles);
                const int from_a = turned_from(g.a_mn, g.a_sym, at.m, at), from_b = turned_from(g.b_mn, g.b_sym, at.n, at);
                const int blocks = (at.k1 - at.k0) * g.passes;
                int kb = at.k0;
                for (int done = 0; done < blocks && ok;) {
                    const int end = stay_end<kPromote>(g, done, blocks);
                    if (!(ok = ptx::bar_wait(acc_empty + 8 * buf, acc_parity, gave_up))) break;
                    ptx::fence_after();
                    const uint32_t d = tmem + buf * kTileN;
                    uint32_t add = 0;
                    while (done < end && ok) {
                        if (kb == at.k1) kb = at.k0;  // the next pass
                        const bool turn_a = kb >= from_a, turn_b = kb >= from_b;
                        const int run = min(end - done, run_end(kb, from_a, from_b, at.k1) - kb);
                        const uint32_t idesc = g.idesc | (turn_a ? 1u << 15 : 0u) | (turn_b ? 1u << 16 : 0u);
                        const uint32_t step_a = turn_a ? 2048 >> 4 : 32 >> 4, step_b = turn_b ? 2048 >> 4 : 32 >> 4;  // 16 along K
                        const uint64_t base_a = operand_desc(ring, turn_a), base_b = operand_desc(ring + kOperandBytes, turn_b);
                        for (int k = 0; k < run; ++k) {
                            if (!(ok = ptx::bar_wait(full + 8 * s, parity, gave_up))) break;
                            ptx::fence_after();
                            const uint64_t da = base_a + s * (kStageBytes >> 4), db = base_b + s * (kStageBytes >> 4);
                            ptx::mma(d, da, db, idesc, add);
                            ptx::mma(d, da + step_a, db + step_b, idesc, 1);
                            ptx::mma(d, da + 2 * step_a, db + 2 * step_b, idesc, 1);
                            ptx::mma(d, da + 3 * step_a, db + 3 * step_b, idesc, 1);
                            ptx::commit_both(empty + 8 * s);
                            add = 1;
                            if (++s == kStages) s = 0, parity ^= 1;
                        }
                        kb += run;
                        done += run;
                    }
                    if (ok) ptx::commit_both(acc_full + 8 * buf);
                    buf ^= 1;
                    if (buf == 0) acc_parity ^= 1;
                }
            }
        }
    } else {
        if constexpr (kPromote) asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        const int quad = warp % 4, half = warp / 4;
        const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16) + half * 128;
        const uint32_t leader_empty = ptx::on_leader(acc_empty);
        float* mine = staging + warp * 32 * kStagePitch;
        uint32_t chunk = 0;
        bool ok = true;
        for (int t = first; t < n_tiles && ok; t += step) {
            const GemmArgs& g = jobs.g[job_of(t)];
            const Tile at = tile_at(g, t - job_of(t) * first_tiles);
            Epi epi(jobs.args[job_of(t)], at, at.m * kTileM + rank * 128 + quad * 32, at.n * kTileN + half * 128, lane, mine);
            uint32_t buf = chunk & 1;
            if constexpr (kPromote) {
                const int blocks = (at.k1 - at.k0) * g.passes;
                if (stay_end<true>(g, 0, blocks) < blocks) {
                    uint64_t sum[64];  // pairs of columns
#pragma unroll
                    for (int k = 0; k < 64; ++k) sum[k] = 0;
                    // what a stay's sums are worth: the first one of a product of words is that of the small terms
                    uint64_t worth = g.passes == 1 ? ptx::pair(1.0f) : ptx::pair(1.0f / kLowUp);
#pragma unroll 1
                    for (int done = 0;;) {
                        buf = chunk & 1;
                        if (!(ok = ptx::bar_wait(acc_full + 8 * buf, (chunk >> 1) & 1, gave_up))) break;
                        ptx::fence_after();
#pragma unroll
                        for (int c = 0; c < 4; c += 2) {
                            uint64_t v[2][16];
                            ptx::tmem_load_pairs(v[0], lanes + buf * kTileN + c * 32);
                            ptx::tmem_load_pairs(v[1], lanes + buf * kTileN + c * 32 + 32);
                            ptx::tmem_load_wait();
#pragma unroll
                            for (int k = 0; k < 32; ++k)
                                asm volatile("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(sum[c * 16 + k]) : "l"(v[k / 16][k % 16]), "l"(worth));
                        }
                        worth = ptx::pair(1.0f);
                        done = stay_end<true>(g, done, blocks);
                        if (done == blocks) break;  // the last stay: the epilogue reads it below
                        ptx::fence_before();
                        __syncwarp();
                        if (lane == 0) ptx::bar_arrive_cluster(leader_empty + 8 * buf);
                        ++chunk;
                    }
                    if (!ok) break;
#pragma unroll
                    for (int c = 0; c < 4; ++c) ptx::tmem_store_pairs(lanes + buf * kTileN + c * 32, sum + c * 16);
                    ptx::tmem_store_wait();
                } else if (!(ok = ptx::bar_wait(acc_full + 8 * buf, (chunk >> 1) & 1, gave_up))) {
                    break;
                }
            } else if (!(ok = ptx::bar_wait(acc_full + 8 * buf, (chunk >> 1) & 1, gave_up))) {
                break;
            }
            ++chunk;
            ptx::fence_after();
            // not unrolled: most launches run the epilogue once or a few times, and fetching its instructions is what it then waits for
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
                float v[32];
                ptx::tmem_load32(v, lanes + buf * kTileN + c * 32);
                ptx::tmem_load_wait();
                if (c == 3) {
                    ptx::fence_before();
                    __syncwarp();
                    if (lane == 0) ptx::bar_arrive_cluster(leader_empty + 8 * buf);
                }
                epi.chunk(c, v);
            }
            epi.finish();
        }
    }
    // neither CTA may leave, or free tensor memory, while the other still reads its shared memory or signals its barriers
    __syncthreads();
    ptx::cluster_sync();
    if (warp == kEpilogueWarps) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

template <class Epi, bool kPromote, int kJobs>
[[nodiscard]] cudaError_t launch_jobs(const Jobs<Epi, kJobs>& jobs, cudaStream_t s) {
    int64_t tiles = 0;
    for (const GemmArgs& g : jobs.g)
        if (g.passes != 1 && !kPromote) return cudaErrorInvalidValue;  // the small terms need a stay of their own
    for (const GemmArgs& g : jobs.g)
        tiles += (int64_t)g.batch * g.splits * (g.lower ? (int64_t)g.tiles_m * (g.tiles_m + 1) / 2 : (int64_t)g.tiles_m * g.tiles_n);
    if (tiles == 0) return cudaSuccess;
    static std::atomic<uint64_t> allowed;
    const cudaError_t e = allow_shared_memory(reinterpret_cast<const void*>(k_gemm<Epi, kPromote, kJobs>), kGemmSmem, allowed);
    if (e != cudaSuccess) return e;
    const int64_t clusters = std::min<int64_t>(tiles, gemm_clusters());
    return launch_chained(k_gemm<Epi, kPromote, kJobs>, dim3((unsigned)(2 * clusters)), kGemmThreads, kGemmSmem, s, jobs);
}
template <class Epi, bool kPromote>
[[nodiscard]] cudaError_t launch_gemm(const GemmArgs& g, const typename Epi::Args& args, cudaStream_t s) {
    return launch_jobs<Epi, kPromote, 1>(Jobs<Epi, 1>{{g}, {args}}, s);
}
// Two independent products of one kind.
template <class Epi, bool kPromote>
[[nodiscard]] cudaError_t launch_gemms(const GemmArgs& g, const typename Epi::Args& args, const GemmArgs& h, const typename Epi::Args& more, cudaStream_t s) {
    return launch_jobs<Epi, kPromote, 2>(Jobs<Epi, 2>{{g, h}, {args, more}}, s);
}
#endif

}  // namespace a2
