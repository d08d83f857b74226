// Matrix products on the 5th-generation tensor cores: C[b] = A[b] B[b]^T summed in fp32, with an epilogue of the caller's.
//
// A pair of CTAs (a cluster of two, cta_group::2) makes one 256 x 256 tile: each CTA holds 128 rows of A and 128 rows of
// B in shared memory and 128 x 256 sums in its tensor memory. Per K step of 16 a CTA's tensor core works 128 cycles on
// 8 KB that come from L2, half of what a CTA alone on a 128 x 256 tile would need with the 12 KB it would load; that is
// what the pair is for. Roles inside a CTA: one thread issues the TMA loads (a ring of kStages blocks of 64 along K), one
// thread of the pair's first CTA issues the MMAs, eight warps read the sums back and run the epilogue while the other half
// of the tensor memory (2 x 256 columns) takes the next tile. Persistent: tiles are handed out round robin.
//
// Operands are 16-bit, either fp16 (in words, see below) or bf16, each K-major (K contiguous) or MN-major (the other
// index contiguous); the 128-byte swizzle of TMA is the one the MMA descriptors name. Everything outside a matrix is
// read as zero, so any M, N and K work.
//
// Words: an fp32 operand x is held as two fp16 words, hi = fp16(s x), lo = fp16(s x - hi), s a power of two that puts the largest
// element just below 2^15. That keeps 22 bits of every element down to 2^-18 of the largest one, and 2^-40 of the largest one
// below. A product is then three passes over K, lo*hi + hi*lo + hi*hi (small terms first).
//
// Sums: the tensor core cuts, rather than rounds, each addition to its fp32 sums, an error that adds up with one sign over
// thousands of steps. With kPromote the sums leave tensor memory every `flush` K blocks and are added up in registers.
//
// Every wait has a limit in time (kWaitNs); a kernel that runs into it sets *gave_up, waits for its copies, frees its
// tensor memory and returns.
#pragma once

#include <cuda.h>
#include <cuda_fp16.h>

#include "lm_ops.h"

namespace a2 {

constexpr int kTileM = 256, kTileN = 256, kBlockK = 64;
constexpr int kStages = 6;
constexpr int kOperandBytes = 128 * kBlockK * 2;           // one CTA's rows of one operand, one stage
constexpr int kStageBytes = 2 * kOperandBytes;             // 32 KB
constexpr int kEpilogueWarps = 8;
constexpr int kGemmThreads = (kEpilogueWarps + 4) * 32;   // loads, products and two idle warps (registers are split by groups of four)
constexpr int kStagePitch = 33;                            // floats; odd, so rows and columns are both free of bank conflicts
constexpr int kStagingBytes = kEpilogueWarps * 32 * kStagePitch * 4;
constexpr int kGemmSmem = kStages * kStageBytes + kStagingBytes + 256 + 1024;  // barriers, alignment
static_assert(kGemmSmem <= 227 * 1024, "shared memory of one CTA");
constexpr unsigned long long kWaitNs = 4000000000ull;

struct GemmArgs {
    CUtensorMap a[2], b[2];  // word 0 (or the only one) and word 1
    int32_t tiles_m, tiles_n, batch;
    int32_t k_blocks;
    int32_t passes;  // 1, or 3 for operands of two words
    int32_t flush;   // K blocks per stay in tensor memory (all of them without kPromote)
    uint32_t idesc;
    uint32_t a_mn, b_mn;  // MN-major operand
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
};
cudaError_t make_gemm(const Operand& a, const Operand& b, int64_t mats, bool bf16, bool lower, int flush, GemmArgs* out);
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
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ unsigned long long now_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ bool bar_wait_slow(uint32_t bar, uint32_t parity, int* gave_up) {
    const unsigned long long start = now_ns();
    while (!bar_try(bar, parity))
        if (now_ns() - start > kWaitNs) {
            atomicExch(gave_up, 1);
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
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

}  // namespace ptx

// Shared-memory descriptor of an operand tile under the 128-byte swizzle. K-major: rows of 128 bytes (64 along K), groups of
// eight rows 1024 bytes apart. MN-major: boxes of 64 along MN by 64 along K, 8 KB each; the leading offset steps from box to
// box along MN, the stride offset over eight steps of K.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, bool mn) {
    const uint64_t leading = mn ? 8192 >> 4 : 1, stride = 1024 >> 4;
    return (uint64_t)((addr & 0x3ffff) >> 4) | leading << 16 | stride << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

struct Tile {
    int b, m, n;  // matrix, tile row, tile column
};
__device__ __forceinline__ Tile tile_at(const GemmArgs& g, int t) {
    const int per = g.lower ? g.tiles_m * (g.tiles_m + 1) / 2 : g.tiles_m * g.tiles_n;
    Tile r;
    r.b = t / per;
    t -= r.b * per;
    if (g.lower) {
        r.m = (int)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
        while (r.m * (r.m + 1) / 2 > t) --r.m;
        while ((r.m + 1) * (r.m + 2) / 2 <= t) ++r.m;
        r.n = t - r.m * (r.m + 1) / 2;
    } else {  // down a column of tiles first: B's rows stream once, A's stay in L2
        r.n = t / g.tiles_m;
        r.m = t - r.n * g.tiles_m;
    }
    return r;
}

// Epilogue: constructed per tile by every thread of the eight warps as
//   Epi(args, matrix, row of lane 0 of the warp, first column of the thread's 128, lane, staging of the warp)
// then chunk(c, v) for c = 0 .. 3 with the sums of row (row0 + lane), columns col0 + 32 c .., then finish().
template <class Epi, bool kPromote>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGemmThreads, 1)
    k_gemm(const __grid_constant__ GemmArgs g, const __grid_constant__ typename Epi::Args args) {
    extern __shared__ char raw[];
    char* smem = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    float* staging = reinterpret_cast<float*>(smem + kStages * kStageBytes);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kStages * kStageBytes + kStagingBytes);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * kStages + 4);
    const uint32_t full = ptx::smem_addr(bars), empty = full + 8 * kStages, acc_full = empty + 8 * kStages, acc_empty = acc_full + 16;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = ptx::cta_rank();

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

    const int n_tiles = g.batch * (g.lower ? g.tiles_m * (g.tiles_m + 1) / 2 : g.tiles_m * g.tiles_n);
    const int first = blockIdx.x / 2, step = gridDim.x / 2;
    const int blocks = g.k_blocks * g.passes;
    const uint32_t ring = ptx::smem_addr(smem);

    // 384 threads start with 168 registers each (64,512). The sums kept in registers need more than that in the epilogue's eight
    // warps: 256 * 232 + 128 * 40 = 64,512.
    if (warp >= kEpilogueWarps) {
        if constexpr (kPromote) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == kEpilogueWarps && lane == 0) {  // loads
            uint32_t it = 0;
            bool ok = true;
            for (int t = first; t < n_tiles && ok; t += step) {
                const Tile at = tile_at(g, t);
                const int row_a = at.m * kTileM + rank * 128, row_b = at.n * kTileN + rank * 128;
                for (int pass = 0; pass < g.passes && ok; ++pass) {
                    const bool one = g.passes == 1;
                    const CUtensorMap* ma = &g.a[one ? 0 : pass == 0];      // lo, hi, hi
                    const CUtensorMap* mb = &g.b[one ? 0 : pass == 1];      // hi, lo, hi
                    for (int kb = 0; kb < g.k_blocks; ++kb, ++it) {
                        const uint32_t s = it % kStages, round = it / kStages;
                        if (round > 0 && !(ok = ptx::bar_wait(empty + 8 * s, (round - 1) & 1, g.gave_up))) break;
                        const uint32_t sa = ring + s * kStageBytes, sb = sa + kOperandBytes;
                        const uint32_t bar = ptx::on_leader(full + 8 * s);
                        if (rank == 0) ptx::bar_expect(full + 8 * s, 2 * kStageBytes);
                        if (g.a_mn) {
                            ptx::tma_load(sa, ma, bar, row_a, kb * kBlockK, at.b);
                            ptx::tma_load(sa + 8192, ma, bar, row_a + 64, kb * kBlockK, at.b);
                        } else {
                            ptx::tma_load(sa, ma, bar, kb * kBlockK, row_a, at.b);
                        }
                        if (g.b_mn) {
                            ptx::tma_load(sb, mb, bar, row_b, kb * kBlockK, at.b);
                            ptx::tma_load(sb + 8192, mb, bar, row_b + 64, kb * kBlockK, at.b);
                        } else {
                            ptx::tma_load(sb, mb, bar, kb * kBlockK, row_b, at.b);
                        }
                    }
                }
            }
            // the last products' signals to this CTA: all of them have arrived once the ring is free again
            for (uint32_t s = 0; s < kStages && s < it && ok; ++s) ok = ptx::bar_wait(empty + 8 * s, ((it - 1 - s) / kStages) & 1, g.gave_up);
            if (!ok) {  // gave up: leave the copies in flight time to land before the CTA goes
                const unsigned long long start = ptx::now_ns();
                while (ptx::now_ns() - start < 10000000ull) {
                }
            }
        }
        if (warp == kEpilogueWarps + 1 && lane == 0 && rank == 0) {  // products
            uint32_t it = 0, chunk = 0;
            bool ok = true;
            const uint32_t step_a = g.a_mn ? 2048 >> 4 : 32 >> 4, step_b = g.b_mn ? 2048 >> 4 : 32 >> 4;  // 16 along K
            for (int t = first; t < n_tiles && ok; t += step) {
                for (int done = 0; done < blocks && ok; ++chunk) {
                    const int end = min(done + g.flush, blocks);
                    const uint32_t buf = chunk & 1, use = chunk >> 1;
                    if (use > 0 && !(ok = ptx::bar_wait(acc_empty + 8 * buf, (use - 1) & 1, g.gave_up))) break;
                    ptx::fence_after();
                    const uint32_t d = tmem + buf * kTileN;
                    for (bool begun = false; done < end; ++done, ++it) {
                        const uint32_t s = it % kStages, round = it / kStages;
                        if (!(ok = ptx::bar_wait(full + 8 * s, round & 1, g.gave_up))) break;
                        ptx::fence_after();
                        const uint32_t sa = ring + s * kStageBytes;
                        uint64_t da = operand_desc(sa, g.a_mn), db = operand_desc(sa + kOperandBytes, g.b_mn);
#pragma unroll
                        for (int k = 0; k < kBlockK / 16; ++k) {
                            ptx::mma(d, da, db, g.idesc, begun);
                            begun = true;
                            da += step_a;
                            db += step_b;
                        }
                        ptx::commit_both(empty + 8 * s);
                    }
                    if (ok) ptx::commit_both(acc_full + 8 * buf);
                }
            }
        }
    } else {
        if constexpr (kPromote) asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
        const int quad = warp % 4, half = warp / 4;
        const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16) + half * 128;
        const uint32_t leader_empty = ptx::on_leader(acc_empty);
        float* mine = staging + warp * 32 * kStagePitch;
        uint32_t chunk = 0;
        bool ok = true;
        for (int t = first; t < n_tiles && ok; t += step) {
            const Tile at = tile_at(g, t);
            Epi epi(args, at.b, at.m * kTileM + rank * 128 + quad * 32, at.n * kTileN + half * 128, lane, mine);
            if constexpr (kPromote) {
                float sum[128];
#pragma unroll
                for (int k = 0; k < 128; ++k) sum[k] = 0.0f;
#pragma unroll 1
                for (int done = 0; done < blocks; done += g.flush, ++chunk) {
                    const uint32_t buf = chunk & 1;
                    if (!(ok = ptx::bar_wait(acc_full + 8 * buf, (chunk >> 1) & 1, g.gave_up))) break;
                    ptx::fence_after();
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float v[32];
                        ptx::tmem_load32(v, lanes + buf * kTileN + c * 32);
                        ptx::tmem_load_wait();
#pragma unroll
                        for (int k = 0; k < 32; ++k) asm volatile("add.f32 %0, %0, %1;" : "+f"(sum[c * 32 + k]) : "f"(v[k]));
                    }
                    ptx::fence_before();
                    __syncwarp();
                    if (lane == 0) ptx::bar_arrive_cluster(leader_empty + 8 * buf);
                }
                if (!ok) break;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float v[32];
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] = sum[c * 32 + k];
                    epi.chunk(c, v);
                }
            } else {
                const uint32_t buf = chunk & 1;
                if (!(ok = ptx::bar_wait(acc_full + 8 * buf, (chunk >> 1) & 1, g.gave_up))) break;
                ++chunk;
                ptx::fence_after();
                float v[2][32];
                ptx::tmem_load32(v[0], lanes + buf * kTileN);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    ptx::tmem_load_wait();
                    if (c < 3) {
                        ptx::tmem_load32(v[(c + 1) & 1], lanes + buf * kTileN + (c + 1) * 32);
                    } else {
                        ptx::fence_before();
                        __syncwarp();
                        if (lane == 0) ptx::bar_arrive_cluster(leader_empty + 8 * buf);
                    }
                    epi.chunk(c, v[c & 1]);
                }
            }
            epi.finish();
        }
    }
    // neither CTA may leave, or free tensor memory, while the other still reads its shared memory or signals its barriers
    __syncthreads();
    ptx::cluster_sync();
    if (warp == kEpilogueWarps) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

template <class Epi, bool kPromote>
cudaError_t launch_gemm(const GemmArgs& g, const typename Epi::Args& args, cudaStream_t s) {
    const int64_t tiles = (int64_t)g.batch * (g.lower ? (int64_t)g.tiles_m * (g.tiles_m + 1) / 2 : (int64_t)g.tiles_m * g.tiles_n);
    if (tiles == 0) return cudaSuccess;
    cudaError_t e = cudaFuncSetAttribute(k_gemm<Epi, kPromote>, cudaFuncAttributeMaxDynamicSharedMemorySize, kGemmSmem);
    if (e != cudaSuccess) return e;
    const int64_t clusters = tiles < gemm_clusters() ? tiles : gemm_clusters();
    k_gemm<Epi, kPromote><<<(unsigned)(2 * clusters), kGemmThreads, kGemmSmem, s>>>(g, args);
    return cudaGetLastError();
}
#endif

}  // namespace a2
