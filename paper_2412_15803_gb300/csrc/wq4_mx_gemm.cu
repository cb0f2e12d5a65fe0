// wq4_mx_gemm.cu -- products of microscaled activations with microscaled 4-bit
// weights on the block-scaled tcgen05 tensor cores of sm_103a.
//
// y[m][n] = fp16( sum_g 2^(sx(m,g) + sw(n,g) - 254) * sum_{k in g} x(m,k) w(n,k) ),
// g a group of 32 k; products are exact, sums in fp32.
//
// Weights are the MMA's A operand (128 rows, a lane of tensor memory each),
// tokens its N.  With e4m3 activations: kind::mxf8f6f4, K = 32 an instruction,
// the weights' nibbles spread to 16 bytes for 16 codes by the tensor copy that
// brings them (shared memory holds 128 K in a 128-byte row, of which 64 bytes
// came from memory).  With e2m1 activations: kind::mxf4, K = 64, packed as they
// lie in memory (256 K in a 128-byte row).  Scales come in the order in which
// the tensor cores read them, 512 bytes for 128 rows by 128 K, and go from
// shared memory to tensor memory by tcgen05.cp, in order with the MMAs.
#include "wq4.h"
#include "wq4_device.cuh"
#include "wq4_host.h"
#include "wq4_tc.cuh"

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>

namespace wq4 {
namespace {

// Warps: 0 the copies, 1 the MMA issuer, 2 lets the next kernel launch, 4-7 the
// epilogue (a warp reads the quarter of tensor memory that its number says).
constexpr int kThreads = 256;
constexpr int kProd = 0, kIssuer = 1, kTrigger = 2, kEpi = 4;
constexpr int kHeader = 1024;
constexpr int kTmemCols = 512;

// Tile of 128 weight rows and T tokens.  A slot of the ring is 128 bytes of each
// row's codes: 128 K for activations of 8 bits, 256 K for 4 (the last slot of
// an odd number of 128 K is half filled, its other half zeros that no MMA reads).
template <int BITS, int T>
struct Cfg {
    static constexpr int kBlocks = BITS == 8 ? 1 : 2;            // blocks of 128 K in a slot
    static constexpr int kW = 128 * 128;
    static constexpr int kX = T * 128;
    static constexpr int kScales = 512 * kBlocks;                // of 128 rows
    static constexpr int kSlot = (kW + kX + 2 * kScales + 1023) / 1024 * 1024;
    static constexpr int kSlots = (220 * 1024 - kHeader) / kSlot;
    static constexpr int kSmem = kHeader + kSlots * kSlot;
    static constexpr uint32_t kBytes = (BITS == 8 ? kW / 2 : kW) + kX;   // what the tensor copies bring a slot
    // tensor memory: two accumulators, then each slot's scales: of the weights, of the tokens
    static constexpr int kScaleCols = 8 * kBlocks;
    static constexpr int kScaleCol0 = 2 * T;
    static_assert(kScaleCol0 + kSlots * kScaleCols <= kTmemCols, "tensor memory");
    static_assert(kSmem <= 227 * 1024, "shared memory");
    static_assert((2 * kSlots + 5) * 8 <= 1008, "barriers");
};

struct Args {
    uint16_t* y;
    const uint8_t* w_scales;
    const uint8_t* x_scales;
    int N, M, kblocks;       // blocks of 128 K
    int rtiles, ttiles;
    uint32_t* err;
    int stall;               // test hook: leaves the copies out
    int bulk;                // y's rows can be written by tensor copies
};

template <int S>
struct RingPos {
    int slot = 0;
    uint32_t par = 0;
    __device__ __forceinline__ void next()
    {
        if (++slot == S) {
            slot = 0;
            par ^= 1u;
        }
    }
};

// As in the other kernels: a wait that gives up (bounded, flagged) leaves
// invalid outputs, but every role goes on to its end, without further waits.
template <int BITS, int T>
__global__ void __launch_bounds__(kThreads, 1)
    mx_gemm_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x, const Args a)
{
    using C = Cfg<BITS, T>;
    constexpr int S = C::kSlots, NB = C::kBlocks;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* full = reinterpret_cast<uint64_t*>(smem);
    uint64_t* empty = full + S;
    uint64_t* dfull = empty + S;       // two accumulators
    uint64_t* dempty = dfull + 2;
    uint64_t* drain = dempty + 2;
    uint32_t* tbase_sh = reinterpret_cast<uint32_t*>(smem + 1008);
    uint8_t* ring = smem + kHeader;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int tiles = a.rtiles * a.ttiles;
    const int slots = (a.kblocks + NB - 1) / NB;
    uint32_t* err = a.err;

    if (threadIdx.x == 0) {
        for (int i = 0; i < S; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&dfull[i], 1);
            mbar_init(&dempty[i], 4);
        }
        mbar_init(drain, 1);
        mbar_fence_init();
    }
    if (warp == kIssuer) tc::tmem_alloc(tbase_sh, kTmemCols);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tbase = *tbase_sh;

    if (warp == kTrigger) {
        grid_dependency_wait();
        grid_dependents_launch();
    } else if (warp == kProd) {
        if (lane == 0) {
            tc::prefetch_map(&tm_w);
            tc::prefetch_map(&tm_x);
            grid_dependency_wait();
            const uint64_t pol = l2_policy_evict_first();
            RingPos<S> p;
            int n = 0;
            bool ok = true;
            for (int u = a.stall ? tiles : static_cast<int>(blockIdx.x); u < tiles && ok; u += gridDim.x) {
                const int n0 = u / a.ttiles * 128, m0 = u % a.ttiles * T;
                const uint8_t* ws = a.w_scales + static_cast<size_t>(n0 >> 7) * a.kblocks * 512;
                const uint8_t* xs = a.x_scales + static_cast<size_t>(m0 >> 7) * a.kblocks * 512;
                for (int k = 0; k < slots; ++k, ++n, p.next()) {
                    if (n >= S && (!mbar_wait(&empty[p.slot], p.par ^ 1u, err) || !mbar_wait(&full[p.slot], p.par ^ 1u, err))) {
                        ok = false;
                        break;
                    }
                    uint8_t* base = ring + static_cast<size_t>(p.slot) * C::kSlot;
                    const uint32_t sb = 512u * min(NB, a.kblocks - k * NB);
                    mbar_arrive_expect_tx(&full[p.slot], C::kBytes + 2 * sb);
                    tc::tma_load_2d(base, &tm_w, k * 128, n0, &full[p.slot]);
                    tc::tma_load_2d(base + C::kW, &tm_x, k * 128, m0, &full[p.slot]);
                    bulk_g2s(base + C::kW + C::kX, ws + static_cast<size_t>(k) * NB * 512, sb, &full[p.slot], pol);
                    bulk_g2s(base + C::kW + C::kX + C::kScales, xs + static_cast<size_t>(k) * NB * 512, sb, &full[p.slot], pol);
                }
            }
            // every copy issued has landed before the CTA's memory goes away
            for (int i = max(0, n - S); i < n; ++i) mbar_wait(&full[i % S], (i / S) & 1, err);
        }
    } else if (warp == kIssuer) {
        constexpr uint32_t idesc = BITS == 8 ? tc::idesc_mx_e2m1_e4m3(128, T) : tc::idesc_mx_e2m1_e2m1(128, T);
        const bool leader = tc::elect_one();
        RingPos<S> p;
        int dit = 0;
        bool ok = true;
        const uint64_t wdesc = tc::sw128_kmajor_desc(smem_addr(ring));
        const uint64_t xdesc = tc::sw128_kmajor_desc(smem_addr(ring + C::kW));
        const uint64_t sdesc = tc::scales_desc(smem_addr(ring + C::kW + C::kX));
        for (int u = blockIdx.x; u < tiles; u += gridDim.x, ++dit) {
            const int buf = dit & 1;
            if (dit >= 2 && ok) ok = mbar_wait(&dempty[buf], ((dit >> 1) - 1) & 1, err);
            tc::fence_after_sync();
            // a tile of 64 tokens may begin at the second half of a block of 128
            const uint32_t shift = (u % a.ttiles * T & 127) >> 5;
            for (int k = 0; k < slots; ++k, p.next()) {
                if (ok) ok = mbar_wait(&full[p.slot], p.par, err);
                tc::fence_after_sync();
                const uint64_t off = static_cast<uint64_t>(p.slot) * (C::kSlot >> 4);
                const uint32_t scol = tbase + C::kScaleCol0 + p.slot * C::kScaleCols;
                const int nb = min(NB, a.kblocks - k * NB);
                if (leader) {
                    for (int b = 0; b < nb; ++b) {
                        tc::cp_scales(scol + 4 * b, sdesc + off + b * 32);
                        tc::cp_scales(scol + 4 * (NB + b), sdesc + off + (C::kScales >> 4) + b * 32);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int b = BITS == 8 ? 0 : j >> 1;
                        if (b >= nb) break;
                        const uint32_t acc = k > 0 || j > 0 ? 1u : 0u;
                        const uint32_t id = idesc | tc::idesc_mx_scale_byte(BITS == 8 ? j : 2 * (j & 1));
                        if constexpr (BITS == 8)
                            tc::mma_mxf8f6f4(tbase + buf * T, wdesc + off + 2 * j, xdesc + off + 2 * j, id, scol, scol + 4 + shift, acc);
                        else
                            tc::mma_mxf4(tbase + buf * T, wdesc + off + 2 * j, xdesc + off + 2 * j, id, scol + 4 * b,
                                         scol + 4 * (NB + b) + shift, acc);
                    }
                    tc::commit(&empty[p.slot]);
                }
                __syncwarp();
            }
            if (leader) tc::commit(&dfull[buf]);
        }
        // all MMAs issued have completed before tensor memory is released
        if (leader) tc::commit(drain);
        mbar_wait(drain, 0, err);
    } else if (warp >= kEpi) {
        grid_dependency_wait();          // y is written after the previous kernel
        const int quad = warp & 3;
        const uint32_t lane_base = tbase + (static_cast<uint32_t>(32 * quad) << 16);
        int dit = 0;
        bool ok = true;
        for (int u = blockIdx.x; u < tiles; u += gridDim.x, ++dit) {
            const int buf = dit & 1;
            const int nn = u / a.ttiles * 128 + 32 * quad + lane, m0 = u % a.ttiles * T;
            if (ok) ok = mbar_wait(&dfull[buf], (dit >> 1) & 1, err);
            __syncwarp();
            tc::fence_after_sync();
            for (int t = 0; t < T; t += 16) {
                uint32_t d[16];
                tc::ld16(lane_base + buf * T + t, d);
                tc::ld_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (nn < a.N && m0 + t + i < a.M)
                        a.y[static_cast<size_t>(m0 + t + i) * a.N + nn] = float_to_half_bits(__uint_as_float(d[i]));
            }
            tc::fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&dempty[buf]);
        }
    }

    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    if (warp == kIssuer) tc::tmem_dealloc(tbase, kTmemCols);
}

template <int BITS, int T>
int launch(const DeviceInfo* di, const CUtensorMap* tm, const Args& a, cudaStream_t stream)
{
    static std::atomic<bool> ready[kMaxDevices];      // per device; setting the attribute twice is harmless
    if (!ready[di->dev].load()) {
        if (cudaFuncSetAttribute(mx_gemm_kernel<BITS, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<BITS, T>::kSmem) !=
            cudaSuccess)
            return WQ4_ERR_CUDA;
        ready[di->dev].store(true);
    }
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(std::min(a.rtiles * a.ttiles, di->sm_count));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Cfg<BITS, T>::kSmem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, mx_gemm_kernel<BITS, T>, tm[0], tm[1], a) == cudaSuccess ? WQ4_OK : WQ4_ERR_CUDA;
}

// ------------------------------------------------------- pairs of CTAs --

// Tile of 256 weight rows and 256 tokens for the two CTAs of a cluster: each
// brings its 128 rows, half of the tokens and the scales of its rows and of all
// the tokens, 34 KB a slot where two CTAs of their own would take 50.
// Tensor memory holds two accumulators that share kOver columns, and the scales
// of each slot: the epilogue takes the shared columns first, and the other
// accumulator's MMAs begin when it has them.
template <int BITS>
struct PairCfg {
    static constexpr int T = 256;
    static constexpr int kBlocks = BITS == 8 ? 1 : 2;
    static constexpr int kW = 128 * 128;
    static constexpr int kX = 128 * 128;
    static constexpr int kScales = 512 * kBlocks;                     // of 128 rows
    static constexpr int kSlot = (kW + kX + 3 * kScales + 1023) / 1024 * 1024;
    static constexpr int kSlots = 5;
    static constexpr int kStage = 32 * 128 * 2;                       // 32 tokens x 128 outputs
    static constexpr int kStage0 = kHeader;
    static constexpr int kRing = kStage0 + 4 * kStage;
    static constexpr int kSmem = kRing + kSlots * kSlot;
    static constexpr uint32_t kBytes = (BITS == 8 ? kW / 2 : kW) + kX + 3 * kScales;   // of one CTA and slot
    static constexpr int kScaleCols = 12 * kBlocks;
    static constexpr int kScaleSpace = 64 * kBlocks;
    static constexpr int kScaleCol0 = kTmemCols - kScaleSpace;
    static constexpr int kD1 = kScaleCol0 - T;                        // the second accumulator's first column
    static constexpr int kOver = T - kD1;                             // shared columns
    static_assert(kSlots * kScaleCols <= kScaleSpace && kOver % 64 == 0, "tensor memory");
    static_assert(kSmem <= 227 * 1024, "shared memory");
};

constexpr int kPairThreads = 384;      // warps 4-11: two groups of four epilogue warps

struct PairMaps {
    CUtensorMap w, x, ws, xs, y;
};

template <int BITS>
__global__ void __launch_bounds__(kPairThreads, 1) mx_gemm_pair_kernel(const __grid_constant__ PairMaps tm, const Args a)
{
    using C = PairCfg<BITS>;
    constexpr int S = C::kSlots, NB = C::kBlocks, T = C::T;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* full = reinterpret_cast<uint64_t*>(smem);     // the first CTA's count, for both
    uint64_t* empty = full + S;
    uint64_t* dfull = empty + S;
    uint64_t* dempty = dfull + 1;      // the first CTA's counts, for both: the shared columns are read
    uint64_t* drain = dempty + 1;
    uint32_t* tbase_sh = reinterpret_cast<uint32_t*>(smem + 1008);
    uint8_t* ring = smem + C::kRing;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = static_cast<int>(blockIdx.x) & 1;
    const int tiles = a.rtiles * a.ttiles, u0 = static_cast<int>(blockIdx.x) >> 1, ustep = static_cast<int>(gridDim.x) >> 1;
    const int slots = (a.kblocks + NB - 1) / NB;
    uint32_t* err = a.err;

    if (threadIdx.x == 0) {
        for (int i = 0; i < S; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        mbar_init(dfull, 1);
        mbar_init(dempty, 16);
        mbar_init(drain, 1);
        mbar_fence_init();
    }
    if (warp == kIssuer) tc::tmem_alloc_pair(tbase_sh, kTmemCols);
    tc::fence_before_sync();
    __syncthreads();
    tc::cluster_sync_all();
    tc::fence_after_sync();
    const uint32_t tbase = *tbase_sh;

    if (warp == kTrigger) {
        grid_dependency_wait();
        grid_dependents_launch();
    } else if (warp == kProd) {
        if (lane == 0) {
            tc::prefetch_map(&tm.w);
            tc::prefetch_map(&tm.x);
            tc::prefetch_map(&tm.ws);
            tc::prefetch_map(&tm.xs);
            grid_dependency_wait();
            RingPos<S> p;
            int n = 0;
            bool ok = true;
            for (int u = a.stall ? tiles : u0; u < tiles && ok; u += ustep) {
                const int n0 = u / a.ttiles * 256 + 128 * rank, m0 = u % a.ttiles * T;
                for (int k = 0; k < slots; ++k, ++n, p.next()) {
                    if (n >= S && !mbar_wait(&empty[p.slot], p.par ^ 1u, err)) {
                        ok = false;
                        break;
                    }
                    uint8_t* base = ring + static_cast<size_t>(p.slot) * C::kSlot;
                    const uint32_t bar = tc::cluster_addr(&full[p.slot], 0);
                    if (rank == 0) mbar_arrive_expect_tx(&full[p.slot], 2 * C::kBytes);
                    tc::tma_load_2d_pair(base, &tm.w, k * 128, n0, bar);
                    tc::tma_load_2d_pair(base + C::kW, &tm.x, k * 128, m0 + 128 * rank, bar);
                    tc::tma_load_2d_pair(base + C::kW + C::kX, &tm.ws, k * NB * 128, n0 >> 7, bar);
                    tc::tma_load_2d_pair(base + C::kW + C::kX + C::kScales, &tm.xs, k * NB * 128, m0 >> 7, bar);
                }
            }
            // every copy issued, the other CTA's too, has landed before the memory goes away
            if (rank == 0)
                for (int i = max(0, n - S); i < n; ++i) mbar_wait(&full[i % S], (i / S) & 1, err);
        }
    } else if (warp == kIssuer) {
        if (rank == 0) {
            constexpr uint32_t idesc = BITS == 8 ? tc::idesc_mx_e2m1_e4m3(256, T) : tc::idesc_mx_e2m1_e2m1(256, T);
            const bool leader = tc::elect_one();
            RingPos<S> p;
            int dit = 0;
            bool ok = true;
            const uint64_t wdesc = tc::sw128_kmajor_desc(smem_addr(ring));
            const uint64_t xdesc = tc::sw128_kmajor_desc(smem_addr(ring + C::kW));
            const uint64_t sdesc = tc::scales_desc(smem_addr(ring + C::kW + C::kX));
            for (int u = u0; u < tiles; u += ustep, ++dit) {
                const uint32_t dcol = tbase + (dit & 1) * C::kD1;
                // the last tile's shared columns are read, and so all of the one before it
                if (dit >= 1 && ok) ok = mbar_wait(dempty, (dit - 1) & 1, err);
                tc::fence_after_sync();
                for (int k = 0; k < slots; ++k, p.next()) {
                    if (ok) ok = mbar_wait(&full[p.slot], p.par, err);
                    tc::fence_after_sync();
                    const uint64_t off = static_cast<uint64_t>(p.slot) * (C::kSlot >> 4);
                    const uint32_t scol = tbase + C::kScaleCol0 + p.slot * C::kScaleCols;
                    const int nb = min(NB, a.kblocks - k * NB);
                    if (leader) {
                        // in tensor memory: the rows' scales of each 128 K, then the tokens' (two blocks of 128) of each
                        for (int b = 0; b < nb; ++b) {
                            tc::cp_scales_pair(scol + 4 * b, sdesc + off + b * 32);
                            tc::cp_scales_pair(scol + 4 * NB + 8 * b, sdesc + off + (C::kScales >> 4) + b * 32);
                            tc::cp_scales_pair(scol + 4 * NB + 8 * b + 4, sdesc + off + 2 * (C::kScales >> 4) + b * 32);
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int b = BITS == 8 ? 0 : j >> 1;
                            if (b >= nb) break;
                            const uint32_t acc = k > 0 || j > 0 ? 1u : 0u;
                            const uint32_t id = idesc | tc::idesc_mx_scale_byte(BITS == 8 ? j : 2 * (j & 1));
                            if constexpr (BITS == 8)
                                tc::mma_mxf8f6f4_pair(dcol, wdesc + off + 2 * j, xdesc + off + 2 * j, id, scol, scol + 4, acc);
                            else
                                tc::mma_mxf4_pair(dcol, wdesc + off + 2 * j, xdesc + off + 2 * j, id, scol + 4 * b,
                                                  scol + 4 * NB + 8 * b, acc);
                        }
                        tc::commit_pair(&empty[p.slot]);
                    }
                    __syncwarp();
                }
                if (leader) tc::commit_pair(dfull);
                __syncwarp();
            }
            // all MMAs issued have completed before tensor memory is released
            if (leader) tc::commit_pair(drain);
            mbar_wait(drain, 0, err);
        }
    } else if (warp >= kEpi) {
        grid_dependency_wait();          // y is written after the previous kernel
        const int quad = warp & 3, grp = (warp - kEpi) >> 2;
        const int row = 32 * quad + lane;
        uint16_t* const stage = reinterpret_cast<uint16_t*>(smem + C::kStage0 + 2 * grp * C::kStage);
        const uint32_t lane_base = tbase + (static_cast<uint32_t>(32 * quad) << 16);
        const uint32_t dempty0 = tc::cluster_addr(dempty, 0);
        constexpr int kOverBlocks = C::kOver / 32;
        int dit = 0, nst = 0;
        bool ok = true;
        for (int u = u0; u < tiles; u += ustep, ++dit) {
            const int n0 = u / a.ttiles * 256 + 128 * rank, m0 = u % a.ttiles * T;
            const uint32_t dcol = lane_base + (dit & 1) * C::kD1;
            if (ok) ok = mbar_wait(dfull, dit & 1, err);
            __syncwarp();
            tc::fence_after_sync();
#pragma unroll 1
            for (int i = 0; i < 4; ++i) {
                // blocks of 32 tokens, the shared columns' first, to the two groups in turn
                const int blk = (((dit & 1) ? 0 : 8 - kOverBlocks) + 2 * i + grp) & 7;
                uint32_t d[32];
                tc::ld32(dcol + 32 * blk, d);
                tc::ld_wait();
                if (i == kOverBlocks / 2 - 1) {
                    tc::fence_before_sync();
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive_cluster(dempty0);
                }
                const int mb = m0 + 32 * blk;
                if (a.bulk) {
                    uint16_t* st = stage + (nst & 1) * (C::kStage / 2);
                    ++nst;
                    if (warp % 4 == 0 && lane == 0) tc::bulk_wait_read<1>();      // the copy that read this block is over
                    named_barrier_sync(1 + grp, 128);
#pragma unroll
                    for (int t = 0; t < 32; ++t) st[t * 128 + row] = float_to_half_bits(__uint_as_float(d[t]));
                    tc::fence_async_smem();
                    named_barrier_sync(1 + grp, 128);
                    if (warp % 4 == 0 && lane == 0) {
                        if (mb < a.M && n0 < a.N) tc::tma_store_2d(&tm.y, n0, mb, st);
                        tc::bulk_commit();
                    }
                } else {
#pragma unroll
                    for (int t = 0; t < 32; ++t)
                        if (n0 + row < a.N && mb + t < a.M)
                            a.y[static_cast<size_t>(mb + t) * a.N + n0 + row] = float_to_half_bits(__uint_as_float(d[t]));
                }
            }
        }
        if (warp % 4 == 0 && lane == 0) tc::bulk_wait<0>();
    }

    tc::fence_before_sync();
    __syncthreads();
    tc::cluster_sync_all();
    tc::fence_after_sync();
    if (warp == kIssuer) tc::tmem_dealloc_pair(tbase, kTmemCols);
}

template <int BITS>
int launch_pair(const DeviceInfo* di, const PairMaps& tm, const Args& a, cudaStream_t stream)
{
    static std::atomic<bool> ready[kMaxDevices];
    if (!ready[di->dev].load()) {
        if (cudaFuncSetAttribute(mx_gemm_pair_kernel<BITS>, cudaFuncAttributeMaxDynamicSharedMemorySize, PairCfg<BITS>::kSmem) !=
            cudaSuccess)
            return WQ4_ERR_CUDA;
        ready[di->dev].store(true);
    }
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * std::min(a.rtiles * a.ttiles, di->sm_count / 2));
    cfg.blockDim = dim3(kPairThreads);
    cfg.dynamicSmemBytes = PairCfg<BITS>::kSmem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, mx_gemm_pair_kernel<BITS>, tm, a) == cudaSuccess ? WQ4_OK : WQ4_ERR_CUDA;
}

}  // namespace
}  // namespace wq4

using namespace wq4;

extern "C" int wq4_mx_gemm(const uint8_t* W, const uint8_t* W_scales, const uint8_t* x, const uint8_t* x_scales, uint16_t* y,
                           int N, int K, int M, int bits, void* stream)
{
    if (!W || !W_scales || !x || !x_scales || !y) return WQ4_ERR_INVALID;
    if (N < 1 || M < 1 || K < 128 || (K % 128) != 0 || (bits != 8 && bits != 4)) return WQ4_ERR_INVALID;
    constexpr int64_t kMost = static_cast<int64_t>(1) << 41;
    if (static_cast<int64_t>(N) * K > kMost || static_cast<int64_t>(M) * K > kMost) return WQ4_ERR_INVALID;
    if (!aligned(W, 32) || !aligned(x, 32) || !aligned(W_scales, 16) || !aligned(x_scales, 16) || !aligned(y, 2)) return WQ4_ERR_ALIGN;
    const size_t yb = static_cast<size_t>(M) * N * 2, wb = static_cast<size_t>(N) * K / 2, xb = static_cast<size_t>(M) * K / 8 * bits;
    if (overlaps(y, yb, W, wb) || overlaps(y, yb, W_scales, wq4_mx_scale_bytes(N, K)) || overlaps(y, yb, x, xb) ||
        overlaps(y, yb, x_scales, wq4_mx_scale_bytes(M, K)))
        return WQ4_ERR_INVALID;
    const DeviceInfo* di = current_device_info(nullptr);
    if (!di) return WQ4_ERR_CUDA;
    const bool pair = M > 128 && static_cast<int64_t>((N - 1) / 256 + 1) * ((M - 1) / 256 + 1) >= di->sm_count / 2;
    const int T = pair ? 256 : M <= 16 ? 16 : M <= 64 ? 64 : 128, rows = pair ? 256 : 128;
    Args a;
    a.y = y;
    a.w_scales = W_scales;
    a.x_scales = x_scales;
    a.N = N;
    a.M = M;
    a.kblocks = K / 128;
    a.rtiles = (N - 1) / rows + 1;
    a.ttiles = (M - 1) / T + 1;
    a.err = di->status;
    a.stall = test_copy_stall() == WQ4_STALL_MX ? 1 : 0;
    a.bulk = (N % 8) == 0 && aligned(y, 16) ? 1 : 0;
    if (static_cast<int64_t>(a.rtiles) * a.ttiles > (static_cast<int64_t>(1) << 30)) return WQ4_ERR_INVALID;
    PairMaps tm;
    const uint64_t k = static_cast<uint64_t>(K), wrow = k / 2, xrow = k / 8 * bits, srow = k / 128 * 512;
    constexpr CUtensorMapDataType kBytes = CU_TENSOR_MAP_DATA_TYPE_UINT8, kWords = CU_TENSOR_MAP_DATA_TYPE_UINT32;
    constexpr CUtensorMapSwizzle kSwz = CU_TENSOR_MAP_SWIZZLE_128B, kPlain = CU_TENSOR_MAP_SWIZZLE_NONE;
    // activations of 8 bits: the weights' codes are spread on their way into shared memory
    const bool w_ok = bits == 8 ? encode_tensor_map_2d(&tm.w, CU_TENSOR_MAP_DATA_TYPE_16U4_ALIGN16B, W, k, N, wrow, 128, 128, kSwz)
                                : encode_tensor_map_2d(&tm.w, kBytes, W, wrow, N, wrow, 128, 128, kSwz);
    if (!w_ok || !encode_tensor_map_2d(&tm.x, kBytes, x, xrow, M, xrow, 128, T < 128 ? T : 128, kSwz)) return WQ4_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (pair) {
        const uint32_t sbox = bits == 8 ? 128 : 256;          // words: of one or two blocks of 128 K
        if (!encode_tensor_map_2d(&tm.ws, kWords, W_scales, srow / 4, (N - 1) / 128 + 1, srow, sbox, 1, kPlain) ||
            !encode_tensor_map_2d(&tm.xs, kWords, x_scales, srow / 4, (M - 1) / 128 + 1, srow, sbox, 2, kPlain))
            return WQ4_ERR_CUDA;
        if (!a.bulk)
            tm.y = tm.x;        // not used
        else if (!encode_tensor_map_2d(&tm.y, CU_TENSOR_MAP_DATA_TYPE_UINT16, y, N, M, static_cast<uint64_t>(N) * 2, 128, 32, kPlain))
            return WQ4_ERR_CUDA;
        return bits == 8 ? launch_pair<8>(di, tm, a, st) : launch_pair<4>(di, tm, a, st);
    }
    const CUtensorMap tms[2] = {tm.w, tm.x};
    if (bits == 8) return T == 16 ? launch<8, 16>(di, tms, a, st) : T == 64 ? launch<8, 64>(di, tms, a, st) : launch<8, 128>(di, tms, a, st);
    return T == 16 ? launch<4, 16>(di, tms, a, st) : T == 64 ? launch<4, 64>(di, tms, a, st) : launch<4, 128>(di, tms, a, st);
}
