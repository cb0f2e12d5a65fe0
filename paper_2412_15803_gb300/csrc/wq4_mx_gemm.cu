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
    const int T = M <= 16 ? 16 : M <= 64 ? 64 : 128;
    Args a;
    a.y = y;
    a.w_scales = W_scales;
    a.x_scales = x_scales;
    a.N = N;
    a.M = M;
    a.kblocks = K / 128;
    a.rtiles = (N - 1) / 128 + 1;
    a.ttiles = (M - 1) / T + 1;
    a.err = di->status;
    a.stall = test_copy_stall() == WQ4_STALL_MX ? 1 : 0;
    if (static_cast<int64_t>(a.rtiles) * a.ttiles > (static_cast<int64_t>(1) << 30)) return WQ4_ERR_INVALID;
    CUtensorMap tm[2];
    const uint64_t k = static_cast<uint64_t>(K), wrow = k / 2, xrow = k / 8 * bits;
    // activations of 8 bits: the weights' codes are spread on their way into shared memory
    const bool w_ok = bits == 8 ? encode_tensor_map_2d(&tm[0], CU_TENSOR_MAP_DATA_TYPE_16U4_ALIGN16B, W, k, N, wrow, 128, 128,
                                                       CU_TENSOR_MAP_SWIZZLE_128B)
                                : encode_tensor_map_2d(&tm[0], CU_TENSOR_MAP_DATA_TYPE_UINT8, W, wrow, N, wrow, 128, 128,
                                                       CU_TENSOR_MAP_SWIZZLE_128B);
    if (!w_ok || !encode_tensor_map_2d(&tm[1], CU_TENSOR_MAP_DATA_TYPE_UINT8, x, xrow, M, xrow, 128, T, CU_TENSOR_MAP_SWIZZLE_128B))
        return WQ4_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (bits == 8) return T == 16 ? launch<8, 16>(di, tm, a, st) : T == 64 ? launch<8, 64>(di, tm, a, st) : launch<8, 128>(di, tm, a, st);
    return T == 16 ? launch<4, 16>(di, tm, a, st) : T == 64 ? launch<4, 64>(di, tm, a, st) : launch<4, 128>(di, tm, a, st);
}
