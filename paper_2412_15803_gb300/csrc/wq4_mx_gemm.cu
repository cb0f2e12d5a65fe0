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
//
// What bounds it, by the number of tokens:
// - one to some: a slot's fixed cost, not its bytes.  A copy costs the thread that
//   issues it ~100 cycles, a wait that is over ~110, the issuer's 128 K ~480 (wait,
//   fence, 2 copies of scales, 4 MMAs, commit), a launch that follows another ~2.5 us
//   from the previous kernel's end to the first MMA, sums over a cluster 1 us.  So few
//   rows are shared by many CTAs (K split over a cluster, two CTAs an SM) and four
//   warps issue copies.  6144 x 4096 over one token 5.8 us (floor 2.0 at the copy
//   rate), 4096 x 14336 over 16 tokens 9.1 (4.7), 128256 x 4096 over one token in 4
//   bits 43.5 (41).
// - a prompt: the power limit.  28672 x 4096 over 2048 tokens in 8 bits 146-153 us
//   (3.2 PFLOP/s) with the SMs at 1.66 GHz, 117 at 2.07 GHz when all codes are zero;
//   over 8192 in 4 bits 281-287 (6.8 PFLOP/s; zeros 246).
// Tried and slower: a warp of its own for the copies of scales to tensor memory
// (6.25 -> 6.7 us), one lane's waits with a shuffle (7.35), test_wait for try_wait (6.6).
#include "wq4.h"
#include "wq4_device.cuh"
#include "wq4_host.h"
#include "wq4_mx.cuh"
#include "wq4_tc.cuh"

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>

namespace wq4 {
namespace {

// Warps: 0, 2, 3 and 12 the copies (in pairs of CTAs 0; 2 lets the next kernel
// launch), 1 the MMA issuer, 4-11 the epilogue (a warp reads the quarter of tensor
// memory that its number says).
constexpr int kThreads = 416, kPairThreads = 384;
constexpr int kProd = 0, kIssuer = 1, kTrigger = 2, kScalesW = 2, kTokens = 3, kEpi = 4, kScalesX = 12;
constexpr int kHeader = 1024;
constexpr int kTmemCols = 512;

struct Args {
    uint16_t* y;
    const uint8_t* w_scales;
    const uint8_t* x_scales;
    int N, M, kblocks;       // blocks of 128 K
    int rtiles, ttiles;
    int tok;                 // tokens of a tile, a multiple of 16
    int split;               // CTAs of a cluster that share a tile's K
    int nslots, slot_bytes, ring;      // of the ring of copies, and where it begins
    int tmem_cols;
    uint32_t* err;
    int stall;               // test hook: leaves the copies out
    int bulk;                // y's rows can be written by tensor copies
    int prefetch;            // fetch weights into L2 early
};

// A ring position: slot and parity of the n-th use of a ring of S slots.
struct RingPos {
    int slot = 0;
    uint32_t par = 0;
    __device__ __forceinline__ void next(int S)
    {
        if (++slot == S) {
            slot = 0;
            par ^= 1u;
        }
    }
};

// Tile of 128 weight rows and `tok` tokens, up to 128.  A slot of the ring is BOXES
// boxes of 128 bytes of each row's codes: 128 or 256 K with activations of 8 bits,
// 256 with 4 (one box).  (Where K is an odd number of 128, the second half of the
// last slot's 256 is zeros that no MMA reads.)
template <int BITS, int BOXES>
struct Cfg {
    static constexpr int kBlocks = BITS == 8 ? BOXES : 2;        // blocks of 128 K in a slot
    static constexpr int kW = BOXES * 128 * 128;
    static constexpr int kScales = 512 * kBlocks;                // of 128 rows
    static constexpr int kMaxSlots = 12;
    static constexpr int kScaleCols = 8 * kBlocks;               // of a slot, in tensor memory: of the weights, of the tokens
    static_assert(2 * 128 + kMaxSlots * kScaleCols <= kTmemCols, "tensor memory");
    static_assert((2 * kMaxSlots + 6) * 8 <= 1008, "barriers");
};

// Shared memory of a CTA: half of an SM's, so that two are resident, of one call or
// of two that follow one another, or all of it.
constexpr int kHalf = 113 * 1024, kWhole = 227 * 1024;

// A persistent grid, or a cluster of `split` CTAs a tile that take consecutive
// parts of its K: each sends its fp32 sums to the CTAs that add them, in rank
// order, consecutive groups of four tokens a CTA.  A CTA leaves when the others'
// sums are in; nothing is sent to it after that.
//
// As in the other kernels: a wait that gives up (bounded, flagged) leaves
// invalid outputs, but every role goes on to its end, without further waits.
template <int BITS, int BOXES>
__global__ void __launch_bounds__(kThreads, 2)
    mx_gemm_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x, const Args a)
{
    using C = Cfg<BITS, BOXES>;
    constexpr int NB = C::kBlocks;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* full = reinterpret_cast<uint64_t*>(smem);
    uint64_t* empty = full + C::kMaxSlots;
    uint64_t* dfull = empty + C::kMaxSlots;       // two accumulators
    uint64_t* dempty = dfull + 2;
    uint64_t* drain = dempty + 2;
    uint64_t* sfull = drain + 1;                  // the cluster's sums for this CTA are in
    uint32_t* tbase_sh = reinterpret_cast<uint32_t*>(smem + 1008);
    float4* sums = reinterpret_cast<float4*>(smem + kHeader);       // [rank][group][row]
    uint8_t* ring = smem + a.ring;
    const int S = a.nslots, tok = a.tok;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int split = a.split, rank = static_cast<int>(blockIdx.x) % split;
    const int tiles = a.rtiles * a.ttiles, u0 = static_cast<int>(blockIdx.x) / split, ustep = static_cast<int>(gridDim.x) / split;
    // this CTA's slots of a tile's K
    const int slots = (a.kblocks + NB - 1) / NB;
    const int k0 = static_cast<int>(static_cast<int64_t>(rank) * slots / split), k1 = static_cast<int>(static_cast<int64_t>(rank + 1) * slots / split);
    uint32_t* err = a.err;

    if (threadIdx.x == 0) {
        for (int i = 0; i < S; ++i) {
            mbar_init(&full[i], 4);       // weights, tokens, the scales of each
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&dfull[i], 1);
            mbar_init(&dempty[i], 8);
        }
        mbar_init(drain, 1);
        mbar_init(sfull, 1);
        mbar_fence_init();
        if (split > 1) {
            // what the cluster's CTAs send here
            const int groups = (min(tok, a.M - u0 % a.ttiles * tok) + 3) / 4, per = (groups + split - 1) / split;
            mbar_arrive_expect_tx(sfull, static_cast<uint32_t>(split * max(0, min(per, groups - rank * per)) * 128 * 16));
        }
    }
    if (warp == kIssuer) tc::tmem_alloc(tbase_sh, a.tmem_cols);
    tc::fence_before_sync();
    __syncthreads();
    if (split > 1) tc::cluster_arrive();          // waited for before the first sums are sent
    tc::fence_after_sync();
    const uint32_t tbase = *tbase_sh, scol0 = tbase + 2 * tok;

    if (warp == kProd || warp == kScalesW || warp == kTokens || warp == kScalesX) {
        // Four warps bring a slot's parts, a lane each.  (6144 x 4096, one token, K in
        // halves, weights copied early: one warp 6.0 us, two 5.7, four 5.45.)
        if (lane == 0) {
            const bool w = warp == kProd || warp == kScalesW, codes = warp == kProd || warp == kTokens;
            tc::prefetch_map(w ? &tm_w : &tm_x);
            const uint64_t pol = l2_policy_evict_first();
            const uint8_t* const sc = w ? a.w_scales : a.x_scales;
            uint8_t* const to = ring + (w ? 0 : C::kW);
            uint8_t* const sc_to = ring + C::kW + BOXES * tok * 128 + (w ? 0 : C::kScales);
            const uint32_t bytes = w ? 128 * 128 * BOXES * (BITS == 8 ? 4 : 8) / 8 : BOXES * tok * 128;   // what the tensor copy brings
            // rows r0 of codes and scales
            auto copy = [&](int slot, int k, int r0) {
                const uint32_t sb = 512u * min(NB, a.kblocks - k * NB);
                uint64_t* bar = &full[slot];
                mbar_arrive_expect_tx(bar, codes ? bytes : sb);
                if (!codes) {
                    bulk_g2s(sc_to + slot * a.slot_bytes, sc + (static_cast<size_t>(r0 >> 7) * a.kblocks + k * NB) * 512, sb, bar, pol);
                } else if constexpr (BITS == 8)
                    tc::tma_load_3d(to + slot * a.slot_bytes, w ? &tm_w : &tm_x, 0, r0, k * BOXES, bar);
                else
                    tc::tma_load_2d(to + slot * a.slot_bytes, w ? &tm_w : &tm_x, k * 128, r0, bar);
            };
            // The previous kernel may write the weights: a small matrix's are fetched into L2
            // while it finishes and copied after it.
            if (w && a.prefetch && u0 < tiles) {
                const int r0 = u0 / a.ttiles * 128, ke = min(k1, k0 + 32);
                if (!codes)
                    bulk_prefetch(sc + (static_cast<size_t>(r0 >> 7) * a.kblocks + k0 * NB) * 512, 512u * (min(ke * NB, a.kblocks) - k0 * NB));
                else
                    for (int k = k0; k < ke; ++k) {
                        if constexpr (BITS == 8)
                            tc::tma_prefetch_3d(&tm_w, 0, r0, k * BOXES);
                        else
                            tc::tma_prefetch_2d(&tm_w, k * 128, r0);
                    }
            }
            grid_dependency_wait();
            if (warp == kTokens) grid_dependents_launch();
            RingPos p;
            int n = 0;
            bool ok = true;
            for (int u = a.stall ? tiles : u0; u < tiles && ok; u += ustep) {
                const int r0 = w ? u / a.ttiles * 128 : u % a.ttiles * tok;
                for (int k = k0; k < k1; ++k, ++n, p.next(S)) {
                    if (n >= S && !mbar_wait(&empty[p.slot], p.par ^ 1u, err)) {
                        ok = false;
                        break;
                    }
                    copy(p.slot, k, r0);
                }
            }
            // every copy issued has landed before the CTA's memory goes away
            for (int i = max(0, n - S); i < n; ++i) mbar_wait(&full[i % S], (i / S) & 1, err);
        }
    } else if (warp == kIssuer) {
        grid_dependency_wait();          // its waits are bounded, the previous kernel's time is not
        const uint32_t idesc = BITS == 8 ? tc::idesc_mx_e2m1_e4m3(128, tok) : tc::idesc_mx_e2m1_e2m1(128, tok);
        const uint32_t leader = tc::elect_one() ? 1u : 0u;
        RingPos p;
        int dit = 0;
        bool ok = true;
        const uint64_t sdesc = tc::scales_desc(smem_addr(ring + C::kW + BOXES * tok * 128));
        const uint64_t wdesc = tc::sw128_kmajor_desc(smem_addr(ring));
        const uint64_t xdesc = tc::sw128_kmajor_desc(smem_addr(ring + C::kW));
        for (int u = u0; u < tiles; u += ustep, ++dit) {
            const int buf = dit & 1;
            const uint32_t dcol = tbase + buf * tok;
            if (dit >= 2 && ok) ok = mbar_wait(&dempty[buf], ((dit >> 1) - 1) & 1, err);
            for (int k = k0; k < k1; ++k) {
                if (ok) ok = mbar_wait(&full[p.slot], p.par, err);
                tc::fence_after_sync();
                const int slot = p.slot, nb = min(NB, a.kblocks - k * NB);
                p.next(S);
                const uint64_t off = static_cast<uint64_t>(slot * a.slot_bytes >> 4);
                const uint32_t scol = scol0 + slot * C::kScaleCols;
                // predicated, not in a branch of one lane: the operands stay warp-uniform
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    if (b > 0 && b >= nb) break;
                    const uint32_t sfw = scol + 4 * b, sfx = scol + 4 * (NB + b);
                    tc::cp_scales(sfw, sdesc + off + b * 32, leader);
                    tc::cp_scales(sfx, sdesc + off + (C::kScales >> 4) + b * 32, leader);
                    if constexpr (BITS == 8) {
                        const uint64_t wd = wdesc + off + b * (128 * 128 >> 4), xd = xdesc + off + static_cast<uint32_t>(b * tok * 8);
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            tc::mma_mxf8f6f4(dcol, wd + 2 * j, xd + 2 * j, idesc | tc::idesc_mx_scale_byte(j), sfw, sfx,
                                             k > k0 || b + j > 0 ? 1u : 0u, leader);
                    } else {
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            tc::mma_mxf4(dcol, wdesc + off + 4 * b + 2 * j, xdesc + off + 4 * b + 2 * j,
                                         idesc | tc::idesc_mx_scale_byte(2 * j), sfw, sfx, k > k0 || b + j > 0 ? 1u : 0u, leader);
                    }
                }
                tc::commit_if(&empty[slot], leader);
                if (k == k1 - 1) tc::commit_if(&dfull[buf], leader);
                __syncwarp();
            }
        }
        // all MMAs issued have completed before tensor memory is released
        if (leader) tc::commit(drain);
        mbar_wait(drain, 0, err);
    } else {
        // two groups of four warps, blocks of 16 tokens in turn
        grid_dependency_wait();          // y is written after the previous kernel
        const int quad = warp & 3, row = 32 * quad + lane, grp = (warp - kEpi) >> 2;
        const uint32_t lane_base = tbase + (static_cast<uint32_t>(32 * quad) << 16);
        int dit = 0;
        bool ok = true;
        for (int u = u0; u < tiles; u += ustep, ++dit) {
            const int buf = dit & 1;
            const int nn = u / a.ttiles * 128 + row, m0 = u % a.ttiles * tok, tv = min(tok, a.M - m0);
            uint16_t* out = a.y + static_cast<size_t>(m0) * a.N + nn;
            const uint32_t dcol = lane_base + buf * tok;
            const int per = ((tv + 3) / 4 + split - 1) / split;       // groups of four tokens that a CTA adds
            if (ok) ok = mbar_wait(&dfull[buf], (dit >> 1) & 1, err);
            if (split > 1) tc::cluster_wait();
            __syncwarp();
            tc::fence_after_sync();
            for (int t = 16 * grp; t < tv; t += 32) {
                uint32_t d[16];
                tc::ld16(dcol + t, d);
                tc::ld_wait();
                if (split > 1) {
                    int to = (t / 4) / per, j = (t / 4) % per;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (t + 4 * i < tv)
                            tc::st_async(tc::cluster_addr(sums + (rank * per + j) * 128 + row, to), d + 4 * i, tc::cluster_addr(sfull, to));
                        if (++j == per) j = 0, ++to;
                    }
                } else if (nn < a.N) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (t + i < tv) out[static_cast<size_t>(t + i) * a.N] = float_to_half_bits(__uint_as_float(d[i]));
                }
            }
            tc::fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&dempty[buf]);
            if (split == 1) continue;
            // a CTA that gives up stays until the others have, too, and sent what they send
            if (!ok || !mbar_wait_cluster(sfull, 0, err))
                for (const uint64_t t0 = globaltimer_ns(); globaltimer_ns() - t0 < 2 * kWaitTimeoutNs;) {}
            __syncwarp();
            for (int j = grp; j < per; j += 2) {
                const int t = 4 * (rank * per + j);
                if (t >= tv) break;
                float4 v = sums[j * 128 + row];
                for (int q = 1; q < split; ++q) {
                    const float4 w = sums[(q * per + j) * 128 + row];
                    v.x += w.x;
                    v.y += w.y;
                    v.z += w.z;
                    v.w += w.w;
                }
                if (nn < a.N) {
                    out[static_cast<size_t>(t) * a.N] = float_to_half_bits(v.x);
                    if (t + 1 < tv) out[static_cast<size_t>(t + 1) * a.N] = float_to_half_bits(v.y);
                    if (t + 2 < tv) out[static_cast<size_t>(t + 2) * a.N] = float_to_half_bits(v.z);
                    if (t + 3 < tv) out[static_cast<size_t>(t + 3) * a.N] = float_to_half_bits(v.w);
                }
            }
            break;
        }
    }
    if (split > 1 && (warp < kEpi || warp == kScalesX)) tc::cluster_wait();

    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    if (warp == kIssuer) tc::tmem_dealloc(tbase, a.tmem_cols);
}

template <int BITS, int BOXES>
bool set_attributes(const DeviceInfo* di)
{
    static std::atomic<bool> ready[kMaxDevices];      // per device; setting the attribute twice is harmless
    if (ready[di->dev].load()) return true;
    if (cudaFuncSetAttribute(mx_gemm_kernel<BITS, BOXES>, cudaFuncAttributeMaxDynamicSharedMemorySize, kWhole) != cudaSuccess) return false;
    ready[di->dev].store(true);
    return true;
}

// Clusters of `split` CTAs, two or more, that fit the device at once (cached per device).
template <int BITS, int BOXES>
int cluster_capacity(const DeviceInfo* di, int split, bool half)
{
    static std::atomic<int> cached[kMaxDevices][9][2];
    if (const int n = cached[di->dev][split][half].load()) return n;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(split);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = half ? kHalf : kWhole;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (!set_attributes<BITS, BOXES>(di) || cudaOccupancyMaxActiveClusters(&n, mx_gemm_kernel<BITS, BOXES>, &cfg) != cudaSuccess) {
        cudaGetLastError();
        n = 0;
    }
    if (n > 0) cached[di->dev][split][half].store(n);
    return n;
}

// Up to this many tokens two CTAs of an SM, by their tensor memory and shared memory.
constexpr int kHalfTok = 80;

template <int BITS, int BOXES>
constexpr int slot_bytes(int tok)
{
    return (Cfg<BITS, BOXES>::kW + BOXES * tok * 128 + 2 * Cfg<BITS, BOXES>::kScales + 1023) / 1024 * 1024;
}

// Behind the header and the cluster's sums: of groups of four tokens by 128 rows, a
// CTA's share from each.
constexpr int ring_at(int tok, int split)
{
    return kHeader + (split > 1 ? (tok / 4 + split - 1) / split * split * 128 * 16 : 0);
}

template <int BITS, int BOXES>
constexpr int ring_slots(int tok, int split, bool half)
{
    const int n = ((half ? kHalf : kWhole) - ring_at(tok, split)) / slot_bytes<BITS, BOXES>(tok);
    return n < Cfg<BITS, BOXES>::kMaxSlots ? n : Cfg<BITS, BOXES>::kMaxSlots;
}

// Every tile and split has two slots at least, and its accumulators and scales lie in
// its tensor memory.  (Slots of two boxes are those of one CTA an SM.)
template <int BITS, int BOXES>
constexpr bool fits()
{
    for (int tok = 16; tok <= 128; tok += 16)
        for (int split = 1; split <= 8; ++split)
            for (int half = 0; half <= (BOXES == 1 && tok <= kHalfTok ? 1 : 0); ++half) {
                const int n = ring_slots<BITS, BOXES>(tok, split, half != 0);
                if (n < 2 || 2 * tok + n * Cfg<BITS, BOXES>::kScaleCols > kTmemCols / (half ? 2 : 1)) return false;
            }
    return true;
}

// A tile's sum must end within the limit of the epilogue's wait for it, 0.5 s: at ~0.25
// us for 128 K, 33 ms here in a CTA that has a tile to itself; 2^31 would take that long
// in a cluster of eight.  (The error that K / 32 additions may add is 2^-3 of the sum.)
constexpr int kMostK = 1 << 24;

struct Plan {
    int tok, split;
    bool half, pair;
};

template <int BITS, int BOXES>
int launch(const DeviceInfo* di, const CUtensorMap& w, const CUtensorMap& x, Args a, const Plan& pl, cudaStream_t stream)
{
    using C = Cfg<BITS, BOXES>;
    if (!set_attributes<BITS, BOXES>(di)) return WQ4_ERR_CUDA;
    const int64_t tiles = static_cast<int64_t>(a.rtiles) * a.ttiles;
    constexpr bool kFits = fits<BITS, BOXES>();
    static_assert(kFits, "rings of two slots and more, tensor memory");
    const int smem = pl.half ? kHalf : kWhole;
    a.tok = pl.tok;
    a.split = pl.split;
    a.slot_bytes = slot_bytes<BITS, BOXES>(pl.tok);
    a.ring = ring_at(pl.tok, pl.split);
    a.nslots = ring_slots<BITS, BOXES>(pl.tok, pl.split, pl.half);
    a.tmem_cols = pl.half ? kTmemCols / 2 : kTmemCols;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = a.split;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.split > 1 ? tiles * a.split : std::min<int64_t>(tiles, pl.half ? 2 * di->sm_count : di->sm_count)));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = a.split > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, mx_gemm_kernel<BITS, BOXES>, w, x, a) == cudaSuccess ? WQ4_OK : WQ4_ERR_CUDA;
}

// What a form takes, in us, with t = tokens of a tile / 128 and f = the share of its
// CTAs that are busy: a + at t, beside k0 + k0t t (alone) .. + k1 + k1t t more (f = 1)
// a slot; each round after the first waits for w, or for as long as the round
// before writes (e t, for rows that 16 bytes do not divide eo t) past its own slots;
// such rows o t at the end; where s CTAs share a tile's K s0 + st t + sf f +
// stf t f + ss (s - 2); where an SM has two CTAs kd a slot and d more.
struct Cost {
    double a, at, k0, k0t, k1, k1t, w, e, eo, o, s0, st, sf, stf, ss, kd, d;
};

// Fitted to 854 measurements (218 sizes of 1 to 8192 tokens, each form and split that
// is possible, over copies of 400 MB), those near the best of a size above all: what
// it picks takes 0.5 % more than the best on average, 16 % at most.  6144 x 4096 over
// one token: whole 6.9 us, K in halves 5.8; 4096 x 14336 over 16 tokens 17.0 whole,
// 9.1 in quarters; 512 tokens of 6144 x 4096 18.3 in single CTAs, 14.3 in pairs.  Over
// a short K the writing decides: 16384 x 512 over 4000 tokens 46.5 in single CTAs,
// 35.6 in pairs; of 16385 rows 53.8 and 69.8.
constexpr Cost kCost[2][3] = {
    // activations of 8 bits: two CTAs an SM, one, pairs
    {{1.873, 0.000, 0.175, 0.218, 0.166, 0.060, 0.000, 1.798, 1.859, 0.110, 0.276, 1.115, 0.001, 5.904, 0.000, 0.000, 0.933},
     {1.843, 1.192, 0.222, 0.151, 0.160, 0.052, 0.000, 1.798, 1.859, 0.110, 0.000, 2.210, 0.779, 1.566, 0.041, 0.000, 0.000},
     {2.084, 1.530, 0.107, 0.069, 0.038, 0.015, 0.698, 1.132, 2.384, 1.784, 0.000, 0.000, 0.000, 0.000, 0.000, 0.000, 0.000}},
    // of 4 bits
    {{2.159, 0.000, 0.159, 0.230, 0.516, 0.000, 0.156, 1.921, 1.921, 0.126, 0.025, 0.433, 0.000, 5.838, 0.000, 0.000, 0.987},
     {1.946, 1.114, 0.213, 0.000, 0.142, 0.000, 0.693, 1.921, 1.921, 0.126, 0.000, 1.445, 0.886, 2.076, 0.023, 0.000, 0.000},
     {2.675, 1.212, 0.126, 0.055, 0.074, 0.018, 0.832, 0.902, 2.464, 1.859, 0.000, 0.000, 0.000, 0.000, 0.000, 0.000, 0.000}}};

double estimate(const Cost& c, int tok, int slots, int64_t ctas, int cap, int s, bool whole_rows)
{
    const double t = tok / 128.0, f = std::min(1.0, static_cast<double>(ctas) / cap), n = (slots + s - 1) / s;
    const double k0 = c.k0 + c.k0t * t, k1 = k0 + c.k1 + c.k1t * t;
    const int64_t full = ctas / cap, rest = ctas % cap, more = std::max<int64_t>(0, full - (rest ? 0 : 1));
    double us = c.a + c.at * t + n * (full * k1 + (rest ? k0 + (k1 - k0) * rest / cap : 0.0));
    us += more * std::max(c.w, (whole_rows ? c.e : c.eo) * t - n * k1) + (whole_rows ? 0.0 : c.o * t);
    if (2 * ctas > cap) us += n * c.kd + c.d;
    if (s > 1) us += c.s0 + c.st * t + c.sf * f + c.stf * t * f + c.ss * (s - 2);
    return us;
}

// Up to this many weights a call fetches them into L2 while the previous kernel
// finishes: 5003 x 2176 over 77 tokens 5.8 us where without it 6.3.  Larger ones take
// bandwidth from that kernel and hold up their own copies (4096 x 14336 over 16 tokens
// 10.2 us with and 9.1 without, a decoder layer of one token 46.0 and 42.2).
constexpr int64_t kPrefetchWeights = 16 << 20;

// The form that calls take (wq4_test_mx_form): 0 the estimate's choice, 1 two CTAs an
// SM, 2 one, 3 pairs, and times 16 the CTAs that share a tile's K (0: the estimate's).
std::atomic<int> g_form{0};

// whole_rows: 16 bytes divide y's address and rows.  A split of 0: the form that a test
// has set does not take the call.
Plan pick(const DeviceInfo* di, int bits, int N, int M, int kblocks, bool whole_rows)
{
    const int tok = M > 112 ? 128 : (M + 15) / 16 * 16;
    const int64_t tiles = (static_cast<int64_t>(N) + 127) / 128 * ((static_cast<int64_t>(M) + tok - 1) / tok);
    const int set = g_form.load(), form = set % 16, cut = set / 16;
    Plan pl = {tok, 0, false, false};
    double best = 1e300;
    for (int half = tok <= kHalfTok ? 1 : 0; half >= 0; --half) {
        if (form && form != (half ? 1 : 2)) continue;
        const int slot = bits == 8 && half ? 1 : 2, slots = (kblocks + slot - 1) / slot;
        for (int s = 1; s <= 8 && s <= slots; ++s) {
            if (cut && s != cut) continue;
            // no more clusters than are on the GPU at once (a split that a test has set: in turns)
            const int fit = s == 1      ? 0
                            : bits == 4 ? cluster_capacity<4, 1>(di, s, half)
                            : half      ? cluster_capacity<8, 1>(di, s, true)
                                        : cluster_capacity<8, 2>(di, s, false);
            if (s > 1 && (fit < 1 || tiles > (cut ? INT32_MAX / s : fit))) continue;
            const double us = estimate(kCost[bits == 4][half ? 0 : 1], tok, slots, tiles * s, di->sm_count * (half ? 2 : 1), s, whole_rows);
            if (us < best) best = us, pl.split = s, pl.half = half != 0;
        }
    }
    if (form ? form == 3 : M > 64) {
        const int64_t pairs = (static_cast<int64_t>(N) + 255) / 256 * ((static_cast<int64_t>(M) + 255) / 256);
        if (estimate(kCost[bits == 4][2], 256, bits == 8 ? kblocks : (kblocks + 1) / 2, pairs, di->sm_count / 2, 1, whole_rows) < best)
            pl = {256, 1, false, true};
    }
    return pl;
}

// ------------------------------------------------------- pairs of CTAs --

// Tile of 256 weight rows and 256 tokens for the two CTAs of a cluster: each
// brings its 128 rows, half of the tokens and the scales of its rows and of all
// the tokens, 34 KB a slot where two CTAs of their own would take 50.
// Tensor memory holds two accumulators that share kOver columns, and the scales
// of each slot: the epilogue takes the shared columns first, and the other
// accumulator's MMAs begin when it has them.  (8192 tokens of 28672 x 4096 in 4 bits:
// 492 us by CTAs of their own with 128 x 128 tiles, 319 in pairs, 311 with predicated
// MMAs, 299 with the shared columns read first, 281 with a relaxed arrival.)  In the
// steady state 128 K of 8-bit activations take 512 cycles, the MMA rate; 256 K of
// 4-bit ones ~655, the 35 KB of a slot from L2.
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
            RingPos p;
            int n = 0;
            bool ok = true;
            for (int u = a.stall ? tiles : u0; u < tiles && ok; u += ustep) {
                const int n0 = u / a.ttiles * 256 + 128 * rank, m0 = u % a.ttiles * T;
                for (int k = 0; k < slots; ++k, ++n, p.next(S)) {
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
            // and so has every arrival on this CTA's barriers by the commits of the pair's
            // MMAs (those on dfull the epilogue has waited for): that CTA 0 has them on its
            // own says nothing of CTA 1's.  Where the waits before gave up, the issuer's
            // may only be giving up now: drain has twice the time.
            if (ok)
                for (int i = max(0, n - S); i < n; ++i) mbar_wait(&empty[i % S], (i / S) & 1, err);
            if (!mbar_wait(drain, 0, err)) mbar_wait(drain, 0, err);
        }
    } else if (warp == kIssuer) {
        if (rank == 0) {
            grid_dependency_wait();      // its waits are bounded, the previous kernel's time is not
            constexpr uint32_t idesc = BITS == 8 ? tc::idesc_mx_e2m1_e4m3(256, T) : tc::idesc_mx_e2m1_e2m1(256, T);
            const uint32_t leader = tc::elect_one() ? 1u : 0u;
            RingPos p;
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
                for (int k = 0; k < slots; ++k, p.next(S)) {
                    if (ok) ok = mbar_wait(&full[p.slot], p.par, err);
                    tc::fence_after_sync();
                    const uint64_t off = static_cast<uint64_t>(p.slot) * (C::kSlot >> 4);
                    const uint32_t scol = tbase + C::kScaleCol0 + p.slot * C::kScaleCols;
                    const int nb = min(NB, a.kblocks - k * NB);
                    // in tensor memory: the rows' scales of each 128 K, then the tokens' (two blocks of 128) of each
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        if (b > 0 && b >= nb) break;
                        tc::cp_scales_pair(scol + 4 * b, sdesc + off + b * 32, leader);
                        tc::cp_scales_pair(scol + 4 * NB + 8 * b, sdesc + off + (C::kScales >> 4) + b * 32, leader);
                        tc::cp_scales_pair(scol + 4 * NB + 8 * b + 4, sdesc + off + 2 * (C::kScales >> 4) + b * 32, leader);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int b = BITS == 8 ? 0 : j >> 1;
                        if (b > 0 && b >= nb) break;
                        const uint32_t acc = k > 0 || j > 0 ? 1u : 0u;
                        const uint32_t id = idesc | tc::idesc_mx_scale_byte(BITS == 8 ? j : 2 * (j & 1));
                        if constexpr (BITS == 8)
                            tc::mma_mxf8f6f4_pair(dcol, wdesc + off + 2 * j, xdesc + off + 2 * j, id, scol, scol + 4, acc, leader);
                        else
                            tc::mma_mxf4_pair(dcol, wdesc + off + 2 * j, xdesc + off + 2 * j, id, scol + 4 * b,
                                              scol + 4 * NB + 8 * b, acc, leader);
                    }
                    tc::commit_pair(&empty[p.slot], leader);
                    if (k == slots - 1) tc::commit_pair(dfull, leader);
                    __syncwarp();
                }
            }
            // all MMAs issued have completed before tensor memory is released
            tc::commit_pair(drain, leader);
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
            // Blocks of 32 tokens, the shared columns' first, to the two groups in turn.
            // Those go to registers before anything else: the next tile's MMAs wait.
            const int first = ((dit & 1) ? 0 : 8 - kOverBlocks) + grp;
            auto store = [&](int blk, const uint32_t d[32]) {
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
            };
            uint32_t d[kOverBlocks / 2][32];
#pragma unroll
            for (int i = 0; i < kOverBlocks / 2; ++i) tc::ld32(dcol + 32 * ((first + 2 * i) & 7), d[i]);
            tc::ld_wait();
            tc::fence_before_sync();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive_cluster_relaxed(dempty0);
#pragma unroll
            for (int i = 0; i < kOverBlocks / 2; ++i) store((first + 2 * i) & 7, d[i]);
#pragma unroll 1
            for (int i = kOverBlocks / 2; i < 4; ++i) {
                const int blk = (first + 2 * i) & 7;
                tc::ld32(dcol + 32 * blk, d[0]);
                tc::ld_wait();
                store(blk, d[0]);
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
    if ((static_cast<int64_t>(N - 1) / 128 + 1) * (static_cast<int64_t>(M - 1) / 128 + 1) > (static_cast<int64_t>(1) << 30)) return WQ4_ERR_UNSUPPORTED;
    if (K > kMostK) return WQ4_ERR_UNSUPPORTED;
    const DeviceInfo* di = current_device_info(nullptr);
    if (!di) return WQ4_ERR_CUDA;
    const bool bulk = (N % 8) == 0 && aligned(y, 16);
    const Plan pl = pick(di, bits, N, M, K / 128, bulk);
    if (pl.split == 0) return WQ4_ERR_UNSUPPORTED;
    const bool pair = pl.pair;
    const int T = pl.tok, rows = pair ? 256 : 128;
    Args a = {};
    a.y = y;
    a.w_scales = W_scales;
    a.x_scales = x_scales;
    a.N = N;
    a.M = M;
    a.kblocks = K / 128;
    a.rtiles = (N - 1) / rows + 1;
    a.ttiles = (M - 1) / T + 1;
    a.err = di->status;
    a.stall = test_copy_stall() == WQ4_STALL_GEMM_W ? 1 : 0;
    a.bulk = bulk ? 1 : 0;
    a.prefetch = !a.stall && static_cast<int64_t>(N) * K <= kPrefetchWeights ? 1 : 0;
    PairMaps tm;
    const uint64_t k = static_cast<uint64_t>(K), wrow = k / 2, xrow = k / 8 * bits, srow = k / 128 * 512;
    constexpr CUtensorMapDataType kBytes = CU_TENSOR_MAP_DATA_TYPE_UINT8, kWords = CU_TENSOR_MAP_DATA_TYPE_UINT32;
    constexpr CUtensorMapSwizzle kSwz = CU_TENSOR_MAP_SWIZZLE_128B, kPlain = CU_TENSOR_MAP_SWIZZLE_NONE;
    // activations of 8 bits: the weights' codes are spread on their way into shared memory
    constexpr CUtensorMapDataType kSpread = CU_TENSOR_MAP_DATA_TYPE_16U4_ALIGN16B;
    const uint32_t box = T < 128 ? T : 128, boxes = pl.half ? 1 : 2;
    const uint64_t n64 = static_cast<uint64_t>(N), m64 = static_cast<uint64_t>(M);
    bool ok;
    if (bits == 8 && !pair)
        ok = encode_tensor_map_3d(&tm.w, kSpread, W, {128, n64, k / 128}, {wrow, 64}, {128, 128, boxes}, kSwz) &&
             encode_tensor_map_3d(&tm.x, kBytes, x, {128, m64, k / 128}, {xrow, 128}, {128, box, boxes}, kSwz);
    else
        ok = encode_tensor_map_2d(&tm.w, bits == 8 ? kSpread : kBytes, W, bits == 8 ? k : wrow, n64, wrow, 128, 128, kSwz) &&
             encode_tensor_map_2d(&tm.x, kBytes, x, xrow, m64, xrow, 128, box, kSwz);
    if (!ok) return WQ4_ERR_CUDA;
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
    if (bits == 4) return launch<4, 1>(di, tm.w, tm.x, a, pl, st);
    return pl.half ? launch<8, 1>(di, tm.w, tm.x, a, pl, st) : launch<8, 2>(di, tm.w, tm.x, a, pl, st);
}

extern "C" int wq4_test_mx_form(int form, int split)
{
    if (form < 0 || form > 3 || split < 0 || split > 8 || (split > 0 && form != 1 && form != 2)) return WQ4_ERR_INVALID;
    g_form.store(16 * split + form);
    return WQ4_OK;
}
