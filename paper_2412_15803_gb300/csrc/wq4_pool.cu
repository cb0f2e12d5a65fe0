// wq4_pool.cu -- the pages of a key/value cache (sm_103a): taken, shared
// between sequences, given back, moved together.
//
// The bookkeeping lives on the device (page table, lengths, and refs[p] = how
// many page-table entries name page p, 0: free), so that every call is
// asynchronous and can be captured.  There is no list of free pages to keep in
// order: a call that needs k pages takes the k lowest-numbered free ones, found
// by a scan of refs that stops at the k-th.  So the same state and call give
// the same pages, whatever ran before.
//
// reserve, fork, compact and copy_pages plan in one block (the scan and the
// prefix sums over the sequences are serial by nature and short: at 16384
// pages a pass), and leave a list of page copies in the workspace; a second
// kernel over the whole GPU moves the bytes.  free and trim touch each table
// entry by itself and need one kernel over all of them.
//
// Measured: compacting 4096 pages of 16 layers (0.9 GB moved) 290 us, 6.2
// TB/s of the 6.8 of a copy, of which the plan takes ~10; eight forks of a
// sequence in 32 layers 13.8 us, trimming and growing 64 sequences 8.3 us, all
// three with the bookkeeping's copy before them: chains of dependent reads of a
// few words, each ~0.7 us.  So what does not depend on an earlier step is read ahead
// of it, and short lists of pages stay in shared memory (16.1 and 9.7 us without).
#include "wq4.h"
#include "wq4_attn.h"
#include "wq4_cache.h"
#include "wq4_device.cuh"
#include "wq4_host.h"

#include <cuda_runtime.h>

#include <algorithm>
#include <climits>

namespace wq4 {
namespace {

constexpr uint32_t kErrPool = 128u;          // status word: a call that could not be done in full
constexpr int kD = 128;
constexpr int kPlan = 1024;                  // threads of a planning block
constexpr int kPlanWarps = kPlan / 32;
constexpr int kScan = 16;                    // pages a lane looks at in a pass
constexpr int kScanPages = kPlan * kScan;
constexpr int kNear = 2048;                  // free pages that reserve lists in shared memory; more go through the workspace
constexpr int kCopyThreads = 256;
constexpr int kHdr = 64;                     // workspace words before the lists

struct PoolArgs {
    int32_t* table;       // [max_seqs][stride]
    int32_t* lens;        // [max_seqs]
    int32_t* refs;        // [num_pages]
    int32_t* hdr;         // workspace: [0] copies planned, [1] live pages (compact)
    int32_t* src;         // [pool_list] copies: from, to, rows of each head (negative from: nothing)
    int32_t* dst;
    int32_t* rows;
    int32_t* list;        // [pool_list] free pages taken / marks / new places
    int stride, page_size, num_pages, max_seqs;
    uint32_t* err;
};

struct PoolLayers {
    uint4* k[WQ4_KV_MAX_LAYERS];
    uint4* v[WQ4_KV_MAX_LAYERS];
};

__device__ __forceinline__ void flag(const PoolArgs& a) { atomicOr(a.err, kErrPool); }

__device__ __forceinline__ int pages_of(const PoolArgs& a, int T)
{
    const unsigned P = a.page_size;             // (the largest length and a page pass an int)
    return min(a.stride, static_cast<int>((static_cast<unsigned>(max(T, 0)) + P - 1u) / P));
}

// One reference of page e less.  A page that had none is flagged and stays at 0.
__device__ __forceinline__ void drop(const PoolArgs& a, int e)
{
    if (e >= a.num_pages || atomicSub(a.refs + e, 1) <= 0) {
        if (e < a.num_pages) atomicAdd(a.refs + e, 1);
        flag(a);
    }
}

// Exclusive prefix sum over the block's threads; *total gets the sum.  red: 32 words.
__device__ __forceinline__ int block_scan(int v, int* red, int* total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += u;
    }
    __syncthreads();               // red is free
    if (lane == 31) red[warp] = incl;
    __syncthreads();
    int w = red[lane], wi = w;     // every warp sums the warps' totals
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, wi, o);
        if (lane >= o) wi += u;
    }
    *total = __shfl_sync(0xffffffffu, wi, 31);
    return __shfl_sync(0xffffffffu, wi - w, warp) + incl - v;
}

// The references of a scan's pass from page `base` on: page base + 512 warp + 32 i + lane.
__device__ __forceinline__ void load_refs(const PoolArgs& a, int base, int r[kScan])
{
    const int p0 = base + (threadIdx.x >> 5) * (32 * kScan) + (threadIdx.x & 31);
#pragma unroll
    for (int i = 0; i < kScan; ++i) r[i] = p0 + 32 * i < a.num_pages ? __ldcg(a.refs + p0 + 32 * i) : 1;
}

// The `want` lowest free pages into list; returns how many there are (at most want).
// r: the first pass's references, which the caller loads as early as they hold.
__device__ int find_free(const PoolArgs& a, int want, int* list, int* red, int r[kScan])
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int found = 0;
    for (int base = 0; base < a.num_pages && found < want; base += kScanPages) {
        const int p0 = base + warp * (32 * kScan) + lane;
        if (base) load_refs(a, base, r);
        int mine = 0;
#pragma unroll
        for (int i = 0; i < kScan; ++i) mine += __popc(__ballot_sync(0xffffffffu, r[i] == 0));
        int total;
        int at = found + block_scan(lane == 0 ? mine : 0, red, &total);
        at = __shfl_sync(0xffffffffu, at, 0);
#pragma unroll
        for (int i = 0; i < kScan; ++i) {
            const uint32_t m = __ballot_sync(0xffffffffu, r[i] == 0);
            const int k = at + __popc(m & ((1u << lane) - 1u));
            if (r[i] == 0 && k < want) list[k] = p0 + 32 * i;
            at += __popc(m);
        }
        found += total;
    }
    __syncthreads();               // the list is written
    return min(found, want);
}

// ------------------------------------------------------------- free, trim --

// A thread a table entry.  whole: the sequence goes; else what the token after
// the last one sees under (window, sinks) stays.
__global__ void __launch_bounds__(256) pool_drop_kernel(const PoolArgs a, const int32_t* seqs, int whole, int window, int sinks)
{
    grid_dependency_wait();
    grid_dependents_launch();
    const int s = seqs[blockIdx.x];
    if (s < 0 || s >= a.max_seqs) {
        if (blockIdx.y == 0 && threadIdx.x == 0) flag(a);
        return;
    }
    const int T = a.lens[s], held = pages_of(a, T);
    for (int j = blockIdx.y * 256 + threadIdx.x; j < held; j += gridDim.y * 256) {
        const int64_t first = static_cast<int64_t>(j) * a.page_size;
        const bool keep = !whole && (first < sinks || first + a.page_size > static_cast<int64_t>(T) + 1 - window);
        if (!keep) {
            // exchanged: a sequence that is listed twice gives each page back once
            const int e = atomicExch(a.table + static_cast<size_t>(s) * a.stride + j, -1);
            if (e >= 0) drop(a, e);
        }
    }
}

__global__ void __launch_bounds__(256) pool_empty_kernel(const PoolArgs a, const int32_t* seqs, int n)
{
    grid_dependency_wait();
    grid_dependents_launch();
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n && seqs[i] >= 0 && seqs[i] < a.max_seqs) a.lens[seqs[i]] = 0;
}

// ---------------------------------------------------------------- reserve --

__global__ void __launch_bounds__(kPlan) pool_reserve_kernel(const PoolArgs a, const int32_t* seqs, const int32_t* new_lens, int n)
{
    __shared__ int red[32];
    __shared__ int first_at[WQ4_KV_MAX_SEQS];
    __shared__ int near_list[kNear];
    __shared__ int off[WQ4_KV_MAX_SEQS], have[WQ4_KV_MAX_SEQS], seq_of[WQ4_KV_MAX_SEQS], need_of[WQ4_KV_MAX_SEQS];
    grid_dependency_wait();
    grid_dependents_launch();
    const int i = threadIdx.x, lane = i & 31, warp = i >> 5;
    first_at[i] = INT_MAX;
    int refs[kScan];
    load_refs(a, 0, refs);
    __syncthreads();
    int s = -1, L = 0, T = 0;
    if (i < n) {
        s = seqs[i];
        L = new_lens[i];
        if (s < 0 || s >= a.max_seqs) {
            s = -1;
        } else {
            atomicMin(&first_at[s], i);
            T = a.lens[s];
        }
    }
    __syncthreads();
    int need = 0, old = 0;
    if (i < n) {
        if (s >= 0 && first_at[s] != i) s = -1;                            // listed before
        if (s >= 0 && (L < 0 || L > static_cast<int64_t>(a.stride) * a.page_size || L < T)) s = -1;
        if (s < 0) flag(a);
        else {
            old = pages_of(a, T);
            need = pages_of(a, L) - old;
        }
    }
    int total;
    const int at = block_scan(need, red, &total);
    off[i] = at;
    have[i] = old;
    need_of[i] = need;
    seq_of[i] = s;
    int* list = total <= kNear ? near_list : a.list;
    const int avail = find_free(a, total, list, red, refs);        // synchronises the block
    // a warp a sequence; from the first that does not fit, none gets any
    for (int k = warp; k < n; k += kPlanWarps) {
        if (seq_of[k] < 0 || need_of[k] == 0) continue;
        if (off[k] + need_of[k] > avail) {
            if (lane == 0) flag(a);
            continue;
        }
        int32_t* row = a.table + static_cast<size_t>(seq_of[k]) * a.stride + have[k];
        for (int j = lane; j < need_of[k]; j += 32) {
            const int p = list[off[k] + j];
            row[j] = p;
            a.refs[p] = 1;
        }
    }
    if (s >= 0 && off[i] + need <= avail) a.lens[s] = L;
    else if (s >= 0 && need == 0) a.lens[s] = L;
}

// ------------------------------------------------------------------- fork --

__global__ void __launch_bounds__(kPlan) pool_fork_kernel(const PoolArgs a, const int32_t* parents, const int32_t* children, int n)
{
    __shared__ int red[32];
    __shared__ int child_at[WQ4_KV_MAX_SEQS];
    __shared__ uint8_t is_parent[WQ4_KV_MAX_SEQS];
    __shared__ int par[WQ4_KV_MAX_SEQS], chi[WQ4_KV_MAX_SEQS], page[WQ4_KV_MAX_SEQS], list[WQ4_KV_MAX_SEQS];
    __shared__ int held[WQ4_KV_MAX_SEQS], len[WQ4_KV_MAX_SEQS];
    grid_dependency_wait();
    grid_dependents_launch();
    const int i = threadIdx.x, lane = i & 31, warp = i >> 5;
    child_at[i] = INT_MAX;
    is_parent[i] = 0;
    __syncthreads();
    int p = -1, c = -1;
    if (i < n) {
        p = parents[i];
        c = children[i];
        if (p < 0 || p >= a.max_seqs || c < 0 || c >= a.max_seqs) p = c = -1;
        else {
            is_parent[p] = 1;
            atomicMin(&child_at[c], i);
        }
    }
    __syncthreads();
    if (i < n) {
        if (c >= 0 && (child_at[c] != i || is_parent[c])) p = c = -1;
        if (c < 0) flag(a);
    }
    // Lengths, and a page of its own where the parent's last one is not full.  (No parent
    // is a child, so what a parent has does not change below.)
    int need = 0, T = 0, last = -1;
    if (c >= 0) {
        held[i] = pages_of(a, a.lens[c]);
        T = a.lens[p];
        if (T < 0 || T > static_cast<int64_t>(a.stride) * a.page_size) {
            flag(a);
            T = 0;
        }
        if (T % a.page_size) {
            last = a.table[static_cast<size_t>(p) * a.stride + T / a.page_size];
            need = last >= 0 && last < a.num_pages ? 1 : 0;
        }
    }
    par[i] = p;
    chi[i] = c;
    len[i] = T;
    __syncthreads();
    // what the children held goes back first; four entries a lane at a time
    for (int k = warp; k < n; k += kPlanWarps) {
        if (chi[k] < 0) continue;
        int32_t* row = a.table + static_cast<size_t>(chi[k]) * a.stride;
        const int np = held[k];
#pragma unroll 4
        for (int j = lane; j < np; j += 32) {
            const int e = row[j];
            row[j] = -1;
            if (e >= 0) drop(a, e);
        }
    }
    __syncthreads();
    int total;
    const int at = block_scan(need, red, &total);
    int refs[kScan];
    load_refs(a, 0, refs);
    const int avail = find_free(a, total, list, red, refs);
    int mine = -1;                                     // the child's own last page
    if (need && at < avail) mine = list[at];
    page[i] = mine;
    if (i < n) {
        a.src[i] = mine >= 0 ? last : -1;
        a.dst[i] = mine;
        a.rows[i] = T % a.page_size;
        if (mine >= 0) a.refs[mine] = 1;
        if (c >= 0) {
            if (need && mine < 0) {                    // no page left: the child stays empty
                flag(a);
                T = 0;
                chi[i] = -1;
            }
            a.lens[c] = T;
        }
    }
    if (i == 0) a.hdr[0] = n;
    __syncthreads();
    for (int k = warp; k < n; k += kPlanWarps) {
        if (chi[k] < 0) continue;
        const int32_t* from = a.table + static_cast<size_t>(par[k]) * a.stride;
        int32_t* row = a.table + static_cast<size_t>(chi[k]) * a.stride;
        const int np = pages_of(a, len[k]);
        for (int j = lane; j < np; j += 32) {
            int e = from[j];
            if (e >= a.num_pages) {
                flag(a);
                e = -1;
            }
            if (page[k] >= 0 && j == np - 1) e = page[k];
            else if (e >= 0) atomicAdd(a.refs + e, 1);
            row[j] = e < 0 ? -1 : e;
        }
    }
}

// ---------------------------------------------------------------- compact --

__global__ void __launch_bounds__(kPlan) pool_compact_kernel(const PoolArgs a)
{
    __shared__ int red[32];
    grid_dependency_wait();
    grid_dependents_launch();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int count = 0;
#pragma unroll 8
    for (int p = threadIdx.x; p < a.num_pages; p += kPlan) count += __ldcg(a.refs + p) > 0 ? 1 : 0;
    int live;
    block_scan(count, red, &live);
    // the k-th live page behind the first `live` ones goes to the k-th free one among them
    int holes = 0, movers = 0;
    for (int base = 0; base < a.num_pages; base += kScanPages) {
        const int p0 = base + warp * (32 * kScan) + lane;
        int r[kScan];
#pragma unroll
        for (int i = 0; i < kScan; ++i) r[i] = p0 + 32 * i < a.num_pages ? __ldcg(a.refs + p0 + 32 * i) : -1;
        int h = 0, m = 0;
#pragma unroll
        for (int i = 0; i < kScan; ++i) {
            const int p = p0 + 32 * i;
            h += __popc(__ballot_sync(0xffffffffu, p < live && r[i] <= 0 && p < a.num_pages));
            m += __popc(__ballot_sync(0xffffffffu, p >= live && r[i] > 0));
        }
        int total;                                     // both counts in one sum: at most 16384 each
        int at = block_scan(lane == 0 ? h | m << 16 : 0, red, &total);
        at = __shfl_sync(0xffffffffu, at, 0);
        int ah = holes + (at & 0xFFFF), am = movers + (at >> 16);
#pragma unroll
        for (int i = 0; i < kScan; ++i) {
            const int p = p0 + 32 * i;
            const bool hole = p < live && r[i] <= 0 && p < a.num_pages, mover = p >= live && r[i] > 0;
            const uint32_t bh = __ballot_sync(0xffffffffu, hole), bm = __ballot_sync(0xffffffffu, mover);
            const uint32_t below = (1u << lane) - 1u;
            if (hole) a.dst[ah + __popc(bh & below)] = p;
            if (mover) a.src[am + __popc(bm & below)] = p;
            else if (p >= live && p < a.num_pages) a.list[p] = -1;
            ah += __popc(bh);
            am += __popc(bm);
        }
        holes += total & 0xFFFF;
        movers += total >> 16;
    }
    __syncthreads();
    // as many holes as movers: both are the live pages that are not among the first `live`
    for (int k = threadIdx.x; k < movers; k += kPlan) {
        const int s = a.src[k], d = a.dst[k];
        a.rows[k] = a.page_size;
        a.list[s] = d;
        a.refs[d] = a.refs[s];
        a.refs[s] = 0;
    }
    if (threadIdx.x == 0) {
        a.hdr[0] = movers;
        a.hdr[1] = live;
    }
}

// ------------------------------------------------------------- copy_pages --

__global__ void __launch_bounds__(kPlan) pool_copy_plan_kernel(const PoolArgs a, const int32_t* src, const int32_t* dst, int n)
{
    grid_dependency_wait();
    grid_dependents_launch();
    auto good = [&](int p) { return p >= 0 && p < a.num_pages; };
    for (int i = threadIdx.x; i < n; i += kPlan) {
        const int s = src[i], d = dst[i];
        if (good(s)) a.list[s] = 0;
        if (good(d)) a.list[d] = 0;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kPlan)
        if (good(src[i]) && good(dst[i])) atomicAdd(a.list + dst[i], 1);
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kPlan) {
        const int s = src[i], d = dst[i];
        // the page has one writer and no reader but it
        const bool ok = good(s) && good(d) && __ldcg(a.list + d) == 1 && __ldcg(a.list + s) == 0;
        a.src[i] = ok ? s : -1;
        a.dst[i] = d;
        a.rows[i] = a.page_size;
        if (!ok) flag(a);
    }
    if (threadIdx.x == 0) a.hdr[0] = n;
}

// ------------------------------------------------------- the bytes moved --

// The planned copies of every layer: a block takes the keys or the values of
// one page in one layer, 16 bytes a thread and step, eight steps' loads ahead of
// their stores.  remap: compact's, the page table's entries go to their pages'
// new places.
__global__ void __launch_bounds__(kCopyThreads) pool_copy_kernel(const PoolArgs a, const __grid_constant__ PoolLayers layers,
                                                                 int num_layers, int Hkv, int remap)
{
    grid_dependency_wait();
    grid_dependents_launch();
    const int n = __ldcg(a.hdr);
    const int P16 = a.page_size * (kD / 8);            // 16-byte words of a head's page
    const int64_t units = static_cast<int64_t>(n) * num_layers * 2;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int i = static_cast<int>(u % n), lv = static_cast<int>(u / n);
        const int s = __ldcg(a.src + i), d = __ldcg(a.dst + i);
        if (s < 0) continue;
        uint4* base = lv & 1 ? layers.v[lv >> 1] : layers.k[lv >> 1];
        const uint4* from = base + static_cast<size_t>(s) * Hkv * P16;
        uint4* to = base + static_cast<size_t>(d) * Hkv * P16;
        const int r16 = __ldcg(a.rows + i) * (kD / 8);
        const int words = Hkv * r16;
        for (int e0 = threadIdx.x; e0 < words; e0 += 8 * kCopyThreads) {
            uint4 w[8];
            int at[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int e = e0 + j * kCopyThreads;
                at[j] = r16 == P16 ? e : e / r16 * P16 + e % r16;
                if (e < words) w[j] = __ldcs(from + at[j]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (e0 + j * kCopyThreads < words) __stcs(to + at[j], w[j]);
        }
    }
    if (remap) {
        const int live = __ldcg(a.hdr + 1);
        const int64_t all = static_cast<int64_t>(a.max_seqs) * a.stride;
        for (int64_t e = static_cast<int64_t>(blockIdx.x) * kCopyThreads + threadIdx.x; e < all;
             e += static_cast<int64_t>(gridDim.x) * kCopyThreads) {
            const int p = a.table[e];
            if (p < live) continue;
            const int to = p < a.num_pages ? __ldcg(a.list + p) : -1;
            a.table[e] = to;
            if (to < 0) flag(a);                       // an entry without a reference, or outside the pool
        }
    }
}

// ------------------------------------------------------------------- host --

// Entries of a list in the workspace: a copy of every page, or of every pair of a fork.
size_t pool_list(int num_pages) { return static_cast<size_t>(std::max(num_pages, WQ4_KV_MAX_SEQS)); }

size_t pool_words(int num_pages) { return kHdr + 4 * pool_list(num_pages); }

int check_pool(const wq4_kv_pool* pool, PoolArgs* a)
{
    if (!pool || !pool->layers || !pool->page_table || !pool->seq_lens || !pool->page_refs || !pool->workspace)
        return WQ4_ERR_INVALID;
    if (pool->num_layers < 1 || pool->max_seqs < 1) return WQ4_ERR_INVALID;
    if (pool->num_layers > WQ4_KV_MAX_LAYERS || pool->max_seqs > WQ4_KV_MAX_SEQS) return WQ4_ERR_UNSUPPORTED;
    const wq4_kv_cache& c0 = pool->layers[0];
    for (int l = 0; l < pool->num_layers; ++l) {
        const wq4_kv_cache& c = pool->layers[l];
        if (!c.k || !c.v || c.num_pages < 1 || c.n_kv_heads < 1 || c.page_size < 16 || c.page_size % 16 ||
            c.page_table_stride < 1 || c.page_table != pool->page_table || c.num_pages != c0.num_pages ||
            c.n_kv_heads != c0.n_kv_heads || c.page_size != c0.page_size || c.head_dim != c0.head_dim ||
            c.page_table_stride != c0.page_table_stride)
            return WQ4_ERR_INVALID;
        if (c.head_dim != kD) return WQ4_ERR_UNSUPPORTED;
        if (!aligned(c.k, 16) || !aligned(c.v, 16)) return WQ4_ERR_ALIGN;
    }
    // what is counted in int: a sequence's tokens, a layer's rows, a page's 16-byte words, the pages of all sequences
    if (static_cast<int64_t>(c0.page_table_stride) * c0.page_size >= (int64_t(1) << 30) || cache_rows(c0) < 0 ||
        static_cast<int64_t>(c0.n_kv_heads) * c0.page_size >= (int64_t(1) << 26) ||
        static_cast<int64_t>(pool->max_seqs) * c0.page_table_stride >= (int64_t(1) << 31))
        return WQ4_ERR_UNSUPPORTED;
    if (!aligned(pool->page_table, 4) || !aligned(pool->seq_lens, 4) || !aligned(pool->page_refs, 4) ||
        !aligned(pool->workspace, 16))
        return WQ4_ERR_ALIGN;
    if (pool->workspace_bytes < pool_words(c0.num_pages) * 4) return WQ4_ERR_INVALID;
    a->table = pool->page_table;
    a->lens = pool->seq_lens;
    a->refs = pool->page_refs;
    a->hdr = static_cast<int32_t*>(pool->workspace);
    a->src = a->hdr + kHdr;
    a->dst = a->src + pool_list(c0.num_pages);
    a->rows = a->dst + pool_list(c0.num_pages);
    a->list = a->rows + pool_list(c0.num_pages);
    a->stride = c0.page_table_stride;
    a->page_size = c0.page_size;
    a->num_pages = c0.num_pages;
    a->max_seqs = pool->max_seqs;
    a->err = nullptr;                // found once the lists are checked too
    return WQ4_OK;
}

// Launch with programmatic dependent launch, as every kernel of the library.
template <typename... Params, typename... Args>
int launch(void (*kernel)(Params...), dim3 grid, int threads, void* stream, Args... args)
{
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.stream = static_cast<cudaStream_t>(stream);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? WQ4_OK : WQ4_ERR_CUDA;
}

// At most `most` copies (the device knows how many): the kernel that makes them.
int launch_copies(const wq4_kv_pool* pool, const PoolArgs& a, int64_t most, bool remap, void* stream)
{
    PoolLayers layers;
    for (int l = 0; l < pool->num_layers; ++l) {
        layers.k[l] = reinterpret_cast<uint4*>(pool->layers[l].k);
        layers.v[l] = reinterpret_cast<uint4*>(pool->layers[l].v);
    }
    int dev = 0;
    const DeviceInfo* di = current_device_info(&dev);
    if (!di) return WQ4_ERR_CUDA;
    const int64_t units = most * pool->num_layers * 2;
    const int grid = static_cast<int>(std::min<int64_t>(std::max<int64_t>(units, 1), 8 * di->sm_count));
    return launch(pool_copy_kernel, dim3(grid), kCopyThreads, stream, a, layers, pool->num_layers, pool->layers[0].n_kv_heads,
                  remap ? 1 : 0);
}

bool bad_list(const void* p, int n, int most) { return n < 0 || n > most || (n > 0 && !p); }

}  // namespace
}  // namespace wq4

using namespace wq4;

extern "C" size_t wq4_kv_pool_workspace_bytes(int num_pages, int max_seqs)
{
    if (num_pages < 1 || max_seqs < 1 || max_seqs > WQ4_KV_MAX_SEQS) return 0;
    return pool_words(num_pages) * 4;
}

extern "C" int wq4_kv_free(const wq4_kv_pool* pool, const int32_t* seqs, int n, void* stream)
{
    PoolArgs a;
    const int rc = check_pool(pool, &a);
    if (rc != WQ4_OK) return rc;
    if (bad_list(seqs, n, WQ4_KV_MAX_SEQS)) return WQ4_ERR_INVALID;
    if (!aligned(seqs, 4)) return WQ4_ERR_ALIGN;
    if (n == 0) return WQ4_OK;
    if (!(a.err = status_word())) return WQ4_ERR_CUDA;
    const int r = launch(pool_drop_kernel, dim3(n, std::min((a.stride + 255) / 256, 1024)), 256, stream, a, seqs, 1, 0, 0);
    return r != WQ4_OK ? r : launch(pool_empty_kernel, dim3((n + 255) / 256), 256, stream, a, seqs, n);
}

extern "C" int wq4_kv_trim(const wq4_kv_pool* pool, const int32_t* seqs, int n, int window, int n_sinks, void* stream)
{
    PoolArgs a;
    const int rc = check_pool(pool, &a);
    if (rc != WQ4_OK) return rc;
    if (bad_list(seqs, n, WQ4_KV_MAX_SEQS) || window < 1 || n_sinks < 0) return WQ4_ERR_INVALID;
    if (!aligned(seqs, 4)) return WQ4_ERR_ALIGN;
    if (n == 0) return WQ4_OK;
    if (!(a.err = status_word())) return WQ4_ERR_CUDA;
    return launch(pool_drop_kernel, dim3(n, std::min((a.stride + 255) / 256, 1024)), 256, stream, a, seqs, 0, window, n_sinks);
}

extern "C" int wq4_kv_reserve(const wq4_kv_pool* pool, const int32_t* seqs, const int32_t* new_lens, int n, void* stream)
{
    PoolArgs a;
    const int rc = check_pool(pool, &a);
    if (rc != WQ4_OK) return rc;
    if (bad_list(seqs, n, WQ4_KV_MAX_SEQS) || bad_list(new_lens, n, WQ4_KV_MAX_SEQS)) return WQ4_ERR_INVALID;
    if (!aligned(seqs, 4) || !aligned(new_lens, 4)) return WQ4_ERR_ALIGN;
    if (n == 0) return WQ4_OK;
    if (!(a.err = status_word())) return WQ4_ERR_CUDA;
    return launch(pool_reserve_kernel, dim3(1), kPlan, stream, a, seqs, new_lens, n);
}

extern "C" int wq4_kv_fork(const wq4_kv_pool* pool, const int32_t* parents, const int32_t* children, int n, void* stream)
{
    PoolArgs a;
    const int rc = check_pool(pool, &a);
    if (rc != WQ4_OK) return rc;
    if (bad_list(parents, n, WQ4_KV_MAX_SEQS) || bad_list(children, n, WQ4_KV_MAX_SEQS)) return WQ4_ERR_INVALID;
    if (!aligned(parents, 4) || !aligned(children, 4)) return WQ4_ERR_ALIGN;
    if (n == 0) return WQ4_OK;
    if (!(a.err = status_word())) return WQ4_ERR_CUDA;
    const int r = launch(pool_fork_kernel, dim3(1), kPlan, stream, a, parents, children, n);
    return r != WQ4_OK ? r : launch_copies(pool, a, n, false, stream);
}

extern "C" int wq4_kv_compact(const wq4_kv_pool* pool, void* stream)
{
    PoolArgs a;
    const int rc = check_pool(pool, &a);
    if (rc != WQ4_OK) return rc;
    if (!(a.err = status_word())) return WQ4_ERR_CUDA;
    const int r = launch(pool_compact_kernel, dim3(1), kPlan, stream, a);
    return r != WQ4_OK ? r : launch_copies(pool, a, a.num_pages, true, stream);
}

extern "C" int wq4_kv_copy_pages(const wq4_kv_pool* pool, const int32_t* src, const int32_t* dst, int n, void* stream)
{
    PoolArgs a;
    const int rc = check_pool(pool, &a);
    if (rc != WQ4_OK) return rc;
    if (bad_list(src, n, a.num_pages) || bad_list(dst, n, a.num_pages)) return WQ4_ERR_INVALID;
    if (!aligned(src, 4) || !aligned(dst, 4)) return WQ4_ERR_ALIGN;
    if (n == 0) return WQ4_OK;
    if (!(a.err = status_word())) return WQ4_ERR_CUDA;
    const int r = launch(pool_copy_plan_kernel, dim3(1), kPlan, stream, a, src, dst, n);
    return r != WQ4_OK ? r : launch_copies(pool, a, n, false, stream);
}
