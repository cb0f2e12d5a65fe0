// wq4_prompt.cu -- the new tokens of prompts (sm_103a): their keys and values
// into a paged cache, and their attention over it, causal, with or without a
// sliding window and first tokens that stay visible.
#include "wq4.h"
#include "wq4_attn.h"
#include "wq4_cache.h"
#include "wq4_device.cuh"
#include "wq4_host.h"
#include "wq4_seen.h"
#include "wq4_tc.cuh"

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cfloat>
#include <climits>
#include <cmath>

namespace wq4 {
namespace {

// ------------------------------------------------------- tensor-core pieces --

// 32 consecutive columns of the lane's own row.
__device__ __forceinline__ void ld32(uint32_t taddr, uint32_t v[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        :
        "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
        "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
        "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
        "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(taddr)
        : "memory");
}

__device__ __forceinline__ void st32(uint32_t taddr, const uint32_t v[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
        "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]),
        "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]),
        "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
        : "memory");
}

// Bits of the instruction descriptor: A negated; B stored with N contiguous.
constexpr uint32_t kIdescNegA = 1u << 13;
constexpr uint32_t kIdescTransB = 1u << 16;

// Shared-memory matrix descriptor of an operand stored with its M or N extent
// contiguous, 128-byte swizzle (rows of 128 bytes = 64 fp16, one row a k): the
// next 64 elements `lead` bytes on (leading byte offset / 16 at bits [16, 30)),
// the next 8 k 1024 bytes on.  A K step of 16 advances the start by 2048 bytes.
__device__ __forceinline__ uint64_t sw128_mnmajor_desc(uint32_t saddr, uint32_t lead)
{
    return static_cast<uint64_t>((saddr >> 4) & 0x3FFFu) | (static_cast<uint64_t>(lead >> 4) << 16) |
           (static_cast<uint64_t>(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

constexpr int kD = 128;
constexpr int kMaxGroup = 8;
constexpr int kMaxHeads = 1 << 16;                 // widths of rows stay within an int

// Rows of the batch: whose each is, and where it stands.
struct Rows {
    const int32_t* starts;   // [batch + 1]
    const int32_t* lens;     // [batch]
    int batch, rows;
};

struct Paged {
    uint16_t* k;
    uint16_t* v;
    const int32_t* table;
    int stride, page_size, num_pages, Hkv;
};

// The sequence that owns row r (-1: none) and the row's position.  (Plain loads here
// and of the page table, not through the read-only path: the previous kernel, which
// this one's launch may overlap, may have written them.)
__device__ __forceinline__ int row_owner(const Rows& R, int r, int* pos)
{
    int lo = 0, hi = R.batch - 1;
    while (lo < hi) {              // the last sequence that starts at or before r
        const int mid = (lo + hi + 1) >> 1;
        if (R.starts[mid] <= r) lo = mid;
        else hi = mid - 1;
    }
    const int s = R.starts[lo], e = R.starts[lo + 1];
    *pos = R.lens[lo] - e + r;
    return r >= s && r < e && r < R.rows ? lo : -1;
}

// ----------------------------------------------------------------- append --

constexpr int kAppThreads = 128;

struct AppendArgs {
    Rows rows;
    Paged c;
    const uint16_t* qkv;
    uint16_t* q_out;                 // null: q is left alone
    int qkv_stride, q_out_stride, Hq, rotate;
    uint32_t* err;
    uint64_t turns[kD / 2];          // angle of position 1 in turns, times 2^64
};

// Cosine and sine as sums of a value of 12 significant bits and a remainder
// (x + y, z + w), each to about 2^-26, of pos times the angle in turns.  The
// product modulo a turn is exact in 64-bit integers (fp64, which GB300 has at 1.25
// TFLOP/s, made the angles cost more than the copy that they are for: 8192 rows of
// 48 heads 68 us); a quarter of a turn is split off and the rest, |x| <= pi / 4,
// goes through the Taylor series, with what rounding x to fp32 leaves over.
__device__ __forceinline__ float4 rotation(int pos, uint64_t turns)
{
    const uint64_t t = static_cast<uint64_t>(pos) * turns;
    const uint32_t quarter = static_cast<uint32_t>((t + (1ull << 61)) >> 62);
    const int r = static_cast<int>(static_cast<int64_t>(t - (static_cast<uint64_t>(quarter) << 62)) >> 31);   // turns * 2^33
    const float rh = static_cast<float>(r), rl = static_cast<float>(r - static_cast<int>(rh));
    constexpr double kTurn = 6.283185307179586476925 / 8589934592.0;          // 2 pi / 2^33
    constexpr float kHi = static_cast<float>(kTurn), kLo = static_cast<float>(kTurn - static_cast<double>(kHi));
    const float x = rh * kHi, xl = fmaf(rh, kHi, -x) + fmaf(rh, kLo, rl * kHi);
    const float z = x * x, zl = fmaf(x, x, -z);
    const float S = fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f);
    const float C = fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f);
    float sh = x, sl = fmaf(x * z, S, fmaf(-0.5f * z, xl, xl));
    float ch = fmaf(-0.5f, z, 1.f), cl = fmaf(z * z, C, fmaf(-0.5f, z, 1.f - ch) - fmaf(0.5f, zl, x * xl));
    if (quarter & 1) {               // (c, s) -> (-s, c)
        const float h = sh, l = sl;
        sh = ch;
        sl = cl;
        ch = -h;
        cl = -l;
    }
    if (quarter & 2) {
        ch = -ch;
        cl = -cl;
        sh = -sh;
        sl = -sl;
    }
    const float c12 = __uint_as_float(__float_as_uint(ch) & 0xFFFFF000u), s12 = __uint_as_float(__float_as_uint(sh) & 0xFFFFF000u);
    return make_float4(c12, (ch - c12) + cl, s12, (sh - s12) + sl);
}

// (x0, x1) turned by the angle whose cosine and sine are t.x + t.y and t.z + t.w.
// t.x and t.z have 12 significant bits, an fp16 value 11: their products are exact
// in fp32, so the difference of the two large products is rounded once and the
// remainders (2^-12 of them) add what they lack.
__device__ __forceinline__ uint32_t turn(uint32_t x, float4 t)
{
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&x));
    const float re = fmaf(v.x, t.x, -(v.y * t.z)) + fmaf(v.x, t.y, -(v.y * t.w));
    const float im = fmaf(v.x, t.z, v.y * t.x) + fmaf(v.x, t.w, v.y * t.y);
    const __half2 h = __floats2half2_rn(re, im);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// A row is taken by 16 kGroups threads: 16 bytes of a head by one thread, every
// kGroups-th head, kAhead heads' loads ahead of their stores.  A thread's four
// rotations serve all its heads in registers (a table in shared memory, read again
// for each head, cost 18 us of 52 over 8192 rows of 48 heads).  The first heads are
// under way while the row's place and rotations are found.  Few rows take four
// groups, whose chains are shorter (512 rows 6.0 us, two groups 7.4), many take two,
// which find half as many rotations (4096 rows 21.2 us, four groups 22.7; 8192 36.6
// and 37.9); they part at ~10 rows an SM (1280 9.0 and 9.6, 1536 12.5 and 10.5).
template <int kGroups, int kAhead>
__global__ void __launch_bounds__(kAppThreads) prompt_append_kernel(const __grid_constant__ AppendArgs a)
{
    grid_dependency_wait();
    grid_dependents_launch();
    constexpr int kRow = 16 * kGroups;                 // threads of a row
    const int row = blockIdx.x * (kAppThreads / kRow) + threadIdx.x / kRow, h0 = threadIdx.x / 16 % kGroups, w = threadIdx.x & 15;
    if (row >= a.rows.rows) return;
    const int heads = a.Hq + 2 * a.c.Hkv;
    const uint4* in = reinterpret_cast<const uint4*>(a.qkv + static_cast<size_t>(row) * a.qkv_stride) + w;
    uint4 x[kAhead];
    auto load = [&](int h) {         // (a row that no sequence owns is in the buffer too)
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (h + kGroups * i < heads) x[i] = __ldcs(in + (h + kGroups * i) * (kD / 8));
    };
    load(h0);
    int pos;
    const int b = row_owner(a.rows, row, &pos);
    if (b < 0) return;
    int64_t dst = -1;                // (page, row) as a row of head 0; -1: not written
    const int page = pos >= 0 && pos < a.c.stride * a.c.page_size
                         ? a.c.table[static_cast<size_t>(b) * a.c.stride + pos / a.c.page_size] : -1;
    if (page >= 0 && page < a.c.num_pages)
        dst = static_cast<int64_t>(page) * a.c.Hkv * a.c.page_size + pos % a.c.page_size;
    else if (threadIdx.x % kRow == 0)
        atomicOr(a.err, kErrAppend);
    float4 rope[4];
    if (a.rotate) {
#pragma unroll
        for (int i = 0; i < 4; ++i) rope[i] = rotation(max(pos, 0), a.turns[4 * w + i]);
    }
    for (int h = h0; h < heads; h += kGroups * kAhead) {
        if (h != h0) load(h);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int head = h + kGroups * i, kv = head - a.Hq;        // kv >= 0: a key or value head
            if (head >= heads || (kv < 0 ? a.q_out == nullptr : dst < 0)) continue;
            if (a.rotate && kv < a.c.Hkv) {
                x[i].x = turn(x[i].x, rope[0]);
                x[i].y = turn(x[i].y, rope[1]);
                x[i].z = turn(x[i].z, rope[2]);
                x[i].w = turn(x[i].w, rope[3]);
            }
            uint16_t* to;
            if (kv < 0)
                to = a.q_out + static_cast<size_t>(row) * a.q_out_stride + head * kD;
            else
                to = (kv < a.c.Hkv ? a.c.k : a.c.v) +
                     (dst + static_cast<int64_t>(kv < a.c.Hkv ? kv : kv - a.c.Hkv) * a.c.page_size) * kD;
            reinterpret_cast<uint4*>(to)[w] = x[i];
        }
    }
}

// -------------------------------------------------------------- attention --
//
// An item is the rows of one key/value head's G query heads over 2 * (128 / G)
// consecutive new tokens of one sequence: two tiles of up to 128 (token, head)
// rows, row = token * G + head, so that a key tile is read once for the group.  It
// walks the tiles of 128 keys that any of its rows sees.  The items' key tiles,
// laid end to end, are cut into equal shares, one a block of the persistent
// grid; an item cut by a share's end leaves partial results (maximum, sum,
// unnormalised output in fp32) that a second kernel joins in their order.
//
// Warps: 0-3 and 4-7 the softmax of row tiles 0 and 1 (a thread a row), 8 the MMA
// issuer, 9 and 10 the copies of queries and keys and of values (with pages of 16
// tokens 32 copies a key tile, ~100 cycles each in one warp), 11 what masks do to
// values (below).  Scores S = Q K^T of 128 x 128 go to tensor memory, one thread
// reads its row's 128, takes the maximum and writes the weights as fp16 over the
// scores; O += P V reads them there.  While one row tile's softmax runs, the
// tensor cores work for the other.  An item of at most one row tile gives both softmax groups that tile,
// one the even and one the odd key tiles, and adds the two results at its end.
//
// What bounds it: 8192 tokens of 32 + 8 heads take 363 us at best (six calls in a
// graph), 1.51 PFLOP/s, 0.80 of the measured cuBLAS burst rate, and 393 back to back,
// 1.40 PFLOP/s, 0.83 of cuBLAS's sustained rate (the power limit); the tensor pipe is
// 69 % active.  A group's turn is a chain, softmax ~1500 cycles, values 512, next
// scores 512, and the other group's fills the gaps but for the handovers; leaving
// out the maximum, half of the exponentials or the stores gains 3 to 4 % each.
// Measured slower: one score buffer for both groups and weights apart, the scores
// three turns ahead (393 us against 375); weights handed over in halves of 64 keys
// (390 against 384); weights by the maximum so far while the tile's own is found
// (383 against 363); scores read twice, 32 at a time, in place of 128 registers
// (451 against 376); the warps' walks in shared memory (395 against 388).
//
// The maximum that weights refer to follows the true one only when that is more
// than 2^kLazy above it, so that O in tensor memory is rarely rescaled; weights carry a
// factor 2^kLift and so lie within [0, 2^(kLift + kLazy)] of fp16's range, 2^15 of
// which is still finite.  Those of 2^-(14 + kLift) of the largest are normal numbers,
// those of 2^-(25 + kLift) vanish; the sums take them unrounded.  The two share 15
// bits: 2^11 and 2^4 take 361 us, 2^9 and 2^6 363, 2^8 364, 2^7 369, 2^6 377 (the best
// of 90 runs; at 2^6 one warp in ten rescales every turn, and its group waits).
//
// Values of masked tokens: a weight of 0 times a NaN or an infinity would reach
// rows that do not see the token.  In a tile that is not seen whole by all of the
// item's rows, tokens that no row sees are set to zero in shared memory; if
// another holds a value that is not finite, the item's rows are computed again
// one by one, without the tokens they do not see (attend_row).

constexpr int kThreads = 384;
constexpr int kMmaWarp = 8, kKeyWarp = 9, kValueWarp = 10, kMaskWarp = 11;
// Registers a thread: the softmax groups take over what the other four warps leave
// of the launch's 384 x 168.  (ptxas spills 348 bytes.  The counters of 8192 and of 2048
// tokens put them at the items' ends: a group's turn holds no local store and four
// local loads, all warps together, among 2660 instructions.)
constexpr int kRegsLaunch = 168, kRegsSoftmax = 208, kRegsOther = 80;
static_assert(256 * kRegsSoftmax + 128 * kRegsOther <= kThreads * kRegsLaunch, "registers");
constexpr int kTileBytes = kKeys * kD * 2;         // Q, K and V tiles: two slabs of 64 dims, 128-byte swizzle
constexpr int kSlab = kTileBytes / 2;
constexpr int kStages = 2;                         // of keys, and of values
constexpr float kLift = 6.f, kLazy = 9.f;
constexpr int kItem = 2;                           // an item's own cost, in key tiles
constexpr int kUncut = 4;                          // key tiles of contexts whose items stay whole, whatever their number
constexpr int kMinShare = 4;                       // places of a block's share, at least
static_assert(kMinShare > kItem, "a share holds a tile");
constexpr int kCut = 6;                            // what cutting an item costs, in key tiles

constexpr int kSlotRows = 256;
constexpr size_t kSlotBytes = static_cast<size_t>(kSlotRows) * (kD + 2) * 4 + 256;   // O, m, l, flag
constexpr int kDescInts = 8;

constexpr int kOffQ = 0;
constexpr int kOffRing = 2 * kTileBytes;
constexpr int kOffBars = kOffRing + 2 * kStages * kTileBytes;
constexpr int kOffMl = kOffBars + 256;             // float [2][128]: m, l of group 1 for group 0
constexpr int kOffMisc = kOffMl + 2 * 128 * 4;     // ints
constexpr int kOffSeq = kOffMisc + 176;            // int [5][batch] + 1: first tile, new tokens, length, first row, longest item

size_t prompt_smem_bytes(int batch) { return 1024 + kOffSeq + (5 * static_cast<size_t>(batch) + 1) * 4; }

struct PromptArgs : View {
    Rows rows;
    Paged c;
    const uint16_t* q;
    uint16_t* out;
    int q_stride, out_stride, G;
    int tok;                         // tokens of a row tile, kKeys / G
    float sl2;                       // |scale| * log2(e), not 0
    uint32_t neg;                    // kIdescNegA for a negative scale
    int uncut;                       // shares of whole items
    int wide;                        // output rows are 32-byte aligned (32 prompts of 100 to 500 tokens 77 us; in 16-byte stores 84)
    int stall;                       // test hook: no key or value is copied
    int32_t* desc;                   // [grid][kDescInts] items to join
    uint8_t* slots;                  // [2 * grid] partial results
    uint32_t* err;
};

struct PromptMaps {
    CUtensorMap q, k, v;
};

// One row and query head by one warp, a token at a time, four dimensions a lane: a
// chain of a page id, a row and a reduction, ~0.6 us a token.  A block's 12 warps take
// ~22 rows each of a whole item of 256, a joining block's 8 warps 4 each: 16 tokens
// over 4096 9 ms in place of 28 us, a prompt of 4096 tokens with one infinity 63 ms in
// place of 123 us.
__device__ __noinline__ void attend_row(const PromptArgs& a, int b, int pos, int row, int head)
{
    const int lane = threadIdx.x & 31, h = head / a.G;
    const int cap = a.cap;
    const float sl2 = a.neg ? -a.sl2 : a.sl2;        // the MMA's sign is in its descriptor
    const uint2 qb = *reinterpret_cast<const uint2*>(a.q + static_cast<size_t>(row) * a.q_stride + head * kD + 4 * lane);
    const float2 q0 = __half22float2(*reinterpret_cast<const __half2*>(&qb.x));
    const float2 q1 = __half22float2(*reinterpret_cast<const __half2*>(&qb.y));
    const int32_t* table = a.c.table + static_cast<size_t>(b) * a.c.stride;
    float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f, o2 = 0.f, o3 = 0.f;
    const int end = min(pos, cap - 1);
    if (pos >= cap && lane == 0) atomicOr(a.err, kErrSeqLen);
    const int first = a.window ? window_first(a, pos) : 0;
    for (int t = a.window && a.sinks ? 0 : first; t <= end; ++t) {
        if (t < first && t >= a.sinks) t = first;
        if (t > end) break;
        const int page = table[t / a.c.page_size];
        uint2 kb = make_uint2(0, 0), vb = make_uint2(0, 0);
        if (page >= 0 && page < a.c.num_pages) {
            const size_t at = ((static_cast<size_t>(page) * a.c.Hkv + h) * a.c.page_size + t % a.c.page_size) * kD + 4 * lane;
            kb = *reinterpret_cast<const uint2*>(a.c.k + at);
            vb = *reinterpret_cast<const uint2*>(a.c.v + at);
        } else if (lane == 0) {
            atomicOr(a.err, kErrPageId);
        }
        const float2 k0 = __half22float2(*reinterpret_cast<const __half2*>(&kb.x));
        const float2 k1 = __half22float2(*reinterpret_cast<const __half2*>(&kb.y));
        const float x = warp_sum(fmaf(q0.x, k0.x, q0.y * k0.y) + fmaf(q1.x, k1.x, q1.y * k1.y)) * sl2;
        const float mn = fmaxf(m, x), ms = mn == -INFINITY ? 0.f : mn;
        const float f = exp2f(m - ms), p = exp2f(x - ms);
        m = mn;
        l = fmaf(l, f, p);
        const float2 v0 = __half22float2(*reinterpret_cast<const __half2*>(&vb.x));
        const float2 v1 = __half22float2(*reinterpret_cast<const __half2*>(&vb.y));
        o0 = fmaf(o0, f, p * v0.x);
        o1 = fmaf(o1, f, p * v0.y);
        o2 = fmaf(o2, f, p * v1.x);
        o3 = fmaf(o3, f, p * v1.y);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const __half2 w0 = __floats2half2_rn(o0 * inv, o1 * inv), w1 = __floats2half2_rn(o2 * inv, o3 * inv);
    uint2 w;
    w.x = *reinterpret_cast<const uint32_t*>(&w0);
    w.y = *reinterpret_cast<const uint32_t*>(&w1);
    *reinterpret_cast<uint2*>(a.out + static_cast<size_t>(row) * a.out_stride + head * kD + 4 * lane) = w;
}

// The batch as every block sees it, in shared memory.
struct Seqs {
    const int* pre;          // [batch + 1] key tiles of one head before sequence b
    const int* n;            // new tokens
    const int* len;
    const int* row0;
    const int* uncut;        // shares of whole items
};

// A block's walk over its share [g, end) of the flattened list.  An item takes
// kItem places before its tiles' (what beginning and ending one costs), so that
// shares with many short items are no longer than others.
struct Walk {
    int g, end, b, h, qt, is;      // is: where the present item begins
};

// The places that an item takes in the list.
__device__ __forceinline__ int item_cost(int uncut, const Seen& s) { return uncut ? 1 : kItem + s.tiles; }

struct Piece {
    Seen seen;
    int t0, t1;                    // its tiles
    int b, h, row0, ntok;          // first row of the batch, tokens
    bool first, dual;              // the share's first piece; both groups on one row tile
    __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == seen.tiles; }
};

__device__ __forceinline__ Seen item_seen(const PromptArgs& a, const Seqs& s, int b, int qt, int tt)
{
    const int pf = s.len[b] - s.n[b] + qt * tt;
    return seen_by(a, pf, pf + min(tt, s.n[b] - qt * tt) - 1);
}

__device__ __forceinline__ bool next_piece(const PromptArgs& a, const Seqs& s, int g_begin, Walk& w, Piece& p)
{
    if (w.g >= w.end) return false;
    const int tok = a.tok, tt = 2 * tok;
    const Seen seen = item_seen(a, s, w.b, w.qt, tt);
    const int uncut = *s.uncut;
    const int t0 = uncut ? 0 : max(0, w.g - w.is - kItem), t1 = uncut ? seen.tiles : min(seen.tiles, w.end - w.is - kItem);
    if (t1 <= t0) {                      // the share ends before the item's first tile; p stays the last piece
        w.g = w.end;
        return false;
    }
    p.seen = seen;
    p.t0 = t0;
    p.t1 = t1;
    p.b = w.b;
    p.h = w.h;
    p.row0 = s.row0[w.b] + w.qt * tt;
    p.ntok = min(tt, s.n[w.b] - w.qt * tt);
    p.dual = p.ntok <= tok;
    p.first = w.g == g_begin;
    w.g = uncut ? w.is + 1 : w.is + kItem + p.t1;
    if (p.t1 == p.seen.tiles) {
        w.is = w.g;
        if (++w.qt * tt >= s.n[w.b]) {
            w.qt = 0;
            if (++w.h == a.c.Hkv) {
                w.h = 0;
                do ++w.b;
                while (w.b < a.rows.batch && s.n[w.b] == 0);
            }
        }
    }
    return true;
}

// Where piece-local key tile i of the group's k-th turn lies: group w of a dual
// item takes every other tile.
__device__ __forceinline__ int turns(const Piece& p, int w)
{
    const int nt = p.t1 - p.t0;
    return p.dual ? (nt + 1 - w) / 2 : nt;
}

__device__ __forceinline__ int turn_tile(const Piece& p, int w, int k) { return p.t0 + (p.dual ? 2 * k + w : k); }

struct Ring {
    int slot = 0;
    uint32_t par = 0;
    __device__ __forceinline__ void next()
    {
        if (++slot == kStages) {
            slot = 0;
            par ^= 1u;
        }
    }
};

// The MMAs and the commit by the one thread for which `on` is set, without a branch:
// the warp stays converged, so that operands stay in uniform registers.
__device__ __forceinline__ void mma_ss_if(uint32_t on, uint32_t d, uint64_t ad, uint64_t bd, uint32_t idesc, uint32_t acc)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(ad), "l"(bd), "r"(idesc), "r"(acc), "r"(on)
        : "memory");
}

__device__ __forceinline__ void mma_ts_if(uint32_t on, uint32_t d, uint32_t at, uint64_t bd, uint32_t idesc, uint32_t acc)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(at), "l"(bd), "r"(idesc), "r"(acc), "r"(on)
        : "memory");
}

__device__ __forceinline__ void commit_if(uint32_t on, uint64_t* bar)
{
    asm volatile(
        "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_addr(bar)),
        "r"(on)
        : "memory");
}

// A wait whose usual case, over or soon over, is one instruction and a branch not
// taken.  ok: no wait has given up yet; after one has, none waits.
__device__ __forceinline__ void wait(uint64_t* bar, uint32_t parity, bool& ok, uint32_t* err)
{
    if (__builtin_expect(!mbar_try_wait(bar, parity), 0)) {
        if (ok) ok = mbar_wait(bar, parity, err);
    }
}

// One arrival, by the lanes for which `on` is set, without a branch.
__device__ __forceinline__ void arrive_if(uint32_t on, uint64_t* bar)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t@q mbarrier.arrive.shared::cta.b64 _, [%0];\n\t}" ::"r"(smem_addr(bar)),
                 "r"(on)
                 : "memory");
}

// Values read from tensor memory are used from here on, not before: the wait names
// no registers, so the uses would not be ordered behind it.
template <int N>
__device__ __forceinline__ void pin(uint32_t* v)
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+r"(v[i]));
}

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

__device__ __forceinline__ uint64_t pair(float lo, float hi)
{
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
    return d;
}

__device__ __forceinline__ void unpair(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }

__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}

__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

__device__ __forceinline__ uint32_t half2_bits(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ __half2 as_half2(uint32_t v) { return *reinterpret_cast<const __half2*>(&v); }

// Whether either of the two is an infinity or a NaN (exponent all ones).
__device__ __forceinline__ bool not_finite(__half2 v)
{
    const uint32_t x = *reinterpret_cast<const uint32_t*>(&v);
    return (x & 0x7C00u) == 0x7C00u || (x & 0x7C000000u) == 0x7C000000u;
}

// 32 bytes by one thread (p 32-byte aligned).
__device__ __forceinline__ void store32(void* p, const uint32_t v[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
                 "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}

// Four blocks of N words by each of four lanes, transposed: lane j's k-th becomes
// lane k's j-th.
template <int N>
__device__ __forceinline__ void turn_quads(uint32_t* v, int lane)
{
#pragma unroll
    for (int s = 1; s < 4; s *= 2) {
        const bool upper = lane & s;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            if (b & s) continue;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                uint32_t &lo = v[b * N + i], &hi = v[(b + s) * N + i];
                const uint32_t got = __shfl_xor_sync(0xffffffffu, upper ? lo : hi, s);
                lo = upper ? got : lo;
                hi = upper ? hi : got;
            }
        }
    }
}

__device__ __forceinline__ int* slot_flag(const PromptArgs& a, int slot)
{
    return reinterpret_cast<int*>(a.slots + static_cast<size_t>(slot) * kSlotBytes + static_cast<size_t>(kSlotRows) * (kD + 2) * 4);
}

__global__ void __launch_bounds__(kThreads, 1)
    prompt_attn_kernel(const __grid_constant__ PromptMaps maps, const __grid_constant__ PromptArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t* kfull = reinterpret_cast<uint64_t*>(smem + kOffBars);  // key tile landed
    uint64_t* kempty = kfull + kStages;                              // ... read by its MMAs
    uint64_t* vfull = kempty + kStages;
    uint64_t* vempty = vfull + kStages;
    uint64_t* fixed = vempty + kStages;                              // value tile looked over
    uint64_t* qfull = fixed + kStages;
    uint64_t* qempty = qfull + 2;
    uint64_t* sfull = qempty + 2;                                    // scores of a row tile written
    uint64_t* pfull = sfull + 2;                                     // ... weights
    uint64_t* ofull = pfull + 2;                                     // ... output of a piece
    uint64_t* drain = ofull + 2;
    float* ml = reinterpret_cast<float*>(smem + kOffMl);
    volatile int* misc = reinterpret_cast<volatile int*>(smem + kOffMisc);   // [0..5] walk, [6] tmem, [7] share, [40] whole items
    uint32_t* again = reinterpret_cast<uint32_t*>(smem + kOffMisc + 32);     // a bit a piece (modulo 1024) whose rows are computed again
    int* seq = reinterpret_cast<int*>(smem + kOffSeq);
    const int batch = a.rows.batch;
    int* pre = seq;
    int* sn = pre + batch + 1;
    int* slen = sn + batch;
    int* srow = slen + batch;
    int* smost = srow + batch;
    const Seqs S = {pre, sn, slen, srow, const_cast<const int*>(misc) + 40};
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cap = a.cap;
    const int tok = a.tok, tt = 2 * tok;
    uint32_t* err = a.err;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&kfull[i], 1);
            mbar_init(&kempty[i], 1);
            mbar_init(&vfull[i], 1);
            mbar_init(&vempty[i], 1);
            mbar_init(&fixed[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&qfull[i], 1);
            mbar_init(&qempty[i], 1);
            mbar_init(&sfull[i], 1);
            mbar_init(&pfull[i], 4);
            mbar_init(&ofull[i], 1);
        }
        mbar_init(drain, 1);
        mbar_fence_init();
    }
    if (threadIdx.x < 32) again[threadIdx.x] = 0;
    if (warp == kKeyWarp && lane == 0) {
        tc::prefetch_map(&maps.q);
        tc::prefetch_map(&maps.k);
        tc::prefetch_map(&maps.v);
    }
    if (warp == kMmaWarp) tc::tmem_alloc(const_cast<uint32_t*>(reinterpret_cast<volatile uint32_t*>(misc + 6)), 512);
    grid_dependency_wait();              // every input may come from the previous kernel
    grid_dependents_launch();

    // the sequences' rows, lengths and key tiles; their prefix
    bool unordered = false;
    for (int b = warp; b < batch; b += kThreads / 32) {
        const int begin = a.rows.starts[b], end = a.rows.starts[b + 1];
        const int s = min(max(begin, 0), a.rows.rows), n = min(max(end, s), a.rows.rows) - s;
        unordered |= end < begin;
        const int L = max(a.rows.lens[b], 0);
        if (lane == 0) {
            sn[b] = n;
            slen[b] = L;
            srow[b] = s;
            if (n > 0 && L > cap && blockIdx.x == 0) atomicOr(err, kErrSeqLen);
        }
        __syncwarp();
        int cost = 0, most = 0;
        for (int qt = lane; qt * tt < n; qt += 32) {
            const int c = item_cost(a.uncut, item_seen(a, S, b, qt, tt));
            cost += c;
            most = max(most, c);
        }
        cost = __reduce_add_sync(0xffffffffu, cost);
        most = __reduce_max_sync(0xffffffffu, most);
        if (lane == 0) {
            pre[b] = cost;
            smost[b] = most;
        }
    }
    // Starts that go down may own rows twice, and more places than an int counts (the
    // host has checked that others do not): no block has any then.
    unordered = __syncthreads_or(unordered) != 0;
    if (unordered && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(err, kErrSeqLen);
    if (warp == 0) {
        // An item a block, whole, where they fill a quarter of the blocks or more and the
        // longest is not much longer than a fair share and what a cut costs (parts written
        // and joined): 1000 tokens of 8 groups of 4 heads 23 us whole, 27 cut, twice 500
        // over 1000 30 and 35; but 16 over 1000, 8 items, 16.5 whole, 14.2 cut.
        bool few = false;
        if (!a.uncut) {
            int sum = 0, items = 0, most = 0;
            for (int b = lane; b < batch; b += 32) {
                sum += pre[b];
                items += (sn[b] + tt - 1) / tt;
                most = max(most, smost[b]);
            }
            sum = __reduce_add_sync(0xffffffffu, sum);
            items = __reduce_add_sync(0xffffffffu, items);
            most = __reduce_max_sync(0xffffffffu, most);
            const int blocks = static_cast<int>(gridDim.x);
            const int64_t all = static_cast<int64_t>(items) * a.c.Hkv;
            few = all <= blocks && 4 * all >= blocks && most <= max(a.c.Hkv * sum / blocks, kMinShare) + kCut;
        }
        const int uncut = a.uncut || few ? 1 : 0;
        __syncwarp();
        int carry = 0;
        for (int b0 = 0; b0 < batch; b0 += 32) {
            const int v = b0 + lane < batch ? (few ? (sn[b0 + lane] + tt - 1) / tt : pre[b0 + lane]) : 0;
            int incl = v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int u = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += u;
            }
            if (b0 + lane < batch) pre[b0 + lane] = carry + incl - v;
            carry += __shfl_sync(0xffffffffu, incl, 31);
        }
        if (lane == 0) pre[batch] = carry;
        __syncwarp();
        const int total = unordered ? 0 : a.c.Hkv * carry, grid = static_cast<int>(gridDim.x);
        const int R = max((total + grid - 1) / grid, uncut ? 1 : kMinShare);
        const int g = min(static_cast<int64_t>(total), static_cast<int64_t>(blockIdx.x) * R);
        if (g < total) {
            int lo = 0, hi = batch - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (a.c.Hkv * pre[mid] <= g) lo = mid;
                else hi = mid - 1;
            }
            const int of_head = pre[lo + 1] - pre[lo];
            const int h = (g - a.c.Hkv * pre[lo]) / of_head;
            int at = a.c.Hkv * pre[lo] + h * of_head, qt = 0;
            for (int q0 = 0;; q0 += 32) {       // ends: g lies within this head's tiles
                const int v = (q0 + lane) * tt < sn[lo] ? item_cost(uncut, item_seen(a, S, lo, q0 + lane, tt)) : 0;
                int incl = v;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int u = __shfl_up_sync(0xffffffffu, incl, o);
                    if (lane >= o) incl += u;
                }
                const uint32_t past = __ballot_sync(0xffffffffu, at + incl > g);
                if (past || (q0 + 32) * tt >= sn[lo]) {
                    const int l = past ? __ffs(past) - 1 : 31;
                    qt = q0 + l;
                    at += __shfl_sync(0xffffffffu, incl - v, l);
                    break;
                }
                at += __shfl_sync(0xffffffffu, incl, 31);
            }
            if (lane == 0) {
                misc[2] = lo;
                misc[3] = h;
                misc[4] = qt;
                misc[5] = at;
            }
        }
        if (lane == 0) {
            misc[0] = g;
            misc[1] = min(static_cast<int64_t>(total), static_cast<int64_t>(g) + R);
            misc[7] = R;
            misc[40] = uncut;
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const int g_begin = misc[0];
    Walk walk = {g_begin, misc[1], misc[2], misc[3], misc[4], misc[5]};
    const int R = misc[7];
    int32_t* desc = a.desc + static_cast<size_t>(blockIdx.x) * kDescInts;
    const uint32_t tbase = static_cast<uint32_t>(misc[6]);
    if (walk.g >= walk.end) {            // more blocks than shares
        if (threadIdx.x == 0) desc[0] = 0;
        if (warp == kMmaWarp) tc::tmem_dealloc(tbase, 512);
        return;
    }
    // tensor memory: scores (and weights over them) of row tile w at 128 w, output at 256 + 128 w

    // After a wait gave up (bounded, flagged) a role waits no more but goes on
    // through every tile with every arrival, so that no other is left behind; the
    // copies stop and are waited for.
    Piece p;
    if (warp >= kMmaWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
        if (warp == kKeyWarp || warp == kValueWarp) {
            // ------------------------------------------------------------ copies
            const bool keys = warp == kKeyWarp;
            uint64_t* const full = keys ? kfull : vfull;
            uint64_t* const empty = keys ? kempty : vempty;
            uint8_t* const tiles = smem + kOffRing + (keys ? 0 : kStages * kTileBytes);
            const CUtensorMap* const map = keys ? &maps.k : &maps.v;
            Ring ring;
            int issued = 0, nq[2] = {0, 0};
            bool ok = true;
            const int boxes = kKeys / a.box;
            const uint32_t qbytes = static_cast<uint32_t>(a.G * tok) * 128u * 2u;
            // A lane a box and half.  Boxes behind the last token, or on a page outside the
            // pool, lie wholly outside the tensor: the copy reads zeros.  The next tile's
            // page ids are under way while this one's copies are issued (nothing is asked of them before).
            auto token = [&](int i) { return p.seen.token(i * kKeys + (lane >> 1) * a.box); };
            auto lookup = [&](const int32_t* table, int i) {
                int page = 0;
                if (lane < 2 * boxes && token(i) <= p.seen.pl) page = table[token(i) / a.c.page_size];
                return page;
            };
            auto tile = [&](int y) {
                if (issued >= kStages && ok) ok = mbar_wait(&empty[ring.slot], ring.par ^ 1u, err);
                if (!ok) return;
                uint8_t* dst = tiles + ring.slot * kTileBytes;
                if (lane == 0) mbar_arrive_expect_tx(&full[ring.slot], kTileBytes);
                __syncwarp();
                if (lane < 2 * boxes)
                    tc::tma_load_2d(dst + (lane & 1) * kSlab + (lane >> 1) * a.box * 128, map, 64 * (lane & 1), y, &full[ring.slot]);
                ++issued;
                ring.next();
            };
            while (ok && a.stall == 0) {
                if (!next_piece(a, S, g_begin, walk, p)) break;
                const int32_t* table = a.c.table + static_cast<size_t>(p.b) * a.c.stride;
                int page = lookup(table, p.t0);
                for (int i = p.t0; i < p.t1 && ok; ++i) {
                    const int next = i + 1 < p.t1 ? lookup(table, i + 1) : 0;
                    int y = -a.box;
                    if (lane < 2 * boxes && token(i) <= p.seen.pl) {
                        if (page >= 0 && page < a.c.num_pages)
                            y = (page * a.c.Hkv + p.h) * a.c.page_size + token(i) % a.c.page_size;
                        else
                            atomicOr(err, kErrPageId);
                    }
                    page = next;
                    tile(y);
                    if (keys && i == p.t0)
                        for (int w = 0; w < (p.dual ? 1 : 2) && ok; ++w) {
                            if (nq[w] >= 1) ok = mbar_wait(&qempty[w], (nq[w] - 1) & 1, err);
                            if (!ok) break;
                            if (lane == 0) {
                                mbar_arrive_expect_tx(&qfull[w], qbytes);
                                for (int s = 0; s < 2; ++s)
                                    tc::tma_load_3d(smem + kOffQ + w * kTileBytes + s * kSlab, &maps.q, 64 * s, p.h * a.G, p.row0 + w * tok,
                                                    &qfull[w]);
                            }
                            ++nq[w];
                        }
                }
            }
            // every copy issued has landed before the block's memory goes away
            for (int i = max(0, issued - kStages); i < issued; ++i) mbar_wait(&full[i % kStages], (i / kStages) & 1, err);
            for (int w = 0; w < 2; ++w)
                if (nq[w]) mbar_wait(&qfull[w], (nq[w] - 1) & 1, err);
        } else if (warp == kMmaWarp) {
            // -------------------------------------------------------- MMA issuer
            // The groups take turns at the key tiles; a group's next scores are issued
            // behind its weights x values, whose weights they overwrite (MMAs run in
            // the order of issue).  An MMA of 128 x 128 x 16 takes 64 cycles and the queue
            // holds about two, so the loop must not lose time: its numbers come through a
            // shuffle, warp-uniform for the compiler too, and MMAs are predicated rather
            // than branched to, or their operands pass through vector registers (8192
            // tokens of 32 heads 724 us with a branch and a search for each turn's kind).
            // One copy of the turn's code serves both groups, both kinds of items and their
            // ends: with one for each (18) 8192 tokens took 1 % less, but short items, where
            // the roles' code passes through the instruction cache all the time, more: 32
            // prompts of 100 to 500 tokens 82.5 us against 77.3, 8 of 500 to 1500 96.3 and
            // 94.5.
            const uint32_t idesc_s = tc::idesc_f16_f32(128, kKeys) | a.neg;
            const uint32_t idesc_o = tc::idesc_f16_f32(128, kD) | kIdescTransB;
            const uint32_t tb = __shfl_sync(0xffffffffu, tbase, 0);
            const uint32_t leader = tc::elect_one() ? 1u : 0u;
            const uint64_t qdesc = tc::sw128_kmajor_desc(smem_addr(smem + kOffQ));
            const uint64_t kdesc = tc::sw128_kmajor_desc(smem_addr(smem + kOffRing));
            const uint64_t vdesc = sw128_mnmajor_desc(smem_addr(smem + kOffRing + kStages * kTileBytes), kSlab);
            Ring kr, vr;                     // the next key tile, the next value tile
            uint32_t qpar = 0, ppar = 0;     // parities, a bit a group
            bool ok = true;
            struct Turns {
                int nt;                      // tiles of the piece
                bool dual;
                __device__ __forceinline__ int count() const { return dual ? nt : 2 * nt; }
            };
            auto fetch = [&](Turns& x) {
                const int more = next_piece(a, S, g_begin, walk, p) ? 1 : 0;
                if (!__shfl_sync(0xffffffffu, more, 0)) return false;
                x.nt = __shfl_sync(0xffffffffu, p.t1 - p.t0, 0);
                x.dual = __shfl_sync(0xffffffffu, p.dual ? 1 : 0, 0) != 0;
                return true;
            };
            // Turn u of a piece is group u & 1's.  Behind its values come the group's next
            // scores, those of turn u + 2 or, where the groups end in their order, of the next
            // piece's first turns; so its softmax finds them when its output is stored.
            // Turns -2 and -1 are the first scores alone.
            Turns x, after;
            bool have = fetch(x), begun = false, more = false;
            while (have) {
                const int turns = x.count();
#pragma unroll 1
                for (int u = begun ? 0 : -2; u < turns; ++u) {
                    const int w = __shfl_sync(0xffffffffu, u & 1, 0);
                    if (u == 0) more = fetch(after);
                    // all that the scores need is known before the wait for the weights
                    const bool here = u + 2 < turns;
                    const int v = here ? u + 2 : w, nt = here ? x.nt : after.nt;
                    const bool dual = here ? x.dual : after.dual;
                    const bool next = (here || (more && !x.dual)) && !(dual && v >= nt);
                    const bool new_q = v < 2 && (w == 0 || !dual), last_q = (dual ? v : v >> 1) + 1 == nt;
                    const bool new_k = w == 0 || dual, last_k = w == 1 || dual;
                    const uint64_t qd = qdesc + (new_k ? 0u : kTileBytes >> 4);
                    const uint64_t kd = kdesc + kr.slot * (kTileBytes >> 4);
                    if (u >= 0) {
                        if (w == 0 || x.dual) wait(&fixed[vr.slot], vr.par, ok, err);
                        wait(&pfull[w], (ppar >> w) & 1u, ok, err);
                        ppar ^= 1u << w;
                        tc::fence_after_sync();
                        const uint64_t vd = vdesc + vr.slot * (kTileBytes >> 4);
#pragma unroll
                        for (int s = 0; s < 8; ++s)
                            mma_ts_if(leader, tb + 256 + 128 * w, tb + 128 * w + 8 * s, vd + s * (2048 >> 4), idesc_o, s > 0 || u >= 2 ? 1u : 0u);
                        if (u + 2 >= turns) commit_if(leader, &ofull[w]);
                        if (w == 1 || x.dual) {
                            commit_if(leader, &vempty[vr.slot]);
                            vr.next();
                        }
                    }
                    if (!next) continue;
                    if (new_q) {
                        wait(&qfull[w], (qpar >> w) & 1u, ok, err);
                        qpar ^= 1u << w;
                    }
                    if (new_k) wait(&kfull[kr.slot], kr.par, ok, err);
                    tc::fence_after_sync();
#pragma unroll
                    for (int s = 0; s < 8; ++s) {
                        const uint64_t step = (s >> 2) * (kSlab >> 4) + (s & 3) * 2;
                        mma_ss_if(leader, tb + 128 * w, qd + step, kd + step, idesc_s, s > 0 ? 1u : 0u);
                    }
                    commit_if(leader, &sfull[w]);
                    if (last_k) {
                        commit_if(leader, &kempty[kr.slot]);
                        kr.next();
                    }
                    if (last_q) commit_if(leader, &qempty[dual ? 0 : w]);
                }
                begun = more && !x.dual;
                x = after;
                have = more;
            }
            commit_if(leader, drain);   // all MMAs have completed before tensor memory is released
            mbar_wait(drain, 0, err);
        } else if (warp == kMaskWarp) {
            // ---------------------------------------------------- masked values
            Ring vr;
            bool ok = true;
            for (int piece = 0; next_piece(a, S, g_begin, walk, p); ++piece) {
                for (int i = p.t0; i < p.t1; ++i) {
                    if (ok) ok = mbar_wait(&vfull[vr.slot], vr.par, err);
                    __syncwarp();
                    const int last = p.seen.pf + p.ntok - 1;
                    if (!sees_all(a, i, p.seen.front, p.seen.gap, p.seen.pf, last, p.seen.pl)) {
                        uint8_t* base = smem + kOffRing + (kStages + vr.slot) * kTileBytes + ((lane >> 3) & 1) * kSlab + (lane & 7) * 16;
                        __half2 big = __float2half2_rn(0.f);
                        auto clip = [&](int x) { return min(max(x - i * kKeys, 0), kKeys); };
                        // places [from, to) of the list, as far as they lie in the tile: 16 lanes a row
                        auto zero = [&](int from, int to) {
                            for (int r = clip(from) + (lane >> 4); r < clip(to); r += 2)
                                *reinterpret_cast<uint4*>(base + r * 128) = make_uint4(0, 0, 0, 0);
                        };
                        auto look = [&](int from, int to) {        // the largest size, NaN above all
                            const int f = clip(from), e = clip(to);
                            for (int r = f + (lane >> 4); r - (lane >> 4) < e; r += 16) {
                                uint4 x[8];
#pragma unroll
                                for (int j = 0; j < 8; ++j) x[j] = *reinterpret_cast<const uint4*>(base + min(r + 2 * j, e - 1) * 128);
#pragma unroll
                                for (int j = 0; j < 8; ++j) {
                                    big = __hmax2_nan(big, __hmax2_nan(__habs2(as_half2(x[j].x)), __habs2(as_half2(x[j].y))));
                                    big = __hmax2_nan(big, __hmax2_nan(__habs2(as_half2(x[j].z)), __habs2(as_half2(x[j].w))));
                                }
                            }
                        };
                        hidden_places(a, p.seen, last, zero, look);
                        if (__any_sync(0xffffffffu, not_finite(big)) && lane == 0) atomicOr(&again[(piece >> 5) & 31], 1u << (piece & 31));
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                    }
                    if (lane == 0) mbar_arrive(&fixed[vr.slot]);
                    vr.next();
                }
            }
            // the item that this share's end cuts, and does not begin in an earlier one: who joins it finds it here
            if (lane == 0) {
                const bool head = p.t0 == 0 && !p.whole();
                desc[0] = head ? (walk.is + kItem + p.seen.tiles - 1) / R - static_cast<int>(blockIdx.x) + 1 : 0;
                desc[1] = p.b;
                desc[2] = p.h;
                desc[3] = p.row0;
                desc[4] = p.ntok;
                desc[5] = p.seen.pf;
                desc[6] = 2 * static_cast<int>(blockIdx.x) + (p.first ? 0 : 1);
                for (int i = 0; i < 2; ++i) *slot_flag(a, 2 * blockIdx.x + i) = 0;
            }
        }
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsLaunch));
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
        // ------------------------------------------------------------ softmax
        const int w = warp >> 2, row = 32 * (warp & 3) + lane;
        const uint32_t lanes = static_cast<uint32_t>(32 * (warp & 3)) << 16;
        const uint32_t ts = tbase + 128 * w + lanes, to = tbase + 256 + 128 * w + lanes;
        const int rtok = row / a.G, rhead = row - rtok * a.G;
        uint32_t spar = 0, opar = 0;
        bool ok = true;
        for (bool more = next_piece(a, S, g_begin, walk, p); more;) {
            const int base = p.dual ? 0 : w * tok;            // first token of the group's row tile
            const int pos = p.seen.pf + base + min(rtok, p.ntok - base - 1);      // (rows behind the last token: its)
            const int pf = p.seen.pf + base, pl = pf + min(tok, p.ntok - base) - 1;
            const int nk = turns(p, w);
            float m = -INFINITY;
            uint64_t l2 = pair(0.f, 0.f);
            for (int k = 0; k < nk; ++k) {
                wait(&sfull[w], spar, ok, err);
                spar ^= 1u;
                __syncwarp();
                tc::fence_after_sync();
                uint32_t s[128];
#pragma unroll
                for (int c = 0; c < 4; ++c) ld32(ts + 32 * c, s + 32 * c);
                tc::ld_wait();
                pin<128>(s);
                const int i = turn_tile(p, w, k);
                if (!sees_all(a, i, p.seen.front, p.seen.gap, pf, pl, p.seen.pl)) {
                    const RowMask mask = row_mask(a, p.seen, i, pos);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const uint32_t see = mask.word(c);
                        if (__all_sync(0xffffffffu, see == 0xFFFFFFFFu)) continue;       // most: a tile has one edge or two
#pragma unroll
                        for (int i = 0; i < 32; ++i) s[32 * c + i] = see & (1u << i) ? s[32 * c + i] : 0xFF800000u;   // -infinity
                    }
                }
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < 128; c += 8)
#pragma unroll
                    for (int i = 0; i < 4; ++i) mx[i] = max3(mx[i], __uint_as_float(s[c + 2 * i]), __uint_as_float(s[c + 2 * i + 1]));
                const float mnew = max3(fmaxf(mx[0], mx[1]), mx[2], mx[3]) * a.sl2;
                const bool up = mnew > m + kLazy;
                const float mref = up ? mnew : m;
                const float ms = mref == -INFINITY ? 0.f : mref;
                const float alpha = up ? ex2(m - ms) : 1.f;
                m = mref;
                const uint64_t sl = pair(a.sl2, a.sl2), off = pair(kLift - ms, kLift - ms);
                uint32_t pk[64];
                uint64_t sum[2] = {pair(0.f, 0.f), pair(0.f, 0.f)};
#pragma unroll
                for (int c = 0; c < 64; ++c) {
                    const uint64_t x = fma2(pair(__uint_as_float(s[2 * c]), __uint_as_float(s[2 * c + 1])), sl, off);
                    float x0, x1;
                    unpair(x, x0, x1);
                    x0 = ex2(x0);
                    x1 = ex2(x1);
                    sum[c & 1] = add2(sum[c & 1], pair(x0, x1));
                    pk[c] = half2_bits(x0, x1);
                }
                l2 = fma2(l2, pair(alpha, alpha), add2(sum[0], sum[1]));
                st32(ts, pk);
                st32(ts + 32, pk + 32);
                if (k > 0 && __any_sync(0xffffffffu, up)) {
#pragma unroll 1
                    for (int c = 0; c < 4; ++c) {
                        uint32_t o[32];
                        ld32(to + 32 * c, o);
                        tc::ld_wait();
                        pin<32>(o);
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                        st32(to + 32 * c, o);
                    }
                }
                tc::st_wait();
                tc::fence_before_sync();
                __syncwarp();
                arrive_if(lane == 0, &pfull[w]);
            }
            float l, lh;
            unpair(l2, l, lh);
            l += lh;
            Piece after;                     // found while the last values are added (later: 8192 tokens 2 % more)
            more = next_piece(a, S, g_begin, walk, after);
            if (nk > 0) {
                wait(&ofull[w], opar, ok, err);
                opar ^= 1u;
                __syncwarp();
                tc::fence_after_sync();
            }
            // factors of this group's output and, in a dual item, of the other's (same lanes)
            float f0 = 1.f, f1 = 0.f;
            const bool joined = p.dual && turns(p, 1) > 0;
            if (joined) {
                if (w == 1) {
                    ml[row] = m;
                    ml[128 + row] = l;
                }
                named_barrier_sync(1, 256);
                if (w == 0) {
                    const float m1 = ml[row], M = fmaxf(m, m1), Ms = M == -INFINITY ? 0.f : M;
                    f0 = ex2(m - Ms);
                    f1 = ex2(m1 - Ms);
                    l = l * f0 + ml[128 + row] * f1;
                    m = M;
                }
            }
            if (!p.dual || w == 0) {
                const bool valid = rtok < tok && base + rtok < p.ntok;
                const float inv = l == 0.f ? 0.f : 1.f / l;
                if (p.whole()) {
                    f0 *= inv;
                    f1 *= inv;
                }
                const int slot = 2 * static_cast<int>(blockIdx.x) + (p.first ? 0 : 1);
                uint8_t* part = a.slots + static_cast<size_t>(slot) * kSlotBytes;
                uint16_t* orow = a.out + static_cast<size_t>(p.row0 + base + (valid ? rtok : 0)) * a.out_stride +
                                 static_cast<size_t>(p.h * a.G + rhead) * kD;
                const int prow = w * 128 + row;
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint32_t o[32];
                    ld32(to + 32 * c, o);
                    if (joined) {
                        uint32_t o1[32];
                        ld32(to + 128 + 32 * c, o1);
                        tc::ld_wait();
                        pin<32>(o);
                        pin<32>(o1);
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            o[i] = __float_as_uint(__uint_as_float(o[i]) * f0 + __uint_as_float(o1[i]) * f1);
                    } else {
                        tc::ld_wait();
                        pin<32>(o);
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f0);
                    }
                    if (p.whole()) {
                        uint32_t v[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[i] = half2_bits(__uint_as_float(o[2 * i]), __uint_as_float(o[2 * i + 1]));
                        if (valid && a.wide) {
                            store32(orow + 32 * c, v);
                            store32(orow + 32 * c + 16, v + 8);
                        } else if (valid) {
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                reinterpret_cast<uint4*>(orow)[4 * c + i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                        }
                    } else if (valid) {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            reinterpret_cast<uint4*>(part)[(8 * c + i) * kSlotRows + prow] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                    }
                }
                if (!p.whole()) {
                    float* mlp = reinterpret_cast<float*>(part + static_cast<size_t>(kSlotRows) * kD * 4);
                    mlp[prow] = m;
                    mlp[kSlotRows + prow] = l;
                }
            }
            if (joined) named_barrier_sync(1, 256);      // group 1's output and m, l are read
            tc::fence_before_sync();
            p = after;
        }
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsLaunch));
    }

    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    if (warp == kMmaWarp) tc::tmem_dealloc(tbase, 512);

    // Rows beside masked values that are not finite, once more: not inside the
    // pipeline, whose waits are bounded.  (A piece that shares its bit with such a
    // one is computed again as well, to the same effect.)
    uint32_t some = again[lane];
    if (!__any_sync(0xffffffffu, some != 0u)) return;
    walk = {g_begin, misc[1], misc[2], misc[3], misc[4], misc[5]};
    for (int piece = 0; next_piece(a, S, g_begin, walk, p); ++piece) {
        if (!(again[(piece >> 5) & 31] >> (piece & 31) & 1u)) continue;
        if (!p.whole()) {
            if (threadIdx.x == 0) *slot_flag(a, 2 * static_cast<int>(blockIdx.x) + (p.first ? 0 : 1)) = 1;   // left to who joins it
            continue;
        }
        for (int i = warp; i < p.ntok * a.G; i += kThreads / 32) {
            const int t = i / a.G;
            attend_row(a, p.b, p.seen.pf + t, p.row0 + t, p.h * a.G + i - t * a.G);
        }
    }
}

// Joins the parts of the items that shares cut, in their order: a block 32 rows
// of one item, a lane a row, a warp 4 kChunks dimensions (gridDim.z blocks for
// all).  Many items are cut in two or three parts each (kChunks = 4: few blocks),
// few items in many (kChunks = 1, the loads of eight parts at once: 16 tokens over
// 32768 39.5 us in all, with four chunks 44.5; 8192 tokens 375 with four, 382 with
// one).
constexpr int kMaxGrid = 256;

template <int kChunks>
__global__ void __launch_bounds__(256) prompt_join_kernel(const PromptArgs a)
{
    __shared__ float sm[8][32], sl[8][32];
    __shared__ __align__(8) uint16_t tile[32][32 * kChunks + 4];
    grid_dependency_wait();
    grid_dependents_launch();
    const int32_t* desc = a.desc + static_cast<size_t>(blockIdx.x) * kDescInts;
    const int parts = __ldcg(desc);
    if (parts < 2) return;
    const int b = __ldcg(desc + 1), h = __ldcg(desc + 2), row0 = __ldcg(desc + 3), ntok = __ldcg(desc + 4), pf = __ldcg(desc + 5);
    const int slot0 = __ldcg(desc + 6), slot1 = 2 * static_cast<int>(blockIdx.x) + 2;    // the following ones: 2 apart
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int tok = a.tok;
    auto place = [&](int r, int& token) {          // row of the item -> its token; whether there is one
        const int rt = (r & 127) / a.G;
        token = (r >> 7) * tok + rt;
        return rt < tok && token < ntok;
    };
    const int r0 = 32 * blockIdx.y;
    int token;
    const bool valid = place(r0 + lane, token);
    if (!__syncthreads_or(valid)) return;
    auto part = [&](int i) { return a.slots + static_cast<size_t>(i == 0 ? slot0 : slot1 + 2 * (i - 1)) * kSlotBytes; };
    auto stats = [&](int i) { return reinterpret_cast<const float*>(part(i) + static_cast<size_t>(kSlotRows) * kD * 4); };
    int slow = 0;
    float M = -INFINITY, L = 0.f;
    for (int i = warp; i < parts; i += 8) {
        const float m = valid ? __ldcg(stats(i) + r0 + lane) : 0.f, l = valid ? __ldcg(stats(i) + kSlotRows + r0 + lane) : 0.f;
        slow |= __ldcg(slot_flag(a, i == 0 ? slot0 : slot1 + 2 * (i - 1)));
        const float Mn = fmaxf(M, m), Ms = Mn == -INFINITY ? 0.f : Mn;
        L = L * ex2(M - Ms) + l * ex2(m - Ms);
        M = Mn;
    }
    sm[warp][lane] = M;
    sl[warp][lane] = L;
    if (__syncthreads_or(slow)) {
        for (int i = 4 * warp; i < 4 * warp + 4 && blockIdx.z == 0; ++i) {
            const int r = r0 + i;
            int t;
            if (place(r, t)) attend_row(a, b, pf + t, row0 + t, h * a.G + (r & 127) % a.G);
        }
        return;
    }
    M = -INFINITY;
    L = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) M = fmaxf(M, sm[w][lane]);
    const float Ms = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int w = 0; w < 8; ++w) L = fmaf(sl[w][lane], ex2(sm[w][lane] - Ms), L);
    float4 acc[kChunks] = {};
#pragma unroll (8 / kChunks)
    for (int i = 0; i < parts; ++i) {
        const float f = valid ? ex2(__ldcg(stats(i) + r0 + lane) - Ms) : 0.f;
        const float4* o = reinterpret_cast<const float4*>(part(i)) + kChunks * (8 * blockIdx.z + warp) * kSlotRows + r0 + lane;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const float4 v = valid ? __ldcg(o + c * kSlotRows) : make_float4(0.f, 0.f, 0.f, 0.f);
            acc[c].x = fmaf(v.x, f, acc[c].x);
            acc[c].y = fmaf(v.y, f, acc[c].y);
            acc[c].z = fmaf(v.z, f, acc[c].z);
            acc[c].w = fmaf(v.w, f, acc[c].w);
        }
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
        *reinterpret_cast<uint2*>(&tile[lane][4 * (kChunks * warp + c)]) =
            make_uint2(half2_bits(acc[c].x * inv, acc[c].y * inv), half2_bits(acc[c].z * inv, acc[c].w * inv));
    __syncthreads();
    for (int e = threadIdx.x; e < 32 * 8 * kChunks; e += 256) {
        const int i = e / (8 * kChunks), c = e % (8 * kChunks), r = r0 + i;
        int t;
        if (place(r, t))
            reinterpret_cast<uint2*>(a.out + static_cast<size_t>(row0 + t) * a.out_stride + (h * a.G + (r & 127) % a.G) * kD +
                                     32 * kChunks * blockIdx.z)[c] = *reinterpret_cast<const uint2*>(&tile[i][4 * c]);
    }
}

// ------------------------------------------------------------------- host --

// What append and attention ask of the cache and the rows alike.
int check_rows(const wq4_kv_cache* c, const int32_t* row_starts, const int32_t* seq_lens, int batch, int rows, int n_q_heads,
               Rows* R, Paged* P)
{
    if (!c || !c->k || !c->v || !c->page_table || c->num_pages < 1 || c->n_kv_heads < 1 || c->page_size < 16 ||
        c->page_size % 16 || c->page_table_stride < 1 || c->head_dim < 1 || !row_starts || !seq_lens || batch < 1 ||
        batch > WQ4_ATTN_MAX_BATCH || rows < 1)
        return WQ4_ERR_INVALID;
    if (n_q_heads < c->n_kv_heads || n_q_heads % c->n_kv_heads) return WQ4_ERR_INVALID;
    if (c->head_dim != kD || n_q_heads / c->n_kv_heads > kMaxGroup || n_q_heads > kMaxHeads) return WQ4_ERR_UNSUPPORTED;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->page_table, 4) || !aligned(row_starts, 4) ||
        !aligned(seq_lens, 4))
        return WQ4_ERR_ALIGN;
    if (cache_rows(*c) < 0 || static_cast<int64_t>(c->page_table_stride) * c->page_size >= (int64_t(1) << 30) || rows >= (1 << 30))
        return WQ4_ERR_UNSUPPORTED;
    *R = {row_starts, seq_lens, batch, rows};
    *P = {c->k, c->v, c->page_table, c->page_table_stride, c->page_size, c->num_pages, c->n_kv_heads};
    return WQ4_OK;
}

size_t cache_bytes(const wq4_kv_cache* c)
{
    return static_cast<size_t>(c->num_pages) * c->n_kv_heads * c->page_size * kD * 2;
}

// Bytes from the first row's start to the last one's end.
size_t rows_bytes(int rows, int stride, int width)
{
    return (static_cast<size_t>(rows - 1) * stride + width) * 2;
}

template <typename... Params, typename... Args>
int launch(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, void* stream, const Args&... args)
{
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? WQ4_OK : WQ4_ERR_CUDA;
}

// A double and what it lacks, to about 2^-94 of the value (not kept normalised).
struct Pair {
    double h, l;
};

Pair operator*(Pair a, Pair b)
{
    const double h = a.h * b.h;
    return {h, std::fma(a.h, b.h, -h) + std::fma(a.h, b.l, a.l * b.h)};
}

// Turns of the 64 pairs at position 1, times 2^64, to 2 of these units: an angle at
// position 2^30 is then within 2^-30, where a frequency rounded to a double leaves
// 2^-24 and more.  The frequencies are powers of theta^(-1 / 64), which one Newton
// step takes from the double's accuracy to the pair's.  (0.18 us on the host; 16 pow
// and products in doubles 0.28.)
void turns_of(double theta, uint64_t* turns)
{
    const double r = std::pow(theta, -1.0 / 64);
    Pair p = {r, 0.0};
    for (int i = 0; i < 5; ++i) p = p * p;                       // r^32: the product below stays near 1
    const Pair one = p * (p * Pair{theta, 0.0});
    const Pair root = {r, r * (((1.0 - one.h) - one.l) / 64)};
    Pair fine[9], coarse[8];
    fine[0] = coarse[0] = {1.0, 0.0};
    for (int i = 1; i < 9; ++i) fine[i] = fine[i - 1] * root;
    for (int i = 1; i < 8; ++i) coarse[i] = coarse[i - 1] * fine[8];
    for (int i = 0; i < kD / 2; ++i) {
        // w / (2 pi): a double and what it leaves
        constexpr double k2Pi = 6.283185307179586476925, k2PiLow = 2.4492935982947064e-16, kInv = 1.0 / k2Pi;
        constexpr double k64 = 18446744073709551616.0;
        const Pair w = coarse[i >> 3] * fine[i & 7];
        const double f = w.h * kInv, rest = (std::fma(-f, k2Pi, w.h) + (w.l - f * k2PiLow)) * kInv;
        turns[i] = static_cast<uint64_t>(f * k64) + static_cast<uint64_t>(static_cast<int64_t>(rest * k64));
    }
}

// The attention kernel's limit of shared memory, set once on each device (twice is harmless).
bool prompt_ready(int dev)
{
    static std::atomic<bool> ready[kMaxDevices];
    if (dev < kMaxDevices && ready[dev].load()) return true;
    if (cudaFuncSetAttribute(prompt_attn_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>(prompt_smem_bytes(WQ4_ATTN_MAX_BATCH))) != cudaSuccess)
        return false;
    if (dev < kMaxDevices) ready[dev].store(true);
    return true;
}

size_t prompt_desc_bytes(int grid) { return align_up(static_cast<size_t>(grid) * kDescInts * 4, 256); }

int prompt_grid(const DeviceInfo* di) { return std::min(di->sm_count, kMaxGrid); }

}  // namespace
}  // namespace wq4

using namespace wq4;

extern "C" int wq4_prompt_append(const wq4_kv_cache* cache, const uint16_t* qkv, int qkv_stride, uint16_t* q_out,
                                 int q_out_stride, const int32_t* row_starts, const int32_t* seq_lens, int batch, int rows,
                                 int n_q_heads, double rope_theta, void* stream)
{
    AppendArgs a = {};
    const int rc = check_rows(cache, row_starts, seq_lens, batch, rows, n_q_heads, &a.rows, &a.c);
    if (rc != WQ4_OK) return rc;
    const bool rotate = rope_theta != 0.0;
    if (!qkv || (rotate && !q_out)) return WQ4_ERR_INVALID;
    if (rotate && (!(rope_theta > 1.0) || !std::isfinite(rope_theta))) return WQ4_ERR_INVALID;
    const int width = (n_q_heads + 2 * cache->n_kv_heads) * kD;
    if (qkv_stride < width || (q_out && q_out_stride < n_q_heads * kD)) return WQ4_ERR_INVALID;
    if (!aligned(qkv, 16) || qkv_stride % 8 || (q_out && (!aligned(q_out, 16) || q_out_stride % 8))) return WQ4_ERR_ALIGN;
    const size_t in = rows_bytes(rows, qkv_stride, width), cb = cache_bytes(cache);
    if (overlaps(cache->k, cb, cache->v, cb) || overlaps(qkv, in, cache->k, cb) || overlaps(qkv, in, cache->v, cb))
        return WQ4_ERR_INVALID;
    if (q_out) {
        const size_t on = rows_bytes(rows, q_out_stride, n_q_heads * kD);
        const bool in_place = q_out == qkv && q_out_stride == qkv_stride;
        if (overlaps(q_out, on, cache->k, cb) || overlaps(q_out, on, cache->v, cb) || (!in_place && overlaps(q_out, on, qkv, in)))
            return WQ4_ERR_INVALID;
        if (in_place && !rotate) q_out = nullptr;      // already there
    }
    a.qkv = qkv;
    a.q_out = q_out;
    a.qkv_stride = qkv_stride;
    a.q_out_stride = q_out_stride;
    a.Hq = n_q_heads;
    a.rotate = rotate ? 1 : 0;
    a.err = status_word();
    if (!a.err) return WQ4_ERR_CUDA;
    if (rotate) turns_of(rope_theta, a.turns);
    int dev = 0;
    const DeviceInfo* di = current_device_info(&dev);
    if (!di) return WQ4_ERR_CUDA;
    return rows < 10 * di->sm_count ? launch(prompt_append_kernel<4, 6>, dim3((rows + 1) / 2), kAppThreads, 0, stream, a)
                                    : launch(prompt_append_kernel<2, 8>, dim3((rows + 3) / 4), kAppThreads, 0, stream, a);
}

extern "C" size_t wq4_prompt_attention_workspace_bytes(int batch, int rows, int n_q_heads, int n_kv_heads, int head_dim)
{
    if (batch < 1 || batch > WQ4_ATTN_MAX_BATCH || rows < 1 || n_kv_heads < 1 || n_q_heads < n_kv_heads ||
        n_q_heads % n_kv_heads || n_q_heads / n_kv_heads > kMaxGroup || head_dim != kD)
        return 0;
    int dev = 0;
    const DeviceInfo* di = current_device_info(&dev);
    if (!di) return 0;
    const int grid = prompt_grid(di);
    return prompt_desc_bytes(grid) + 2 * static_cast<size_t>(grid) * kSlotBytes;
}

extern "C" int wq4_prompt_attention(const wq4_kv_cache* cache, const uint16_t* q, int q_stride, const int32_t* row_starts,
                                    const int32_t* seq_lens, uint16_t* out, int out_stride, int batch, int rows,
                                    int n_q_heads, float scale, int window, int n_sinks, void* workspace,
                                    size_t workspace_bytes, void* stream)
{
    PromptArgs a;
    const int rc = check_rows(cache, row_starts, seq_lens, batch, rows, n_q_heads, &a.rows, &a.c);
    if (rc != WQ4_OK) return rc;
    if (!q || !out || !workspace) return WQ4_ERR_INVALID;
    const int width = n_q_heads * kD;
    if (q_stride < width || out_stride < width || !std::isfinite(scale) || window < 0 || n_sinks < 0) return WQ4_ERR_INVALID;
    if (!aligned(q, 16) || q_stride % 8 || !aligned(out, 16) || out_stride % 8 || !aligned(workspace, 256)) return WQ4_ERR_ALIGN;
    const int Hkv = cache->n_kv_heads, G = n_q_heads / Hkv, tok = kKeys / G;
    const int cap = cache->page_table_stride * cache->page_size;
    // the list of key tiles is indexed in int
    const int64_t items = static_cast<int64_t>(Hkv) * ((rows + 2 * tok - 1) / (2 * tok) + batch);
    // Short contexts: an item of few tiles is not worth cutting, and without cuts there is
    // nothing to join, which needs no launch then (512 tokens of 32 + 8 heads 14.4 us, cut
    // 21.0; eight sequences of 500 44.3 either way).
    a.uncut = (cap + kKeys - 1) / kKeys <= kUncut ? 1 : 0;
    const int64_t span = window ? std::min<int64_t>(cap, int64_t(window) + n_sinks + 2 * tok + 2 * kKeys) : cap;   // an item sees at most
    const int64_t most = a.uncut ? items : items * (span / kKeys + 1 + kItem);
    if (most >= (int64_t(1) << 30)) return WQ4_ERR_UNSUPPORTED;
    const size_t need = wq4_prompt_attention_workspace_bytes(batch, rows, n_q_heads, cache->n_kv_heads, kD);
    if (need == 0) return WQ4_ERR_CUDA;
    if (workspace_bytes < need) return WQ4_ERR_INVALID;
    const size_t ob = rows_bytes(rows, out_stride, width), cb = cache_bytes(cache);
    if (overlaps(out, ob, cache->k, cb) || overlaps(out, ob, cache->v, cb) || overlaps(out, ob, workspace, need) ||
        overlaps(out, ob, q, rows_bytes(rows, q_stride, width)))
        return WQ4_ERR_INVALID;
    int dev = 0;
    const DeviceInfo* di = current_device_info(&dev);
    if (!di || !prompt_ready(dev)) return WQ4_ERR_CUDA;
    const int grid = static_cast<int>(std::min<int64_t>(prompt_grid(di), a.uncut ? most : (most + kMinShare - 1) / kMinShare));
    a.q = q;
    a.out = out;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.G = G;
    a.tok = tok;
    a.cap = cap;
    a.window = window;           // (of the table's capacity too: rows behind its end outgrow it)
    a.sinks = std::min(n_sinks, cap);
    a.sl2 = static_cast<float>(std::fabs(static_cast<double>(scale)) * 1.4426950408889634);
    if (a.sl2 < FLT_MIN) a.sl2 = FLT_MIN;        // every weight alike, and masked scores still -infinity
    a.neg = scale < 0.f ? kIdescNegA : 0u;
    a.box = 16;
    while (a.box < kKeys && cache->page_size % (2 * a.box) == 0) a.box *= 2;
    a.wide = aligned(out, 32) && out_stride % 16 == 0 ? 1 : 0;
    a.stall = test_copy_stall() == WQ4_STALL_ATTN ? 1 : 0;
    a.desc = static_cast<int32_t*>(workspace);
    a.slots = static_cast<uint8_t*>(workspace) + prompt_desc_bytes(prompt_grid(di));
    a.err = status_word();
    if (!a.err) return WQ4_ERR_CUDA;
    PromptMaps maps;
    const uint64_t crows = static_cast<uint64_t>(cache->num_pages) * Hkv * cache->page_size;
    if (!encode_tensor_map_2d(&maps.k, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, cache->k, kD, crows, kD * 2, 64, a.box,
                              CU_TENSOR_MAP_SWIZZLE_128B) ||
        !encode_tensor_map_2d(&maps.v, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, cache->v, kD, crows, kD * 2, 64, a.box,
                              CU_TENSOR_MAP_SWIZZLE_128B) ||
        !encode_tensor_map_3d(&maps.q, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, q,
                              {kD, static_cast<uint64_t>(n_q_heads), static_cast<uint64_t>(rows)},
                              {kD * 2, static_cast<uint64_t>(q_stride) * 2},
                              {64, static_cast<uint32_t>(G), static_cast<uint32_t>(tok)}, CU_TENSOR_MAP_SWIZZLE_128B))
        return WQ4_ERR_CUDA;
    const int r = launch(prompt_attn_kernel, dim3(grid), kThreads, prompt_smem_bytes(batch), stream, maps, a);
    if (r != WQ4_OK || a.uncut || grid == 1) return r;      // one block cuts nothing
    // Rows of an item in blocks of 32 (fewer with few rows), dimensions over four blocks
    // where the items, were every row owned, are at most a quarter of the blocks, so
    // that each is cut in many parts.  (A block with nothing to join costs a launch:
    // 4832 of them 6 us.)
    const int chunks = rows * G <= 128 ? (rows * G + 31) / 32 : kSlotRows / 32;
    return static_cast<int64_t>(Hkv) * ((rows + 2 * tok - 1) / (2 * tok)) * 4 <= grid
               ? launch(prompt_join_kernel<1>, dim3(grid - 1, chunks, 4), 256, 0, stream, a)
               : launch(prompt_join_kernel<4>, dim3(grid - 1, chunks), 256, 0, stream, a);
}
