// wq4_prompt.cu -- the new tokens of prompts (sm_103a): their keys and values
// into a paged cache, and their attention over it, causal, with or without a
// sliding window and first tokens that stay visible.
#include "wq4.h"
#include "wq4_attn.h"
#include "wq4_device.cuh"
#include "wq4_host.h"

#include <cuda_runtime.h>

#include <cmath>

namespace wq4 {
namespace {

constexpr int kD = 128;
constexpr int kMaxGroup = 8;

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

// The sequence that owns row r (-1: none) and the row's position.
__device__ __forceinline__ int row_owner(const Rows& R, int r, int* pos)
{
    int lo = 0, hi = R.batch - 1;
    while (lo < hi) {              // the last sequence that starts at or before r
        const int mid = (lo + hi + 1) >> 1;
        if (__ldg(R.starts + mid) <= r) lo = mid;
        else hi = mid - 1;
    }
    const int s = __ldg(R.starts + lo), e = __ldg(R.starts + lo + 1);
    *pos = __ldg(R.lens + lo) - e + r;
    return r >= s && r < e && r < R.rows ? lo : -1;
}

// ----------------------------------------------------------------- append --

constexpr int kAppRows = 8;
constexpr int kAppThreads = 256;

struct AppendArgs {
    Rows rows;
    Paged c;
    const uint16_t* qkv;
    uint16_t* q_out;                 // null: q is left alone
    int qkv_stride, q_out_stride, Hq, rotate;
    uint32_t* err;
    double inv_freq[kD / 2];
};

// (x0, x1) turned by the angle whose cosine and sine are t.x + t.y and t.z + t.w.
// t.x and t.z have 12 significant bits, an fp16 value 11: their products are exact
// in fp32, so the difference of the two large products is rounded once and the
// remainders (2^-12 of them) add what they lack.  The fp64 rotation costs more
// than the copy that it rides on (GB300 has 1.25 TFLOP/s of fp64).
__device__ __forceinline__ uint32_t turn(uint32_t x, float4 t)
{
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&x));
    const float re = fmaf(v.x, t.x, -(v.y * t.z)) + fmaf(v.x, t.y, -(v.y * t.w));
    const float im = fmaf(v.x, t.z, v.y * t.x) + fmaf(v.x, t.w, v.y * t.y);
    const __half2 h = __floats2half2_rn(re, im);
    return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ float2 split12(double v)
{
    const float hi = __uint_as_float(__float_as_uint(static_cast<float>(v)) & 0xFFFFF000u);
    return make_float2(hi, static_cast<float>(v - hi));
}

// A block takes kAppRows rows: their owners and cache rows, the 64 rotations of
// each, then 16 bytes a thread and step.
__global__ void __launch_bounds__(kAppThreads) prompt_append_kernel(const __grid_constant__ AppendArgs a)
{
    __shared__ float4 rope[kAppRows][kD / 2];
    __shared__ int64_t dst[kAppRows];       // (page, row) as a row of head 0; -1: not written
    __shared__ int pos_of[kAppRows], owner[kAppRows];
    grid_dependency_wait();
    grid_dependents_launch();
    const int r0 = blockIdx.x * kAppRows, tid = threadIdx.x;
    if (tid < kAppRows) {
        int pos = 0;
        const int b = r0 + tid < a.rows.rows ? row_owner(a.rows, r0 + tid, &pos) : -1;
        int64_t d = -1;
        if (b >= 0) {
            const int page = pos >= 0 && pos < a.c.stride * a.c.page_size
                                 ? __ldg(a.c.table + static_cast<size_t>(b) * a.c.stride + pos / a.c.page_size) : -1;
            if (page >= 0 && page < a.c.num_pages)
                d = static_cast<int64_t>(page) * a.c.Hkv * a.c.page_size + pos % a.c.page_size;
            else
                atomicOr(a.err, kErrAppend);
        }
        owner[tid] = b;
        pos_of[tid] = pos < 0 ? 0 : pos;
        dst[tid] = d;
    }
    __syncthreads();
    if (a.rotate) {
        for (int e = tid; e < kAppRows * (kD / 2); e += kAppThreads) {
            const int r = e / (kD / 2), i = e % (kD / 2);
            if (owner[r] < 0) continue;
            double s, c;
            sincos(pos_of[r] * a.inv_freq[i], &s, &c);
            const float2 cc = split12(c), ss = split12(s);
            rope[r][i] = make_float4(cc.x, cc.y, ss.x, ss.y);
        }
        __syncthreads();
    }
    const int heads = a.Hq + 2 * a.c.Hkv, words = heads * (kD / 8);
    for (int r = 0; r < kAppRows; ++r) {
        if (owner[r] < 0) continue;
        const uint4* row = reinterpret_cast<const uint4*>(a.qkv + static_cast<size_t>(r0 + r) * a.qkv_stride);
        for (int e = tid; e < words; e += kAppThreads) {
            const int head = e / (kD / 8), w = e % (kD / 8);
            const int kv = head - a.Hq;                  // >= 0: a key or value head
            if (kv < 0 ? !a.q_out : dst[r] < 0) continue;
            uint4 x = row[e];
            if (a.rotate && kv < a.c.Hkv) {
                x.x = turn(x.x, rope[r][4 * w]);
                x.y = turn(x.y, rope[r][4 * w + 1]);
                x.z = turn(x.z, rope[r][4 * w + 2]);
                x.w = turn(x.w, rope[r][4 * w + 3]);
            }
            uint16_t* to;
            if (kv < 0)
                to = a.q_out + static_cast<size_t>(r0 + r) * a.q_out_stride + head * kD;
            else
                to = (kv < a.c.Hkv ? a.c.k : a.c.v) +
                     (dst[r] + static_cast<int64_t>(kv < a.c.Hkv ? kv : kv - a.c.Hkv) * a.c.page_size) * kD;
            reinterpret_cast<uint4*>(to)[w] = x;
        }
    }
}

// -------------------------------------------------------------- attention --

struct PromptArgs {
    Rows rows;
    Paged c;
    const uint16_t* q;
    uint16_t* out;
    int q_stride, out_stride, G;
    int window, sinks;               // window 0: none
    float sl2;                       // scale * log2(e)
    uint32_t* err;
};

// One row and query head by one warp, a token at a time, four dimensions a lane.
__device__ void attend_row(const PromptArgs& a, int b, int pos, int row, int head)
{
    const int lane = threadIdx.x & 31, h = head / a.G;
    const int cap = a.c.stride * a.c.page_size;
    const uint2 qb = *reinterpret_cast<const uint2*>(a.q + static_cast<size_t>(row) * a.q_stride + head * kD + 4 * lane);
    const float2 q0 = __half22float2(*reinterpret_cast<const __half2*>(&qb.x));
    const float2 q1 = __half22float2(*reinterpret_cast<const __half2*>(&qb.y));
    const int32_t* table = a.c.table + static_cast<size_t>(b) * a.c.stride;
    float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f, o2 = 0.f, o3 = 0.f;
    const int end = min(pos, cap - 1);
    if (pos >= cap && lane == 0) atomicOr(a.err, kErrSeqLen);
    const int first = a.window ? max(0, pos - a.window + 1) : 0;
    for (int t = a.window && a.sinks ? 0 : first; t <= end; ++t) {
        if (t < first && t >= a.sinks) t = first;
        if (t > end) break;
        const int page = __ldg(table + t / a.c.page_size);
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
        const float x = warp_sum(fmaf(q0.x, k0.x, q0.y * k0.y) + fmaf(q1.x, k1.x, q1.y * k1.y)) * a.sl2;
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

__global__ void __launch_bounds__(256) prompt_attn_kernel(const PromptArgs a)
{
    grid_dependency_wait();
    grid_dependents_launch();
    const int Hq = a.G * a.c.Hkv;
    const int64_t item = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    if (item >= static_cast<int64_t>(a.rows.rows) * Hq) return;
    const int row = static_cast<int>(item / Hq), head = static_cast<int>(item % Hq);
    int pos;
    const int b = row_owner(a.rows, row, &pos);
    if (b >= 0) attend_row(a, b, pos, row, head);
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
    if (c->head_dim != kD || n_q_heads / c->n_kv_heads > kMaxGroup) return WQ4_ERR_UNSUPPORTED;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->page_table, 4) || !aligned(row_starts, 4) ||
        !aligned(seq_lens, 4))
        return WQ4_ERR_ALIGN;
    if (static_cast<int64_t>(c->num_pages) * c->n_kv_heads * c->page_size >= (int64_t(1) << 31) ||
        static_cast<int64_t>(c->page_table_stride) * c->page_size >= (int64_t(1) << 30) || rows >= (1 << 30))
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

template <typename Args>
int launch(void (*kernel)(Args), dim3 grid, int threads, void* stream, const Args& args)
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
    return cudaLaunchKernelEx(&cfg, kernel, args) == cudaSuccess ? WQ4_OK : WQ4_ERR_CUDA;
}

}  // namespace
}  // namespace wq4

using namespace wq4;

extern "C" int wq4_prompt_append(const wq4_kv_cache* cache, const uint16_t* qkv, int qkv_stride, uint16_t* q_out,
                                 int q_out_stride, const int32_t* row_starts, const int32_t* seq_lens, int batch, int rows,
                                 int n_q_heads, double rope_theta, void* stream)
{
    AppendArgs a;
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
    for (int i = 0; i < kD / 2; ++i) a.inv_freq[i] = rotate ? std::pow(rope_theta, -2.0 * i / kD) : 0.0;
    return launch(prompt_append_kernel, dim3((rows + kAppRows - 1) / kAppRows), kAppThreads, stream, a);
}

extern "C" size_t wq4_prompt_attention_workspace_bytes(int batch, int rows, int n_q_heads, int n_kv_heads, int head_dim)
{
    if (batch < 1 || batch > WQ4_ATTN_MAX_BATCH || rows < 1 || n_kv_heads < 1 || n_q_heads < n_kv_heads ||
        n_q_heads % n_kv_heads || n_q_heads / n_kv_heads > kMaxGroup || head_dim != kD)
        return 0;
    return 256;
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
    const size_t need = wq4_prompt_attention_workspace_bytes(batch, rows, n_q_heads, cache->n_kv_heads, kD);
    if (need == 0) return WQ4_ERR_CUDA;
    if (workspace_bytes < need) return WQ4_ERR_INVALID;
    const size_t ob = rows_bytes(rows, out_stride, width), cb = cache_bytes(cache);
    if (overlaps(out, ob, cache->k, cb) || overlaps(out, ob, cache->v, cb) || overlaps(out, ob, workspace, need) ||
        overlaps(out, ob, q, rows_bytes(rows, q_stride, width)))
        return WQ4_ERR_INVALID;
    a.q = q;
    a.out = out;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.G = n_q_heads / cache->n_kv_heads;
    a.window = window;
    a.sinks = n_sinks;
    a.sl2 = static_cast<float>(static_cast<double>(scale) * 1.4426950408889634);
    a.err = status_word();
    if (!a.err) return WQ4_ERR_CUDA;
    const int64_t items = static_cast<int64_t>(rows) * n_q_heads;
    if (items >= (int64_t(1) << 33)) return WQ4_ERR_UNSUPPORTED;
    return launch(prompt_attn_kernel, dim3(static_cast<unsigned>((items + 7) / 8)), 256, stream, a);
}
