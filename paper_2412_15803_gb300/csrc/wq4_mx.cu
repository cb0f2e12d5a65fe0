// wq4_mx.cu -- rows of fp16 into microscaled codes and back: quantize, the
// residual's addition with the root-mean-square norm, silu(gate) * up.
//
// A group of 32 consecutive values of a row shares one power of two, the least
// 2^e with amax <= top * 2^e (top = 448 for e4m3, 6 for e2m1); a code is the
// value times 2^-e, rounded once.  amax = 2^E (1 + f), so e = E - 8 (or - 2),
// and one more where 1 + f is over top's own 1.75 (1.5): integer work on the
// bits of amax.  Eight values a lane, so that a group is four lanes, one
// 16-byte load is coalesced over a warp and the four scale bytes of 128
// columns, which lie side by side in the layout that the tensor cores read,
// leave as one word of 16 lanes.
//
// No load goes through the read-only path, and no pointer says that it has no
// aliases: the kernel before, which a launch here may overlap, may still be writing
// what is read after the wait for it, and nothing keeps a load of memory that is said
// not to change behind that wait.
#include "wq4.h"
#include "wq4_device.cuh"
#include "wq4_host.h"

#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>

namespace wq4 {
namespace {

constexpr unsigned kAll = 0xffffffffu;

// Two fp32 values an instruction.
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 d;
    asm("mul.rn.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<uint64_t&>(d))
        : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
    return d;
}

__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("add.rn.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<uint64_t&>(d))
        : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
    return d;
}

// Eight fp16 values of a 16-byte load.
__device__ __forceinline__ void to_floats(uint4 q, float2 v[4])
{
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
}

__device__ __forceinline__ uint4 to_halves(const float2 v[4])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 h = __floats2half2_rn(v[i].x, v[i].y);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Sixteen bytes, in the order of the program.
__device__ __forceinline__ uint4 load16(const uint16_t* p)
{
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

// Where the scales of row r's columns [128 kb, 128 kb + 128) lie.
__device__ __forceinline__ size_t scale_word(int r, int kb, int K)
{
    return (static_cast<size_t>(r >> 7) * (K >> 7) + kb) * 512 + (r & 31) * 16 + ((r >> 5) & 3) * 4;
}

// The largest magnitude of three, NaN if one is.
__device__ __forceinline__ float max_abs(float a, float b, float c)
{
    float d;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// The scale byte of a group whose largest magnitude has the bits mb.
template <int BITS>
__device__ __forceinline__ uint32_t scale_of(uint32_t mb)
{
    constexpr int kTop = BITS == 8 ? 8 : 2;                       // top = 1.75 * 2^8, 1.5 * 2^2
    constexpr uint32_t kUp = BITS == 8 ? 0x1FFFFFu : 0x3FFFFFu;   // carries into the exponent where 1 + f is over that
    const int e = max(static_cast<int>((mb + kUp) >> 23) - kTop, 0);
    return mb == 0 ? 127u : mb >= 0x7F800000u ? 255u : static_cast<uint32_t>(e);
}

// Codes of columns [8 c, 8 c + 8) of row r, zeros where the group's scale is NaN.
template <int BITS>
__device__ __forceinline__ void put_codes(uint2 o, uint32_t byte, uint8_t* codes, int r, int c, int K, bool live)
{
    if (byte == 255u) o = make_uint2(0, 0);
    if (!live) return;
    if constexpr (BITS == 8)
        *reinterpret_cast<uint2*>(codes + static_cast<size_t>(r) * K + 8 * c) = o;
    else
        *reinterpret_cast<uint32_t*>(codes + static_cast<size_t>(r) * (K >> 1) + 4 * c) = o.x;
}

// The word of scales of a lane's 128 columns, group j's byte at place j (in each of
// its 16 lanes).
__device__ __forceinline__ uint32_t scale_bytes_of(uint32_t byte, int c)
{
    uint32_t w = byte << (8 * ((c >> 2) & 3));
    w |= __shfl_xor_sync(kAll, w, 4);
    w |= __shfl_xor_sync(kAll, w, 8);
    return w;
}

// Codes of the eight values that each lane has of columns [8 c, 8 c + 8) of row
// r, and the word of scales of its 128 columns; all lanes of a warp, 16 in turn
// with 16 consecutive c.  Lanes without `live` store nothing.
template <int BITS>
__device__ __forceinline__ uint32_t store_codes(const float2 v[4], uint8_t* codes, int r, int c, int K, bool live)
{
    float m = max_abs(max_abs(v[0].x, v[0].y, v[1].x), max_abs(v[1].y, v[2].x, v[2].y), max_abs(v[3].x, v[3].y, 0.f));
    m = max_abs(m, __shfl_xor_sync(kAll, m, 1), 0.f);
    m = max_abs(m, __shfl_xor_sync(kAll, m, 2), 0.f);
    const uint32_t byte = scale_of<BITS>(__float_as_uint(m));
    const float inv = __uint_as_float((254u - byte) << 23);       // (a NaN scale's codes are not used)
    float2 q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = mul2(v[i], make_float2(inv, inv));
    uint2 o = make_uint2(0, 0);
    if constexpr (BITS == 8) {
        asm("{\n\t.reg .b16 a, b, c, d;\n\t"
            "cvt.rn.satfinite.e4m3x2.f32 a, %3, %2;\n\tcvt.rn.satfinite.e4m3x2.f32 b, %5, %4;\n\t"
            "cvt.rn.satfinite.e4m3x2.f32 c, %7, %6;\n\tcvt.rn.satfinite.e4m3x2.f32 d, %9, %8;\n\t"
            "mov.b32 %0, {a, b};\n\tmov.b32 %1, {c, d};\n\t}"
            : "=r"(o.x), "=r"(o.y)
            : "f"(q[0].x), "f"(q[0].y), "f"(q[1].x), "f"(q[1].y), "f"(q[2].x), "f"(q[2].y), "f"(q[3].x), "f"(q[3].y));
    } else {
        asm("{\n\t.reg .b8 a, b, c, d;\n\t"
            "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
            "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
            "mov.b32 %0, {a, b, c, d};\n\t}"
            : "=r"(o.x)
            : "f"(q[0].x), "f"(q[0].y), "f"(q[1].x), "f"(q[1].y), "f"(q[2].x), "f"(q[2].y), "f"(q[3].x), "f"(q[3].y));
    }
    put_codes<BITS>(o, byte, codes, r, c, K, live);
    return scale_bytes_of(byte, c);
}

// The same for fp16 values as they were loaded.  Magnitudes are compared as
// integers (NaN is over all numbers), and where 2^-e is a normal fp16 number the
// values are scaled in fp16: exactly, but for those that become smaller than 2^-14,
// whose codes are 0 either way.
template <int BITS>
__device__ __forceinline__ uint32_t store_codes(uint4 x, uint8_t* codes, int r, int c, int K, bool live)
{
    auto max2 = [](uint32_t a, uint32_t b) {
        uint32_t d;
        asm("max.u16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
        return d;
    };
    constexpr uint32_t kAbs = 0x7FFF7FFFu;
    uint32_t m = max2(max2(x.x & kAbs, x.y & kAbs), max2(x.z & kAbs, x.w & kAbs));
    m = max2(m, __shfl_xor_sync(kAll, m, 1));
    m = max2(m, __shfl_xor_sync(kAll, m, 2));
    const uint32_t byte = scale_of<BITS>(__float_as_uint(half_bits_to_float(static_cast<uint16_t>(max(m & 0xFFFFu, m >> 16)))));
    const bool normal = byte >= 127u - 15u;       // 2^-e at most 2^15 (and at least 2^-14: e is 14 at most)
    uint2 o = make_uint2(0, 0);
    if (__all_sync(kAll, normal)) {
        const uint32_t inv = (127u + 15u - min(byte, 127u + 14u)) << 10;
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(h[i]) : "r"(w[i]), "r"(inv | (inv << 16)));
        if constexpr (BITS == 8)
            asm("{\n\t.reg .b16 a, b, c, d;\n\t"
                "cvt.rn.satfinite.e4m3x2.f16x2 a, %2;\n\tcvt.rn.satfinite.e4m3x2.f16x2 b, %3;\n\t"
                "cvt.rn.satfinite.e4m3x2.f16x2 c, %4;\n\tcvt.rn.satfinite.e4m3x2.f16x2 d, %5;\n\t"
                "mov.b32 %0, {a, b};\n\tmov.b32 %1, {c, d};\n\t}"
                : "=r"(o.x), "=r"(o.y)
                : "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]));
        else
            asm("{\n\t.reg .b8 a, b, c, d;\n\t"
                "cvt.rn.satfinite.e2m1x2.f16x2 a, %1;\n\tcvt.rn.satfinite.e2m1x2.f16x2 b, %2;\n\t"
                "cvt.rn.satfinite.e2m1x2.f16x2 c, %3;\n\tcvt.rn.satfinite.e2m1x2.f16x2 d, %4;\n\t"
                "mov.b32 %0, {a, b, c, d};\n\t}"
                : "=r"(o.x)
                : "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]));
        put_codes<BITS>(o, byte, codes, r, c, K, live);
        return scale_bytes_of(byte, c);
    }
    float2 v[4];
    to_floats(x, v);
    return store_codes<BITS>(v, codes, r, c, K, live);
}

__device__ __forceinline__ void store_scales(uint32_t w, uint8_t* scales, int r, int c, int K, bool live)
{
    if (live && (c & 15) == 0) *reinterpret_cast<uint32_t*>(scales + scale_word(r, c >> 4, K)) = w;
}

// silu(g) u = g u / (1 + 2^(-g log2 e)) of two values, with the approximate
// exponential and reciprocal: relative errors of 2^-22 and 2^-23, and of |g| 2^-23
// from the exponent's product, far below the half step (2^-4) that the code is off
// by.  Under g = -87 the reciprocal is 0.  (expf and exact quotients: 70 us where
// these take 44, 4096 rows of 14336 in 8 bits.)
__device__ __forceinline__ float2 silu_times(float2 g, float2 u)
{
    const float2 t = mul2(g, make_float2(-1.44269504f, -1.44269504f));
    float2 e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(t.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(t.y));
    e = add2(e, make_float2(1.f, 1.f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(e.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(e.y));
    return mul2(mul2(g, u), r);
}

// A lane's place in a call on rows: eight columns, and rows r, r + 32, r + 64 and
// r + 96 (R = 4) or r alone.  Those four's scales are 16 consecutive bytes.
struct Place {
    int r, c;
    bool live;
};

template <int R>
__device__ __forceinline__ Place place(int M, int chunks)
{
    const int64_t groups = R == 1 ? M : (static_cast<int64_t>(M) + 127) / 128 * 32;
    const int64_t n = groups * chunks, i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
    int g, c;
    if (n <= 0x7FFFFFFF) {
        const uint32_t j = min(static_cast<uint32_t>(i), static_cast<uint32_t>(n - 1));
        g = j / static_cast<uint32_t>(chunks);
        c = j % static_cast<uint32_t>(chunks);
    } else {
        const int64_t j = min(i, n - 1);
        g = static_cast<int>(j / chunks);
        c = static_cast<int>(j % chunks);
    }
    const int r = R == 1 ? g : (g >> 5) * 128 + (g & 31);
    return {r, c, i < n && r < M};
}

// Rows without a sum over them: quantize, and silu(gate) * up.  Bound by memory:
// 4096 rows of 14336 silu in 44.0 us (6.7 TB/s) in 8 bits and 40.6 in 4, quantize in
// 25.6 in 4 bits (5.8 TB/s).  Before two values an instruction they were bound by
// issue (49.1, 43.7 and 26.0 at 0.72 of it).  Four rows a thread (two, then: 52.5, 48.7
// and 30.4), in blocks of 128 threads but for silu in 8 bits (256: 42.5 and 25.8 in 4
// bits, then; silu in 8 bits with 128 50.9).  Quantize has all four rows' loads in
// flight, silu two rows': the next one's loads go out behind a row's stores (all four
// 47.8 and 44.6, three 44.6 and 42.6; loads that the compiler may move 44.1 and 44.0).
template <int BITS, bool SILU>
constexpr int kRowThreads = BITS == 8 && SILU ? 256 : 128;

template <int BITS, int R>
__device__ __forceinline__ void silu_rows(const Place& p, const uint16_t* x, int stride, uint8_t* codes, int M, int K, uint32_t w[R])
{
    uint4 a[R], b[R];
    auto load = [&](int q) {          // behind the last row, that one again
        const uint16_t* row = x + static_cast<size_t>(min(p.r + 32 * q, M - 1)) * stride + 8 * p.c;
        a[q] = load16(row);
        b[q] = load16(row + K);
    };
#pragma unroll
    for (int q = 0; q < min(R, 2); ++q) load(q);
#pragma unroll
    for (int q = 0; q < R; ++q) {
        float2 v[4], u[4];
        to_floats(a[q], v);
        to_floats(b[q], u);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = silu_times(v[i], u[i]);
        w[q] = store_codes<BITS>(v, codes, p.r + 32 * q, p.c, K, p.live && p.r + 32 * q < M);
        if (q + 2 < R) load(q + 2);
    }
}

template <int BITS, bool SILU, int R>
__global__ void __launch_bounds__(kRowThreads<BITS, SILU>) rows_kernel(const uint16_t* x, int stride, uint8_t* codes, uint8_t* scales, int M, int K)
{
    grid_dependency_wait();
    grid_dependents_launch();
    const Place p = place<R>(M, K >> 3);
    uint32_t w[R];
    if constexpr (SILU) {
        silu_rows<BITS, R>(p, x, stride, codes, M, K, w);
    } else {
        uint4 a[R];
#pragma unroll
        for (int q = 0; q < R; ++q) {
            a[q] = make_uint4(0, 0, 0, 0);
            if (p.live && p.r + 32 * q < M) a[q] = load16(x + static_cast<size_t>(p.r + 32 * q) * stride + 8 * p.c);
        }
#pragma unroll
        for (int q = 0; q < R; ++q) w[q] = store_codes<BITS>(a[q], codes, p.r + 32 * q, p.c, K, p.live && p.r + 32 * q < M);
    }
    if (R == 4 && p.r + 96 < M) {
        if (p.live && (p.c & 15) == 0)
            *reinterpret_cast<uint4*>(scales + scale_word(p.r, p.c >> 4, K)) = make_uint4(w[0], w[R > 1 ? 1 : 0], w[R > 2 ? 2 : 0], w[R > 3 ? 3 : 0]);
    } else {
#pragma unroll
        for (int q = 0; q < R; ++q) store_scales(w[q], scales, p.r + 32 * q, p.c, K, p.live && p.r + 32 * q < M);
    }
}

struct NormArgs {
    const uint16_t* x;
    const uint16_t* residual;
    const uint16_t* gain;
    uint16_t* sum;
    uint8_t* codes;
    uint8_t* scales;
    int x_stride, residual_stride, sum_stride, M, K;
    float eps;
};

__device__ __forceinline__ uint32_t add_half2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// fp16(x + residual) of eight values.
__device__ __forceinline__ uint4 add_halves(uint4 x, uint4 r)
{
    return make_uint4(add_half2(x.x, r.x), add_half2(x.y, r.y), add_half2(x.z, r.z), add_half2(x.w, r.w));
}

// fp32 c + a b of the lower and of the upper halves: products of fp16 values are
// exact in fp32, and need no conversion first (sm_100 and later).
__device__ __forceinline__ float2 fma_halves(uint32_t a, uint32_t b, float2 c)
{
    asm("{\n\t.reg .f16 a0, a1, b0, b1;\n\tmov.b32 {a0, a1}, %2;\n\tmov.b32 {b0, b1}, %3;\n\t"
        "fma.rn.f32.f16 %0, a0, b0, %0;\n\tfma.rn.f32.f16 %1, a1, b1, %1;\n\t}"
        : "+f"(c.x), "+f"(c.y)
        : "r"(a), "r"(b));
    return c;
}

__device__ __forceinline__ uint4 load_h(const NormArgs& a, int r, int c)
{
    const uint4 x = *reinterpret_cast<const uint4*>(a.x + static_cast<size_t>(r) * a.x_stride + 8 * c);
    if (!a.residual) return x;
    return add_halves(x, *reinterpret_cast<const uint4*>(a.residual + static_cast<size_t>(r) * a.residual_stride + 8 * c));
}

__device__ __forceinline__ float squares(uint4 h, float ss)
{
    float2 t = fma_halves(h.x, h.x, make_float2(ss, 0.f));
    t = fma_halves(h.y, h.y, t);
    t = fma_halves(h.z, h.z, t);
    t = fma_halves(h.w, h.w, t);
    return t.x + t.y;
}

// f h g
__device__ __forceinline__ void norm_codes(uint4 h, uint4 g, float f, float2 o[4])
{
    const uint32_t a[4] = {h.x, h.y, h.z, h.w}, b[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = mul2(fma_halves(a[j], b[j], make_float2(0.f, 0.f)), make_float2(f, f));
}

constexpr uint32_t kOnes = 0x3C003C00u;      // fp16 1, 1

__device__ __forceinline__ uint4 load_gain(const NormArgs& a, int c)
{
    return a.gain && c < (a.K >> 3) ? *reinterpret_cast<const uint4*>(a.gain + 8 * c) : make_uint4(kOnes, kOnes, kOnes, kOnes);
}

// Rows of up to 512: a warp a row, eight rows a block, NC chunks of eight a lane.
template <int BITS, int NC>
__global__ void __launch_bounds__(256) norm_warp_kernel(const NormArgs a)
{
    grid_dependency_wait();
    grid_dependents_launch();
    const int64_t r = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    if (r >= a.M) return;
    const int lane = threadIdx.x & 31, chunks = a.K >> 3;
    uint4 h[NC];
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = lane + 32 * i;
        h[i] = make_uint4(0, 0, 0, 0);
        if (c < chunks) {
            h[i] = load_h(a, static_cast<int>(r), c);
            if (a.sum) *reinterpret_cast<uint4*>(a.sum + static_cast<size_t>(r) * a.sum_stride + 8 * c) = h[i];
        }
        ss = squares(h[i], ss);
    }
    const float f = rsqrtf(warp_sum(ss) / static_cast<float>(a.K) + a.eps);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = lane + 32 * i;
        float2 o[4];
        norm_codes(h[i], load_gain(a, c), f, o);
        const uint32_t w = store_codes<BITS>(o, a.codes, static_cast<int>(r), c, a.K, c < chunks);
        store_scales(w, a.scales, static_cast<int>(r), c, a.K, c < chunks);
    }
}

// A block a row, the row in registers, NC
// chunks of eight a thread (NC = 0, rows of more than 32768: read again for the
// second pass, from `sum` where there is one, since it may be x or residual).
template <int BITS, int NC>
__global__ void __launch_bounds__(1024) norm_kernel(const NormArgs a)
{
    __shared__ float part[2][32];
    grid_dependency_wait();
    grid_dependents_launch();
    const int nt = static_cast<int>(blockDim.x), chunks = a.K >> 3, t = static_cast<int>(threadIdx.x);
    const int n = NC ? NC : (chunks + nt - 1) / nt;
    int buf = 0;
    for (int r = blockIdx.x; r < a.M; r += gridDim.x, buf ^= 1) {
        uint4 h[NC ? NC : 1];
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const int c = t + i * nt;
            uint4& v = h[NC ? i : 0];
            v = make_uint4(0, 0, 0, 0);
            if (c < chunks) {
                v = load_h(a, r, c);
                if (a.sum) *reinterpret_cast<uint4*>(a.sum + static_cast<size_t>(r) * a.sum_stride + 8 * c) = v;
            }
            ss = squares(v, ss);
        }
        ss = warp_sum(ss);
        if ((t & 31) == 0) part[buf][t >> 5] = ss;
        __syncthreads();
        ss = warp_sum((t & 31) < (nt >> 5) ? part[buf][t & 31] : 0.f);
        const float f = rsqrtf(ss / static_cast<float>(a.K) + a.eps);
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const int c = t + i * nt;
            const bool live = c < chunks;
            uint4 v = h[NC ? i : 0];
            if (NC == 0) {
                v = make_uint4(0, 0, 0, 0);
                if (live) v = a.sum ? *reinterpret_cast<const uint4*>(a.sum + static_cast<size_t>(r) * a.sum_stride + 8 * c) : load_h(a, r, c);
            }
            float2 o[4];
            norm_codes(v, load_gain(a, c), f, o);
            const uint32_t w = store_codes<BITS>(o, a.codes, r, c, a.K, live);
            store_scales(w, a.scales, r, c, a.K, live);
        }
    }
}

constexpr int kCopyMost = 16384;      // columns: four chunks for each of 512 threads

// Many long rows: a bulk copy brings a block's next row (and the residual's) into shared
// memory while this one is in registers, so that what is in flight does not end at a
// block's barrier; one barrier a row, after which the buffer is free.  (Two to six rows
// in shared memory: no gain at any width from 6272 to 16384.)
template <int BITS, int NC>
__global__ void __launch_bounds__(512) norm_copy_kernel(const NormArgs a, uint32_t* err)
{
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ float part[2][32];
    __shared__ __align__(8) uint64_t full;
    const int nt = static_cast<int>(blockDim.x), chunks = a.K >> 3, t = static_cast<int>(threadIdx.x);
    const uint32_t row_bytes = 2 * a.K;
    const int step = static_cast<int>(gridDim.x);
    uint64_t pol = 0;
    auto fetch = [&](int64_t r) {
        mbar_arrive_expect_tx(&full, a.residual ? 2 * row_bytes : row_bytes);
        bulk_g2s(smem, a.x + static_cast<size_t>(r) * a.x_stride, row_bytes, &full, pol);
        if (a.residual) bulk_g2s(smem + row_bytes, a.residual + static_cast<size_t>(r) * a.residual_stride, row_bytes, &full, pol);
    };
    if (t == 0) {
        mbar_init(&full, 1);
        mbar_fence_init();
    }
    grid_dependency_wait();
    grid_dependents_launch();
    if (t == 0) {
        pol = l2_policy_evict_first();
        fetch(blockIdx.x);
    }
    uint4 g[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) g[i] = load_gain(a, t + i * nt);
    __syncthreads();                 // the barrier is there
    const uint4* const xs = reinterpret_cast<const uint4*>(smem);
    uint32_t par = 0;
    for (int64_t r = blockIdx.x; r < a.M; r += step, par ^= 1u) {
        mbar_wait(&full, par, err);
        uint4 h[NC];
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = t + i * nt;
            h[i] = make_uint4(0, 0, 0, 0);
            if (c < chunks) {
                h[i] = xs[c];
                if (a.residual) h[i] = add_halves(h[i], xs[chunks + c]);
                if (a.sum) __stcs(reinterpret_cast<uint4*>(a.sum + static_cast<size_t>(r) * a.sum_stride + 8 * c), h[i]);
            }
            ss = squares(h[i], ss);
        }
        ss = warp_sum(ss);
        if ((t & 31) == 0) part[par][t >> 5] = ss;
        __syncthreads();
        if (t == 0 && r + step < a.M) fetch(r + step);
        ss = warp_sum((t & 31) < (nt >> 5) ? part[par][t & 31] : 0.f);
        const float f = rsqrtf(ss / static_cast<float>(a.K) + a.eps);
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = t + i * nt;
            float2 o[4];
            norm_codes(h[i], g[i], f, o);
            const uint32_t w = store_codes<BITS>(o, a.codes, static_cast<int>(r), c, a.K, c < chunks);
            store_scales(w, a.scales, static_cast<int>(r), c, a.K, c < chunks);
        }
    }
}

template <int BITS, int R>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t* codes, const uint8_t* scales,
                                                         uint16_t* y, int stride, int M, int K)
{
    grid_dependency_wait();
    grid_dependents_launch();
    const Place p = place<R>(M, K >> 3);
    if (!p.live) return;
    uint2 code[R];
    uint32_t sb[R];
#pragma unroll
    for (int q = 0; q < R; ++q) {
        const int r = min(p.r + 32 * q, M - 1);
        sb[q] = scales[scale_word(r, p.c >> 4, K) + ((p.c >> 2) & 3)];
        if constexpr (BITS == 8)
            code[q] = *reinterpret_cast<const uint2*>(codes + static_cast<size_t>(r) * K + 8 * p.c);
        else
            code[q].x = *reinterpret_cast<const uint32_t*>(codes + static_cast<size_t>(r) * (K >> 1) + 4 * p.c);
    }
#pragma unroll
    for (int q = 0; q < R; ++q) {
        if (p.r + 32 * q >= M) break;
        // 2^(sb - 127); sb = 0 is 2^-127, below the normal range
        const float s = sb[q] == 255 ? __uint_as_float(0x7FC00000u) : sb[q] == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(sb[q] << 23);
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (BITS == 8) {
                const uint16_t c2 = static_cast<uint16_t>((i < 2 ? code[q].x : code[q].y) >> (16 * (i & 1)));
                asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h[i]) : "h"(c2));
            } else {
                const uint16_t c2 = static_cast<uint16_t>((code[q].x >> (8 * i)) & 0xFFu);
                asm("{\n\t.reg .b8 t, u;\n\tmov.b16 {t, u}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, t;\n\t}" : "=r"(h[i]) : "h"(c2));
            }
        }
        float2 v[4];
        to_floats(make_uint4(h[0], h[1], h[2], h[3]), v);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], make_float2(s, s));
        *reinterpret_cast<uint4*>(y + static_cast<size_t>(p.r + 32 * q) * stride + 8 * p.c) = to_halves(v);
    }
}

size_t scale_bytes(int rows, int K)
{
    return (static_cast<size_t>(rows) + 127) / 128 * 128 * (static_cast<size_t>(K) / 32);
}

size_t code_bytes(int rows, int K, int bits)
{
    return static_cast<size_t>(rows) * K / 8 * bits;
}

// Bytes from a strided matrix's first element to its last.
size_t row_bytes(int rows, int stride, int width)
{
    return (static_cast<size_t>(rows - 1) * stride + width) * 2;
}

int check_sizes(int M, int K, int bits)
{
    if (M < 1 || K < 128 || (K % 128) != 0 || (bits != 8 && bits != 4)) return WQ4_ERR_INVALID;
    if (static_cast<int64_t>(M) * K > (static_cast<int64_t>(1) << 41)) return WQ4_ERR_INVALID;
    return WQ4_OK;
}

int check_held(const uint8_t* codes, const uint8_t* scales, int M, int K, int bits)
{
    if (!aligned(codes, 32) || !aligned(scales, 16)) return WQ4_ERR_ALIGN;
    if (overlaps(codes, code_bytes(M, K, bits), scales, scale_bytes(M, K))) return WQ4_ERR_INVALID;
    return WQ4_OK;
}

// A call's launch: with programmatic dependent launch, on `stream`.
template <typename... P, typename... A>
int launch(void (*kernel)(P...), int64_t grid, int threads, size_t smem, void* stream, A... args)
{
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(grid));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? WQ4_OK : WQ4_ERR_CUDA;
}

// Four rows a thread from the size on where that many threads fill the GPU twice.
bool four_rows(const DeviceInfo* di, int M, int K)
{
    return static_cast<int64_t>(M) * (K / 8) >= static_cast<int64_t>(di->sm_count) * 2048 * 8;
}

int64_t rows_grid(int M, int K, int R, int threads)
{
    const int64_t groups = R == 1 ? M : (static_cast<int64_t>(M) + 127) / 128 * 32;
    return (groups * (K / 8) + threads - 1) / threads;
}

template <bool SILU>
int run_rows(const uint16_t* x, int stride, uint8_t* codes, uint8_t* scales, int M, int K, int bits, void* stream)
{
    if (!x || !codes || !scales) return WQ4_ERR_INVALID;
    int rc = check_sizes(M, K, bits);
    if (rc != WQ4_OK) return rc;
    const int64_t width = SILU ? 2 * static_cast<int64_t>(K) : K;
    if (stride < width) return WQ4_ERR_INVALID;
    if (!aligned(x, 16) || (stride % 8) != 0) return WQ4_ERR_ALIGN;
    rc = check_held(codes, scales, M, K, bits);
    if (rc != WQ4_OK) return rc;
    const size_t xb = row_bytes(M, stride, static_cast<int>(width));
    if (overlaps(x, xb, codes, code_bytes(M, K, bits)) || overlaps(x, xb, scales, scale_bytes(M, K))) return WQ4_ERR_INVALID;
    const DeviceInfo* di = current_device_info(nullptr);
    if (!di) return WQ4_ERR_CUDA;
    const int t = bits == 8 ? kRowThreads<8, SILU> : kRowThreads<4, SILU>;
    if (four_rows(di, M, K))
        return launch(bits == 8 ? rows_kernel<8, SILU, 4> : rows_kernel<4, SILU, 4>, rows_grid(M, K, 4, t), t, 0, stream, x, stride, codes,
                      scales, M, K);
    return launch(bits == 8 ? rows_kernel<8, SILU, 1> : rows_kernel<4, SILU, 1>, rows_grid(M, K, 1, t), t, 0, stream, x, stride, codes,
                  scales, M, K);
}

// Blocks of an SM: two to five are resident at a time (56 or 64 registers a thread), the
// others begin as those end, so that no SM is left with one row more than the next.
// With a residual and without, us, 64 Mi values of 8192 / 16384 columns: as many as are
// resident 77.6 / 78.6 and 40.5 / 40.0, 2048 threads' worth 77.9 / 78.7 and 39.8 / 40.8,
// 16 75.6 / 74.3 and 40.5 / 46.1; in 4 bits with a residual 71.7 / 72.1 as many as are
// resident, 69.9 / 69.1 16.
template <int BITS, int NC>
int launch_norm_copy(const NormArgs& a, const DeviceInfo* di, void* stream)
{
    static std::atomic<bool> ready[kMaxDevices];      // per device; setting the attribute twice is harmless
    if (!ready[di->dev].load()) {
        if (cudaFuncSetAttribute(norm_copy_kernel<BITS, NC>, cudaFuncAttributeMaxDynamicSharedMemorySize, 4 * kCopyMost) != cudaSuccess)
            return WQ4_ERR_CUDA;
        ready[di->dev].store(true);
    }
    const int threads = (a.K / 8 + 32 * NC - 1) / (32 * NC) * 32;
    const int64_t grid = std::min<int64_t>(a.M, static_cast<int64_t>(di->sm_count) * (a.residual ? 16 : 2048 / threads));
    return launch(norm_copy_kernel<BITS, NC>, grid, threads, static_cast<size_t>(a.residual ? 4 : 2) * a.K, stream, a, di->status);
}

// Measured, 8 bits, us: by a block a row and by copies 8192 rows of 4096 38.4 and
// 38.9, 8000 of 5120 48.5 and 49.2, 6000 of 8192 58.1 and 57.3, 5000 of 11008 79.8 and
// 64.1; by a block and by a warp a row 16384 of 1024 20.2 and 22.0, of 512 12.7 and
// 11.1, of 128 9.3 and 5.4.  (8192 of 4096: 38.0 with packed products, 6.2 TB/s; 46.7
// with conversions before every product.)  Bound by memory, then by the barrier
// between a row's two halves (0.61 of the issue rate).
template <int BITS>
int launch_norm(const NormArgs& a, const DeviceInfo* di, void* stream)
{
    const int chunks = a.K / 8;
    if (chunks <= 64) {
        const int64_t grid = (static_cast<int64_t>(a.M) + 7) / 8;
        return chunks <= 32 ? launch(norm_warp_kernel<BITS, 1>, grid, 256, 0, stream, a)
                            : launch(norm_warp_kernel<BITS, 2>, grid, 256, 0, stream, a);
    }
    if (a.M > 4 * di->sm_count && a.K > 6144 && a.K <= kCopyMost) return launch_norm_copy<BITS, 4>(a, di, stream);
    const int threads = chunks < 1024 ? (chunks + 31) / 32 * 32 : 1024;
    const int n = (chunks + threads - 1) / threads;
    const int grid = std::min(a.M, di->sm_count * 16);
    switch (n) {
        case 1: return launch(norm_kernel<BITS, 1>, grid, threads, 0, stream, a);
        case 2: return launch(norm_kernel<BITS, 2>, grid, threads, 0, stream, a);
        case 3:
        case 4: return launch(norm_kernel<BITS, 4>, grid, threads, 0, stream, a);
        default: return launch(norm_kernel<BITS, 0>, grid, threads, 0, stream, a);
    }
}

}  // namespace
}  // namespace wq4

using namespace wq4;

extern "C" size_t wq4_mx_scale_bytes(int rows, int K)
{
    return check_sizes(rows, K, 8) == WQ4_OK ? scale_bytes(rows, K) : 0;
}

extern "C" int wq4_mx_quantize(const uint16_t* x, int x_stride, uint8_t* codes, uint8_t* scales, int M, int K, int bits,
                               void* stream)
{
    return run_rows<false>(x, x_stride, codes, scales, M, K, bits, stream);
}

extern "C" int wq4_mx_silu(const uint16_t* gate_up, int stride, uint8_t* codes, uint8_t* scales, int M, int K, int bits,
                           void* stream)
{
    return run_rows<true>(gate_up, stride, codes, scales, M, K, bits, stream);
}

extern "C" int wq4_mx_norm(const uint16_t* x, int x_stride, const uint16_t* residual, int residual_stride,
                           const uint16_t* gain, float eps, uint16_t* sum, int sum_stride, uint8_t* codes, uint8_t* scales,
                           int M, int K, int bits, void* stream)
{
    if (!x || !codes || !scales) return WQ4_ERR_INVALID;
    int rc = check_sizes(M, K, bits);
    if (rc != WQ4_OK) return rc;
    if (!(eps > 0.f) || !std::isfinite(eps)) return WQ4_ERR_INVALID;
    if (x_stride < K || (residual && residual_stride < K) || (sum && sum_stride < K)) return WQ4_ERR_INVALID;
    if (!aligned(x, 16) || (x_stride % 8) != 0 || !aligned(gain, 16)) return WQ4_ERR_ALIGN;
    if (residual && (!aligned(residual, 16) || (residual_stride % 8) != 0)) return WQ4_ERR_ALIGN;
    if (sum && (!aligned(sum, 16) || (sum_stride % 8) != 0)) return WQ4_ERR_ALIGN;
    rc = check_held(codes, scales, M, K, bits);
    if (rc != WQ4_OK) return rc;
    const struct {
        const void* p;
        size_t n;
    } in[3] = {{x, row_bytes(M, x_stride, K)}, {residual, residual ? row_bytes(M, residual_stride, K) : 0}, {gain, gain ? 2 * static_cast<size_t>(K) : 0}};
    const size_t cb = code_bytes(M, K, bits), sb = scale_bytes(M, K), hb = sum ? row_bytes(M, sum_stride, K) : 0;
    for (int i = 0; i < 3; ++i) {
        if (!in[i].p) continue;
        if (overlaps(in[i].p, in[i].n, codes, cb) || overlaps(in[i].p, in[i].n, scales, sb)) return WQ4_ERR_INVALID;
        const bool same = (i == 0 && sum == x && sum_stride == x_stride) || (i == 1 && sum == residual && sum_stride == residual_stride);
        if (sum && !same && overlaps(in[i].p, in[i].n, sum, hb)) return WQ4_ERR_INVALID;
    }
    if (sum && (overlaps(sum, hb, codes, cb) || overlaps(sum, hb, scales, sb))) return WQ4_ERR_INVALID;
    const DeviceInfo* di = current_device_info(nullptr);
    if (!di) return WQ4_ERR_CUDA;
    const NormArgs a = {x, residual, gain, sum, codes, scales, x_stride, residual_stride, sum_stride, M, K, eps};
    return bits == 8 ? launch_norm<8>(a, di, stream) : launch_norm<4>(a, di, stream);
}

extern "C" int wq4_mx_dequantize(const uint8_t* codes, const uint8_t* scales, uint16_t* y, int y_stride, int M, int K,
                                 int bits, void* stream)
{
    if (!codes || !scales || !y) return WQ4_ERR_INVALID;
    int rc = check_sizes(M, K, bits);
    if (rc != WQ4_OK) return rc;
    if (y_stride < K) return WQ4_ERR_INVALID;
    if (!aligned(y, 16) || (y_stride % 8) != 0) return WQ4_ERR_ALIGN;
    rc = check_held(codes, scales, M, K, bits);
    if (rc != WQ4_OK) return rc;
    const size_t yb = row_bytes(M, y_stride, K);
    if (overlaps(y, yb, codes, code_bytes(M, K, bits)) || overlaps(y, yb, scales, scale_bytes(M, K))) return WQ4_ERR_INVALID;
    const DeviceInfo* di = current_device_info(nullptr);
    if (!di) return WQ4_ERR_CUDA;
    if (four_rows(di, M, K))
        return launch(bits == 8 ? dequantize_kernel<8, 4> : dequantize_kernel<4, 4>, rows_grid(M, K, 4, 256), 256, 0, stream, codes, scales, y,
                      y_stride, M, K);
    return launch(bits == 8 ? dequantize_kernel<8, 1> : dequantize_kernel<4, 1>, rows_grid(M, K, 1, 256), 256, 0, stream, codes, scales, y,
                  y_stride, M, K);
}
