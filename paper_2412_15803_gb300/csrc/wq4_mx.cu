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
#include "wq4.h"
#include "wq4_device.cuh"
#include "wq4_host.h"

#include <cuda_runtime.h>

#include <cmath>

namespace wq4 {
namespace {

constexpr unsigned kAll = 0xffffffffu;

// Eight fp16 values of a 16-byte load.
__device__ __forceinline__ void to_floats(uint4 q, float v[8])
{
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = half_bits_to_float(static_cast<uint16_t>(w[i] & 0xFFFFu));
        v[2 * i + 1] = half_bits_to_float(static_cast<uint16_t>(w[i] >> 16));
    }
}

__device__ __forceinline__ uint4 to_halves(const float v[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = static_cast<uint32_t>(float_to_half_bits(v[2 * i])) |
               (static_cast<uint32_t>(float_to_half_bits(v[2 * i + 1])) << 16);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// (b, a) as two e4m3 codes, a in the lower byte.
__device__ __forceinline__ uint32_t e4m3x2(float a, float b)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
    return r;
}

// (b, a) as two e2m1 codes, a in the lower nibble.
__device__ __forceinline__ uint32_t e2m1x2(float a, float b)
{
    uint16_t r;
    asm("{\n\t.reg .b8 t;\n\tcvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n\tcvt.u16.u8 %0, t;\n\t}" : "=h"(r) : "f"(b), "f"(a));
    return r;
}

// Where the scales of row r's columns [128 kb, 128 kb + 128) lie.
__device__ __forceinline__ size_t scale_word(int r, int kb, int K)
{
    return (static_cast<size_t>(r >> 7) * (K >> 7) + kb) * 512 + (r & 31) * 16 + ((r >> 5) & 3) * 4;
}

// Codes and scales of the eight values that each lane has of columns [8 c, 8 c +
// 8) of row r; all lanes of a warp, 16 in turn with 16 consecutive c.  Lanes
// without `live` store nothing.
template <int BITS>
__device__ __forceinline__ void store_codes(const float v[8], uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                                            int r, int c, int K, bool live)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);   // NaN is over all numbers here
    m = max(m, __shfl_xor_sync(kAll, m, 1));
    m = max(m, __shfl_xor_sync(kAll, m, 2));
    constexpr int kTop = BITS == 8 ? 8 : 2;                       // top = 1.75 * 2^8, 1.5 * 2^2
    constexpr uint32_t kFrac = BITS == 8 ? 0x600000u : 0x400000u;
    const bool bad = m >= 0x7F800000u;
    int e = static_cast<int>(m >> 23) - 127 - kTop + ((m & 0x7FFFFFu) > kFrac ? 1 : 0);
    e = m == 0 ? 0 : max(e, -127);
    const float inv = bad ? 0.f : __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = bad ? 0.f : v[i] * inv;
    if constexpr (BITS == 8) {
        const uint2 o = make_uint2(e4m3x2(q[0], q[1]) | (e4m3x2(q[2], q[3]) << 16), e4m3x2(q[4], q[5]) | (e4m3x2(q[6], q[7]) << 16));
        if (live) *reinterpret_cast<uint2*>(codes + static_cast<size_t>(r) * K + 8 * c) = o;
    } else {
        const uint32_t o = e2m1x2(q[0], q[1]) | (e2m1x2(q[2], q[3]) << 8) | (e2m1x2(q[4], q[5]) << 16) | (e2m1x2(q[6], q[7]) << 24);
        if (live) *reinterpret_cast<uint32_t*>(codes + static_cast<size_t>(r) * (K >> 1) + 4 * c) = o;
    }
    // group j's byte at place j of the word of 128 columns
    uint32_t w = static_cast<uint32_t>(bad ? 255 : e + 127) << (8 * ((c >> 2) & 3));
    w |= __shfl_xor_sync(kAll, w, 4);
    w |= __shfl_xor_sync(kAll, w, 8);
    if (live && (c & 15) == 0) *reinterpret_cast<uint32_t*>(scales + scale_word(r, c >> 4, K)) = w;
}

__device__ __forceinline__ float silu(float g)
{
    return g / (1.f + expf(-g));
}

// Rows without a sum over them: quantize, and silu(gate) * up.  A block's
// threads take consecutive columns, gridDim.y rows at a time.
template <int BITS, bool SILU>
__global__ void __launch_bounds__(256) rows_kernel(const uint16_t* __restrict__ x, int stride, uint8_t* __restrict__ codes,
                                                   uint8_t* __restrict__ scales, int M, int K)
{
    grid_dependency_wait();
    grid_dependents_launch();
    const int c = static_cast<int>(blockIdx.x * blockDim.x + threadIdx.x), chunks = K >> 3;
    const bool live = c < chunks;
    for (int r = blockIdx.y; r < M; r += gridDim.y) {
        float v[8] = {};
        if (live) {
            const uint16_t* row = x + static_cast<size_t>(r) * stride + 8 * c;
            to_floats(*reinterpret_cast<const uint4*>(row), v);
            if constexpr (SILU) {
                float u[8];
                to_floats(*reinterpret_cast<const uint4*>(row + K), u);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = silu(v[i]) * u[i];
            }
        }
        store_codes<BITS>(v, codes, scales, r, c, K, live);
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

__device__ __forceinline__ void load_h(const NormArgs& a, int r, int c, float h[8])
{
    to_floats(*reinterpret_cast<const uint4*>(a.x + static_cast<size_t>(r) * a.x_stride + 8 * c), h);
    if (!a.residual) return;
    float t[8];
    to_floats(*reinterpret_cast<const uint4*>(a.residual + static_cast<size_t>(r) * a.residual_stride + 8 * c), t);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = half_bits_to_float(float_to_half_bits(h[i] + t[i]));
}

// A block a row.  The row stays in registers, NC chunks of eight a thread
// (NC = 0, rows of more than 32768: read again for the second pass, from `sum`
// where there is one, since it may be x or residual).
template <int BITS, int NC>
__global__ void __launch_bounds__(1024) norm_kernel(const NormArgs a)
{
    __shared__ float part[32];
    grid_dependency_wait();
    grid_dependents_launch();
    const int nt = static_cast<int>(blockDim.x), chunks = a.K >> 3, t = static_cast<int>(threadIdx.x);
    const int n = NC ? NC : (chunks + nt - 1) / nt;
    for (int r = blockIdx.x; r < a.M; r += gridDim.x) {
        float h[NC ? NC : 1][8];
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const int c = t + i * nt;
            float* v = h[NC ? i : 0];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = 0.f;
            if (c < chunks) {
                load_h(a, r, c, v);
                if (a.sum) *reinterpret_cast<uint4*>(a.sum + static_cast<size_t>(r) * a.sum_stride + 8 * c) = to_halves(v);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) ss = fmaf(v[j], v[j], ss);
        }
        ss = warp_sum(ss);
        if ((t & 31) == 0) part[t >> 5] = ss;
        __syncthreads();
        ss = warp_sum((t & 31) < (nt >> 5) ? part[t & 31] : 0.f);
        __syncthreads();
        const float f = rsqrtf(ss / static_cast<float>(a.K) + a.eps);
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const int c = t + i * nt;
            const bool live = c < chunks;
            float* v = h[NC ? i : 0];
            float g[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
            if (live) {
                if (NC == 0) {
                    if (a.sum)
                        to_floats(*reinterpret_cast<const uint4*>(a.sum + static_cast<size_t>(r) * a.sum_stride + 8 * c), v);
                    else
                        load_h(a, r, c, v);
                }
                if (a.gain) to_floats(*reinterpret_cast<const uint4*>(a.gain + 8 * c), g);
            }
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = v[j] * f * g[j];
            store_codes<BITS>(o, a.codes, a.scales, r, c, a.K, live);
        }
    }
}

template <int BITS>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                         uint16_t* __restrict__ y, int stride, int M, int K)
{
    grid_dependency_wait();
    grid_dependents_launch();
    const int c = static_cast<int>(blockIdx.x * blockDim.x + threadIdx.x);
    if (c >= (K >> 3)) return;
    for (int r = blockIdx.y; r < M; r += gridDim.y) {
        const uint32_t sb = scales[scale_word(r, c >> 4, K) + ((c >> 2) & 3)];
        // 2^(sb - 127); sb = 0 is 2^-127, below the normal range
        const float s = sb == 255 ? __uint_as_float(0x7FC00000u) : sb == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(sb << 23);
        uint32_t h[4];
        if constexpr (BITS == 8) {
            const uint2 q = *reinterpret_cast<const uint2*>(codes + static_cast<size_t>(r) * K + 8 * c);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint16_t p = static_cast<uint16_t>((i < 2 ? q.x : q.y) >> (16 * (i & 1)));
                asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h[i]) : "h"(p));
            }
        } else {
            const uint32_t q = *reinterpret_cast<const uint32_t*>(codes + static_cast<size_t>(r) * (K >> 1) + 4 * c);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint16_t p = static_cast<uint16_t>((q >> (8 * i)) & 0xFFu);
                asm("{\n\t.reg .b8 t, u;\n\tmov.b16 {t, u}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, t;\n\t}" : "=r"(h[i]) : "h"(p));
            }
        }
        float v[8];
        to_floats(make_uint4(h[0], h[1], h[2], h[3]), v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= s;
        *reinterpret_cast<uint4*>(y + static_cast<size_t>(r) * stride + 8 * c) = to_halves(v);
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
int launch(void (*kernel)(P...), dim3 grid, int threads, void* stream, A... args)
{
    if (!current_device_info(nullptr)) return WQ4_ERR_CUDA;
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

dim3 rows_grid(int M, int K)
{
    return dim3((K / 8 + 255) / 256, M < 65535 ? M : 65535);
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
    return launch(bits == 8 ? rows_kernel<8, SILU> : rows_kernel<4, SILU>, rows_grid(M, K), 256, stream, x, stride, codes, scales, M, K);
}

template <int BITS>
int launch_norm(const NormArgs& a, int sms, void* stream)
{
    const int chunks = a.K / 8;
    int threads = chunks < 1024 ? (chunks + 31) / 32 * 32 : 1024;
    const int n = (chunks + threads - 1) / threads;
    const dim3 grid(a.M < sms * 16 ? a.M : sms * 16);
    switch (n) {
        case 1: return launch(norm_kernel<BITS, 1>, grid, threads, stream, a);
        case 2: return launch(norm_kernel<BITS, 2>, grid, threads, stream, a);
        case 3:
        case 4: return launch(norm_kernel<BITS, 4>, grid, threads, stream, a);
        default: return launch(norm_kernel<BITS, 0>, grid, threads, stream, a);
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
    return bits == 8 ? launch_norm<8>(a, di->sm_count, stream) : launch_norm<4>(a, di->sm_count, stream);
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
    return launch(bits == 8 ? dequantize_kernel<8> : dequantize_kernel<4>, rows_grid(M, K), 256, stream, codes, scales, y, y_stride,
                  M, K);
}
