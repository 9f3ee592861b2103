// Norm of whole rows with the residual's addition, and rows in 8 bits with a scale each.
//
//     h = x + residual (rounded to the residual's type, as it is stored),  r = 1 / sqrt(mean(h^2) + eps),
//     y = h w r,  scale = max(max |y| / 448, 2^-126),  q = e4m3(y / scale).
// One pass: a row stays in the registers of the threads that read it, and its two statistics, sum h^2 and max |h w|, are
// taken in one round: max |y| = r max |h w|, since r does not depend on the element.  Sums are binary32.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "geocache.h"
#include "geocache_device.cuh"
#include "geocache_internal.h"

namespace geocache {

namespace {

constexpr int kThreads = 256;   // of a block, or as many as a wide row takes
constexpr float kLargest = 448.0f, kTiny = 0x1p-126f;  // of e4m3; the least scale (the least normal number)

__device__ __forceinline__ void unpack2(uint32_t w, float* v, __nv_bfloat16) {
    v[0] = __uint_as_float(w << 16);
    v[1] = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ void unpack2(uint32_t w, float* v, __half) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    v[0] = f.x;
    v[1] = f.y;
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __nv_bfloat16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __half) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T>
__device__ __forceinline__ T rounded(float x) {
    if constexpr (std::is_same<T, float>::value) return x;
    else if constexpr (std::is_same<T, __half>::value) return __float2half_rn(x);
    else return __float2bfloat16_rn(x);
}

// 8 elements of a row, n of them inside it (the others are zero)
template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, bool aligned, float* v) {
    if (aligned && n == 8) {
        if constexpr (std::is_same<T, float>::value) {
            const float4 a = __ldcs(reinterpret_cast<const float4*>(p)), b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
            v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
            const uint4 w = __ldcs(reinterpret_cast<const uint4*>(p));
            unpack2(w.x, v, T());
            unpack2(w.y, v + 2, T());
            unpack2(w.z, v + 4, T());
            unpack2(w.w, v + 6, T());
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < n ? to_float(p[e]) : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int n, bool aligned, const float* v) {
    if (aligned && n == 8) {
        if constexpr (std::is_same<T, float>::value) {
            reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            *reinterpret_cast<uint4*>(p) =
                make_uint4(pack2(v[0], v[1], T()), pack2(v[2], v[3], T()), pack2(v[4], v[5], T()), pack2(v[6], v[7], T()));
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = rounded<T>(v[e]);
    }
}
// two floats as e4m3, `lo` in the low byte, values over 448 as 448
__device__ __forceinline__ uint32_t pack_e4m3(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

// The rows of a block: `lanes` threads (a power of two) each, kWords words of 8 elements a thread, the words of a row
// side by side over its threads.
template <typename X, bool kNorm, bool kQuant, int kWords>
__global__ void __launch_bounds__(1024) norm_rows_kernel(const __grid_constant__ NormRowsArgs a) {
    __shared__ float2 shared[32];
    const int lane = threadIdx.x & (a.lanes - 1), row_in = threadIdx.x / a.lanes;
    const long long row = (long long)blockIdx.x * (blockDim.x / a.lanes) + row_in;
    const bool active = row < a.T;
    pdl_wait();
    float v[kWords][8];
    const X* x = static_cast<const X*>(a.x.data) + row * a.x.stride;
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
        const int at = 8 * (lane + i * a.lanes), n = active ? min(8, a.C - at) : 0;
        load8(x + at, n, a.x_aligned, v[i]);
    }
    if (kNorm && a.residual.data) {
        float r[kWords][8];
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            const int at = 8 * (lane + i * a.lanes), n = active ? min(8, a.C - at) : 0;
            if (std::is_same<X, float>::value || a.residual_f32)
                load8(static_cast<const float*>(a.residual.data) + row * a.residual.stride + at, n, a.residual_aligned, r[i]);
            else
                load8(static_cast<const X*>(a.residual.data) + row * a.residual.stride + at, n, a.residual_aligned, r[i]);
        }
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            const int at = 8 * (lane + i * a.lanes), n = active ? min(8, a.C - at) : 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[i][e] += r[i][e];
                if (!a.residual_f32) v[i][e] = to_float(rounded<X>(v[i][e]));
            }
            if (std::is_same<X, float>::value || a.residual_f32)
                store8(static_cast<float*>(a.residual_out.data) + row * a.residual_out.stride + at, n, a.residual_aligned, v[i]);
            else
                store8(static_cast<X*>(a.residual_out.data) + row * a.residual_out.stride + at, n, a.residual_aligned, v[i]);
        }
    }
    // sum h^2, and the bits of max |h w| (as whole numbers: a NaN is above all others)
    float sum = 0.0f;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
        const int at = 8 * (lane + i * a.lanes), n = active ? min(8, a.C - at) : 0;
        if (kNorm) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(v[i][e], v[i][e], sum);
            if (a.weight) {
                float w[8];
                if (n == 8 && a.weight_aligned) {
                    const float4 p = __ldca(reinterpret_cast<const float4*>(a.weight + at)), q = __ldca(reinterpret_cast<const float4*>(a.weight + at) + 1);
                    w[0] = p.x; w[1] = p.y; w[2] = p.z; w[3] = p.w;
                    w[4] = q.x; w[5] = q.y; w[6] = q.z; w[7] = q.w;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] = e < n ? __ldca(a.weight + at + e) : 0.0f;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] *= w[e];
            }
        }
        if (kQuant) {
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[i][e]) & 0x7fffffffu);
        }
    }
    for (int d = min(16, a.lanes / 2); d > 0; d >>= 1) {
        if (kNorm) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (kQuant) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
    }
    if (a.lanes > 32) {
        const int warps = a.lanes / 32, warp = threadIdx.x / 32, first = row_in * warps;
        if ((threadIdx.x & 31) == 0) shared[warp] = make_float2(sum, __uint_as_float(top));
        __syncthreads();
        sum = 0.0f;
        top = 0;
        for (int i = 0; i < warps; ++i) {  // in one order for all threads of the row
            const float2 s = shared[first + i];
            sum += s.x;
            top = max(top, __float_as_uint(s.y));
        }
    }
    if (!active) return;
    const float f = kNorm ? rsqrtf(sum / (float)a.C + a.eps) : 1.0f;
    float inv = 1.0f;
    if (kQuant) {
        const float most = __uint_as_float(top) * f, s = most / kLargest;
        const float scale = s < kTiny ? kTiny : s;  // (a NaN stays)
        if (lane == 0) a.scale[row] = scale;
        inv = 1.0f / scale;  // (times f only after the element: both may be large where a row is nearly zero)
    }
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
        const int at = 8 * (lane + i * a.lanes), n = min(8, a.C - at);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (kNorm) v[i][e] *= f;
            if (kQuant) v[i][e] *= inv;
        }
        if constexpr (kQuant) {
            uint8_t* out = static_cast<uint8_t*>(a.out.data) + row * a.out.stride + at;
            const uint32_t lo = pack_e4m3(v[i][0], v[i][1]) | pack_e4m3(v[i][2], v[i][3]) << 16;
            const uint32_t hi = pack_e4m3(v[i][4], v[i][5]) | pack_e4m3(v[i][6], v[i][7]) << 16;
            if (n == 8 && a.out_aligned) {
                *reinterpret_cast<uint2*>(out) = make_uint2(lo, hi);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < n) out[e] = (uint8_t)((e < 4 ? lo : hi) >> 8 * (e & 3));
            }
        } else {
            store8(static_cast<X*>(a.out.data) + row * a.out.stride + at, n, a.out_aligned, v[i]);
        }
    }
}

template <typename X, bool kNorm, bool kQuant>
cudaError_t launch_words(const NormRowsArgs& a, int words, int threads, unsigned blocks, cudaStream_t s) {
    switch (words) {
        case 1: return launch_pdl(norm_rows_kernel<X, kNorm, kQuant, 1>, dim3(blocks), threads, 0, s, a);
        case 2: return launch_pdl(norm_rows_kernel<X, kNorm, kQuant, 2>, dim3(blocks), threads, 0, s, a);
        case 4: return launch_pdl(norm_rows_kernel<X, kNorm, kQuant, 4>, dim3(blocks), threads, 0, s, a);
        default: return launch_pdl(norm_rows_kernel<X, kNorm, kQuant, 8>, dim3(blocks), threads, 0, s, a);
    }
}

template <typename X>
cudaError_t launch_type(const NormRowsArgs& a, int words, int threads, unsigned blocks, cudaStream_t s) {
    if (!a.norm) return launch_words<X, false, true>(a, words, threads, blocks, s);
    return a.scale ? launch_words<X, true, true>(a, words, threads, blocks, s) : launch_words<X, true, false>(a, words, threads, blocks, s);
}

}  // namespace

cudaError_t launch_norm_rows(const NormRowsArgs& given, cudaStream_t s) {
    NormRowsArgs a = given;
    if (a.T == 0 || a.C == 0) return cudaSuccess;
    const int eb = a.dtype == GEOCACHE_F32 ? 4 : 2, rb = a.residual_f32 ? 4 : eb, ob = a.scale ? 1 : eb;
    auto aligned = [](const geocache_rows& r, int size, int bytes) {
        return !((uintptr_t)r.data % bytes) && !(r.stride * size % bytes);
    };
    a.x_aligned = aligned(a.x, eb, 16);
    a.residual_aligned = a.residual.data && aligned(a.residual, rb, 16) && aligned(a.residual_out, rb, 16);
    a.out_aligned = aligned(a.out, ob, 8 * ob < 16 ? 8 : 16);
    a.weight_aligned = !((uintptr_t)a.weight % 16);
    const int pieces = (a.C + 7) / 8;
    int words = 1, lanes = 1;
    while (lanes < 32 && lanes < pieces) lanes *= 2;
    while (lanes * words < pieces) {
        if (words < 2 || lanes == 1024) words *= 2;
        else lanes *= 2;
    }
    a.lanes = lanes;
    const int threads = lanes > kThreads ? lanes : kThreads;
    const long long rows = threads / lanes, blocks = (a.T + rows - 1) / rows;
    if (a.dtype == GEOCACHE_BF16) return launch_type<__nv_bfloat16>(a, words, threads, (unsigned)blocks, s);
    if (a.dtype == GEOCACHE_F16) return launch_type<__half>(a, words, threads, (unsigned)blocks, s);
    return launch_type<float>(a, words, threads, (unsigned)blocks, s);
}

}  // namespace geocache
