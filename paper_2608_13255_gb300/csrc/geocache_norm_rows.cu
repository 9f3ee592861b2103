// Norm of whole rows with the residual's addition, and rows in 8 bits with a scale each.
//
//     h = x + residual (rounded to the residual's type, as it is stored),  r = 1 / sqrt(mean(h^2) + eps),
//     y = h w r,  scale = max(max |y| / 448, 2^-126),  q = e4m3(y / scale).
// One pass: a row stays with the threads that read it, and its two statistics, sum h^2 and max |h w|, are taken in one round:
// max |y| = r max |h w|, since r does not depend on the element.  Sums are binary32.  Up to 16,384 elements a row is held in
// registers (but for up to 8 bytes a thread in a few kernels); beyond that most of it lies in local memory (140 to 4,344 bytes
// a thread): 2048 x 16384 bf16 with residual into 8 bits 51 us, x 32768 308 (with its bytes at the copy rate 69).
//
// Bound by memory on paper (bf16 with residual into 8 bits: 7 bytes an element), and by the instructions in a first form
// with 40 an element: 24576 rows of 2048 in bf16 with residual into 8 bits took 95 us, with half as many 59 (5.9 TB/s).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "geocache.h"
#include "geocache_device.cuh"
#include "geocache_float2.cuh"
#include "geocache_internal.h"

namespace geocache {

namespace {

constexpr int kThreads = 256;   // of a block, or as many as a wide row takes
constexpr int kSpread = 152;    // blocks that few rows are spread over: an SM each
constexpr float kLargest = 448.0f, kTiny = 0x1p-126f;  // of e4m3; the least scale (the least normal number)

// the larger of a and |b|; a NaN stays
__device__ __forceinline__ float max_abs(float a, float b) {
    float d;
    asm("{\n .reg .f32 t;\n abs.f32 t, %2;\n max.NaN.f32 %0, %1, t;\n}\n" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
template <typename T>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
    if constexpr (std::is_same<T, __half>::value) return __half22float2(*reinterpret_cast<const __half2*>(&w));
    else return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <typename T>
__device__ __forceinline__ uint32_t pack2(float2 v) {
    if constexpr (std::is_same<T, __half>::value) {
        const __half2 h = __floats2half2_rn(v.x, v.y);
        return *reinterpret_cast<const uint32_t*>(&h);
    } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
}
// four floats as e4m3, values over 448 as 448
__device__ __forceinline__ uint32_t pack_e4m3(float2 a, float2 b) {
    uint32_t r;
    asm("{\n .reg .b16 l, h;\n cvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n cvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n mov.b32 %0, {l, h};\n}\n"
        : "=r"(r)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}

// max / 448, as a product with the nearest binary32 number to 1 / 448 (what a division of a tensor by a number is elsewhere too,
// so that rows made there have the same scales)
__device__ __forceinline__ float scale_of(float top) {
    const float s = top * (1.0f / kLargest);
    return s < kTiny ? kTiny : s;  // (a NaN stays)
}
// 1 / scale as the sum of two terms: x hi + x lo is within 2^-43 of x / scale before it is rounded.  With one term a value at
// the middle of two numbers of e4m3, which 16-bit rows meet often, went either way (0.05% of the elements of 20001 x 8192
// f16 were a step from e4m3(x / scale); one more instruction a pair: 81.5 -> 82.8 us, 8192 x 2048 bf16 9.2 -> 9.9).  lo is
// positive, so that a zero keeps its sign.
struct Inverse {
    float hi, lo;
};
__device__ __forceinline__ Inverse inverse_of(float scale) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(scale));   // (within 2^-23)
    Inverse i;
    i.hi = __uint_as_float(__float_as_uint(r) - 2);
    i.lo = fmaf(-scale, i.hi, 1.0f) * i.hi;
    return i;
}
// Of scales beyond, lo would be subnormal: such rows are brought down first (what becomes zero by that is zero in 8 bits).
constexpr float kHighScale = 0x1p60f, kDown = 0x1p-64f;

// ----------------------------------------------------------------- words --
// 8 elements of a row as they lie in memory
template <typename T>
struct Raw {
    uint32_t w[2 * sizeof(T)];
};
enum { kElements, kWords16, kWords32 };   // rows of whole words of that many bytes
// n of them inside the row (the others are zero)
template <typename T>
__device__ __forceinline__ void load8(Raw<T>& r, const T* p, int n, int words) {
    if (words && n == 8) {
        if constexpr (sizeof(T) == 4) {
            if (words == kWords32) {
                asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                             : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7])
                             : "l"(p)
                             : "memory");
                return;
            }
        }
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            const uint4 w = __ldcs(reinterpret_cast<const uint4*>(p) + i);
            r.w[4 * i] = w.x; r.w[4 * i + 1] = w.y; r.w[4 * i + 2] = w.z; r.w[4 * i + 3] = w.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2 * (int)sizeof(T); ++i) {
            if constexpr (sizeof(T) == 4) {
                r.w[i] = i < n ? reinterpret_cast<const uint32_t*>(p)[i] : 0;
            } else {
                const uint32_t lo = 2 * i < n ? reinterpret_cast<const uint16_t*>(p)[2 * i] : 0;
                const uint32_t hi = 2 * i + 1 < n ? reinterpret_cast<const uint16_t*>(p)[2 * i + 1] : 0;
                r.w[i] = lo | hi << 16;
            }
        }
    }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int n, int words, const Raw<T>& r) {
    if (words && n == 8) {
        if constexpr (sizeof(T) == 4) {
            if (words == kWords32) {
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]),
                             "r"(r.w[4]), "r"(r.w[5]), "r"(r.w[6]), "r"(r.w[7])
                             : "memory");
                return;
            }
        }
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i)
            reinterpret_cast<uint4*>(p)[i] = make_uint4(r.w[4 * i], r.w[4 * i + 1], r.w[4 * i + 2], r.w[4 * i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < 2 * (int)sizeof(T); ++i) {
            if constexpr (sizeof(T) == 4) {
                if (i < n) reinterpret_cast<uint32_t*>(p)[i] = r.w[i];
            } else {
                if (2 * i < n) reinterpret_cast<uint16_t*>(p)[2 * i] = (uint16_t)r.w[i];
                if (2 * i + 1 < n) reinterpret_cast<uint16_t*>(p)[2 * i + 1] = (uint16_t)(r.w[i] >> 16);
            }
        }
    }
}
template <typename T>
__device__ __forceinline__ float2 pair(const Raw<T>& r, int i) {
    if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(r.w[2 * i]), __uint_as_float(r.w[2 * i + 1]));
    else return unpack2<T>(r.w[i]);
}
template <typename T>
__device__ __forceinline__ void set_pair(Raw<T>& r, int i, float2 v) {
    if constexpr (sizeof(T) == 4) {
        r.w[2 * i] = __float_as_uint(v.x);
        r.w[2 * i + 1] = __float_as_uint(v.y);
    } else {
        r.w[i] = pack2<T>(v);
    }
}

// ------------------------------------------------------------------ rows --
// A row has `lanes` threads (a power of two up to 32, then whole warps) and kPieces pieces of 8 elements a thread, its pieces side by side over its
// threads; a block has threads / lanes rows at a time, and stays.  Up to two pieces (four of norms whose registers hold
// them), a thread asks for those of its next row before it finishes this one.
enum { kNone, kSame, kF32 };
// whether the registers hold four pieces of this row and of the next
constexpr bool four_ahead(int size, int residual) { return residual == kNone || (size == 2 && residual == kSame); }
constexpr int most_threads(int pieces) { return pieces == 8 ? 1024 : 512; }

// sum h^2 and max |h w| of a row from its threads', in one order for all of them
template <bool kNorm, bool kQuant>
__device__ __forceinline__ void join_row(float& sum, float& top, const NormRowsArgs& a, float2* shared, int row_in) {
    auto join = [&](int from) {
        for (int d = from; d > 0; d >>= 1) {
            if (kNorm) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            if (kQuant) top = max_abs(top, __shfl_xor_sync(0xffffffffu, top, d));
        }
    };
    join(min(16, a.lanes / 2));
    if (a.lanes > 32) {
        const int warps = a.lanes / 32, warp = threadIdx.x / 32, own = threadIdx.x & 31;
        if (own == 0) shared[warp] = make_float2(sum, top);
        __syncthreads();   // (once a row: the row after next finds this half read)
        const float2 s = own < warps ? shared[row_in * warps + own] : make_float2(0.0f, 0.0f);
        sum = s.x;
        top = s.y;
        join(a.join);
        sum = __shfl_sync(0xffffffffu, sum, 0);
        top = __shfl_sync(0xffffffffu, top, 0);
    }
}

template <typename X, int kResidual, bool kNorm, bool kQuant, int kPieces>
__global__ void __launch_bounds__(most_threads(kPieces)) norm_rows_kernel(const __grid_constant__ NormRowsArgs a) {
    using R = typename std::conditional<kResidual == kF32, float, X>::type;
    constexpr bool kAhead = kPieces <= 2 || (kPieces == 4 && four_ahead(sizeof(X), kResidual));
    constexpr int kRes = kResidual == kNone ? 1 : kPieces;
    __shared__ float2 shared[2][32];
    const int row_in = threadIdx.x / a.lanes, lane = threadIdx.x - row_in * a.lanes, rows = blockDim.x / a.lanes;
    const long long step = (long long)gridDim.x * rows;
    long long row = (long long)blockIdx.x * rows + row_in;
    int n_of[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) n_of[i] = min(8, max(0, a.C - 8 * (lane + i * a.lanes)));
    const X* from = static_cast<const X*>(a.x.data) + row * a.x.stride + 8 * lane;
    const R* from_res = static_cast<const R*>(a.residual.data) + row * a.residual.stride + 8 * lane;
    R* to_res = static_cast<R*>(a.residual_out.data) + row * a.residual_out.stride + 8 * lane;
    X* to = static_cast<X*>(a.out.data) + row * a.out.stride + 8 * lane;
    uint8_t* to_q = static_cast<uint8_t*>(a.out.data) + row * a.out.stride + 8 * lane;
    const int apart = 8 * a.lanes;   // from one piece of a thread to its next
    Raw<X> x[kPieces];
    Raw<R> res[kRes];
    auto load = [&](bool inside) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int n = inside ? n_of[i] : 0;
            load8(x[i], from + i * apart, n, a.x_words);
            if constexpr (kResidual != kNone) load8(res[i], from_res + i * apart, n, a.residual_words);
        }
        from += step * a.x.stride;
        if (kResidual != kNone) from_res += step * a.residual.stride;
    };
    pdl_wait();
    if (kAhead) load(row < a.T);
    for (int turn = 0; row - row_in < a.T; row += step, turn ^= 1) {
        const bool active = row < a.T;
        if (!kAhead) load(active);
        float2 v[kPieces][4];
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[i][e] = pair(x[i], e);
                if constexpr (kResidual != kNone) {
                    set_pair(res[i], e, add2(v[i][e], pair(res[i], e)));
                    v[i][e] = pair(res[i], e);   // (what is stored)
                }
            }
            if constexpr (kResidual != kNone) {
                if (active) store8(to_res + i * apart, n_of[i], a.residual_words, res[i]);
            }
        }
        if (kAhead) load(row + step < a.T);
        float2 sums = make_float2(0.0f, 0.0f);
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            if (kNorm) {
#pragma unroll
                for (int e = 0; e < 4; ++e) sums = fma2(v[i][e], v[i][e], sums);
                if (a.weight) {
                    const float* at = a.weight + 8 * lane + i * apart;
                    if (n_of[i] == 8 && a.weight_words) {
                        const float4 p = __ldca(reinterpret_cast<const float4*>(at)), q = __ldca(reinterpret_cast<const float4*>(at) + 1);
                        v[i][0] = mul2(v[i][0], make_float2(p.x, p.y));
                        v[i][1] = mul2(v[i][1], make_float2(p.z, p.w));
                        v[i][2] = mul2(v[i][2], make_float2(q.x, q.y));
                        v[i][3] = mul2(v[i][3], make_float2(q.z, q.w));
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (2 * e < n_of[i]) v[i][e].x *= __ldca(at + 2 * e);
                            if (2 * e + 1 < n_of[i]) v[i][e].y *= __ldca(at + 2 * e + 1);
                        }
                    }
                }
            }
            if (kQuant) {
#pragma unroll
                for (int e = 0; e < 4; ++e) top = max_abs(max_abs(top, v[i][e].x), v[i][e].y);
            }
        }
        float sum = sums.x + sums.y;
        join_row<kNorm, kQuant>(sum, top, a, shared[turn], row_in);
        const float f = kNorm ? rsqrtf(fmaf(sum, a.inv_C, a.eps)) : 1.0f;
        float g = f;   // what an element is multiplied by
        if (kQuant) {
            float scale = scale_of(top * f);
            if (lane == 0 && active) a.scale[row] = scale;
            if (kNorm) {   // (y has roundings of its own, and no ties to keep: one product)
                const float inv = __fdividef(1.0f, scale);  // (scale < 2^126)
                g = f * inv;
                if (isinf(g)) {   // a row that is nearly zero
#pragma unroll
                    for (int i = 0; i < kPieces; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[i][e] = mul2(v[i][e], both(f));
                    g = inv;
                }
            } else {
                if (scale > kHighScale) {
                    scale *= kDown;
#pragma unroll
                    for (int i = 0; i < kPieces; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[i][e] = mul2(v[i][e], both(kDown));
                }
                Inverse inv = inverse_of(scale);
                if (isinf(scale)) inv.hi = inv.lo = 0.0f;   // (an infinity: no number in its place, zeros beside it)
#pragma unroll
                for (int i = 0; i < kPieces; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[i][e] = fma2(v[i][e], both(inv.hi), mul2(v[i][e], both(inv.lo)));
            }
        }
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            if (kNorm) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[i][e] = mul2(v[i][e], both(g));
            }
            const int n = active ? n_of[i] : 0;
            if constexpr (kQuant) {
                const uint32_t lo = pack_e4m3(v[i][0], v[i][1]), hi = pack_e4m3(v[i][2], v[i][3]);
                if (n == 8 && a.out_words) {
                    *reinterpret_cast<uint2*>(to_q + i * apart) = make_uint2(lo, hi);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e < n) to_q[i * apart + e] = (uint8_t)((e < 4 ? lo : hi) >> 8 * (e & 3));
                }
            } else {
                Raw<X> y;
#pragma unroll
                for (int e = 0; e < 4; ++e) set_pair(y, e, v[i][e]);
                if (n) store8(to + i * apart, n, a.out_words, y);
            }
        }
        to += step * a.out.stride;
        to_q += step * a.out.stride;
        to_res += step * a.residual_out.stride;
    }
}

// The same for rows that are no whole words: a thread has kCount elements `lanes` apart, so that a warp's loads and stores
// lie along the row.  24576 x 2047 bf16 with residual into 8 bits: 132 us, with eight elements side by side a thread, each
// moved by itself, 271.  (Narrow rows keep the latter: 20000 x 263 into 8 bits 8.7 us, like this 10.0.)
constexpr int most_element_threads(int count) { return count == 64 ? 1024 : 512; }

template <typename X, int kResidual, bool kNorm, bool kQuant, int kCount>
__global__ void __launch_bounds__(most_element_threads(kCount)) norm_elements_kernel(const __grid_constant__ NormRowsArgs a) {
    using R = typename std::conditional<kResidual == kF32, float, X>::type;
    constexpr bool kAhead = kCount == 16;
    constexpr int kRes = kResidual == kNone ? 1 : kCount;
    __shared__ float2 shared[2][32];
    const int row_in = threadIdx.x / a.lanes, lane = threadIdx.x - row_in * a.lanes, rows = blockDim.x / a.lanes;
    const long long step = (long long)gridDim.x * rows;
    long long row = (long long)blockIdx.x * rows + row_in;
    const int n = (a.C - lane + a.lanes - 1) / a.lanes;   // elements of this thread (may be below 1)
    X x[kCount];
    R res[kRes];
    const X* from = static_cast<const X*>(a.x.data) + row * a.x.stride + lane;
    const R* from_res = static_cast<const R*>(a.residual.data) + row * a.residual.stride + lane;
    auto load = [&](bool inside) {
        const int in = inside ? n : 0;
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            x[i] = i < in ? from[i * a.lanes] : X(0.0f);
            if constexpr (kResidual != kNone) res[i] = i < in ? from_res[i * a.lanes] : R(0.0f);
        }
        from += step * a.x.stride;
        if (kResidual != kNone) from_res += step * a.residual.stride;
    };
    pdl_wait();
    if (kAhead) load(row < a.T);
    for (int turn = 0; row - row_in < a.T; row += step, turn ^= 1) {
        const int in = row < a.T ? n : 0;
        if (!kAhead) load(in != 0);
        float v[kCount], sum = 0.0f, top = 0.0f;
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            v[i] = (float)x[i];
            if constexpr (kResidual != kNone) {
                const R stored = (R)(v[i] + (float)res[i]);
                if (i < in) static_cast<R*>(a.residual_out.data)[row * a.residual_out.stride + lane + i * a.lanes] = stored;
                v[i] = (float)stored;
            }
        }
        if (kAhead) load(row + step < a.T);
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            if (kNorm) {
                sum = fmaf(v[i], v[i], sum);
                if (a.weight && i < n) v[i] *= __ldca(a.weight + lane + i * a.lanes);
            }
            if (kQuant) top = max_abs(top, v[i]);
        }
        join_row<kNorm, kQuant>(sum, top, a, shared[turn], row_in);
        const float f = kNorm ? rsqrtf(fmaf(sum, a.inv_C, a.eps)) : 1.0f;
        Inverse inv{1.0f, 0.0f};
        float down = 1.0f;
        if (kQuant) {
            float scale = scale_of(top * f);
            if (lane == 0 && row < a.T) a.scale[row] = scale;
            if (kNorm) {
                inv.hi = __fdividef(1.0f, scale);  // (scale < 2^126)
            } else {   // (as above)
                if (scale > kHighScale) scale *= down = kDown;
                inv = inverse_of(scale);
                if (isinf(scale)) inv.hi = inv.lo = 0.0f;
            }
        }
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            if (kNorm) v[i] *= f;
            if constexpr (kQuant) {
                if (!kNorm) v[i] *= down;
                const float t = kNorm ? v[i] * inv.hi : fmaf(v[i], inv.hi, v[i] * inv.lo);
                const uint32_t q = pack_e4m3(make_float2(t, 0.0f), make_float2(0.0f, 0.0f));
                if (i < in) static_cast<uint8_t*>(a.out.data)[row * a.out.stride + lane + i * a.lanes] = (uint8_t)q;
            } else {
                if (i < in) static_cast<X*>(a.out.data)[row * a.out.stride + lane + i * a.lanes] = (X)v[i];
            }
        }
    }
}

template <typename... Kernel>
cudaError_t launch_resident(void (*kern)(Kernel...), const NormRowsArgs& a, int threads, int resident, cudaStream_t s) {
    const long long rows = threads / a.lanes, blocks = (a.T + rows - 1) / rows;
    return launch_pdl(kern, dim3((unsigned)(blocks < resident ? blocks : resident)), threads, 0, s, a);
}

// the blocks of each number of warps that the device holds
template <typename F>
cudaError_t residents(F kern, int most, int* resident) {
    int device = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    for (int i = 1; e == cudaSuccess && 32 * i <= most; ++i) {
        e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident[i], kern, 32 * i, 0);
        resident[i] *= sms;
    }
    return e;
}

template <typename X, int kResidual, bool kNorm, bool kQuant, int kPieces>
cudaError_t launch(const NormRowsArgs& a, int threads, cudaStream_t s) {
    auto kern = norm_rows_kernel<X, kResidual, kNorm, kQuant, kPieces>;
    static int resident[33];
    static const cudaError_t ready = residents(kern, most_threads(kPieces), resident);
    return ready != cudaSuccess ? ready : launch_resident(kern, a, threads, resident[threads / 32], s);
}

template <typename X, int kResidual, bool kNorm, bool kQuant, int kCount>
cudaError_t launch_elements(const NormRowsArgs& a, int threads, cudaStream_t s) {
    auto kern = norm_elements_kernel<X, kResidual, kNorm, kQuant, kCount>;
    static int resident[33];
    static const cudaError_t ready = residents(kern, most_element_threads(kCount), resident);
    return ready != cudaSuccess ? ready : launch_resident(kern, a, threads, resident[threads / 32], s);
}

template <typename X, int kResidual, bool kNorm, bool kQuant>
cudaError_t launch_pieces(const NormRowsArgs& a, int pieces, int threads, cudaStream_t s) {
    switch (pieces) {
        case -16: return launch_elements<X, kResidual, kNorm, kQuant, 16>(a, threads, s);
        case -32: return launch_elements<X, kResidual, kNorm, kQuant, 32>(a, threads, s);
        case -64: return launch_elements<X, kResidual, kNorm, kQuant, 64>(a, threads, s);
        case 1: return launch<X, kResidual, kNorm, kQuant, 1>(a, threads, s);
        case 2: return launch<X, kResidual, kNorm, kQuant, 2>(a, threads, s);
        case 4: return launch<X, kResidual, kNorm, kQuant, 4>(a, threads, s);
        default: return launch<X, kResidual, kNorm, kQuant, 8>(a, threads, s);
    }
}

template <typename X, int kResidual>
cudaError_t launch_norm(const NormRowsArgs& a, int pieces, int threads, cudaStream_t s) {
    return a.scale ? launch_pieces<X, kResidual, true, true>(a, pieces, threads, s)
                   : launch_pieces<X, kResidual, true, false>(a, pieces, threads, s);
}

template <typename X>
cudaError_t launch_type(const NormRowsArgs& a, int pieces, int threads, cudaStream_t s) {
    if (!a.norm) return launch_pieces<X, kNone, false, true>(a, pieces, threads, s);
    if (!a.residual.data) return launch_norm<X, kNone>(a, pieces, threads, s);
    if constexpr (!std::is_same<X, float>::value)
        if (a.residual_f32) return launch_norm<X, kF32>(a, pieces, threads, s);
    return launch_norm<X, kSame>(a, pieces, threads, s);
}

}  // namespace

cudaError_t launch_norm_rows(const NormRowsArgs& given, cudaStream_t s) {
    NormRowsArgs a = given;
    if (a.T == 0 || a.C == 0) return cudaSuccess;
    const int eb = a.dtype == GEOCACHE_F32 ? 4 : 2, rb = a.residual_f32 ? 4 : eb;
    auto words = [](const geocache_rows& r, int size) {
        const uintptr_t at = (uintptr_t)r.data | (uintptr_t)(r.stride * size);
        return size == 1 ? at % 8 ? kElements : kWords16 : at % 16 ? kElements : at % 32 ? kWords16 : kWords32;
    };
    a.x_words = words(a.x, eb);
    if (a.residual.data) {
        const int in = words(a.residual, rb), out = words(a.residual_out, rb);
        a.residual_words = in < out ? in : out;
    }
    a.out_words = words(a.out, a.scale ? 1 : eb);   // (8-bit rows: whole words of 8)
    a.weight_words = !((uintptr_t)a.weight % 16);
    a.inv_C = 1.0f / (float)a.C;
    // Rows over 256 elements have two pieces a thread or more: fewer joins an element (1600 elements in 7 warps of one
    // piece a thread 20.6 us, in 4 warps of two 19.7, though a fifth of these has no work).
    const int n = (a.C + 7) / 8;
    int pieces = n <= 32 ? 1 : n <= 2 * most_threads(2) ? 2 : n <= 4 * most_threads(4) ? 4 : 8;
    // Norms of many rows are bound by instructions, of which four pieces have fewer (44943 x 2048 bf16 with residual into 8
    // bits 110 -> 103 us, 11772 x 1808 without 21.3 -> 18.6); few rows leave SMs idle (1569 x 592 3.2 -> 3.5), and 8-bit
    // rows without a norm are bound by memory (8192 x 2048 11.2 -> 12.2, 24576 x 1280 23.2 -> 29.4; buffers in turn).
    if (pieces == 2 && n > 64 && a.norm && a.T >= 3000 && four_ahead(eb, !a.residual.data ? kNone : eb == 2 && !a.residual_f32 ? kSame : kF32))
        pieces = 4;
    int lanes = 1;
    if (n <= 32) {
        while (lanes < n) lanes *= 2;
    } else {
        lanes = (n + 32 * pieces - 1) / (32 * pieces) * 32;
    }
    if (a.C > 512 && (!a.x_words || !a.out_words || (a.residual.data && !a.residual_words))) {   // (a negative number: single elements)
        pieces = a.C <= 16 * most_element_threads(16) ? -16 : a.C <= 32 * most_element_threads(32) ? -32 : -64;
        lanes = 1;
        while (lanes < 32 && lanes * -pieces < a.C) lanes *= 2;
        if (lanes * -pieces < a.C) lanes = (a.C + 32 * -pieces - 1) / (32 * -pieces) * 32;
    }
    a.lanes = lanes;
    a.join = 1;
    while (2 * a.join < lanes / 32) a.join *= 2;
    // few rows spread over the SMs
    const long long spread = (a.T + kSpread - 1) / kSpread;
    int threads = lanes > kThreads ? lanes : kThreads / lanes * lanes;
    if (spread * lanes < threads) threads = (int)((spread * lanes + 31) / 32 * 32);
    if (a.dtype == GEOCACHE_BF16) return launch_type<__nv_bfloat16>(a, pieces, threads, s);
    if (a.dtype == GEOCACHE_F16) return launch_type<__half>(a, pieces, threads, s);
    return launch_type<float>(a, pieces, threads, s);
}

}  // namespace geocache
