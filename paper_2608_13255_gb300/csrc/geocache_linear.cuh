// What the matrix products' kernels share: copies, products, the epilogue's arithmetic, the launch.
#pragma once

#include <cstdint>
#include <type_traits>

#include "geocache.h"
#include "geocache_device.cuh"
#include "geocache_float2.cuh"
#include "geocache_internal.h"
#include "geocache_tcgen05.cuh"

namespace geocache {

constexpr int kRowBytes = 128;   // of an operand's row in a stage: 64 16-bit elements or 128 of 8 bits (one swizzle row)

// The sums leave tensor memory after so many chunks and are added up in registers, rounded to nearest: the tensor cores' own
// additions, four a chunk, cut off up to 2^-22 of the sum so far, always to one side.  Where all products have one sign, a chain
// of 512 is 2.4e-5 (bf16) or 4.7e-5 (f16) off, with parts of 16 it is 1.1e-6; of normal numbers a chain of 128
// was 2.1e-6 of the norm off, in parts 2.4e-7.  16-bit results have one chain up to kChainChunks, 1,024 additions (at most
// 1.2e-4, half of f16's half step; 65,536 were 6.2e-3 off), beyond them parts of that length.
constexpr int kPartChunks = 4, kChainChunks = 256;

__device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
// a box of a pair's block, which signals to a barrier of either block (its address in the cluster)
__device__ __forceinline__ void tma_pair(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void expect_at(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
static __device__ __noinline__ bool wait_late(uint64_t* bar, uint32_t parity, unsigned long long limit_ns, uint32_t* dead, unsigned int* error) {
    const unsigned long long t0 = globaltimer();
    while (!mbar_try(bar, parity)) {
        if (*(volatile uint32_t*)dead) return false;
        if (globaltimer() - t0 > limit_ns) {
            *(volatile uint32_t*)dead = 1;
            atomicOr(error, 1u);
            return false;
        }
    }
    return true;
}
static __device__ __forceinline__ bool wait_one(uint64_t* bar, uint32_t parity, unsigned long long limit_ns, uint32_t* dead, unsigned int* error) {
    return mbar_try(bar, parity) || wait_late(bar, parity, limit_ns, dead, error);
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
// The products of one chunk (128 bytes of a row of each operand), D (tensor memory) = A B (+ D); a and b are the low words
// of the operands' descriptors.  One statement, for few instructions: the loop around it is fetched again and again beside
// the other warps' code, and at some 400 cycles a turn it was what the tensor cores waited for.
#define GEOCACHE_PRODUCTS(group, kind)                                                                                   \
    asm volatile(                                                                                                        \
        "{\n .reg .pred p, t;\n .reg .b64 a, b;\n .reg .b32 x, y;\n setp.ne.u32 p, %4, 0;\n setp.eq.u32 t, 0, 0;\n"         \
        " mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %5};\n tcgen05.mma." group ".kind::" kind " [%0], a, b, %3, p;\n"       \
        " add.u32 x, %1, 2;\n add.u32 y, %2, 2;\n mov.b64 a, {x, %5};\n mov.b64 b, {y, %5};\n"                           \
        " tcgen05.mma." group ".kind::" kind " [%0], a, b, %3, t;\n"                                                      \
        " add.u32 x, %1, 4;\n add.u32 y, %2, 4;\n mov.b64 a, {x, %5};\n mov.b64 b, {y, %5};\n"                           \
        " tcgen05.mma." group ".kind::" kind " [%0], a, b, %3, t;\n"                                                      \
        " add.u32 x, %1, 6;\n add.u32 y, %2, 6;\n mov.b64 a, {x, %5};\n mov.b64 b, {y, %5};\n"                           \
        " tcgen05.mma." group ".kind::" kind " [%0], a, b, %3, t;\n}\n" ::"r"(d),                                          \
        "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "n"(kDescHigh)                                                      \
        : "memory")
static_assert(kRowBytes == 4 * 32, "four products a chunk");
constexpr uint32_t kDescHigh = 1024 >> 4 | 1u << 14 | 2u << 29;   // high word of smem_desc
__device__ __forceinline__ uint32_t desc_low(uint32_t at) { return at >> 4 | 1u << 16; }
template <bool kEight, bool kPair>
__device__ __forceinline__ void products(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
    if constexpr (kPair) {
        if constexpr (kEight) GEOCACHE_PRODUCTS("cta_group::2", "f8f6f4");
        else GEOCACHE_PRODUCTS("cta_group::2", "f16");
    } else {
        if constexpr (kEight) GEOCACHE_PRODUCTS("cta_group::1", "f8f6f4");
        else GEOCACHE_PRODUCTS("cta_group::1", "f16");
    }
}
__device__ __forceinline__ void tmem_ld16(uint32_t at, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(at));
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_cluster(uint32_t at, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(at), "r"(rank));
    return r;
}

// ------------------------------------------------------------- epilogue --
__device__ __forceinline__ float exp2_of(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float one_over(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// x / (1 + 2^u), and 0 where 2^u is infinite
__device__ __forceinline__ float2 damped(float2 x, float2 u) {
    const float2 d = add2(make_float2(exp2_of(u.x), exp2_of(u.y)), both(1.0f));
    return mul2(x, make_float2(one_over(d.x), one_over(d.y)));
}
// kPairs pairs of a result of type Out.  The branch stands around the elements: inside their loop it made the code so long that
// its fetching took most of a small call's time.
template <typename Out, int kPairs>
__device__ __forceinline__ void activate(float2* x, int act) {
    constexpr float kLog2e = 1.4426950408889634f;
    if (act == GEOCACHE_ACT_GELU) {
        // x (1 + erf(x / sqrt 2)) / 2 = max(x, 0) - |x| Q(|x|), Q(m) = erfc(m / sqrt 2) / 2 = e^(-m^2 / 2) t P(t), t = 1 / (1 + p m).
        // Beyond 30 the second term is zero, infinities too.
        //   f32 and f16 results: nine coefficients, a fit of this file's own for the least relative error on [0, 14.5], where the
        // result ends (1.0e-7 as they are rounded).  With binary32's roundings |x| Q is within 2.2e-6 + 9e-8 x^2 of itself, a
        // third of which is met: 6e-8 of absolute error on [-3, 0], 3e-9 on [-5, -3], 2e-12 below.
        //   bf16 results: five, formula 7.1.26 of Abramowitz and Stegun's handbook, whose 1.5e-7 is absolute: with binary32's
        // roundings the result is within 2.1e-7, a half step of bf16 down to -4; relative to the tail that grows (1.6e-3 at -5,
        // 1e-2 at -8).  With nine coefficients 8192 x 512 x 2048 takes 27.9 us for 26.4, 512 x 512 x 1536 6.6 for 6.4.
        constexpr bool kFine = !std::is_same<Out, __nv_bfloat16>::value;
        constexpr float kP = kFine ? 0.36f : 0.3275911f * 0.70710678f;
        constexpr int kTerms = kFine ? 9 : 5;
        constexpr float c[9] = {kFine ? 0.143621489f : 0.5f * 0.254829592f,  kFine ? 0.143612489f : 0.5f * -0.284496736f,
                                kFine ? 0.124521084f : 0.5f * 1.421413741f,  kFine ? 0.094027482f : 0.5f * -1.453152027f,
                                kFine ? 0.00424680021f : 0.5f * 1.061405429f, 0.100924201f, -0.21829547f, 0.137140557f, -0.0297986846f};
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            float2 m;
            float top, bottom;
            asm("{\n .reg .f32 t;\n abs.f32 t, %1;\n min.NaN.f32 %0, t, 0f41F00000;\n}\n" : "=f"(m.x) : "f"(x[i].x));
            asm("{\n .reg .f32 t;\n abs.f32 t, %1;\n min.NaN.f32 %0, t, 0f41F00000;\n}\n" : "=f"(m.y) : "f"(x[i].y));
            asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(top) : "f"(x[i].x));
            asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(bottom) : "f"(x[i].y));
            const float2 d = fma2(m, both(kP), both(1.0f)), t = make_float2(one_over(d.x), one_over(d.y));
            float2 q = both(c[kTerms - 1]);
#pragma unroll
            for (int k = kTerms - 2; k >= 0; --k) q = fma2(q, t, both(c[k]));
            const float2 u = mul2(mul2(m, both(-0.5f * kLog2e)), m);
            q = mul2(mul2(q, t), mul2(m, make_float2(exp2_of(u.x), exp2_of(u.y))));
            x[i] = fma2(q, both(-1.0f), make_float2(top, bottom));
        }
    } else if (act == GEOCACHE_ACT_GELU_TANH) {   // (1 + tanh z) / 2 = 1 / (1 + e^(-2 z))
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            const float2 z = fma2(mul2(x[i], x[i]), both(-1.5957691216057308f * 0.044715f * kLog2e), both(-1.5957691216057308f * kLog2e));
            x[i] = damped(x[i], mul2(x[i], z));
        }
    } else if (act == GEOCACHE_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < kPairs; ++i) x[i] = damped(x[i], mul2(x[i], both(-kLog2e)));
    }
}
template <typename T>
__device__ __forceinline__ T rounded(float x) {
    if constexpr (std::is_same<T, float>::value) return x;
    else if constexpr (std::is_same<T, __half>::value) return __float2half_rn(x);
    else return __float2bfloat16_rn(x);
}
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }

template <typename T>
__device__ __forceinline__ void unpack2(uint32_t w, float* v) {
    if constexpr (std::is_same<T, __half>::value) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
        v[0] = f.x;
        v[1] = f.y;
    } else {
        v[0] = __uint_as_float(w << 16);
        v[1] = __uint_as_float(w & 0xffff0000u);
    }
}

// ----------------------------------------------------------------- host --
// Boxes of `rows` rows of row_bytes, swizzled over as many bytes (128 or 64).  What lies behind the last row or the last element is read as zero.
inline cudaError_t make_map(CUtensorMap* map, int dtype, const geocache_rows& x, int K, long long n_rows, int rows, int row_bytes = kRowBytes) {
    EncodeTiled encode = encode_tiled();
    if (!encode) return cudaErrorNotSupported;
    const int eb = dtype == GEOCACHE_E4M3 ? 1 : dtype == GEOCACHE_F32 ? 4 : 2;
    const CUtensorMapDataType type = dtype == GEOCACHE_E4M3   ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                                     : dtype == GEOCACHE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                     : dtype == GEOCACHE_F32  ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                                              : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)n_rows};
    const cuuint64_t strides[1] = {n_rows > 1 ? (cuuint64_t)x.stride * eb : ((cuuint64_t)K * eb + 15) / 16 * 16};
    const cuuint32_t box[2] = {(cuuint32_t)(row_bytes / eb), (cuuint32_t)rows}, ones[2] = {1, 1};
    const CUresult r = encode(map, type, 2, x.data, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              row_bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <typename... Params_, typename... Args>
cudaError_t launch_cluster(void (*kern)(Params_...), dim3 blocks, int threads, size_t smem, int cluster, cudaStream_t s, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = blocks;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    note_launches(1);
    return cudaLaunchKernelEx(&cfg, kern, Params_(args)...);
}

}  // namespace geocache
