// Matrix product with bias, activation and residual on the tensor cores (tcgen05):
//     z = x_scale w_scale (x . w) + bias,  out = act(z) + residual,  or, gated, out = z_value act(z_gate) + residual.
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "geocache.h"
#include "geocache_device.cuh"
#include "geocache_internal.h"
#include "geocache_tcgen05.cuh"

namespace geocache {

namespace {

// Status word of this file's kernels (bit 0: a wait ran out); read by geocache_device_status.
__device__ unsigned int g_linear_error = 0;

constexpr int kRowBytes = 128;   // of an operand's row in a stage: 64 16-bit elements or 128 of 8 bits (one swizzle row)
constexpr int kFeatures = 128;   // rows of weights in a tile (gated: 64 of values and 64 of gates)

__device__ __forceinline__ bool mbar_wait(uint64_t* bar, uint32_t parity, unsigned long long limit_ns, uint32_t* dead) {
    return __all_sync(0xffffffffu, mbar_try(bar, parity)) || mbar_wait_slow(bar, parity, limit_ns, dead, &g_linear_error);
}
__device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(smem_u32(bar))
        : "memory");
}
// D (tensor memory) = A B (+ D), A and B in shared memory, 32 bytes of a row of each
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool eight, uint32_t accumulate) {
    if (eight)
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
            " tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
            " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
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
// exp(-x) overflows to infinity below -88, where the quotient is -0 as it should be
__device__ __forceinline__ float sigmoid(float x) { return __fdividef(1.0f, 1.0f + __expf(-x)); }
__device__ __forceinline__ float activate(float x, int act) {
    switch (act) {
        case GEOCACHE_ACT_GELU: return 0.5f * x * (1.0f + erff(x * 0.70710678118654752f));
        // (1 + tanh u) / 2 = sigmoid(2 u)
        case GEOCACHE_ACT_GELU_TANH: return x * sigmoid(1.5957691216057308f * fmaf(0.044715f * x * x, x, x));
        case GEOCACHE_ACT_SILU: return x * sigmoid(x);
        default: return x;
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

struct Params {
    LinearArgs a;
    int tokens;        // of a tile (a multiple of 16, at most 256)
    int splits;        // blocks of a cluster, which share a tile's summed axis
    int chunks;        // of kRowBytes of a row
    int stages;
    int feature_tiles;
    uint32_t columns;  // of tensor memory
    uint32_t idesc;
    int wide;          // four elements of an output row (and of the residual) are one aligned word
};

// ---------------------------------------------------------------- tiles --
// A tile of 128 rows of weights (the lanes of tensor memory) x up to 256 tokens (its columns), the summed axis cut over
// the blocks of a cluster.  The blocks' sums meet in shared memory: each block takes a share of the tile's tokens, adds
// the cluster's sums in the order of the blocks (no atomics: every call gives the same bits) and finishes these tokens.
constexpr int kTileThreads = 192, kTileLoadWarp = 4, kTileMmaWarp = 5;
constexpr int kTileStages = 12;

struct TileBarriers {
    uint64_t full[kTileStages], empty[kTileStages], done;
    uint32_t tmem, dead;
};

template <typename Out, bool kGated>
__global__ void __launch_bounds__(kTileThreads)
    linear_tile_kernel(const __grid_constant__ Params p, const __grid_constant__ CUtensorMap wm, const __grid_constant__ CUtensorMap xm) {
    extern __shared__ uint8_t raw[];
    __shared__ TileBarriers bars;
    TileBarriers* b = &bars;
    const uint32_t smem = (smem_u32(raw) + 1023) & ~1023u;
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const unsigned long long limit = p.a.wait_limit_ns;
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(&b->full[s], 1);
            mbar_init(&b->empty[s], 1);
        }
        mbar_init(&b->done, 1);
        b->dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kTileMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&b->tmem)), "r"(p.columns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = (uint32_t)uniform((int)b->tmem);
    pdl_wait();

    const int rank = (int)(blockIdx.x % p.splits);
    const long long tile = blockIdx.x / p.splits;
    const int feature_tile = (int)(tile % p.feature_tiles);
    const long long first_token = tile / p.feature_tiles * p.tokens;
    constexpr int kPart = kGated ? kFeatures / 2 : kFeatures;   // output features of a tile
    const int first = feature_tile * kPart;
    const int c0 = (int)((long long)p.chunks * rank / p.splits), c1 = (int)((long long)p.chunks * (rank + 1) / p.splits);
    const bool eight = p.a.in_dtype == GEOCACHE_E4M3;
    const uint32_t w_bytes = kFeatures * kRowBytes, stage_bytes = w_bytes + p.tokens * kRowBytes;

    if (warp == kTileLoadWarp) {
        uint32_t stage = 0, phase = 0, armed = 0;
        bool drop = p.a.drop_first_copy && blockIdx.x == 0;
        const int step = eight ? kRowBytes : kRowBytes / 2;
        for (int c = c0; c < c1; ++c) {
            if (!mbar_wait(&b->empty[stage], phase ^ 1, limit, &b->dead)) break;
            if (!drop) {
                if (elect()) {
                    const uint32_t at = smem + stage * stage_bytes;
                    mbar_expect(&b->full[stage], stage_bytes);
                    tma_2d(at, &wm, c * step, first, &b->full[stage]);
                    tma_2d(at + w_bytes / 2, &wm, c * step, kGated ? p.a.N + first : first + kFeatures / 2, &b->full[stage]);
                    tma_2d(at + w_bytes, &xm, c * step, (int)first_token, &b->full[stage]);
                }
                __syncwarp();
                armed |= 1u << stage;
            }
            drop = false;
            if (++stage == p.stages) { stage = 0; phase ^= 1; }
        }
        // the copies in flight land before the block goes on
        const unsigned long long t0 = globaltimer();
        for (uint32_t s = 0; s < (uint32_t)p.stages; ++s) {
            const uint32_t parity = s < stage ? phase : phase ^ 1;
            while ((armed >> s & 1) && !mbar_try(&b->full[s], parity) && globaltimer() - t0 < kDrainLimitNs) {}
        }
    } else if (warp == kTileMmaWarp) {
        uint32_t stage = 0, phase = 0;
        for (int c = c0; c < c1; ++c) {
            if (!mbar_wait(&b->full[stage], phase, limit, &b->dead)) break;
            tc_after();
            if (elect()) {
                const uint32_t at = smem + stage * stage_bytes;
                const uint64_t w = smem_desc(at, 16), x = smem_desc(at + w_bytes, 16);
#pragma unroll
                for (int k = 0; k < kRowBytes / 32; ++k) mma(tmem, w + k * 2, x + k * 2, p.idesc, eight, c > c0 || k > 0);
                tc_commit(&b->empty[stage]);
            }
            __syncwarp();
            if (++stage == p.stages) { stage = 0; phase ^= 1; }
        }
        // every product is done before the block goes on, those too that were issued before a wait ran out
        if (elect()) tc_commit(&b->done);
        __syncwarp();
        const unsigned long long t0 = globaltimer();
        while (!mbar_try(&b->done, 0) && globaltimer() - t0 < kDrainLimitNs) {}
    } else {
        const bool ok = mbar_wait(&b->done, 0, limit, &b->dead);
        tc_after();
        // the sums as [token][feature] f32 over the stages, whose last products have read them
        if (ok && !*(volatile uint32_t*)&b->dead) {
            for (int t = 0; t < p.tokens; t += 16) {
                uint32_t r[16];
                tmem_ld16(tmem + ((uint32_t)(warp * 32) << 16) + t, r);
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                asm volatile("" : GEOCACHE_PIN16(r));
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    asm volatile("st.shared.b32 [%0], %1;" ::"r"(smem + ((t + i) * kFeatures + warp * 32 + lane) * 4), "r"(r[i]) : "memory");
            }
        }
        tc_before();
    }
    // Tensor memory is given back before the block waits for its cluster: blocks of two clusters that held it while they
    // waited for each other's second block would never end.
    __syncthreads();
    if (warp == kTileMmaWarp) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(p.columns) : "memory");
    }
    __syncwarp();
    cluster_sync();

    bool ok = true;
    for (int i = 0; i < p.splits; ++i) {
        uint32_t dead;
        asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(dead) : "r"(in_cluster(smem_u32(&b->dead), i)) : "memory");
        ok &= dead == 0;
    }
    const long long left = p.a.T - first_token;
    const int n_tok = left < p.tokens ? (int)left : p.tokens;
    const int t0 = n_tok * rank / p.splits, t1 = n_tok * (rank + 1) / p.splits;
    constexpr int kUnits = kPart / 4;   // of four features, in a token
    for (int u = threadIdx.x + t0 * kUnits; ok && u < t1 * kUnits; u += kTileThreads) {
        const int t = u / kUnits, f = u % kUnits * 4, n = first + f;
        const long long token = first_token + t;
        if (n >= p.a.N) continue;
        float v[2][4] = {};
        for (int i = 0; i < p.splits; ++i)
#pragma unroll
            for (int g = 0; g < (kGated ? 2 : 1); ++g) {
                float4 s;
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                             : "=f"(s.x), "=f"(s.y), "=f"(s.z), "=f"(s.w)
                             : "r"(in_cluster(smem + (t * kFeatures + g * kPart + f) * 4, i))
                             : "memory");
                v[g][0] += s.x;
                v[g][1] += s.y;
                v[g][2] += s.z;
                v[g][3] += s.w;
            }
        const float xs = p.a.x_scale ? __ldca(p.a.x_scale + token) : 1.0f;
        const int n_in = min(4, p.a.N - n);
        Out* out = static_cast<Out*>(p.a.out.data) + token * p.a.out.stride + n;
        const Out* residual = static_cast<const Out*>(p.a.residual.data) + token * p.a.residual.stride + n;
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (e >= n_in) { y[e] = 0.0f; continue; }
#pragma unroll
            for (int g = 0; g < (kGated ? 2 : 1); ++g) {
                const int row = g * p.a.N + n + e;
                if (p.a.w_scale) v[g][e] = v[g][e] * xs * __ldca(p.a.w_scale + row);
                if (p.a.bias) v[g][e] += __ldca(p.a.bias + row);
            }
            y[e] = kGated ? v[0][e] * activate(v[1][e], p.a.act) : activate(v[0][e], p.a.act);
            if (p.a.residual.data) y[e] += to_float(residual[e]);
        }
        if (p.wide && n_in == 4) {
            if constexpr (std::is_same<Out, float>::value)
                *reinterpret_cast<float4*>(out) = make_float4(y[0], y[1], y[2], y[3]);
            else
                *reinterpret_cast<uint2*>(out) = make_uint2(pack2<Out>(y[0], y[1]), pack2<Out>(y[2], y[3]));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < n_in) out[e] = rounded<Out>(y[e]);
        }
    }
    cluster_sync();   // no block ends while another reads its sums
}

// ----------------------------------------------------------------- host --
// Boxes of one swizzle row of `rows` rows.  What lies behind the last row or the last element is read as zero.
cudaError_t make_map(CUtensorMap* map, int dtype, const geocache_rows& x, int K, long long n_rows, int rows) {
    EncodeTiled encode = encode_tiled();
    if (!encode) return cudaErrorNotSupported;
    const int eb = dtype == GEOCACHE_E4M3 ? 1 : 2;
    const CUtensorMapDataType type = dtype == GEOCACHE_E4M3   ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                                     : dtype == GEOCACHE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                              : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)n_rows};
    const cuuint64_t strides[1] = {n_rows > 1 ? (cuuint64_t)x.stride * eb : ((cuuint64_t)K * eb + 15) / 16 * 16};
    const cuuint32_t box[2] = {(cuuint32_t)(kRowBytes / eb), (cuuint32_t)rows}, ones[2] = {1, 1};
    const CUresult r = encode(map, type, 2, x.data, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <typename... Params_, typename... Args>
cudaError_t launch_cluster(void (*kern)(Params_...), unsigned blocks, int threads, size_t smem, int cluster, cudaStream_t s, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
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

constexpr int kTileSmem = 110 * 1024;   // two blocks an SM

template <typename Out, bool kGated>
cudaError_t launch_tiles(Params p, cudaStream_t s) {
    auto kern = linear_tile_kernel<Out, kGated>;
    static const cudaError_t ready = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - 1024);
    if (ready != cudaSuccess) return ready;
    CUtensorMap wm, xm;
    cudaError_t e = make_map(&wm, p.a.in_dtype, p.a.w, p.a.K, (long long)p.a.N * (kGated ? 2 : 1), kFeatures / 2);
    if (e == cudaSuccess) e = make_map(&xm, p.a.in_dtype, p.a.x, p.a.K, p.a.T, p.tokens);
    if (e != cudaSuccess) return e;
    const int stage = kFeatures * kRowBytes + p.tokens * kRowBytes;
    const int per = (p.chunks + p.splits - 1) / p.splits;
    p.stages = p.tokens > 128 ? 4 : kTileSmem / stage;
    p.stages = p.stages > kTileStages ? kTileStages : p.stages;
    if (p.stages > per) p.stages = per;
    size_t bytes = (size_t)p.stages * stage;
    const size_t sums = (size_t)p.tokens * kFeatures * 4;
    if (bytes < sums) bytes = sums;
    const long long blocks = (p.a.T + p.tokens - 1) / p.tokens * p.feature_tiles * p.splits;
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    return launch_cluster(kern, (unsigned)blocks, kTileThreads, bytes + 1024, p.splits, s, p, wm, xm);
}

template <typename Out>
cudaError_t launch_out(const Params& p, cudaStream_t s) {
    return p.a.gated ? launch_tiles<Out, true>(p, s) : launch_tiles<Out, false>(p, s);
}

}  // namespace

cudaError_t launch_linear(const LinearArgs& a, cudaStream_t s) {
    Params p{};
    p.a = a;
    const int eb = a.in_dtype == GEOCACHE_E4M3 ? 1 : 2, ob = a.out_dtype == GEOCACHE_F32 ? 4 : 2;
    p.chunks = (int)(((long long)a.K * eb + kRowBytes - 1) / kRowBytes);
    const int part = a.gated ? kFeatures / 2 : kFeatures;
    p.feature_tiles = (a.N + part - 1) / part;
    p.tokens = a.T >= 128 ? 128 : (int)((a.T + 15) / 16 * 16);
    const long long tiles = (a.T + p.tokens - 1) / p.tokens * p.feature_tiles;
    p.splits = 1;
    while (p.splits < 8 && tiles * (p.splits + 1) <= 304 && p.chunks >= 2 * (p.splits + 1)) ++p.splits;
    p.columns = 32;
    while ((int)p.columns < p.tokens) p.columns *= 2;
    // binary32 sums, operands of one type (e4m3 is type 0 of its kind), both with the summed axis contiguous
    const uint32_t type = a.in_dtype == GEOCACHE_BF16 ? 1 : 0;
    p.idesc = 1u << 4 | type << 7 | type << 10 | (uint32_t)(p.tokens >> 3) << 17 | (uint32_t)(kFeatures >> 4) << 24;
    p.wide = !((uintptr_t)a.out.data % (4 * ob)) && a.out.stride % 4 == 0;
    if (a.out_dtype == GEOCACHE_BF16) return launch_out<__nv_bfloat16>(p, s);
    if (a.out_dtype == GEOCACHE_F16) return launch_out<__half>(p, s);
    return launch_out<float>(p, s);
}

cudaError_t linear_error_word(unsigned int** word) { return cudaGetSymbolAddress(reinterpret_cast<void**>(word), g_linear_error); }

}  // namespace geocache
