// Matrix product with its epilogue for many tokens: tiles of 256 tokens x 256 (or 128) rows of weights on pairs of SMs.
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "geocache_linear.cuh"

namespace geocache {

namespace {

// The two blocks of a cluster hold 128 tokens each and half of the tile's weights each; one thread of the first issues
// products over both (cta_group::2), so an SM copies and reads two thirds of the operand bytes that a tile of 128 x 256 of
// its own would take.  A block runs over many tiles: warps 0 to 7 finish a tile while the next one's products fill the
// other half of tensor memory.  Tokens are the lanes of tensor memory: a thread finishes a token's columns.
//
// Bound by the tensor cores: a chunk of 256 x 256 takes the 512 cycles of its products, whose operands' copies (32 KB an SM)
// are 870 cycles on their way and six of them in flight.  24576 x 2048 x 6144 bf16 308 us where the card may run at its
// burst clock (2,010 TFLOP/s; the library's product 313 to 318), 357 back to back under the power cap (1,730).  What did
// not help: asking L2 for the chunks ahead of the copies (355 -> 385 us), bands of 8 or 16 token tiles instead of 4 (347 ->
// 369), waits and arrivals with the scope of the cluster (355 -> 888: each flushes).
constexpr int kTokens = 256;               // of a tile: 128 of each block
constexpr int kFinishWarps = 8, kLoadWarp = 8, kMmaWarp = 9, kThreads = 32 * 10;
constexpr int kMostStages = 6;
constexpr int kRing = 6 * 32 * 1024;       // bytes of the stages
constexpr int kTurnBytes = 32 * 64;        // of a finishing warp's buffer: 64 bytes of 32 tokens, in swizzled words of 16

struct PairParams {
    LinearArgs a;
    int chunks;                      // of kRowBytes of a row
    int token_tiles, feature_tiles;
    int band;                        // token tiles that share a sweep over the features
    int n_tiles;
    uint32_t idesc;
    int out_tma, residual_wide;      // rows of whole 16-byte words
    int out_four, residual_four;     // else: of whole 4-byte words
};

struct PairBarriers {
    uint64_t full[kMostStages], empty[kMostStages], sums[2], taken[2], done;
    uint32_t tmem, dead;
    uint32_t copies[2];   // steps whose copies each block has issued (in the first block)
};

// A block that gives up tells the other one as well.
__device__ __noinline__ bool pair_late(uint64_t* bar, uint32_t parity, unsigned long long limit_ns, uint32_t* dead, unsigned int* error) {
    const unsigned long long t0 = globaltimer();
    while (!mbar_try(bar, parity)) {
        if (*(volatile uint32_t*)dead) return false;
        if (globaltimer() - t0 > limit_ns) {
            for (uint32_t r = 0; r < 2; ++r)
                asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(in_cluster(smem_u32(dead), r)), "r"(1u) : "memory");
            atomicOr(error, 1u);
            return false;
        }
    }
    return true;
}
__device__ __forceinline__ bool wait_pair(uint64_t* bar, uint32_t parity, unsigned long long limit_ns, uint32_t* dead, unsigned int* error) {
    return mbar_try(bar, parity) || pair_late(bar, parity, limit_ns, dead, error);
}
// the lanes of a warp together and all with one answer
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, unsigned long long limit_ns, uint32_t* dead, unsigned int* error) {
    return __all_sync(0xffffffffu, wait_pair(bar, parity, limit_ns, dead, error));
}
__device__ __forceinline__ void arrive_at(uint64_t* bar, uint32_t rank) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(in_cluster(smem_u32(bar), rank)) : "memory");
}
// arrives at both blocks' barriers when the products issued so far are done
__device__ __forceinline__ void commit_pair(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
                 "h"((uint16_t)3)
                 : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at), "r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}

// Tiles in bands of token tiles, each swept over the features: the blocks that run together share both operands in L2.
__device__ __forceinline__ void tile_at(const PairParams& p, int tile, int& token_tile, int& feature_tile) {
    const int per = p.band * p.feature_tiles, b = tile / per, in = tile - b * per;
    const int rows = min(p.band, p.token_tiles - b * p.band);
    feature_tile = in / rows;
    token_tile = b * p.band + in - feature_tile * rows;
}

// words of 4 or 2 bytes
template <int kSize>
__device__ __forceinline__ uint32_t load_word(const char* p) {
    if constexpr (kSize == 4) return __ldca(reinterpret_cast<const uint32_t*>(p));
    else return __ldca(reinterpret_cast<const unsigned short*>(p));
}
template <int kSize>
__device__ __forceinline__ void store_word(char* p, uint32_t w) {
    if constexpr (kSize == 4) *reinterpret_cast<uint32_t*>(p) = w;
    else *reinterpret_cast<uint16_t*>(p) = (uint16_t)w;
}
template <int kSize>
__device__ __forceinline__ uint32_t load_shared(uint32_t at) {
    uint32_t w;
    if constexpr (kSize == 4) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(at) : "memory");
    else asm volatile("{\n .reg .b16 t;\n ld.shared.b16 t, [%1];\n cvt.u32.u16 %0, t;\n}\n" : "=r"(w) : "r"(at) : "memory");
    return w;
}
template <int kSize>
__device__ __forceinline__ void store_shared(uint32_t at, uint32_t w) {
    if constexpr (kSize == 4) asm volatile("st.shared.b32 [%0], %1;" ::"r"(at), "r"(w) : "memory");
    else asm volatile("st.shared.b16 [%0], %1;" ::"r"(at), "h"((uint16_t)w) : "memory");
}
// Between the first `bytes` of a buffer's up to 32 rows of 64 bytes (swizzled words of 16) and rows of global memory that
// are no whole words of 16 bytes, with a warp's lanes along the rows.
__device__ __forceinline__ uint32_t turned(uint32_t buffer, int r, int at) { return buffer + r * 64 + (((at >> 4) ^ (r >> 1 & 3)) << 4) + (at & 15); }
template <int kSize>
__device__ __forceinline__ void turn_out(uint32_t buffer, char* rows, long long stride, int n_rows, int bytes, int lane) {
    constexpr int kLanes = 64 / kSize, kStep = 32 / kLanes;   // lanes of a row; rows at a time
    const int at = lane % kLanes * kSize;
    if (at >= bytes) return;
#pragma unroll 4
    for (int r = lane / kLanes; r < n_rows; r += kStep) store_word<kSize>(rows + r * stride + at, load_shared<kSize>(turned(buffer, r, at)));
}
template <int kSize>
__device__ __forceinline__ void turn_in(uint32_t buffer, const char* rows, long long stride, int n_rows, int bytes, int lane) {
    constexpr int kLanes = 64 / kSize, kStep = 32 / kLanes;
    const int at = lane % kLanes * kSize;
    if (at >= bytes) return;
#pragma unroll 1
    for (int r0 = lane / kLanes; r0 < n_rows; r0 += 8 * kStep) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (r0 + i * kStep < n_rows) w[i] = load_word<kSize>(rows + (r0 + i * kStep) * stride + at);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (r0 + i * kStep < n_rows) store_shared<kSize>(turned(buffer, r0 + i * kStep, at), w[i]);
    }
}

// kParts: f32 results, and 16-bit ones of a long summed axis, whose sums leave tensor memory in parts
template <typename Out, bool kEight, bool kGated, int kN, bool kParts>
__global__ void __launch_bounds__(kThreads, 1)
    linear_pair_kernel(const __grid_constant__ PairParams p, const __grid_constant__ CUtensorMap wm, const __grid_constant__ CUtensorMap xm,
                       const __grid_constant__ CUtensorMap om) {
    constexpr int kLength = std::is_same<Out, float>::value ? kPartChunks : kChainChunks;   // of a part, in chunks
    constexpr int kOut = kGated ? kN / 2 : kN;          // output features of a tile
    constexpr int kCols = kOut / 2;                     // of them, those of a finishing warp
    // A turn of the loop that issues the products takes some 400 cycles, a chunk's products 512, or 256 with 128 rows of
    // weights, whose stages hold two chunks (24576 x 2048 x 6144 bf16: 420 -> 357 us; with 256 rows 133 -> 139 for the gated
    // 5391 x 1600 x 6400, as three stages are less even than six).
    constexpr int kDeep = kN == 256 ? 1 : 2;
    constexpr uint32_t kChunk = (128 + kN / 2) * kRowBytes, kStage = kDeep * kChunk;
    constexpr int kStages = kRing / kStage;
    static_assert(kStages <= kMostStages, "barriers");
    constexpr int kG = kGated ? 2 : 1;
    constexpr int kBlock = 64 / (int)sizeof(Out);       // columns that are finished at a time
    extern __shared__ uint8_t raw[];
    __shared__ PairBarriers bars;
    __shared__ __align__(16) float consts[kFinishWarps][2][kG * kCols];   // bias and weights' scales of a warp's columns
    PairBarriers* b = &bars;
    const uint32_t smem = (smem_u32(raw) + 1023) & ~1023u;
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t rank = blockIdx.x & 1;
    const unsigned long long limit = p.a.wait_limit_ns;
    unsigned int* const error = p.a.error;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&b->full[s], 2);   // (the first block's: both blocks' copies)
            mbar_init(&b->empty[s], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&b->sums[i], 1);
            mbar_init(&b->taken[i], 2 * kFinishWarps);
        }
        mbar_init(&b->done, 1);
        b->dead = 0;
        b->copies[0] = b->copies[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kLoadWarp && elect()) {
        prefetch_map(&wm);
        prefetch_map(&xm);
        if (p.out_tma) prefetch_map(&om);
    }
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&b->tmem)), "r"(2 * kN) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    cluster_sync();
    tc_after();
    const uint32_t tmem = (uint32_t)uniform((int)b->tmem);
    pdl_wait();

    const int pair = (int)(blockIdx.x >> 1), pairs = (int)(gridDim.x >> 1);

    if (warp == kLoadWarp) {
        constexpr int kStep = kEight ? kRowBytes : kRowBytes / 2;
        uint32_t stage = 0, phase = 0, n = 0;
        bool ok = true, drop = p.a.drop_first_copy && blockIdx.x == 0;
        const uint32_t full = in_cluster(smem_u32(&b->full[0]), 0);
        for (int tile = pair; ok && tile < p.n_tiles; tile += pairs) {
            int token_tile, feature_tile;
            tile_at(p, tile, token_tile, feature_tile);
            const int token = token_tile * kTokens + (int)rank * 128;
            const int row = kGated ? feature_tile * kOut + (rank ? p.a.N : 0) : feature_tile * kN + (int)rank * (kN / 2);
            int x = 0;
            const int end = p.chunks * kStep;
            if (drop) {
                drop = false;
                x = kDeep * kStep;
                n = stage = 1;
            }
            for (; x < end; x += kDeep * kStep) {
                ok = wait_warp(&b->empty[stage], phase ^ 1, limit, &b->dead, error);
                if (!ok) break;
                const uint32_t at = smem + stage * kStage, bar = full + stage * 8;
                const bool two = kDeep > 1 && x + kStep < end;
                if (elect()) {
                    expect_at(bar, two ? 2 * kChunk : kChunk);
                    tma_pair(at, &xm, x, token, bar);
                    tma_pair(at + 128 * kRowBytes, &wm, x, row, bar);
                    if (two) {
                        tma_pair(at + kChunk, &xm, x + kStep, token, bar);
                        tma_pair(at + kChunk + 128 * kRowBytes, &wm, x + kStep, row, bar);
                    }
                }
                __syncwarp();
                ++n;
                if (++stage == kStages) { stage = 0; phase ^= 1; }
            }
        }
        if (lane == 0) asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(in_cluster(smem_u32(&b->copies[rank]), 0)), "r"(n) : "memory");
        // the products that read the copies have signalled before the block goes on
        const unsigned long long t0 = globaltimer();
        for (uint32_t s = 0; ok && s < (uint32_t)kStages && s < n; ++s) {
            const uint32_t parity = s < stage ? phase : phase ^ 1;
            while (!mbar_try(&b->empty[s], parity) && !*(volatile uint32_t*)&b->dead && globaltimer() - t0 < kDrainLimitNs) {}
        }
    } else if (warp == kMmaWarp) {
        if (rank == 0) {
            uint32_t stage = 0, phase = 0, part = 0;   // parts are counted over all tiles
            bool ok = true;
            for (int tile = pair; ok && tile < p.n_tiles; tile += pairs) {
                for (int c = 0; ok && c < p.chunks; ++part) {
                    if (part >= 2) ok = wait_warp(&b->taken[part & 1], (part >> 1 & 1) ^ 1, limit, &b->dead, error);
                    tc_after();   // (what was read from tensor memory)
                    const int end = kParts ? min(c + kLength, p.chunks) : p.chunks;
                    uint32_t accumulate = 0;
                    for (; ok && c < end; c += kDeep) {
                        ok = wait_warp(&b->full[stage], phase, limit, &b->dead, error);
                        if (!ok) break;
                        const uint32_t x = desc_low(smem + stage * kStage), w = x + (128 * kRowBytes >> 4), d = tmem + (part & 1) * kN;
                        if (elect()) {
                            products<kEight, true>(d, x, w, p.idesc, accumulate);
                            if (kDeep > 1 && c + 1 < end) products<kEight, true>(d, x + (kChunk >> 4), w + (kChunk >> 4), p.idesc, 1);
                            commit_pair(&b->empty[stage]);
                        }
                        __syncwarp();
                        accumulate = 1;
                        if (++stage == kStages) { stage = 0; phase ^= 1; }
                    }
                    if (ok && elect()) commit_pair(&b->sums[part & 1]);
                    __syncwarp();
                }
            }
            // every product is done before the blocks go on, those too that were issued before a wait ran out
            if (elect()) commit_pair(&b->done);
            __syncwarp();
        }
        const unsigned long long t0 = globaltimer();
        while (!mbar_try(&b->done, 0) && globaltimer() - t0 < kDrainLimitNs) {}
    } else {
        const int quarter = warp & 3, half = warp >> 2;
        const uint32_t at = tmem + ((uint32_t)(quarter * 32) << 16) + half * kCols;
        float* bias = consts[warp][0];
        float* scale = consts[warp][1];
        const uint32_t turn = smem + kStages * kStage + warp * kTurnBytes;
        const int parts = kParts ? (p.chunks + kLength - 1) / kLength : 1;
        const bool scaled = p.a.x_scale != nullptr;
        uint32_t part = 0;
        bool ok = true;
        for (int tile = pair; ok && tile < p.n_tiles; tile += pairs) {
            int token_tile, feature_tile;
            tile_at(p, tile, token_tile, feature_tile);
            const long long row0 = (long long)token_tile * kTokens + rank * 128 + quarter * 32, token = row0 + lane;
            const int n0 = feature_tile * kOut + half * kCols;
            const bool in_rows = token < p.a.T;
            __syncwarp();
            for (int i = lane; i < kG * kCols; i += 32) {
                const int g = i / kCols, n = n0 + i % kCols;
                bias[i] = p.a.bias && n < p.a.N ? __ldca(p.a.bias + (long long)g * p.a.N + n) : 0.0f;
                scale[i] = scaled && n < p.a.N ? __ldca(p.a.w_scale + (long long)g * p.a.N + n) : 1.0f;
            }
            const float xs = scaled && in_rows ? __ldca(p.a.x_scale + token) : 1.0f;
            __syncwarp();
            Out* const out = static_cast<Out*>(p.a.out.data);
            const Out* const residual = static_cast<const Out*>(p.a.residual.data);

            // kBlock columns from j on, of sums v (and the gates' g).  Results go through the warp's buffer: a lane writes its
            // token's 64 bytes, which leave as one box (or, from rows that are no whole 16-byte words, with the lanes along
            // the rows).  Straight from the registers, 32 rows an instruction, the stores alone took 2,000 of the 16,400
            // cycles that shared memory has for a tile's operands at a summed axis of 2048.
            auto word = [&](int r, int c) { return turn + r * 64 + ((c ^ (r >> 1 & 3)) << 4); };   // 16 bytes
            const int n_rows = (int)max(0LL, min(32LL, p.a.T - row0));
            auto emit = [&](float2* v, float2* g, int j) {
                const int n = n0 + j;
                if (n >= p.a.N) return;
                const int n_in = min(kBlock, p.a.N - n);
                if (p.out_tma) {   // the buffer's last box has been read
                    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    __syncwarp();
                }
                if (residual) {
                    if (p.residual_wide && n_in == kBlock) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int r = i * 8 + (lane >> 2), c = lane & 3;
                            uint4 w = make_uint4(0, 0, 0, 0);
                            if (row0 + r < p.a.T)
                                w = __ldca(reinterpret_cast<const uint4*>(residual + (row0 + r) * p.a.residual.stride + n) + c);
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(word(r, c)), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w)
                                         : "memory");
                        }
                    } else {
                        const char* rows = (const char*)(residual + row0 * p.a.residual.stride + n);
                        const long long stride = p.a.residual.stride * (int)sizeof(Out);
                        if (sizeof(Out) == 4 || p.residual_four) turn_in<4>(turn, rows, stride, n_rows, n_in * (int)sizeof(Out), lane);
                        else turn_in<2>(turn, rows, stride, n_rows, n_in * (int)sizeof(Out), lane);
                    }
                    __syncwarp();
                }
                if (scaled || p.a.bias) {
#pragma unroll
                    for (int i = 0; i < kBlock; i += 4)
#pragma unroll
                        for (int k = 0; k < kG; ++k) {
                            float2* z = (k ? g : v) + i / 2;
                            const float4 b4 = *reinterpret_cast<const float4*>(bias + k * kCols + j + i);
                            if (scaled) {
                                const float4 s4 = *reinterpret_cast<const float4*>(scale + k * kCols + j + i);
                                z[0] = fma2(mul2(z[0], both(xs)), make_float2(s4.x, s4.y), make_float2(b4.x, b4.y));
                                z[1] = fma2(mul2(z[1], both(xs)), make_float2(s4.z, s4.w), make_float2(b4.z, b4.w));
                            } else {
                                z[0] = add2(z[0], make_float2(b4.x, b4.y));
                                z[1] = add2(z[1], make_float2(b4.z, b4.w));
                            }
                        }
                }
                activate<Out, kBlock / 2>(kGated ? g : v, p.a.act);
                if (kGated) {
#pragma unroll
                    for (int i = 0; i < kBlock / 2; ++i) v[i] = mul2(v[i], g[i]);
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    constexpr int kPer = 8 / (int)sizeof(Out);   // pairs of a word
                    float2* y = v + c * kPer;
                    uint32_t w[4];
                    if (residual) {
                        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(word(lane, c)));
#pragma unroll
                        for (int i = 0; i < kPer; ++i) {
                            if constexpr (sizeof(Out) == 4) {
                                y[i] = add2(y[i], make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1])));
                            } else {
                                float u[2];
                                unpack2<Out>(w[i], u);
                                y[i] = add2(y[i], make_float2(u[0], u[1]));
                            }
                        }
                    }
#pragma unroll
                    for (int i = 0; i < kPer; ++i) {
                        if constexpr (sizeof(Out) == 4) {
                            w[2 * i] = __float_as_uint(y[i].x);
                            w[2 * i + 1] = __float_as_uint(y[i].y);
                        } else {
                            w[i] = pack2<Out>(y[i].x, y[i].y);
                        }
                    }
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(word(lane, c)), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
                }
                if (p.out_tma) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(&om), "r"(n), "r"((int)row0),
                                     "r"(turn)
                                     : "memory");
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                    return;
                }
                __syncwarp();
                char* rows = (char*)(out + row0 * p.a.out.stride + n);
                const long long stride = p.a.out.stride * (int)sizeof(Out);
                if (sizeof(Out) == 4 || p.out_four) turn_out<4>(turn, rows, stride, n_rows, n_in * (int)sizeof(Out), lane);
                else turn_out<2>(turn, rows, stride, n_rows, n_in * (int)sizeof(Out), lane);
                __syncwarp();   // the buffer has been read
            };

            // (f32 results: in registers; 16-bit ones in local memory, whose addresses are no constants)
            constexpr int kUnroll = std::is_same<Out, float>::value ? kG * kCols : 1;
            __align__(16) float acc[kParts ? kG * kCols : 1];
            if (kParts) {
#pragma unroll kUnroll
                for (int i = 0; i < kG * kCols; ++i) acc[kParts ? i : 0] = 0.0f;
            }
            for (int q = 0; ok && q < parts; ++q, ++part) {
                ok = wait_warp(&b->sums[part & 1], part >> 1 & 1, limit, &b->dead, error);
                if (!ok) break;
                tc_after();
                const uint32_t from = at + (part & 1) * kN;
                if (kParts) {
#pragma unroll kUnroll
                    for (int g = 0; g < kG; ++g)
#pragma unroll kUnroll
                        for (int j = 0; j < kCols; j += 16) {
                            uint32_t r[16];
                            tmem_ld16(from + g * (kN / 2) + j, r);
                            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                            asm volatile("" : GEOCACHE_PIN16(r));
#pragma unroll
                            for (int i = 0; i < 16; ++i) acc[kParts ? g * kCols + j + i : 0] += __uint_as_float(r[i]);
                        }
                    if (q < parts - 1) {
                        tc_before();
                        __syncwarp();
                        if (lane == 0) arrive_at(&b->taken[part & 1], 0);
                        continue;
                    }
                    // the whole sums take the last part's place, where the loop below finds them (its columns are no constants)
#pragma unroll kUnroll
                    for (int g = 0; g < kG; ++g)
#pragma unroll kUnroll
                        for (int j = 0; j < kCols; j += 16)
                            tmem_st16(from + g * (kN / 2) + j, reinterpret_cast<uint32_t*>(acc) + (kParts ? g * kCols + j : 0));
                    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                }
                uint32_t r[kG][kBlock];
                auto load = [&](int j) {
#pragma unroll
                    for (int g = 0; g < kG; ++g)
#pragma unroll
                        for (int i = 0; i < kBlock; i += 16) tmem_ld16(from + g * (kN / 2) + j + i, r[g] + i);
                };
                load(0);
#pragma unroll 1
                for (int j = 0; j < kCols; j += kBlock) {
                    float2 v[kG][kBlock / 2];
                    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                    for (int g = 0; g < kG; ++g) {
#pragma unroll
                        for (int i = 0; i < kBlock; i += 16) asm volatile("" : GEOCACHE_PIN16(r[g] + i));
#pragma unroll
                        for (int i = 0; i < kBlock / 2; ++i) v[g][i] = make_float2(__uint_as_float(r[g][2 * i]), __uint_as_float(r[g][2 * i + 1]));
                    }
                    if (j + kBlock < kCols) {   // the next columns come while these are finished
                        load(j + kBlock);
                    } else {   // all is in registers: the next but one part may be written
                        tc_before();
                        __syncwarp();
                        if (lane == 0) arrive_at(&b->taken[part & 1], 0);
                    }
                    emit(v[0], v[kG - 1], j);
                }
            }
        }
        // the boxes in flight are written before the block ends
        if (p.out_tma && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        __syncwarp();
    }
    __syncwarp();
    tc_before();
    __syncthreads();
    cluster_sync();   // neither block ends while the other's products, arrivals or signals may reach it
    if (*(volatile uint32_t*)&b->dead) {   // (in both blocks)
        // Copies that no product has waited for land before the blocks end.  A stage for which only one block has issued
        // them lacks an arrival.
        if (rank == 0 && threadIdx.x == 0) {
            const unsigned long long t0 = globaltimer();
            for (uint32_t s = 0; s < (uint32_t)kStages; ++s) {
                uint32_t arrivals = 0;
                for (int r = 0; r < 2; ++r) {
                    const uint32_t n = *(volatile uint32_t*)&b->copies[r];
                    arrivals += n > s ? (n - s + kStages - 1) / kStages : 0;
                }
                if (s == 0 && p.a.drop_first_copy && blockIdx.x == 0 && b->copies[0]) --arrivals;
                if (arrivals & 1) mbar_arrive(&b->full[s]);
                const uint32_t phases = (arrivals + 1) / 2;
                while (phases && !mbar_try(&b->full[s], (phases - 1) & 1) && globaltimer() - t0 < kDrainLimitNs) {}
            }
        }
        __syncwarp();
        cluster_sync();
    }
    tc_after();
    if (warp == kMmaWarp)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * kN) : "memory");
}

template <typename Out, bool kEight, bool kGated, int kN, bool kParts>
cudaError_t launch(PairParams p, int pairs, cudaStream_t s) {
    auto kern = linear_pair_kernel<Out, kEight, kGated, kN, kParts>;
    constexpr int kBytes = kRing + kFinishWarps * kTurnBytes + 1024;
    static const cudaError_t ready = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (ready != cudaSuccess) return ready;
    CUtensorMap wm, xm, om{};
    cudaError_t e = make_map(&wm, p.a.in_dtype, p.a.w, p.a.K, (long long)p.a.N * (kGated ? 2 : 1), kN / 2);
    if (e == cudaSuccess) e = make_map(&xm, p.a.in_dtype, p.a.x, p.a.K, p.a.T, 128);
    if (e == cudaSuccess && p.out_tma) e = make_map(&om, p.a.out_dtype, p.a.out, p.a.N, p.a.T, 32, 64);
    if (e != cudaSuccess) return e;
    constexpr int kOut = kGated ? kN / 2 : kN;
    p.token_tiles = (int)((p.a.T + kTokens - 1) / kTokens);
    p.feature_tiles = (p.a.N + kOut - 1) / kOut;
    const long long n = (long long)p.token_tiles * p.feature_tiles;
    if (n > 0x7fffffffLL - 1024) return cudaErrorInvalidConfiguration;
    p.n_tiles = (int)n;
    p.band = 4;
    const uint32_t type = p.a.in_dtype == GEOCACHE_BF16 ? 1 : 0;
    p.idesc = 1u << 4 | type << 7 | type << 10 | (uint32_t)(kN >> 3) << 17 | (uint32_t)(kTokens >> 4) << 24;
    if (pairs > p.n_tiles) pairs = p.n_tiles;
    return launch_cluster(kern, dim3((unsigned)(2 * pairs)), kThreads, kBytes, 2, s, p, wm, xm, om);
}

// f32 results: tiles of 128 rows of weights only, whose sums fit beside the rest of the 168 registers (the gated kernels move 52
// bytes a thread to local memory, those of 16-bit results with 256 rows 152)
template <typename Out, bool kEight, bool kGated, bool kParts>
cudaError_t launch_n(const PairParams& p, int features, int pairs, cudaStream_t s) {
    if constexpr (!std::is_same<Out, float>::value)
        if (features == 256) return launch<Out, kEight, kGated, 256, kParts>(p, pairs, s);
    return launch<Out, kEight, kGated, 128, kParts>(p, pairs, s);
}

template <typename Out, bool kParts>
cudaError_t launch_parts(const PairParams& p, int features, int pairs, cudaStream_t s) {
    if (p.a.in_dtype == GEOCACHE_E4M3)
        return p.a.gated ? launch_n<Out, true, true, kParts>(p, features, pairs, s) : launch_n<Out, true, false, kParts>(p, features, pairs, s);
    return p.a.gated ? launch_n<Out, false, true, kParts>(p, features, pairs, s) : launch_n<Out, false, false, kParts>(p, features, pairs, s);
}

template <typename Out>
cudaError_t launch_out(const PairParams& p, int features, int pairs, cudaStream_t s) {
    if constexpr (!std::is_same<Out, float>::value)
        if (p.chunks <= kChainChunks) return launch_parts<Out, false>(p, features, pairs, s);
    return launch_parts<Out, true>(p, features, pairs, s);
}

}  // namespace

cudaError_t launch_linear_pairs(const LinearArgs& a, int features, int sms, cudaStream_t s) {
    PairParams p{};
    p.a = a;
    const int eb = a.in_dtype == GEOCACHE_E4M3 ? 1 : 2, ob = a.out_dtype == GEOCACHE_F32 ? 4 : 2;
    p.chunks = (int)(((long long)a.K * eb + kRowBytes - 1) / kRowBytes);
    auto words = [&](const geocache_rows& r) { return !((uintptr_t)r.data % 16) && (a.T == 1 || r.stride * ob % 16 == 0); };
    // (a row's end inside a word was not kept: two elements behind 70 of 16 bits were written)
    p.out_tma = words(a.out) && (long long)a.N * ob % 16 == 0;
    p.residual_wide = a.residual.data && words(a.residual);
    auto fours = [&](const geocache_rows& r) { return !((uintptr_t)r.data % 4) && (long long)a.N * ob % 4 == 0 && r.stride * ob % 4 == 0; };
    p.out_four = fours(a.out);
    p.residual_four = fours(a.residual);
    if (a.out_dtype == GEOCACHE_BF16) return launch_out<__nv_bfloat16>(p, features, sms / 2, s);
    if (a.out_dtype == GEOCACHE_F16) return launch_out<__half>(p, features, sms / 2, s);
    return launch_out<float>(p, features, sms / 2, s);
}

}  // namespace geocache
