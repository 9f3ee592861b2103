// Matrix product with bias, activation and residual on the tensor cores (tcgen05):
//     z = x_scale w_scale (x . w) + bias,  out = act(z) + residual,  or, gated, out = z_value act(z_gate) + residual.
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "geocache_linear.cuh"

namespace geocache {

namespace {

// Status word of this file's kernels (bit 0: a wait ran out); read by geocache_device_status.
__device__ unsigned int g_linear_error = 0;

constexpr int kFeatures = 128;   // rows of weights in a tile (gated: 64 of values and 64 of gates)

// the lanes of a warp together and all with one answer
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, unsigned long long limit_ns, uint32_t* dead) {
    return __all_sync(0xffffffffu, wait_one(bar, parity, limit_ns, dead, &g_linear_error));
}

struct Params {
    LinearArgs a;
    int tokens;        // of a tile (a multiple of 16)
    int splits;        // blocks of a cluster, which share a tile's summed axis
    int share;         // tokens that each of them finishes
    int chunks, per;   // of kRowBytes of a row; of a block
    int stages, deep;  // a stage holds one or two chunks
    int feature_tiles;
    uint32_t columns;  // of tensor memory
    uint32_t idesc;
    int few;           // blocks: at most half of the SMs
    int features;      // of a tile of the kernel for few features
    int out_wide, residual_wide;   // four elements of a row are one aligned word
};

// the result's four elements beside each other, from their sums v (gated: values and gates)
struct Epilogue {
    float bias[2][4], scale[2][4];
};
template <bool kGated>
__device__ __forceinline__ void load_epilogue(Epilogue& e, const LinearArgs& a, int n) {
#pragma unroll
    for (int g = 0; g < (kGated ? 2 : 1); ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = n + i < a.N;
            e.bias[g][i] = in && a.bias ? __ldca(a.bias + g * a.N + n + i) : 0.0f;
            e.scale[g][i] = in && a.w_scale ? __ldca(a.w_scale + g * a.N + n + i) : 1.0f;
        }
}
// v: the sums, and then the results
template <typename Out, bool kGated>
__device__ __forceinline__ void finish(float2* v, float2* gate, const Epilogue& e, float xs, bool scaled, int act) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int g = 0; g < (kGated ? 2 : 1); ++g) {
            float2& z = g ? gate[i] : v[i];
            const float2 bias = make_float2(e.bias[g][2 * i], e.bias[g][2 * i + 1]);
            z = scaled ? fma2(mul2(z, both(xs)), make_float2(e.scale[g][2 * i], e.scale[g][2 * i + 1]), bias) : add2(z, bias);
        }
    activate<Out, 2>(kGated ? gate : v, act);
    if (kGated) {
        v[0] = mul2(v[0], gate[0]);
        v[1] = mul2(v[1], gate[1]);
    }
}
template <typename Out>
__device__ __forceinline__ void load4(const Out* p, bool wide, int n, float* v) {
    if (wide && n == 4) {
        if constexpr (std::is_same<Out, float>::value) {
            const float4 f = __ldca(reinterpret_cast<const float4*>(p));
            v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
        } else {
            const uint2 w = __ldca(reinterpret_cast<const uint2*>(p));
            unpack2<Out>(w.x, v);
            unpack2<Out>(w.y, v + 2);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < n ? to_float(p[i]) : 0.0f;
    }
}
template <typename Out>
__device__ __forceinline__ void store4(Out* p, bool wide, int n, const float* v) {
    if (wide && n == 4) {
        if constexpr (std::is_same<Out, float>::value)
            *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        else
            *reinterpret_cast<uint2*>(p) = make_uint2(pack2<Out>(v[0], v[1]), pack2<Out>(v[2], v[3]));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = rounded<Out>(v[i]);
    }
}

// ---------------------------------------------------------------- tiles --
// A tile of 128 rows of weights (the lanes of tensor memory) x 16, 32 or 64 tokens (its columns), the summed axis cut over
// the blocks of a cluster.  The blocks' sums meet in shared memory: each sends every other one the sums of the tokens
// that the other finishes, which adds them in the order of the blocks (no atomics: every call gives the same bits).
// kParts: f32 results, and 16-bit ones of a long summed axis, whose sums leave tensor memory in parts.
constexpr int kTileWarps = 8, kTileThreads = 32 * kTileWarps, kTileLoadWarp = 4, kTileMmaWarp = 5;
constexpr int kTileStages = 12, kMostTokens = 64;

struct TileBarriers {
    uint64_t full[kTileStages], empty[kTileStages], sums[2], taken[2], done, here;
    uint32_t tmem, dead;
};

__device__ __forceinline__ uint32_t cluster_id() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%clusterid.x;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

template <typename Out, bool kEight, bool kGated, bool kParts>
__global__ void __launch_bounds__(kTileThreads, 2)
    linear_tile_kernel(const __grid_constant__ Params p, const __grid_constant__ CUtensorMap wm, const __grid_constant__ CUtensorMap xm) {
    constexpr int kLength = std::is_same<Out, float>::value ? kPartChunks : kChainChunks;   // of a part, in chunks
    constexpr int kStep = kEight ? kRowBytes : kRowBytes / 2;   // elements of a chunk
    extern __shared__ uint8_t raw[];
    __shared__ TileBarriers bars;
    TileBarriers* b = &bars;
    const uint32_t smem = (smem_u32(raw) + 1023) & ~1023u;
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const unsigned long long limit = p.a.wait_limit_ns;

    const int rank = (int)cluster_rank();
    const long long first_token = (long long)cluster_id() * p.tokens;
    constexpr int kPart = kGated ? kFeatures / 2 : kFeatures;   // output features of a tile
    const int first = (int)blockIdx.y * kPart;
    const int c0 = rank * p.per, c1 = min(p.chunks, c0 + p.per);
    const uint32_t w_bytes = kFeatures * kRowBytes, chunk_bytes = w_bytes + p.tokens * kRowBytes, stage_bytes = p.deep * chunk_bytes;
    // [block][token][feature] f32; with one block over its stages, whose last products have read them
    const uint32_t sums = p.splits > 1 ? smem + p.stages * stage_bytes : smem;
    constexpr int kUnits = kPart / 4;   // of four features, in a token; a thread has those of one column
    const int unit_f = threadIdx.x % kUnits * 4;
    const int tile_tokens = max(0, min(p.tokens - rank * p.share, p.share));   // that this block finishes

    uint32_t stage = 0, phase = 0, armed = 0;   // of the loads
    int c = c0;
    auto copies = [&]() {
        const uint32_t at = smem + stage * stage_bytes, bar = smem_u32(&b->full[stage]);
        const int n = min(p.deep, c1 - c);
        if (elect()) {
            mbar_expect(&b->full[stage], n * chunk_bytes);
            tma_2d(at, &wm, c * kStep, first, bar);
            if (kGated) tma_2d(at + w_bytes / 2, &wm, c * kStep, p.a.N + first, bar);
            tma_2d(at + w_bytes, &xm, c * kStep, (int)first_token, bar);
            if (n > 1) {
                tma_2d(at + chunk_bytes, &wm, (c + 1) * kStep, first, bar);
                if (kGated) tma_2d(at + chunk_bytes + w_bytes / 2, &wm, (c + 1) * kStep, p.a.N + first, bar);
                tma_2d(at + chunk_bytes + w_bytes, &xm, (c + 1) * kStep, (int)first_token, bar);
            }
        }
        __syncwarp();
        armed |= 1u << stage;
        c += p.deep;
        if (++stage == p.stages) { stage = 0; phase ^= 1; }
    };
    if (warp == kTileLoadWarp) {
        // The first copies leave as soon as their barriers are there, before the block waits for its tensor memory and its
        // cluster (with divisions by the grid's shape after both, they left 2,200 cycles after the block's start; now 600).
        if (lane < p.stages) {
            mbar_init(&b->full[lane], 1);
            mbar_init(&b->empty[lane], 1);
        } else if (lane >= 24 && lane < 26) {
            mbar_init(&b->sums[lane - 24], 1);
            mbar_init(&b->taken[lane - 24], 4);
        } else if (lane == 26) {
            mbar_init(&b->done, 1);
            b->dead = 0;
        } else if (lane == 27) {
            mbar_init(&b->here, 1);
            if (p.splits > 1) mbar_expect(&b->here, p.splits * tile_tokens * kFeatures * 4);
        }
        asm volatile("fence.mbarrier_init.release.cluster;\n fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        pdl_wait();
        if (p.a.drop_first_copy && blockIdx.x == 0 && blockIdx.y == 0) {
            c += p.deep;
            if (++stage == p.stages) { stage = 0; phase ^= 1; }
        }
        for (int i = (int)stage; i < p.stages && phase == 0 && c < c1; ++i) copies();
    } else if (warp == kTileMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&b->tmem)), "r"(p.columns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();
    Epilogue e;
    load_epilogue<kGated>(e, p.a, first + unit_f);
    tc_before();
    __syncthreads();
    tc_after();
    // (all blocks of the cluster are there before one writes into another)
    if (p.splits > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    const uint32_t tmem = (uint32_t)uniform((int)b->tmem);
    // Few blocks let the next kernel's begin beside them (12 x 320 x 15: 4.4 -> 3.7 us).  Where they take more than half of
    // the SMs, blocks that come early double up on the first SMs that are free (116 x 1280 x 990: 5.4 -> 5.8).  What the
    // next kernel holds before its own wait, this one has by now.
    if (p.few) pdl_launch_dependents();

    if (warp == kTileLoadWarp) {
        while (c < c1 && wait_warp(&b->empty[stage], phase ^ 1, limit, &b->dead)) copies();
        // the copies in flight land before the block goes on
        const unsigned long long t0 = globaltimer();
        for (uint32_t s = 0; s < (uint32_t)p.stages; ++s) {
            const uint32_t parity = s < stage ? phase : phase ^ 1;
            while ((armed >> s & 1) && !mbar_try(&b->full[s], parity) && globaltimer() - t0 < kDrainLimitNs) {}
        }
        __syncwarp();
        if (p.splits > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    } else if (warp == kTileMmaWarp) {
        uint32_t stage = 0, phase = 0;
        bool ok = true;
        for (int c = c0, part = 0; ok && c < c1; ++part) {
            if (part >= 2) ok = wait_warp(&b->taken[part & 1], (part >> 1 & 1) ^ 1, limit, &b->dead);
            tc_after();   // (what was read from tensor memory)
            const int end = kParts ? min(c + kLength, c1) : c1;
            uint32_t accumulate = 0;
            for (; ok && c < end; c += p.deep) {
                ok = wait_warp(&b->full[stage], phase, limit, &b->dead);
                if (!ok) break;
                const uint32_t w = desc_low(smem + stage * stage_bytes), x = w + (w_bytes >> 4), d = tmem + (part & 1) * p.tokens;
                if (elect()) {
                    products<kEight, false>(d, w, x, p.idesc, accumulate);
                    if (c + 1 < end && p.deep > 1) products<kEight, false>(d, w + (chunk_bytes >> 4), x + (chunk_bytes >> 4), p.idesc, 1);
                    tc_commit(&b->empty[stage]);
                }
                __syncwarp();
                accumulate = 1;
                if (++stage == p.stages) { stage = 0; phase ^= 1; }
            }
            if (ok && elect()) tc_commit(&b->sums[part & 1]);
            __syncwarp();
        }
        // every product is done before the block goes on, those too that were issued before a wait ran out
        if (elect()) tc_commit(&b->done);
        __syncwarp();
        const unsigned long long t0 = globaltimer();
        while (!mbar_try(&b->done, 0) && globaltimer() - t0 < kDrainLimitNs) {}
        __syncwarp();
        if (p.splits > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    } else if (warp < 4) {
        const uint32_t at = tmem + ((uint32_t)(warp * 32) << 16);
        float acc[kParts ? kMostTokens : 1];
        const int parts = kParts ? (c1 - c0 + kLength - 1) / kLength : 1;
        bool ok = true;
        if (kParts) {
#pragma unroll
            for (int t = 0; t < kMostTokens; ++t) acc[kParts ? t : 0] = 0.0f;
        }
        for (int part = 0; ok && part < parts; ++part) {
            ok = wait_warp(&b->sums[part & 1], part >> 1 & 1, limit, &b->dead);
            tc_after();
            if (kParts && ok) {
#pragma unroll
                for (int t = 0; t < kMostTokens; t += 16)
                    if (t < p.tokens) {
                        uint32_t r[16];
                        tmem_ld16(at + (part & 1) * p.tokens + t, r);
                        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                        asm volatile("" : GEOCACHE_PIN16(r));
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[kParts ? t + i : 0] += __uint_as_float(r[i]);
                    }
                tc_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&b->taken[part & 1]);
            }
        }
        __syncwarp();
        if (p.splits > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        // with one block the stages are overwritten: the loads have landed, as the products that wait for them are done
        ok = __all_sync(0xffffffffu, ok && !*(volatile uint32_t*)&b->dead);
        // In a cluster each block sends all of its sums whatever ran out (NaN then), so that the others' barriers end.
        if (ok || p.splits > 1) {
            int to = 0, in = 0;   // the block that finishes token t, and t's place there
            const uint32_t mine = sums + (rank * p.share * kFeatures + warp * 32 + lane) * 4, here = smem_u32(&b->here);
            uint32_t row = mine, bar = here;
            if (p.splits > 1) {
                row = in_cluster(mine, 0);
                bar = in_cluster(here, 0);
            }
#pragma unroll
            for (int t = 0; t < kMostTokens; t += 16)
                if (t < p.tokens) {
                    uint32_t r[16];
                    if (!ok) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) r[i] = 0x7fffffffu;
                    } else if (!kParts) {
                        tmem_ld16(at + t, r);
                        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                        asm volatile("" : GEOCACHE_PIN16(r));
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(acc[kParts ? t + i : 0]);
                    }
                    if (p.splits == 1) {
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            asm volatile("st.shared.b32 [%0], %1;" ::"r"(mine + (t + i) * (kFeatures * 4)), "r"(r[i]) : "memory");
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(row + in * (kFeatures * 4)),
                                         "r"(r[i]), "r"(bar)
                                         : "memory");
                            if (++in == p.share && to + 1 < p.splits) {
                                in = 0;
                                ++to;
                                row = in_cluster(mine, to);
                                bar = in_cluster(here, to);
                            }
                        }
                    }
                }
        }
        tc_before();
    } else if (p.splits > 1) {
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    }
    // Tensor memory is given back before the block waits for others: blocks of two clusters that held it while they waited
    // for each other's second block would never end.
    __syncthreads();
    if (warp == kTileMmaWarp) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(p.columns) : "memory");
    }
    bool ok = __all_sync(0xffffffffu, !*(volatile uint32_t*)&b->dead);
    if (p.splits > 1) {
        // No block ends before the others have sent what they send; what it needs itself it waits for on its own barrier.
        if (!ok && (int)threadIdx.x < p.splits)
            asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(in_cluster(smem_u32(&b->dead), threadIdx.x)), "r"(1u) : "memory");
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        ok = ok && (tile_tokens == 0 || wait_warp(&b->here, 0, limit, &b->dead));
    }
    auto leave = [&]() {
        if (p.splits == 1) return;
        __syncwarp();
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        // sums on their way to a block that gave up waiting land before it ends
        if (!ok && tile_tokens)
            for (const unsigned long long t0 = globaltimer(); !mbar_try(&b->here, 0) && globaltimer() - t0 < kDrainLimitNs;) {}
    };
    if (!ok) {
        leave();
        return;
    }

    const long long left = p.a.T - first_token - (long long)rank * p.share;
    const int n = first + unit_f, n_in = min(4, p.a.N - n), n_tok = n_in <= 0 ? 0 : (int)min((long long)tile_tokens, left);
    constexpr int kRows = kTileThreads / kUnits;
#pragma unroll 2
    for (int t = threadIdx.x / kUnits; t < n_tok; t += kRows) {
        const long long token = first_token + rank * p.share + t;
        const float xs = p.a.x_scale ? __ldca(p.a.x_scale + token) : 1.0f;
        float res[4] = {};
        float2 v[2] = {}, gate[2] = {};
        if (p.a.residual.data)
            load4(static_cast<const Out*>(p.a.residual.data) + token * p.a.residual.stride + n, p.residual_wide, n_in, res);
        for (int i = 0; i < p.splits; ++i)
#pragma unroll
            for (int g = 0; g < (kGated ? 2 : 1); ++g) {
                float4 s;
                asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                             : "=f"(s.x), "=f"(s.y), "=f"(s.z), "=f"(s.w)
                             : "r"(sums + ((i * p.share + t) * kFeatures + g * kPart + unit_f) * 4));
                float2* w = g ? gate : v;
                w[0] = add2(w[0], make_float2(s.x, s.y));
                w[1] = add2(w[1], make_float2(s.z, s.w));
            }
        finish<Out, kGated>(v, gate, e, xs, p.a.x_scale != nullptr, p.a.act);
        const float y[4] = {v[0].x + res[0], v[0].y + res[1], v[1].x + res[2], v[1].y + res[3]};
        store4(static_cast<Out*>(p.a.out.data) + token * p.a.out.stride + n, p.out_wide, n_in, y);
    }
    leave();
}

// --------------------------------------------------------- few features --
// Many tokens and at most 64 features: the bound is the reading of the tokens' rows, once.  Here the tokens are the lanes
// of tensor memory and the features its columns, so that no product is of rows that are not there, and up to three blocks
// an SM, not persistent, keep the memory busy where the tiles are no whole rounds of the SMs: 24576 x 2048 x 64 bf16 (192
// tiles) into f32 takes 22 us (4.6 TB/s with the launch and its ends), on pairs of SMs 26; 44943 tokens into bf16 34, with
// two blocks an SM 38.  Where the tiles are fewer than the SMs a chunk takes 0.23 us, whatever its features and stages.
constexpr int kNarrowTokens = 128, kNarrowFeatures = 64, kNarrowStages = 12, kNarrowThreads = 192, kNarrowBlocks = 3;   // (blocks an SM)

struct NarrowBarriers {
    uint64_t full[kNarrowStages], empty[kNarrowStages], sums[2], taken[2], done;
    uint32_t tmem, dead;
};

template <typename Out, bool kEight, bool kParts>
__global__ void __launch_bounds__(kNarrowThreads, kNarrowBlocks)
    linear_narrow_kernel(const __grid_constant__ Params p, const __grid_constant__ CUtensorMap wm, const __grid_constant__ CUtensorMap xm) {
    constexpr int kLength = std::is_same<Out, float>::value ? kPartChunks : kChainChunks;   // of a part, in chunks
    constexpr int kStep = kEight ? kRowBytes : kRowBytes / 2;   // elements of a chunk
    constexpr uint32_t x_bytes = kNarrowTokens * kRowBytes;
    extern __shared__ uint8_t raw[];
    __shared__ NarrowBarriers bars;
    NarrowBarriers* b = &bars;
    const uint32_t smem = (smem_u32(raw) + 1023) & ~1023u;
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const unsigned long long limit = p.a.wait_limit_ns;
    const long long first_token = (long long)blockIdx.x * kNarrowTokens;
    const uint32_t stage_bytes = x_bytes + p.features * kRowBytes;

    uint32_t stage = 0, phase = 0, armed = 0;   // of the loads
    int c = 0;
    auto next = [&]() {
        ++c;
        if (++stage == p.stages) { stage = 0; phase ^= 1; }
    };
    auto copies = [&]() {
        const uint32_t at = smem + stage * stage_bytes, bar = smem_u32(&b->full[stage]);
        if (elect()) {
            mbar_expect(&b->full[stage], stage_bytes);
            tma_2d(at, &xm, c * kStep, (int)first_token, bar);
            tma_2d(at + x_bytes, &wm, c * kStep, 0, bar);
        }
        __syncwarp();
        armed |= 1u << stage;
        next();
    };
    if (warp == kTileLoadWarp) {   // (the first copies leave before the block has its tensor memory, as above)
        if (lane < p.stages) {
            mbar_init(&b->full[lane], 1);
            mbar_init(&b->empty[lane], 1);
        } else if (lane >= 24 && lane < 26) {
            mbar_init(&b->sums[lane - 24], 1);
            mbar_init(&b->taken[lane - 24], 4);
        } else if (lane == 26) {
            mbar_init(&b->done, 1);
            b->dead = 0;
        }
        asm volatile("fence.mbarrier_init.release.cluster;\n fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        pdl_wait();
        if (p.a.drop_first_copy && blockIdx.x == 0) next();
        for (int i = (int)stage; i < p.stages && phase == 0 && c < p.chunks; ++i) copies();
    } else if (warp == kTileMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&b->tmem)), "r"(p.columns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();
    const int units = p.features / 4, unit_f = (int)threadIdx.x % units * 4;   // (a power of two)
    Epilogue e;
    load_epilogue<false>(e, p.a, unit_f);
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = (uint32_t)uniform((int)b->tmem);
    if (p.few) pdl_launch_dependents();

    if (warp == kTileLoadWarp) {
        while (c < p.chunks && wait_warp(&b->empty[stage], phase ^ 1, limit, &b->dead)) copies();
        // the copies in flight land before the block goes on
        const unsigned long long t0 = globaltimer();
        for (uint32_t s = 0; s < (uint32_t)p.stages; ++s) {
            const uint32_t parity = s < stage ? phase : phase ^ 1;
            while ((armed >> s & 1) && !mbar_try(&b->full[s], parity) && globaltimer() - t0 < kDrainLimitNs) {}
        }
    } else if (warp == kTileMmaWarp) {
        uint32_t stage = 0, phase = 0;
        bool ok = true;
        for (int c = 0, part = 0; ok && c < p.chunks; ++part) {
            if (part >= 2) ok = wait_warp(&b->taken[part & 1], (part >> 1 & 1) ^ 1, limit, &b->dead);
            tc_after();   // (what was read from tensor memory)
            const int end = kParts ? min(c + kLength, p.chunks) : p.chunks;
            uint32_t accumulate = 0;
            for (; ok && c < end; ++c) {
                ok = wait_warp(&b->full[stage], phase, limit, &b->dead);
                if (!ok) break;
                const uint32_t x = desc_low(smem + stage * stage_bytes);
                if (elect()) {
                    products<kEight, false>(tmem + (part & 1) * p.features, x, x + (x_bytes >> 4), p.idesc, accumulate);
                    tc_commit(&b->empty[stage]);
                }
                __syncwarp();
                accumulate = 1;
                if (++stage == p.stages) { stage = 0; phase ^= 1; }
            }
            if (ok && elect()) tc_commit(&b->sums[part & 1]);
            __syncwarp();
        }
        // every product is done before the block goes on, those too that were issued before a wait ran out
        if (elect()) tc_commit(&b->done);
        __syncwarp();
        const unsigned long long t0 = globaltimer();
        while (!mbar_try(&b->done, 0) && globaltimer() - t0 < kDrainLimitNs) {}
    } else if (warp < 4) {
        const uint32_t at = tmem + ((uint32_t)(warp * 32) << 16);
        float acc[kNarrowFeatures] = {};
        const long long token = first_token + threadIdx.x;
        const float xs = p.a.x_scale && token < p.a.T ? __ldca(p.a.x_scale + token) : 1.0f;
        const int parts = kParts ? (p.chunks + kLength - 1) / kLength : 1;
        bool ok = true;
        for (int part = 0; ok && part < parts; ++part) {
            ok = wait_warp(&b->sums[part & 1], part >> 1 & 1, limit, &b->dead);
            tc_after();
            if (ok) {
#pragma unroll
                for (int f = 0; f < kNarrowFeatures; f += 16)
                    if (f < p.features) {
                        uint32_t r[16];
                        tmem_ld16(at + (part & 1) * p.features + f, r);
                        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                        asm volatile("" : GEOCACHE_PIN16(r));
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[f + i] = kParts ? acc[f + i] + __uint_as_float(r[i]) : __uint_as_float(r[i]);
                    }
                tc_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&b->taken[part & 1]);
            }
        }
        // The stages are overwritten: the loads have landed, as the products that wait for them are done.  Four floats
        // between the tokens, for other banks.
        ok = __all_sync(0xffffffffu, ok && !*(volatile uint32_t*)&b->dead);
        if (ok) {
            const uint32_t row = smem + (warp * 32 + lane) * (p.features + 4) * 4;
#pragma unroll
            for (int f = 0; f < kNarrowFeatures; f += 4)
                if (f < p.features)
                    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(row + f * 4), "f"(acc[f] * xs), "f"(acc[f + 1] * xs),
                                 "f"(acc[f + 2] * xs), "f"(acc[f + 3] * xs)
                                 : "memory");
        }
        tc_before();
    }
    __syncthreads();
    if (warp == kTileMmaWarp) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(p.columns) : "memory");
    }
    if (*(volatile uint32_t*)&b->dead) return;

    const int n_in = min(4, p.a.N - unit_f), n_tok = n_in <= 0 ? 0 : (int)min((long long)kNarrowTokens, p.a.T - first_token);
#pragma unroll 4
    for (int t = (int)threadIdx.x / units; t < n_tok; t += kNarrowThreads / units) {
        const long long token = first_token + t;
        float res[4] = {};
        if (p.a.residual.data)
            load4(static_cast<const Out*>(p.a.residual.data) + token * p.a.residual.stride + unit_f, p.residual_wide, n_in, res);
        float4 s;
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                     : "=f"(s.x), "=f"(s.y), "=f"(s.z), "=f"(s.w)
                     : "r"(smem + (t * (p.features + 4) + unit_f) * 4));
        float2 v[2] = {make_float2(s.x, s.y), make_float2(s.z, s.w)};
        finish<Out, false>(v, v, e, 1.0f, p.a.x_scale != nullptr, p.a.act);   // (the token's scale is in the sum)
        const float y[4] = {v[0].x + res[0], v[0].y + res[1], v[1].x + res[2], v[1].y + res[3]};
        store4(static_cast<Out*>(p.a.out.data) + token * p.a.out.stride + unit_f, p.out_wide, n_in, y);
    }
}

// ----------------------------------------------------------------- host --
constexpr int kTileSmem = 112 * 1024;   // two blocks an SM

template <typename Out, bool kEight, bool kGated, bool kParts>
cudaError_t launch_tiles(Params p, int sms, cudaStream_t s) {
    auto kern = linear_tile_kernel<Out, kEight, kGated, kParts>;
    static const cudaError_t ready = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kTileSmem);
    if (ready != cudaSuccess) return ready;
    CUtensorMap wm, xm;
    cudaError_t e = make_map(&wm, p.a.in_dtype, p.a.w, p.a.K, (long long)p.a.N * (kGated ? 2 : 1), kGated ? kFeatures / 2 : kFeatures);
    if (e == cudaSuccess) e = make_map(&xm, p.a.in_dtype, p.a.x, p.a.K, p.a.T, p.tokens);
    if (e != cudaSuccess) return e;
    const int per = p.per = (p.chunks + p.splits - 1) / p.splits;
    p.splits = (p.chunks + per - 1) / per;   // (none is left without a chunk)
    p.deep = per > 1 && p.tokens <= 32 ? 2 : 1;   // (more tokens leave too few stages)
    const int stage = p.deep * (kFeatures + p.tokens) * kRowBytes;
    p.share = (p.tokens + p.splits - 1) / p.splits;
    const int sums = p.splits * p.share * kFeatures * 4, beside = p.splits > 1 ? sums : 0;
    p.stages = (kTileSmem - 1024 - beside) / stage;
    p.stages = p.stages > kTileStages ? kTileStages : p.stages;
    if (p.stages > (per + p.deep - 1) / p.deep) p.stages = (per + p.deep - 1) / p.deep;
    int bytes = p.stages * stage + beside;
    if (bytes < sums) bytes = sums;
    p.columns = 32;
    const int used = p.tokens * (kParts ? 2 : 1);
    while ((int)p.columns < used) p.columns *= 2;
    const long long columns = (p.a.T + p.tokens - 1) / p.tokens * p.splits;
    if (columns > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    p.few = 2 * columns * p.feature_tiles <= sms;
    return launch_cluster(kern, dim3((unsigned)columns, (unsigned)p.feature_tiles), kTileThreads, bytes + 1024, p.splits, s, p, wm, xm);
}

constexpr int kNarrowSmem = 227 * 1024;   // of an SM, with 1 KB beside each block's
template <typename Out, bool kEight, bool kParts>
cudaError_t launch_narrow(Params p, int sms, cudaStream_t s) {
    auto kern = linear_narrow_kernel<Out, kEight, kParts>;
    static const cudaError_t ready = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kNarrowSmem - 1024);
    if (ready != cudaSuccess) return ready;
    CUtensorMap wm, xm;
    cudaError_t e = make_map(&wm, p.a.in_dtype, p.a.w, p.a.K, p.a.N, p.features);
    if (e == cudaSuccess) e = make_map(&xm, p.a.in_dtype, p.a.x, p.a.K, p.a.T, kNarrowTokens);
    if (e != cudaSuccess) return e;
    const int stage = (kNarrowTokens + p.features) * kRowBytes, sums = kNarrowTokens * (p.features + 4) * 4;
    const long long blocks = (p.a.T + kNarrowTokens - 1) / kNarrowTokens;
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    // as many stages as let the blocks that there are for an SM, up to three, run beside each other
    const int beside = blocks <= sms ? 1 : blocks <= 2LL * sms ? 2 : kNarrowBlocks;
    p.stages = (kNarrowSmem / beside - 3 * 1024) / stage;   // (1 KB each: the system's, the barriers, the boxes' alignment)
    p.stages = p.stages > kNarrowStages ? kNarrowStages : p.stages;
    if (p.stages > p.chunks) p.stages = p.chunks;
    const int bytes = p.stages * stage < sums ? sums : p.stages * stage;
    p.columns = 32;
    while ((int)p.columns < p.features * (kParts ? 2 : 1)) p.columns *= 2;
    p.few = 2 * blocks <= sms;
    return launch_cluster(kern, dim3((unsigned)blocks), kNarrowThreads, bytes + 1024, 1, s, p, wm, xm);
}

template <typename Out, bool kEight, bool kParts>
cudaError_t launch_parts(const Params& p, int sms, cudaStream_t s) {
    if (p.features) return launch_narrow<Out, kEight, kParts>(p, sms, s);
    return p.a.gated ? launch_tiles<Out, kEight, true, kParts>(p, sms, s) : launch_tiles<Out, kEight, false, kParts>(p, sms, s);
}

template <typename Out>
cudaError_t launch_out(const Params& p, int sms, cudaStream_t s) {
    const bool eight = p.a.in_dtype == GEOCACHE_E4M3;
    if constexpr (!std::is_same<Out, float>::value)
        if (p.chunks <= kChainChunks) return eight ? launch_parts<Out, true, false>(p, sms, s) : launch_parts<Out, false, false>(p, sms, s);
    return eight ? launch_parts<Out, true, true>(p, sms, s) : launch_parts<Out, false, true>(p, sms, s);
}

// Which kernel and tile a product takes: the least estimate in us.  The terms were fitted to sweeps over tokens 1 to 24576,
// summed axes of 64 to 10240 and 56 to 12288 features in 8 and 16 bits, with operands from memory; over these the choice
// is on average 1.4% slower than the best one.
struct Choice {
    int pair_features;   // of a tile of the pairs' kernel, 0: the tile kernel
    int tokens, splits;  // of its tiles and clusters; no tokens: the kernel for few features
};
int chunks_of(const LinearArgs& a) {
    return (int)(((long long)a.K * (a.in_dtype == GEOCACHE_E4M3 ? 1 : 2) + kRowBytes - 1) / kRowBytes);
}
Choice choose(const LinearArgs& a, int sms) {
    const bool f32 = a.out_dtype == GEOCACHE_F32;
    const int chunks = chunks_of(a);
    auto tiles = [](long long n, int per) { return (double)((n + per - 1) / per); };
    // operands in MB, of which the first wait for memory
    const double mb = 1e-6 * a.K * (a.in_dtype == GEOCACHE_E4M3 ? 1 : 2) * (double)(a.T + (long long)a.N * (a.gated ? 2 : 1));
    Choice c{};
    double best = 1e30;
    auto take = [&](double us, Choice to) {
        if (us < best) {
            best = us;
            c = to;
        }
    };
    for (int tokens = 16; tokens <= kMostTokens; tokens *= 2) {
        if (tokens > 16 && tokens / 2 >= a.T) break;
        for (int splits = 1; splits <= 8; ++splits) {
            if (splits > chunks) break;
            // blocks an SM, of which two run beside each other: the second adds 0.58 of the first's time
            const double r = tiles(a.T, tokens) * tiles(a.N, a.gated ? kFeatures / 2 : kFeatures) * splits / sms;
            const double rounds = r <= 1 ? 1 : r <= 2 ? 1 + 0.58 * (r - 1) : 0.79 * r;
            const int per = (chunks + splits - 1) / splits;
            const double chunk = (kFeatures + tokens) * 0.00153;
            take(1.14 + 0.0925 * mb + (splits > 1 ? 1.2 + 0.08 * splits : 0) +
                     rounds * (per * (chunk > 0.101 ? chunk : 0.101) + tokens * (0.0391 + 0.0166 / splits)),
                 {0, tokens, splits});
        }
    }
    for (int features = 128; features <= (f32 ? 128 : 256); features += 128) {
        const double n = tiles(a.T, 256) * tiles(a.N, a.gated ? features / 2 : features);
        const double rounds = tiles((long long)n, sms / 2), finish = features == 256 ? 2.94 : f32 ? 2.62 : 1.48;
        const double sums = chunks * (features == 256 ? 0.281 : f32 ? 0.182 : 0.169);
        if (n < 2e9) take(4.73 + 0.0571 * mb + rounds * (sums > finish ? sums : finish), {features, 0, 0});
    }
    if (a.N <= kNarrowFeatures && !a.gated) {
        // a block's chain or the memory, and rounds of blocks
        const double part = (a.N <= 16 ? 16 : a.N <= 32 ? 32 : 64) / 64.0, copies = 3.5 + 0.135 * mb;
        const double chain = 3 + 1.2 * part + chunks * (0.23 + 0.02 * part), rounds = tiles(a.T, kNarrowTokens * kNarrowBlocks * sms);
        take((chain > copies ? chain : copies) + 2 * (rounds - 1), {0, 0, 1});
    }
    return c;
}

LinearKernel g_set{};                 // by a test (0: the estimate)
thread_local LinearKernel g_taken{};

}  // namespace

void set_debug_linear(const LinearKernel& k) { g_set = k; }
LinearKernel last_linear() { return g_taken; }
bool debug_linear_fits(const LinearArgs& a) {
    return !(g_set.kernel == 1 && g_set.splits > chunks_of(a)) && !(g_set.kernel == 2 && g_set.size == 256 && a.out_dtype == GEOCACHE_F32) &&
           !(g_set.kernel == 3 && (a.N > kNarrowFeatures || a.gated));
}

cudaError_t launch_linear(const LinearArgs& given, cudaStream_t s) {
    LinearArgs a = given;
    static unsigned int* word = nullptr;
    static int sms = 0;
    static const cudaError_t ready = [] {
        int device = 0;
        cudaError_t e = linear_error_word(&word);
        if (e == cudaSuccess) e = cudaGetDevice(&device);
        return e == cudaSuccess ? cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) : e;
    }();
    if (ready != cudaSuccess) return ready;
    a.error = word;
    Choice c = choose(a, sms);
    if (g_set.kernel) c = {g_set.kernel == 2 ? g_set.size : 0, g_set.kernel == 1 ? g_set.size : 0, g_set.splits};
    g_taken = c.pair_features ? LinearKernel{2, c.pair_features, 0} : c.tokens ? LinearKernel{1, c.tokens, c.splits} : LinearKernel{3, 0, 0};
    if (c.pair_features) return launch_linear_pairs(a, c.pair_features, sms, s);
    Params p{};
    p.a = a;
    const int ob = a.out_dtype == GEOCACHE_F32 ? 4 : 2;
    p.chunks = chunks_of(a);
    const int part = a.gated ? kFeatures / 2 : kFeatures;
    p.feature_tiles = (a.N + part - 1) / part;
    p.tokens = c.tokens;
    p.splits = c.splits;
    // binary32 sums, operands of one type (e4m3 is type 0 of its kind), both with the summed axis contiguous
    const uint32_t type = a.in_dtype == GEOCACHE_BF16 ? 1 : 0;
    if (!p.tokens)
        for (p.features = 16; p.features < a.N;) p.features *= 2;
    // the first operand's rows are the lanes, here weights; with few features tokens
    const int columns = p.features ? p.features : p.tokens, lanes = p.features ? kNarrowTokens : kFeatures;
    p.idesc = 1u << 4 | type << 7 | type << 10 | (uint32_t)(columns >> 3) << 17 | (uint32_t)(lanes >> 4) << 24;
    p.out_wide = !((uintptr_t)a.out.data % (4 * ob)) && a.out.stride % 4 == 0;
    p.residual_wide = !((uintptr_t)a.residual.data % (4 * ob)) && a.residual.stride % 4 == 0;
    if (a.out_dtype == GEOCACHE_BF16) return launch_out<__nv_bfloat16>(p, sms, s);
    if (a.out_dtype == GEOCACHE_F16) return launch_out<__half>(p, sms, s);
    return launch_out<float>(p, sms, s);
}

cudaError_t linear_error_word(unsigned int** word) { return cudaGetSymbolAddress(reinterpret_cast<void**>(word), g_linear_error); }

}  // namespace geocache
