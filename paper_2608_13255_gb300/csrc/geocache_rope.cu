// Norms of queries and keys with the rotation of their positions, and the table of the rotation.
//
// norm_rope_kernel reads each row (one head of one token) once and writes it once; the sum of squares
// runs over the lanes that hold the row, so nothing else moves but one table row a token and the weights,
// which the L1 serves to all heads.  It is bound by HBM.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "geocache.h"
#include "geocache_device.cuh"
#include "geocache_internal.h"

namespace geocache {

namespace {

// Status word of this file's kernels (bit 32: a slot outside the table); read by geocache_device_status.
__device__ unsigned int g_rope_error = 0;

// One thread per (slot, pair); double throughout, since an angle of 10^5 turns keeps 2^-53 * 10^6 of itself.
__global__ void __launch_bounds__(256) rope_table_kernel(const __grid_constant__ RopeTableArgs a) {
    const long long n = a.n_slots * a.pairs;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < n; i += gridDim.x * 256LL) {
        const long long slot = i / a.pairs;
        const int pair = (int)(i - slot * a.pairs);
        const double p = a.pos ? (double)a.pos[slot] : (double)slot;
        double s, c;
        sincos(p * a.freq[pair], &s, &c);
        a.table[slot * a.row_pairs + a.first_pair + pair] = make_float2((float)(a.magnitude * c), (float)(a.magnitude * s));
    }
}

enum Rotation { kNone, kInterleaved, kHalfShuffle, kHalfShared };

template <typename T>
struct Elements {  // 16 bytes of a row
    static constexpr int kN = 16 / sizeof(T);
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

template <typename T, bool kAligned>
__device__ __forceinline__ uint4 load_words(const T* p) {
    if (kAligned) return __ldcs(reinterpret_cast<const uint4*>(p));
    union { uint4 w; T e[Elements<T>::kN]; } u;
#pragma unroll
    for (int e = 0; e < Elements<T>::kN; ++e) u.e[e] = p[e];
    return u.w;
}

template <typename T, bool kAligned>
__device__ __forceinline__ void store_words(T* p, const float* x) {
    union { uint4 w; T e[Elements<T>::kN]; } u;
#pragma unroll
    for (int e = 0; e < Elements<T>::kN; ++e) u.e[e] = from_float<T>(x[e]);
    if (kAligned) {
        *reinterpret_cast<uint4*>(p) = u.w;
    } else {
#pragma unroll
        for (int e = 0; e < Elements<T>::kN; ++e) p[e] = u.e[e];
    }
}

constexpr int kWarps = 8;

// n consecutive floats, in 16-byte words where `wide`
template <int kN>
__device__ __forceinline__ void load_floats(const float* p, bool wide, float* x) {
    static_assert(kN % 4 == 0, "whole words");
    if (wide) {
#pragma unroll
        for (int i = 0; i < kN; i += 4) {
            const float4 w = *reinterpret_cast<const float4*>(p + i);
            x[i] = w.x; x[i + 1] = w.y; x[i + 2] = w.z; x[i + 3] = w.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kN; ++i) x[i] = p[i];
    }
}

// A warp takes one unit: up to `heads` heads of one token's queries or keys.  G lanes hold a row, kNV words of 16 bytes
// each (word w of a row lies in lane w % G), and kU rows a lane are loaded before any is used.  A lane's cosines and
// sines are the same for all heads of the token and stay in registers, as the weights do.
// Rotation: out = x * c + partner * s, s signed by the element's place in its pair.  Interleaved pairs lie in one
// lane; halves that are whole words lie in two lanes (shuffle); other halves meet in shared memory.
template <typename T, int G, int kNV, int kRot, int kU, bool kAligned>
__global__ void __launch_bounds__(32 * kWarps) norm_rope_kernel(const __grid_constant__ NormRopeArgs a, int heads,
                                                                unsigned q_units, unsigned units, unsigned n_blocks) {
    constexpr int V = Elements<T>::kN, R = 32 / G;
    __shared__ float rows[kRot == kHalfShared ? kWarps : 1][kRot == kHalfShared ? 32 * kNV * V : 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane % G, r = lane / G;
    const float inv_d = 1.0f / (float)a.D;
    const int half = a.rot / 2;
    pdl_wait();
    for (unsigned block = blockIdx.x; block < n_blocks; block += gridDim.x) {
        const unsigned group = block / units, c = block - group * units;
        const long long t = (long long)group * kWarps + warp;
        if (t >= a.T) continue;
        const int side = c >= q_units, H = side ? a.Hk : a.Hq;
        const int first = (int)(side ? c - q_units : c) * heads, last = min(H, first + heads);
        const T* in = static_cast<const T*>(a.in[side]) + t * a.in_ts[side];
        T* out = static_cast<T*>(a.out[side]) + t * a.out_ts[side];
        // a round of rows, on its way while the table is read and while the round before it is worked on
        uint4 w[kU][kNV];
        auto load_round = [&](int h1) {
#pragma unroll
            for (int i = 0; i < kU; ++i)
#pragma unroll
                for (int v = 0; v < kNV; ++v) {
                    const int h = h1 + i * R, d = (l + v * G) * V;
                    w[i][v] = make_uint4(0, 0, 0, 0);
                    if (h < last && d < a.D) w[i][v] = load_words<T, kAligned>(in + h * a.in_hs[side] + d);
                }
        };
        load_round(first + r);

        float cs[kNV][V], sn[kNV][V], wt[kNV][V];
        bool turn = kRot != kNone;
        if (kRot != kNone) {
            const long long slot = a.slots ? a.slots[t] : t;
            if (slot < 0 || slot >= a.n_slots) {
                turn = false;
                if (lane == 0) atomicOr(&g_rope_error, 32u);
            } else {
                const float* tab = reinterpret_cast<const float*>(a.table + slot * half);
                // words of a lane's pairs: whole and 16-byte aligned (but for shared halves, which are rare)
                const bool wide = kRot != kHalfShared && !((uintptr_t)tab & 15);
#pragma unroll
                for (int v = 0; v < kNV; ++v) {
                    const int d0 = (l + v * G) * V;
                    if (kRot == kInterleaved) {
                        float x[V];
                        // (a word that the rotation ends in is read pair by pair)
                        if (d0 + V <= a.rot) load_floats<V>(tab + d0, wide, x);
#pragma unroll
                        for (int e = 0; e < V; e += 2) {
                            if (d0 + V > a.rot) {
                                const bool in_row = d0 + e < a.rot;
                                x[e] = in_row ? tab[d0 + e] : 1.0f;
                                x[e + 1] = in_row ? tab[d0 + e + 1] : 0.0f;
                            }
                            cs[v][e] = cs[v][e + 1] = x[e];
                            sn[v][e] = -x[e + 1];
                            sn[v][e + 1] = x[e + 1];
                        }
                    } else if (kRot == kHalfShuffle) {
                        float x[2 * V];
                        const bool second = d0 >= half;
                        if (d0 < a.rot) load_floats<2 * V>(tab + 2 * (second ? d0 - half : d0), wide, x);
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            cs[v][e] = d0 < a.rot ? x[2 * e] : 1.0f;
                            sn[v][e] = d0 < a.rot ? (second ? x[2 * e + 1] : -x[2 * e + 1]) : 0.0f;
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            const int d = d0 + e;
                            const bool second = d >= half, in_row = d < a.rot;
                            const float* x = tab + 2 * (second ? d - half : d);
                            cs[v][e] = in_row ? x[0] : 1.0f;
                            sn[v][e] = in_row ? (second ? x[1] : -x[1]) : 0.0f;
                        }
                    }
                }
            }
        }
        const float* weight = a.norm ? a.weight[side] : nullptr;
        if (weight) {
            const bool wide = !((uintptr_t)weight & 15);
#pragma unroll
            for (int v = 0; v < kNV; ++v)
                if ((l + v * G) * V < a.D) load_floats<V>(weight + (l + v * G) * V, wide, wt[v]);
        }

#pragma unroll 1
        for (int h1 = first + r; h1 - r < last; h1 += kU * R) {
            uint4 now[kU][kNV];
#pragma unroll
            for (int i = 0; i < kU; ++i)
#pragma unroll
                for (int v = 0; v < kNV; ++v) now[i][v] = w[i][v];
            if (h1 - r + kU * R < last) load_round(h1 + kU * R);
#pragma unroll
            for (int i = 0; i < kU; ++i) {
                const int h = h1 + i * R;
                float x[kNV][V];
#pragma unroll
                for (int v = 0; v < kNV; ++v) {
                    const T* p = reinterpret_cast<const T*>(&now[i][v]);
#pragma unroll
                    for (int e = 0; e < V; ++e) x[v][e] = to_float(p[e]);
                }
                if (a.norm) {
                    float sum = 0.0f;
#pragma unroll
                    for (int v = 0; v < kNV; ++v)
#pragma unroll
                        for (int e = 0; e < V; ++e) sum = fmaf(x[v][e], x[v][e], sum);
#pragma unroll
                    for (int m = G / 2; m > 0; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
                    const float inv = rsqrtf(fmaf(sum, inv_d, a.eps));
#pragma unroll
                    for (int v = 0; v < kNV; ++v)
#pragma unroll
                        for (int e = 0; e < V; ++e) x[v][e] *= weight ? inv * wt[v][e] : inv;
                }
                if (turn) {  // the same for the whole warp
                    float y[kNV][V];
                    if (kRot == kInterleaved) {
#pragma unroll
                        for (int v = 0; v < kNV; ++v)
#pragma unroll
                            for (int e = 0; e < V; ++e) y[v][e] = x[v][e ^ 1];
                    } else if (kRot == kHalfShuffle) {
                        const int hop = half / V, from = l < hop ? l + hop : l - hop;
#pragma unroll
                        for (int e = 0; e < V; ++e) y[0][e] = __shfl_sync(0xffffffffu, x[0][e], from, G);
                    } else {
                        float* row = rows[warp] + r * (G * kNV * V);
                        __syncwarp();
#pragma unroll
                        for (int v = 0; v < kNV; ++v)
#pragma unroll
                            for (int e = 0; e < V; ++e) row[(l + v * G) * V + e] = x[v][e];
                        __syncwarp();
#pragma unroll
                        for (int v = 0; v < kNV; ++v)
#pragma unroll
                            for (int e = 0; e < V; ++e) {
                                const int d = (l + v * G) * V + e;
                                y[v][e] = d < a.rot ? row[d < half ? d + half : d - half] : 0.0f;
                            }
                    }
#pragma unroll
                    for (int v = 0; v < kNV; ++v)
#pragma unroll
                        for (int e = 0; e < V; ++e)
                            if ((l + v * G) * V + e < a.rot) x[v][e] = fmaf(x[v][e], cs[v][e], y[v][e] * sn[v][e]);
                }
                if (h < last)
#pragma unroll
                    for (int v = 0; v < kNV; ++v) {
                        const int d = (l + v * G) * V;
                        if (d < a.D) store_words<T, kAligned>(out + h * a.out_hs[side] + d, x[v]);
                    }
            }
        }
    }
}

int sm_count() {
    static const int n = [] {  // one device per process
        int dev = 0, sms = 0;
        cudaGetDevice(&dev);
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
        return sms > 0 ? sms : 1;
    }();
    return n;
}

template <typename T, int G, int kNV, int kRot, int kU, bool kAligned>
cudaError_t launch(const NormRopeArgs& a, cudaStream_t s) {
    // As many heads a warp as leave the device two rounds of its warps (the table's row and the weights are then read
    // once for them), in even shares: small calls still fill the device.
    constexpr int round = kU * (32 / G);
    const long long warps = 2LL * 32 * sm_count();
    const int most = a.Hq > a.Hk ? a.Hq : a.Hk;
    int shares = 1;
    while (shares * round < most && (long long)a.T * shares * 2 < warps) ++shares;
    const int heads = (most + shares * round - 1) / (shares * round) * round;
    const unsigned q_units = (unsigned)((a.Hq + heads - 1) / heads), units = q_units + (unsigned)((a.Hk + heads - 1) / heads);
    const long long blocks = ((long long)a.T + kWarps - 1) / kWarps * units;
    if (blocks > 0xffffffffLL - (1LL << 30)) return cudaErrorInvalidValue;  // over 2^31 tokens x 2^16 heads
    const unsigned grid = (unsigned)(blocks < (1LL << 30) ? blocks : (1LL << 30));
    return launch_pdl(norm_rope_kernel<T, G, kNV, kRot, kU, kAligned>, dim3(grid), 32 * kWarps, 0, s, a, heads, q_units, units,
                      (unsigned)blocks);
}

template <typename T, int G, int kNV, int kRot>
cudaError_t launch_rows(const NormRopeArgs& a, bool aligned, cudaStream_t s) {
    if (!aligned) return launch<T, G, kNV, kRot, 1, false>(a, s);
    constexpr int R = 32 / G;
    const int most = a.Hq > a.Hk ? a.Hq : a.Hk;
    // four rows a lane where there are heads for them
    if (most > R) return launch<T, G, kNV, kRot, 4, true>(a, s);
    return launch<T, G, kNV, kRot, 1, true>(a, s);
}

template <typename T, int G, int kNV>
cudaError_t launch_rotation(const NormRopeArgs& a, bool aligned, cudaStream_t s) {
    if (a.rot == 0) return launch_rows<T, G, kNV, kNone>(a, aligned, s);
    if (a.layout == GEOCACHE_ROPE_INTERLEAVED) return launch_rows<T, G, kNV, kInterleaved>(a, aligned, s);
    if (kNV == 1 && a.rot / 2 % Elements<T>::kN == 0) return launch_rows<T, G, 1, kHalfShuffle>(a, aligned, s);
    return launch_rows<T, G, kNV, kHalfShared>(a, aligned, s);
}

template <typename T>
cudaError_t launch_type(const NormRopeArgs& a, cudaStream_t s) {
    constexpr int V = Elements<T>::kN;
    bool aligned = true;
    for (int i = 0; i < 2; ++i) {
        if (!(i ? a.Hk : a.Hq)) continue;
        aligned = aligned && !(((uintptr_t)a.in[i] | (uintptr_t)a.out[i]) & 15) &&
                  !((a.in_ts[i] | a.in_hs[i] | a.out_ts[i] | a.out_hs[i]) % V);
    }
    const int words = a.D / V;
    if (words <= 4) return launch_rotation<T, 4, 1>(a, aligned, s);
    if (words <= 8) return launch_rotation<T, 8, 1>(a, aligned, s);
    if (words <= 16) return launch_rotation<T, 16, 1>(a, aligned, s);
    if (words <= 32) return launch_rotation<T, 32, 1>(a, aligned, s);
    if constexpr (V == 4) return launch_rotation<T, 32, 2>(a, aligned, s);
    return cudaErrorInvalidValue;  // not reached: D <= 256
}

}  // namespace

cudaError_t launch_rope_table(const RopeTableArgs& a, cudaStream_t s) {
    const long long n = a.n_slots * a.pairs;
    if (n == 0) return cudaSuccess;
    const long long blocks = (n + 255) / 256, most = 32LL * sm_count();
    note_launches(1);
    rope_table_kernel<<<(unsigned)(blocks < most ? blocks : most), 256, 0, s>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_norm_rope(const NormRopeArgs& a, cudaStream_t s) {
    if (a.T == 0 || (a.Hq == 0 && a.Hk == 0)) return cudaSuccess;
    if (a.dtype == GEOCACHE_BF16) return launch_type<__nv_bfloat16>(a, s);
    if (a.dtype == GEOCACHE_F16) return launch_type<__half>(a, s);
    return launch_type<float>(a, s);
}

cudaError_t read_rope_error(unsigned int* out, bool clear, cudaStream_t s) {
    cudaError_t e = cudaMemcpyFromSymbolAsync(out, g_rope_error, sizeof(unsigned int), 0, cudaMemcpyDeviceToHost, s);
    if (e != cudaSuccess) return e;
    e = cudaStreamSynchronize(s);
    if (e != cudaSuccess || !clear || *out == 0) return e;
    static const unsigned int zero = 0;
    e = cudaMemcpyToSymbolAsync(g_rope_error, &zero, sizeof(unsigned int), 0, cudaMemcpyHostToDevice, s);
    if (e != cudaSuccess) return e;
    return cudaStreamSynchronize(s);
}

}  // namespace geocache
