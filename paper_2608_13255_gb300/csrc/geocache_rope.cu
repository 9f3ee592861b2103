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

// A warp takes one unit: kU * (32 / G) heads of one token's queries or keys.  G lanes hold a row, kNV words of
// 16 bytes each (word w of a row lies in lane w % G), so one round of kU loads a lane is in flight before any
// is used.  A lane's cosines and sines are the same for all heads of the token and stay in registers.
// Rotation: out = x * c + partner * s, s signed by the element's place in its pair.  Interleaved pairs lie in one
// lane; halves that are whole words lie in two lanes (shuffle); other halves meet in shared memory.
template <typename T, int G, int kNV, int kRot, int kU, bool kAligned>
__global__ void __launch_bounds__(32 * kWarps) norm_rope_kernel(const __grid_constant__ NormRopeArgs a, int q_units,
                                                                int units) {
    constexpr int V = Elements<T>::kN, R = 32 / G;
    __shared__ float rows[kRot == kHalfShared ? kWarps : 1][kRot == kHalfShared ? 32 * kNV * V : 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane % G, r = lane / G;
    pdl_wait();
    const long long n = (long long)a.T * units;
    for (long long u = (long long)blockIdx.x * kWarps + warp; u < n; u += (long long)gridDim.x * kWarps) {
        const long long t = u / units;
        const int c = (int)(u - t * units), side = c >= q_units;
        const int h0 = (side ? c - q_units : c) * (kU * R) + r, H = side ? a.Hk : a.Hq;
        const T* in = static_cast<const T*>(a.in[side]) + t * a.in_ts[side];
        T* out = static_cast<T*>(a.out[side]) + t * a.out_ts[side];

        uint4 w[kU][kNV];
#pragma unroll
        for (int i = 0; i < kU; ++i)
#pragma unroll
            for (int v = 0; v < kNV; ++v) {
                const int h = h0 + i * R, d = (l + v * G) * V;
                w[i][v] = make_uint4(0, 0, 0, 0);
                if (h < H && d < a.D) w[i][v] = load_words<T, kAligned>(in + h * a.in_hs[side] + d);
            }

        float cs[kNV][V], sn[kNV][V], wt[kNV][V];
#pragma unroll
        for (int v = 0; v < kNV; ++v)
#pragma unroll
            for (int e = 0; e < V; ++e) { cs[v][e] = 1.0f; sn[v][e] = 0.0f; wt[v][e] = 1.0f; }
        bool turn = kRot != kNone;
        if (kRot != kNone) {
            const long long slot = a.slots ? a.slots[t] : t;
            if (slot < 0 || slot >= a.n_slots) {
                turn = false;
                if (lane == 0) atomicOr(&g_rope_error, 32u);
            } else {
                const float2* tab = a.table + slot * (a.rot / 2);
                const int half = a.rot / 2;
#pragma unroll
                for (int v = 0; v < kNV; ++v)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const int d = (l + v * G) * V + e;
                        if (d >= a.rot) continue;
                        const bool second = kRot == kInterleaved ? e & 1 : d >= half;
                        const float2 x = tab[kRot == kInterleaved ? d / 2 : (second ? d - half : d)];
                        cs[v][e] = x.x;
                        sn[v][e] = second ? x.y : -x.y;
                    }
            }
        }
        const float* weight = a.norm ? a.weight[side] : nullptr;
        if (weight)
#pragma unroll
            for (int v = 0; v < kNV; ++v)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const int d = (l + v * G) * V + e;
                    if (d < a.D) wt[v][e] = weight[d];
                }

#pragma unroll
        for (int i = 0; i < kU; ++i) {
            const int h = h0 + i * R;
            float x[kNV][V];
#pragma unroll
            for (int v = 0; v < kNV; ++v) {
                const T* p = reinterpret_cast<const T*>(&w[i][v]);
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
                const float inv = 1.0f / sqrtf(sum / (float)a.D + a.eps);
#pragma unroll
                for (int v = 0; v < kNV; ++v)
#pragma unroll
                    for (int e = 0; e < V; ++e) x[v][e] *= inv * wt[v][e];
            }
            if (turn) {  // the same for the whole warp
                float y[kNV][V];
                if (kRot == kInterleaved) {
#pragma unroll
                    for (int v = 0; v < kNV; ++v)
#pragma unroll
                        for (int e = 0; e < V; ++e) y[v][e] = x[v][e ^ 1];
                } else if (kRot == kHalfShuffle) {
                    const int hop = a.rot / 2 / V, from = l < hop ? l + hop : l - hop;
#pragma unroll
                    for (int e = 0; e < V; ++e) y[0][e] = __shfl_sync(0xffffffffu, x[0][e], from, G);
                } else {
                    float* row = rows[warp] + r * (G * kNV * V);
                    const int half = a.rot / 2;
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
            if (h < H)
#pragma unroll
                for (int v = 0; v < kNV; ++v) {
                    const int d = (l + v * G) * V;
                    if (d < a.D) store_words<T, kAligned>(out + h * a.out_hs[side] + d, x[v]);
                }
        }
    }
}

int sm_count() {
    int dev = 0, sms = 0;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    return sms > 0 ? sms : 1;
}

template <typename T, int G, int kNV, int kRot, int kU, bool kAligned>
cudaError_t launch(const NormRopeArgs& a, cudaStream_t s) {
    constexpr int heads = kU * (32 / G);
    const int q_units = (a.Hq + heads - 1) / heads, units = q_units + (a.Hk + heads - 1) / heads;
    const long long blocks = ((long long)a.T * units + kWarps - 1) / kWarps;
    const unsigned grid = (unsigned)(blocks < (1LL << 30) ? blocks : (1LL << 30));
    return launch_pdl(norm_rope_kernel<T, G, kNV, kRot, kU, kAligned>, dim3(grid), 32 * kWarps, 0, s, a, q_units, units);
}

template <typename T, int G, int kNV, int kRot>
cudaError_t launch_rows(const NormRopeArgs& a, bool aligned, cudaStream_t s) {
    if (!aligned) return launch<T, G, kNV, kRot, 1, false>(a, s);
    constexpr int R = 32 / G;
    const int most = a.Hq > a.Hk ? a.Hq : a.Hk;
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
