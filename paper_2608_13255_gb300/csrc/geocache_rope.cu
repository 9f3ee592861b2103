// Norms of queries and keys with the rotation of their positions, and the table of the rotation.
//
// Both kernels read each row (one head of one token) once and write it once; the sum of squares runs over the lanes that
// hold the row, and beside the rows only one table row a token and the weights move, which the L1 serves to all heads.
// Back to back on one set of buffers 24,576 tokens x 32 heads of 128 take 68 (interleaved) and 74 us (halves) in bf16, 6.1
// and 5.6 of 6.7 TB/s (72 us interleaved where the inputs change), and 120 us in f32, which is all of HBM.  Narrower heads
// are bound by issue, a lane's coefficients being made for two rows only: 32 heads of 64 43 and 47 us (4.9 and 4.4 TB/s),
// of 40, 72 and 80 39, 64 and 66 us (3.4, 3.6 and 3.9 TB/s, lanes without words besides).  norm_rope_kernel takes the rows
// that norm_rope_pairs_kernel does not (halves that end inside a word of 8 bytes, no alignment, a head of one word) and
// is bound by issue.
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

// Status word of this file's kernels (bit 5: a slot outside the table); read by geocache_device_status.
__device__ unsigned int g_rope_error = 0;

// One thread per (slot, pair); double throughout, since an angle of 10^5 turns keeps 2^-53 * 10^6 of itself.  Made once
// per model and bound by the few binary64 units: 24,576 slots x 32 pairs 50 us, x 64 pairs 92 us, 17 pairs a ns (the
// writes alone would take 1 and 2 us).
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
    if constexpr (kAligned) {
        return __ldcs(reinterpret_cast<const uint4*>(p));
    } else {
        union { uint4 w; T e[Elements<T>::kN]; } u;
#pragma unroll
        for (int e = 0; e < Elements<T>::kN; ++e) u.e[e] = p[e];
        return u.w;
    }
}

// 16 bytes of a row as floats, and back (two values a conversion)
__device__ __forceinline__ void widen(const uint4& w, float* x, __nv_bfloat16) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void widen(const uint4& w, float* x, __half) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ void widen(const uint4& w, float* x, float) {
    x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
}
__device__ __forceinline__ uint32_t narrow(float lo, float hi, __nv_bfloat16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t narrow(float lo, float hi, __half) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// 8 bytes of a 16-bit row
template <typename T>
__device__ __forceinline__ void widen(const uint2& w, float* x, T t) {
    float y[8];
    widen(make_uint4(w.x, w.y, 0, 0), y, t);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = y[i];
}
template <typename T>
__device__ __forceinline__ void store_word(uint2* p, const float* x) {
    if constexpr (sizeof(T) == 2) *p = make_uint2(narrow(x[0], x[1], T()), narrow(x[2], x[3], T()));
}
template <typename T>
__device__ __forceinline__ uint4 narrow_words(const float* x) {
    if constexpr (sizeof(T) == 4)
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    else
        return make_uint4(narrow(x[0], x[1], T()), narrow(x[2], x[3], T()), narrow(x[4], x[5], T()), narrow(x[6], x[7], T()));
}

template <typename T>
__device__ __forceinline__ void store_word(uint4* p, const float* x) { *p = narrow_words<T>(x); }

template <typename T, bool kAligned>
__device__ __forceinline__ void store_words(T* p, const float* x) {
    if constexpr (kAligned) {
        *reinterpret_cast<uint4*>(p) = narrow_words<T>(x);
    } else {
#pragma unroll
        for (int e = 0; e < Elements<T>::kN; ++e) p[e] = from_float<T>(x[e]);
    }
}

constexpr int kWarps = 8;
constexpr int kLargestHead = 256;  // elements

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
                    widen(now[i][v], x[v], T());
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
                        // element e of word w at [e][w]: neither side meets a bank twice
                        float* row = rows[warp] + r * (G * kNV * V);
                        __syncwarp();
#pragma unroll
                        for (int v = 0; v < kNV; ++v)
#pragma unroll
                            for (int e = 0; e < V; ++e) row[e * (G * kNV) + l + v * G] = x[v][e];
                        __syncwarp();
#pragma unroll
                        for (int v = 0; v < kNV; ++v)
#pragma unroll
                            for (int e = 0; e < V; ++e) {
                                const int d = (l + v * G) * V + e;
                                const int at = d < half ? d + half : d - half;
                                y[v][e] = d < a.rot ? row[at % V * (G * kNV) + at / V] : 0.0f;
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

// The rows of a token whose slot is outside the table: the norm alone, a warp a row.  Out of line and taken before the
// rows are loaded, for the kernel below is bound by issue and registers where every element is rotated (24,576 tokens x 32
// heads of 128 in bf16, interleaved and halves: 68 and 74 us; 73 and 76 with a flag beside the coefficients).
template <typename T>
__device__ __noinline__ void norm_rows(const NormRopeArgs& a, int side, long long t, int first, int last) {
    const int lane = threadIdx.x & 31;
    const float* weight = a.norm ? a.weight[side] : nullptr;
    for (int h = first; h < last; ++h) {
        const T* in = static_cast<const T*>(a.in[side]) + t * a.in_ts[side] + h * a.in_hs[side];
        T* out = static_cast<T*>(a.out[side]) + t * a.out_ts[side] + h * a.out_hs[side];
        float inv = 1.0f;
        if (a.norm) {
            float sum = 0.0f;
            for (int d = lane; d < a.D; d += 32) sum = fmaf((float)in[d], (float)in[d], sum);
#pragma unroll
            for (int m = 16; m > 0; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
            inv = rsqrtf(fmaf(sum, 1.0f / (float)a.D, a.eps));
        }
        for (int d = lane; d < a.D; d += 32) out[d] = from_float<T>((float)in[d] * (weight ? weight[d] : 1.0f) * inv);
    }
}

// The common rows: an even number of words, two a lane, and a rotation that whole words take part in.  Rotated halves lie
// in one lane as interleaved pairs do (lane l: word l of each half; the unrotated words two by two behind them), and
// nothing but the sum of squares crosses lanes.  With the weights folded into the rotation a pair (a, b) becomes
//     inv (a ca - b sb, a sa + b cb),  ca = w_a c, sa = w_a s, cb = w_b c, sb = w_b s,
// three products and three sums an element in place of about ten operations of the general kernel, which is bound by
// issue (24,576 tokens x 32 heads of 128 in bf16: 84 -> 73 us; halves of 64: 74 -> 51 us).
// kFull: all lanes have words and the whole head is rotated (heads of 64, 128 and 256 in 16 bits), known to the compiler
// (73 us; 79 without).  Two rows of 16-byte words of 16-bit elements a lane want more than the 80 registers that three
// blocks an SM leave: these instances spill 36 to 60 bytes a thread, the others nothing.  V: elements of a word; 16-bit
// rows that have an odd number of 16-byte words, or halves that are not whole ones, take words of 8 bytes (24,576 tokens x
// 20 heads of 80, half rotated: 103 -> 53 us; 32 heads of 40: 95 -> 45 us).
template <typename T, int V, int G, bool kInter, bool kFull, int kU>
__global__ void __launch_bounds__(32 * kWarps, 3) norm_rope_pairs_kernel(const __grid_constant__ NormRopeArgs a, int heads,
                                                                         unsigned q_units, unsigned units, unsigned n_blocks) {
    using Word = std::conditional_t<V * sizeof(T) == 16, uint4, uint2>;
    constexpr int R = 32 / G;
    const int D = kFull ? 2 * G * V : a.D, rot = kFull ? D : a.rot;
    const int lane_words = D / (2 * V), turned = kInter ? 0 : rot / (2 * V);  // lanes with words; with rotated halves
    const float inv_d = 1.0f / (float)D;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane % G, r = lane / G;
    const bool on = kFull || l < lane_words;
    // the lane's two words, by their first elements
    const int da = V * (kFull || kInter || l < turned ? l : turned + l), db = V * (kInter || kFull || l >= turned ? lane_words + l : turned + l);
    pdl_wait();
    for (unsigned block = blockIdx.x; block < n_blocks; block += gridDim.x) {
        const unsigned group = block / units, c = block - group * units;
        const long long t = (long long)group * kWarps + warp;
        if (t >= a.T) continue;
        const int side = c >= q_units, H = side ? a.Hk : a.Hq;
        const int first = (int)(side ? c - q_units : c) * heads, last = min(H, first + heads);
        const long long in_hs = a.in_hs[side], out_hs = a.out_hs[side];
        const int slot = rot == 0 ? 0 : a.slots ? a.slots[t] : (int)t;
        const bool lost = rot && (slot < 0 || slot >= (int)a.n_slots);
        if (lost && lane == 0) atomicOr(&g_rope_error, 32u);
        if (kFull && __builtin_expect(lost, 0)) {
            norm_rows<T>(a, side, t, first, last);
            continue;
        }
        const T* in = static_cast<const T*>(a.in[side]) + t * a.in_ts[side] + (first + r) * in_hs;
        T* out = static_cast<T*>(a.out[side]) + t * a.out_ts[side] + (first + r) * out_hs;
        Word w[kU][2];
        auto load_round = [&](int h1) {
#pragma unroll
            for (int i = 0; i < kU; ++i)
                if (on && h1 + i * R < last) {
                    w[i][0] = __ldcs(reinterpret_cast<const Word*>(in + i * R * in_hs + da));
                    w[i][1] = __ldcs(reinterpret_cast<const Word*>(in + i * R * in_hs + db));
                }
            in += kU * R * in_hs;
        };
#pragma unroll
        for (int i = 0; i < kU; ++i) w[i][0] = w[i][1] = Word{};
        load_round(first + r);

        // pair i: elements (2 i, 2 i + 1) of the lane's words, or (i, i) of the first and the second
        float ca[V], sa[V], cb[V], sb[V];
        // which of the lane's words are rotated (halves: both or neither); the others meet no partner, since that need not
        // be finite
        bool turn[2] = {kFull, kFull};
        {
            float cs[2 * V];
#pragma unroll
            for (int i = 0; i < V; ++i) { cs[2 * i] = 1.0f; cs[2 * i + 1] = 0.0f; }
            if (rot && !lost && on) {
                turn[0] = kFull || (kInter ? da < rot : l < turned);
                turn[1] = kFull || (kInter && db < rot);
                const float* tab = reinterpret_cast<const float*>(a.table + (long long)slot * (rot / 2));
                const bool wide = !((uintptr_t)tab & 15);
                if (kInter) {
                    if (turn[0]) load_floats<V>(tab + da, wide, cs);
                    if (turn[1]) load_floats<V>(tab + db, wide, cs + V);
                } else if (turn[0]) {
                    load_floats<2 * V>(tab + 2 * da, wide, cs);
                }
            }
            float wt[2][V];
#pragma unroll
            for (int e = 0; e < V; ++e) wt[0][e] = wt[1][e] = 1.0f;
            const float* weight = a.norm ? a.weight[side] : nullptr;
            if (weight && on) {
                const bool wide = !((uintptr_t)weight & 15);
                load_floats<V>(weight + da, wide, wt[0]);
                load_floats<V>(weight + db, wide, wt[1]);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float wa = kInter ? wt[i / (V / 2)][2 * i % V] : wt[0][i], wb = kInter ? wt[i / (V / 2)][2 * i % V + 1] : wt[1][i];
                ca[i] = wa * cs[2 * i];
                sa[i] = wa * cs[2 * i + 1];
                cb[i] = wb * cs[2 * i];
                sb[i] = wb * cs[2 * i + 1];
            }
        }

#pragma unroll 1
        for (int h1 = first + r; h1 - r < last; h1 += kU * R) {
            Word now[kU][2];
#pragma unroll
            for (int i = 0; i < kU; ++i) { now[i][0] = w[i][0]; now[i][1] = w[i][1]; }
            if (h1 - r + kU * R < last) load_round(h1 + kU * R);
#pragma unroll
            for (int i = 0; i < kU; ++i) {
                float x[2][V];
                widen(now[i][0], x[0], T());
                widen(now[i][1], x[1], T());
                float inv = 1.0f;
                if (a.norm) {
                    float sum[2] = {0.0f, 0.0f};
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        sum[0] = fmaf(x[0][e], x[0][e], sum[0]);
                        sum[1] = fmaf(x[1][e], x[1][e], sum[1]);
                    }
                    sum[0] += sum[1];
#pragma unroll
                    for (int m = G / 2; m > 0; m >>= 1) sum[0] += __shfl_xor_sync(0xffffffffu, sum[0], m);
                    inv = rsqrtf(fmaf(sum[0], inv_d, a.eps));
                }
                float z[2][V];
#pragma unroll
                for (int p = 0; p < V; ++p) {
                    const int va = kInter ? p / (V / 2) : 0, ea = kInter ? 2 * p % V : p;
                    const int vb = kInter ? va : 1, eb = kInter ? ea + 1 : p;
                    const float xa = x[va][ea], xb = x[vb][eb];
                    if (turn[va]) {
                        z[va][ea] = fmaf(xa, ca[p], -(xb * sb[p])) * inv;
                        z[vb][eb] = fmaf(xa, sa[p], xb * cb[p]) * inv;
                    } else {
                        z[va][ea] = xa * ca[p] * inv;
                        z[vb][eb] = xb * cb[p] * inv;
                    }
                }
                if (on && h1 + i * R < last) {
                    store_word<T>(reinterpret_cast<Word*>(out + i * R * out_hs + da), z[0]);
                    store_word<T>(reinterpret_cast<Word*>(out + i * R * out_hs + db), z[1]);
                }
            }
            out += kU * R * out_hs;
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

using Kernel = void (*)(const NormRopeArgs, int, unsigned, unsigned, unsigned);

// `round`: the rows that a warp has in flight
cudaError_t launch(Kernel kernel, int round, const NormRopeArgs& a, cudaStream_t s) {
    // As many heads a warp as leave the device two rounds of its warps (the table's row and the weights are then read
    // once for them), in even shares: small calls still fill the device.
    const long long warps = 2LL * 32 * sm_count();
    const int most = a.Hq > a.Hk ? a.Hq : a.Hk;
    int shares = 1;
    while (shares * round < most && (long long)a.T * shares * 2 < warps) ++shares;
    const int heads = (most + shares * round - 1) / (shares * round) * round;
    const unsigned q_units = (unsigned)((a.Hq + heads - 1) / heads), units = q_units + (unsigned)((a.Hk + heads - 1) / heads);
    const long long blocks = ((long long)a.T + kWarps - 1) / kWarps * units;
    if (blocks > 0xffffffffLL - (1LL << 30)) return cudaErrorInvalidValue;  // over 2^31 tokens x 2^16 heads
    const unsigned grid = (unsigned)(blocks < (1LL << 30) ? blocks : (1LL << 30));
    return launch_pdl(kernel, dim3(grid), 32 * kWarps, 0, s, a, heads, q_units, units, (unsigned)blocks);
}

template <typename T, int V, int G>
cudaError_t launch_pairs(const NormRopeArgs& a, cudaStream_t s) {
    static_assert(G == 4 || G * V < kLargestHead, "rows that fill no more than half of the lanes take fewer");
    constexpr int R = 32 / G;
    const bool inter = a.layout == GEOCACHE_ROPE_INTERLEAVED;
    const int most = a.Hq > a.Hk ? a.Hq : a.Hk;
    // two rows (four words) a lane where there are heads for them
    if constexpr (V == Elements<T>::kN) {
        if (a.rot == a.D && a.D == 2 * G * V) {
            if (most > R)
                return launch(inter ? norm_rope_pairs_kernel<T, V, G, true, true, 2> : norm_rope_pairs_kernel<T, V, G, false, true, 2>,
                              2 * R, a, s);
            return launch(inter ? norm_rope_pairs_kernel<T, V, G, true, true, 1> : norm_rope_pairs_kernel<T, V, G, false, true, 1>, R,
                          a, s);
        }
    }
    return launch(inter ? norm_rope_pairs_kernel<T, V, G, true, false, 2> : norm_rope_pairs_kernel<T, V, G, false, false, 2>, 2 * R,
                  a, s);
}

// Rows of whole pairs of V-element words, aligned to them; false where they are not.
template <typename T, int V>
bool try_pairs(const NormRopeArgs& a, cudaStream_t s, cudaError_t* e) {
    const int step = a.layout == GEOCACHE_ROPE_INTERLEAVED ? V : 2 * V;
    if (a.D % (2 * V) || a.rot % step) return false;
    for (int i = 0; i < 2; ++i) {
        if (!(i ? a.Hk : a.Hq)) continue;
        if (((uintptr_t)a.in[i] | (uintptr_t)a.out[i]) % (V * sizeof(T)) ||
            (a.in_ts[i] | a.in_hs[i] | a.out_ts[i] | a.out_hs[i]) % V)
            return false;
    }
    const int lanes = a.D / (2 * V);
    if (lanes <= 4)
        *e = launch_pairs<T, V, 4>(a, s);
    else if (lanes <= 8)
        *e = launch_pairs<T, V, 8>(a, s);
    else if (V * 32 >= kLargestHead || lanes <= 16)
        *e = launch_pairs<T, V, 16>(a, s);
    else if constexpr (V * 32 < kLargestHead)
        *e = launch_pairs<T, V, 32>(a, s);
    return true;
}

template <typename T, int G, int kNV, int kRot>
cudaError_t launch_rows(const NormRopeArgs& a, bool aligned, cudaStream_t s) {
    constexpr int R = 32 / G;
    // (aligned rows without a rotation, or with halves of whole words, are norm_rope_pairs_kernel's)
    if constexpr (kRot == kInterleaved || kRot == kHalfShared) {
        const int most = a.Hq > a.Hk ? a.Hq : a.Hk;
        // four rows a lane where there are heads for them
        if (aligned && most > R) return launch(norm_rope_kernel<T, G, kNV, kRot, 4, true>, 4 * R, a, s);
        if (aligned) return launch(norm_rope_kernel<T, G, kNV, kRot, 1, true>, R, a, s);
    }
    return launch(norm_rope_kernel<T, G, kNV, kRot, 1, false>, R, a, s);
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
    cudaError_t e;
    if (try_pairs<T, V>(a, s, &e)) return e;
    if constexpr (sizeof(T) == 2) {
        if (try_pairs<T, V / 2>(a, s, &e)) return e;
    }
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

cudaError_t rope_error_word(unsigned int** word) { return cudaGetSymbolAddress(reinterpret_cast<void**>(word), g_rope_error); }

}  // namespace geocache
