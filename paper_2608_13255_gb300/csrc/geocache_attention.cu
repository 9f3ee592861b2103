// Attention over packed sequences on the tensor cores (tcgen05), planned by geocache_plan_attention.
//
// A thread block takes its pieces of the schedule one after the other.  A piece is one or two tiles of 128 query rows
// against a run of 128-key tiles; the two tiles share every load of keys and values and take turns, so that the tensor
// cores work on one while the other's softmax runs:
//   warp 10     loads queries (once a piece), keys and values (a ring of stages) by TMA;
//   warps 8, 9  issue the products of tile 0 and of tile 1: S = Q K^T into tensor memory, O += P V with P read from there;
//   warps 0-3   softmax of tile 0, one row a thread: S from tensor memory, the running maximum and sum in registers,
//   warps 4-7   the same of tile 1;   P = exp2((S - m) scale log2 e) as 16-bit pairs in tensor memory.
// O stays in tensor memory over the whole piece.  It is rescaled only when a row's weights of one tile of keys sum to more
// than 2^15: until then the sums and P are kept relative to an older maximum, which changes no result beyond rounding,
// and the maximum itself need not be taken in every tile.  S, the statistics and O are binary32; P is rounded to the
// inputs' type, as the product with the values needs, while its sum is taken before that rounding (f16: a weight below
// 2^-14 of the row's reference keeps fewer bits, off by at most 2^-25 of it).
//
// What bounds it.  Heads over 64, many rows: the tensor cores (24,576 tokens x 16 heads of 128: 2.69 to 2.86 ms from box
// to box, 1,730 to 1,840 TFLOP/s; 8,192: 319 to 332 us, 1,660 to 1,720).  Heads up to 64: no unit is above half use
// (tensor cores 48%, MUFU 48%, issue 46%; 8,192 tokens x 8 heads of 64 133 us, 1,030 TFLOP/s).  A pair of key tiles
// takes about 2,190 cycles, of which the products need 1,060, and the softmax of both tiles 1,490 (820 for one alone; its
// exponentials 1,090): the chain score - softmax - product is what takes the time, some 700 cycles of it between the
// roles.  Few rows: HBM (298,000 keys of 4 heads of 128: 100 us, 6.1 TB/s).
//
// 128 x 128 tiles, since a tile's S and O for two tiles fill the 512 columns of tensor memory; two tiles a
// block, so that products and softmax overlap; one block an SM, with a ring of 5 (8) stages in what the queries leave.
#include <cuda_runtime.h>

#include <cstdint>

#include "geocache.h"
#include "geocache_attention_turns.h"
#include "geocache_device.cuh"
#include "geocache_internal.h"
#include "geocache_tcgen05.cuh"

namespace geocache {

namespace {

// Status word of this file's kernels (bit 0: a wait ran out); read by geocache_device_status.
__device__ unsigned int g_attention_error = 0;

constexpr int kRows = kAttentionRows, kKeys = kAttentionKeys;
constexpr int kThreads = 384;  // three warpgroups: two of softmax, one of which three warps work
constexpr int kMmaWarp = 8, kLoadWarp = 10;  // warps 8 and 9 issue the products of tiles 0 and 1
// Registers a thread: 168 at launch (65536 / 384); the softmax warps hold a row of 128 scores and take the others' share
// (8 * 208 + 4 * 88 = 12 * 168).
constexpr int kSoftmaxRegs = 208, kOtherRegs = 88;
static_assert(8 * kSoftmaxRegs + 4 * kOtherRegs <= 12 * 168, "no more than the block was launched with");
constexpr uint32_t kTmemColumns = 512;
constexpr uint32_t kBox = 128 * 128;    // bytes of 128 rows of 64 elements (one swizzled box)

template <int DP>
struct Shape {  // heads padded to DP = 64 or 128 elements
    static constexpr int kBoxes = DP / 64;
    static constexpr uint32_t kTileBytes = kBoxes * kBox;
    static constexpr int kStages = DP == 128 ? 5 : 8;
    // Tensor memory, in columns: S of tile t at 128 t, and behind both O.  Heads up to 64 leave room for P beside S: the
    // scores of the next keys are then multiplied while the softmax of these runs.  Wider heads have P over S.
    static constexpr bool kApart = DP == 64;
    static constexpr uint32_t kWeights = kApart ? 256 : 0, kWeightsStep = kApart ? 64 : 128;
    static constexpr uint32_t kOut = kApart ? 384 : 256;
    static constexpr uint32_t kBytes = (2 + kStages) * kTileBytes + 1024;  // and room to align to 1024
};

constexpr int kCached = 16;  // pieces that a block reads from shared memory

struct Barriers {
    uint64_t q_full[2], q_empty[2], s_full[2], s_read[2], p_full[2], o_full[2], turn[2], drained;
    uint64_t kv_full[8], kv_empty[8];
    AttentionItem items[kCached];  // the block's first pieces
    uint32_t tmem;
    uint32_t dead;
};

// ------------------------------------------------------------------ PTX --
__device__ __forceinline__ bool mbar_wait(uint64_t* bar, uint32_t parity, unsigned long long limit_ns, Barriers* b) {
    return __all_sync(0xffffffffu, mbar_try(bar, parity)) || mbar_wait_slow(bar, parity, limit_ns, &b->dead, &g_attention_error);
}

__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
            dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void tma_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], "
        "[%6];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
        : "memory");
}

// D (tensor memory) = A B (+ D), A and B in shared memory
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
// the same with A in tensor memory
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t at, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(at),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// pairs of floats: one issue slot for two operations
__device__ __forceinline__ uint64_t pair(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t r, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(r)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
struct Params {
    AttentionArgs a;
    int tok;              // tokens of a tile
    int k_steps;          // of 16 elements of a head
    uint32_t qk_idesc, pv_idesc;
    float c;              // scale * log2(e)
    int wide_out;         // rows of `out` are whole 32-byte sectors
};

struct Items {  // a block's pieces [first, last)
    const AttentionItem* all;
    const Barriers* b;
    int first, last;
};
__device__ __forceinline__ void load_item(const Items& p, int i, AttentionItem& it) {
    const int4* s = reinterpret_cast<const int4*>(i - p.first < kCached ? p.b->items + (i - p.first) : p.all + i);
    int4* d = reinterpret_cast<int4*>(&it);
#pragma unroll
    for (int i = 0; i < 3; ++i) d[i] = s[i];
}

constexpr float kLargest = 32768.0f;  // of the weights of a row and tile: half of what f16 holds
constexpr int kEarly = 1;  // products of a go that are issued after the turn has passed to the other tile (of five at
                           // least: turns are for heads over 64)

// ---------------------------------------------------------------- roles --
// Each role walks the block's pieces with its own count of the phases; a wait that gives up ends it.
template <int DP>
__device__ void load_role(const Params& p, const CUtensorMap* qm, const CUtensorMap* km, const CUtensorMap* vm, uint32_t smem,
                          Barriers* b, const Items& items) {
    using S = Shape<DP>;
    const unsigned long long limit = p.a.wait_limit_ns;
    const uint32_t q_bytes = S::kBoxes * 128u * p.a.pack * p.tok;
    uint32_t stage = 0, phase = 0, q_n[2] = {0, 0}, armed = 0;
    bool drop = p.a.drop_first_copy && blockIdx.x == 0, ok = true;
    for (int i = items.first; i < items.last && ok; ++i) {
        AttentionItem it;
        load_item(items, i, it);
        const int n_kv[2] = {uniform(it.n_kv[0]), uniform(it.n_kv[1])}, n_tok[2] = {uniform(it.n_tok[0]), uniform(it.n_tok[1])};
        const int n = max(n_kv[0], n_kv[1]), q_row = uniform(it.q_row), group = uniform(it.head) / p.a.pack;
        const int kv_head = uniform(it.kv_head), kv_row = uniform(it.kv_row);
        auto queries = [&](int t) {
            if (!n_tok[t] || !n_kv[t]) return true;
            if (!mbar_wait(&b->q_empty[t], (q_n[t] & 1) ^ 1, limit, b)) return false;
            if (elect()) {
                mbar_expect(&b->q_full[t], q_bytes);
#pragma unroll
                for (int x = 0; x < S::kBoxes; ++x)
                    tma_4d(smem + t * S::kTileBytes + x * kBox, qm, 64 * x, 0, group, q_row + t * p.tok, &b->q_full[t]);
            }
            __syncwarp();
            ++q_n[t];
            return true;
        };
        auto keys = [&](const CUtensorMap* map, int j) {
            if (!mbar_wait(&b->kv_empty[stage], phase ^ 1, limit, b)) return false;
            if (!drop) {
                if (elect()) {
                    mbar_expect(&b->kv_full[stage], S::kTileBytes);
#pragma unroll
                    for (int x = 0; x < S::kBoxes; ++x)
                        tma_3d(smem + (2 + stage) * S::kTileBytes + x * kBox, map, 64 * x, kv_head, kv_row + j * kKeys,
                               &b->kv_full[stage]);
                }
                __syncwarp();
                armed |= 1u << stage;
            }
            drop = false;
            if (++stage == S::kStages) { stage = 0; phase ^= 1; }
            return true;
        };
        if (!queries(0)) break;
        for (int j = 0; j < n; ++j) {
            ok = keys(km, j);
            if (ok && j == 0) ok = queries(1);
            if (ok) ok = keys(vm, j);
            if (!ok) break;
        }
    }
    // The copies in flight land before the block ends: the last phase of every barrier is waited for.  On every path, since
    // this warp is up to a ring ahead and cannot know that another will give up later.
    const unsigned long long t0 = globaltimer();
    for (int t = 0; t < 2; ++t)
        while (q_n[t] && !mbar_try(&b->q_full[t], (q_n[t] & 1) ^ 1) && globaltimer() - t0 < kDrainLimitNs) {}
    for (uint32_t s = 0; s < S::kStages; ++s) {
        // stages below `stage` were last armed in this round, the others in the one before
        const uint32_t parity = s < stage ? phase : phase ^ 1;
        while ((armed >> s & 1) && !mbar_try(&b->kv_full[s], parity) && globaltimer() - t0 < kDrainLimitNs) {}
    }
}

// One warp issues the products of one query tile: S = Q K_0, and then for each key tile O += P V_j and S = Q K_{j+1} in one
// go.  The tensor cores' queue is short (issuing waits for room), so one warp waits for P and does the ring's bookkeeping
// while the other's products are issued.  The goes alternate: products of both tiles mixed would end together, and the
// softmax of both would then run while the tensor cores idle (measured: 4.0 ms for what takes 3.1 by one warp in turn).
// Each warp waits for every stage of the ring and gives every stage back, those that only the other tile reads too: a
// phase's parity tells it from the next one only, so neither warp may fall behind.
//
// With P apart from S (heads up to 64) the scores of the next keys are issued as soon as the softmax has read these, and
// the goes need no order: no tile's softmax waits for the other's products (8,192 tokens x 8 heads of 64: 141 -> 133 us).
template <int DP>
__device__ void mma_role(const Params& p, uint32_t smem, uint32_t tmem, Barriers* b, const Items& items, int t, int lane) {
    using S = Shape<DP>;
    const unsigned long long limit = p.a.wait_limit_ns;
    uint32_t stage = 0, phase = 0, q_n = 0, p_n = 0, r_n = 0, turn_n = 0;
    bool first = true;  // no piece of two tiles with keys so far
    // the next stage of the ring, once its copy has landed
    auto next_stage = [&](uint32_t& at) {
        at = stage;
        const bool ok = mbar_wait(&b->kv_full[stage], phase, limit, b);
        if (++stage == S::kStages) { stage = 0; phase ^= 1; }
        return ok;
    };
    auto scores = [&](uint32_t k_at, bool hand_over) {
        const uint64_t q = smem_desc(smem + t * S::kTileBytes, 16), k = smem_desc(k_at, 16);
#pragma unroll
        for (int s = 0; s < DP / 16; ++s)
            if (s < p.k_steps) {
                const uint32_t off = ((s >> 2) * kBox + (s & 3) * 32) >> 4;
                mma_ss(tmem + t * 128, q + off, k + off, p.qk_idesc, s > 0);
                if (hand_over && s + kEarly + 1 == p.k_steps) mbar_arrive(&b->turn[t ^ 1]);
            }
        tc_commit(&b->s_full[t]);
    };
    for (int i = items.first; i < items.last; ++i) {
        AttentionItem it;
        load_item(items, i, it);
        const int n = uniform(t ? it.n_kv[1] : it.n_kv[0]), n_other = uniform(t ? it.n_kv[0] : it.n_kv[1]);
        const int n_keys = uniform(it.n_keys);
        if (n > 0) {
            uint32_t v_stage = 0, k_stage = 0;
            if (!next_stage(k_stage) || !mbar_wait(&b->q_full[t], q_n++ & 1, limit, b)) return;
            tc_after();
            if (elect()) {
                scores(smem + (2 + k_stage) * S::kTileBytes, false);
                if (n == 1) tc_commit(&b->q_empty[t]);
                tc_commit(&b->kv_empty[k_stage]);
            }
            __syncwarp();
            for (int j = 0; j < n; ++j) {
                if (!next_stage(v_stage) || (j + 1 < n && !next_stage(k_stage))) return;
                if (S::kApart && j + 1 < n) {
                    if (!mbar_wait(&b->s_read[t], r_n++ & 1, limit, b)) return;
                    tc_after();
                    if (elect()) {
                        scores(smem + (2 + k_stage) * S::kTileBytes, false);
                        if (j + 2 == n) tc_commit(&b->q_empty[t]);
                        tc_commit(&b->kv_empty[k_stage]);
                    }
                    __syncwarp();
                }
                const uint32_t v_at = smem + (2 + v_stage) * S::kTileBytes, k_at = smem + (2 + k_stage) * S::kTileBytes;
                int v_steps = kKeys / 16;
                if (n_keys - j * kKeys < kKeys) {
                    // what lies behind the sequence's last key is another's: the rest of the last step of 16 keys is
                    // cleared (by both warps), so that 0 * v is 0 whatever it holds, and later steps are left out
                    const int keys = n_keys - j * kKeys;
                    v_steps = (keys + 15) / 16;
                    const int words = (v_steps * 16 - keys) * 8;
                    for (int x = 0; x < S::kBoxes; ++x)
                        for (int w = lane; w < words; w += 32)
                            asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(v_at + x * kBox + keys * 128 + w * 16), "r"(0)
                                         : "memory");
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                }
                // tile 0's go j comes before tile 1's and after its go j - 1
                if (!S::kApart && turn_taken(t, j, n_other, first))
                    if (!mbar_wait(&b->turn[t], turn_n++ & 1, limit, b)) return;
                const bool at_once = turn_given_at_once(t, j, n_other), turn_over = turn_given(t, j, n_other) && !at_once;
                if (!S::kApart && at_once) {
                    if (elect()) mbar_arrive(&b->turn[t ^ 1]);
                    __syncwarp();
                }
                if (!mbar_wait(&b->p_full[t], p_n++ & 1, limit, b)) return;
                tc_after();
                if (elect()) {
                    const uint64_t v = smem_desc(v_at, kBox);
#pragma unroll
                    for (int s = 0; s < kKeys / 16; ++s)
                        if (s < v_steps)
                            mma_ts(tmem + S::kOut + t * DP, tmem + S::kWeights + t * S::kWeightsStep + s * 8, v + s * (2048 >> 4),
                                   p.pv_idesc, j > 0 || s > 0);
                    tc_commit(&b->kv_empty[v_stage]);
                    if (S::kApart) {
                        tc_commit(&b->o_full[t]);
                    } else if (j + 1 < n) {
                        scores(k_at, turn_over);
                        if (j + 2 == n) tc_commit(&b->q_empty[t]);
                        tc_commit(&b->kv_empty[k_stage]);
                    } else {
                        if (turn_over) mbar_arrive(&b->turn[t ^ 1]);
                        tc_commit(&b->o_full[t]);
                    }
                }
                __syncwarp();
            }
        }
        if (n > 0 && n_other > 0) first = false;
        if (S::kApart && n > 0 && !mbar_wait(&b->s_read[t], r_n++ & 1, limit, b)) return;  // of the last scores
        for (int x = 2 * n; x < 2 * n_other; ++x) {  // stages that the other tile alone reads
            uint32_t at = 0;
            if (!next_stage(at)) return;
            if (elect()) mbar_arrive(&b->kv_empty[at]);
            __syncwarp();
        }
    }
}

// 8 columns of a row of O
template <typename T>
__device__ __forceinline__ void store8(T* out, const uint32_t* o, float inv) {
    uint4 w;
    uint32_t* r = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = pack2<T>(__uint_as_float(o[2 * i]) * inv, __uint_as_float(o[2 * i + 1]) * inv);
    *reinterpret_cast<uint4*>(out) = w;
}

template <int DP, typename T>
__device__ void softmax_role(const Params& p, uint32_t tmem, Barriers* b, const Items& items, int t, int warp, int lane) {
    const unsigned long long limit = p.a.wait_limit_ns;
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    using S = Shape<DP>;
    constexpr bool kApart = S::kApart;
    const uint32_t s_at = tmem + t * 128 + lanes, w_at = tmem + S::kWeights + t * S::kWeightsStep + lanes;
    const uint32_t o_at = tmem + S::kOut + t * DP + lanes;
    const int row = warp * 32 + lane, tok = row / p.a.pack, head = row - tok * p.a.pack;
    uint32_t s_n = 0, o_n = 0;
    for (int i = items.first; i < items.last; ++i) {
        AttentionItem it;
        load_item(items, i, it);
        const int n_tok = t ? it.n_tok[1] : it.n_tok[0], n = t ? it.n_kv[1] : it.n_kv[0], slot = t ? it.slot[1] : it.slot[0];
        if (!n_tok) continue;
        const bool active = tok < n_tok, warp_active = warp * 32 < n_tok * p.a.pack;
        const int sees = p.a.causal ? min(it.n_keys, it.sees + t * p.tok + tok) : it.n_keys;
        const int least = uniform(sees);  // the rows of a warp see more and more
        float m = -INFINITY, l = 0.0f;
        for (int j = 0; j < n; ++j) {
            if (!mbar_wait(&b->s_full[t], s_n++ & 1, limit, b)) return;
            tc_after();
            // P apart from S: its last product has to be done before the next weights are stored (P over S: the scores came
            // after that product)
            auto product_done = [&]() { return !kApart || j == 0 || mbar_wait(&b->o_full[t], o_n++ & 1, limit, b); };
            if (warp_active) {
                uint32_t s[128];
#pragma unroll
                for (int x = 0; x < 4; ++x) tmem_ld32(s_at + 32 * x, s + 32 * x);
                tmem_wait_ld(s);
#pragma unroll
                for (int x = 1; x < 4; ++x) tmem_pin32(s + 32 * x);
                if (kApart) {
                    tc_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&b->s_read[t]);
                }
                const int here = sees - j * kKeys;
                if (least - j * kKeys < kKeys) {
#pragma unroll
                    for (int x = 0; x < 128; ++x)
                        if (x >= here) s[x] = 0xff800000u;
                }
                if (j == 0) {
#pragma unroll
                    for (int x = 0; x < 128; x += 2) m = max3(m, __uint_as_float(s[x]), __uint_as_float(s[x + 1]));
                }
                // The weights are formed relative to the maximum of the first tile of keys, or of the last one that made
                // them large: while a row's weights sum to at most 2^15 in a tile they lose nothing by not being relative
                // to the latest maximum (the sums are binary32, and each is rounded relative to itself).
                float sum;
                for (bool again = false;; again = true) {
                    const float base = m == -INFINITY ? 0.0f : m * p.c;
                    const uint64_t c2 = pair(p.c, p.c), base2 = pair(-base, -base);
                    uint64_t sums[2] = {0, 0};
                    constexpr int kPart = kApart ? 32 : 16;  // pairs of weights stored at a time
#pragma unroll
                    for (int h = 0; h < 64 / kPart; ++h) {
                        uint32_t w[kPart];
#pragma unroll
                        for (int x = 0; x < kPart; ++x) {
                            const int y = 2 * (kPart * h + x);
                            float e0, e1;
                            unpair(fma2(pair(__uint_as_float(s[y]), __uint_as_float(s[y + 1])), c2, base2), e0, e1);
                            e0 = exp2_fast(e0);
                            e1 = exp2_fast(e1);
                            sums[x & 1] = add2(sums[x & 1], pair(e0, e1));
                            w[x] = pack2<T>(e0, e1);
                        }
                        if (kApart && h == 0 && !again) {
                            if (!product_done()) return;
                            tc_after();
                        }
                        if constexpr (kApart)
                            tmem_st32(w_at + 32 * h, w);
                        else
                            tmem_st16(w_at + 16 * h, w);
                    }
                    float l0, l1;
                    unpair(add2(sums[0], sums[1]), l0, l1);
                    sum = l0 + l1;
                    const bool large = active && (sum > kLargest || m == -INFINITY);
                    if (!__any_sync(0xffffffffu, large)) break;
                    // they did not (a row without keys so far counts as such): O and the sum follow the new maximum (the
                    // product into O is complete: see above), and the weights are formed again; each row by its own
                    // scores alone, so that its result does not depend on the rows beside it
                    float top = m;
#pragma unroll
                    for (int x = 0; x < 128; x += 2) top = max3(top, __uint_as_float(s[x]), __uint_as_float(s[x + 1]));
                    const bool grown = large && top > m;
                    if (!__any_sync(0xffffffffu, grown)) break;  // an infinite sum that no maximum mends
                    const float f = grown ? exp2_fast((m - top) * p.c) : 1.0f;
                    if (grown) m = top;
                    l *= f;
                    tmem_wait_st();  // the weights in flight go to where the new ones will
#pragma unroll 1
                    for (int x = 0; x < p.a.D; x += 32) {
                        uint32_t o[32];
                        tmem_ld32(o_at + x, o);
                        tmem_wait_ld(o);
#pragma unroll
                        for (int y = 0; y < 32; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * f);
                        tmem_st32(o_at + x, o);
                    }
                }
                l += sum;
                tmem_wait_st();
            } else if (kApart) {
                if (lane == 0) mbar_arrive(&b->s_read[t]);
                if (!product_done()) return;
            }
            tc_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&b->p_full[t]);
        }
        if (n && !mbar_wait(&b->o_full[t], o_n++ & 1, limit, b)) return;
        tc_after();
        if (!warp_active) continue;
        const long long token = (long long)it.q_row + t * p.tok + tok;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        const float lse = l == 0.0f ? -INFINITY : m * p.a.scale + logf(l);
        T* out = static_cast<T*>(p.a.out.data) + token * p.a.out.token_stride + (it.head + head) * p.a.out.head_stride;
        const long long part = (long long)slot * kRows + row;
        const bool wide = p.wide_out;
#pragma unroll 1
        for (int x = 0; x < p.a.D; x += 32) {
            uint32_t o[32];
            tmem_ld32(o_at + x, o);  // (of a tile without keys what a piece before left)
            tmem_wait_ld(o);
            // a row without weights is zero, also where its neighbours' values are not finite (0 * NaN in the product)
            if (inv == 0.0f) {
#pragma unroll
                for (int y = 0; y < 32; ++y) o[y] = 0;
            }
            // a lane has a row to itself: whole 32-byte sectors where the rows begin on them
            if (active && slot < 0) {
                if (wide) {
#pragma unroll
                    for (int y = 0; y < 32; y += 16)
                        if (x + y < p.a.D) {
                            uint32_t w[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                w[i] = pack2<T>(__uint_as_float(o[y + 2 * i]) * inv, __uint_as_float(o[y + 2 * i + 1]) * inv);
                            store32(out + x + y, w);
                        }
                } else {
#pragma unroll
                    for (int y = 0; y < 32; y += 8)
                        if (x + y < p.a.D) store8<T>(out + x + y, o + y, inv);
                }
            } else if (active) {
                float* dst = p.a.parts + part * p.a.D + x;
#pragma unroll
                for (int y = 0; y < 32; y += 8)
                    if (x + y < p.a.D) {
                        uint32_t w[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(__uint_as_float(o[y + i]) * inv);
                        store32(dst + y, w);
                    }
            }
            __syncwarp();
        }
        if (active) {
            if (slot >= 0)
                p.a.part_lse[part] = lse;
            else if (p.a.lse)
                p.a.lse[token * p.a.Hq + it.head + head] = lse;
        }
        tc_before();
    }
}

template <int DP, typename T>
__global__ void __launch_bounds__(kThreads, 1)
    attention_kernel(const __grid_constant__ Params p, const __grid_constant__ CUtensorMap qm,
                     const __grid_constant__ CUtensorMap km, const __grid_constant__ CUtensorMap vm) {
    extern __shared__ uint8_t raw[];
    __shared__ Barriers bars;
    Barriers* b = &bars;
    const uint32_t smem = (smem_u32(raw) + 1023) & ~1023u;
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int t = 0; t < 2; ++t) {
            mbar_init(&b->q_full[t], 1);
            mbar_init(&b->q_empty[t], 1);
            mbar_init(&b->s_full[t], 1);
            mbar_init(&b->s_read[t], 4);
            mbar_init(&b->p_full[t], 4);
            mbar_init(&b->o_full[t], 1);
            mbar_init(&b->turn[t], 1);
        }
        mbar_init(&b->drained, 2);
        for (int s = 0; s < 8; ++s) {
            mbar_init(&b->kv_full[s], 1);
            mbar_init(&b->kv_empty[s], 2);
        }
        b->dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&b->tmem)), "r"(kTmemColumns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = (uint32_t)uniform((int)b->tmem);
    pdl_wait();
    const Items items{p.a.items, b, uniform(p.a.cta_ptr[blockIdx.x]), uniform(p.a.cta_ptr[blockIdx.x + 1])};
    if (threadIdx.x < 4 * kCached && items.first + (int)threadIdx.x / 4 < items.last)
        reinterpret_cast<int4*>(b->items)[threadIdx.x] = reinterpret_cast<const int4*>(p.a.items + items.first)[threadIdx.x];
    __syncthreads();
    if (warp < kMmaWarp) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        softmax_role<DP, T>(p, tmem, b, items, warp >> 2, warp & 3, lane);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (warp == kLoadWarp) load_role<DP>(p, &qm, &km, &vm, smem, b, items);
        if (warp == kMmaWarp || warp == kMmaWarp + 1) {
            mma_role<DP>(p, smem, tmem, b, items, warp - kMmaWarp, lane);
            // every product and every arrival that it announced is done before the block ends
            __syncwarp();
            if (elect()) tc_commit(&b->drained);
            const unsigned long long t0 = globaltimer();
            while (!mbar_try(&b->drained, 0) && globaltimer() - t0 < kDrainLimitNs) {}
        }
        __syncwarp();
    }
    tc_before();
    __syncthreads();
    tc_after();
    if (warp == kMmaWarp)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemColumns) : "memory");
}

// Joins the parts of rows split along the keys, in their order: a warp takes a row, a lane four of its columns.  Bound by
// its launch and one round of loads (about 4 us behind the parts; launched while the attention drains).
template <typename T>
__global__ void __launch_bounds__(256) attention_join_kernel(const __grid_constant__ Params p) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    pdl_wait();
    const AttentionJoin join = p.a.joins[blockIdx.x];
    const int row = blockIdx.y * 8 + warp;
    if (row < join.n_tok * p.a.pack) {
        const int tok = row / p.a.pack, head = join.head + row - tok * p.a.pack;
        const float* lse = p.a.part_lse + (long long)join.slot * kRows + row;
        float top = -INFINITY;
        for (int i = 0; i < join.n_parts; ++i) {
            const float x = lse[(long long)i * kRows];
            top = x > top || x != x ? x : top;  // a NaN stays
        }
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        float sum = 0.0f;
        if (top != -INFINITY)
            for (int i = 0; i < join.n_parts; ++i) {
                const float w = expf(lse[(long long)i * kRows] - top);
                sum += w;
                if (4 * lane < p.a.D) {
                    const float4 x =
                        *reinterpret_cast<const float4*>(p.a.parts + (((long long)join.slot + i) * kRows + row) * p.a.D + 4 * lane);
                    o.x = fmaf(w, x.x, o.x);
                    o.y = fmaf(w, x.y, o.y);
                    o.z = fmaf(w, x.z, o.z);
                    o.w = fmaf(w, x.w, o.w);
                }
            }
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        const long long token = (long long)join.q_row + tok;
        if (4 * lane < p.a.D) {
            T* out = static_cast<T*>(p.a.out.data) + token * p.a.out.token_stride + head * p.a.out.head_stride + 4 * lane;
            *reinterpret_cast<uint2*>(out) = make_uint2(pack2<T>(o.x * inv, o.y * inv), pack2<T>(o.z * inv, o.w * inv));
        }
        if (lane == 0 && p.a.lse) p.a.lse[token * p.a.Hq + head] = sum == 0.0f ? -INFINITY : top + logf(sum);
    }
}

// ----------------------------------------------------------------- host --
// Boxes of 64 elements of a head x `heads` heads x `tokens` tokens.  The stride of an axis of one entry is never used
// but has to be a valid one.
cudaError_t make_map(CUtensorMap* map, int dtype, const geocache_heads& x, int D, int pack, int H, long long T, int tokens) {
    EncodeTiled encode = encode_tiled();
    if (!encode) return cudaErrorNotSupported;
    const cuuint64_t row = (cuuint64_t)D * 2, hs = H > 1 ? x.head_stride * 2 : row, ts = T > 1 ? x.token_stride * 2 : row;
    const CUtensorMapDataType type = dtype == GEOCACHE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    CUresult r;
    const cuuint32_t ones[4] = {1, 1, 1, 1};
    if (pack > 0) {
        const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)pack, (cuuint64_t)(H / pack), (cuuint64_t)T};
        const cuuint64_t strides[3] = {hs, H / pack > 1 ? hs * pack : row, ts};
        const cuuint32_t box[4] = {64, (cuuint32_t)pack, 1, (cuuint32_t)tokens};
        r = encode(map, type, 4, x.data, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                   CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    } else {
        const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)H, (cuuint64_t)T};
        const cuuint64_t strides[2] = {hs, ts};
        const cuuint32_t box[3] = {64, 1, (cuuint32_t)tokens};
        r = encode(map, type, 3, x.data, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                   CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    }
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int DP, typename T>
cudaError_t launch(const Params& p, const CUtensorMap& qm, const CUtensorMap& km, const CUtensorMap& vm, cudaStream_t s) {
    auto kern = attention_kernel<DP, T>;
    static const cudaError_t ready = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<DP>::kBytes);
    if (ready != cudaSuccess) return ready;
    cudaError_t e = launch_pdl(kern, dim3((unsigned)p.a.n_ctas), kThreads, Shape<DP>::kBytes, s, p, qm, km, vm);
    if (e != cudaSuccess || p.a.n_joins == 0) return e;
    // a block for every 8 rows of a tile
    const int rows = p.tok * p.a.pack;
    return launch_pdl(attention_join_kernel<T>, dim3((unsigned)p.a.n_joins, (unsigned)((rows + 7) / 8)), 256, 0, s, p);
}

}  // namespace

cudaError_t launch_attention(const AttentionArgs& a, cudaStream_t s) {
    Params p{};
    p.a = a;
    p.tok = kRows / a.pack;
    p.k_steps = (a.D + 15) / 16;
    // kind f16: binary32 accumulators, operands of `dtype`, 128 rows; the keys' head axis and the queries' are summed
    // (contiguous), the values' is not
    const uint32_t type = a.dtype == GEOCACHE_BF16 ? 1 : 0;
    const uint32_t idesc = 1u << 4 | type << 7 | type << 10 | (uint32_t)(kRows >> 4) << 24;
    p.qk_idesc = idesc | (uint32_t)(kKeys >> 3) << 17;
    p.pv_idesc = idesc | 1u << 16 | (uint32_t)(2 * p.k_steps) << 17;
    p.c = (float)((double)a.scale * 1.4426950408889634);
    p.wide_out = !((uintptr_t)a.out.data & 31) && !((a.out.token_stride | a.out.head_stride | a.D) % 16);
    CUtensorMap qm, km, vm;
    cudaError_t e = make_map(&qm, a.dtype, a.q, a.D, a.pack, a.Hq, a.q_tokens, p.tok);
    if (e != cudaSuccess) return e;
    if (a.k_tokens) {
        e = make_map(&km, a.dtype, a.k, a.D, 0, a.Hk, a.k_tokens, kKeys);
        if (e == cudaSuccess) e = make_map(&vm, a.dtype, a.v, a.D, 0, a.Hk, a.k_tokens, kKeys);
        if (e != cudaSuccess) return e;
    } else {
        km = vm = qm;  // no key is loaded
    }
    if (a.dtype == GEOCACHE_BF16)
        return a.D > 64 ? launch<128, __nv_bfloat16>(p, qm, km, vm, s) : launch<64, __nv_bfloat16>(p, qm, km, vm, s);
    return a.D > 64 ? launch<128, __half>(p, qm, km, vm, s) : launch<64, __half>(p, qm, km, vm, s);
}

cudaError_t attention_error_word(unsigned int** word) { return cudaGetSymbolAddress(reinterpret_cast<void**>(word), g_attention_error); }

}  // namespace geocache
