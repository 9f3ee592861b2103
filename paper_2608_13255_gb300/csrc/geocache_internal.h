// Internal interface between the C ABI layer (geocache_api.cu) and the
// kernels (geocache_kernels.cu).  Not installed; not part of the ABI.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "geocache.h"

namespace geocache {

// Per-step sampler constants, formed in double on the host and rounded once.
struct ReconCoef {
    int enabled;     // 0: transport only
    int sampler;     // GEOCACHE_DDIM / GEOCACHE_FM_EULER
    int pred_kind;   // geocache_pred
    float st, s1t, inv_s1t, sp, s1p;   // DDIM: sqrt(ab_t), sqrt(1-ab_t), 1/sqrt(1-ab_t), sqrt(ab_prev), sqrt(1-ab_prev)
    float inv_sigma, dsigma;           // FM: 1/sigma, sigma_next - sigma
};

struct TransportArgs {
    int B, N, H, W, C, K, a;
    int c0, cn;                         // channel window [c0, c0 + cn) handled by this launch
    int mode;                           // geocache_corr_mode
    int write_anchor_rows;              // 0 when x0_out aliases x0_prev (rows written afterwards)
    int lat_dtype;                      // geocache_dtype
    int update;                         // geocache_update (Eq. 1 or the value-copy ablation)
    int drop_first_copy;                // test hook: unit 0's staged copies are not issued
    unsigned long long wait_limit_ns;   // limit of the bounded waits
    const float* pos;
    const uint8_t* valid;
    const geocache_camera* cams;
    const float* tau;
    const int32_t* idx;
    const float* w;
    const uint8_t* keep;
    const int32_t* tile_ptr;
    const geocache_tap_record* records;
    long long max_records;
    const int32_t* src_ptr;             // source index of the records (optional; see geocache_corr)
    const int32_t* src_rec;
    float* workspace;
    const float* x0_new;
    const float* x0_prev;
    float* x0_out;
    const void* x_t;
    void* x_next;
    float* pred_out;
    ReconCoef coef;
    int32_t anchors[GEOCACHE_MAX_VIEWS];
    int32_t slot_of[GEOCACHE_MAX_VIEWS];   // slot in `anchors`, -1 for non-anchors
    int32_t others[GEOCACHE_MAX_VIEWS];    // the views outside the anchor set, ascending
    long long workspace_floats;            // size of `workspace` (0 without one)
};

// The sparse step with wide latents (C >= kPlaneMinChannels) keeps the
// anchors' increments as a plane [b][anchor slot][channel group][token] x 4
// channels at the start of the workspace.  It takes that path only when the
// workspace holds max_records * C floats plus the plane, so that a minimal
// workspace keeps the per-record rows (see geocache_transport_workspace).
constexpr int kPlaneMinChannels = 8;
inline long long plane_floats(long long B, long long a, int C, long long HW) {
    return B * a * (long long)((C + 3) / 4) * 4 * HW;
}

struct RowAnchors {
    int32_t v[GEOCACHE_MAX_VIEWS];
};
cudaError_t launch_copy_rows(const void* src, void* dst, long long row_bytes, int B, int N, int a,
                             const RowAnchors& anc, bool pack, cudaStream_t s);

cudaError_t launch_tau(const float* pos, const uint8_t* valid, int B, int N, int H, int W,
                       float tol_frac, float* tau, cudaStream_t s);
cudaError_t launch_build_corr(const geocache_corr& c, cudaStream_t s);
// sparse form: per-tile record counts and their exclusive prefix sum in
// tile_ptr (tile_ptr[n] = total, or -1 when the total exceeds INT32_MAX)
cudaError_t launch_tile_ptr(const geocache_corr& c, cudaStream_t s);
cudaError_t launch_fill_records(const geocache_corr& c, cudaStream_t s);
// source index of the records (c.src_ptr, c.src_rec), after the records
cudaError_t launch_src_index(const geocache_corr& c, cudaStream_t s);
cudaError_t launch_permute_records(const geocache_tap_record* src, const int32_t* perm, geocache_tap_record* dst,
                                   long long n, cudaStream_t s);
__host__ __device__ int tiles_per_view(int H, int W);
cudaError_t launch_transport(const TransportArgs& t, cudaStream_t s);
cudaError_t launch_copy_anchor_rows(const TransportArgs& t, cudaStream_t s);
cudaError_t launch_reconstruct(const void* x_t, const float* x0, void* x_next, int lat_dtype, int64_t n,
                               const ReconCoef& coef, float* pred_out, float* x0_store, cudaStream_t s);

// Reads the status words of all sources (one copy and one wait), and clears them with `clear`.
cudaError_t read_device_error(unsigned int* out, bool clear, cudaStream_t s);
cudaError_t raster_error_word(unsigned int** word);     // their device addresses
cudaError_t rope_error_word(unsigned int** word);
cudaError_t attention_error_word(unsigned int** word);
cudaError_t linear_error_word(unsigned int** word);
// test hook of the bounded waits (geocache_debug_set_wait)
void set_debug_wait(unsigned long long limit_ns, int drop_first_copy);
// position maps at the token grid H x W; ss > 1: rendered at ss x H by
// ss x W (zbuf holds B*N*H*W*ss*ss words) and pooled to the token grid
cudaError_t launch_raster(const float* V, long long nv, const int32_t* F, long long nf, const int64_t* face_off,
                          int B, const geocache_camera* cams, int N, int H, int W, int ss, unsigned long long* zbuf,
                          float* pos, uint8_t* valid, cudaStream_t s);
cudaError_t launch_pool_posmaps(const float* pos_hi, const uint8_t* valid_hi, long long n_maps, int H, int W, int ss,
                                float* pos, uint8_t* valid, cudaStream_t s);

struct RopeTableArgs {
    double freq[128];        // of the pairs
    double magnitude;
    const int32_t* pos;      // or nullptr: the slot's index
    float2* table;           // [n_slots][row_pairs], written at [first_pair, first_pair + pairs)
    long long n_slots;
    int pairs, row_pairs, first_pair;
};
cudaError_t launch_rope_table(const RopeTableArgs& a, cudaStream_t s);

// Heads [0, H) of the queries are followed by those of the keys.
struct NormRopeArgs {
    const void* in[2];       // queries, keys
    void* out[2];
    long long in_ts[2], in_hs[2], out_ts[2], out_hs[2];   // strides in elements
    const float* weight[2];  // [D] or nullptr
    const float2* table;     // [n_slots][rot / 2]
    const int32_t* slots;    // [T] or nullptr
    long long n_slots;
    int T, Hq, Hk, D, rot, layout, norm;
    float eps;
    int dtype;
};
cudaError_t launch_norm_rope(const NormRopeArgs& a, cudaStream_t s);

// One piece of an attention launch: up to two tiles of 128 query rows (tile t's tokens start at q_row + t *
// (128 / pack); a row is one of `pack` heads of a token) of one sequence and key/value head, over a range of its
// keys in tiles of 128.
struct alignas(16) AttentionItem {
    int32_t q_row;      // first token of tile 0
    int32_t head;       // first query head
    int32_t kv_head;
    int32_t kv_row;     // first key
    int32_t n_keys;     // keys from kv_row to the sequence's end
    int32_t sees;       // causal: keys from kv_row on that tile 0's first token sees (may be <= 0)
    int32_t n_tok[2];   // tokens of a tile; 0: the tile takes no part
    int32_t n_kv[2];    // key tiles that the tile sees
    int32_t slot[2];    // the tile's part of the workspace, -1: it writes the output
    int32_t unused[4];
};
static_assert(sizeof(AttentionItem) == 64, "read as four 16-byte words");
// The parts slot .. slot + n_parts of a tile's rows.
struct AttentionJoin {
    int32_t q_row, n_tok, head, slot, n_parts, unused[3];
};
static_assert(sizeof(AttentionJoin) == 32, "layout of the schedule");
constexpr int kAttentionRows = 128;   // query rows of a tile
constexpr int kAttentionKeys = 128;   // keys of a tile
constexpr long long kAttentionTokens = 0x7fffffffLL - 1023;   // rows: an int32 index may run over the end by some tiles
// schedule: n_ctas + 1 int32 offsets of the blocks' items (padded to 64 bytes), the items, the joins
inline long long attention_items_at(int n_ctas) { return ((long long)n_ctas + 1 + 15) / 16 * 64; }
// workspace: n_slots tiles of [128][D] f32, then their [128] f32 lse
inline long long attention_slot_bytes(int D) { return 128LL * D * 4 + 128 * 4; }

struct AttentionArgs {
    const int32_t* cta_ptr;
    const AttentionItem* items;
    const AttentionJoin* joins;
    int n_ctas, n_joins, pack, D, Hq, Hk, causal, dtype;
    long long q_tokens, k_tokens, n_slots;
    geocache_heads q, k, v, out;
    float* lse;
    float scale;
    float* parts;       // workspace
    float* part_lse;
    unsigned long long wait_limit_ns;
    int drop_first_copy;
};
cudaError_t launch_attention(const AttentionArgs& a, cudaStream_t s);

struct NormRowsArgs {
    geocache_rows x, residual, residual_out, out;   // residual.data = nullptr: none
    const float* weight;     // [C] or nullptr
    float* scale;            // [T]: the output is e4m3; nullptr: of the input's type
    long long T;
    int C, norm, dtype, residual_f32;
    float eps;
    // set by the launch: threads of a row, the first distance of its warps' join, which rows are whole
    // words, 1 / C
    int lanes, join, x_words, residual_words, out_words, weight_words;
    float inv_C;
};
cudaError_t launch_norm_rows(const NormRowsArgs& a, cudaStream_t s);

struct LinearArgs {
    geocache_rows x, w, out, residual;   // residual.data = nullptr: none
    long long T;
    int K, N, in_dtype, out_dtype, act, gated;
    const float *bias, *x_scale, *w_scale;
    unsigned long long wait_limit_ns;
    int drop_first_copy;
    unsigned int* error;   // status word, set by the launch
};
cudaError_t launch_linear(const LinearArgs& a, cudaStream_t s);
// the kernel that products are to take or took (geocache_debug_set_linear); kernel 0: none
struct LinearKernel {
    int kernel, size, splits;
};
void set_debug_linear(const LinearKernel& k);
LinearKernel last_linear();
// whether the kernel that is set can take the product
bool debug_linear_fits(const LinearArgs& a);
// the kernel for many tokens, with tiles of 256 or 128 rows of weights
cudaError_t launch_linear_pairs(const LinearArgs& a, int features, int sms, cudaStream_t s);
// the limit of bounded waits, and the test hook's pending request (consumed)
unsigned long long debug_wait_limit_ns();
int take_drop_first_copy();

// Counts kernels that the calling thread's current library call enqueues
// (geocache_last_launches).
void note_launches(int n);

// Launch with programmatic stream serialization: the kernel may become resident
// while the one before it in the stream drains, and begins with pdl_wait, before
// it touches memory.  It hides the launch behind the predecessor's tail (us a
// call among others of its kind: full step of 64 assets 47.2 -> 44.8, MASK step
// of 8 assets 14.7 -> 12.7, pooling of 96 maps 35.2 -> 32.9).
template <typename... Params, typename... Args>
cudaError_t launch_pdl(void (*kern)(Params...), dim3 grid, int threads, size_t dyn_smem, cudaStream_t s, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = dyn_smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    note_launches(1);
    return cudaLaunchKernelEx(&cfg, kern, Params(args)...);
}

// Records a status and its message for geocache_last_error(); returns status.
int set_error(int status, const char* fmt, ...);

}  // namespace geocache
