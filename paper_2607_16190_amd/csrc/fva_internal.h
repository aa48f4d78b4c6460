// Internal launch interface between the C ABI layer and the HIP kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "fva_geometry.h"

namespace fva {

struct RouteArgs {
  const void* Q;
  const void* K;
  int batch, heads, tokens;
  int64_t stride_b, stride_h, stride_n;
  int T, H, W, bt, bh, bw;
  double p;
  int k_min;
  uint8_t* mask;
  int32_t* counts;
  int32_t* kv_idx;  // may be null
  // slack-aware augmentation (null rank_of: plain routing)
  const int32_t* rank_of = nullptr;  // [batch * heads] rank of every head (device)
  int n_ranks = 0;
  double n1 = 0.0, n2 = 0.0;
  int32_t* rank_extra = nullptr;  // [n_ranks] extra blocks per row of each rank (device) or null
  int32_t* extra_head = nullptr;  // [batch * heads] workspace tail
  void* row_cuts = nullptr;       // [batch * heads * nb] last kept block of each routed row (augmentation)
  void* workspace;
  hipStream_t stream;
};

struct AttnArgs {
  const void* Q;
  const void* K;
  const void* V;
  void* O;
  int batch, heads, tokens;
  int64_t stride_b, stride_h, stride_n;
  int T, H, W, bt, bh, bw;
  const uint8_t* V8;      // E4M3 V tiles (FP8 variant) or null
  const int32_t* vexp;    // per-channel exponents of V8 (FP8 variant)
  const uint8_t* mask;
  const int32_t* counts;  // null: rebuilt from mask in the workspace
  const int32_t* kv_idx;  // null together with counts
  float scale;
  uint32_t flags;
  int64_t* trace;  // null unless tracing
  void* workspace;
  hipStream_t stream;
  bool lean = false;  // workspace laid out without list copies and chunk items
};

struct QuantizeArgs {
  const void* V;
  int batch, heads, tokens;
  int64_t stride_b, stride_h, stride_n;
  int T, H, W, bt, bh, bw;
  uint8_t* V8;
  int32_t* vexp;
  void* workspace;
  hipStream_t stream;
};

size_t route_workspace_bytes(int batch, int heads, int nb);
size_t route_sasa_workspace_bytes(int batch, int heads, int nb);
size_t attn_workspace_bytes(int batch, int heads, const Geometry& g, uint32_t flags);
int64_t attn_trace_words(int batch, int heads, int nb);

hipError_t launch_route(const RouteArgs& a);
hipError_t launch_attn(const AttnArgs& a);

// Allocation-free attention: scratch bytes a shape needs, the capacity of
// the library's static device scratch, and the launch (persistent scheduler,
// caller's counts and kept lists, no split rows) on that scratch.
size_t attn_noalloc_bytes(int batch, int heads, const Geometry& g);
size_t attn_noalloc_capacity();
hipError_t launch_attn_noalloc(const AttnArgs& a);

// E4M3 V quantisation for the FP8 attention variant (fp8_kernels.hip).
size_t quantize_v_workspace_bytes(int batch, int heads);
hipError_t launch_quantize_v(const QuantizeArgs& a);

// Hilbert-curve token order and row permutation (curve_kernels.hip).
size_t curve_workspace_bytes(int T, int H, int W);
hipError_t launch_curve_order(int T, int H, int W, int32_t* perm, void* workspace, hipStream_t stream);
hipError_t launch_permute_rows(const void* src, void* dst, int batch, int heads, int tokens, int64_t sb, int64_t sh,
                               int64_t sn, const int32_t* perm, int direction, hipStream_t stream);

// Rotary positions (rope_kernels.hip). One of Q and K; `out` may be `in`.
struct RopeTensor {
  const void* in = nullptr;
  void* out = nullptr;
  int heads = 0;
  int64_t sb = 0, sh = 0, sn = 0;
};

struct RopeArgs {
  RopeTensor q, k;  // k.heads == 0: Q alone
  int dtype;        // FVA_BF16, FVA_FP16 or FVA_FP32
  int batch, tokens;
  int H, W, dim_t, dim_y, dim_x, t0, y0, x0;
  double log2_theta;
  bool halves, inverse;
  const int32_t* ids;  // token ids, or null: 0, 1, ..
  int64_t ids_stride;  // between batches
  hipStream_t stream;
};

hipError_t launch_rope(const RopeArgs& a);

// Paged 8-bit cache (cache_kernels.hip).
constexpr int kPlanStreams = 2048;   // streams of a plan: their prefix sums are kept in LDS
constexpr int kCacheExpMin = -100;   // smallest exponent of a scale: 448 * 2^-100 is far below any activation, and
                                     // every scaled code stays a normal fp32 and bf16 number

struct PlanArgs {
  const int32_t* held;
  const int32_t* fresh;
  int streams, page;
  const int32_t* state;
  int32_t* ring;
  int ring_size;
  int32_t* table;
  int width, tokens;
  int32_t* kv_len;
  int32_t* q_start;
  int32_t* slots;
  int32_t* ids;
  int32_t* state_out;
  hipStream_t stream;
};

struct StoreArgs {
  const void* K;
  const void* V;
  int batch, heads, tokens;
  int64_t stride_b, stride_h, stride_n;
  const int32_t* slots;
  uint8_t* k8;
  uint8_t* v8;
  int32_t* k_exp;
  int32_t* v_exp;
  int pages, page;
  int window = 0;  // token rows a wave looks through for the runs it stores
  hipStream_t stream;
};

// A divisor of non-negative 32-bit integers as a multiplier and a shift.
struct Divisor {
  uint32_t mul;
  int shift;
};

struct CacheAttnArgs {
  const void* Q;
  void* O;
  int heads, kv_heads, tokens;
  int64_t stride_h, stride_n;
  const uint8_t* k8;
  const uint8_t* v8;
  const int32_t* k_exp;
  const int32_t* v_exp;
  int pages, page, page_shift;
  const int32_t* table;
  int width;
  const int32_t* kv_len;
  const int32_t* q_start;
  int streams, max_q, frame, window;
  float scale;
  float* partial;
  hipStream_t stream;
  // set by the launcher
  int group = 1;       // query heads per K/V head
  int rows = 16, row_shift = 4;  // query rows of a tile, a power of two
  int slots = 0;       // workgroups per K/V head that the keys are split for (large tiles: at most); 0: not split
  int32_t* chunk = nullptr;  // the chunk length the attention came to, for the merge
  double inv_slots = 0.0;  // 1 / slots
  bool ramp = false;   // rows of a stream see more and more keys: its tiles are weighed by their mean
  int64_t items = 0;   // items there can be
  int partials = 0;    // partial results there is room for, per K/V head
  int64_t items_per_head = 0;
  int most_keys = 0;   // that any tile sees, at most
  Divisor by_group, by_heads, by_frame;
};

hipError_t launch_cache_plan(const PlanArgs& a);
hipError_t launch_cache_store(StoreArgs a);
// Workgroups of up to 256 threads of a call: a grid of 2^32 threads and more is cut to 32 bits
// without an error.
constexpr int64_t kCacheWorkgroups = ((int64_t)1 << 24) - 1;
bool cache_attn_fits(int tokens, int heads, int kv_heads, int streams, int max_q, int64_t most_keys);
size_t cache_attn_workspace_bytes(int tokens, int heads, int kv_heads, int streams, int max_q, int64_t most_keys);
hipError_t launch_cache_attn(CacheAttnArgs a);

}  // namespace fva
