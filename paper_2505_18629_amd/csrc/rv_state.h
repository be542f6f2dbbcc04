// The model and cache handles behind the C ABI, and the error helpers of the
// files that implement it.
#pragma once
#include <string>
#include <vector>

#include "rv_internal.h"
#include "rv_tiles.h"

inline rv_status hip_fail(hipError_t e, const char* what) {
  return rv_fail(RV_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

#define HIP_TRY(expr, what)                 \
  do {                                      \
    hipError_t e_ = (expr);                 \
    if (e_ != hipSuccess) return hip_fail(e_, what); \
  } while (0)

struct rv_model {
  rv_config cfg;
  uint64_t seed;
  char* base;
  size_t bytes;
  int es;
  MatDesc qkv, o, gateup, down, lm;
  void* embed;
  float* norm_f;
  void* lm_head;
  std::vector<void*> w_qkv, w_o, w_gateup, w_down;
  std::vector<float*> n1, n2;
  const float *q_gain = nullptr, *k_gain = nullptr;  // [n_layers][head_dim] norms of queries and keys, the caller's
};

struct rv_cache {
  rv_model* m;
  int B, max_len, max_block, max_drafts;
  int kv_len;  // cached positions per (sequence, kv head): max_len rounded up to whole 64-key tiles
  char* base;
  size_t bytes;
  int rows_cap, out_rows_cap, r1_cap, nchunk;
  size_t kv_layer_elems;
  char* kc;   // K cache [layer][b][kv_head][kv_len x hd] (order: put_k4 / put_v4): bf16 hi plane, or fp32
  char* vc;
  char* kc2;  // bf16 lo planes (bf16 models)
  char* vc2;
  int* tile_own;     // [b][kv_len / 64]: slot that holds the tile (the device's copy of `tiles`)
  TileOwners tiles;  // as of the last call
  int* ids;
  float* rope_cos;
  float* rope_sin;
  int* seq_bad;
  int *row_pos, *row_seq, *row_bad;
  int *seg_b, *seg_row0, *seg_n, *seg_pos0;
  float* h;
  // matmul operands: first plane (bf16 hi, or fp32) and bf16 lo plane
  void *xn, *xn2, *qbuf, *qbuf2, *att, *att2, *act, *act2, *lm_x, *lm_x2;
  size_t part_entries;
  float *part_o, *part_ml;
  float* gpart;  // k-group partials of a split matmul [gk][rows][max(d_model, qkv rows)], gk*rows <= gpart_rows
  int gpart_rows;
  float *logits, *z, *lp, *hpart, *lse, *margins, *entropy;
  int* lm_src;                      // block row of each LM-head row of the last verify
  int last_R1;                      // fused rows of the last verify
  uint8_t last_kb[RV_MAX_BATCH];    // its per-sequence draft counts
  int* argmax;
  int last_k = -1;
  int force_rows = 0, force_mt = 0, force_gk = 0;  // rv_debug_force_matmul
  // event profiler
  bool prof = false;
  std::vector<hipEvent_t> prof_ev;   // pairs: start, stop
  std::vector<int> prof_cls;
  size_t prof_used = 0;
  ~rv_cache() {
    for (hipEvent_t e : prof_ev) (void)hipEventDestroy(e);
  }
};

// ---------------------------------------------------------------- shared tiles
// Every tile back in its sequence's own slot (what they held is not copied).
rv_status reset_owners(rv_cache* c, hipStream_t st);
// RV_E_STATE where another sequence reads what positions pos .. pos + rows - 1 of b overwrite.
rv_status check_writable(const rv_cache* c, int b, int pos, int rows);
// Everything of a but the layer's planes and the rows themselves.  rows: row0[B] > 0.
void plan_attend(const rv_cache* c, const int* pos0, const int* row0, ShareArgs& a);
