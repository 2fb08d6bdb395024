// Internal declarations of the calls for trees of drafts over a bfloat16 cache:
// the launchers of their kernels (tree.hip), used by the C ABI (api.cpp).
#pragma once

#include "spade_internal.h"

namespace spade {

constexpr int kTreeMaxLen = 1 << 20;
constexpr int kTreeMaxRows = 64;  // rows per request of attend and commit: a row's ancestors are one word

// The [batch][KVH] heads of one layer, keys and values apart (k_cache_index,
// v_cache_index); head_elems from one to the next.
struct TreeCache {
  uint16_t* k;
  uint16_t* v;
  int64_t head_elems;
};

struct TreeAppend {
  TreeCache cache;
  int B, R, H, KVH, hd, max_len;
  const void* q;  // NULL: no queries
  const void* k;
  const void* v;
  int64_t q_ld, k_ld, v_ld;
  int bf16;            // inputs and q_out: bfloat16, else float32
  const double* freq;  // [pairs] angle per position
  int pairs;           // 0: no rotation
  int interleaved;
  float amplitude;
  const int32_t* pos;    // [B], or NULL: lens
  const int32_t* depth;  // [B][R], or NULL: i
  const int32_t* lens;
  const int32_t* rows;
  void* q_out;
  int64_t qo_ld;
  uint32_t* err;
  // set by the launcher
  int run;        // heads that a wave of the rotated part goes through
  int qk_blocks;  // workgroups of that part; the values' follow
};
hipError_t launch_tree_append(const TreeAppend& a, hipStream_t st);

struct TreeRead {
  TreeCache cache;
  int B, R, KVH, hd, max_len, bf16;
  const int32_t* start;
  const int32_t* rows;
  void* k;
  void* v;
  int k_blocks;  // set by the launcher
};
hipError_t launch_tree_read(const TreeRead& a, hipStream_t st);

struct TreeAttend {
  TreeCache cache;
  int B, R, H, KVH, G, hd;
  const void* q;
  int64_t q_ld;
  int bf16;  // q and out
  float scale;
  const int32_t* parents;  // [B][R], or NULL: i - 1
  const int32_t* lens;
  const int32_t* rows;
  int max_keys;
  void* out;
  int64_t out_ld;
  float* part_o;      // [request, K/V head, split, packed row][hd]
  float* part_ml;     // ... [2]
  int32_t* plan;      // [B + 1] blocks of 32 positions of a split; a request's first row in part_o
  size_t part_rows;   // rows that part_o holds
  uint32_t* err;
  // set by the launcher
  int tile;  // packed rows of a workgroup
  int RB;    // workgroups over the packed rows of a K/V head
  int WG;    // 0: a workgroup takes all keys; else most workgroups of a call whose keys are split
};
// rows of part_o that any call of up to max_rows rows needs
size_t tree_part_rows(int G, int max_rows);
hipError_t launch_tree_attend(const TreeAttend& a, hipStream_t st);

struct TreeCommit {
  TreeCache cache;  // of layer 0
  int64_t layer_elems;
  int L, B, R, KVH, hd, max_len;
  const int32_t* tokens;
  const int32_t* parents;
  const int32_t* next;
  const int32_t* rows;
  const int32_t* lens;
  int32_t* lens_out;
  int32_t* n_accepted;
  int32_t* path;
  int32_t* correction;
  uint32_t* err;
};
hipError_t launch_tree_commit(const TreeCommit& a, hipStream_t st);

}  // namespace spade
