// Internal declarations of the 4-bit K/V cache: its layout and the launchers
// of its kernels (kvq.hip), shared with the C ABI (api.cpp) and the model's
// forward (kernels.hip).
#pragma once

#include "spade_internal.h"

namespace spade {

// A cache row (one position of one K/V head) is x_f = m + n_f s: codes n_f of
// 4 bits, one scale s and one minimum m (bfloat16) for the keys and one pair
// for the values.  Positions are stored in blocks of 32, each one contiguous
// run: the keys' codes, the values' codes, then (key pair, value pair) per
// position.
//   keys    position t: head_dim / 2 bytes at t head_dim / 2, feature f in
//           nibble f % 8 of word f / 8.  Sixteen positions are the A operand of
//           S^T = K Q^T: lane 16 q + c loads the q-th quarter of position c.
//   values  word (f / 8) of position t at ((t / 4) (head_dim / 8) + f / 8) 16
//           + (t % 4) 4: four positions of eight features are one 16-byte
//           piece, so a lane's load holds four positions (the k index of O^T =
//           V^T P^T) of its own eight features, and appending a position
//           writes whole words.  A half word has features 4 i .. 4 i + 3, each
//           as the sign of n - 7.5 and k = |n - 7.5| - 1/2 in 0 .. 7: the signs
//           at bits 15, 11, 7 and 3, k at bits 4 .. 6, 0 .. 2, 12 .. 14 and
//           8 .. 10, so that shifts by 0 and 4 of the half word and of its
//           bytes swapped bring every one to bits 15 and 4 .. 6.
//   pairs   8 bytes per position: scale and minimum (low and high half) of
//           the keys, then of the values.
constexpr int kKvqBlock = 32;
__host__ __device__ inline uint32_t kvq_block_bytes(int hd) { return (uint32_t)kKvqBlock * (hd + 8); }
__host__ __device__ inline uint32_t kvq_k_word(int t, int w, int hd) { return (uint32_t)(t * (hd >> 1) + 4 * w); }
__host__ __device__ inline uint32_t kvq_v_word(int t, int w, int hd) {
  return (uint32_t)(kKvqBlock * (hd >> 1) + ((t >> 2) * (hd >> 3) + w) * 16 + (t & 3) * 4);
}
__host__ __device__ inline uint32_t kvq_pair(int t, int hd) { return (uint32_t)(kKvqBlock * hd + 8 * t); }
// bytes of one (layer, request, K/V head)
inline size_t kvq_head_bytes(int max_len, int hd) {
  return (size_t)((max_len + kKvqBlock - 1) / kKvqBlock) * kvq_block_bytes(hd);
}
constexpr int kKvqMaxLen = 1 << 20;
constexpr int kKvqMaxRows = 16;  // rows per request of one attention call

// Rows of heads: element (request b, row i, head h, feature f) at b sb + i si +
// h sh + f.
struct KvqRows {
  const void* p;
  int64_t sb, si, sh;
};

struct KvqAppend {
  uint8_t* cache;  // the layer's [batch][KVH] heads
  size_t head_bytes;
  int B, R, H, KVH, hd, max_len;
  KvqRows q, k, v;  // q.p NULL: no queries
  int v_feature;    // distance of neighbouring features of v: 1, or float32 columns
  int bf16;         // inputs and q_out: bfloat16, else float32
  const float* gain_q;
  const float* gain_k;
  float eps;
  const float* rope;
  int rope_len;
  const int32_t* pos;
  const int32_t* shift;  // added to the position of every row, or NULL
  const int32_t* lens;
  const int32_t* rows;
  void* q_out;
  int64_t qo_ld;
  float* weights;  // the layer's [batch][KVH][max_len], or NULL
  uint32_t* err;
  int run;  // set by the launcher: row groups of a workgroup
};
hipError_t launch_kvq_append(const KvqAppend& a, hipStream_t st);

struct KvqRead {
  const uint8_t* cache;
  size_t head_bytes;
  int B, R, KVH, hd, max_len, bf16;
  const int32_t* start;
  const int32_t* rows;
  void* k;
  void* v;
};
hipError_t launch_kvq_read(const KvqRead& a, hipStream_t st);

struct KvqAttend {
  const uint8_t* cache;
  size_t head_bytes;
  int B, R, H, KVH, G, hd, max_len;
  const void* q;
  int64_t q_ld;
  int bf16;  // q and out
  float scale;
  const int32_t* lens;
  const int32_t* rows;
  int max_keys;  // bound of lens + rows in use, in 1 .. max_len (may be below R)
  void* out;
  int64_t out_ld;
  size_t split;  // 0, or float32 calls: out is the two bf16 terms of a GEMM operand, this many elements apart
  const float* w_in;
  float* w_out;  // the layer's [batch][KVH][max_len], or NULL
  int w_rows;
  float* part_o;   // [slot][G R][hd] segments' partials
  float* part_ml;  // [slot][G R][2]
  float* lse;      // [B][KVH][G R]
  size_t part_rows;  // rows that part_o holds
  uint32_t* err;
  // set by the launcher
  int WG;     // ranges
  int parts;  // > 0: ranges are equal parts of a head, this many; 0: of the whole batch
  int TG;  // 16-row tiles of a K/V head's rows
};
size_t kvq_attend_floats(int B, int H, int KVH, int hd, int R, size_t* part_ml, size_t* lse);
hipError_t launch_kvq_attend(const KvqAttend& a, hipStream_t st);

struct KvqEvict {
  const uint8_t* cache;
  size_t head_bytes;
  uint8_t* out;
  size_t out_head_bytes;
  int L, batch, B, KVH, hd, max_len, out_batch, out_max_len;
  int budget, recent;
  const float* w;
  float* w_out;
  const int32_t* lens;
  int32_t* lens_out;
  int32_t* kept;  // [L][batch][KVH][budget]
  int32_t* evicted;  // [B] positions evicted so far, or NULL
};
hipError_t launch_kvq_evict(const KvqEvict& a, hipStream_t st);

// counts of requests that start over: evicted[b] = 0 where lens[b] is 0
hipError_t launch_kvq_restart(int B, const int32_t* lens, int32_t* evicted, hipStream_t st);
// rows[b] of a prefill forward of R rows per request: the prompt tokens left, at most R
hipError_t launch_kvq_prefill_rows(int b0, int nb, int R, const int32_t* n_cache, const int32_t* base,
                                   const int32_t* lens, int32_t* rows, hipStream_t st);

}  // namespace spade
