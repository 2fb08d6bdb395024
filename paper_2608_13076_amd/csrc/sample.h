// Internal declarations of the filtered sampler: the launcher of its kernels
// (sample.hip), used by the C ABI (api.cpp).
#pragma once

#include "spade_internal.h"

namespace spade {

constexpr int kSampleMaxVocab = 1 << 20;
constexpr int kSampleSlice = 4096;  // tokens of a workgroup of the first pass: 16 per thread
constexpr int kSampleBins = 128;    // of a slice's weights
constexpr int kSampleList = 8192;   // candidates of a row kept apart
constexpr int kSampleSub = 256;     // parts of the border's bins, where they hold more
constexpr int kSampleParts = 32;    // most workgroups of a row in the second pass

// What the passes of a row hand on.
struct SampleRow {
  double mass;    // of the tokens above bin `lo`, over the largest weight
  double total;   // of all (tail: but those of the window's last bin)
  float max;
  int lo, hi;     // bins whose tokens are listed (below the top bin)
  int above;      // tokens above bin lo
  int k_in;       // whether the first top_k end in the list
  int bits;       // of a listed weight, an integer of 2^-bits of the first listed bin's edge
  int tail;       // whether the weight of the window's last bin is added up by itself
  int sub;        // bits of a place of these bins below a part of theirs (-1: their tokens are listed)
  float least, below;  // logits of these bins: from `least` on, below `below`
  double inv_T, cut, inv_sum;  // probabilities: exp(-d) inv_sum where d <= cut
  uint32_t key, id;            // and the token comes no later than this one
};

// A token of the draw.
struct SampleDraw {
  double s;  // its score
  int id;
  double d;  // its distance from the largest logit
};

struct SampleArgs {
  int rows, V, bf16;
  const void* logits;
  int64_t ld;
  int per;  // rows of a request
  float temperature, top_p, min_p;
  int top_k;
  const float* d_temperature;  // [requests], or NULL: the value above
  const int32_t* d_top_k;
  const float* d_top_p;
  const float* d_min_p;
  const float* u;
  int32_t* tokens;
  float* chosen;  // or NULL
  float* probs;   // or NULL
  uint32_t* err;
  // workspace
  float* smax;          // [rows][NS] largest logit of a slice
  int32_t* sarg;        // ... its lowest token (greedy rows)
  uint64_t* hist;       // [rows][NS][kSampleBins] count and weight
  SampleDraw* best;     // [rows][NS] of a part (or slice)
  double* sum;          // ... the weight of its kept tokens
  SampleRow* row;       // [rows]
  uint32_t* count;      // [rows] listed tokens
  uint64_t* tail;       // [rows] weight in the window's last bin
  uint2* list;          // [rows][kSampleList] token and logit
  uint64_t* sub_mass;   // [rows][kSampleSub] weight of a part of the border's bins
  uint32_t* sub_count;  // ... its tokens
  int NS, NW, spw;      // slices, parts, slices of a part
};
size_t sample_workspace(int rows, int V, SampleArgs* a, uint8_t* base);
hipError_t launch_sample(const SampleArgs& a, hipStream_t st);

}  // namespace spade
