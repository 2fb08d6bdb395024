// Kernels of the calls for trees of drafts over a bfloat16 cache in the model's
// layout (k_cache_index, v_cache_index):
//   tree_append_kernel  rotation by position, keys and values of new rows
//   tree_read_kernel    rows of the cache
//   tree_attend_kernel  rows that see the context, their ancestors and themselves
//   tree_merge_kernel   the partials of a row's splits
//   tree_walk_kernel    the path whose tokens were drawn
//   tree_move_kernel    closes the path's rows up
#include "tree.h"

#include <float.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "device_lanes.h"

namespace spade {

namespace {

__device__ __forceinline__ uint32_t pk_bf16(float a, float b) {
  typedef __attribute__((ext_vector_type(2))) float f2;
  typedef __attribute__((ext_vector_type(2))) __bf16 b2;
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2){a, b}, b2));  // one v_cvt_pk_bf16_f32
}
__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// lengths come from the caller's device memory: sums stop at the type's ends
__device__ __forceinline__ int add_sat(int a, int b) { return __builtin_elementwise_add_sat(a, b); }

// STREAM: what a large call reads or writes once goes past the caches.
typedef __attribute__((ext_vector_type(2))) uint32_t Words2;
typedef __attribute__((ext_vector_type(4))) float Floats4;
template <bool STREAM, typename T>
__device__ __forceinline__ T get(const T* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(p);
  else return *p;
}
template <bool STREAM, typename T>
__device__ __forceinline__ void set(T* p, T v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, p);
  else *p = v;
}

template <bool BF16, bool STREAM = false>
__device__ __forceinline__ void load4(const void* base, int64_t at, float* x) {
  if constexpr (BF16) {
    const Words2 w = get<STREAM>((const Words2*)((const uint16_t*)base + at));
    x[0] = lo_f(w.x);
    x[1] = hi_f(w.x);
    x[2] = lo_f(w.y);
    x[3] = hi_f(w.y);
  } else {
    const Floats4 w = get<STREAM>((const Floats4*)((const float*)base + at));
    x[0] = w.x;
    x[1] = w.y;
    x[2] = w.z;
    x[3] = w.w;
  }
}

template <bool BF16, bool STREAM = false>
__device__ __forceinline__ void store4(void* base, int64_t at, const float* x) {
  if constexpr (BF16) set<STREAM>((Words2*)((uint16_t*)base + at), Words2{pk_bf16(x[0], x[1]), pk_bf16(x[2], x[3])});
  else set<STREAM>((Floats4*)((float*)base + at), Floats4{x[0], x[1], x[2], x[3]});
}

// ---------------------------------------------------------------------------
// Append.  hd / 8 lanes hold a head: pair group p < pairs / 4 the features of
// pairs 4 p .. + 3 (halves: 4 p .. + 3 and pairs + 4 p .. + 3; neighbours: 8 p ..
// + 7), the lanes behind the eight features each that are not rotated.  A workgroup
// takes 16 rows (hd 64: 32) and goes through heads: each lane computes its row's
// four angles once, and the 16-byte pieces of neighbouring positions, which share
// the keys' cache lines, leave from one place.  The angle pos f is a product in
// double whose whole turns are taken off exactly, so far positions lose nothing but
// the product's rounding (2^-53 of the angle; a float32 angle is off by 0.004 at 100
// thousand positions); sine and cosine are rounded once to float32.
//
// Values are stored by feature: a lane takes two features of eight neighbouring
// positions, whole 16-byte pieces where the rows cover them.
//
// Bound by memory: 4003 rows of 32 + 32 heads of 128 in bfloat16 read and write
// 197 MB in 47 us, 4.2 TB/s (a large copy: 5.1).  A wave that takes four heads of one
// row instead, so that a line of keys is written from eight places, took 78 us where this
// took 55 (both through the caches).  More loads in flight, other numbers of heads per workgroup (a twentieth to a
// quarter of them) and 16-byte loads change less than a tenth; without the angles
// it takes as long.
// ---------------------------------------------------------------------------
template <int HD, bool BF16, bool STREAM>
__device__ __forceinline__ void append_qk(const TreeAppend& p, int block) {
  constexpr int LPH = HD / 8, RPW = 64 / LPH;  // lanes a head, rows a wave
  const int lane = threadIdx.x & 63, c = lane % LPH;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int HQ = p.q != nullptr ? p.H : 0, heads = HQ + p.KVH, parts = (heads + p.run - 1) / p.run;
  const int rows16 = block / parts, part = block - rows16 * parts;
  const int64_t row = ((int64_t)rows16 * 4 + wave) * RPW + lane / LPH;
  if (row >= (int64_t)p.B * p.R) return;
  const int b = (int)(row / p.R), i = (int)(row - (int64_t)b * p.R);
  const int L = p.lens[b], n = p.rows != nullptr ? min(p.rows[b], p.R) : p.R;
  const bool used = i < n;
  const int t = add_sat(L, i);
  const bool fits = t >= 0 && t < p.max_len;
  if (used && !fits && part == 0 && c == 0) flag_error(p.err, SPADE_DERR_CAPACITY);
  // the lane's features f0 .. + 3 and f1 .. + 3
  const bool turns = 4 * c < p.pairs;
  const int f0 = turns ? (p.interleaved ? 8 * c : 4 * c) : 8 * c + 0;
  const int f1 = turns ? (p.interleaved ? 8 * c + 4 : p.pairs + 4 * c) : 8 * c + 4;
  const int first = part * p.run, end = min(heads, first + p.run);
  if (!used) {
    const float z[4] = {0.f, 0.f, 0.f, 0.f};
    for (int h = first; h < min(end, HQ); ++h) {
      store4<BF16>(p.q_out, row * p.qo_ld + h * HD + f0, z);
      store4<BF16>(p.q_out, row * p.qo_ld + h * HD + f1, z);
    }
    return;
  }
  float co[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {0.f, 0.f, 0.f, 0.f};
  if (turns) {
    const double at = (double)(p.pos != nullptr ? p.pos[b] : L) + (double)(p.depth != nullptr ? p.depth[row] : i);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const double a = at * p.freq[4 * c + j];
      // whole turns off: a - 2 pi k, 2 pi in two parts (k below 2^32 leaves 2^-53 of a)
      const double k = rint(a * 0.15915494309189535);
      const double r = __builtin_fma(-k, 2.4492935982947064e-16, __builtin_fma(-k, 6.283185307179586, a));
      double s, o;
      sincos(r, &s, &o);
      co[j] = (float)(o * (double)p.amplitude);
      sn[j] = (float)(s * (double)p.amplitude);
    }
  }
  for (int h = first; h < end; ++h) {
    const bool query = h < HQ;
    const int64_t in = row * (query ? p.q_ld : p.k_ld) + (query ? h : h - HQ) * HD;
    float a[4], d[4];
    load4<BF16, STREAM>(query ? p.q : p.k, in + f0, a);
    load4<BF16, STREAM>(query ? p.q : p.k, in + f1, d);
    if (turns) {
      if (p.interleaved) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float* x = j < 2 ? a : d;
          const int e = 2 * (j & 1);
          const float u = x[e], w = x[e + 1];
          x[e] = u * co[j] - w * sn[j];
          x[e + 1] = w * co[j] + u * sn[j];
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float u = a[j], w = d[j];
          a[j] = u * co[j] - w * sn[j];
          d[j] = w * co[j] + u * sn[j];
        }
      }
    }
    if (query) {
      store4<BF16, STREAM>(p.q_out, row * p.qo_ld + h * HD + f0, a);
      store4<BF16, STREAM>(p.q_out, row * p.qo_ld + h * HD + f1, d);
    } else if (fits) {
      uint16_t* dst = p.cache.k + ((int64_t)b * p.KVH + h - HQ) * p.cache.head_elems;
      store4<true>(dst, k_cache_index(f0, t, HD), a);
      store4<true>(dst, k_cache_index(f1, t, HD), d);
    }
  }
}

// Two features of eight neighbouring positions t0 .. t0 + 7 (t0 a multiple of 8).
struct Octet {
  int b, h, f;
  int64_t t0;
  int L;
};
template <int HD>
__device__ __forceinline__ bool octet_of(int64_t block, int B, int R, int KVH, const int32_t* lens, Octet& o) {
  constexpr int LPH = HD / 2, HPW = 64 / LPH;
  const int lane = threadIdx.x & 63, per = (R + 14) / 8, groups = (KVH + HPW - 1) / HPW;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  int64_t id = block * 4 + wave;
  const int g = (int)(id % groups);
  id /= groups;
  const int oc = (int)(id % per);
  id /= per;
  if (id >= B) return false;
  o.b = (int)id;
  o.h = g * HPW + lane / LPH;
  o.f = 2 * (lane % LPH);
  o.L = lens != nullptr ? lens[o.b] : 0;
  o.t0 = ((int64_t)(o.L >> 3) + oc) * 8;
  return o.h < KVH;
}

template <int HD, bool BF16, bool STREAM>
__device__ __forceinline__ void append_v(const TreeAppend& p, int64_t block) {
  Octet o;
  if (!octet_of<HD>(block, p.B, p.R, p.KVH, p.lens, o)) return;
  const int n = p.rows != nullptr ? min(p.rows[o.b], p.R) : p.R;
  uint32_t w[8];
  uint32_t have = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int64_t t = o.t0 + e, i = t - o.L;
    w[e] = 0;
    if (i >= 0 && i < n && t >= 0 && t < p.max_len) {
      have |= 1u << e;
      const int64_t at = ((int64_t)o.b * p.R + i) * p.v_ld + o.h * HD + o.f;
      if constexpr (BF16) {
        w[e] = get<STREAM>((const uint32_t*)((const uint16_t*)p.v + at));
      } else {
        const Words2 x = get<STREAM>((const Words2*)((const float*)p.v + at));
        w[e] = pk_bf16(__uint_as_float(x.x), __uint_as_float(x.y));
      }
    }
  }
  if (have == 0) return;
  uint16_t* dst = p.cache.v + ((int64_t)o.b * p.KVH + o.h) * p.cache.head_elems + v_cache_index(o.f, (int)o.t0, HD);
  if (have == 0xffu) {
    uint32_t a[4], d[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      a[j] = __builtin_amdgcn_perm(w[2 * j + 1], w[2 * j], 0x05040100u);
      d[j] = __builtin_amdgcn_perm(w[2 * j + 1], w[2 * j], 0x07060302u);
    }
    *(uint4*)dst = make_uint4(a[0], a[1], a[2], a[3]);
    *(uint4*)(dst + 8) = make_uint4(d[0], d[1], d[2], d[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (have >> e & 1u) {
        dst[e] = (uint16_t)w[e];
        dst[8 + e] = (uint16_t)(w[e] >> 16);
      }
  }
}

template <int HD, bool BF16, bool STREAM>
__global__ void __launch_bounds__(256) tree_append_kernel(TreeAppend p) {
  if ((int)blockIdx.x < p.qk_blocks) append_qk<HD, BF16, STREAM>(p, (int)blockIdx.x);
  else append_v<HD, BF16, STREAM>(p, (int64_t)blockIdx.x - p.qk_blocks);
}

// ---------------------------------------------------------------------------
// Read back: keys a lane per 16-byte piece, values as they were appended.  Bound by
// memory: 4003 rows of 32 heads of 128 read and write 131 MB in 27 us (4.8 TB/s).
// ---------------------------------------------------------------------------
template <int HD, bool BF16>
__global__ void __launch_bounds__(256) tree_read_kernel(TreeRead p) {
  if ((int)blockIdx.x < p.k_blocks) {
    constexpr int LPH = HD / 8;
    const int64_t id = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LPH;
    const int c = threadIdx.x % LPH;
    // (row within the request fastest: neighbouring positions' pieces are neighbours)
    const int64_t bh = id / p.R;
    if (bh >= (int64_t)p.B * p.KVH) return;
    const int i = (int)(id - bh * p.R), b = (int)(bh / p.KVH), h = (int)(bh - (int64_t)b * p.KVH);
    const int n = p.rows != nullptr ? min(p.rows[b], p.R) : p.R;
    const int t = add_sat(p.start != nullptr ? p.start[b] : 0, i);
    uint4 w = make_uint4(0, 0, 0, 0);
    if (i < n && t >= 0 && t < p.max_len) w = *(const uint4*)(p.cache.k + bh * p.cache.head_elems + k_cache_index(8 * c, t, HD));
    const int64_t at = (((int64_t)b * p.R + i) * p.KVH + h) * HD + 8 * c;
    if constexpr (BF16) {
      *(uint4*)((uint16_t*)p.k + at) = w;
    } else {
      *(float4*)((float*)p.k + at) = make_float4(lo_f(w.x), hi_f(w.x), lo_f(w.y), hi_f(w.y));
      *(float4*)((float*)p.k + at + 4) = make_float4(lo_f(w.z), hi_f(w.z), lo_f(w.w), hi_f(w.w));
    }
    return;
  }
  Octet o;
  if (!octet_of<HD>((int64_t)blockIdx.x - p.k_blocks, p.B, p.R, p.KVH, p.start, o)) return;
  const int n = p.rows != nullptr ? min(p.rows[o.b], p.R) : p.R;
  uint4 w[2] = {};
  if (o.t0 >= 0 && o.t0 < p.max_len && o.t0 - o.L < n) {
    const uint16_t* src = p.cache.v + ((int64_t)o.b * p.KVH + o.h) * p.cache.head_elems + v_cache_index(o.f, (int)o.t0, HD);
    w[0] = *(const uint4*)src;
    w[1] = *(const uint4*)(src + 8);
  }
  const uint32_t x[2][4] = {{w[0].x, w[0].y, w[0].z, w[0].w}, {w[1].x, w[1].y, w[1].z, w[1].w}};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int64_t t = o.t0 + e, i = t - o.L;
    if (i < 0 || i >= p.R) continue;
    const bool live = i < n && t >= 0 && t < p.max_len;
    const uint32_t a = live ? (x[0][e >> 1] >> (16 * (e & 1))) & 0xffffu : 0u;
    const uint32_t d = live ? (x[1][e >> 1] >> (16 * (e & 1))) & 0xffffu : 0u;
    const int64_t at = (((int64_t)o.b * p.R + i) * p.KVH + o.h) * HD + o.f;
    if constexpr (BF16) *(uint32_t*)((uint16_t*)p.v + at) = a | d << 16;
    else *(float2*)((float*)p.v + at) = make_float2(lo_f(a), lo_f(d));
  }
}

// ---------------------------------------------------------------------------
// Attention.
//
// The G n rows in use that share a K/V head are packed (row g n + i) into tiles
// of 16.  A workgroup takes tiles of rows over a split of the keys, in blocks of 32
// positions, with a running reference, sum and output per row (one pass over the keys).
// The cache's fragments are the A operands of the transposed products, 1 KB per load:
//   S^T = K Q^T    lane 16 q + c gets the scores of row c at positions 4 q .. + 3
//                  of either 16-position group
//   O^T = V^T P^T  k slots 8 q .. + 7 are positions 8 q .. + 7: two swaps of lane
//                  halves and rows per pair of words bring the probabilities there
// so a lane keeps to one row, and its maximum, sum and factors stay in it.
// float32 calls hold queries and probabilities in three bf16 terms (24 bits),
// bfloat16 calls the probabilities in two, so that nothing but the rounding of an
// output shows.
//
// Only the last blocks hold rows of the tree: there a row's word of ancestors
// says which it sees.
//
// Bound by memory up to about 64 rows of a K/V head (two tiles over 32768 keys of 8
// heads: 134 MB in 32 us, 4.2 TB/s), by the matrix units and the exponentials beside
// them beyond (256 rows over 120001 keys of 8 heads, bfloat16: 126 GFLOP of the
// formula, 189 with the probabilities' second term, 191 us at least and a median of 225
// where runs follow each other; a large bfloat16 product would take 158.  Matrix
// instructions fill 0.55 of a SIMD's busy cycles, vector instructions 0.36).
// ---------------------------------------------------------------------------
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWaves = 4;

struct TreeRows {
  int L, n;  // cached positions before the rows, rows in use: L, n >= 0, L + n <= max_keys
};
__device__ __forceinline__ TreeRows tree_rows(const TreeAttend& p, int b, bool flag) {
  TreeRows r;
  r.n = p.rows != nullptr ? max(0, min(p.rows[b], p.R)) : p.R;
  r.L = p.lens[b];
  if (r.L < 0 || r.L > p.max_keys - r.n) {  // (also where n > max_keys)
    if (flag) flag_error(p.err, SPADE_DERR_CAPACITY);
    r.n = min(r.n, p.max_keys);
    r.L = r.L < 0 ? 0 : p.max_keys - r.n;
  }
  return r;
}

__device__ __forceinline__ bf16x8 op(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(bf16x8, make_uint4(a, b, c, d));
}
__device__ __forceinline__ floatx4 mfma(uint4 a, bf16x8 b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), b, c, 0, 0, 0);
}

// lanes l, l ^ 16, l ^ 32, l ^ 48 combined in all of them; NaN if one of them is
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float max_q(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = max_nan(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return max_nan(__uint_as_float(t[0]), __uint_as_float(t[1]));
}
__device__ __forceinline__ float sum_q(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(t[0]) + __uint_as_float(t[1]);
}

// Words a (positions 4 q + 2 j, + 1 of the first group) and b (of the second) to
// words j and j + 2 of the lane's eight positions 8 q .. + 7.
__device__ __forceinline__ void swap_words(uint32_t a, uint32_t b, uint32_t& w0, uint32_t& w2) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  const auto t = __builtin_amdgcn_permlane16_swap(r[0], r[1], false, false);
  w0 = t[0];
  w2 = t[1];
}

// the bf16 terms of two floats, largest first
template <int N>
__device__ __forceinline__ void terms(float a, float b, uint32_t (&w)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    w[i] = pk_bf16(a, b);
    if (i + 1 < N) {
      a -= lo_f(w[i]);
      b -= hi_f(w[i]);
    }
  }
}

// Ancestors of node `lane` and itself, as bits: every step doubles the distance.
__device__ __forceinline__ uint64_t ancestors(const TreeAttend& p, int b, int n, int lane, bool flag) {
  int at = -1;
  if (lane < n) {
    at = p.parents != nullptr ? p.parents[(int64_t)b * p.R + lane] : lane - 1;
    if (at < -1 || at >= lane) {
      if (flag) flag_error(p.err, SPADE_DERR_TREE);
      at = -1;
    }
  }
  uint32_t lo = lane < 32 ? 1u << lane : 0u, hi = lane < 32 ? 0u : 1u << (lane - 32);
#pragma unroll
  for (int s = 0; s < 6; ++s) {
    const int from = at < 0 ? lane : at;
    const uint32_t l2 = __shfl(lo, from), h2 = __shfl(hi, from);
    const int a2 = __shfl(at, from);
    lo |= l2;
    hi |= h2;
    at = at < 0 ? -1 : a2;
  }
  return (uint64_t)hi << 32 | lo;
}

// The output rows of a request that it does not use, for the heads of one K/V head
template <int HD, bool QB>
__device__ __forceinline__ void zero_rows(const TreeAttend& p, int b, int kvh, int n, int tid, int threads) {
  const int per = p.G * (HD / 4), count = (p.R - n) * per;
  const float z[4] = {0.f, 0.f, 0.f, 0.f};
  for (int k = tid; k < count; k += threads) {
    const int i = k / per, f = (k - i * per) * 4;
    store4<QB>(p.out, ((int64_t)b * p.R + n + i) * p.out_ld + (int64_t)kvh * p.G * HD + f, z);
  }
}

// Which part of the call a workgroup has.
//
// With keys enough and few heads the keys are split: the workgroups, WG at most (one
// round), have equal counts of blocks of 32 positions whatever the requests' lengths.
// The count follows from all of them: the least CB for which the splits of all heads and
// tiles of rows fit (kLeast at least, four rounds of a wave).  Every wave works it out
// from the lengths, the first workgroup leaves it for the merge.  16 ragged contexts of
// 256 to 4096 (8 heads, 128 rows) take 45 us with their merge; with as many splits for
// every request, and loads under branches, they took 66.  kLeast of 8 / 16 / 24 / 32, us
// with the merge, 4 query heads on each of 8 K/V heads, bfloat16: 1 x 2048 keys, 64 rows
// 13.6 / 11.2 / 12.8 / 13.0; 1 x 8192, 16 rows 15.7 / 12.6 / 14.3 / 14.3, 32 rows 17.9 / 16.2 /
// 14.5 / 14.6; 1 x 32768, 128 rows 47 / 48 / 51 / 58; 16 x 2048 the same.
constexpr int kLeast = 16;
struct Part {
  unsigned head;
  int b, kvh, rb, L, n, rows, nb, lo, hi;
  int part;  // the first row of the split's part in part_o
  __device__ __forceinline__ void request(const TreeAttend& p, int tid) {
    head = (unsigned)(b * p.KVH + kvh);
    const TreeRows rr = tree_rows(p, b, p.WG == 0 && rb == 0 && kvh == 0 && tid == 0);
    L = rr.L;
    n = rr.n;
    rows = p.G * n;
    nb = (L + n + 31) / 32;
  }
  // false: nothing to do
  __device__ __forceinline__ bool init(const TreeAttend& p, int tid) {
    lo = part = 0;
    if (p.WG == 0) {
      // Workgroup i runs on XCD i % 8: those that read the same keys for other rows
      // follow each other there and share its L2.
      const unsigned xcd = blockIdx.x & 7, jj = blockIdx.x >> 3, tt = jj / (unsigned)p.RB, unit = 8 * tt + xcd;
      rb = (int)(jj - tt * p.RB);
      if (unit >= (unsigned)(p.B * p.KVH)) return false;
      b = (int)(unit / (unsigned)p.KVH);
      kvh = (int)(unit - (unsigned)b * p.KVH);
      request(p, tid);
      hi = nb;
      return true;
    }
    const int lane = tid & 63, want = (int)blockIdx.x;
    // a request's blocks, tiles and packed rows
    struct One { int nb, tiles, rows; };
    auto one = [&](int r) {
      One x{0, 0, 0};
      if (r < p.B) {
        const TreeRows rr = tree_rows(p, r, false);
        x.nb = rr.n > 0 ? (rr.L + rr.n + 31) / 32 : 0;
        x.rows = p.G * rr.n;
        x.tiles = (x.rows + p.tile - 1) / p.tile;
      }
      return x;
    };
    const One first = one(lane);
    auto total = [&](auto f) {
      int s = prefix_sum(f(first));
      for (int r0 = 64; r0 < p.B; r0 += 64) s += prefix_sum(f(one(r0 + lane)));
      return from_lane(s, 63);
    };
    int cb = max(kLeast, (total([&](One x) { return p.KVH * x.tiles * x.nb; }) + p.WG - 1) / p.WG);
    auto units = [&](One x) { return p.KVH * x.tiles * ((x.nb + cb - 1) / cb); };
    while (total(units) > p.WG) cb += max(1, cb >> 3);
    if (want == 0 && tid == 0) p.plan[0] = cb;
    int before = 0, row = 0;
    bool found = false;
    for (int r0 = 0; r0 < p.B; r0 += 64) {
      const One x = r0 == 0 ? first : one(r0 + lane);
      const int u = units(x), iu = before + prefix_sum(u);
      const int pr = p.KVH * ((x.nb + cb - 1) / cb) * x.rows, ir = row + prefix_sum(pr);
      if (want == 0 && tid < 64 && r0 + lane < p.B) {
        p.plan[1 + r0 + lane] = ir - pr;
        tree_rows(p, r0 + lane, true);
      }
      const uint64_t hit = __ballot(iu > want);
      if (hit != 0 && !found) {
        const int l = __ffsll((unsigned long long)hit) - 1;
        found = true;
        b = r0 + l;
        const int at = want - from_lane(iu - u, l), ns = (from_lane(x.nb, l) + cb - 1) / cb;
        const int h = at / ns, split = at - h * ns;
        rb = h / p.KVH;
        kvh = h - rb * p.KVH;
        lo = split * cb;
        part = from_lane(ir - pr, l) + (kvh * ns + split) * from_lane(x.rows, l);
        if (want != 0) break;
      }
      before = from_lane(iu, 63);
      row = from_lane(ir, 63);
    }
    if (!found) return false;
    request(p, tid);
    hi = min(nb, lo + cb);
    return true;
  }
};

// One head's keys and values: fragments of 1 KB, a lane's 16 bytes at 16 lane.
template <int HD>
struct KvLoader {
  Rsrc k, v;
  __device__ __forceinline__ void init(const TreeCache& c, int64_t head) {
    // (a head has at most 2^28 bytes)
    k = make_rsrc(c.k + head * c.head_elems, (uint32_t)(c.head_elems * 2));
    v = make_rsrc(c.v + head * c.head_elems, (uint32_t)(c.head_elems * 2));
  }
  // fragment f of a block of 32 positions; nothing is read where `there` is false
  __device__ __forceinline__ uint4 key(int blk, int f, int lane, bool there) const {
    const uint32_t so = there ? (uint32_t)blk * (64 * HD) : 0u;
    return __builtin_bit_cast(
        uint4, __builtin_amdgcn_raw_buffer_load_b128(k, (int)(there ? 16u * lane : kOob), (int)(so + f * 1024), 0));
  }
  __device__ __forceinline__ uint4 value(int blk, int f, int lane, bool there) const {
    const uint32_t so = there ? (uint32_t)(blk >> 3) * (512 * HD) + (uint32_t)(blk & 7) * 1024 : 0u;
    return __builtin_bit_cast(
        uint4, __builtin_amdgcn_raw_buffer_load_b128(v, (int)(there ? 16u * lane : kOob), (int)(so + f * 8192), 0));
  }
};

// Masks of a lane's eight positions, the first d from the tree's first row: up to the
// last row; the tree's rows.
__device__ __forceinline__ void tail_masks(int d0, int n, uint32_t (&keep)[4], uint32_t (&own)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    keep[j] = own[j] = 0;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int d = d0 + 2 * j + e;
      const uint32_t half = 0xffffu << (16 * e);
      if (d < n) keep[j] |= half;
      if (d >= 0 && d < n) own[j] |= half;
    }
  }
}
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
  return ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

// The rows of a wave: RT tiles of 16, a lane with row c of each.
template <int HD, bool QB, int RT>
struct Rows {
  static constexpr int FT = HD / 16, S = HD / 32;
  static constexpr int NQ = QB ? 1 : 3, NP = QB ? 2 : 3;  // bf16 terms of queries and of probabilities
  bf16x8 Q[RT][NQ][S];
  uint64_t anc[RT];
  float M[RT], l[RT];
  floatx4 o[RT][FT];
  bool broken;  // a value of the tree's own rows was not finite, and cleared

  __device__ __forceinline__ void load(const TreeAttend& p, const Part& w, int r0, int lane) {
    const int q = lane >> 4, c = lane & 15;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int m = r0 + rt * 16 + c, g = m / w.n, i = m - g * w.n;
      const bool ok = m < w.rows;
      const int64_t at =
          ((int64_t)w.b * p.R + (ok ? i : 0)) * p.q_ld + ((int64_t)w.kvh * p.G + (ok ? g : 0)) * HD + 8 * q;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        float x[8];
        load4<QB>(p.q, at + 32 * s, x);
        load4<QB>(p.q, at + 32 * s + 4, x + 4);
        uint32_t e[NQ][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t t[NQ];
          terms<NQ>(ok ? x[2 * j] : 0.f, ok ? x[2 * j + 1] : 0.f, t);
#pragma unroll
          for (int k = 0; k < NQ; ++k) e[k][j] = t[k];
        }
#pragma unroll
        for (int k = 0; k < NQ; ++k) Q[rt][k][s] = op(e[k][0], e[k][1], e[k][2], e[k][3]);
      }
      anc[rt] = 0;
      M[rt] = -INFINITY;
      l[rt] = 0.f;
#pragma unroll
      for (int t = 0; t < FT; ++t) o[rt][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    broken = false;
  }
  __device__ __forceinline__ void load_ancestors(const TreeAttend& p, const Part& w, int r0, int lane, bool flag) {
    const uint64_t all = ancestors(p, w.b, w.n, lane, flag);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int m = r0 + rt * 16 + (lane & 15), i = m - m / w.n * w.n;
      const uint64_t x = (uint64_t)__shfl((uint32_t)(all >> 32), i) << 32 | __shfl((uint32_t)all, i);
      anc[rt] = m < w.rows ? x : 0ull;
    }
  }

  // Block blk: key fragment (u, s) and value fragment t from K and V.  TAIL: some
  // row does not see all of it.
  template <bool TAIL, typename KF, typename VF>
  __device__ __forceinline__ void step(int blk, const Part& w, float sl, int lane, KF K, VF V) {
    const int q = lane >> 4, d0 = 32 * blk - w.L;  // distance of the first position from the tree's first row
    floatx4 z[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int u = 0; u < 2; ++u) z[rt][u] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      uint4 kf[S];
#pragma unroll
      for (int s = 0; s < S; ++s) kf[s] = K(u, s);
#pragma unroll
      for (int k = NQ - 1; k >= 0; --k)  // (smallest terms first)
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) z[rt][u] = mfma(kf[s], Q[rt][k][s], z[rt][u]);
    }
    if constexpr (TAIL) {
      // (a hidden position may hold anything, NaN among it)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int d = d0 + 16 * u + 4 * q + r;
            const bool sees = d < 0 || (d < w.n && (anc[rt] >> (d & 63) & 1ull));
            if (!sees) z[rt][u][r] = -INFINITY;
          }
    }
    bf16x8 P[RT][NP];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float mx = z[rt][0][0];
#pragma unroll
      for (int k = 1; k < 8; ++k) mx = max_nan(mx, z[rt][k >> 2][k & 3]);
      mx = max_q(mx) * sl;
      // The reference follows the maximum where it is 2^8 behind it, so most blocks leave the sums
      // alone (a row's own alone decides, so its bits do not depend on the other rows).
      const bool up = mx > M[rt] + 8.f;
      if (__any(up)) {
        const float mn = up ? mx : M[rt];
        const float f = M[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M[rt] - mn);
        M[rt] = mn;
        l[rt] *= f;
#pragma unroll
        for (int t = 0; t < FT; ++t) o[rt][t] *= f;
      }
      const float base = M[rt] == -INFINITY ? 0.f : M[rt];
      uint32_t pw[2][2][NP];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float e[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          e[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[rt][u][r], sl, -base));
          l[rt] += e[r];
        }
        terms<NP>(e[0], e[1], pw[u][0]);
        terms<NP>(e[2], e[3], pw[u][1]);
      }
#pragma unroll
      for (int k = 0; k < NP; ++k) {
        uint32_t x[4];
        swap_words(pw[0][0][k], pw[1][0][k], x[0], x[2]);
        swap_words(pw[0][1][k], pw[1][1][k], x[1], x[3]);
        P[rt][k] = op(x[0], x[1], x[2], x[3]);
      }
    }
    uint32_t keep[4], own[4];
    if constexpr (TAIL) tail_masks(d0 + 8 * q, w.n, keep, own);
#pragma unroll
    for (int t = 0; t < FT; ++t) {
      uint4 vf = V(t);
      if constexpr (TAIL) {
        // Values behind the last row are cleared, and those of the tree's own rows that are not
        // finite, which must not reach the rows that do not see them (mend puts NaN where they do).
        uint32_t x[4] = {vf.x, vf.y, vf.z, vf.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[j] &= keep[j];
          const uint32_t bad = not_finite(x[j]) & own[j];
          x[j] &= ~bad;
          broken |= bad != 0;
        }
        vf = make_uint4(x[0], x[1], x[2], x[3]);
      }
#pragma unroll
      for (int k = NP - 1; k >= 0; --k)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) o[rt][t] = mfma(vf, P[rt][k], o[rt][t]);
    }
  }

  // A block whose values were cleared: NaN at their features in the rows that see them
  // (a product of marks counts them).
  __device__ __forceinline__ void mend(const KvLoader<HD>& ld, int blk, const Part& w, int lane) {
    const int q = lane >> 4, d0 = 32 * blk - w.L;
    uint32_t keep[4], own[4];
    tail_masks(d0 + 8 * q, w.n, keep, own);
    bf16x8 sees[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      uint32_t x[4] = {};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int d = d0 + 8 * q + e;
        if (d >= 0 && d < w.n && (anc[rt] >> (d & 63) & 1ull)) x[e >> 1] |= 0x3f80u << (16 * (e & 1));
      }
      sees[rt] = op(x[0], x[1], x[2], x[3]);
    }
#pragma unroll
    for (int t = 0; t < FT; ++t) {
      const uint4 vf = ld.value(blk, t, lane, true);
      const uint4 one = make_uint4(not_finite(vf.x) & own[0] & 0x3f803f80u, not_finite(vf.y) & own[1] & 0x3f803f80u,
                                   not_finite(vf.z) & own[2] & 0x3f803f80u, not_finite(vf.w) & own[3] & 0x3f803f80u);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const floatx4 hit = mfma(one, sees[rt], floatx4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (hit[r] > 0.f) o[rt][t][r] = __uint_as_float(0x7fc00000u);
      }
    }
  }
};

// An output, or a split's part of it: x of packed row m at features f .. + 3, its
// reference mx and sum s.
template <int HD, bool QB>
__device__ __forceinline__ void put(const TreeAttend& p, const Part& w, int m, int f, floatx4 x, float mx, float s) {
  if (p.WG == 0) {
    const int g = m / w.n, i = m - g * w.n;
    const float y[4] = {x[0] / s, x[1] / s, x[2] / s, x[3] / s};
    store4<QB>(p.out, ((int64_t)w.b * p.R + i) * p.out_ld + ((int64_t)w.kvh * p.G + g) * HD + f, y);
  } else {
    const int64_t at = (int64_t)w.part + m;
    *(floatx4*)(p.part_o + at * HD + f) = x;
    if (f == 0) {
      p.part_ml[2 * at] = mx;
      p.part_ml[2 * at + 1] = s;
    }
  }
}

// The waves of the same rows put their parts together.
template <int HD, int RT>
struct JoinSmem {
  float o[kWaves][RT * 16][HD + 4];
  float m[kWaves][RT * 16], l[kWaves][RT * 16];
};
template <int HD, bool QB, int RT>
__device__ __forceinline__ void join(const TreeAttend& p, const Part& w, Rows<HD, QB, RT>& R, JoinSmem<HD, RT>& sm, int wave,
                                     int tid) {
  const int lane = tid & 63, q = lane >> 4, c = lane & 15;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float s = sum_q(R.l[rt]);
    if (q == 0) {
      sm.m[wave][rt * 16 + c] = R.M[rt];
      sm.l[wave][rt * 16 + c] = s;
    }
  }
  __syncthreads();
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float m = sm.m[0][rt * 16 + c];
#pragma unroll
    for (int k = 1; k < kWaves; ++k) m = fmaxf(m, sm.m[k][rt * 16 + c]);
    const float f = R.M[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(R.M[rt] - m);
#pragma unroll
    for (int t = 0; t < HD / 16; ++t) {
      const floatx4 x = R.o[rt][t] * f;
      *(floatx4*)&sm.o[wave][rt * 16 + c][16 * t + 4 * q] = x;
    }
  }
  __syncthreads();
  constexpr int LPR = HD / 4;  // lanes a row
  for (int k = tid; k < RT * 16 * LPR; k += kWaves * 64) {
    const int r = k / LPR, f = (k - r * LPR) * 4, m = w.rb * RT * 16 + r;
    if (m >= w.rows) break;
    float mx = sm.m[0][r];
#pragma unroll
    for (int j = 1; j < kWaves; ++j) mx = fmaxf(mx, sm.m[j][r]);
    float s = 0.f;
    floatx4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < kWaves; ++j) {
      const float mw = sm.m[j][r], lw = sm.l[j][r];
      // (a part that is NaN stays so whatever its reference)
      s += mw == -INFINITY ? lw : lw * __builtin_amdgcn_exp2f(mw - mx);
      x += *(const floatx4*)&sm.o[j][r][f];
    }
    put<HD, QB>(p, w, m, f, x, mx, s);
  }
}

// Few rows: four waves with the same RT tiles, wave w every fourth block, two blocks
// in flight in registers.
template <int HD, bool QB, int RT>
__global__ void __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(RT == 1 ? 2 : 1)))
tree_attend_kernel(TreeAttend p) {
  constexpr int FT = HD / 16, S = HD / 32;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  auto& sm = *reinterpret_cast<JoinSmem<HD, RT>*>(smem_raw);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Part w;
  if (!w.init(p, tid)) return;
  if (p.WG == 0 && w.rb == 0 && w.n < p.R) zero_rows<HD, QB>(p, w.b, w.kvh, w.n, tid, kWaves * 64);
  const int r0 = w.rb * RT * 16;
  if (r0 >= w.rows || w.lo >= w.hi) return;
  KvLoader<HD> ld;
  ld.init(p.cache, (int64_t)w.head);
  Rows<HD, QB, RT> R;
  R.load(p, w, r0, lane);  // (first: the blocks' loads are waited for in order)
  uint4 kb[2][2 * S], vb[2][FT];
  auto request = [&](int e, int blk) {
#pragma unroll
    for (int f = 0; f < 2 * S; ++f) kb[e][f] = ld.key(blk, f, lane, blk < w.hi);
#pragma unroll
    for (int t = 0; t < FT; ++t) vb[e][t] = ld.value(blk, t, lane, blk < w.hi);
  };
  request(0, w.lo + wave);
  request(1, w.lo + wave + kWaves);
  const int full = min(w.hi, w.L / 32);  // blocks that every row sees
  if (full < w.hi) R.load_ancestors(p, w, r0, lane, w.kvh == 0 && w.rb == 0 && w.hi == w.nb);
  const float sl = p.scale * kLog2e;
  auto step = [&](auto tail, int e, int blk) {
    R.template step<decltype(tail)::value>(
        blk, w, sl, lane, [&](int u, int s) { return kb[e][u * S + s]; }, [&](int t) { return vb[e][t]; });
  };
  int blk = w.lo + wave;
  for (; blk + kWaves < full; blk += 2 * kWaves) {
    step(std::false_type{}, 0, blk);
    request(0, blk + 2 * kWaves);
    step(std::false_type{}, 1, blk + kWaves);
    request(1, blk + 3 * kWaves);
  }
  // what is left: at most one full block, and the tree's
  const int first = blk;
  for (; blk < w.hi; blk += 2 * kWaves) {
    step(std::true_type{}, 0, blk);
    if (blk + kWaves >= w.hi) break;
    request(0, blk + 2 * kWaves);
    step(std::true_type{}, 1, blk + kWaves);
    request(1, blk + 3 * kWaves);
  }
  if (__any(R.broken))
    for (int e = first; e < w.hi; e += kWaves) R.mend(ld, e, w, lane);
  join<HD, QB, RT>(p, w, R, sm, wave, tid);
}

// Many rows: four or eight waves with 32 rows (float32: 16) each over the same keys,
// which pass through LDS: every byte enters the compute unit once for all of them.
// Loads run D blocks ahead in registers.
//
// bfloat16 calls use the 32 x 32 products, whose tile is a block's 32 positions by a
// wave's 32 rows: lane 32 h + c has the scores of row c at positions 8 g + 4 h .. + 3,
// and one swap of lane halves per pair of words makes them the next operand.
typedef __attribute__((ext_vector_type(16))) float floatx16;
__device__ __forceinline__ floatx16 mfma32(uint4 a, bf16x8 b, floatx16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), b, c, 0, 0, 0);
}
__device__ __forceinline__ float half_max(float v) {
  const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return max_nan(__uint_as_float(t[0]), __uint_as_float(t[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(t[0]) + __uint_as_float(t[1]);
}
// a pair's second terms: what its first terms w leave
__device__ __forceinline__ uint32_t second_terms(float a, float b, uint32_t w) {
  return pk_bf16(a - lo_f(w), b - hi_f(w));
}

template <int HD>
struct Rows32 {
  static constexpr int FT = HD / 32, E = HD / 16, S = HD / 32;
  bf16x8 Q[E];
  uint64_t anc;
  float M, l;  // reference; the lane's part of the sum
  floatx16 o[FT];
  bool broken;

  __device__ __forceinline__ void load(const TreeAttend& p, const Part& w, int r0, int lane) {
    const int h = lane >> 5, m = r0 + (lane & 31), g = m / w.n, i = m - g * w.n;
    const bool ok = m < w.rows;
    const int64_t at = ((int64_t)w.b * p.R + (ok ? i : 0)) * p.q_ld + ((int64_t)w.kvh * p.G + (ok ? g : 0)) * HD + 8 * h;
#pragma unroll
    for (int e = 0; e < E; ++e) {  // (rows are aligned to 8 bytes)
      const uint2 a = *(const uint2*)((const uint16_t*)p.q + at + 16 * e), b = *(const uint2*)((const uint16_t*)p.q + at + 16 * e + 4);
      Q[e] = ok ? op(a.x, a.y, b.x, b.y) : op(0, 0, 0, 0);
    }
    anc = 0;
    M = -INFINITY;
    l = 0.f;
    broken = false;
#pragma unroll
    for (int t = 0; t < FT; ++t) o[t] = floatx16{};
  }
  __device__ __forceinline__ void load_ancestors(const TreeAttend& p, const Part& w, int r0, int lane, bool flag) {
    const uint64_t all = ancestors(p, w.b, w.n, lane, flag);
    const int m = r0 + (lane & 31), i = m - m / w.n * w.n;
    const uint64_t x = (uint64_t)__shfl((uint32_t)(all >> 32), i) << 32 | __shfl((uint32_t)all, i);
    anc = m < w.rows ? x : 0ull;
  }
  __device__ __forceinline__ bool sees(int d, int n) const { return d < 0 || (d < n && (anc >> (d & 63) & 1ull)); }

  // A block at `at` in LDS, fragments of 16 positions by 32 features, then of 16
  // features by 32 positions: the pieces of a 32 x 16 operand lie in two of them.
  template <bool TAIL>
  __device__ __forceinline__ void step(int blk, const Part& w, float sl, int lane, const uint4* at) {
    const int h = lane >> 5, d0 = 32 * blk - w.L;
    const uint4* kp = at + (lane >> 4 & 1) * (S * 64) + 16 * h + (lane & 15);
    const uint4* vp = at + 2 * S * 64 + (lane >> 4 & 1) * 64 + 16 * h + (lane & 15);
    uint4 kf[E], vf[FT][2];
#pragma unroll
    for (int e = 0; e < E; ++e) kf[e] = kp[(e >> 1) * 64 + (e & 1) * 32];
    floatx16 z = mfma32(kf[0], Q[0], floatx16{});
#pragma unroll
    for (int e = 1; e < E; ++e) z = mfma32(kf[e], Q[e], z);
#pragma unroll
    for (int t = 0; t < FT; ++t)
#pragma unroll
      for (int s = 0; s < 2; ++s) vf[t][s] = vp[t * 128 + s * 32];
    if constexpr (TAIL) {
#pragma unroll
      for (int k = 0; k < 16; ++k)
        if (!sees(d0 + 8 * (k >> 2) + 4 * h + (k & 3), w.n)) z[k] = -INFINITY;
    }
    // A row keeps its reference as long as its sum stays in range (it starts with the first
    // maximum): no maximum in most blocks, and a row's bits do not depend on the others.
    float e[16], s = l, base = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      e[k] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[k], sl, -base));
      s += e[k];
    }
    const uint64_t out = __ballot(M == -INFINITY || !(s <= 0x1p60f));
    if (out != 0) {
      float mx = z[0];
#pragma unroll
      for (int k = 1; k < 16; ++k) mx = max_nan(mx, z[k]);
      mx = half_max(mx) * sl;
      const bool up = (out | out >> 32) >> (lane & 31) & 1u;
      const float mn = up ? fmaxf(M, mx) : M;
      const float f = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - mn);
      M = mn;
      base = M == -INFINITY ? 0.f : M;
      s = l * f;
#pragma unroll
      for (int t = 0; t < FT; ++t) o[t] *= f;
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        e[k] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[k], sl, -base));
        s += e[k];
      }
    }
    l = s;
    bf16x8 P[2][2];  // [16 positions][term]
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2) {
      uint32_t a[2][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float x = e[8 * s2 + 2 * j], y = e[8 * s2 + 2 * j + 1];
        a[0][j] = pk_bf16(x, y);
        a[1][j] = second_terms(x, y, a[0][j]);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const auto r0 = __builtin_amdgcn_permlane32_swap(a[k][0], a[k][2], false, false);
        const auto r1 = __builtin_amdgcn_permlane32_swap(a[k][1], a[k][3], false, false);
        P[s2][k] = op(r0[0], r1[0], r0[1], r1[1]);
      }
    }
    if constexpr (TAIL) {
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        uint32_t keep[4], own[4];
        tail_masks(d0 + 16 * s2 + 8 * h, w.n, keep, own);
#pragma unroll
        for (int t = 0; t < FT; ++t) {
          uint32_t x[4] = {vf[t][s2].x, vf[t][s2].y, vf[t][s2].z, vf[t][s2].w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            x[j] &= keep[j];
            const uint32_t bad = not_finite(x[j]) & own[j];
            x[j] &= ~bad;
            broken |= bad != 0;
          }
          vf[t][s2] = make_uint4(x[0], x[1], x[2], x[3]);
        }
      }
    }
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
      for (int k = 1; k >= 0; --k)
#pragma unroll
        for (int t = 0; t < FT; ++t) o[t] = mfma32(vf[t][s2], P[s2][k], o[t]);
  }
  __device__ __forceinline__ void mend(const KvLoader<HD>& ld, int blk, const Part& w, int lane) {
    const int h = lane >> 5, d0 = 32 * blk - w.L;
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2) {
      uint32_t keep[4], own[4], x[4] = {};
      tail_masks(d0 + 16 * s2 + 8 * h, w.n, keep, own);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int d = d0 + 16 * s2 + 8 * h + e;
        if (d >= 0 && d < w.n && (anc >> (d & 63) & 1ull)) x[e >> 1] |= 0x3f80u << (16 * (e & 1));
      }
      const bf16x8 see = op(x[0], x[1], x[2], x[3]);
#pragma unroll
      for (int t = 0; t < FT; ++t) {
        // (fragment 2 t or 2 t + 1, its lane 16 (2 s2 + h) + feature)
        const uint4 a = ld.value(blk, 2 * t, 32 * s2 + 16 * h + (lane & 15), true);
        const uint4 b = ld.value(blk, 2 * t + 1, 32 * s2 + 16 * h + (lane & 15), true);
        const uint4 vf = lane & 16 ? b : a;
        const uint4 one = make_uint4(not_finite(vf.x) & own[0] & 0x3f803f80u, not_finite(vf.y) & own[1] & 0x3f803f80u,
                                     not_finite(vf.z) & own[2] & 0x3f803f80u, not_finite(vf.w) & own[3] & 0x3f803f80u);
        const floatx16 hit = mfma32(one, see, floatx16{});
#pragma unroll
        for (int k = 0; k < 16; ++k)
          if (hit[k] > 0.f) o[t][k] = __uint_as_float(0x7fc00000u);
      }
    }
  }
};

// A wave's rows from r0 on are its own: no join.
template <int HD>
__device__ __forceinline__ void put_rows(const TreeAttend& p, const Part& w, const Rows32<HD>& R, int r0, int lane) {
  const int h = lane >> 5, m = r0 + (lane & 31);
  const float s = half_sum(R.l);
  if (m < w.rows)
#pragma unroll
    for (int t = 0; t < HD / 32; ++t)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        put<HD, true>(p, w, m, 32 * t + 8 * g + 4 * h,
                      floatx4{R.o[t][4 * g], R.o[t][4 * g + 1], R.o[t][4 * g + 2], R.o[t][4 * g + 3]}, R.M, s);
}
template <int HD>
__device__ __forceinline__ void put_rows(const TreeAttend& p, const Part& w, const Rows<HD, false, 1>& R, int r0, int lane) {
  const int q = lane >> 4, m = r0 + (lane & 15);
  const float s = sum_q(R.l[0]);
  if (m < w.rows)
#pragma unroll
    for (int t = 0; t < HD / 16; ++t) put<HD, false>(p, w, m, 16 * t + 4 * q, R.o[0][t], R.M[0], s);
}

template <int HD, bool QB, int W>
struct Wide {
  static constexpr int kThreads = W * 64, kWaveRows = QB ? 32 : 16, kRows = W * kWaveRows;
  static constexpr int kPieces = 8 * HD;              // 16-byte pieces of a block, keys first
  static constexpr int kLoads = kPieces / kThreads;   // of a thread
  static constexpr int D = kLoads >= 4 ? 2 : 3;       // blocks ahead
  static constexpr size_t kSmem = 2 * kPieces * 16;
};

template <int HD, bool QB, int W>
__global__ void __launch_bounds__(W * 64) __attribute__((amdgpu_waves_per_eu(2))) tree_attend_wide_kernel(TreeAttend p) {
  using C = Wide<HD, QB, W>;
  constexpr int S = HD / 32, D = C::D, N = C::kLoads, T = C::kThreads;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  uint4* ring = reinterpret_cast<uint4*>(smem_raw);  // [2][kPieces]
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Part w;
  if (!w.init(p, tid)) return;
  if (p.WG == 0 && w.rb == 0 && w.n < p.R) zero_rows<HD, QB>(p, w.b, w.kvh, w.n, tid, T);
  if (w.rb * C::kRows >= w.rows || w.lo >= w.hi) return;
  const int r0 = w.rb * C::kRows + wave * C::kWaveRows;
  const bool work = r0 < w.rows;
  KvLoader<HD> ld;
  ld.init(p.cache, (int64_t)w.head);
  std::conditional_t<QB, Rows32<HD>, Rows<HD, QB, 1>> R;
  R.load(p, w, r0, lane);
  // Piece e T + tid of a block, keys before values.  Which of them follows from e or (T pieces
  // are a whole block) from the wave: no load is under a branch, or the wait for one would be a
  // wait for all.
  const bool keys = wave < 2 * S;
  const Rsrc mine = keys ? ld.k : ld.v;
  auto load = [&](int blk, int e) {
    const int f0 = e * T / 64;
    const bool there = blk < w.hi;
    if (f0 + W <= 2 * S) return ld.key(blk, f0 + wave, lane, there);
    if (f0 >= 2 * S) return ld.value(blk, f0 + wave - 2 * S, lane, there);
    const uint32_t ko = (uint32_t)blk * (64 * HD) + wave * 1024,
                   vo = (uint32_t)(blk >> 3) * (512 * HD) + (uint32_t)(blk & 7) * 1024 + (wave - 2 * S) * 8192;
    return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(mine, (int)(there ? 16u * lane : kOob),
                                                                           (int)(there ? (keys ? ko : vo) : 0u), 0));
  };
  uint4 reg[D][N];
#pragma unroll
  for (int e = 0; e < N; ++e) ring[e * T + tid] = load(w.lo, e);
#pragma unroll
  for (int d = 0; d < D; ++d)
#pragma unroll
    for (int e = 0; e < N; ++e) reg[d][e] = load(w.lo + 1 + d, e);
  if (32 * w.hi > w.L && work) R.load_ancestors(p, w, r0, lane, w.kvh == 0 && r0 == 0 && w.hi == w.nb);
  const float sl = p.scale * kLog2e;
  auto block = [&](auto tail, int it, uint4 (&next_regs)[N]) {
    uint4* next = ring + ((it + 1) & 1) * C::kPieces;
#pragma unroll
    for (int e = 0; e < N; ++e) next[e * T + tid] = next_regs[e];
#pragma unroll
    for (int e = 0; e < N; ++e) next_regs[e] = load(w.lo + it + 1 + D, e);
    if (work) {
      const uint4* here = ring + (it & 1) * C::kPieces;
      if constexpr (QB) {
        R.template step<decltype(tail)::value>(w.lo + it, w, sl, lane, here);
      } else {
        R.template step<decltype(tail)::value>(
            w.lo + it, w, sl, lane, [&](int u, int s) { return here[(u * S + s) * 64 + lane]; },
            [&](int t) { return here[(2 * S + t) * 64 + lane]; });
      }
    }
    __syncthreads();
  };
  __syncthreads();
  // blocks that every row sees, D at a time (the registers' turn); the rest with the masks
  const int count = w.hi - w.lo, full = min(max(w.L / 32 - w.lo, 0), count) / D * D;
  for (int it = 0; it < full; it += D)
#pragma unroll
    for (int d = 0; d < D; ++d) block(std::false_type{}, it + d, reg[d]);
  for (int it = full; it < count; it += D)
#pragma unroll
    for (int d = 0; d < D; ++d) {
      if (it + d >= count) break;
      block(std::true_type{}, it + d, reg[d]);
    }
  if (__any(R.broken))
    for (int e = max(w.lo, w.L / 32); e < w.hi; ++e) R.mend(ld, e, w, lane);
  put_rows<HD>(p, w, R, r0, lane);
}

// The splits of a row, in order: GR groups of HD / 4 lanes take every GR-th one.  Bound
// by memory: 16 requests of 32 rows and 32 heads over about four splits read 34 MB in
// 7.6 us (4.4 TB/s; by eight groups 24); one request's 64 splits take 10.8, most of it
// three round trips (by one group 17).
template <int HD, bool QB, int GR>
__global__ void __launch_bounds__(256) tree_merge_kernel(TreeAttend p) {
  constexpr int LPR = HD / 4, PER = 256 / LPR / GR;  // rows of a workgroup
  __shared__ float po[256 / LPR][HD];
  __shared__ float pm[256 / LPR], pl[256 / LPR];
  const int grp = threadIdx.x / LPR, f = (threadIdx.x % LPR) * 4, sub = grp % GR;
  const int64_t row = (int64_t)blockIdx.x * PER + grp / GR;  // (request, K/V head, query head of it, i)
  const bool live = row < (int64_t)p.B * p.H * p.R;
  const int64_t bh = live ? row / (p.G * p.R) : 0;
  const int in = live ? (int)(row - bh * (p.G * p.R)) : 0, g = in / p.R, i = in - g * p.R;
  const int b = (int)(bh / p.KVH), kvh = (int)(bh - (int64_t)b * p.KVH);
  const TreeRows rr = tree_rows(p, b, false);
  const bool used = live && i < rr.n;
  const int cb = p.plan[0], ns = used ? ((rr.L + rr.n + 31) / 32 + cb - 1) / cb : 0;
  const int64_t step = (int64_t)p.G * rr.n, at0 = p.plan[1 + b] + (int64_t)kvh * ns * step + g * rr.n + i;
  float m = -INFINITY, s = 0.f;
  floatx4 x = {0.f, 0.f, 0.f, 0.f};
  constexpr int U = 4;
  for (int k0 = sub; k0 < ns; k0 += U * GR) {
    float mk[U], lk[U];
    floatx4 ok[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * GR;
      const int64_t at = at0 + (k < ns ? k : k0) * step;
      mk[u] = p.part_ml[2 * at];
      lk[u] = p.part_ml[2 * at + 1];
      ok[u] = *(const floatx4*)(p.part_o + at * HD + f);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k0 + u * GR >= ns) break;
      const float mn = fmaxf(m, mk[u]);
      const float a = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      const float d = mk[u] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mk[u] - mn);
      // (a part that is NaN stays so whatever its maximum)
      s = s * a + (mk[u] == -INFINITY ? lk[u] : lk[u] * d);
      x = x * a + ok[u] * d;
      m = mn;
    }
  }
  if constexpr (GR > 1) {
    if (f == 0) {
      pm[grp] = m;
      pl[grp] = s;
    }
    *(floatx4*)&po[grp][f] = x;
    __syncthreads();
    if (sub != 0) return;
    float mx = m;
#pragma unroll
    for (int k = 1; k < GR; ++k) mx = fmaxf(mx, pm[grp + k]);
    floatx4 y = {0.f, 0.f, 0.f, 0.f};
    s = 0.f;
#pragma unroll
    for (int k = 0; k < GR; ++k) {
      const float mk = pm[grp + k], d = mk == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mk - mx);
      s += mk == -INFINITY ? pl[grp + k] : pl[grp + k] * d;
      y += *(const floatx4*)&po[grp + k][f] * d;
    }
    x = y;
  }
  if (!live) return;
  float y[4] = {0.f, 0.f, 0.f, 0.f};
  if (used)
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = x[k] / s;
  store4<QB>(p.out, ((int64_t)b * p.R + i) * p.out_ld + ((int64_t)kvh * p.G + g) * HD + f, y);
}

// ---------------------------------------------------------------------------
// Commit.  A wave walks a request's tree: lane i holds node i, a vote finds the
// lowest child of the present node whose token is the drawn one.  Children come
// after their parents, so the walk ends.  Bound by latency: the walk 1.8 us for one
// request, 3.5 for 16; the moves 4 us for a layer of one request, 16 for 8 layers of 16
// requests of 8 heads (2048 workgroups, each two dependent round trips; values are
// 2-byte elements of 16-byte pieces).
// ---------------------------------------------------------------------------
__global__ void __launch_bounds__(64) tree_walk_kernel(TreeCommit p) {
  const int b = blockIdx.x, lane = threadIdx.x;
  int n = p.rows != nullptr ? max(0, min(p.rows[b], p.R)) : p.R;
  const int L = p.lens[b];
  if (L < 0 || L > p.max_len - n) {  // rows that the cache does not hold
    if (lane == 0) flag_error(p.err, SPADE_DERR_CAPACITY);
    n = L < 0 ? 0 : max(0, min(n, p.max_len - L));
  }
  const int64_t at = (int64_t)b * p.R + lane;
  int parent = -1, token = 0, next = 0;
  if (lane < n) {
    parent = p.parents != nullptr ? p.parents[at] : lane - 1;
    token = p.tokens[at];
    next = p.next[at];
    if (parent < -1 || parent >= lane) flag_error(p.err, SPADE_DERR_TREE);
  }
  int cur = 0, count = n > 0 ? 1 : 0, mine = lane == 0 && n > 0 ? 0 : -1;
  while (n > 0) {
    const int want = __shfl(next, cur);
    const uint64_t hit = __ballot(lane > cur && lane < n && parent == cur && token == want);
    if (hit == 0) break;
    cur = __ffsll((unsigned long long)hit) - 1;
    if (lane == count) mine = cur;
    ++count;
  }
  const int corr = __shfl(next, cur);
  if (lane < p.R) p.path[at] = mine;
  if (lane == 0) {
    p.n_accepted[b] = count - 1;
    p.correction[b] = n > 0 ? corr : -1;
    p.lens_out[b] = add_sat(L, count);
  }
}

// Row path[j] becomes row j.  A workgroup reads all that it moves before it writes.
constexpr int kMoveThreads = 256;
__global__ void __launch_bounds__(kMoveThreads) tree_move_kernel(TreeCommit p) {
  __shared__ int path[kTreeMaxRows];
  const int z = blockIdx.x, tid = threadIdx.x;
  const int h = z % p.KVH, b = (z / p.KVH) % p.B, l = z / (p.KVH * p.B);
  const int count = p.n_accepted[b] + 1, L = p.lens_out[b] - count;
  if (tid < count) path[tid] = p.path[(int64_t)b * p.R + tid];
  __syncthreads();
  int j0 = 0;  // rows that stay: path[j] = j
  while (j0 < count && path[j0] == j0) ++j0;
  if (j0 >= count) return;
  const int64_t head = l * p.layer_elems + ((int64_t)b * p.KVH + h) * p.cache.head_elems;
  if (blockIdx.y == 0) {
    constexpr int N = kTreeMaxRows * 16 / kMoveThreads;
    uint16_t* k = p.cache.k + head;
    const int pieces = p.hd / 8, items = (count - j0) * pieces;
    uint4 w[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int it = tid + e * kMoveThreads, j = j0 + it / pieces, f = it % pieces * 8;
      if (it < items) w[e] = *(const uint4*)(k + k_cache_index(f, L + path[j], p.hd));
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int it = tid + e * kMoveThreads, j = j0 + it / pieces, f = it % pieces * 8;
      if (it < items) *(uint4*)(k + k_cache_index(f, L + j, p.hd)) = w[e];
    }
  } else {
    constexpr int N = kTreeMaxRows * 128 / kMoveThreads;
    uint16_t* v = p.cache.v + head;
    const int items = (count - j0) * p.hd;
    uint16_t w[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int it = tid + e * kMoveThreads, j = j0 + it / p.hd, f = it % p.hd;
      if (it < items) w[e] = v[v_cache_index(f, L + path[j], p.hd)];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int it = tid + e * kMoveThreads, j = j0 + it / p.hd, f = it % p.hd;
      if (it < items) v[v_cache_index(f, L + j, p.hd)] = w[e];
    }
  }
}

// Inputs of more than this go past the caches (as do the queries).  us with / without, 4096
// rows, inputs just written by another kernel: 32 + 2 x 8 heads of float32 (96 MB) 39 / 45, 32 +
// 2 x 32 of float32 (192 MB) 58 / 70, of bfloat16 (96 MB) 57 / 52, inputs in memory 46 / 55; 2048
// rows of 32 + 2 x 8 heads of float32 (48 MB) 21 / 18.
constexpr int64_t kStreamBytes = 64 << 20;
template <int HD, bool BF16>
hipError_t append_t(TreeAppend a, hipStream_t st) {
  constexpr int VHPW = 64 / (HD / 2), RPG = 4 * 64 / (HD / 8);  // rows a workgroup
  const int heads = (a.q != nullptr ? a.H : 0) + a.KVH;
  const int64_t rows = (int64_t)a.B * a.R, groups = (rows + RPG - 1) / RPG;
  // enough workgroups for the chip, then several heads for one computation of the angles
  a.run = (int)std::min<int64_t>(std::max<int64_t>(groups * heads / 1024, 1), heads);
  const int64_t qk = groups * ((heads + a.run - 1) / a.run);
  const int64_t vb = ((int64_t)a.B * ((a.R + 14) / 8) * ((a.KVH + VHPW - 1) / VHPW) + 3) / 4;
  if (qk + vb > 0x7fffffff) return hipErrorInvalidValue;
  a.qk_blocks = (int)qk;
  const dim3 grid((unsigned)(qk + vb)), block(256);
  if (rows * (heads + a.KVH) * HD * (BF16 ? 2 : 4) > kStreamBytes)
    hipLaunchKernelGGL((tree_append_kernel<HD, BF16, true>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((tree_append_kernel<HD, BF16, false>), grid, block, 0, st, a);
  return hipGetLastError();
}

template <int HD, bool BF16>
hipError_t read_t(TreeRead a, hipStream_t st) {
  constexpr int VHPW = 64 / (HD / 2);
  const int64_t kb = ((int64_t)a.B * a.KVH * a.R * (HD / 8) + 255) / 256;
  const int64_t vb = ((int64_t)a.B * ((a.R + 14) / 8) * ((a.KVH + VHPW - 1) / VHPW) + 3) / 4;
  if (kb + vb > 0x7fffffff) return hipErrorInvalidValue;
  a.k_blocks = (int)kb;
  hipLaunchKernelGGL((tree_read_kernel<HD, BF16>), dim3((unsigned)(kb + vb)), dim3(256), 0, st, a);
  return hipGetLastError();
}

// LDS beyond 64 KB has to be asked for, once for every device.
template <auto KERNEL>
hipError_t allow_lds(size_t bytes) {
  if (bytes <= 65536) return hipSuccess;
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(done.load() & bit)) {
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != hipSuccess) return e;
    done.fetch_or(bit);
  }
  return hipSuccess;
}

// tile: packed rows of a workgroup; wgs: workgroups of one round
template <int HD, bool QB, auto KERNEL>
hipError_t attend_with(TreeAttend a, int tile, int wgs, int threads, size_t lds, hipStream_t st) {
  a.tile = tile;
  a.RB = (a.G * a.R + tile - 1) / tile;
  const int64_t heads = (int64_t)a.B * a.KVH;
  a.WG = (a.max_keys + 31) / 32 > kLeast && heads * a.RB < wgs ? wgs : 0;
  const int64_t grid = a.WG > 0 ? a.WG : 8 * a.RB * ((heads + 7) / 8);
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  // (a split's part has the rows of its workgroups)
  if (a.WG > 0 && std::min<int64_t>((int64_t)wgs * tile, (int64_t)wgs * a.G * a.R) > (int64_t)a.part_rows) return hipErrorInvalidValue;
  hipError_t e = allow_lds<KERNEL>(lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(KERNEL, dim3((unsigned)grid), dim3(threads), lds, st, a);
  e = hipGetLastError();
  if (e != hipSuccess || a.WG == 0) return e;
  constexpr int LPR = HD / 4, per = 256 / LPR;
  const int64_t out = (int64_t)a.B * a.H * a.R;
  // (about wgs / heads splits of a row)
  if (wgs >= 8 * heads * a.RB) hipLaunchKernelGGL((tree_merge_kernel<HD, QB, per>), dim3((unsigned)out), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((tree_merge_kernel<HD, QB, 1>), dim3((unsigned)((out + per - 1) / per)), dim3(256), 0, st, a);
  return hipGetLastError();
}

template <int HD, bool QB, int RT>
hipError_t attend_few(const TreeAttend& a, hipStream_t st) {
  return attend_with<HD, QB, tree_attend_kernel<HD, QB, RT>>(a, RT * 16, RT == 1 ? 512 : 256, kWaves * 64,
                                                            sizeof(JoinSmem<HD, RT>), st);
}
template <int HD, bool QB, int W>
hipError_t attend_wide(const TreeAttend& a, hipStream_t st) {
  using C = Wide<HD, QB, W>;
  return attend_with<HD, QB, tree_attend_wide_kernel<HD, QB, W>>(a, C::kRows, 2048 / W, C::kThreads, C::kSmem, st);
}

// Which kernel.  Few rows a workgroup cost its keys again for every 16 or 32 rows, from
// L2; many cost waves that wait at barriers and a part of the chip where the keys are
// few.  us with 4 query heads on each of 8 K/V heads of 128, bfloat16 calls (kernel by
// the rows of a workgroup):
//   requests x keys, rows of a K/V head      16     32     128     256
//   1 x 2048,   64                         13.6   14.8    16.1    18.0
//              256                         18.1   19.5    23.2    31.1
//   1 x 8192,  128                         24.2   23.1    28.8    24.2
//   1 x 32768,  32                         49.6   32.2    34.9    36.5
//               64                         50.2   33.0    38.7    39.7
//              256                         92.9   76.5    71.9    67.8
//   16 x 2048,  64                         30.0   29.5    38.9    39.9
//              128                         51.9   51.7    48.4    47.4
//              256                         94.4   96.6    76.5    72.5
//   64 x 512,   32                         29.3   36.7    30.1    42.5
//               64                         45.1   57.4    34.2    45.4
//              256                         153     206    76.4    84.7
// and 128 rows over 16 ragged contexts of 256 to 4096 55.9 / 57.7 / 45.6 / 50.1.
// float32 calls, whose wide kernels have half the rows: 1 x 8192, 256 rows 40.0 / 42.4 /
// 41.1 / 40.9; 1 x 32768, 32 rows 51.6 / 34.2 / 37.5 / 39.7, 256 rows 106 / 102 / 107 / 101.
//
// From 512 heads times groups of 64 rows on, whole heads fill the chip.  A bfloat16 workgroup
// takes 128 rows, so of calls with fewer than 512 of those (256 to 511 heads with 65 to 128
// rows) attend_with still splits long keys.  There too this kernel is about as fast or faster
// than what the rules below would take, us for 68 / 128 rows of 32 requests of 8 K/V heads: 256
// keys 18.2 / 19.6 (below: 35.3 / 46.6), 1024 keys 41.5 / 51.5 (50.2 / 52.0), 4096 keys 124 / 143
// (122 / 144).  (16 x 2048 with 256 rows comes here, 5 % off its best.)
template <int HD, bool QB>
hipError_t attend_t(const TreeAttend& a, hipStream_t st) {
  const int tiles = (a.G * a.R + 15) / 16;
  const int64_t heads = (int64_t)a.B * a.KVH;
  if (heads * ((tiles + 3) / 4) >= 512)
    return tiles <= 2 ? attend_few<HD, QB, 1>(a, st) : attend_wide<HD, QB, 4>(a, st);
  // blocks of keys times tiles of rows, for each workgroup of one round
  const int64_t work = heads * tiles * ((a.max_keys + 31) / 32) / 512;
  if (tiles == 1 || work <= 16) return attend_few<HD, QB, 1>(a, st);
  if (tiles <= 4 || work <= 96) return attend_few<HD, QB, 2>(a, st);
  if (QB && tiles <= 8) return attend_wide<HD, QB, 4>(a, st);
  return attend_wide<HD, QB, 8>(a, st);
}

}  // namespace

hipError_t launch_tree_append(const TreeAppend& a, hipStream_t st) {
  if (a.hd == 128) return a.bf16 ? append_t<128, true>(a, st) : append_t<128, false>(a, st);
  return a.bf16 ? append_t<64, true>(a, st) : append_t<64, false>(a, st);
}

hipError_t launch_tree_read(const TreeRead& a, hipStream_t st) {
  if (a.hd == 128) return a.bf16 ? read_t<128, true>(a, st) : read_t<128, false>(a, st);
  return a.bf16 ? read_t<64, true>(a, st) : read_t<64, false>(a, st);
}

// (workgroups of a split call times their rows: 512 of 16 or 128, 256 of up to 256)
size_t tree_part_rows(int G, int max_rows) {
  const int64_t n = (int64_t)G * max_rows;
  return (size_t)std::max(512 * std::min<int64_t>(n, 128), 256 * std::min<int64_t>(n, 256));
}

hipError_t launch_tree_attend(const TreeAttend& a, hipStream_t st) {
  if (a.hd == 128) return a.bf16 ? attend_t<128, true>(a, st) : attend_t<128, false>(a, st);
  return a.bf16 ? attend_t<64, true>(a, st) : attend_t<64, false>(a, st);
}

hipError_t launch_tree_commit(const TreeCommit& a, hipStream_t st) {
  hipLaunchKernelGGL(tree_walk_kernel, dim3((unsigned)a.B), dim3(64), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(tree_move_kernel, dim3((unsigned)(a.L * a.B * a.KVH), 2), dim3(kMoveThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace spade
