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

#include "device_util.h"

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

template <bool BF16>
__device__ __forceinline__ void load4(const void* base, int64_t at, float* x) {
  if constexpr (BF16) {
    const uint2 w = *(const uint2*)((const uint16_t*)base + at);
    x[0] = lo_f(w.x);
    x[1] = hi_f(w.x);
    x[2] = lo_f(w.y);
    x[3] = hi_f(w.y);
  } else {
    const float4 w = *(const float4*)((const float*)base + at);
    x[0] = w.x;
    x[1] = w.y;
    x[2] = w.z;
    x[3] = w.w;
  }
}

template <bool BF16>
__device__ __forceinline__ void store4(void* base, int64_t at, const float* x) {
  if constexpr (BF16) *(uint2*)((uint16_t*)base + at) = make_uint2(pk_bf16(x[0], x[1]), pk_bf16(x[2], x[3]));
  else *(float4*)((float*)base + at) = make_float4(x[0], x[1], x[2], x[3]);
}

// ---------------------------------------------------------------------------
// Append.  hd / 8 lanes hold a head: pair group p < pairs / 4 the features of
// pairs 4 p .. + 3 (halves: 4 p .. + 3 and pairs + 4 p .. + 3; neighbours: 8 p ..
// + 7), the lanes behind the eight features each that are not rotated.  A wave
// takes a row and computes its lanes' four angles once, for all heads that it
// goes through.  The angle pos f is a product in double whose whole turns are
// taken off exactly, so far positions lose nothing but the product's rounding
// (2^-53 of the angle; a float32 angle is off by 0.004 at 100 thousand
// positions); sine and cosine are rounded once to float32.
//
// Values are stored by feature: a lane takes two features of eight neighbouring
// positions, whole 16-byte pieces where the rows cover them.
// ---------------------------------------------------------------------------
template <int HD, bool BF16>
__device__ __forceinline__ void append_qk(const TreeAppend& p, int block) {
  constexpr int LPH = HD / 8, HPW = 64 / LPH;  // lanes a head, heads at a time
  const int lane = threadIdx.x & 63, c = lane % LPH, slot = lane / LPH;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int HQ = p.q != nullptr ? p.H : 0, heads = HQ + p.KVH;
  const int groups = (heads + HPW - 1) / HPW, parts = (groups + p.run - 1) / p.run;
  const int64_t id = (int64_t)block * 4 + wave, row = id / parts;
  const int part = (int)(id - row * parts);
  if (row >= (int64_t)p.B * p.R) return;
  const int b = (int)(row / p.R), i = (int)(row - (int64_t)b * p.R);
  const int L = p.lens[b], n = p.rows != nullptr ? min(p.rows[b], p.R) : p.R;
  const bool used = i < n;
  const int t = add_sat(L, i);
  const bool fits = t >= 0 && t < p.max_len;
  if (used && !fits && part == 0 && lane == 0) flag_error(p.err, SPADE_DERR_CAPACITY);
  // the lane's features f0 .. + 3 and f1 .. + 3
  const bool turns = 4 * c < p.pairs;
  const int f0 = turns ? (p.interleaved ? 8 * c : 4 * c) : 8 * c + 0;
  const int f1 = turns ? (p.interleaved ? 8 * c + 4 : p.pairs + 4 * c) : 8 * c + 4;
  float co[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {0.f, 0.f, 0.f, 0.f};
  if (turns && used) {
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
  for (int g = part * p.run, end = min(groups, g + p.run); g < end; ++g) {
    const int h = g * HPW + slot;
    if (h >= heads) break;
    const bool query = h < HQ;
    const int hh = query ? h : h - HQ;
    if (!used) {
      if (query) {
        const float z[4] = {0.f, 0.f, 0.f, 0.f};
        store4<BF16>(p.q_out, row * p.qo_ld + hh * HD + f0, z);
        store4<BF16>(p.q_out, row * p.qo_ld + hh * HD + f1, z);
      }
      continue;
    }
    const int64_t in = row * (query ? p.q_ld : p.k_ld) + hh * HD;
    float a[4], d[4];
    load4<BF16>(query ? p.q : p.k, in + f0, a);
    load4<BF16>(query ? p.q : p.k, in + f1, d);
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
      store4<BF16>(p.q_out, row * p.qo_ld + hh * HD + f0, a);
      store4<BF16>(p.q_out, row * p.qo_ld + hh * HD + f1, d);
    } else if (fits) {
      uint16_t* dst = p.cache.k + ((int64_t)b * p.KVH + hh) * p.cache.head_elems;
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

template <int HD, bool BF16>
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
        w[e] = *(const uint32_t*)((const uint16_t*)p.v + at);
      } else {
        const float2 x = *(const float2*)((const float*)p.v + at);
        w[e] = pk_bf16(x.x, x.y);
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

template <int HD, bool BF16>
__global__ void __launch_bounds__(256) tree_append_kernel(TreeAppend p) {
  if ((int)blockIdx.x < p.qk_blocks) append_qk<HD, BF16>(p, (int)blockIdx.x);
  else append_v<HD, BF16>(p, (int64_t)blockIdx.x - p.qk_blocks);
}

// ---------------------------------------------------------------------------
// Read back: keys a lane per 16-byte piece, values as they were appended.
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
// of 16; a workgroup of four waves takes RT tiles over a split of the keys, wave
// w every fourth block of 32 positions, with a running maximum, sum and output
// of its own.  The cache's fragments are the A operands of the transposed
// products, straight from memory, 1 KB per load:
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

// One block of 32 positions: two 16-position groups of keys, HD / 16 tiles of values.
template <int HD>
struct KvBlock {
  uint4 k[2][HD / 32];
  uint4 v[HD / 16];
};

template <int HD>
struct KvLoader {
  Rsrc k, v;
  uint32_t lane16;
  __device__ __forceinline__ void init(const TreeCache& c, int64_t head, int lane) {
    // (a head has at most 2^28 bytes)
    k = make_rsrc(c.k + head * c.head_elems, (uint32_t)(c.head_elems * 2));
    v = make_rsrc(c.v + head * c.head_elems, (uint32_t)(c.head_elems * 2));
    lane16 = 16u * lane;
  }
  // blk at or past `end`: nothing is read
  __device__ __forceinline__ void keys(KvBlock<HD>& b, int blk, int end) const {
    const uint32_t so = blk < end ? (uint32_t)blk * (64 * HD) : 0u, vo = blk < end ? lane16 : kOob;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int s = 0; s < HD / 32; ++s)
        b.k[u][s] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(
                                                  k, (int)vo, (int)(so + (u * (HD / 32) + s) * 1024), 0));
  }
  __device__ __forceinline__ void values(KvBlock<HD>& b, int blk, int end) const {
    const uint32_t so = blk < end ? (uint32_t)(blk >> 3) * (512 * HD) + (uint32_t)(blk & 7) * 1024 : 0u, vo = blk < end ? lane16 : kOob;
#pragma unroll
    for (int t = 0; t < HD / 16; ++t)
      b.v[t] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(v, (int)vo, (int)(so + t * 8192), 0));
  }
};

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

template <int HD, int RT>
struct TreeSmem {
  float o[kWaves][RT * 16][HD + 4];
  float m[kWaves][RT * 16], l[kWaves][RT * 16];
};

template <int HD, bool QB, int RT>
__global__ void __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(RT == 1 ? 2 : 1)))
tree_attend_kernel(TreeAttend p) {
  constexpr int FT = HD / 16, S = HD / 32;
  constexpr int NQ = QB ? 1 : 3, NP = QB ? 2 : 3;  // bf16 terms of queries and of probabilities
  extern __shared__ __align__(16) uint8_t smem_raw[];
  TreeSmem<HD, RT>& sm = *reinterpret_cast<TreeSmem<HD, RT>*>(smem_raw);
  const int tid = threadIdx.x, lane = tid & 63, q = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Workgroup i runs on XCD i % 8: those that read the same keys for other rows
  // follow each other there and share its L2.
  const unsigned xcd = blockIdx.x & 7, jj = blockIdx.x >> 3;
  const unsigned tt = jj / (unsigned)p.RB, rb = jj - tt * p.RB, unit = 8 * tt + xcd;
  if (unit >= (unsigned)(p.B * p.KVH * p.NS)) return;
  const unsigned head = unit / (unsigned)p.NS, split = unit - head * p.NS;
  const int b = (int)(head / (unsigned)p.KVH), kvh = (int)(head - (unsigned)b * p.KVH);
  const bool first = split == 0 && rb == 0;
  const TreeRows rr = tree_rows(p, b, first && kvh == 0 && tid == 0);
  const int L = rr.L, n = rr.n, total = L + n, rows = p.G * n, r0 = (int)rb * RT * 16;
  if (p.NS == 1 && rb == 0 && n < p.R) zero_rows<HD, QB>(p, b, kvh, n, tid, kWaves * 64);
  const int nb = (total + 31) / 32, lo = (int)split * p.CB, hi = min(nb, lo + p.CB);
  if (r0 >= rows || lo >= hi) return;

  KvLoader<HD> ld;
  ld.init(p.cache, (int64_t)head, lane);
  KvBlock<HD> buf[2];
  bf16x8 Q[RT][NQ][S];
  int node[RT];
  // queries first: the blocks' loads are waited for in order
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int m = r0 + rt * 16 + c, g = m / n, i = m - g * n;
    const bool ok = m < rows;
    node[rt] = ok ? i : -1;
    const int64_t at = ((int64_t)b * p.R + (ok ? i : 0)) * p.q_ld + ((int64_t)kvh * p.G + (ok ? g : 0)) * HD + 8 * q;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      float x[8];
      load4<QB>(p.q, at + 32 * s, x);
      load4<QB>(p.q, at + 32 * s + 4, x + 4);
      uint32_t w[NQ][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t e[NQ];
        terms<NQ>(ok ? x[2 * j] : 0.f, ok ? x[2 * j + 1] : 0.f, e);
#pragma unroll
        for (int k = 0; k < NQ; ++k) w[k][j] = e[k];
      }
#pragma unroll
      for (int k = 0; k < NQ; ++k) Q[rt][k][s] = op(w[k][0], w[k][1], w[k][2], w[k][3]);
    }
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    ld.keys(buf[k], lo + wave + k * kWaves, hi);
    ld.values(buf[k], lo + wave + k * kWaves, hi);
  }
  uint64_t anc[RT] = {};
  if (32 * hi > L) {
    const uint64_t all = ancestors(p, b, n, lane, kvh == 0 && rb == 0 && hi == nb);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int from = max(node[rt], 0);
      const uint64_t w = (uint64_t)(uint32_t)__shfl((uint32_t)(all >> 32), from) << 32 | (uint32_t)__shfl((uint32_t)all, from);
      anc[rt] = node[rt] >= 0 ? w : 0ull;
    }
  }
  const float sl = p.scale * kLog2e;
  float M[RT], l[RT];
  floatx4 o[RT][FT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    M[rt] = -INFINITY;
    l[rt] = 0.f;
#pragma unroll
    for (int t = 0; t < FT; ++t) o[rt][t] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  auto step = [&](KvBlock<HD>& cur, int blk) {
    const int p0 = 32 * blk, nxt = blk + 2 * kWaves;
    const bool tail = p0 + 32 > L;
    floatx4 z[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        z[rt][u] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = NQ - 1; k >= 0; --k)  // (smallest terms first)
#pragma unroll
          for (int s = 0; s < S; ++s) z[rt][u] = mfma(cur.k[u][s], Q[rt][k][s], z[rt][u]);
      }
    ld.keys(cur, nxt, hi);
    if (tail) {
      // A hidden position may hold anything, NaN among it: its score is replaced,
      // and values behind the last row are cleared.  A value of the tree's own rows
      // that is not finite must not reach the rows that do not see it: it is cleared
      // too, and the rows that see it get NaN at its feature.
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int d = p0 + 16 * u + 4 * q + r - L;
            const bool sees = d < 0 || (d < n && (anc[rt] >> (d & 63) & 1ull));
            if (!sees) z[rt][u][r] = -INFINITY;
          }
      uint32_t keep[4], own[4], any = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        keep[j] = own[j] = 0;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int d = p0 + 8 * q + 2 * j + e - L;
          const uint32_t half = 0xffffu << (16 * e);
          if (d < n) keep[j] |= half;
          if (d >= 0 && d < n) own[j] |= half;
        }
      }
      auto broken = [&](uint32_t w, int j) {
        uint32_t m = 0;
        if ((w & 0x7f80u) == 0x7f80u) m |= 0xffffu;
        if ((w & 0x7f800000u) == 0x7f800000u) m |= 0xffff0000u;
        return m & own[j];
      };
#pragma unroll
      for (int t = 0; t < FT; ++t) {
        uint32_t* w = (uint32_t*)&cur.v[t];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          w[j] &= keep[j];
          any |= broken(w[j], j);
        }
      }
      if (__any(any != 0)) {
        bf16x8 sees[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          uint32_t w[4] = {};
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int d = p0 + 8 * q + e - L;
            if (d >= 0 && d < n && (anc[rt] >> (d & 63) & 1ull)) w[e >> 1] |= 0x3f80u << (16 * (e & 1));
          }
          sees[rt] = op(w[0], w[1], w[2], w[3]);
        }
#pragma unroll
        for (int t = 0; t < FT; ++t) {
          uint32_t* w = (uint32_t*)&cur.v[t];
          uint32_t one[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t m = broken(w[j], j);
            one[j] = m & 0x3f803f80u;
            w[j] &= ~m;
          }
          const uint4 a = make_uint4(one[0], one[1], one[2], one[3]);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            const floatx4 hit = mfma(a, sees[rt], floatx4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (hit[r] > 0.f) o[rt][t][r] = __uint_as_float(0x7fc00000u);
          }
        }
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
        uint32_t w[4];
        swap_words(pw[0][0][k], pw[1][0][k], w[0], w[2]);
        swap_words(pw[0][1][k], pw[1][1][k], w[1], w[3]);
        P[rt][k] = op(w[0], w[1], w[2], w[3]);
      }
    }
#pragma unroll
    for (int t = 0; t < FT; ++t)
#pragma unroll
      for (int k = NP - 1; k >= 0; --k)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) o[rt][t] = mfma(cur.v[t], P[rt][k], o[rt][t]);
    ld.values(cur, nxt, hi);
  };

  for (int blk = lo + wave; blk < hi; blk += 2 * kWaves) {
    step(buf[0], blk);
    if (blk + kWaves >= hi) break;
    step(buf[1], blk + kWaves);
  }

  // the waves' parts
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float s = sum_q(l[rt]);
    if (q == 0) {
      sm.m[wave][rt * 16 + c] = M[rt];
      sm.l[wave][rt * 16 + c] = s;
    }
  }
  __syncthreads();
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float m = sm.m[0][rt * 16 + c];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = fmaxf(m, sm.m[w][rt * 16 + c]);
    const float f = M[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M[rt] - m);
#pragma unroll
    for (int t = 0; t < FT; ++t) {
      const floatx4 x = o[rt][t] * f;
      *(floatx4*)&sm.o[wave][rt * 16 + c][16 * t + 4 * q] = x;
    }
  }
  __syncthreads();
  constexpr int LPR = HD / 4;  // lanes a row
  for (int k = tid; k < RT * 16 * LPR; k += kWaves * 64) {
    const int r = k / LPR, f = (k - r * LPR) * 4, m = r0 + r;
    if (m >= rows) break;
    float mx = sm.m[0][r];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) mx = fmaxf(mx, sm.m[w][r]);
    float s = 0.f;
    floatx4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float mw = sm.m[w][r];
      s += mw == -INFINITY ? sm.l[w][r] : sm.l[w][r] * __builtin_amdgcn_exp2f(mw - mx);
      x += *(const floatx4*)&sm.o[w][r][f];
    }
    if (p.NS == 1) {
      const int g = m / n, i = m - g * n;
      const float y[4] = {x[0] / s, x[1] / s, x[2] / s, x[3] / s};
      store4<QB>(p.out, ((int64_t)b * p.R + i) * p.out_ld + ((int64_t)kvh * p.G + g) * HD + f, y);
    } else {
      const int64_t at = (int64_t)unit * p.G * p.R + m;
      *(floatx4*)(p.part_o + at * HD + f) = x;
      if (f == 0) {
        p.part_ml[2 * at] = mx;
        p.part_ml[2 * at + 1] = s;
      }
    }
  }
}

// The splits of a row, in order: GR groups of HD / 4 lanes take every GR-th one.
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
  const int nb = (rr.L + rr.n + 31) / 32, ns = used ? (nb + p.CB - 1) / p.CB : 0;
  const int64_t at0 = bh * p.NS * p.G * p.R + (int64_t)g * rr.n + i, step = (int64_t)p.G * p.R;
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
// after their parents, so the walk ends.
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

template <int HD, bool BF16>
hipError_t append_t(TreeAppend a, hipStream_t st) {
  constexpr int HPW = 64 / (HD / 8), VHPW = 64 / (HD / 2);
  const int heads = (a.q != nullptr ? a.H : 0) + a.KVH, groups = (heads + HPW - 1) / HPW;
  const int64_t rows = (int64_t)a.B * a.R;
  // enough waves for the chip, then several groups of heads for one computation of the angles
  a.run = (int)std::min<int64_t>(std::max<int64_t>(rows * groups / 8192, 1), groups);
  const int64_t qk = (rows * ((groups + a.run - 1) / a.run) + 3) / 4;
  const int64_t vb = ((int64_t)a.B * ((a.R + 14) / 8) * ((a.KVH + VHPW - 1) / VHPW) + 3) / 4;
  if (qk + vb > 0x7fffffff) return hipErrorInvalidValue;
  a.qk_blocks = (int)qk;
  hipLaunchKernelGGL((tree_append_kernel<HD, BF16>), dim3((unsigned)(qk + vb)), dim3(256), 0, st, a);
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

constexpr int kTreeWgs = 1024;  // most workgroups of a call whose keys are split

template <int HD, bool QB, int RT>
hipError_t attend_rt(TreeAttend a, hipStream_t st) {
  const int tiles = (a.G * a.R + 15) / 16;
  a.RB = (tiles + RT - 1) / RT;
  const int blocks = (a.max_keys + 31) / 32;
  const int64_t items = (int64_t)a.B * a.KVH * a.RB;
  const int64_t want = RT == 1 ? 512 : 256;
  int64_t ns = std::min<int64_t>((a.B > 1 ? 2 : 1) * want / items, (blocks + 2 * kWaves - 1) / (2 * kWaves));
  ns = std::max<int64_t>(ns, 1);
  a.CB = (int)((blocks + ns - 1) / ns);
  a.NS = (blocks + a.CB - 1) / a.CB;
  const int64_t units = (int64_t)a.B * a.KVH * a.NS, grid = 8 * a.RB * ((units + 7) / 8);
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  if (a.NS > 1 && units * a.G * a.R > (int64_t)a.part_rows) return hipErrorInvalidValue;
  const void* fn = reinterpret_cast<const void*>(&tree_attend_kernel<HD, QB, RT>);
  constexpr int lds = (int)sizeof(TreeSmem<HD, RT>);
  if (lds > 65536) {  // once for every device
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (!(done.load() & bit)) {
      if ((e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, lds)) != hipSuccess) return e;
      done.fetch_or(bit);
    }
  }
  hipLaunchKernelGGL((tree_attend_kernel<HD, QB, RT>), dim3((unsigned)grid), dim3(kWaves * 64), lds, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.NS == 1) return e;
  constexpr int LPR = HD / 4, per = 256 / LPR;
  const int64_t rows = (int64_t)a.B * a.H * a.R;
  if (a.NS >= 8) hipLaunchKernelGGL((tree_merge_kernel<HD, QB, per>), dim3((unsigned)rows), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((tree_merge_kernel<HD, QB, 1>), dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, st, a);
  return hipGetLastError();
}

template <int HD, bool QB>
hipError_t attend_t(const TreeAttend& a, hipStream_t st) {
  const int tiles = (a.G * a.R + 15) / 16;
  if (tiles == 1) return attend_rt<HD, QB, 1>(a, st);
  if (!QB || tiles == 2) return attend_rt<HD, QB, 2>(a, st);
  return attend_rt<HD, QB, QB ? 4 : 2>(a, st);
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

// (a workgroup of a split call has at most 64 packed rows)
size_t tree_part_rows(int G, int max_rows) {
  return (size_t)kTreeWgs * std::min<int64_t>((int64_t)G * max_rows, 64);
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
