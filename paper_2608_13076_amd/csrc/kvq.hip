// Kernels of the 4-bit K/V cache (layout in kvq.h):
//   kvq_append_kernel   head norms, rotation and the 4-bit rows of new positions
//   kvq_read_kernel     rows of the cache as the values they stand for
//   kvq_attend_kernel   causal attention of a few rows per request, by chunks of keys
//   kvq_merge_kernel    the chunks' partials in chunk order
//   kvq_weights_kernel  the attention weight every position received
//   kvq_select_kernel   the positions a cache keeps: the last and the heaviest
//   kvq_move_kernel     closes the kept positions up
#include "kvq.h"

#include <float.h>

#include <algorithm>

#include "device_util.h"

namespace spade {

namespace {

// ---------------------------------------------------------------------------
// Append.  A row is a request's position i; hd / 8 lanes hold one head of it,
// lane c features 4 c .. + 3 and their rotary partners hd / 2 + 4 c .. + 3.
//
// A key's codes have to be those of its definition, so that a cache does not
// depend on how a sum was ordered: the norm and the rotation of keys run in
// double, the result is rounded once to float32 (v), and with m = bf16(min v),
// s = bf16((max v - m) * (1 / 15)) the code is the integer nearest to (v - m) /
// s, ties to even, clamped to 0..15.  The quotient comes from a reciprocal and is
// corrected by its exact remainder.  Queries stay in float32.
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t bf_bits(float f) { return (uint32_t)f2bf(f); }

template <int LPH>
__device__ __forceinline__ float min_lanes(float v) {
#pragma unroll
  for (int o = LPH / 2; o >= 1; o >>= 1) v = fminf(v, __shfl_xor(v, o));
  return v;
}
template <int LPH>
__device__ __forceinline__ float max_lanes(float v) {
#pragma unroll
  for (int o = LPH / 2; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
template <int LPH, typename F>
__device__ __forceinline__ F sum_lanes(F v) {
#pragma unroll
  for (int o = LPH / 2; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

template <bool BF16>
__device__ __forceinline__ void load4(const void* base, int64_t at, float* x) {
  if constexpr (BF16) {
    const uint2 w = *(const uint2*)((const uint16_t*)base + at);
    x[0] = __uint_as_float(w.x << 16);
    x[1] = __uint_as_float(w.x & 0xffff0000u);
    x[2] = __uint_as_float(w.y << 16);
    x[3] = __uint_as_float(w.y & 0xffff0000u);
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
  if constexpr (BF16) {
    *(uint2*)((uint16_t*)base + at) =
        make_uint2(bf_bits(x[0]) | (bf_bits(x[1]) << 16), bf_bits(x[2]) | (bf_bits(x[3]) << 16));
  } else {
    *(float4*)((float*)base + at) = make_float4(x[0], x[1], x[2], x[3]);
  }
}

// x: a lane's features (0..3 and their partners 4..7) of one head; norm (gain
// g != NULL) and rotation (rope row cs != NULL) in F.
template <int HD, typename F>
__device__ __forceinline__ void norm_rotate(F (&x)[8], const float* g, float eps, const float* cs, int c) {
  if (g != nullptr) {
    F ss = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) ss += x[j] * x[j];
    ss = sum_lanes<HD / 8>(ss);
    F r;
    if constexpr (sizeof(F) == 8) r = 1.0 / sqrt(ss / HD + (F)eps);
    else r = 1.0f / sqrtf(ss / HD + eps);
    float ga[4], gb[4];
    load4<false>(g, 4 * c, ga);
    load4<false>(g, HD / 2 + 4 * c, gb);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[j] = x[j] * r * ga[j];
      x[4 + j] = x[4 + j] * r * gb[j];
    }
  }
  if (cs != nullptr) {
    float t[8];
    load4<false>(cs, 8 * c, t);
    load4<false>(cs, 8 * c + 4, t + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const F co = t[2 * j], sn = t[2 * j + 1];
      const F a = x[j], b = x[4 + j];
      x[j] = a * co - b * sn;
      x[4 + j] = b * co + a * sn;
    }
  }
}

// Codes of a lane's features: nibbles 0..3 of word c / 2 (even lanes' half) in
// the low half, those of the partners in the high half; pair = scale | minimum.
template <int HD>
__device__ __forceinline__ uint32_t quantise(const float (&v)[8], uint32_t* pair) {
  float lo = fminf(fminf(fminf(v[0], v[1]), fminf(v[2], v[3])), fminf(fminf(v[4], v[5]), fminf(v[6], v[7])));
  float hi = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
  // NaN where a feature is not finite (min and max pass NaN over)
  float bad = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) bad += v[j] * 0.f;
  lo = min_lanes<HD / 8>(lo);
  hi = max_lanes<HD / 8>(hi);
  bad = sum_lanes<HD / 8>(bad);
  const uint16_t mb = f2bf(lo);
  const float m = bf2f(mb);
  const float span = fmaxf(hi - m, 0.f);
  bad += span * 0.f;  // a span beyond float32
  const uint16_t sb = f2bf(span * (1.0f / 15.0f));
  const float s = bf2f(sb);
  uint32_t code = 0;
  if (bad == 0.f && s > 0.f) {
    const double ds = s, inv = 1.0 / ds;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const double d = (double)v[j] - (double)m;
      double n = rint(d * inv);
      // exact remainder: the nearest integer, ties to even
      const double e = __builtin_fma(-n, ds, d), h = 0.5 * ds;
      const bool odd = ((int)n) & 1;
      if (e > h || (e == h && odd)) n += 1.0;
      else if (e < -h || (e == -h && odd)) n -= 1.0;
      const int ni = (int)fmin(fmax(n, 0.0), 15.0);
      code |= (uint32_t)ni << (j < 4 ? 4 * j : 16 + 4 * (j - 4));
    }
  }
  *pair = bad == 0.f ? ((uint32_t)sb | ((uint32_t)mb << 16)) : 0x7fc07fc0u;
  return code;
}

template <int HD, bool BF16>
__global__ void __launch_bounds__(256) kvq_append_kernel(KvqAppend p) {
  constexpr int LPH = HD / 8;
  const int c = threadIdx.x % LPH;
  const int HQ = p.q != nullptr ? p.H : 0;
  const int heads = HQ + 2 * p.KVH;
  const int64_t items = (int64_t)p.B * p.R * heads;
  const int64_t it = (int64_t)blockIdx.x * (256 / LPH) + threadIdx.x / LPH;
  if (it >= items) return;  // whole groups of LPH lanes
  const int64_t row = it / heads;
  int h = (int)(it - row * heads);
  const int b = (int)(row / p.R), i = (int)(row - (int64_t)b * p.R);
  const int n_rows = p.rows != nullptr ? min(p.rows[b], p.R) : p.R;
  const int f0 = 4 * c, f1 = HD / 2 + 4 * c;
  if (i >= n_rows) {  // a row the request does not use
    if (h < HQ) {
      const float z[4] = {0.f, 0.f, 0.f, 0.f};
      store4<BF16>(p.q_out, row * p.qo_ld + h * HD + f0, z);
      store4<BF16>(p.q_out, row * p.qo_ld + h * HD + f1, z);
    }
    return;
  }
  const int t = p.lens[b] + i;
  const float* cs = nullptr;
  if (p.rope != nullptr) {
    int pos = (p.pos != nullptr ? p.pos[b] : p.lens[b]) + i;
    if (pos < 0 || pos >= p.rope_len) {
      if (c == 0) flag_error(p.err, SPADE_DERR_CAPACITY);
      pos = pos < 0 ? 0 : p.rope_len - 1;
    }
    cs = p.rope + (size_t)pos * HD;
  }
  if (h < HQ) {
    float x[8];
    load4<BF16>(p.q, row * p.q_ld + h * HD + f0, x);
    load4<BF16>(p.q, row * p.q_ld + h * HD + f1, x + 4);
    norm_rotate<HD, float>(x, p.gain_q, p.eps, cs, c);
    store4<BF16>(p.q_out, row * p.qo_ld + h * HD + f0, x);
    store4<BF16>(p.q_out, row * p.qo_ld + h * HD + f1, x + 4);
    return;
  }
  h -= HQ;
  const bool key = h < p.KVH;
  if (!key) h -= p.KVH;
  float x[8];
  const void* src = key ? p.k : p.v;
  const int64_t at = row * (key ? p.k_ld : p.v_ld) + h * HD;
  load4<BF16>(src, at + f0, x);
  load4<BF16>(src, at + f1, x + 4);
  if (key && (p.gain_k != nullptr || cs != nullptr)) {
    double y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = x[j];
    norm_rotate<HD, double>(y, p.gain_k, p.eps, cs, c);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (float)y[j];
  }
  uint32_t pair;
  const uint32_t code = quantise<HD>(x, &pair);
  const uint32_t other = __shfl_xor(code, 1);
  if (t < 0 || t >= p.max_len) {
    if (c == 0) flag_error(p.err, SPADE_DERR_CAPACITY);
    return;
  }
  // even lanes put the word of features 8 (c / 2) .. + 7 together, odd lanes
  // that of their partners
  const bool odd = c & 1;
  const uint32_t word = odd ? ((other >> 16) | (code & 0xffff0000u)) : ((code & 0xffffu) | (other << 16));
  const int w = (odd ? HD / 16 : 0) + c / 2;
  uint8_t* blk = p.cache + (size_t)((int64_t)b * p.KVH + h) * p.head_bytes +
                 (size_t)(t / kKvqBlock) * kvq_block_bytes(HD);
  const int tb = t % kKvqBlock;
  *(uint32_t*)(blk + (key ? kvq_k_word(tb, w, HD) : kvq_v_word(tb, w, HD))) = word;
  if (c == 0) {
    *(uint32_t*)(blk + kvq_pair(tb, HD) + (key ? 0 : 4)) = pair;
    if (key && p.weights != nullptr) p.weights[((int64_t)b * p.KVH + h) * p.max_len + t] = 0.f;
  }
}

// ---------------------------------------------------------------------------
// Read back: lanes as in the append.
// ---------------------------------------------------------------------------
template <int HD, bool BF16>
__global__ void __launch_bounds__(256) kvq_read_kernel(KvqRead p) {
  constexpr int LPH = HD / 8;
  const int c = threadIdx.x % LPH;
  const int64_t items = (int64_t)p.B * p.R * p.KVH;
  const int64_t it = (int64_t)blockIdx.x * (256 / LPH) + threadIdx.x / LPH;
  if (it >= items) return;
  const int64_t row = it / p.KVH;
  const int h = (int)(it - row * p.KVH);
  const int b = (int)(row / p.R), i = (int)(row - (int64_t)b * p.R);
  const int n_rows = p.rows != nullptr ? min(p.rows[b], p.R) : p.R;
  const int t = (p.start != nullptr ? p.start[b] : 0) + i;
  const bool live = i < n_rows && t >= 0 && t < p.max_len;
  float x[2][8] = {};
  if (live) {
    const uint8_t* blk = p.cache + (size_t)((int64_t)b * p.KVH + h) * p.head_bytes +
                         (size_t)(t / kKvqBlock) * kvq_block_bytes(HD);
    const int tb = t % kKvqBlock;
    const uint2 pr = *(const uint2*)(blk + kvq_pair(tb, HD));
    const uint32_t w[2] = {*(const uint32_t*)(blk + kvq_k_word(tb, c, HD)), *(const uint32_t*)(blk + kvq_v_word(tb, c, HD))};
#pragma unroll
    for (int o = 0; o < 2; ++o) {
      const uint32_t pp = o ? pr.y : pr.x;
      const float s = __uint_as_float(pp << 16), m = __uint_as_float(pp & 0xffff0000u);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[o][j] = m + (float)((w[o] >> (4 * j)) & 15u) * s;
    }
  }
  const int64_t at = it * HD + 8 * c;
  store4<BF16>(p.k, at, x[0]);
  store4<BF16>(p.k, at + 4, x[0] + 4);
  store4<BF16>(p.v, at, x[1]);
  store4<BF16>(p.v, at + 4, x[1] + 4);
}

// ---------------------------------------------------------------------------
// Attention.
//
// Row i of request b (i < rows[b]) sees positions 0 .. lens[b] + i.  The G R
// rows that share a K/V head are packed (row g R + i) into 16-row tiles; a
// workgroup of W waves takes T tiles over a chunk of keys, wave w every W-th
// block of 32 positions, with a running maximum, sum and output of its own
// (one pass over the codes; the waves meet once, at the end of the chunk).
//
// Both products are transposed, so nothing crosses lanes between them:
//   S^T = K Q^T   A = codes of 16 positions, B = queries; lane 16 q + c gets
//                 the scores of row c at positions 4 q .. + 3
//   O^T = V^T P^T B = probabilities of 2 x 16 positions straight from those
//                 registers (k slots 8 q .. + 7 are positions 4 q .. + 3 of
//                 either half), A = codes of features 8 c + j, j the product
// A code n enters as the bf16 number 16 + n (one shift, one and-or for two
// codes), exact; with x = m + n s the scores are
//   q . x = s (sum_f q_f (16 + n_f) - 16 sum_f q_f) + m sum_f q_f
// (the sum over 16 + n starts at -16 sum q), and with x = c + (n - 8) s,
//   sum_t p_t x_t = sum_t p_t s_t (16 + n_t) - 24 sum_t p_t s_t + sum_t p_t c_t.
// Float32 queries enter as three bf16 terms, which hold all of their 24 bits,
// and so do the products p s; bfloat16 calls take their queries as they are and
// round p s to bfloat16 once (2^-9 of a weight, half a step of their outputs).
// ---------------------------------------------------------------------------
constexpr int kWaves = 4;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ uint32_t pk_bf16(float a, float b) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)a) | ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)b) << 16);
}
__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// the codes at bits 3..6 and 19..22 of x as the bf16 pair (16 + n, 16 + n')
__device__ __forceinline__ uint32_t code16(uint32_t x) { return (x & 0x00780078u) | 0x41804180u; }
__device__ __forceinline__ uint32_t code_pair(uint32_t w, int j) { return code16(j == 0 ? w << 3 : w >> (4 * j - 3)); }

__device__ __forceinline__ bf16x8 op(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(bf16x8, make_uint4(a, b, c, d));
}
__device__ __forceinline__ floatx4 mfma(bf16x8 a, bf16x8 b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// the bf16 terms of two floats, largest first
template <int N>
__device__ __forceinline__ void terms(float a, float b, uint32_t (&w)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    w[i] = pk_bf16(a, b);
    a -= lo_f(w[i]);
    b -= hi_f(w[i]);
  }
}

// lanes l, l ^ 16, l ^ 32, l ^ 48 combined in all of them
__device__ __forceinline__ float max_q(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
}
__device__ __forceinline__ float sum_q(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(t[0]) + __uint_as_float(t[1]);
}

// Queries of one row in a lane: its quarter of the features (HD / 4 from q HD / 4
// on), as the B operands of the HD / 32 steps; dword j of step s holds
// features 8 s + j and 8 s + j + 4 of the quarter, the order of a code word.
template <int HD, bool QB>
struct Queries {
  static constexpr int S = HD / 32, N = QB ? 1 : 3;
  uint32_t w[N][S][4];
  float sum;  // of the row's features
  __device__ __forceinline__ void load(const void* base, int64_t at, bool ok, int q) {
    float x[8], t = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = 0.f;
      if (ok) {
        load4<QB>(base, at + q * (HD / 4) + 8 * s, x);
        load4<QB>(base, at + q * (HD / 4) + 8 * s + 4, x + 4);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t e[N];
        terms<N>(x[j], x[j + 4], e);
#pragma unroll
        for (int n = 0; n < N; ++n) w[n][s][j] = e[n];
        t += x[j] + x[j + 4];
      }
    }
    sum = sum_q(t);
  }
};

// A wave's part of one block of 32 positions.
template <int HD>
struct Block {
  static constexpr int KW = HD / 32;  // words of a lane's quarter of a key
  uint32_t k[2][KW];
  uint4 v[2];
  uint4 pr[2][2];  // (key pair, value pair) of positions 16 u + 4 q .. + 3
};

template <int HD>
__device__ __forceinline__ void load_keys(Block<HD>& b, const uint8_t* blk, int q, int c) {
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const uint8_t* p = blk + (16 * u + c) * (HD / 2) + q * (HD / 8);
    if constexpr (HD == 128) {
      const uint4 w = *(const uint4*)p;
      b.k[u][0] = w.x;
      b.k[u][1] = w.y;
      b.k[u][2] = w.z;
      b.k[u][3] = w.w;
    } else {
      const uint2 w = *(const uint2*)p;
      b.k[u][0] = w.x;
      b.k[u][1] = w.y;
    }
    const uint4* pr = (const uint4*)(blk + kvq_pair(16 * u + 4 * q, HD));
    b.pr[u][0] = pr[0];
    b.pr[u][1] = pr[1];
  }
}

template <int HD>
__device__ __forceinline__ void load_values(Block<HD>& b, const uint8_t* blk, int q, int c) {
#pragma unroll
  for (int u = 0; u < 2; ++u)
    b.v[u] = *(const uint4*)(blk + kvq_v_word(16 * u + 4 * q, HD == 128 ? c : c / 2, HD));
}

__device__ __forceinline__ uint32_t key_pair_of(const uint4 (&pr)[2], int r) {
  return r == 0 ? pr[0].x : r == 1 ? pr[0].z : r == 2 ? pr[1].x : pr[1].z;
}
__device__ __forceinline__ uint32_t value_pair_of(const uint4 (&pr)[2], int r) {
  return r == 0 ? pr[0].y : r == 1 ? pr[0].w : r == 2 ? pr[1].y : pr[1].w;
}

// z[u][r]: the (unscaled) score of the lane's row at position 16 u + 4 q + r
template <int HD, bool QB, int T>
__device__ __forceinline__ void scores(const Block<HD>& b, const Queries<HD, QB> (&Q)[T], float (&z)[T][2][4]) {
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    floatx4 acc[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const float o = -16.f * Q[t].sum;
      acc[t] = floatx4{o, o, o, o};
    }
#pragma unroll
    for (int s = 0; s < HD / 32; ++s) {
      const uint32_t w = b.k[u][s];
      const bf16x8 a = op(code_pair(w, 0), code_pair(w, 1), code_pair(w, 2), code_pair(w, 3));
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int n = 0; n < Queries<HD, QB>::N; ++n)
          acc[t] = mfma(a, op(Q[t].w[n][s][0], Q[t].w[n][s][1], Q[t].w[n][s][2], Q[t].w[n][s][3]), acc[t]);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint32_t pr = key_pair_of(b.pr[u], r);
      const float s = lo_f(pr), m = hi_f(pr);
#pragma unroll
      for (int t = 0; t < T; ++t) z[t][u][r] = __builtin_fmaf(s, acc[t][r], m * Q[t].sum);
    }
  }
}

struct RequestRows {
  int L, n;  // cached positions before the rows, rows in use
};

__device__ __forceinline__ RequestRows request_rows(const KvqAttend& p, int b) {
  RequestRows r;
  r.n = p.rows != nullptr ? max(0, min(p.rows[b], p.R)) : p.R;
  r.L = p.lens[b];
  if (r.L < 0 || r.L + r.n > p.max_keys) {
    flag_error(p.err, SPADE_DERR_CAPACITY);
    r.L = r.L < 0 ? 0 : max(0, p.max_keys - r.n);
  }
  return r;
}

template <int HD>
struct AttendSmem {
  float o[kWaves][16][HD + 4];
  float m[kWaves][16], l[kWaves][16];
};

// Output of (request b, packed row pr, features f .. + 3)
__device__ __forceinline__ void store_out(const KvqAttend& p, int b, int kvh, int pr, int f, const float* x) {
  const int g = pr / p.R, i = pr - g * p.R;
  const int64_t at = ((int64_t)b * p.R + i) * p.out_ld + (kvh * p.G + g) * p.hd + f;
  if (p.bf16) store4<true>(p.out, at, x);
  else store4<false>(p.out, at, x);
}

template <int HD, int T, bool QB>
__global__ void __launch_bounds__(kWaves * 64) kvq_attend_kernel(KvqAttend p) {
  constexpr int FT = HD / 16;  // O^T products: features (HD / 16) c + j
  __shared__ AttendSmem<HD> sm;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, q = lane >> 4, c = lane & 15;
  // the tile groups of one chunk run on one XCD (workgroup i on XCD i % 8)
  const int x = (int)blockIdx.x & 7, jj = (int)blockIdx.x >> 3;
  const int tt = jj / p.TG, tg = jj - tt * p.TG;
  const int64_t item = 8ll * tt + x;
  const int chunk = (int)(item % p.NC);
  const int64_t bh = item / p.NC;
  if (bh >= (int64_t)p.B * p.KVH) return;
  const int b = (int)(bh / p.KVH), kvh = (int)(bh - (int64_t)b * p.KVH);
  const RequestRows rr = request_rows(p, b);
  const int NR = p.G * p.R, keys = rr.L + rr.n;
  const int k_lo = chunk * p.CK, k_hi = min(k_lo + p.CK, keys);
  if (p.NC > 1 && (rr.n == 0 || k_lo >= keys)) return;  // (one chunk: it writes the zeros)

  Queries<HD, QB> Q[T];
  int vis[T];  // positions the lane's row sees
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const int pr = (tg * T + t) * 16 + c, g = pr / p.R, i = pr - g * p.R;
    const bool ok = pr < NR && i < rr.n;
    vis[t] = ok ? rr.L + i + 1 : 0;
    Q[t].load(p.q, ((int64_t)b * p.R + i) * p.q_ld + (kvh * p.G + g) * HD, ok, q);
  }
  float M[T], l[T], cs[T];
  floatx4 o[T][FT], ps[T];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    M[t] = -INFINITY;
    l[t] = cs[t] = 0.f;
    ps[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < FT; ++j) o[t][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  const float sl = p.scale * kLog2e;
  const uint8_t* head = p.cache + (size_t)bh * p.head_bytes;
  const uint32_t bb = kvq_block_bytes(HD);
  const int blk_hi = (k_hi + kKvqBlock - 1) / kKvqBlock;
  int blk = k_lo / kKvqBlock + wave;
  Block<HD> cur;
  if (blk < blk_hi) {
    load_keys<HD>(cur, head + (size_t)blk * bb, q, c);
    load_values<HD>(cur, head + (size_t)blk * bb, q, c);
  }
  for (; blk < blk_hi; blk += kWaves) {
    Block<HD> nxt;
    {  // (the last round loads its own block again)
      const int nb = blk + kWaves < blk_hi ? blk + kWaves : blk;
      load_keys<HD>(nxt, head + (size_t)nb * bb, q, c);
      load_values<HD>(nxt, head + (size_t)nb * bb, q, c);
    }
    float z[T][2][4];
    scores<HD, QB, T>(cur, Q, z);
    const int p0 = blk * kKvqBlock;
    const bool tail = p0 + kKvqBlock > rr.L + 1;  // some row does not see all of the block
    if (tail) {
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (p0 + 16 * u + 4 * q + r >= vis[t]) z[t][u][r] = -INFINITY;
    }
    constexpr int N = QB ? 1 : 3;
    uint32_t pw[T][N][4];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      float mx = fmaxf(fmaxf(fmaxf(z[t][0][0], z[t][0][1]), fmaxf(z[t][0][2], z[t][0][3])),
                       fmaxf(fmaxf(z[t][1][0], z[t][1][1]), fmaxf(z[t][1][2], z[t][1][3])));
      mx = max_q(mx);
      if (__any(mx > M[t])) {
        const float mn = fmaxf(M[t], mx);
        const float f = M[t] == -INFINITY ? 0.f : exp2f((M[t] - mn) * sl);
        M[t] = mn;
        l[t] *= f;
        cs[t] *= f;
        ps[t] *= f;
#pragma unroll
        for (int j = 0; j < FT; ++j) o[t][j] *= f;
      }
      const float base = M[t] == -INFINITY ? 0.f : M[t] * sl;
      float w[8];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(z[t][u][r], sl, -base));
          const uint32_t pr = value_pair_of(cur.pr[u], r);
          float s = lo_f(pr), m = hi_f(pr);
          // a hidden position may hold anything, NaN among it
          if (tail && p0 + 16 * u + 4 * q + r >= vis[t]) s = m = 0.f;
          l[t] += e;
          cs[t] = __builtin_fmaf(e, __builtin_fmaf(8.f, s, m), cs[t]);
          w[4 * u + r] = e * s;
        }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t x[N];
        terms<N>(w[2 * e], w[2 * e + 1], x);
#pragma unroll
        for (int n = 0; n < N; ++n) pw[t][n][e] = x[n];
      }
    }
    // V^T: for the pairs of positions (2 e, 2 e + 1) of the lane's eight, the
    // halves of their words side by side
    uint32_t half[2][4];
    {
      const uint32_t vw[8] = {cur.v[0].x, cur.v[0].y, cur.v[0].z, cur.v[0].w,
                              cur.v[1].x, cur.v[1].y, cur.v[1].z, cur.v[1].w};
      const uint32_t sel = HD == 128 ? 0x05040100u : (c & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        half[0][e] = __builtin_amdgcn_perm(vw[2 * e + 1], vw[2 * e], sel);
        half[1][e] = HD == 128 ? __builtin_amdgcn_perm(vw[2 * e + 1], vw[2 * e], 0x07060302u) : 0u;
      }
    }
    const bf16x8 ones = op(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int n = 0; n < N; ++n) ps[t] = mfma(ones, op(pw[t][n][0], pw[t][n][1], pw[t][n][2], pw[t][n][3]), ps[t]);
#pragma unroll
    for (int j = 0; j < FT; ++j) {
      const uint32_t(&hf)[4] = half[j >> 2];
      const bf16x8 a = op(code_pair(hf[0], j & 3), code_pair(hf[1], j & 3), code_pair(hf[2], j & 3), code_pair(hf[3], j & 3));
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int n = 0; n < N; ++n)
          o[t][j] = mfma(a, op(pw[t][n][0], pw[t][n][1], pw[t][n][2], pw[t][n][3]), o[t][j]);
    }
    cur = nxt;
  }

  // the waves' parts, tile by tile; lane 16 q + c holds row c, features
  // q HD / 4 + FT r + j
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const float lt = sum_q(l[t]), off = sum_q(cs[t]) - 24.f * ps[t][0];
    if (t > 0) __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < FT; j += 4)
        *(float4*)&sm.o[wave][c][q * (HD / 4) + r * FT + j] =
            make_float4(o[t][j][r] + off, o[t][j + 1][r] + off, o[t][j + 2][r] + off, o[t][j + 3][r] + off);
    if (q == 0) {
      sm.m[wave][c] = M[t];
      sm.l[wave][c] = lt;
    }
    __syncthreads();
    const int row0 = (tg * T + t) * 16;
    for (int e = tid; e < 16 * (HD / 4); e += kWaves * 64) {
      const int row = e / (HD / 4), f = 4 * (e - row * (HD / 4)), pr = row0 + row;
      if (pr >= NR) continue;
      float mm = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) mm = fmaxf(mm, sm.m[w][row]);
      float ll = 0.f, a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float mw = sm.m[w][row];
        if (mw == -INFINITY && sm.l[w][row] == 0.f) continue;  // the wave saw nothing of this row
        const float s = exp2f((mw - mm) * sl);
        const float4 v = *(const float4*)&sm.o[w][row][f];
        ll += sm.l[w][row] * s;
        a[0] += v.x * s;
        a[1] += v.y * s;
        a[2] += v.z * s;
        a[3] += v.w * s;
      }
      if (p.NC == 1) {
        const bool live = pr - pr / p.R * p.R < rr.n;
        const float inv = 1.0f / ll;
#pragma unroll
        for (int k = 0; k < 4; ++k) a[k] = live ? a[k] * inv : 0.f;
        store_out(p, b, kvh, pr, f, a);
        if (f == 0 && p.w_out != nullptr) p.lse[bh * NR + pr] = live ? mm * sl + log2f(ll) : INFINITY;
      } else {
        const int64_t at = (bh * p.NC + chunk) * NR + pr;
        *(float4*)(p.part_o + at * HD + f) = make_float4(a[0], a[1], a[2], a[3]);
        if (f == 0) *(float2*)(p.part_ml + at * 2) = make_float2(mm, ll);
      }
    }
  }
}

// Merge of the chunks of one (request, K/V head, packed row), in chunk order:
// HD / 4 lanes per row.
template <int HD>
__global__ void __launch_bounds__(256) kvq_merge_kernel(KvqAttend p) {
  constexpr int LPR = HD / 4;
  const int NR = p.G * p.R;
  const int64_t row = (int64_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
  if (row >= (int64_t)p.B * p.KVH * NR) return;
  const int f = 4 * (threadIdx.x % LPR);
  const int64_t bh = row / NR;
  const int pr = (int)(row - bh * NR);
  const int b = (int)(bh / p.KVH), kvh = (int)(bh - (int64_t)b * p.KVH);
  const RequestRows rr = request_rows(p, b);
  const int i = pr - pr / p.R * p.R;
  float a[4] = {0.f, 0.f, 0.f, 0.f};
  float lse = INFINITY;
  if (i < rr.n) {
    const float sl = p.scale * kLog2e;
    // chunks with a position that the row sees
    const int nc = min((rr.L + i + p.CK) / p.CK, p.NC);
    const float* ml = p.part_ml + ((bh * p.NC) * NR + pr) * 2;
    const float* po = p.part_o + ((bh * p.NC) * NR + pr) * HD + f;
    float M = -INFINITY;
    for (int k = 0; k < nc; ++k) M = fmaxf(M, ml[(int64_t)k * NR * 2]);
    float l = 0.f;
#pragma unroll 4
    for (int k = 0; k < nc; ++k) {
      const float2 v = *(const float2*)(ml + (int64_t)k * NR * 2);
      const float s = exp2f((v.x - M) * sl);
      const float4 o = *(const float4*)(po + (int64_t)k * NR * HD);
      l += v.y * s;
      a[0] += o.x * s;
      a[1] += o.y * s;
      a[2] += o.z * s;
      a[3] += o.w * s;
    }
    const float inv = 1.0f / l;
#pragma unroll
    for (int k = 0; k < 4; ++k) a[k] *= inv;
    lse = M * sl + log2f(l);
  }
  store_out(p, b, kvh, pr, f, a);
  if (f == 0 && p.w_out != nullptr) p.lse[bh * NR + pr] = lse;
}

// Weights: out = in + the probabilities of the first w_rows rows, summed over
// the rows and the query heads of the K/V head.  The scores are taken again
// from the keys' codes (half of the cache) now that the rows' log-sum-exp is
// known; a wave owns its block of 32 positions, so nothing is added twice and
// the order of the sum is fixed.
template <int HD, bool QB>
__global__ void __launch_bounds__(kWaves * 64) kvq_weights_kernel(KvqAttend p) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, q = lane >> 4, c = lane & 15;
  const int64_t bh = blockIdx.x;
  const int b = (int)(bh / p.KVH), kvh = (int)(bh - (int64_t)b * p.KVH);
  const RequestRows rr = request_rows(p, b);
  const int keys = rr.L + rr.n, blocks = (keys + kKvqBlock - 1) / kKvqBlock;
  const int per = p.CK / kKvqBlock;
  const int lo = (int)blockIdx.y * per, hi = min(lo + per, blocks);
  const int nw = min(p.w_rows, rr.n), NW = p.G * nw;
  const float sl = p.scale * kLog2e;
  const uint8_t* head = p.cache + (size_t)bh * p.head_bytes;
  const uint32_t bb = kvq_block_bytes(HD);
  const float* lse = p.lse + bh * p.G * p.R;
  for (int blk = lo + wave; blk < hi; blk += kWaves) {
    Block<HD> cur;
    load_keys<HD>(cur, head + (size_t)blk * bb, q, c);
    const int p0 = blk * kKvqBlock;
    float add[2][4] = {};
    for (int r0 = 0; r0 < NW; r0 += 16) {
      const int pr = r0 + c, g = pr / nw, i = pr - g * nw;
      const bool ok = pr < NW;
      Queries<HD, QB> Q[1];
      Q[0].load(p.q, ((int64_t)b * p.R + i) * p.q_ld + (kvh * p.G + g) * HD, ok, q);
      const float ls = ok ? lse[g * p.R + i] : INFINITY;
      const int vis = ok ? rr.L + i + 1 : 0;
      float z[1][2][4];
      scores<HD, QB, 1>(cur, Q, z);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(z[0][u][r], sl, -ls));
          add[u][r] += p0 + 16 * u + 4 * q + r < vis ? e : 0.f;
        }
    }
    // over the sixteen rows; lane 16 q + 4 u + r stores position 16 u + 4 q + r
    float mine = 0.f;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float t = sum_lanes<16>(add[u][r]);
        if (c == 4 * u + r) mine = t;
      }
    const int pos = p0 + 16 * (c >> 2) + 4 * q + (c & 3);
    if (c < 8 && pos < keys) {
      const int64_t at = bh * p.max_len + pos;
      p.w_out[at] = (p.w_in != nullptr ? p.w_in[at] : 0.f) + mine;
    }
  }
}

// ---------------------------------------------------------------------------
// Eviction.
//
// kvq_select_kernel, a workgroup per (layer, request, K/V head): of n cached
// positions the last `recent` stay, and of the others the budget - recent
// heaviest, ties to the lower position.  The weight that decides is found by
// four passes over 8 bits of an order-preserving key, then one pass takes the
// positions in order.
// ---------------------------------------------------------------------------
constexpr int kSelThreads = 1024;

// larger key: heavier (NaN above everything, -0 as 0)
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0xffffffffu;
  uint32_t u = __float_as_uint(w);
  if (u == 0x80000000u) u = 0;
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__global__ void __launch_bounds__(kSelThreads) kvq_select_kernel(KvqEvict p) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t s_prefix, s_need;
  __shared__ uint32_t wsum[2][kSelThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int h = blockIdx.x % p.KVH, b = (blockIdx.x / p.KVH) % p.B, l = blockIdx.x / (p.KVH * p.B);
  const int64_t lbh = ((int64_t)l * p.batch + b) * p.KVH + h;
  const int64_t lbh_out = ((int64_t)l * p.out_batch + b) * p.KVH + h;
  const float* w = p.w + lbh * p.max_len;
  float* wo = p.w_out != nullptr ? p.w_out + lbh_out * p.out_max_len : nullptr;
  int32_t* kept = p.kept + lbh * p.budget;
  const int n = max(0, min(p.lens[b], p.max_len));
  if (n <= p.budget) {
    for (int j = tid; j < p.budget; j += kSelThreads) {
      kept[j] = j < n ? j : -1;
      if (j < n && wo != nullptr && wo != w) wo[j] = w[j];
    }
    return;
  }
  const int cand = n - p.recent;
  uint32_t need = (uint32_t)(p.budget - p.recent), prefix = 0, mask = 0;
  if (need > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int j = tid; j < cand; j += kSelThreads) {
        const uint32_t k = weight_key(w[j]);
        if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255], 1u);
      }
      __syncthreads();
      if (tid == 0) {  // from the heaviest bin down, the one that holds the last kept position
        uint32_t left = need;
        int d = 255;
        while (d > 0 && hist[d] < left) left -= hist[d--];
        s_prefix = prefix | ((uint32_t)d << shift);
        s_need = left;
      }
      __syncthreads();
      prefix = s_prefix;
      need = s_need;
      mask |= 0xffu << shift;
    }
  } else {
    prefix = 0xffffffffu;  // nothing but the last positions (need = 0: no ties are taken)
  }
  // every position heavier than the key, and the first `need` of those equal to it
  uint32_t base_k = 0, base_e = 0;
  for (int j0 = 0; j0 < n; j0 += kSelThreads) {
    const int j = j0 + tid;
    float wj = 0.f;
    bool gt = false, eq = false;
    if (j < n) {
      wj = w[j];
      const uint32_t k = weight_key(wj);
      gt = j >= cand || (k > prefix);
      eq = j < cand && k == prefix;
    }
    const uint64_t be = __ballot(eq);
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    if (lane == 0) wsum[0][wave] = (uint32_t)__popcll(be);
    __syncthreads();
    uint32_t e_at = base_e, e_all = 0;
    for (int k = 0; k < kSelThreads / 64; ++k) {
      if (k < wave) e_at += wsum[0][k];
      e_all += wsum[0][k];
    }
    e_at += (uint32_t)__popcll(be & below);
    const bool take = gt || (eq && e_at < need);
    const uint64_t bk = __ballot(take);
    if (lane == 0) wsum[1][wave] = (uint32_t)__popcll(bk);
    __syncthreads();
    uint32_t at = base_k, k_all = 0;
    for (int k = 0; k < kSelThreads / 64; ++k) {
      if (k < wave) at += wsum[1][k];
      k_all += wsum[1][k];
    }
    at += (uint32_t)__popcll(bk & below);
    if (take) {  // (at <= j, and every weight up to j has been read: in place is fine)
      kept[at] = j;
      if (wo != nullptr) wo[at] = wj;
    }
    base_k += k_all;
    base_e += e_all;
  }
}

// kvq_move_kernel: kept position j of the source becomes position j.  Grid
// ((layer, request, K/V head), part, column): a column is a quarter of the
// keys' codes, a quarter of the values' or the pairs.  In place one workgroup
// goes through its column in order: a row moves to a lower or the same place,
// and a round reads all of its rows before it writes the first.
constexpr int kMoveThreads = 256;
constexpr int kMoveCols = 9;

template <int HD>
__global__ void __launch_bounds__(kMoveThreads) kvq_move_kernel(KvqEvict p, int in_place) {
  const int z = blockIdx.x, col = blockIdx.z, tid = threadIdx.x;
  const int h = z % p.KVH, b = (z / p.KVH) % p.B, l = z / (p.KVH * p.B);
  const int64_t lbh = ((int64_t)l * p.batch + b) * p.KVH + h;
  const int64_t lbh_out = ((int64_t)l * p.out_batch + b) * p.KVH + h;
  // (lens may be lens_out: the minimum with the budget is the same before and after)
  const int m = max(0, min(min(p.lens[b], p.max_len), p.budget));
  const int32_t* kept = p.kept + lbh * p.budget;
  const uint8_t* src = p.cache + (size_t)lbh * p.head_bytes;
  uint8_t* dst = p.out + (size_t)lbh_out * p.out_head_bytes;
  constexpr uint32_t bb = (uint32_t)kKvqBlock * (HD + 8);
  constexpr int W = HD / 32;  // words of a column
  // rows of a round: threads are (row, word) of the column; the pairs' column has 2 words
  const int cw = col == 8 ? 2 : W;
  const int rpr = kMoveThreads / cw;
  const int r = tid / cw, wd = tid - r * cw;
  for (int j0 = (int)blockIdx.y * rpr; j0 < m; j0 += (int)gridDim.y * rpr) {
    const int j = j0 + r;
    uint32_t v = 0;
    size_t to = 0;
    bool move = j < m;
    if (move) {
      const int t = kept[j];
      const int tb = t % kKvqBlock, jb = j % kKvqBlock;
      uint32_t from;
      if (col < 4) {
        from = kvq_k_word(tb, col * W + wd, HD);
        to = kvq_k_word(jb, col * W + wd, HD);
      } else if (col < 8) {
        from = kvq_v_word(tb, (col - 4) * W + wd, HD);
        to = kvq_v_word(jb, (col - 4) * W + wd, HD);
      } else {
        from = kvq_pair(tb, HD) + 4 * wd;
        to = kvq_pair(jb, HD) + 4 * wd;
      }
      to += (size_t)(j / kKvqBlock) * bb;
      v = *(const uint32_t*)(src + (size_t)(t / kKvqBlock) * bb + from);
      if (in_place && t == j) move = false;
    }
    if (in_place) __syncthreads();
    if (move) *(uint32_t*)(dst + to) = v;
    if (in_place) __syncthreads();
  }
  if (col == 8 && blockIdx.y == 0 && l == 0 && h == 0 && tid == 0) p.lens_out[b] = m;
}

}  // namespace

hipError_t launch_kvq_append(const KvqAppend& a, hipStream_t st) {
  const int heads = (a.q != nullptr ? a.H : 0) + 2 * a.KVH;
  const int per = 256 / (a.hd / 8);
  const int64_t items = (int64_t)a.B * a.R * heads, grid = (items + per - 1) / per;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  const dim3 g((unsigned)grid);
  if (a.hd == 128) {
    if (a.bf16) hipLaunchKernelGGL((kvq_append_kernel<128, true>), g, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((kvq_append_kernel<128, false>), g, dim3(256), 0, st, a);
  } else {
    if (a.bf16) hipLaunchKernelGGL((kvq_append_kernel<64, true>), g, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((kvq_append_kernel<64, false>), g, dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

hipError_t launch_kvq_read(const KvqRead& a, hipStream_t st) {
  const int per = 256 / (a.hd / 8);
  const int64_t items = (int64_t)a.B * a.R * a.KVH, grid = (items + per - 1) / per;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  const dim3 g((unsigned)grid);
  if (a.hd == 128) {
    if (a.bf16) hipLaunchKernelGGL((kvq_read_kernel<128, true>), g, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((kvq_read_kernel<128, false>), g, dim3(256), 0, st, a);
  } else {
    if (a.bf16) hipLaunchKernelGGL((kvq_read_kernel<64, true>), g, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((kvq_read_kernel<64, false>), g, dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

namespace {

constexpr int kChunk = 512;  // keys per workgroup of the attention

template <int HD, int T>
void attend_t(const KvqAttend& a, unsigned grid, hipStream_t st) {
  if (a.bf16) hipLaunchKernelGGL((kvq_attend_kernel<HD, T, true>), dim3(grid), dim3(kWaves * 64), 0, st, a);
  else hipLaunchKernelGGL((kvq_attend_kernel<HD, T, false>), dim3(grid), dim3(kWaves * 64), 0, st, a);
}

template <int HD>
hipError_t attend_hd(KvqAttend a, hipStream_t st) {
  const int NR = a.G * a.R, tiles = (NR + 15) / 16, T = tiles > 1 ? 2 : 1;
  a.TG = (tiles + T - 1) / T;
  a.CK = kChunk;
  a.NC = std::max(1, (a.max_keys + a.CK - 1) / a.CK);
  const int64_t items = (int64_t)a.B * a.KVH * a.NC, grid = 8 * a.TG * ((items + 7) / 8);
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  if (T == 1) attend_t<HD, 1>(a, (unsigned)grid, st);
  else attend_t<HD, 2>(a, (unsigned)grid, st);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.NC > 1) {
    const int per = 256 / (HD / 4);
    const int64_t rows = (int64_t)a.B * a.KVH * NR;
    hipLaunchKernelGGL((kvq_merge_kernel<HD>), dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.w_out != nullptr) {
    const dim3 g((unsigned)(a.B * a.KVH), (unsigned)a.NC);
    if (a.bf16) hipLaunchKernelGGL((kvq_weights_kernel<HD, true>), g, dim3(kWaves * 64), 0, st, a);
    else hipLaunchKernelGGL((kvq_weights_kernel<HD, false>), g, dim3(kWaves * 64), 0, st, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

size_t kvq_attend_floats(int B, int H, int KVH, int hd, int max_len, int R, size_t* part_ml, size_t* lse) {
  const size_t rows = (size_t)B * H * R, nc = (size_t)std::max(1, (max_len + kChunk - 1) / kChunk);
  *part_ml = rows * nc * 2;
  *lse = rows;
  return rows * nc * hd;
}

hipError_t launch_kvq_attend(const KvqAttend& a, hipStream_t st) {
  return a.hd == 128 ? attend_hd<128>(a, st) : attend_hd<64>(a, st);
}

hipError_t launch_kvq_evict(const KvqEvict& a, hipStream_t st) {
  const int64_t heads = (int64_t)a.L * a.B * a.KVH;
  if (heads > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL(kvq_select_kernel, dim3((unsigned)heads), dim3(kSelThreads), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int in_place = a.cache == a.out;
  const dim3 g((unsigned)heads, in_place ? 1u : (unsigned)std::max(1, std::min((a.budget + 63) / 64, 64)), kMoveCols);
  if (a.hd == 128) hipLaunchKernelGGL((kvq_move_kernel<128>), g, dim3(kMoveThreads), 0, st, a, in_place);
  else hipLaunchKernelGGL((kvq_move_kernel<64>), g, dim3(kMoveThreads), 0, st, a, in_place);
  return hipGetLastError();
}

}  // namespace spade
