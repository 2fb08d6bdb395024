// Kernels of the 4-bit K/V cache (layout in kvq.h):
//   kvq_append_kernel   head norms, rotation and the 4-bit rows of new positions
//   kvq_read_kernel     rows of the cache as the values they stand for
//   kvq_attend_kernel   causal attention of a few rows per request, by ranges of keys
//   kvq_merge_kernel    the partials of a head's ranges, in order
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
// lane c features 4 c .. + 3 and their rotary partners hd / 2 + 4 c .. + 3.  With
// more than a few rows per request neighbouring lane groups take ROWS = 4 or 8
// rows of one head (a wave), whose value words are 16-byte pieces; else heads of
// one row.
//
// A key's codes have to be those of its definition, so that a cache does not
// depend on how a sum was ordered: the norm and the rotation of keys run in
// double, the result is rounded once to float32 (v), and with m = bf16(min v),
// s = bf16((max v - m) * (1 / 15)) the code is the integer nearest to (v - m) /
// s, ties to even, clamped to 0..15.  The quotient comes from a reciprocal and is
// corrected by its exact remainder.  Queries are normed in double too, whose squares
// stay in range; those that are only rotated stay in float32.
//
// 2048 rows of 32 + 64 bf16 heads take 26 us (76 MB, 2.9 TB/s; 25 with the inputs in
// the caches): by counters the vector units issue in 0.71 and the scalar unit in 0.47
// of the cycles, and waves wait for memory for 0.45 of theirs.  The same in float32
// 28 us (143 MB, 5.1 TB/s); one row of 48 heads 4 us, a launch and two memory
// latencies.
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t pk_bf16(float a, float b) {
  typedef __attribute__((ext_vector_type(2))) float f2;
  typedef __attribute__((ext_vector_type(2))) __bf16 b2;
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2){a, b}, b2));  // one v_cvt_pk_bf16_f32
}

// lengths come from the caller's device memory: sums stop at the type's ends
__device__ __forceinline__ int add_sat(int a, int b) { return __builtin_elementwise_add_sat(a, b); }

// v of another lane of the wave's groups of 16: step 0 and 1 swap neighbours and
// pairs, step 2 and 3 mirror eight and sixteen lanes (data-parallel moves, so a
// reduction that does not care for its order needs no LDS traffic)
template <int STEP>
__device__ __forceinline__ float lane_step(float v) {
  constexpr int ctrl = STEP == 0 ? 0xb1 : STEP == 1 ? 0x4e : STEP == 2 ? 0x141 : 0x140;
  const int i = __builtin_bit_cast(int, v);
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, ctrl, 0xf, 0xf, false));
}
template <int STEP>
__device__ __forceinline__ double lane_step(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __float_as_uint(lane_step<STEP>(__uint_as_float((uint32_t)u)));
  const uint32_t hi = __float_as_uint(lane_step<STEP>(__uint_as_float((uint32_t)(u >> 32))));
  return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}

// over the LPH = 8 or 16 lanes of a head, in all of them; NaN if one of them is
__device__ __forceinline__ float min_nan(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }
template <int LPH>
__device__ __forceinline__ float min_lanes(float v) {
  v = min_nan(v, lane_step<0>(v));
  v = min_nan(v, lane_step<1>(v));
  v = min_nan(v, lane_step<2>(v));
  if constexpr (LPH == 16) v = min_nan(v, lane_step<3>(v));
  return v;
}
template <int LPH>
__device__ __forceinline__ float max_lanes(float v) {
  v = max_nan(v, lane_step<0>(v));
  v = max_nan(v, lane_step<1>(v));
  v = max_nan(v, lane_step<2>(v));
  if constexpr (LPH == 16) v = max_nan(v, lane_step<3>(v));
  return v;
}
template <int LPH, typename F>
__device__ __forceinline__ F sum_lanes(F v) {
  v += lane_step<0>(v);
  v += lane_step<1>(v);
  v += lane_step<2>(v);
  if constexpr (LPH == 16) v += lane_step<3>(v);
  return v;
}
__device__ __forceinline__ float max_wave(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
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
    *(uint2*)((uint16_t*)base + at) = make_uint2(pk_bf16(x[0], x[1]), pk_bf16(x[2], x[3]));
  } else {
    *(float4*)((float*)base + at) = make_float4(x[0], x[1], x[2], x[3]);
  }
}

template <bool BF16>
__device__ __forceinline__ void store8(void* base, int64_t at, const float* x) {
  if constexpr (BF16) {
    *(uint4*)((uint16_t*)base + at) =
        make_uint4(pk_bf16(x[0], x[1]), pk_bf16(x[2], x[3]), pk_bf16(x[4], x[5]), pk_bf16(x[6], x[7]));
  } else {
    store4<false>(base, at, x);
    store4<false>(base, at + 4, x + 4);
  }
}

// Codes 0 .. 15 in nibbles to value codes and back (kvq.h), for both halves of a
// word: n is sign and magnitude of n - 7.5 in a nibble, then magnitudes of
// neighbouring nibbles change places and the signs of a half reverse.
__device__ __forceinline__ uint32_t sign_nibbles(uint32_t n) {
  const uint32_t low = ~n & 0x88888888u;  // n < 8
  return n ^ 0x88888888u ^ (low - (low >> 3));
}
__device__ __forceinline__ uint32_t nibbles_of_signs(uint32_t w) {
  const uint32_t neg = w & 0x88888888u;
  return w ^ 0x88888888u ^ (neg - (neg >> 3));
}
__device__ __forceinline__ uint32_t place_values(uint32_t w) {  // its own inverse
  const uint32_t s = __builtin_amdgcn_perm(w, w, 0x02030001u);
  return ((w & 0x07070707u) << 4) | ((w >> 4) & 0x07070707u) | ((s & 0x08080808u) << 4) | ((s >> 4) & 0x08080808u);
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
    if constexpr (sizeof(F) == 8) r = rsqrt(ss / HD + (F)eps);
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

// The integer nearest to (v - m) / s, ties to even, by its exact remainder.
__device__ __noinline__ float exact_code(float v, float m, float s) {
  const double ds = s, d = (double)v - (double)m;
  double n = rint(d / ds);
  const double e = __builtin_fma(-n, ds, d), h = 0.5 * ds;
  const bool odd = fmod(n, 2.0) != 0.0;
  if (e > h || (e == h && odd)) n += 1.0;
  else if (e < -h || (e == -h && odd)) n -= 1.0;
  return (float)fmin(fmax(n, -1.0), 16.0);
}

// Codes of a lane's features: nibbles 0..3 of word c / 2 (even lanes' half) in
// the low half, those of the partners in the high half; pair = scale | minimum.
template <int HD>
__device__ __forceinline__ uint32_t quantise(const float (&v)[8], uint32_t* pair) {
  float lo = v[0], hi = v[0];
#pragma unroll
  for (int j = 1; j < 8; ++j) {
    lo = min_nan(lo, v[j]);
    hi = max_nan(hi, v[j]);
  }
  lo = min_lanes<HD / 8>(lo);
  hi = max_lanes<HD / 8>(hi);
  const uint16_t mb = f2bf(lo);
  const float m = bf2f(mb);
  const bool bad = !(fabsf(hi - m) < INFINITY);  // a feature, the minimum as bfloat16 or the span is not finite
  const float span = max_nan(hi - m, 0.f);
  const uint16_t sb = f2bf(span * (1.0f / 15.0f));
  const float s = bf2f(sb);
  uint32_t code = 0;
  if (!bad && s > 0.f) {
    // a reciprocal within 2^-23 and two roundings of a quotient below 16: within 4e-6
    const float inv = __builtin_amdgcn_rcpf(s), h = 0.5f * s;
    float n[8];
    float far = s >= 0x1p-120f ? 0.f : 1.f;  // (1 / s may overflow)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float t = (v[j] - m) * inv;
      n[j] = rintf(t);
      far = fmaxf(far, fabsf(t - n[j]));
    }
    if (far > 0.49999f) {
      // next to a border (bfloat16 rows hit many exactly) n is at most one off and
      // put right by its remainder e, which float32 holds exactly where it holds
      // v - m
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = v[j] - m, back = v[j] - d, lost = (v[j] - (d + back)) + (back - m);
        if (lost != 0.f || !(s >= 0x1p-120f)) {
          n[j] = exact_code(v[j], m, s);
        } else {
          const float e = __builtin_fmaf(-n[j], s, d), ae = fabsf(e);
          const bool odd = (int)n[j] & 1;
          n[j] += ae > h || (ae == h && odd) ? copysignf(1.f, e) : 0.f;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t ni = (uint32_t)__builtin_amdgcn_fmed3f(n[j], 0.f, 15.f);
      code |= ni << (j < 4 ? 4 * j : 16 + 4 * (j - 4));
    }
  }
  *pair = bad ? 0x7fc07fc0u : (uint32_t)sb | ((uint32_t)mb << 16);
  return code;
}

// The head of a lane (LPH lanes a head, ROWS rows of it side by side); with rows
// enough for a wave it is the wave's, and all that follows from it scalar.
template <int LPH, int ROWS>
__device__ __forceinline__ int head_of() {
  const int h = (int)blockIdx.y * (256 / LPH / ROWS) + threadIdx.x / LPH / ROWS;
  return LPH * ROWS == 64 ? __builtin_amdgcn_readfirstlane(h) : h;
}

template <int HD, bool BF16, int ROWS>
__global__ void __launch_bounds__(256) kvq_append_kernel(KvqAppend p) {
  constexpr int LPH = HD / 8;
  const int c = threadIdx.x % LPH;
  const int HQ = p.q.p != nullptr ? p.H : 0, heads = HQ + 2 * p.KVH;
  int h = head_of<LPH, ROWS>();
  const int step = ROWS * p.run, per = (p.R + step - 1) / step, b = (int)blockIdx.x / per;
  const int first = ((int)blockIdx.x - b * per) * step;
  if (h >= heads) return;  // whole groups of LPH lanes
  const uint32_t f0 = 4 * c, f1 = HD / 2 + 4 * c;
  const bool query = h < HQ, key = !query && h < HQ + p.KVH;
  if (!query) h -= key ? HQ : HQ + p.KVH;
  // (selected member by member: a reference would be a load of its own)
  const void* in = query ? p.q.p : key ? p.k.p : p.v.p;
  const int64_t sb = query ? p.q.sb : key ? p.k.sb : p.v.sb, si = query ? p.q.si : key ? p.k.si : p.v.si,
                sh = query ? p.q.sh : key ? p.k.sh : p.v.sh;
  const int L = p.lens[b], n_rows = p.rows != nullptr ? min(p.rows[b], p.R) : p.R;
  const int pos0 = p.pos != nullptr ? p.pos[b] : L, shift = p.shift != nullptr ? p.shift[b] : 0;
  // (a head has less than 2^31 bytes)
  uint8_t* head = p.cache + (size_t)((int64_t)b * p.KVH + h) * p.head_bytes;
  for (int i = first + threadIdx.x / LPH % ROWS, end = min(first + step, p.R); i < end; i += ROWS) {
    const int64_t row = (int64_t)b * p.R + i;
    const int t = add_sat(L, i);
    float x[8];
    {
      const int64_t at = b * sb + i * si + h * sh;
      if (!BF16 && !query && !key && p.v_feature != 1) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[j] = ((const float*)in)[at + (int64_t)(f0 + j) * p.v_feature];
          x[4 + j] = ((const float*)in)[at + (int64_t)(f1 + j) * p.v_feature];
        }
      } else {
        load4<BF16>(in, at + f0, x);
        load4<BF16>(in, at + f1, x + 4);
      }
    }
    if (i >= n_rows) {  // a row the request does not use
      if (query) {
        const float z[4] = {0.f, 0.f, 0.f, 0.f};
        store4<BF16>(p.q_out, row * p.qo_ld + h * HD + f0, z);
        store4<BF16>(p.q_out, row * p.qo_ld + h * HD + f1, z);
      }
      continue;
    }
    const float* cs = nullptr;
    if (p.rope != nullptr) {
      int pos = add_sat(add_sat(pos0, i), shift);
      if (pos < 0 || pos >= p.rope_len) {
        if (c == 0) flag_error(p.err, SPADE_DERR_CAPACITY);
        pos = pos < 0 ? 0 : p.rope_len - 1;
      }
      cs = p.rope + (size_t)pos * HD;
    }
    const float* gain = query ? p.gain_q : key ? p.gain_k : nullptr;
    if (gain != nullptr || (key && cs != nullptr)) {
      double y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = x[j];
      norm_rotate<HD, double>(y, gain, p.eps, cs, c);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = (float)y[j];
    } else if (query) {
      norm_rotate<HD, float>(x, nullptr, p.eps, cs, c);
    }
    if (query) {
      store4<BF16>(p.q_out, row * p.qo_ld + h * HD + f0, x);
      store4<BF16>(p.q_out, row * p.qo_ld + h * HD + f1, x + 4);
      continue;
    }
    uint32_t pair;
    const uint32_t code = quantise<HD>(x, &pair);
    const uint32_t other = __float_as_uint(lane_step<0>(__uint_as_float(code)));
    if (t < 0 || t >= p.max_len) {
      if (c == 0) flag_error(p.err, SPADE_DERR_CAPACITY);
      continue;
    }
    // even lanes put the word of features 8 (c / 2) .. + 7 together, odd lanes
    // that of their partners
    const bool odd = c & 1;
    const uint32_t word = odd ? ((other >> 16) | (code & 0xffff0000u)) : ((code & 0xffffu) | (other << 16));
    const int w = (odd ? HD / 16 : 0) + c / 2;
    uint8_t* blk = head + (uint32_t)t / kKvqBlock * kvq_block_bytes(HD);
    const int tb = (uint32_t)t % kKvqBlock;
    if (key) *(uint32_t*)(blk + kvq_k_word(tb, w, HD)) = word;
    else *(uint32_t*)(blk + kvq_v_word(tb, w, HD)) = place_values(sign_nibbles(word));
    if (c == 0) {
      *(uint32_t*)(blk + kvq_pair(tb, HD) + (key ? 0 : 4)) = pair;
      if (key && p.weights != nullptr) p.weights[((int64_t)b * p.KVH + h) * p.max_len + t] = 0.f;
    }
  }
}

// ---------------------------------------------------------------------------
// Read back: lanes as in the append (2048 bf16 rows of 32 heads: 42 MB in 9.8 us).
// ---------------------------------------------------------------------------
template <int HD, bool BF16, int ROWS>
__global__ void __launch_bounds__(256) kvq_read_kernel(KvqRead p) {
  constexpr int LPH = HD / 8;
  const int c = threadIdx.x % LPH;
  const int h = head_of<LPH, ROWS>();
  const int per = (p.R + ROWS - 1) / ROWS, b = (int)blockIdx.x / per;
  const int i = ((int)blockIdx.x - b * per) * ROWS + threadIdx.x / LPH % ROWS;
  if (h >= p.KVH || i >= p.R) return;
  const int n_rows = p.rows != nullptr ? min(p.rows[b], p.R) : p.R;
  const int t = add_sat(p.start != nullptr ? p.start[b] : 0, i);
  const bool live = i < n_rows && t >= 0 && t < p.max_len;
  float x[2][8] = {};
  if (live) {
    const uint8_t* blk = p.cache + (size_t)((int64_t)b * p.KVH + h) * p.head_bytes +
                         (uint32_t)t / kKvqBlock * kvq_block_bytes(HD);
    const int tb = (uint32_t)t % kKvqBlock;
    const uint2 pr = *(const uint2*)(blk + kvq_pair(tb, HD));
    const uint32_t vw = place_values(*(const uint32_t*)(blk + kvq_v_word(tb, c, HD)));
    const uint32_t w[2] = {*(const uint32_t*)(blk + kvq_k_word(tb, c, HD)), nibbles_of_signs(vw)};
#pragma unroll
    for (int o = 0; o < 2; ++o) {
      const uint32_t pp = o ? pr.y : pr.x;
      const float s = __uint_as_float(pp << 16), m = __uint_as_float(pp & 0xffff0000u);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[o][j] = m + (float)((w[o] >> (4 * j)) & 15u) * s;
    }
  }
  const int64_t at = (((int64_t)b * p.R + i) * p.KVH + h) * HD + 8 * c;
  store8<BF16>(p.k, at, x[0]);
  store8<BF16>(p.v, at, x[1]);
}

// ---------------------------------------------------------------------------
// Attention.
//
// Row i of request b (i < rows[b]) sees positions 0 .. lens[b] + i.  The G R
// rows that share a K/V head are packed (row g R + i) into 16-row tiles; a
// workgroup of W waves takes one tile over a range of keys, wave w every W-th
// block of 32 positions, with a running maximum, sum and output of its own
// (one pass over the codes; the waves meet once, at the end of the range).
//
// Both products are transposed, so nothing crosses lanes between them:
//   S^T = K Q^T   A = codes of 16 positions, B = queries; lane 16 q + c gets
//                 the scores of row c at positions 4 q .. + 3
//   O^T = V^T P^T B = probabilities of 2 x 16 positions straight from those
//                 registers (k slots 8 q .. + 7 are positions 4 q .. + 3 of
//                 either half), A = codes of features 8 c + j, j the product
// Bits 0 .. 7 of a half word alone are a bf16 number, their value times 2^-133:
// subnormal up to 127, the first normal numbers from there (the matrix
// instructions keep subnormal inputs, and these products come out exact).  So a
// key code n in a nibble is the operand n 2^-133 or 16 n 2^-133 after a mask, and
// a shift by 8 for every other mask; queries of the features that enter sixteen
// times as large are divided by 16.  Value codes are held as sign and magnitude
// of n - 7.5 (kvq.h) so that a shift by 4, a swap of bytes and one and-or leave
// them at bits 15 and 3 .. 6: 16 (n - 7.5) 2^-133.  Queries carry 2^60 and
// probabilities 2^50 to keep the products in float32's normal range; with x = m +
// n s,
//   2^-73 q . x = s sum_f (2^60 q_f) (2^-133 n_f) + m 2^-73 sum_f q_f
//   sum_t p_t x_t = 2^129 sum_t (p_t s_t) (2^-129 (n_t - 7.5)) + sum_t p_t (m_t + 7.5 s_t).
// Float32 queries enter as three bf16 terms, which hold all of their 24 bits,
// and so do the products p s; bfloat16 calls take their queries as they are and
// hold p s in two terms, 16 bits (2^-17), so that nothing but the rounding of an
// output shows: 1.65e-3 of its size in norm, 2.1e-3 with one term, which costs less
// (us, one term / two: one row of 16 requests of 5000 to 16000 positions 34.3 /
// 35.5, of 120 thousand 29.7 / 30.3, of 129 5.2 / 5.3; 9 rows of 16 requests of 256
// to 4096 29.7 / 31.4).
// The matrix instructions cut the smaller of 32 products short by their operands'
// exponents: codes of both signs keep that from adding up, scores take their
// smallest terms first.  The 2^50 of the probabilities is a factor, not part of the
// exponent, which would be rounded at 50's step.  Error of float32 outputs relative
// to their size 5.5e-7 to 7.6e-7, of the weights 1.9e-7 to 6.9e-7 (200 to 30000
// positions; 2^50 in the exponent, of the weights too: 8.9e-7 to 1.1e-6, 1.3e-6 to
// 2.1e-6; the other choices cost more, measured earlier: codes of one sign, less
// eight times the sum of p s, 3.5e-6, largest terms first 1.1e-6).
// ---------------------------------------------------------------------------
constexpr int kWaves = 4;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kQScale = 0x1p60f, kZScale = 0x1p-73f;  // of queries; of the scores that come out
constexpr float kPScale = 0x1p50f;                     // of the probabilities
// sums of p (n - 7.5) as they come out, back in units of p
__device__ __forceinline__ float code_sum(float x) { return x * 0x1p100f * 0x1p29f; }

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// key codes j and j + 4 of a word as a bf16 pair; odd j sixteen times as large
__device__ __forceinline__ uint32_t code_pair(uint32_t w, int j) {
  return (j < 2 ? w : w >> 8) & (j & 1 ? 0x00f000f0u : 0x000f000fu);
}
__device__ __forceinline__ float code_scale(int j) { return j & 1 ? 0.0625f : 1.f; }
// value codes j of two half words, sixteen times n - 7.5 (swapped: the bytes of
// both halves)
__device__ __forceinline__ uint32_t value_pair(uint32_t w, uint32_t swapped, int j) {
  const uint32_t v = j < 2 ? w : swapped;
  uint32_t r;  // (one instruction, which takes one constant from a scalar register)
  asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(r) : "v"(j & 1 ? v << 4 : v), "s"(0x80708070u), "v"(0x00080008u));
  return r;
}

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

// A lane's quarter of a query as loaded (nothing waits for it before get).
template <int HD, bool QB>
struct RawQuery {
  static constexpr int V = HD / 32 * (QB ? 1 : 2);  // 16-byte (QB: eight-feature) pieces
  uint4 v[V];
  __device__ __forceinline__ void load(const void* base, int64_t at, int q) {
    if constexpr (QB) {
      const uint16_t* p = (const uint16_t*)base + at + q * (HD / 4);
#pragma unroll
      for (int i = 0; i < V; ++i) {  // (rows are aligned to 8 bytes)
        const uint2 a = *(const uint2*)(p + 8 * i), b = *(const uint2*)(p + 8 * i + 4);
        v[i] = make_uint4(a.x, a.y, b.x, b.y);
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = *(const uint4*)((const float*)base + at + q * (HD / 4) + 4 * i);
    }
  }
  __device__ __forceinline__ void get(int s, float (&x)[8]) const {
    if constexpr (QB) {
      const uint32_t w[4] = {v[s].x, v[s].y, v[s].z, v[s].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[2 * j] = lo_f(w[j]);
        x[2 * j + 1] = hi_f(w[j]);
      }
    } else {
      const uint4 a = v[2 * s], b = v[2 * s + 1];
      const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(w[j]);
    }
  }
};

// Queries of one row in a lane: its quarter of the features (HD / 4 from q HD / 4
// on), as the B operands of the HD / 32 steps; dword j of step s holds
// features 8 s + j and 8 s + j + 4 of the quarter, the order of a code word.
template <int HD, bool QB>
struct Queries {
  static constexpr int S = HD / 32, N = QB ? 1 : 3;
  uint32_t w[N][S][4];
  float sum;  // of the row's features, times kZScale
  __device__ __forceinline__ void convert(const RawQuery<HD, QB>& raw, bool ok) {
    float t = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      float x[8];
      raw.get(s, x);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float a = ok ? x[j] : 0.f, b = ok ? x[j + 4] : 0.f;
        uint32_t e[N];
        terms<N>(a * (kQScale * code_scale(j)), b * (kQScale * code_scale(j)), e);
#pragma unroll
        for (int n = 0; n < N; ++n) w[n][s][j] = e[n];
        t += a + b;
      }
    }
    sum = sum_q(t) * kZScale;
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

// Loads of block `blk` of a head (r: its region).  Values and pairs go by with
// the nt policy; keys may stay, and are in the Infinity Cache when the weights
// read them again (16 requests of 5000 to 16000 positions with weights: 62.0 us,
// 66.2 with nt for the keys too, 68.4 with it for nothing).
template <int HD>
struct BlockLoader {
  Rsrc r;
  uint32_t k, v, pr;  // the lane's offsets
  __device__ __forceinline__ void init(const uint8_t* head, size_t bytes, int q, int c) {
    r = make_rsrc(head, (uint32_t)bytes);
    k = (uint32_t)(c * (HD / 2) + q * (HD / 8));
    v = kvq_v_word(4 * q, HD == 128 ? c : c / 2, HD);
    pr = kvq_pair(4 * q, HD);
  }
  template <int AUX = kAuxStream>
  __device__ __forceinline__ uint4 b128(uint32_t off, uint32_t so) const {
    return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, (int)so, AUX));
  }
  __device__ __forceinline__ void keys(Block<HD>& b, int blk) const {
    const uint32_t so = (uint32_t)blk * kvq_block_bytes(HD);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if constexpr (HD == 128) {
        const uint4 w = b128<0>(k + 16 * u * (HD / 2), so);
        b.k[u][0] = w.x;
        b.k[u][1] = w.y;
        b.k[u][2] = w.z;
        b.k[u][3] = w.w;
      } else {
        const auto w = __builtin_amdgcn_raw_buffer_load_b64(r, (int)(k + 16 * u * (HD / 2)), (int)so, 0);
        b.k[u][0] = w[0];
        b.k[u][1] = w[1];
      }
    }
  }
  __device__ __forceinline__ void pairs(Block<HD>& b, int blk) const {
    const uint32_t so = (uint32_t)blk * kvq_block_bytes(HD);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      b.pr[u][0] = b128(pr + 128 * u, so);
      b.pr[u][1] = b128(pr + 128 * u + 16, so);
    }
  }
  __device__ __forceinline__ void values(Block<HD>& b, int blk) const {
    const uint32_t so = (uint32_t)blk * kvq_block_bytes(HD);
#pragma unroll
    for (int u = 0; u < 2; ++u) b.v[u] = b128(v + 4 * u * (HD / 8) * 16, so);
  }
};

__device__ __forceinline__ uint32_t key_pair_of(const uint4 (&pr)[2], int r) {
  return r == 0 ? pr[0].x : r == 1 ? pr[0].z : r == 2 ? pr[1].x : pr[1].z;
}
__device__ __forceinline__ uint32_t& value_pair_of(uint4 (&pr)[2], int r) {
  return r == 0 ? pr[0].y : r == 1 ? pr[0].w : r == 2 ? pr[1].y : pr[1].w;
}

// z[u][r]: kZScale times the (unscaled) score of the lane's row at position 16
// u + 4 q + r
template <int HD, bool QB>
__device__ __forceinline__ void scores(const Block<HD>& b, const Queries<HD, QB>& Q, float (&z)[2][4]) {
  floatx4 acc[2] = {};
  bf16x8 a[HD / 32][2];
#pragma unroll
  for (int n = Queries<HD, QB>::N - 1; n >= 0; --n)  // (smallest terms first)
#pragma unroll
    for (int s = 0; s < HD / 32; ++s) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint32_t w = b.k[u][s];
        if (n == Queries<HD, QB>::N - 1) a[s][u] = op(code_pair(w, 0), code_pair(w, 1), code_pair(w, 2), code_pair(w, 3));
        acc[u] = mfma(a[s][u], op(Q.w[n][s][0], Q.w[n][s][1], Q.w[n][s][2], Q.w[n][s][3]), acc[u]);
      }
    }
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint32_t pr = key_pair_of(b.pr[u], r);
      z[u][r] = __builtin_fmaf(lo_f(pr), acc[u][r], hi_f(pr) * Q.sum);
    }
}

struct RequestRows {
  int L, n;  // cached positions before the rows, rows in use: L, n >= 0, L + n <= max_keys
};

__device__ __forceinline__ RequestRows request_rows(const KvqAttend& p, int b) {
  RequestRows r;
  r.n = p.rows != nullptr ? max(0, min(p.rows[b], p.R)) : p.R;
  r.L = p.lens[b];
  if (r.L < 0 || r.L > p.max_keys - r.n) {  // (also where n > max_keys)
    flag_error(p.err, SPADE_DERR_CAPACITY);
    r.n = min(r.n, p.max_keys);
    r.L = r.L < 0 ? 0 : p.max_keys - r.n;
  }
  return r;
}

// Work of an attention call: the blocks of 32 positions of request 0's first
// K/V head, its second, .., request 1's, .., T in all, cut into WG ranges whose
// sizes differ by one at most, whatever the requests' lengths.  Every head
// counts kHeadCost blocks more, before its first: what its queries and its
// partial cost, about three blocks of each wave (ranges over many short requests
// took the longest without: 16 requests of 256 to 4096 positions, 9 rows, 40 us;
// 37 with 4, 34 with 8 to 16).
// Head bh's part of range w (a segment) leaves its partial in slot w + bh:
// along the cut one of the two moves on by one, so slots do not meet and a
// head's are contiguous.  The last bits of a row's result follow the cut, and
// so the batch.
constexpr int kHeadCost = 12;
struct Plan {
  uint32_t T, q, r;  // the first r ranges hold q + 1 blocks, the others q
  __device__ __forceinline__ uint32_t start(uint32_t w) const { return w * q + min(w, r); }
  __device__ __forceinline__ uint32_t range_of(uint32_t block) const {
    const uint32_t big = r * (q + 1);
    return block < big ? block / (q + 1) : r + (block - big) / q;
  }
};

// first block of part `part` of a head of nb blocks (parts may be empty)
__device__ __forceinline__ int even_start(int nb, unsigned part, int parts) {
  const unsigned q = (unsigned)nb / (unsigned)parts, r = (unsigned)nb - q * parts;
  return (int)(part * q + min(part, r));
}

// blocks that request b brings per K/V head (ALL: also without rows in use)
template <bool ALL>
__device__ __forceinline__ uint32_t request_blocks(const RequestRows& rr) {
  return !ALL && rr.n == 0 ? 0u : (uint32_t)(rr.L + rr.n + kKvqBlock - 1) / kKvqBlock;
}
// what they count in a plan
__device__ __forceinline__ uint32_t planned_blocks(uint32_t nb) { return nb > 0 ? nb + kHeadCost : 0u; }

// Planned blocks per K/V head of requests b0 .. b0 + 63, one per lane, and
// their inclusive prefix.
template <bool ALL>
__device__ __forceinline__ uint32_t scan_blocks(const KvqAttend& p, int b0, int lane, uint32_t* incl) {
  const uint32_t n = b0 + lane < p.B ? planned_blocks(request_blocks<ALL>(request_rows(p, b0 + lane))) : 0u;
  uint32_t v = n;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t t = __shfl_up(v, o);
    if (lane >= o) v += t;
  }
  *incl = v;
  return n;
}

__device__ __forceinline__ uint32_t lane_of(uint32_t v, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); }

__device__ __forceinline__ Plan make_plan(const KvqAttend& p, uint32_t blocks) {
  Plan pl;
  pl.T = blocks * (uint32_t)p.KVH;
  pl.q = pl.T / (uint32_t)p.WG;
  pl.r = pl.T - pl.q * (uint32_t)p.WG;
  return pl;
}

// The plan, and the request that holds the first block of range w with the
// blocks before that request (b = B: the range is empty).
template <bool ALL>
__device__ __forceinline__ Plan find_range(const KvqAttend& p, int lane, uint32_t w, int* b_out, uint32_t* before_out) {
  uint32_t incl;
  uint32_t n = scan_blocks<ALL>(p, 0, lane, &incl), sum = lane_of(incl, 63);
  for (int b0 = 64; b0 < p.B; b0 += 64) {
    uint32_t v;
    scan_blocks<ALL>(p, b0, lane, &v);
    sum += lane_of(v, 63);
  }
  const Plan pl = make_plan(p, sum);
  const uint32_t want = pl.start(w) / (uint32_t)p.KVH;  // of the requests' blocks per head
  uint32_t before = 0;
  *b_out = p.B;
  for (int b0 = 0;;) {
    const uint64_t hit = __ballot(before + incl > want);
    if (hit != 0) {
      const int l = __ffsll((unsigned long long)hit) - 1;
      *b_out = b0 + l;
      before += lane_of(incl - n, l);
      break;
    }
    before += lane_of(incl, 63);
    b0 += 64;
    if (b0 >= p.B) break;
    n = scan_blocks<ALL>(p, b0, lane, &incl);
  }
  *before_out = before * (uint32_t)p.KVH;
  return pl;
}

// The plan and the blocks before request b.
__device__ __forceinline__ Plan find_request(const KvqAttend& p, int lane, int b, uint32_t* before_out) {
  uint32_t sum = 0, before = 0;
  for (int b0 = 0; b0 < p.B; b0 += 64) {
    uint32_t incl;
    const uint32_t n = scan_blocks<false>(p, b0, lane, &incl);
    if (b >= b0 && b < b0 + 64) before = sum + lane_of(incl - n, b - b0);
    sum += lane_of(incl, 63);
  }
  *before_out = before * (uint32_t)p.KVH;
  return make_plan(p, sum);
}

// One segment after the other of range w: (request, K/V head, blocks lo .. hi - 1
// of nb).
template <bool ALL>
struct Segments {
  uint32_t left;  // planned blocks of the range still to go
  int b, h, lo, hi, nb;
  RequestRows rr;
  __device__ __forceinline__ bool init(const KvqAttend& p, int lane, uint32_t w) {
    uint32_t before;
    const Plan pl = find_range<ALL>(p, lane, w, &b, &before);
    const uint32_t s = pl.start(w);
    left = pl.start(w + 1) - s;
    if (b >= p.B || left == 0) return false;
    rr = request_rows(p, b);
    nb = (int)request_blocks<ALL>(rr);
    const uint32_t per = planned_blocks((uint32_t)nb);
    h = (int)((s - before) / per);
    return take(s - before - (uint32_t)h * per);
  }
  __device__ __forceinline__ bool next(const KvqAttend& p) {
    if (left == 0) return false;
    if (++h == p.KVH) {
      h = 0;
      do {  // (the plan counted these blocks, so there is such a request)
        if (++b >= p.B) return false;
        rr = request_rows(p, b);
        nb = (int)request_blocks<ALL>(rr);
      } while (nb == 0);
    }
    return take(0);
  }
  // the head's part from its planned block `at` on; false: the range ends
  // before the head's first block
  __device__ __forceinline__ bool take(uint32_t at) {
    const uint32_t end = min(planned_blocks((uint32_t)nb), at + left);
    left -= end - at;
    lo = max((int)at - kHeadCost, 0);
    hi = (int)end - kHeadCost;
    return hi > lo;
  }
};

template <int HD, int W>
struct AttendSmem {
  float o[W][16][HD + 4];
  float m[W][16], l[W][16];
};

// Output of (request b, packed row pr, features f .. + 3)
__device__ __forceinline__ void store_out(const KvqAttend& p, int b, int kvh, int pr, int f, const float* x) {
  const int g = pr / p.R, i = pr - g * p.R;
  const int64_t at = ((int64_t)b * p.R + i) * p.out_ld + (kvh * p.G + g) * p.hd + f;
  if (p.bf16) {
    store4<true>(p.out, at, x);
  } else if (p.split != 0) {  // hi = rne(x), lo = rne(x - hi)
    float lo[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) lo[k] = x[k] - bf2f(f2bf(x[k]));
    store4<true>(p.out, at, x);
    store4<true>(p.out, at + (int64_t)p.split, lo);
  } else {
    store4<false>(p.out, at, x);
  }
}

template <int HD, bool QB, int W>
__global__ void __launch_bounds__(W * 64) __attribute__((amdgpu_waves_per_eu(2))) kvq_attend_kernel(KvqAttend p) {
  constexpr bool WHOLE = W != kWaves;  // a workgroup takes all of a head
  constexpr int FT = HD / 16;        // O^T products: features (HD / 16) c + j
  constexpr int N = QB ? 2 : 3;      // bf16 terms of p s
  __shared__ AttendSmem<HD, W> sm;
  const int tid = threadIdx.x, lane = tid & 63, q = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Workgroup i runs on XCD i % 8: the row tiles of one range follow each other
  // on one XCD and share its L2.
  const unsigned xcd = blockIdx.x & 7, jj = blockIdx.x >> 3;
  const unsigned tt = jj / (unsigned)p.TG, tile = jj - tt * p.TG, range = 8 * tt + xcd;
  const int NR = p.G * p.R;
  const float sl = p.scale * kLog2e / kZScale;
  Segments<false> sg;
  const bool even = WHOLE || p.parts > 0;  // every head in so many equal parts
  if (even) {
    const unsigned head = range / (unsigned)p.parts, part = range - head * p.parts;
    if (head >= (unsigned)(p.B * p.KVH)) return;
    sg.b = (int)(head / (unsigned)p.KVH);
    sg.h = (int)(head - (unsigned)sg.b * p.KVH);
    sg.rr = request_rows(p, sg.b);
    sg.nb = (int)request_blocks<false>(sg.rr);
    sg.lo = even_start(sg.nb, part, p.parts);
    sg.hi = even_start(sg.nb, part + 1, p.parts);
  } else {
    if (range >= (unsigned)p.WG || !sg.init(p, lane, range)) return;
  }
  const unsigned my = tile * 16 + c, g = my / (unsigned)p.R;  // the lane's packed row
  const int i = (int)(my - g * p.R);
  const bool row_ok = my < (unsigned)NR;

  BlockLoader<HD> ld;
  RawQuery<HD, QB> qx;
  // The wave's blocks lo + wave, + W, ..: two in flight, a part of the next one
  // requested as soon as its registers are free (past the end: the last one
  // again).
  Block<HD> buf[2];
  auto request = [&]() {  // a segment's queries and first blocks
    ld.init(p.cache + (size_t)(sg.b * p.KVH + sg.h) * p.head_bytes, p.head_bytes, q, c);
    qx.load(p.q, ((int64_t)sg.b * p.R + (row_ok ? i : 0)) * p.q_ld + (sg.h * p.G + (row_ok ? (int)g : 0)) * HD, q);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int nb = max(min(sg.lo + wave + n * W, sg.hi - 1), 0);
      ld.keys(buf[n], nb);
      // (in the order of the loop, or its head would have to wait for more)
      asm volatile("" ::: "memory");
      ld.pairs(buf[n], nb);
      asm volatile("" ::: "memory");
      ld.values(buf[n], nb);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  request();
  for (;;) {
    const RequestRows rr = sg.rr;
    const int b = sg.b, kvh = sg.h, blk_hi = sg.hi;
    const unsigned bh = (unsigned)(b * p.KVH + kvh);
    const bool all = WHOLE || (even ? p.parts == 1 : sg.lo == 0 && sg.hi == sg.nb), ok = row_ok && i < rr.n;
    const int vis = ok ? rr.L + i + 1 : 0;  // positions the lane's row sees
    Queries<HD, QB> Q;
    Q.convert(qx, ok);
    float M = -INFINITY, l = 0.f, cs = 0.f;
    floatx4 o[FT];
#pragma unroll
    for (int j = 0; j < FT; ++j) o[j] = floatx4{0.f, 0.f, 0.f, 0.f};

    auto block = [&](Block<HD>& cur, int blk) {
      const int nb = min(blk + 2 * W, blk_hi - 1);  // the buffer's next block
      float z[2][4];
      scores<HD, QB>(cur, Q, z);
      ld.keys(cur, nb);
      asm volatile("" ::: "memory");  // (the compiler would request all parts at the block's end)
      const int p0 = blk * kKvqBlock;
      if (p0 + kKvqBlock > rr.L + 1) {  // some row does not see all of the block
        // a hidden position may hold anything, NaN among it
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (p0 + 16 * u + 4 * q + r >= vis) {
              z[u][r] = -INFINITY;
              value_pair_of(cur.pr[u], r) = 0;
            }
      }
      // (a row with a NaN is lost anyway: what becomes of its maximum is of no matter)
      float mx = z[0][0];
#pragma unroll
      for (int k = 1; k < 8; ++k) mx = max_nan(mx, z[k >> 2][k & 3]);
      mx = max_q(mx) * sl;
      if (__any(mx > M)) {
        const float mn = fmaxf(M, mx);
        const float f = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - mn);
        M = mn;
        l *= f;
        cs *= f;
#pragma unroll
        for (int j = 0; j < FT; ++j) o[j] *= f;
      }
      const float base = M == -INFINITY ? 0.f : M;
      float w[8];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          // (2^50 in the exponent would round it at 50's step: 1e-6 of every p)
          const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(z[u][r], sl, -base)) * kPScale;
          const uint32_t pr = value_pair_of(cur.pr[u], r);
          l += e;
          cs = __builtin_fmaf(e, __builtin_fmaf(7.5f, lo_f(pr), hi_f(pr)), cs);
          w[4 * u + r] = e * lo_f(pr);
        }
      ld.pairs(cur, nb);
      asm volatile("" ::: "memory");
      bf16x8 P[N];
      {
        uint32_t pw[N][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t t[N];
          terms<N>(w[2 * e], w[2 * e + 1], t);
#pragma unroll
          for (int n = 0; n < N; ++n) pw[n][e] = t[n];
        }
#pragma unroll
        for (int n = 0; n < N; ++n) P[n] = op(pw[n][0], pw[n][1], pw[n][2], pw[n][3]);
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
      ld.values(cur, nb);
#pragma unroll
      for (int jh = 0; jh < FT / 4; ++jh) {
        const uint32_t(&hf)[4] = half[jh];
        uint32_t sw[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) sw[e] = __builtin_amdgcn_perm(hf[e], hf[e], 0x02030001u);
        bf16x8 a[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          a[j] = op(value_pair(hf[0], sw[0], j), value_pair(hf[1], sw[1], j), value_pair(hf[2], sw[2], j),
                    value_pair(hf[3], sw[3], j));
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j) o[4 * jh + j] = mfma(a[j], P[n], o[4 * jh + j]);
      }
    };
    for (int blk = sg.lo + wave; blk < blk_hi; blk += 2 * W) {
      block(buf[0], blk);
      __builtin_amdgcn_sched_barrier(0);
      if (blk + W >= blk_hi) break;
      block(buf[1], blk + W);
      __builtin_amdgcn_sched_barrier(0);
    }

    // the waves' parts; lane 16 q + c holds row c, features q HD / 4 + FT r + j
    const float lt = sum_q(l), off = sum_q(cs);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < FT; j += 4)
        *(float4*)&sm.o[wave][c][q * (HD / 4) + r * FT + j] =
            make_float4(code_sum(o[j][r]) + off, code_sum(o[j + 1][r]) + off, code_sum(o[j + 2][r]) + off,
                        code_sum(o[j + 3][r]) + off);
    if (q == 0) {
      sm.m[wave][c] = M;
      sm.l[wave][c] = lt;
    }
    const bool more = !even && sg.next(p);
    if (more) request();  // (in flight while this segment is put together)
    __syncthreads();
    for (int e = tid; e < 16 * (HD / 4); e += W * 64) {
      const int row = e / (HD / 4), f = 4 * (e - row * (HD / 4)), pr = (int)tile * 16 + row;
      if (pr >= NR) continue;
      float mm = -INFINITY;
#pragma unroll
      for (int w = 0; w < W; ++w) mm = fmaxf(mm, sm.m[w][row]);
      float ll = 0.f, a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float mw = sm.m[w][row], lw = sm.l[w][row];
        // (a wave that saw nothing of this row holds zeros)
        const float s = mw == -INFINITY && lw == 0.f ? 0.f : __builtin_amdgcn_exp2f(mw - mm);
        const float4 v = *(const float4*)&sm.o[w][row][f];
        ll += lw * s;
        a[0] += v.x * s;
        a[1] += v.y * s;
        a[2] += v.z * s;
        a[3] += v.w * s;
      }
      if (all) {  // the segment is all of the head
        const bool live = pr - pr / p.R * p.R < rr.n;
        const float inv = 1.0f / ll;
#pragma unroll
        for (int k = 0; k < 4; ++k) a[k] = live ? a[k] * inv : 0.f;
        store_out(p, b, kvh, pr, f, a);
        if (f == 0 && p.w_out != nullptr) p.lse[(int64_t)bh * NR + pr] = live ? mm + log2f(ll / kPScale) : INFINITY;
      } else {
        const int64_t at = (int64_t)(range + bh) * NR + pr;
        *(float4*)(p.part_o + at * HD + f) = make_float4(a[0], a[1], a[2], a[3]);
        if (f == 0) *(float2*)(p.part_ml + at * 2) = make_float2(mm, ll);
      }
    }
    if (!more) break;
    __syncthreads();
  }
}

// Merge of a head's segments, in order.  A head that lies in one range is
// complete already (parts: there are several); rows that are not in use get their zeros here.  ROWS = 1:
// a workgroup takes one row, its GR groups of HD / 4 lanes every GR-th segment,
// and the groups are added in order (few rows of many segments); ROWS = GR: a
// row per group (many rows of a few segments: 4608 of 2, 5 us, 10 with ROWS = 1).
template <int HD, bool SPLIT>
__global__ void __launch_bounds__(256) kvq_merge_kernel(KvqAttend p) {
  constexpr int LPR = HD / 4, GR = 256 / LPR, ROWS = SPLIT ? 1 : GR;
  __shared__ float so[SPLIT ? GR : 1][HD];
  __shared__ float sm[4], sl[GR];
  const int NR = p.G * p.R, tid = threadIdx.x, f = 4 * (tid % LPR), g = tid / LPR;
  const unsigned per = (unsigned)(NR + ROWS - 1) / ROWS, bh = blockIdx.x / per;
  const int pr = (int)(blockIdx.x - bh * per) * ROWS + (SPLIT ? 0 : g);
  const int b = (int)(bh / (unsigned)p.KVH), kvh = (int)(bh - (unsigned)b * p.KVH);
  const RequestRows rr = request_rows(p, b);
  uint32_t w0, w1;  // the head's first and last range
  if (p.parts > 0) {
    w0 = bh * (unsigned)p.parts;
    w1 = w0 + p.parts - 1;
  } else {
    const uint32_t nb = request_blocks<false>(rr);
    uint32_t before;
    const Plan pl = find_request(p, tid & 63, b, &before);
    before += (uint32_t)kvh * planned_blocks(nb) + kHeadCost;
    w0 = nb > 0 ? pl.range_of(before) : 0;
    w1 = nb > 0 ? pl.range_of(before + nb - 1) : 0;
  }
  const int i = pr - pr / p.R * p.R, nc = (int)(w1 - w0) + 1;
  if (pr < NR && i >= rr.n && (!SPLIT || g == 0)) {
    const float z[4] = {0.f, 0.f, 0.f, 0.f};
    store_out(p, b, kvh, pr, f, z);
    if (f == 0 && p.w_out != nullptr) p.lse[(int64_t)bh * NR + pr] = INFINITY;
  }
  const bool mine = pr < NR && i < rr.n && nc > 1;
  if (SPLIT && !mine) return;  // (the workgroup's one row)
  const float* ml = p.part_ml + ((int64_t)(w0 + bh) * NR + (mine ? pr : 0)) * 2;
  const float* po = p.part_o + ((int64_t)(w0 + bh) * NR + (mine ? pr : 0)) * HD + f;
  float M = -INFINITY;
  if constexpr (SPLIT) {
    for (int k = tid; k < nc; k += 256) M = fmaxf(M, ml[(int64_t)k * NR * 2]);
    M = max_wave(M);
    if ((tid & 63) == 0) sm[tid >> 6] = M;
    __syncthreads();
    M = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  } else {
    if (!mine) return;
    for (int k = 0; k < nc; ++k) M = fmaxf(M, ml[(int64_t)k * NR * 2]);
  }
  float l = 0.f, a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
  for (int k = SPLIT ? g : 0; k < nc; k += SPLIT ? GR : 1) {
    const float2 v = *(const float2*)(ml + (int64_t)k * NR * 2);
    const float s = v.x == -INFINITY && v.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(v.x - M);  // (0: it sees none of them)
    const float4 o = *(const float4*)(po + (int64_t)k * NR * HD);
    l += v.y * s;
    a[0] += o.x * s;
    a[1] += o.y * s;
    a[2] += o.z * s;
    a[3] += o.w * s;
  }
  if constexpr (SPLIT) {
    *(float4*)&so[g][f] = make_float4(a[0], a[1], a[2], a[3]);
    if (f == 0) sl[g] = l;
    __syncthreads();
    if (g != 0) return;
#pragma unroll
    for (int k = 1; k < GR; ++k) {
      const float4 o = *(const float4*)&so[k][f];
      a[0] += o.x;
      a[1] += o.y;
      a[2] += o.z;
      a[3] += o.w;
      l += sl[k];
    }
  }
  const float inv = 1.0f / l;
#pragma unroll
  for (int k = 0; k < 4; ++k) a[k] *= inv;
  store_out(p, b, kvh, pr, f, a);
  if (f == 0 && p.w_out != nullptr) p.lse[(int64_t)bh * NR + pr] = M + log2f(l / kPScale);
}

// Weights: out = in + the probabilities of the first w_rows rows, summed over
// the rows and the query heads of the K/V head.  The scores are taken again
// from the keys' codes (half of the cache) now that the rows' log-sum-exp is
// known, here as S = Q K^T: lane 16 q + c gets position c of rows 4 q .. + 3, so
// a position's sum is three adds and two swaps.  A wave owns its blocks of 32
// positions: nothing is added twice and the order of the sum is fixed.  The
// cut is a plan of its own (requests without rows in use copy their weights).
// Bound by the stream of keys and weights (80 bytes a position and head: 16
// requests of 5000 to 16000 positions, 8 heads, 22 us, 5.3 TB/s).  Scores kept by
// the attention would be read instead of the keys, 16 bytes a position for 4
// query heads and one row, but need a workspace of rows x positions.
template <int HD, bool QB>
__global__ void __launch_bounds__(kWaves * 64) kvq_weights_kernel(KvqAttend p) {
  constexpr int S = HD / 32;
  const int tid = threadIdx.x, lane = tid & 63, q = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const float sl = p.scale * kLog2e / kZScale;
  Segments<true> sg;
  if (!sg.init(p, lane, blockIdx.x)) return;
  do {
    const RequestRows rr = sg.rr;
    const int b = sg.b, kvh = sg.h, keys = rr.L + rr.n;
    const int64_t bh = b * p.KVH + kvh;
    const int first = sg.lo + wave, hi = sg.hi;
    if (first >= hi) continue;
    const int nw = min(p.w_rows, rr.n), NW = p.G * nw;
    BlockLoader<HD> ld;
    ld.init(p.cache + (size_t)bh * p.head_bytes, p.head_bytes, q, c);
    const float* lse = p.lse + bh * p.G * p.R;
    struct Part {
      Block<HD> b;
      uint2 pr[2];  // key pair (and value pair) of positions 16 u + c
      float w;      // weight so far of position lane % 32 (none: 0)
    };
    Rsrc from;
    auto weights_from = [&](const float* w) {
      from = make_rsrc(w + (w != nullptr ? bh * p.max_len : 0), w != nullptr ? (uint32_t)keys * 4 : 0u);
    };
    auto request = [&](Part& x, int blk) {
      blk = blk < hi ? blk : first;
      ld.keys(x.b, blk);
      x.w = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(from, 4 * (blk * kKvqBlock + lane % kKvqBlock), 0, 0));
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const auto w = __builtin_amdgcn_raw_buffer_load_b64(ld.r, (int)kvq_pair(16 * u + c, HD),
                                                            (int)((uint32_t)blk * kvq_block_bytes(HD)), kAuxStream);
        x.pr[u] = make_uint2(w[0], w[1]);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    Part buf[2];
    weights_from(p.w_in);
    request(buf[0], first);
    request(buf[1], first + kWaves);
    // sixteen counted rows at a time; the first tile (there is one even without
    // rows) starts from w_in, the others from what the tile before stored
    for (int r0 = 0; r0 == 0 || r0 < NW; r0 += 16) {
      Queries<HD, QB> Q;
      {
        const int pr = r0 + c, g = nw > 0 ? pr / nw : 0, i = pr - g * nw;
        const bool ok = pr < NW;
        RawQuery<HD, QB> x;
        x.load(p.q, ((int64_t)b * p.R + (ok ? i : 0)) * p.q_ld + (kvh * p.G + (ok ? g : 0)) * HD, q);
        Q.convert(x, ok);
      }
      float ls[4], sq[4];
      int vis[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int pr = r0 + 4 * q + r, g = nw > 0 ? pr / nw : 0, i = pr - g * nw;
        const bool ok = pr < NW;
        ls[r] = ok ? lse[g * p.R + i] : INFINITY;
        vis[r] = ok ? rr.L + i + 1 : 0;
        sq[r] = __shfl(Q.sum, 4 * q + r);
      }
      auto block = [&](Part& cur, int blk) {
        floatx4 acc[2] = {};
#pragma unroll
        for (int n = Queries<HD, QB>::N - 1; n >= 0; --n)  // (as in the attention)
#pragma unroll
          for (int s = 0; s < S; ++s)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const uint32_t w = cur.b.k[u][s];
              acc[u] = mfma(op(Q.w[n][s][0], Q.w[n][s][1], Q.w[n][s][2], Q.w[n][s][3]),
                            op(code_pair(w, 0), code_pair(w, 1), code_pair(w, 2), code_pair(w, 3)), acc[u]);
            }
        const float s[2] = {lo_f(cur.pr[0].x), lo_f(cur.pr[1].x)}, m[2] = {hi_f(cur.pr[0].x), hi_f(cur.pr[1].x)};
        const float before = cur.w;
        request(cur, blk + 2 * kWaves);
        float t[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          t[u] = 0.f;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float z = __builtin_fmaf(s[u], acc[u][r], m[u] * sq[r]);
            const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(z, sl, -ls[r]));
            t[u] += blk * kKvqBlock + 16 * u + c < vis[r] ? e : 0.f;
          }
          t[u] = sum_q(t[u]);
        }
        // lanes 0 .. 31 store the block's positions
        const int pos = blk * kKvqBlock + lane;
        if (lane < kKvqBlock && pos < keys) {
          const int64_t at = bh * p.max_len + pos;
          p.w_out[at] = before + (q == 0 ? t[0] : t[1]);
        }
      };
      for (int blk = first; blk < hi; blk += 2 * kWaves) {
        block(buf[0], blk);
        if (blk + kWaves >= hi) break;
        block(buf[1], blk + kWaves);
      }
      if (r0 + 16 < NW) {
        weights_from(p.w_out);
        request(buf[0], first);
        request(buf[1], first + kWaves);
      }
    }
  } while (sg.next(p));
}

// ---------------------------------------------------------------------------
// Eviction.
//
// kvq_select_kernel, a workgroup per (layer, request, K/V head): of n cached
// positions the last `recent` stay, and of the others the budget - recent
// heaviest, ties to the lower position.  The weight that decides is found by
// four passes over 8 bits of an order-preserving key, then one pass takes the
// positions in order.  A workgroup reads its weights five times, from the second
// on from L2 (4 layers of 16 requests of 900 to 12000 positions, 8 heads: 31 us).
// ---------------------------------------------------------------------------
constexpr int kSelThreads = 1024;
constexpr int kSelAhead = 4;  // weights a thread requests at once
constexpr int kSelRun = 4;    // positions in a row per thread of the last pass

// larger key: heavier (NaN above everything, -0 as 0)
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0xffffffffu;
  uint32_t u = __float_as_uint(w);
  if (u == 0x80000000u) u = 0;
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__global__ void __launch_bounds__(kSelThreads) kvq_select_kernel(KvqEvict p) {
  __shared__ uint32_t hist[4][256];  // (lanes 4 apart count apart: equal weights meet less often)
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
  if (p.evicted != nullptr && l == 0 && h == 0 && tid == 0) p.evicted[b] += n - p.budget;
  const int cand = n - p.recent;
  uint32_t need = (uint32_t)(p.budget - p.recent), prefix = 0, mask = 0;
  if (need > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      ((uint32_t*)hist)[tid] = 0;
      __syncthreads();
      for (int j0 = 0; j0 < cand; j0 += kSelThreads * kSelAhead) {
        float v[kSelAhead];
#pragma unroll
        for (int u = 0; u < kSelAhead; ++u) {
          const int j = j0 + u * kSelThreads + tid;
          v[u] = j < cand ? w[j] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < kSelAhead; ++u) {
          const uint32_t k = weight_key(v[u]);
          if (j0 + u * kSelThreads + tid < cand && (k & mask) == prefix) atomicAdd(&hist[tid & 3][(k >> shift) & 255], 1u);
        }
      }
      __syncthreads();
      if (wave == 0) {
        // from the heaviest bin down, the one that holds the last kept position:
        // lane i has bins 255 - 4 i .. 252 - 4 i
        uint32_t n[4], t = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int d = 255 - 4 * lane - k;
          n[k] = hist[0][d] + hist[1][d] + hist[2][d] + hist[3][d];
          t += n[k];
        }
        uint32_t above = t;  // inclusive prefix over the lanes
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const uint32_t v = __shfl_up(above, o);
          if (lane >= o) above += v;
        }
        above -= t;
        if (above < need && need <= above + t) {
          uint32_t left = need - above;
          int k = 0;
          while (k < 3 && n[k] < left) left -= n[k++];
          s_prefix = prefix | ((uint32_t)(255 - 4 * lane - k) << shift);
          s_need = left;
        }
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
  // (a thread has kSelRun positions in a row; a position's place counts those
  // before it: other rounds', other waves', lower lanes', the lane's own)
  uint32_t base_k = 0, base_e = 0;
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  for (int j0 = 0; j0 < n; j0 += kSelThreads * kSelRun) {
    const int j = j0 + tid * kSelRun;
    float v[kSelRun];
#pragma unroll
    for (int u = 0; u < kSelRun; ++u) v[u] = j + u < n ? w[j + u] : 0.f;
    bool gt[kSelRun], eq[kSelRun];
    uint32_t e_at = base_e, e_wave = 0, at = base_k, k_wave = 0;
#pragma unroll
    for (int u = 0; u < kSelRun; ++u) {
      const uint32_t k = weight_key(v[u]);
      gt[u] = j + u < n && (j + u >= cand || k > prefix);
      eq[u] = j + u < cand && k == prefix;
      const uint64_t m = __ballot(eq[u]);
      e_at += (uint32_t)__popcll(m & below);
      e_wave += (uint32_t)__popcll(m);
    }
    if (lane == 0) wsum[0][wave] = e_wave;
    __syncthreads();
    uint32_t all = 0;
#pragma unroll
    for (int k = 0; k < kSelThreads / 64; ++k) {
      const uint32_t c = wsum[0][k];
      if (k < wave) e_at += c;
      all += c;
    }
    base_e += all;
    bool take[kSelRun];
#pragma unroll
    for (int u = 0; u < kSelRun; ++u) {
      take[u] = gt[u] || (eq[u] && e_at < need);
      e_at += eq[u] ? 1 : 0;
      const uint64_t m = __ballot(take[u]);
      at += (uint32_t)__popcll(m & below);
      k_wave += (uint32_t)__popcll(m);
    }
    if (lane == 0) wsum[1][wave] = k_wave;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int k = 0; k < kSelThreads / 64; ++k) {
      const uint32_t c = wsum[1][k];
      if (k < wave) at += c;
      all += c;
    }
    base_k += all;
#pragma unroll
    for (int u = 0; u < kSelRun; ++u)
      if (take[u]) {  // (at <= j + u, and every weight up to the round's end has been read: in place is fine)
        kept[at] = j + u;
        if (wo != nullptr) wo[at] = v[u];
        ++at;
      }
  }
}

// kvq_move_kernel: kept position j of the source becomes position j.  Grid
// ((layer, request, K/V head), part, column).  Column 0 is the keys' codes, a
// thread a 16-byte piece of a position; column 1 the values', a thread the
// piece of four positions and eight features (from four places); column 2 the
// pairs.  In place one workgroup goes through its column in order: a row moves
// to a lower or the same position, and a round reads all of its rows before it
// writes the first.  2048 kept positions of the 512 heads above: 142 MB out and at
// least as many in, 94 us, 3.0 TB/s (a value piece holds four positions, so
// scattered ones bring their neighbours along).
constexpr int kMoveThreads = 512;

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
  constexpr int KP = HD / 32, VP = HD / 8;  // pieces of a position's keys, of four positions' values
  // positions of a round
  const int per = col == 0 ? kMoveThreads / KP : col == 1 ? kMoveThreads / VP * 4 : kMoveThreads;
  for (int j0 = (int)blockIdx.y * per; j0 < m; j0 += (int)gridDim.y * per) {
    uint4 v = make_uint4(0, 0, 0, 0);
    int j, n = 0;  // first position and count of the thread's positions
    uint8_t* to;
    if (col == 0) {
      j = j0 + tid / KP;
      n = j < m;
      to = dst + (size_t)(j / kKvqBlock) * bb + kvq_k_word(j % kKvqBlock, 4 * (tid % KP), HD);
      if (n) {
        const int t = kept[j];
        v = *(const uint4*)(src + (size_t)(t / kKvqBlock) * bb + kvq_k_word(t % kKvqBlock, 4 * (tid % KP), HD));
      }
    } else if (col == 1) {
      j = j0 + tid / VP * 4;
      n = max(0, min(m - j, 4));
      to = dst + (size_t)(j / kKvqBlock) * bb + kvq_v_word(j % kKvqBlock, tid % VP, HD);
      uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < n) {
          const int t = kept[j + k];
          w[k] = *(const uint32_t*)(src + (size_t)(t / kKvqBlock) * bb + kvq_v_word(t % kKvqBlock, tid % VP, HD));
        }
      v = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      j = j0 + tid;
      n = j < m;
      to = dst + (size_t)(j / kKvqBlock) * bb + kvq_pair(j % kKvqBlock, HD);
      if (n) {
        const int t = kept[j];
        const uint2 w = *(const uint2*)(src + (size_t)(t / kKvqBlock) * bb + kvq_pair(t % kKvqBlock, HD));
        v.x = w.x;
        v.y = w.y;
      }
    }
    if (in_place) __syncthreads();
    if (col == 2) {
      if (n) *(uint2*)to = make_uint2(v.x, v.y);
    } else if (col == 1 && n < 4) {  // positions behind the last stay as they were
      uint32_t* o = (uint32_t*)to;
      if (n > 0) o[0] = v.x;
      if (n > 1) o[1] = v.y;
      if (n > 2) o[2] = v.z;
    } else if (n) {
      *(uint4*)to = v;
    }
    if (in_place) __syncthreads();
  }
  if (col == 2 && blockIdx.y == 0 && l == 0 && h == 0 && tid == 0) p.lens_out[b] = m;
}

__global__ void kvq_restart_kernel(int B, const int32_t* lens, int32_t* evicted) {
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b < B && lens[b] == 0) evicted[b] = 0;
}

__global__ void kvq_prefill_rows_kernel(int b0, int nb, int R, const int32_t* n_cache, const int32_t* base,
                                        const int32_t* lens, int32_t* rows) {
  const int b = b0 + blockIdx.x * blockDim.x + threadIdx.x;
  if (b < b0 + nb) rows[b] = max(0, min(n_cache[b] - (lens[b] - base[b]), R));
}

// Row groups of a wave of the append, where there are waves enough (as many as
// the compute units hold): what a wave does once, some 170 instructions, is half
// of a group's work (2048 rows of 96 heads: 24 to 25 us, 26 with one).
constexpr int kAppendWaves = 8192, kAppendRun = 4;

template <int HD, bool BF16>
hipError_t append_t(KvqAppend a, hipStream_t st) {
  constexpr int kWaveRows = 64 / (HD / 8);
  const int heads = (a.q.p != nullptr ? a.H : 0) + 2 * a.KVH, rows = a.R > kWaveRows / 2 ? kWaveRows : 1;
  const int per = 256 / (HD / 8) / rows, gy = (heads + per - 1) / per;
  if (gy > 65535) return hipErrorInvalidValue;
  const int64_t groups = (int64_t)a.B * ((a.R + rows - 1) / rows), waves = groups * gy * 4;
  a.run = (int)std::min<int64_t>(std::max<int64_t>(waves / kAppendWaves, 1), kAppendRun);
  const dim3 g((unsigned)(a.B * ((a.R + rows * a.run - 1) / (rows * a.run))), (unsigned)gy);
  if (rows > 1) hipLaunchKernelGGL((kvq_append_kernel<HD, BF16, kWaveRows>), g, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((kvq_append_kernel<HD, BF16, 1>), g, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kvq_append(const KvqAppend& a, hipStream_t st) {
  if (a.hd == 128) return a.bf16 ? append_t<128, true>(a, st) : append_t<128, false>(a, st);
  return a.bf16 ? append_t<64, true>(a, st) : append_t<64, false>(a, st);
}

namespace {

template <int HD, bool BF16>
hipError_t read_t(const KvqRead& a, hipStream_t st) {
  constexpr int kWaveRows = 64 / (HD / 8);
  const int rows = a.R > kWaveRows / 2 ? kWaveRows : 1, per = 256 / (HD / 8) / rows, gy = (a.KVH + per - 1) / per;
  if (gy > 65535) return hipErrorInvalidValue;
  const dim3 g((unsigned)(a.B * ((a.R + rows - 1) / rows)), (unsigned)gy);
  if (rows > 1) hipLaunchKernelGGL((kvq_read_kernel<HD, BF16, kWaveRows>), g, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((kvq_read_kernel<HD, BF16, 1>), g, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kvq_read(const KvqRead& a, hipStream_t st) {
  if (a.hd == 128) return a.bf16 ? read_t<128, true>(a, st) : read_t<128, false>(a, st);
  return a.bf16 ? read_t<64, true>(a, st) : read_t<64, false>(a, st);
}

namespace {

// Workgroups of the attention's ranges: two per compute unit (what their
// registers allow) over all row tiles, one round; fewer where that left less
// than two blocks per wave.  A workgroup costs about 5 us before and after its
// stream, so one round of long ranges beats several of short ones, and ranges of
// equal size beat chunks of equal length where the requests' lengths differ (one
// bf16 token, 8 K/V heads, 16 requests of 5000 to 16000 positions: 35 us, 40 to
// 75 with chunks of 2048 to 256 keys).  Equal parts of every head never straddle
// two heads and need no plan: they are taken for a single request, and where
// parts of two blocks per wave all fit the round (6 float32 rows over 1024
// positions, 32 heads: 7.3 us and 3.8 for the merge, 8.2 and 4.7 as ranges).  One
// part per head (up to 256 keys) needs no merge (250 positions: 5.8 us, 6.5 and
// 3.8 as ranges).
//
// Workgroups of eight waves take whole heads where every compute unit gets one
// at most and the heads are short for their number: it is the merge and its
// launch against fewer workgroups.  While parts of two blocks per wave leave a
// workgroup per compute unit, that pays up to 20 blocks of keys (28 for bfloat16),
// where they do not, longer.  Row tiles, blocks, us with whole heads / without: 32
// float32 tiles, 20 blocks 8.9 / 9.6, 22 9.8 / 9.5; 64, 20 9.1 / 9.8, 24 10.1 / 9.8;
// 80, 24 10.1 / 10.0, 28 10.7 / 12.3, 40 13.1 / 12.6; 96, 36 12.3 / 12.9, 64 17.7 /
// 17.7; 128, 48 14.8 / 18.0, 80 20.8 / 21.2; 256, 96 25.4 / 32.5; bfloat16, 8 tiles,
// 28 blocks 8.2 / 8.4, 32 9.0 / 8.5; 64, 28 8.7 / 9.0, 32 9.5 / 9.0; 96, 36 10.1 /
// 11.2; 128, 48 12.1 / 15.5, 96 19.3 / 20.1; 256, 96 22.5 / 28.4.  The bound for many
// tiles stays below what pays for equal lengths, since a long request among short
// ones holds its workgroup alone.
//
// What bounds it: long caches the stream (bf16 calls: 120 thousand positions, 130
// MB, 26.7 us, 4.9 TB/s; the 16 requests above 38 us, 5.2 TB/s; a plain copy of 512
// MB reaches 5.3); float32 calls the vector instructions beside it (three terms: 43
// us for the 120 thousand positions, and of 16 requests of 256 to 4096 positions, 9
// rows, 4 query heads a K/V head, 30 us, with vector issue in 0.58 and the matrix
// units busy in 0.25 of the cycles); a short request the launch and four dependent
// round trips to memory.
constexpr int kAttendWgs = 512;
constexpr int kWeightWgs = 1024;

int64_t attend_blocks(const KvqAttend& a) {
  return (int64_t)a.B * a.KVH * ((a.max_keys + kKvqBlock - 1) / kKvqBlock + kHeadCost);
}

template <int HD>
hipError_t attend_hd(KvqAttend a, hipStream_t st) {
  const int64_t heads = (int64_t)a.B * a.KVH, rows = heads * a.G * a.R;
  a.TG = (a.G * a.R + 15) / 16;
  const int blocks = (a.max_keys + kKvqBlock - 1) / kKvqBlock;
  const int64_t fill = (attend_blocks(a) + 2 * kWaves - 1) / (2 * kWaves);
  // (whole rounds of the eight XCDs)
  int64_t wgs = std::min<int64_t>(fill, std::max(8, kAttendWgs / 8 / a.TG * 8));
  const int64_t pieces = (blocks + 2 * kWaves - 1) / (2 * kWaves), fit = kAttendWgs / a.TG / heads;
  a.parts = a.B == 1 || pieces <= std::max<int64_t>(fit, 1) ? (int)std::max<int64_t>(1, std::min(pieces, fit)) : 0;
  if (a.parts > 0) wgs = heads * a.parts;
  const int64_t tiles = heads * a.TG;
  const int64_t most = std::max<int64_t>(a.bf16 ? 28 : 20, tiles * pieces > kAttendWgs / 2 ? tiles * 3 / 8 : 0);
  const bool whole = tiles <= kAttendWgs / 2 && blocks > 2 * kWaves && blocks <= most;
  if (whole) {
    a.parts = 1;
    wgs = heads;
  }
  a.WG = (int)wgs;
  const int64_t grid = 8 * a.TG * ((wgs + 7) / 8);
  if (grid > 0x7fffffff || rows > 0x7fffffff || attend_blocks(a) > 0x7fffffff) return hipErrorInvalidValue;
  if (a.parts != 1 && (heads + wgs) * a.G * a.R > (int64_t)a.part_rows) return hipErrorInvalidValue;
  auto launch = [&](auto kernel, int waves) { hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(waves * 64), 0, st, a); };
  constexpr int W = kWaves, W2 = 2 * kWaves;
  if (whole) launch(a.bf16 ? kvq_attend_kernel<HD, true, W2> : kvq_attend_kernel<HD, false, W2>, W2);
  else launch(a.bf16 ? kvq_attend_kernel<HD, true, W> : kvq_attend_kernel<HD, false, W>, W);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.parts != 1) {
    // about wgs / heads segments per head
    constexpr int kRows = 256 / (HD / 4);
    if (wgs >= 4 * heads) hipLaunchKernelGGL((kvq_merge_kernel<HD, true>), dim3((unsigned)rows), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((kvq_merge_kernel<HD, false>), dim3((unsigned)(heads * ((a.G * a.R + kRows - 1) / kRows))), dim3(256), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.w_out != nullptr) {
    a.WG = (int)std::min<int64_t>(fill, kWeightWgs);
    if (a.bf16) hipLaunchKernelGGL((kvq_weights_kernel<HD, true>), dim3((unsigned)a.WG), dim3(kWaves * 64), 0, st, a);
    else hipLaunchKernelGGL((kvq_weights_kernel<HD, false>), dim3((unsigned)a.WG), dim3(kWaves * 64), 0, st, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

// (grows with every argument, so a workspace for the largest call holds any)
size_t kvq_attend_floats(int B, int H, int KVH, int hd, int R, size_t* part_ml, size_t* lse) {
  const size_t rows = (size_t)B * H * R, TG = ((size_t)(H / KVH) * R + 15) / 16;
  const size_t parts = rows + std::max<size_t>(16 * kAttendWgs, 8 * 16 * TG);
  *part_ml = parts * 2;
  *lse = rows;
  return parts * hd;
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
  const dim3 g((unsigned)heads, in_place ? 1u : (unsigned)std::min((a.budget + 127) / 128, 64), 3);
  if (a.hd == 128) hipLaunchKernelGGL((kvq_move_kernel<128>), g, dim3(kMoveThreads), 0, st, a, in_place);
  else hipLaunchKernelGGL((kvq_move_kernel<64>), g, dim3(kMoveThreads), 0, st, a, in_place);
  return hipGetLastError();
}

hipError_t launch_kvq_restart(int B, const int32_t* lens, int32_t* evicted, hipStream_t st) {
  hipLaunchKernelGGL(kvq_restart_kernel, dim3((B + 63) / 64), dim3(64), 0, st, B, lens, evicted);
  return hipGetLastError();
}

hipError_t launch_kvq_prefill_rows(int b0, int nb, int R, const int32_t* n_cache, const int32_t* base,
                                   const int32_t* lens, int32_t* rows, hipStream_t st) {
  hipLaunchKernelGGL(kvq_prefill_rows_kernel, dim3((nb + 63) / 64), dim3(64), 0, st, b0, nb, R, n_cache, base, lens, rows);
  return hipGetLastError();
}

}  // namespace spade
