// Filtered sampling: a token per row of logits.
//
// Tokens of a row are ordered by logit, equal ones by id.  With d = (max - l) / T
// and weights w = exp(-d) in 64 bits a token is kept if d <= 32, it is among the
// first top_k of those, the weight before it is below top_p of theirs, and w >=
// min_p; the token is the largest of -d + G over the kept ones, G the Gumbel noise
// of the acceptance step (SplitMix64 of the uniform's bits).  All filters keep the
// beginning of the order, so a row's result is one border (logit, id).
//
//   sample_slice_kernel   a slice's maximum, and its tokens' counts and weights by
//                         bins of their logit over T
//   sample_scan_kernel    the row's bins: which hold the border; tokens above them
//                         draw, theirs are listed
//   sample_finish_kernel  the border among the listed tokens, the draw
//   sample_probs_kernel   the distribution, where asked
#include "sample.h"

#include <float.h>

#include <algorithm>

#include "device_accept.h"

namespace spade {

namespace {

constexpr int kThreads = 256;
constexpr double kSpan = 32.0;                       // of d: weights from e^-32 on
constexpr double kBinsPerUnit = 126.0 / kSpan, kBin = kSpan / 126.0;
constexpr int kSteps = 256;                          // of the table of a bin's weights
constexpr double kSlack = 0x1p-40;                   // of top_p: equal masses count as reached

struct Request {
  double inv_T, top_p, min_d;  // min_d: largest d that min_p allows
  int top_k;
  bool greedy, use_k, use_p;
  __device__ __forceinline__ bool listed() const { return use_k || use_p; }
};

__device__ __forceinline__ Request request_of(const SampleArgs& a, int row) {
  const int r = row / a.per;
  Request q;
  const float T = a.d_temperature != nullptr ? a.d_temperature[r] : a.temperature;
  const float p = a.d_top_p != nullptr ? a.d_top_p[r] : a.top_p;
  const float m = a.d_min_p != nullptr ? a.d_min_p[r] : a.min_p;
  q.top_k = a.d_top_k != nullptr ? a.d_top_k[r] : a.top_k;
  q.greedy = !(T > 0.f);
  q.inv_T = q.greedy ? 0.0 : 1.0 / (double)T;
  q.use_k = !q.greedy && q.top_k > 0 && q.top_k < a.V;
  q.use_p = !q.greedy && p < 1.f;
  q.top_p = (double)p;
  q.min_d = m > 0.f ? -log((double)fminf(m, 1.f)) : kSpan;
  if (!(q.min_d < kSpan)) q.min_d = kSpan;
  return q;
}

// 1 / T of a row whose largest logit is m, held to |m| / T <= 2^34: there two
// different logits are 512 apart, so nothing changes.
__device__ __forceinline__ double row_inv_T(double inv_T, float m) {
  const double most = 0x1p34 / fmax(fabs((double)m), 0x1p-140);
  return fmin(inv_T, most);
}

// Bins of l / T on a grid that all slices share, and their upper edges.
__device__ __forceinline__ double bin_of(float l, double inv_T) { return floor((double)l * inv_T * kBinsPerUnit); }
__device__ __forceinline__ double edge_of(double bin) { return (bin + 1.0) * kBin; }

// exp(x) for x in a bin below its edge: a table's step and a short series of the
// rest (|r| < 0.001: 2^-34 of the value; float32's exponential would leave the
// border of a fine distribution to its rounding).
__device__ __forceinline__ double bin_weight(const double* table, double x) {
  constexpr float scale = (float)(kSteps / kBin);
  const int i = min(max((int)((float)x * -scale), 0), kSteps - 1);
  const float r = (float)__builtin_fma((double)i, kBin / kSteps, x);
  const float e = r * __builtin_fmaf(r, __builtin_fmaf(r, 1.f / 6.f, 0.5f), 1.f);
  const double t = table[i];
  return __builtin_fma(t, (double)e, t);
}
__device__ __forceinline__ void fill_table(double* table, int tid) {
  static_assert(kSteps == kThreads, "a step per thread");
  table[tid] = exp(-(double)tid * (kBin / kSteps));
}

// w 2^n as an integer, w 2^n < 2^51
template <int N>
__device__ __forceinline__ uint64_t fixed(double w) {
  return (uint64_t)__double_as_longlong(__builtin_fma(w, (double)(1ull << N), 0x1p52)) & 0xfffffffffffffull;
}
constexpr int kMassBits = 38;  // of a slice's bins: 4096 weights up to 1 below the count at bit 51

// Order-preserving integer of a float.
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t b = __float_as_uint(l + 0.f);  // (-0 is 0)
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// The thread's 16 tokens of a slice: NaN (flagged) and tokens past the end as -inf,
// infinity as the largest number.
template <bool BF16>
__device__ __forceinline__ int token_of(int base, int tid, int k) {
  return BF16 ? base + ((k >> 3) * kThreads + tid) * 8 + (k & 7) : base + ((k >> 2) * kThreads + tid) * 4 + (k & 3);
}
template <bool BF16>
__device__ __forceinline__ bool load16(const SampleArgs& a, int row, int base, int tid, float (&x)[16]) {
  const int64_t at = (int64_t)row * a.ld;
  if constexpr (BF16) {
    const uint16_t* p = (const uint16_t*)a.logits + at;
    const bool vec = ((uintptr_t)p & 15) == 0;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int v = token_of<true>(base, tid, 8 * j);
      if (vec && v + 8 <= a.V) {
        const uint4 w = *(const uint4*)(p + v);
        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[8 * j + 2 * i] = __uint_as_float(ww[i] << 16);
          x[8 * j + 2 * i + 1] = __uint_as_float(ww[i] & 0xffff0000u);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[8 * j + i] = v + i < a.V ? bf2f(p[v + i]) : -INFINITY;
      }
    }
  } else {
    const float* p = (const float*)a.logits + at;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int v = token_of<false>(base, tid, 4 * j);
      if (v + 4 <= a.V) {
        const Float4u w = *(const Float4u*)(p + v);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * j + i] = w.v[i];
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * j + i] = v + i < a.V ? p[v + i] : -INFINITY;
      }
    }
  }
  bool nan = false;
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    nan |= x[k] != x[k];
    x[k] = x[k] != x[k] ? -INFINITY : fminf(x[k], FLT_MAX);
  }
  return nan;
}
template <bool BF16>
__device__ __forceinline__ float load1(const SampleArgs& a, int row, int v) {
  const int64_t at = (int64_t)row * a.ld + v;
  const float x = BF16 ? bf2f(((const uint16_t*)a.logits)[at]) : ((const float*)a.logits)[at];
  return x != x ? -INFINITY : fminf(x, FLT_MAX);
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = min(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

struct Draw {
  double s;
  int id;
};
__device__ __forceinline__ Draw better_draw(Draw x, Draw y) { return y.s > x.s || (y.s == x.s && y.id < x.id) ? y : x; }
__device__ __forceinline__ Draw wave_draw(Draw v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = better_draw(v, Draw{__shfl_xor(v.s, o), __shfl_xor(v.id, o)});
  return v;
}

// Token `id` at distance d takes part in the draw.  It wins with U above
// exp(-exp(-(best + d))) only, so 1 - U below exp(-(best + d)): most tokens end
// there, without a logarithm, and those that no noise could lift (1 - U is at
// least 2^-24) without their hash.
__device__ __forceinline__ void draw(Draw& best, float& bestf, uint64_t seed, int id, double d) {
  const float t = __builtin_amdgcn_exp2f(-(bestf + (float)d) * 1.44269504f) * 1.001f;
  if (t < 0x1p-24f) return;
  const uint32_t x = (uint32_t)(splitmix64_at(seed, (uint64_t)id) >> 41);
  if (((float)(0x7fffffu - x) + 0.5f) * 0x1p-23f > t) return;
  const double U = ((double)x + 0.5) * 0x1p-23;
  const Draw n{-log(-log(U)) - d, id};
  best = better_draw(best, n);
  bestf = (float)best.s;
}

// ---------------------------------------------------------------------------
template <bool BF16>
__global__ void __launch_bounds__(kThreads) sample_slice_kernel(SampleArgs a) {
  __shared__ float wm[4];
  __shared__ int wi[4];
  __shared__ double table[kSteps];
  __shared__ uint64_t bins[kSampleBins];
  const int row = blockIdx.x / a.NS, s = blockIdx.x - row * a.NS, tid = threadIdx.x, wave = tid >> 6;
  const Request q = request_of(a, row);
  float x[16];
  const bool nan = load16<BF16>(a, row, s * kSampleSlice, tid, x);
  if (nan) flag_error(a.err, SPADE_DERR_NAN);
  if (q.listed()) {
    fill_table(table, tid);
    if (tid < kSampleBins) bins[tid] = 0;
  }
  float m = x[0];
#pragma unroll
  for (int k = 1; k < 16; ++k) m = fmaxf(m, x[k]);
  m = wave_max(m);
  if ((tid & 63) == 0) wm[wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(wm[0], wm[1]), fmaxf(wm[2], wm[3]));
  const int64_t at = (int64_t)row * a.NS + s;
  if (tid == 0) {
    a.smax[at] = m;
    if (s == 0) a.count[row] = 0;
  }
  if (q.greedy) {
    int id = 0x7fffffff;
#pragma unroll
    for (int k = 15; k >= 0; --k)
      if (x[k] == m) id = min(id, token_of<BF16>(s * kSampleSlice, tid, k));
    id = wave_min(id);
    if ((tid & 63) == 0) wi[wave] = id;
    __syncthreads();
    if (tid == 0) a.sarg[at] = min(min(wi[0], wi[1]), min(wi[2], wi[3]));
    return;
  }
  if (!q.listed()) return;
  const double inv_T = row_inv_T(q.inv_T, m), top = bin_of(m, inv_T);
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const double bin = bin_of(x[k], inv_T), j = top - bin;
    if (x[k] > -INFINITY && j < (double)kSampleBins) {
      const double w = bin_weight(table, __builtin_fma((double)x[k], inv_T, -edge_of(bin)));
      atomicAdd((unsigned long long*)&bins[(int)j], (unsigned long long)(fixed<kMassBits>(w) | 1ull << 51));
    }
  }
  __syncthreads();
  if (tid < kSampleBins) a.hist[at * kSampleBins + tid] = bins[tid];
}

// ---------------------------------------------------------------------------
// Inclusive prefix of two values per lane over 128 bins.
struct ScanSmem {
  double table[kSteps];
  double factor[kSampleBins];  // weight of a bin's edge over the largest weight
  uint64_t mass[2][kSampleBins];
  uint32_t cnt[2][kSampleBins];
  int off[256];  // bins between a slice's top and the row's (1000: out of reach)
  float wm[4];
  double ws[4];
  Draw wd[4];
  SampleRow row;
};

template <bool BF16>
__global__ void __launch_bounds__(kThreads) sample_scan_kernel(SampleArgs a) {
  __shared__ ScanSmem sm;
  const int row = blockIdx.x / a.NW, part = blockIdx.x - row * a.NW, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Request q = request_of(a, row);
  if (q.greedy) return;
  const float ms = tid < a.NS ? a.smax[(int64_t)row * a.NS + tid] : -INFINITY;  // (at most 256 slices)
  const float m0 = wave_max(ms);
  if (lane == 0) sm.wm[wave] = m0;
  fill_table(sm.table, tid);
  __syncthreads();
  const float M = fmaxf(fmaxf(sm.wm[0], sm.wm[1]), fmaxf(sm.wm[2], sm.wm[3]));
  if (M == -INFINITY) return;
  const double inv_T = row_inv_T(q.inv_T, M), top = bin_of(M, inv_T);
  {
    const double d = ((double)M - (double)ms) * inv_T;
    sm.off[tid] = ms > -INFINITY && d <= kSpan ? (int)(top - bin_of(ms, inv_T)) : 1000;
    if (tid < kSampleBins) sm.factor[tid] = exp(__builtin_fma(-(double)M, inv_T, edge_of(top - tid)));
  }
  __syncthreads();
  int lo = kSampleBins, hi = kSampleBins;
  if (q.listed()) {
    const int j = tid & (kSampleBins - 1), half = tid / kSampleBins;
    uint64_t mass = 0;
    uint32_t cnt = 0;
    const uint64_t* h = a.hist + (int64_t)row * a.NS * kSampleBins;
#pragma unroll 4
    for (int s = half; s < a.NS; s += 2) {
      const int jj = j - sm.off[s];
      const uint64_t w = jj >= 0 ? h[s * kSampleBins + jj] : 0ull;
      mass += w & 0x7ffffffffffffull;
      cnt += (uint32_t)(w >> 51);
    }
    sm.mass[half][j] = mass;
    sm.cnt[half][j] = cnt;
    __syncthreads();
    if (wave == 0) {
      double w[2], wi[2];
      int c[2], ci[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int b = 2 * lane + e;
        w[e] = (double)(sm.mass[0][b] + sm.mass[1][b]) * 0x1p-38 * sm.factor[b];
        c[e] = (int)(sm.cnt[0][b] + sm.cnt[1][b]);
      }
      double sw = w[0] + w[1];
      int sc = c[0] + c[1];
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double tw = __shfl_up(sw, o);
        const int tc = __shfl_up(sc, o);
        if (lane >= o) {
          sw += tw;
          sc += tc;
        }
      }
      wi[1] = sw;
      wi[0] = sw - w[1];
      ci[1] = sc;
      ci[0] = sc - c[1];
      const double total = __shfl(sw, 63);
      // the first bin with f, and the counts and weights before it
      auto first = [&](bool f0, bool f1) {
        const uint64_t hit = __ballot(f0 || f1);
        if (hit == 0) return kSampleBins - 1;
        const int l = __ffsll((unsigned long long)hit) - 1;
        return 2 * l + (__shfl((int)f0, l) ? 0 : 1);
      };
      int k_bin = kSampleBins - 1, k_in = 0;
      double least = total, most = total;  // of the weight that top_p refers to
      if (q.use_k && __shfl(ci[1], 63) > q.top_k) {  // (else all are among the first top_k)
        k_in = 1;
        k_bin = first(ci[0] >= q.top_k, ci[1] >= q.top_k);
        const double in = __shfl(k_bin & 1 ? wi[1] : wi[0], k_bin >> 1);
        most = in;
        least = in - __shfl(k_bin & 1 ? w[1] : w[0], k_bin >> 1);
      }
      lo = hi = k_bin;
      if (q.use_p) {
        // (a little more on either side, so that rounding cannot move the border out)
        const double t0 = (q.top_p - 0x1p-30) * least, t1 = (q.top_p + 0x1p-30) * most;
        lo = min(lo, first(wi[0] >= t0, wi[1] >= t0));
        hi = min(hi, first(wi[0] >= t1, wi[1] >= t1));
        if (k_in) hi = k_bin;  // the first top_k tokens' weight ends there
      }
      const double in = __shfl(lo & 1 ? wi[1] : wi[0], lo >> 1), ex = in - __shfl(lo & 1 ? w[1] : w[0], lo >> 1);
      const int above = __shfl(lo & 1 ? ci[1] : ci[0], lo >> 1) - __shfl(lo & 1 ? c[1] : c[0], lo >> 1);
      if (lane == 0) {
        sm.row.mass = lo == 0 ? 0.0 : ex;
        sm.row.total = total;
        sm.row.lo = lo;
        sm.row.hi = hi;
        sm.row.above = above;
        sm.row.k_in = k_in;
      }
    }
    __syncthreads();
    lo = sm.row.lo;
    hi = sm.row.hi;
  }
  if (part == 0 && tid == 0) {
    SampleRow r = sm.row;
    if (!q.listed()) {
      r.mass = r.total = 0.0;
      r.lo = r.hi = kSampleBins;
      r.above = r.k_in = 0;
    }
    r.max = M;
    r.inv_T = inv_T;
    a.row[row] = r;
  }
  const uint64_t seed = (uint64_t)__float_as_uint(a.u[row]);
  Draw best{-INFINITY, 0x7fffffff};
  float bestf = -INFINITY;
  double sum = 0.0;
  const int s1 = min(a.NS, (part + 1) * a.spw);
  for (int s = part * a.spw; s < s1; ++s) {
    if (sm.off[s] > min(hi, kSampleBins - 1)) continue;
    float x[16];
    load16<BF16>(a, row, s * kSampleSlice, tid, x);
    uint32_t listed = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const double d = ((double)M - (double)x[k]) * inv_T;
      if (!(x[k] > -INFINITY && d <= kSpan)) continue;
      const double bin = bin_of(x[k], inv_T);
      const int j = min((int)(top - bin), kSampleBins - 1);
      if (j > hi) continue;
      if (j >= lo) {
        listed |= 1u << k;
      } else if (d <= q.min_d) {
        sum += bin_weight(sm.table, __builtin_fma((double)x[k], inv_T, -edge_of(bin))) * sm.factor[j];
        draw(best, bestf, seed, token_of<BF16>(s * kSampleSlice, tid, k), d);
      }
    }
    bestf = wave_max(bestf);  // (a bound for the other lanes' tokens, not their best)
    if (__any(listed != 0)) {
      const int n = __popc(listed);
      int in = n;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_up(in, o);
        if (lane >= o) in += t;
      }
      uint32_t at = 0;
      if (lane == 63) at = atomicAdd(a.count + row, (uint32_t)in);
      at = (uint32_t)__shfl((int)at, 63) + (uint32_t)(in - n);
#pragma unroll
      for (int k = 0; k < 16; ++k)
        if (listed >> k & 1u) {
          if (at < kSampleList)
            a.list[(int64_t)row * kSampleList + at] = make_uint2((uint32_t)token_of<BF16>(s * kSampleSlice, tid, k), __float_as_uint(x[k]));
          ++at;
        }
    }
  }
  best = wave_draw(best);
  sum = wave_sum(sum);
  if (lane == 0) {
    sm.wd[wave] = best;
    sm.ws[wave] = sum;
  }
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < 4; ++w) {
      best = better_draw(best, sm.wd[w]);
      sum += sm.ws[w];
    }
    const int64_t at = (int64_t)row * kSampleParts + part;
    a.best[at] = best.s;
    a.best_id[at] = best.id;
    a.sum[at] = sum;
  }
}

// ---------------------------------------------------------------------------
struct FinishSmem {
  uint2 list[2048];
  uint64_t mass[256];
  uint32_t cnt[256];
  Draw wd[4];
  double ws[4];
  float wm[4];
  int wi[4];
  // of a selection
  int digit;
  uint32_t cnt_in;
  uint64_t before, total;
};

// The listed tokens of a row: in LDS, in the list, or, where there are more, all
// tokens of the row again.
template <bool BF16>
struct Listed {
  const SampleArgs& a;
  FinishSmem& sm;
  int row, tid;
  uint32_t n;
  double top, inv_T, M;
  int lo, hi;
  __device__ __forceinline__ void stage() {
    if (n <= 2048) {
      for (uint32_t i = tid; i < n; i += kThreads) sm.list[i] = a.list[(int64_t)row * kSampleList + i];
    }
    __syncthreads();
  }
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    if (n <= 2048) {
      for (uint32_t i = tid; i < n; i += kThreads) f((int)sm.list[i].x, __uint_as_float(sm.list[i].y));
    } else if (n <= kSampleList) {
      for (uint32_t i = tid; i < n; i += kThreads) {
        const uint2 e = a.list[(int64_t)row * kSampleList + i];
        f((int)e.x, __uint_as_float(e.y));
      }
    } else {
      for (int v = tid; v < a.V; v += kThreads) {
        const float l = load1<BF16>(a, row, v);
        if (!(l > -INFINITY && (M - (double)l) * inv_T <= kSpan)) continue;
        const int j = min((int)(top - bin_of(l, inv_T)), kSampleBins - 1);
        if (j >= lo && j <= hi) f(v, l);
      }
    }
  }
};

constexpr int kListBits = 40;  // of a listed weight: 2^20 of them stay below 2^61

// The digit at which `target` (a count, or a weight) is reached, from the highest
// down (UP: from the lowest up), with what comes before it.  False: never.
template <bool MASS, bool UP>
__device__ __forceinline__ bool find_digit(FinishSmem& sm, int tid, uint64_t target) {
  __syncthreads();
  if (tid < 64) {
    uint64_t v[4], s = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int b = UP ? 4 * tid + e : 255 - 4 * tid - e;
      v[e] = MASS ? sm.mass[b] : (uint64_t)sm.cnt[b];
      s += v[e];
    }
    uint64_t in = s;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint64_t t = __shfl_up((unsigned long long)in, o);
      if (tid >= o) in += t;
    }
    const uint64_t hit = __ballot(in >= target);
    if (hit == 0) {
      if (tid == 0) sm.digit = -1;
    } else if (tid == __ffsll((unsigned long long)hit) - 1) {
      uint64_t before = in - s;
      int e = 0;
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (e == k && before + v[k] < target) {
          before += v[k];
          e = k + 1;
        }
      const int b = UP ? 4 * tid + e : 255 - 4 * tid - e;
      sm.digit = b;
      sm.before = before;
      sm.cnt_in = sm.cnt[b];
    }
  }
  __syncthreads();
  return sm.digit >= 0;
}

// Among the listed tokens that `in` allows, the key at which the target is reached
// in descending order: the key, what is before it and how many tokens have it.
struct Border {
  uint32_t key, ties;
  uint64_t before;
  bool found;
};
template <bool MASS, typename L, typename In>
__device__ __forceinline__ Border find_key(const L& ls, FinishSmem& sm, int tid, uint64_t target, double ref, In in) {
  Border b{0u, 0u, 0u, true};
#pragma unroll 1
  for (int shift = 24; shift >= 0; shift -= 8) {
    sm.cnt[tid] = 0;
    sm.mass[tid] = 0;
    __syncthreads();
    ls.each([&](int id, float l) {
      const uint32_t key = key_of(l);
      if (!in(id, key) || (shift < 24 && (key ^ b.key) >> (shift + 8) != 0)) return;
      const uint32_t dg = key >> shift & 255u;
      atomicAdd(&sm.cnt[dg], 1u);
      if (MASS)
        atomicAdd((unsigned long long*)&sm.mass[dg], (unsigned long long)fixed<kListBits>(exp(__builtin_fma((double)l, ls.inv_T, -ref))));
    });
    if (!find_digit<MASS, false>(sm, tid, target)) {
      b.found = false;
      __syncthreads();
      return b;
    }
    b.key |= (uint32_t)sm.digit << shift;
    b.before += sm.before;
    target -= sm.before;
    b.ties = sm.cnt_in;
    __syncthreads();
  }
  return b;
}

// The n-th lowest id (from 1) of the listed tokens with this key.
template <typename L>
__device__ __forceinline__ uint32_t find_id(const L& ls, FinishSmem& sm, int tid, uint32_t key, uint32_t n) {
  uint32_t found = 0;
  uint64_t target = n;
#pragma unroll 1
  for (int shift = 16; shift >= 0; shift -= 8) {
    sm.cnt[tid] = 0;
    __syncthreads();
    ls.each([&](int id, float l) {
      if (key_of(l) == key && (shift == 16 || ((uint32_t)id ^ found) >> (shift + 8) == 0)) atomicAdd(&sm.cnt[(uint32_t)id >> shift & 255u], 1u);
    });
    if (!find_digit<false, true>(sm, tid, target)) {
      __syncthreads();
      return 0xffffffffu;
    }
    found |= (uint32_t)sm.digit << shift;
    target -= sm.before;
    __syncthreads();
  }
  return found;
}

template <bool BF16>
__global__ void __launch_bounds__(kThreads) sample_finish_kernel(SampleArgs a) {
  __shared__ FinishSmem sm;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Request q = request_of(a, row);
  // the row's maximum
  const float ms = tid < a.NS ? a.smax[(int64_t)row * a.NS + tid] : -INFINITY;
  const float m0 = wave_max(ms);
  if (lane == 0) sm.wm[wave] = m0;
  __syncthreads();
  const float M = fmaxf(fmaxf(sm.wm[0], sm.wm[1]), fmaxf(sm.wm[2], sm.wm[3]));
  if (M == -INFINITY || q.greedy) {
    int id = 0x7fffffff;
    if (q.greedy && ms == M && tid < a.NS) id = a.sarg[(int64_t)row * a.NS + tid];
    id = wave_min(id);
    if (lane == 0) sm.wi[wave] = id;
    __syncthreads();
    if (tid == 0) {
      id = min(min(sm.wi[0], sm.wi[1]), min(sm.wi[2], sm.wi[3]));
      const bool none = M == -INFINITY;
      if (none) {
        flag_error(a.err, SPADE_DERR_NAN);
        id = 0;
      }
      a.tokens[row] = id;
      if (a.chosen != nullptr) a.chosen[row] = none ? 0.f : 1.f;
      SampleRow r{};
      r.max = M;
      r.inv_T = 0.0;
      r.cut = none ? -1.0 : 0.0;
      r.inv_sum = 1.0;
      r.key = key_of(M);
      r.id = (uint32_t)id;
      a.row[row] = r;
    }
    return;
  }
  SampleRow r = a.row[row];
  const uint64_t seed = (uint64_t)__float_as_uint(a.u[row]);
  Draw best{-INFINITY, 0x7fffffff};
  double sum = 0.0;
  if (tid < a.NW) {
    const int64_t at = (int64_t)row * kSampleParts + tid;
    best = Draw{a.best[at], a.best_id[at]};
    sum = a.sum[at];
  }
  uint32_t key = 0, id_to = 0xffffffffu;
  if (q.listed()) {
    Listed<BF16> ls{a, sm, row, tid, a.count[row], bin_of(M, r.inv_T), r.inv_T, (double)M, r.lo, r.hi};
    ls.stage();
    const double ref = edge_of(ls.top - r.lo), factor = exp(__builtin_fma(-(double)M, r.inv_T, ref));
    double total = r.total;
    uint32_t ties_k = 0xffffffffu;
    if (r.k_in) {
      const Border b = find_key<false>(ls, sm, tid, (uint64_t)(q.top_k - r.above), ref, [](int, uint32_t) { return true; });
      if (b.found) {
        key = b.key;
        ties_k = (uint32_t)(q.top_k - r.above) - (uint32_t)b.before;
        if (ties_k < b.ties) id_to = find_id(ls, sm, tid, key, ties_k);
      }
      // the weight of the first top_k
      if (tid == 0) sm.total = 0;
      __syncthreads();
      uint64_t mine = 0;
      ls.each([&](int id, float l) {
        const uint32_t k = key_of(l);
        if (k > key || (k == key && (uint32_t)id <= id_to)) mine += fixed<kListBits>(exp(__builtin_fma((double)l, r.inv_T, -ref)));
      });
      atomicAdd((unsigned long long*)&sm.total, (unsigned long long)mine);
      __syncthreads();
      total = r.mass + (double)sm.total * 0x1p-40 * factor;
      __syncthreads();
    }
    if (q.use_p) {
      const uint64_t target = (uint64_t)fmax(ceil(((q.top_p - kSlack) * total - r.mass) / factor * 0x1p40), 1.0);
      const uint32_t k_key = key, k_id = id_to;
      const Border b = find_key<true>(ls, sm, tid, target, ref, [&](int id, uint32_t k) {
        return k > k_key || (k == k_key && (uint32_t)id <= k_id);
      });
      if (b.found) {
        key = b.key;
        // as many of the equal tokens as it takes, in their order
        const uint32_t bits = key & 0x80000000u ? key ^ 0x80000000u : ~key;
        const uint64_t w = fixed<kListBits>(exp(__builtin_fma((double)__uint_as_float(bits), r.inv_T, -ref)));
        const uint64_t need = w > 0 ? (target - b.before + w - 1) / w : b.ties;
        const uint32_t n = (uint32_t)(need < 1 ? 1 : need > b.ties ? b.ties : need);
        id_to = n < b.ties || b.key == k_key ? find_id(ls, sm, tid, key, n) : 0xffffffffu;
      }
    }
    float bestf = -INFINITY;
    ls.each([&](int id, float l) {
      const uint32_t k = key_of(l);
      if (!(k > key || (k == key && (uint32_t)id <= id_to))) return;
      const double d = ((double)M - (double)l) * r.inv_T;
      if (d > q.min_d) return;
      sum += exp(-d);
      draw(best, bestf, seed, id, d);
    });
  }
  best = wave_draw(best);
  sum = wave_sum(sum);
  if (lane == 0) {
    sm.wd[wave] = best;
    sm.ws[wave] = sum;
  }
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < 4; ++w) {
      best = better_draw(best, sm.wd[w]);
      sum += sm.ws[w];
    }
    best.id = min(best.id, a.V - 1);
    a.tokens[row] = best.id;
    const double d = ((double)M - (double)load1<BF16>(a, row, best.id)) * r.inv_T;
    if (a.chosen != nullptr) a.chosen[row] = (float)(exp(-d) / sum);
    r.cut = q.min_d;
    r.inv_sum = 1.0 / sum;
    r.key = key;
    r.id = id_to;
    a.row[row] = r;
  }
}

template <bool BF16>
__global__ void __launch_bounds__(kThreads) sample_probs_kernel(SampleArgs a) {
  const int row = blockIdx.x / a.NS, s = blockIdx.x - row * a.NS, tid = threadIdx.x;
  const SampleRow r = a.row[row];
  float x[16];
  load16<BF16>(a, row, s * kSampleSlice, tid, x);
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const int v = token_of<BF16>(s * kSampleSlice, tid, k);
    const uint32_t key = key_of(x[k]);
    const double d = ((double)r.max - (double)x[k]) * r.inv_T;
    const bool kept = x[k] > -INFINITY && (key > r.key || (key == r.key && (uint32_t)v <= r.id)) && d <= r.cut;
    x[k] = kept ? (float)(exp(-d) * r.inv_sum) : 0.f;
  }
  float* out = a.probs + (int64_t)row * a.V;
  constexpr int W = BF16 ? 8 : 4;
#pragma unroll
  for (int j = 0; j < 16 / W; ++j) {
    const int v = token_of<BF16>(s * kSampleSlice, tid, j * W);
    if (v + W <= a.V) {
#pragma unroll
      for (int i = 0; i < W; i += 4) {
        Float4u w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w.v[e] = x[j * W + i + e];
        *(Float4u*)(out + v + i) = w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < W; ++i)
        if (v + i < a.V) out[v + i] = x[j * W + i];
    }
  }
}

template <bool BF16>
hipError_t sample_t(const SampleArgs& a, hipStream_t st) {
  const int64_t slices = (int64_t)a.rows * a.NS, parts = (int64_t)a.rows * a.NW;
  if (slices > 0x7fffffff || parts > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL((sample_slice_kernel<BF16>), dim3((unsigned)slices), dim3(kThreads), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((sample_scan_kernel<BF16>), dim3((unsigned)parts), dim3(kThreads), 0, st, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL((sample_finish_kernel<BF16>), dim3((unsigned)a.rows), dim3(kThreads), 0, st, a);
  if ((e = hipGetLastError()) != hipSuccess || a.probs == nullptr) return e;
  hipLaunchKernelGGL((sample_probs_kernel<BF16>), dim3((unsigned)slices), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t sample_workspace(int rows, int V, SampleArgs* a, uint8_t* base) {
  const size_t R = (size_t)rows, NS = (size_t)(V + kSampleSlice - 1) / kSampleSlice;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += (bytes + 255) & ~(size_t)255;
    return base + o;
  };
  uint8_t* smax = take(R * NS * 4);
  uint8_t* sarg = take(R * NS * 4);
  uint8_t* hist = take(R * NS * kSampleBins * 8);
  uint8_t* best = take(R * kSampleParts * 8);
  uint8_t* best_id = take(R * kSampleParts * 4);
  uint8_t* sum = take(R * kSampleParts * 8);
  uint8_t* row = take(R * sizeof(SampleRow));
  uint8_t* count = take(R * 4);
  uint8_t* list = take(R * kSampleList * 8);
  if (a != nullptr) {
    a->smax = (float*)smax;
    a->sarg = (int32_t*)sarg;
    a->hist = (uint64_t*)hist;
    a->best = (double*)best;
    a->best_id = (int32_t*)best_id;
    a->sum = (double*)sum;
    a->row = (SampleRow*)row;
    a->count = (uint32_t*)count;
    a->list = (uint2*)list;
  }
  return off;
}

hipError_t launch_sample(const SampleArgs& in, hipStream_t st) {
  SampleArgs a = in;
  a.NS = (a.V + kSampleSlice - 1) / kSampleSlice;
  // every part reads the row's bins (1 KB a slice): few rows take many parts, many rows few
  const int parts = std::max(1, std::min({kSampleParts, a.NS, 2048 / a.rows}));
  a.spw = (a.NS + parts - 1) / parts;
  a.NW = (a.NS + a.spw - 1) / a.spw;
  return a.bf16 ? sample_t<true>(a, st) : sample_t<false>(a, st);
}

}  // namespace spade
