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
//                         bins of their logit over T; rows without filters draw here
//   sample_scan_kernel    the row's bins: which hold the border; tokens above them
//                         draw, theirs are listed
//   sample_finish_kernel  the border among the listed tokens, the draw
//   sample_probs_kernel   the distribution, where asked
//
// One float32 row of 128256 (top_k 50, top_p 0.9): 5.1 + 10.8 + 8.6 us, each a chain
// of a few round trips on at most 32 compute units.  400 rows, us of the three passes:
//   greedy                 40 + 5 + 6     the stream, 5.2 TB/s
//   no filter             132 + 5 + 14    the noise's hash (two 64-bit products a token)
//   top_k 50, top_p 0.9    60 + 78 + 20   the stream twice; vector instructions
//   min_p                  40 + 50 + 14   the stream twice
// and of bfloat16, of all kinds, 59 + 42 + 28 (a stream of 103 MB: 20).
#include "sample.h"

#include <float.h>

#include <algorithm>
#include <type_traits>

#include "device_accept.h"
#include "device_lanes.h"
#include "sample_grid.h"

namespace spade {

template <int STEP>
__device__ __forceinline__ SampleDraw prefix_step(SampleDraw v, SampleDraw) {
  return SampleDraw{prefix_step<STEP>(v.s, v.s), prefix_step<STEP>(v.id, v.id), prefix_step<STEP>(v.d, v.d)};
}

namespace {

constexpr int kThreads = 256;
constexpr double kSlack = 0x1p-40;                   // of top_p: equal masses count as reached

struct Request {
  double inv_T, top_p, min_d;  // min_d: largest d that min_p allows
  int top_k;
  bool greedy, use_k, use_p;
  __device__ __forceinline__ bool listed() const { return use_k || use_p; }
  // neither borders nor the row's maximum matter to a slice's draw: tokens that the other slices'
  // maxima leave out could not win (32 below them; the noise spans 19.5), and weigh 2^-46
  __device__ __forceinline__ bool plain() const { return !greedy && !listed() && min_d >= kSpan; }
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

// exp of what the tables hold: by its series at x / 64
constexpr double const_exp(double x) {
  double t = 1.0, s = 1.0;
  for (int i = 1; i < 24; ++i) {
    t *= x / 64.0 / i;
    s += t;
  }
  for (int i = 0; i < 6; ++i) s *= s;
  return s;
}
struct Tables {
  double step[kSteps];       // weight of a step over its bin's upper edge's
  double edge[kSampleBins];  // weight of the upper edge of the bin j below the first over that bin's lower edge's
  double rel[kSampleBins];   // ... over the first's upper edge's
};
constexpr Tables make_tables() {
  Tables t{};
  for (int i = 0; i < kSteps; ++i) t.step[i] = const_exp((i - kSteps) * kStep);
  for (int j = 0; j < kSampleBins; ++j) t.edge[j] = const_exp((1 - j) * kBin);
  for (int j = 0; j < kSampleBins; ++j) t.rel[j] = t.edge[j] / t.edge[0];
  return t;
}
__device__ const Tables kTables = make_tables();
// weight of a place over its bin's upper edge's
__device__ __forceinline__ double place_weight(const double* table, int step, float rest) {
  const float r = rest * (float)kStep;
  const float e = r * __builtin_fmaf(r, __builtin_fmaf(r, 1.f / 6.f, 0.5f), 1.f);
  const double t = table[step];
  return __builtin_fma(t, (double)e, t);
}
static_assert(kSteps == kThreads && kSteps == 256, "a step per thread, 8 bits");
// The lower edge of the top bin over the largest logit, whose weight is 1.
__device__ __forceinline__ double top_scale(const Grid& g, const double* table, float m) {
  int step;
  float rest;
  g.place(m, step, rest);
  return 1.0 / (place_weight(table, step, rest) * const_exp(kBin));
}

// w 2^n as an integer, w 2^n < 2^51
template <int N>
__device__ __forceinline__ uint64_t fixed(double w) {
  return (uint64_t)__double_as_longlong(__builtin_fma(w, (double)(1ull << N), 0x1p52)) & 0xfffffffffffffull;
}
constexpr int kMassBits = 38;  // of a slice's bins: 4096 weights up to 1 below the count at bit 51
// A listed token's weight over that of the first listed bin's edge, times `scale` (2^bits):
// in the bins' own steps first, so that equal weights add up to exactly what the bins
// hold.  The row's bits are as many as all the listed weights leave in 63, 50 at most: a list
// from the largest weight down to e^-32 of it keeps sums to 2^-50 a token.
constexpr int kListBits = 50;
__device__ __forceinline__ double power_of_2(int n) { return __longlong_as_double((long long)(1023 + n) << 52); }
__device__ __forceinline__ uint64_t listed_weight(const double* table, int step, float rest, double rel, double scale) {
  const double w = (double)fixed<kMassBits>(place_weight(table, step, rest)) * 0x1p-38 * rel;
  return (uint64_t)__double_as_longlong(__builtin_fma(w, scale, 0x1p52)) & 0xfffffffffffffull;
}
// A place of the listed bins, j below the first of them, in steps from its upper edge.
__device__ __forceinline__ int listed_place(int j, int step) { return j * kSteps + (kSteps - 1 - step); }
constexpr int kSubBits = 8;
static_assert(kSampleSub == 1 << kSubBits && kSampleSub == 2 * kSampleBins && kSampleSub == kThreads, "two bins' places; in the bins' memory");
constexpr int kCopies = 4;     // of a slice's bins, by lane, which often meet in a bin (2 to 16: the same time)

// Order-preserving integer of a float.
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t b = __float_as_uint(l + 0.f);  // (-0 is 0)
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// a key's logit
__device__ __forceinline__ float logit_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
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
  return from_lane(all_lanes(v, [](float x, float y) { return fmaxf(x, y); }), 63);
}
__device__ __forceinline__ int wave_min(int v) {
  return from_lane(all_lanes(v, [](int x, int y) { return min(x, y); }), 63);
}
__device__ __forceinline__ double wave_sum(double v) { return from_lane(prefix_sum(v), 63); }

using Draw = SampleDraw;
constexpr Draw kNoDraw{-INFINITY, 0x7fffffff, 0.0};
__device__ __forceinline__ Draw better_draw(Draw x, Draw y) { return y.s > x.s || (y.s == x.s && y.id < x.id) ? y : x; }
__device__ __forceinline__ Draw wave_draw(Draw v) {
  v = all_lanes(v, [](Draw x, Draw y) { return better_draw(x, y); });
  return Draw{from_lane(v.s, 63), from_lane(v.id, 63), from_lane(v.d, 63)};
}

// The draw as a race: argmax(G - d) is the token with the least e = -log(U) exp(d).
// 1 - U <= -log(U), so most tokens end without a logarithm.  e is good to 2^-17 in
// float32: tokens closer than that are told apart in double.
__device__ __noinline__ double score_of(uint32_t x, double d) {
  const double U = ((double)x + 0.5) * 0x1p-23;
  return -log(-log(U)) - d;
}
constexpr float kNear = 0x1p-15f;
constexpr uint64_t kGolden = 0x9E3779B97F4A7C15ull;  // of SplitMix64's state
// The 23 bits of the noise: output n of the stream from z = seed + (n + 1) golden (its
// last step leaves the upper bits alone).
__device__ __forceinline__ uint32_t noise_bits(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return (uint32_t)(z >> 32) >> 9;
}
// 1 - U, exact
__device__ __forceinline__ float noise_rest(uint32_t x) { return ((float)(0x7fffffu - x) + 0.5f) * 0x1p-23f; }

struct Race {
  float bound = INFINITY;  // nothing above it can win
  float e = INFINITY;      // the lane's best
  uint32_t x = 0;
  int id = 0x7fffffff;
  double d = INFINITY;
  // Token n at distance dn with noise xn (y = 1 - U) and f = exp(dn).
  __device__ __forceinline__ void enter(int n, double dn, float f, uint32_t xn, float y) {
    if (y * f > bound) return;
    // -log(1 - y): a series below 1/8
    float g = __builtin_fmaf(y, 1.f / 6.f, 0.2f);
    g = __builtin_fmaf(y, g, 0.25f);
    g = __builtin_fmaf(y, g, 1.f / 3.f);
    g = __builtin_fmaf(y, g, 0.5f);
    g = __builtin_fmaf(y, g, 1.f) * y;
    if (y >= 0.125f) g = __builtin_amdgcn_logf(1.f - y) * -0.69314718f;
    const float en = g * f;
    bool first = en < e;
    if (en >= e * (1.f - kNear) && en <= e * (1.f + kNear)) {
      const double a = score_of(xn, dn), b = score_of(x, d);
      first = a > b || (a == b && n < id);
    }
    if (first) {
      e = en;
      x = xn;
      id = n;
      d = dn;
      bound = fminf(bound, e * (1.f + 4.f * kNear));
    }
  }
  // the lanes' bounds to all (all lanes of the wave call it)
  __device__ __forceinline__ void share() {
    bound = from_lane(all_lanes(bound, [](float a, float b) { return fminf(a, b); }), 63);
  }
  // the wave's token
  __device__ __forceinline__ Draw best() {
    share();
    Draw r = kNoDraw;
    if (e <= bound) r = Draw{score_of(x, d), id, d};
    return wave_draw(r);
  }
};

// A workgroup's draws and weights to one place.
template <int W>
__device__ __forceinline__ void store_draw(const SampleArgs& a, int64_t at, Race& race, double sum, Draw* wd, double* ws, int tid) {
  Draw best = race.best();
  sum = wave_sum(sum);
  if ((tid & 63) == 0) {
    wd[tid >> 6] = best;
    ws[tid >> 6] = sum;
  }
  __syncthreads();
  if (tid == 0) {
#pragma unroll
    for (int w = 1; w < W; ++w) {
      best = better_draw(best, wd[w]);
      sum += ws[w];
    }
    a.best[at] = best;
    a.sum[at] = sum;
  }
}

// ---------------------------------------------------------------------------
// A slice of a row.  Tokens are looked up one by one (80 registers, six waves a SIMD): four or
// sixteen at a time need more and take 65 to 75 us where one by one takes 59 (400 rows of
// 128256, bfloat16; vector instructions fill the time).
template <bool BF16>
__global__ void __launch_bounds__(kThreads) sample_slice_kernel(SampleArgs a) {
  __shared__ float wm[4];
  __shared__ int wi[4];
  __shared__ double table[kSteps], edge[kSampleBins];
  __shared__ uint64_t bins[kSampleBins * kCopies];
  __shared__ Draw wd[4];
  __shared__ double ws[4];
  const int row = blockIdx.x / a.NS, s = blockIdx.x - row * a.NS, tid = threadIdx.x, wave = tid >> 6;
  float x[16];
  const bool nan = load16<BF16>(a, row, s * kSampleSlice, tid, x);
  const Request q = request_of(a, row);
  if (nan) flag_error(a.err, SPADE_DERR_NAN);
  table[tid] = kTables.step[tid];
  if (tid < kSampleBins) edge[tid] = kTables.edge[tid];
#pragma unroll
  for (int c = 0; c < kSampleBins * kCopies; c += kThreads) bins[c + tid] = 0;
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
    if (s == 0) {
      a.count[row] = 0;
      a.tail[row] = 0;
    }
  }
  if (s == 0 && q.listed())
    for (int i = tid; i < kSampleSub; i += kThreads) {
      a.sub_mass[(int64_t)row * kSampleSub + i] = 0;
      a.sub_count[(int64_t)row * kSampleSub + i] = 0;
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
  const double inv_T = row_inv_T(q.inv_T, m);
  const Grid grid(inv_T, m);
  if (q.plain()) {
    const int base = token_of<BF16>(s * kSampleSlice, tid, 0);
    const uint64_t z0 = (uint64_t)__float_as_uint(a.u[row]) + (uint64_t)(base + 1) * kGolden;
    Race race;
    double sum = 0.0;
    const double scale = top_scale(grid, table, m);
    auto draw = [&](auto wide) {
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        int step;
        float rest;
        const int j = grid.template place<wide.value>(x[k], step, rest);
        if (j < kSampleBins) {
          const double w = place_weight(table, step, rest) * (edge[j] * scale);
          sum += w;
          const float f = __builtin_amdgcn_rcpf((float)w);
          if (f * 0x1p-24f <= race.bound) {  // (1 - U is at least 2^-24: no noise brings the others ahead)
            const int off = token_of<BF16>(0, 0, k);
            const uint32_t xn = noise_bits(z0 + (uint64_t)off * kGolden);
            race.enter(base + off, ((double)m - (double)x[k]) * inv_T, f, xn, noise_rest(xn));
          }
        }
        if (k == 0 || k == 4) race.share();
      }
    };
    if (grid.wide)
      draw(std::true_type{});
    else
      draw(std::false_type{});
    store_draw<4>(a, (int64_t)row * a.NS + s, race, sum, wd, ws, tid);
    return;
  }
  if (!q.listed()) return;
  auto count = [&](auto wide) {
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      int step;
      float rest;
      const int j = grid.template place<wide.value>(x[k], step, rest);
      if (j < kSampleBins)
        atomicAdd((unsigned long long*)&bins[j * kCopies + (tid & (kCopies - 1))],
                  (unsigned long long)(fixed<kMassBits>(place_weight(table, step, rest)) | 1ull << 51));
    }
  };
  if (grid.wide)
    count(std::true_type{});
  else
    count(std::false_type{});
  __syncthreads();
  if (tid < kSampleBins) {
    uint64_t w = 0;
#pragma unroll
    for (int c = 0; c < kCopies; ++c) w += bins[tid * kCopies + c];
    a.hist[at * kSampleBins + tid] = w;
  }
}

// ---------------------------------------------------------------------------
// Inclusive prefix of two values per lane over 128 bins.
struct ScanSmem {
  double table[kSteps];
  double factor[kSampleBins];  // weight of a bin's upper edge over the largest weight
  uint64_t mass[2][kSampleBins];
  uint32_t cnt[2][kSampleBins];
  int off[256];  // bins between a slice's top and the row's (1000: out of reach)
  float x[16][kThreads];
  float wm[4];
  double ws[4];
  Draw wd[4];
  SampleRow row;
};

// The least finite logit that `in`, true from some logit on, holds for (infinity: none).
// Among the 64 numbers around a guess at once; rounding can put it further away near 0,
// then by all numbers, 64 parts at a time.
template <typename In>
__device__ __forceinline__ float least_logit(double guess, In in) {
  const int64_t first = key_of(-FLT_MAX), last = key_of(FLT_MAX);
  const int64_t at = key_of((float)fmin(fmax(guess, -(double)FLT_MAX), (double)FLT_MAX)) - 32;
  const int lane = threadIdx.x & 63;
  auto number = [&](int64_t key) { return logit_of((uint32_t)min(max(key, first), last)); };
  uint64_t hits = __ballot(in(number(at + lane)));
  if (hits != 0 && (hits & 1) == 0) return number(at + __ffsll((unsigned long long)hits) - 1);
  int64_t below = first - 1;  // (below, below + 64 step] holds it
#pragma unroll 1
  for (int bits = 27;; bits = max(0, bits - 6)) {
    hits = __ballot(in(number(below + ((int64_t)(lane + 1) << bits))));
    if (hits == 0) return INFINITY;
    below += (int64_t)(__ffsll((unsigned long long)hits) - 1) << bits;
    if (bits == 0) return number(below + 1);
  }
}

// A part of a row: every part puts the slices' bins together for itself, then reads its
// slices that reach the border.  Tokens are told apart by thresholds of their logits,
// so that only those that draw or are listed have their place and weight worked out,
// every lane its own next one (400 rows: 42 us; all tokens' places: 47).
template <bool BF16>
__global__ void __launch_bounds__(kThreads) sample_scan_kernel(SampleArgs a) {
  __shared__ ScanSmem sm;
  const int row = blockIdx.x / a.NW, part = blockIdx.x - row * a.NW, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Request q = request_of(a, row);
  if (q.greedy || q.plain()) return;
  const float ms = tid < a.NS ? a.smax[(int64_t)row * a.NS + tid] : -INFINITY;  // (at most 256 slices)
  const float m0 = wave_max(ms);
  if (lane == 0) sm.wm[wave] = m0;
  sm.table[tid] = kTables.step[tid];
  const double ej = kTables.edge[tid & (kSampleBins - 1)];
  __syncthreads();
  const float M = fmaxf(fmaxf(sm.wm[0], sm.wm[1]), fmaxf(sm.wm[2], sm.wm[3]));
  if (M == -INFINITY) return;
  const double inv_T = row_inv_T(q.inv_T, M);
  const Grid grid(inv_T, M);
  {
    int step;
    float rest;
    const double d = ((double)M - (double)ms) * inv_T;
    sm.off[tid] = ms > -INFINITY && d <= kSpan ? grid.place(ms, step, rest) : 1000;
    if (tid < kSampleBins) sm.factor[tid] = ej * top_scale(grid, sm.table, M);
  }
  __syncthreads();
  int lo = kSampleBins, hi = kSampleBins;
  if (q.listed()) {
    const int j = tid & (kSampleBins - 1), half = tid / kSampleBins;
    uint64_t mass = 0;
    uint32_t cnt = 0;
    const uint64_t* h = a.hist + (int64_t)row * a.NS * kSampleBins;
    for (int s0 = half; s0 < a.NS; s0 += 32) {  // (sixteen loads in flight)
      uint64_t w[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int s = s0 + 2 * e, jj = s < a.NS && j <= kLastBin ? j - sm.off[s] : -1;
        w[e] = jj >= 0 ? h[s * kSampleBins + jj] : 0ull;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        mass += w[e] & 0x7ffffffffffffull;
        cnt += (uint32_t)(w[e] >> 51);
      }
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
      const double sw = prefix_sum(w[0] + w[1]);
      const int sc = prefix_sum(c[0] + c[1]);
      wi[1] = sw;
      wi[0] = sw - w[1];
      ci[1] = sc;
      ci[0] = sc - c[1];
      const double total = from_lane(sw, 63);
      // the first bin with f, and the counts and weights before it
      auto first = [&](bool f0, bool f1) {
        const uint64_t hit = __ballot(f0 || f1);
        if (hit == 0) return kSampleBins - 1;
        const int l = __ffsll((unsigned long long)hit) - 1;
        return 2 * l + (from_lane((int)f0, l) ? 0 : 1);
      };
      int k_bin = kSampleBins - 1, k_in = 0;
      // The window ends within its last bin: what that holds in all is only a bound.
      const double last = from_lane(w[kLastBin & 1], kLastBin >> 1);
      double least = total - last, most = total;  // of the weight that top_p refers to
      if (q.use_k && from_lane(ci[1], 63) > q.top_k) {  // (else all are among the first top_k)
        k_in = 1;
        k_bin = first(ci[0] >= q.top_k, ci[1] >= q.top_k);
        most = from_lane(k_bin & 1 ? wi[1] : wi[0], k_bin >> 1);
        least = most - from_lane(k_bin & 1 ? w[1] : w[0], k_bin >> 1);
      }
      lo = hi = k_bin;
      if (q.use_p) {
        // (a little more on either side, so that rounding cannot move the border out)
        const double t0 = (q.top_p - 0x1p-30) * least, t1 = (q.top_p + 0x1p-30) * most;
        lo = min(lo, first(wi[0] >= t0, wi[1] >= t0));
        hi = min(hi, first(wi[0] >= t1, wi[1] >= t1));
        if (k_in) hi = k_bin;  // the first top_k tokens' weight ends there
      }
      const double in = from_lane(lo & 1 ? wi[1] : wi[0], lo >> 1), ex = in - from_lane(lo & 1 ? w[1] : w[0], lo >> 1);
      const double upto = from_lane(hi & 1 ? wi[1] : wi[0], hi >> 1);
      const int above = from_lane(lo & 1 ? ci[1] : ci[0], lo >> 1) - from_lane(lo & 1 ? c[1] : c[0], lo >> 1);
      // more than the list holds: their counts and weights by finer parts instead
      const int n = from_lane(hi & 1 ? ci[1] : ci[0], hi >> 1) - above, span = (hi - lo + 1) * kSteps;
      const int sub = n > kSampleList ? max(0, 32 - __clz(span - 1) - kSubBits) : -1;
      if (lane == 0) {
        sm.row.mass = lo == 0 ? 0.0 : ex;
        sm.row.tail = q.use_p && !k_in && last > total * 0x1p-46;
        sm.row.total = sm.row.tail ? total - last : total;
        sm.row.lo = lo;
        sm.row.hi = hi;
        sm.row.above = above;
        sm.row.k_in = k_in;
        sm.row.sub = sub;
        const int exponent = (int)(__double_as_longlong((upto - sm.row.mass) / sm.factor[lo]) >> 52) - 1022;
        sm.row.bits = min(kListBits, 62 - max(exponent, 0));
      }
    }
    __syncthreads();
    lo = sm.row.lo;
    hi = sm.row.hi;
  }
  // The least logits of the window, of the bins up to hi, of those above lo and of min_p
  auto within = [&](double most) {
    return least_logit((double)M - most / inv_T, [&](float l) { return ((double)M - (double)l) * inv_T <= most; });
  };
  auto from_bin = [&](int bin) {  // of the bins up to `bin` below the top
    return least_logit((grid.top - bin) * kSteps / grid.c, [&](float l) { return grid.reaches(l, bin); });
  };
  float t_window = -FLT_MAX, t_list = -FLT_MAX, t_sure = -FLT_MAX, t_min = -FLT_MAX, t_tail = -FLT_MAX;
  const bool tail = q.listed() && sm.row.tail;
  if (inv_T > 0.0) {
    t_window = within(kSpan);
    if (q.min_d < kSpan) t_min = within(q.min_d);
    if (hi < kSampleBins - 1) t_list = from_bin(hi);
    if (lo < kSampleBins) t_sure = lo > 0 ? from_bin(lo - 1) : INFINITY;
    if (tail) t_tail = from_bin(kLastBin - 1);
  } else if (q.listed()) {
    t_sure = INFINITY;  // (all logits are in one bin)
  }
  t_list = fmaxf(t_list, t_window);
  t_sure = fmaxf(t_sure, t_window);
  if (part == 0 && tid == 0) {
    SampleRow r = sm.row;
    if (!q.listed()) {
      r.mass = r.total = 0.0;
      r.lo = r.hi = kSampleBins;
      r.above = r.k_in = r.tail = 0;
      r.sub = -1;
    }
    r.max = M;
    r.inv_T = inv_T;
    r.least = t_list;
    r.below = t_sure;
    a.row[row] = r;
  }
  const int sub = q.listed() ? sm.row.sub : -1;
  uint64_t* sub_mass = &sm.mass[0][0];  // (the bins' are used)
  uint32_t* sub_count = &sm.cnt[0][0];
  if (sub >= 0) {
    sub_mass[tid] = 0;
    sub_count[tid] = 0;
    __syncthreads();
  }
  const uint64_t z0 = (uint64_t)__float_as_uint(a.u[row]);
  Race race;
  const double scale = q.listed() ? power_of_2(sm.row.bits) : 0.0;
  double sum = 0.0;
  uint64_t in_tail = 0;
  const int s1 = min(a.NS, (part + 1) * a.spw), reach = tail ? kLastBin : min(hi, kSampleBins - 1);
  // the slices that reach these bins, one ahead
  auto after = [&](int s) {
    while (s < s1 && sm.off[s] > reach) ++s;
    return s;
  };
  float next[16];
  int s = after(part * a.spw);
  if (s < s1) load16<BF16>(a, row, s * kSampleSlice, tid, next);
  while (s < s1) {
    float x[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) x[k] = next[k];
    const int here = s;
    s = after(s + 1);
    if (s < s1) load16<BF16>(a, row, s * kSampleSlice, tid, next);
    uint32_t listed = 0, sure = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      sm.x[k][tid] = x[k];
      const bool above = x[k] >= t_sure;
      sure |= (above && x[k] >= t_min ? 1u : 0u) << k;
      listed |= (!above && x[k] >= t_list && q.listed() ? 1u : 0u) << k;
    }
    if (tail) {
      uint32_t in = 0;
#pragma unroll
      for (int k = 0; k < 16; ++k) in |= (x[k] >= t_window && x[k] < t_tail ? 1u : 0u) << k;
      while (in != 0) {
        const int k = __builtin_ctz(in);
        in &= in - 1;
        int step;
        float rest;
        grid.place(sm.x[k][tid], step, rest);
        in_tail += fixed<kMassBits>(place_weight(sm.table, step, rest));
      }
    }
    // the tokens above, every lane its own
    while (__any(sure != 0)) {
      if (sure != 0) {
        const int k = __builtin_ctz(sure);
        sure &= sure - 1;
        const float l = sm.x[k][tid];
        int step;
        float rest;
        const int j = min(max(grid.place(l, step, rest), 0), kSampleBins - 1), id = token_of<BF16>(here * kSampleSlice, tid, k);
        const double w = place_weight(sm.table, step, rest) * sm.factor[j];
        sum += w;
        const uint32_t xn = noise_bits(z0 + (uint64_t)(id + 1) * kGolden);
        race.enter(id, ((double)M - (double)l) * inv_T, __builtin_amdgcn_rcpf((float)w), xn, noise_rest(xn));
      }
      race.share();
    }
    if (sub >= 0) {
      while (listed != 0) {
        const int k = __builtin_ctz(listed);
        listed &= listed - 1;
        int step;
        float rest;
        const int j = min(max(grid.place(sm.x[k][tid], step, rest) - lo, 0), hi - lo);
        const int at = listed_place(j, step) >> sub;
        atomicAdd((unsigned long long*)(sub_mass + at), (unsigned long long)listed_weight(sm.table, step, rest, kTables.rel[j], scale));
        atomicAdd(sub_count + at, 1u);
      }
    } else if (__any(listed != 0)) {
      const int n = __popc(listed);
      const int in = prefix_sum(n);
      uint32_t at = 0;
      if (lane == 63) at = atomicAdd(a.count + row, (uint32_t)in);
      at = from_lane(at, 63) + (uint32_t)(in - n);
#pragma unroll
      for (int k = 0; k < 16; ++k)
        if (listed >> k & 1u) {
          if (at < kSampleList)
            a.list[(int64_t)row * kSampleList + at] = make_uint2((uint32_t)token_of<BF16>(here * kSampleSlice, tid, k), __float_as_uint(x[k]));
          ++at;
        }
    }
  }
  if (tail) {
    in_tail = from_lane(prefix_sum(in_tail), 63);
    if (lane == 0 && in_tail != 0) atomicAdd((unsigned long long*)(a.tail + row), (unsigned long long)in_tail);
  }
  if (sub >= 0) {
    __syncthreads();
    if (sub_count[tid] != 0) {
      atomicAdd((unsigned long long*)(a.sub_mass + (int64_t)row * kSampleSub + tid), (unsigned long long)sub_mass[tid]);
      atomicAdd(a.sub_count + (int64_t)row * kSampleSub + tid, sub_count[tid]);
    }
  }
  store_draw<4>(a, (int64_t)row * a.NS + part, race, sum, sm.wd, sm.ws, tid);
}

// ---------------------------------------------------------------------------
// (400 rows of mixed filters, 128256 tokens: 27 us; 256 or 512 threads 41 to 65 where 1024 took
// 32, for one row 13 where they took 16; weights looked up again in every pass 32)
constexpr int kFinish = 1024;                     // threads of a row's last workgroup
constexpr int kStaged = kSampleList;               // listed tokens, all kept in LDS
static_assert(kSampleList >= kFinish, "an entry per thread");

struct FinishSmem {
  uint2 list[kStaged];  // key, id
  uint64_t weight[kStaged];
  double table[kSteps];
  double factor[kSampleBins];  // weight of a bin's edge over that of the list's first
  uint64_t mass[2][256];  // of this digit and, cleared meanwhile, of the next
  uint32_t cnt[2][256];
  Draw wd[kFinish / 64];
  double ws[kFinish / 64];
  uint64_t wl[kFinish / 64];
  float wm[kFinish / 64];
  int wi[kFinish / 64];
  uint32_t key_lo, key_hi;
  // of a selection
  int digit;
  uint32_t cnt_in;
  uint64_t before, total;
  // of the border's parts
  uint64_t part_mass[kSampleSub / 64];
  uint32_t part_cnt[kSampleSub / 64];
  int k_part, p_part[2];
  uint64_t k_mass[2], mass_before;
  uint32_t cnt_before, count;
};

// The listed tokens of a row: in LDS, from the list, or, where that was too short
// for them, all tokens of the row again.
template <bool BF16>
struct Tokens {
  const SampleArgs& a;
  FinishSmem& sm;
  int row, tid;
  uint32_t n;
  double M, inv_T;
  Grid grid;
  int lo, hi;
  double scale;
  __device__ __forceinline__ void stage(uint2 e, double step, double rel) {
    if (tid < kSteps) sm.table[tid] = step;
    if (tid < kSampleBins) sm.factor[tid] = rel;
    __syncthreads();
    if (n <= kStaged)
      for (uint32_t i = tid; i < n; i += kFinish) {
        if (i >= kFinish) e = a.list[(int64_t)row * kSampleList + i];
        const float l = __uint_as_float(e.y);
        sm.list[i] = make_uint2(key_of(l), e.x);
        sm.weight[i] = weight(l);
      }
    __syncthreads();
  }
  __device__ __forceinline__ uint64_t weight(float l) const {
    int step;
    float rest;
    const int j = min(max(grid.place(l, step, rest) - lo, 0), kSampleBins - 1);
    return listed_weight(sm.table, step, rest, sm.factor[j], scale);
  }
  // f(id, key, weight()) of every listed token
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    if (n <= kStaged) {
#pragma unroll 1
      for (uint32_t i = tid; i < n; i += kFinish) {
        const uint2 e = sm.list[i];
        f((int)e.y, e.x, [&] { return sm.weight[i]; });
      }
      return;
    }
#pragma unroll 1
    for (int v = tid; v < a.V; v += kFinish) {
      const float l = load1<BF16>(a, row, v);
      if (!(l > -INFINITY && (M - (double)l) * inv_T <= kSpan)) continue;
      int step;
      float rest;
      const int j = min(grid.place(l, step, rest), kSampleBins - 1);
      if (j >= lo && j <= hi) f(v, key_of(l), [&] { return weight(l); });
    }
  }
};

// More tokens in the border's bins than the list holds.  Their counts and weights by
// parts of those bins tell which parts the border is in: one pass over the row draws
// the tokens above them and lists theirs (if these are still too many, as where all
// are equal, every later pass reads the row).  One row of 128256 logits of N(0, 1) with
// top_p 0.9, 13 thousand of them in the border's bin: 69 us in all, with every pass over
// the row 304.  For lists that fit it gains nothing: what the last pass saves (27 -> 24
// us, 400 rows) the second one pays.
template <bool BF16>
__device__ __forceinline__ void narrow(Tokens<BF16>& ls, FinishSmem& sm, int tid, const Request& q, SampleRow& r, uint64_t z0,
                                       double unit, Race& race, uint64_t& sum) {
  const SampleArgs& a = ls.a;
  const int lane = tid & 63, wave = tid >> 6;
  const bool mine = tid < kSampleSub;
  const int64_t at = (int64_t)ls.row * kSampleSub + (mine ? tid : 0);
  const uint64_t w = mine ? a.sub_mass[at] : 0ull;
  const uint32_t c = mine ? a.sub_count[at] : 0u;
  uint64_t wi = prefix_sum(w);
  uint32_t ci = prefix_sum(c);
  if (mine && lane == 63) {
    sm.part_mass[wave] = wi;
    sm.part_cnt[wave] = ci;
  }
  if (tid == 0) {
    sm.k_part = sm.p_part[0] = sm.p_part[1] = kSampleSub - 1;
    sm.k_mass[0] = sm.k_mass[1] = 0;
    sm.count = 0;
  }
  __syncthreads();
  if (mine)
    for (int v = 0; v < wave; ++v) {
      wi += sm.part_mass[v];
      ci += sm.part_cnt[v];
    }
  if (r.k_in && mine) {
    const uint32_t n = (uint32_t)(q.top_k - r.above);
    if (ci >= n && ci - c < n) {
      sm.k_part = tid;
      sm.k_mass[0] = wi - w;
      sm.k_mass[1] = wi;
    }
  }
  __syncthreads();
  int lo = sm.k_part, hi = lo;
  if (q.use_p) {
    // (a little more on either side, as for the bins)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const double of = r.k_in ? r.mass + (double)sm.k_mass[e] * unit : r.total;
      const double t = ((q.top_p + (e == 0 ? -0x1p-30 : 0x1p-30)) * of - r.mass) / unit;
      if (mine && (double)wi >= t && (tid == 0 || (double)(wi - w) < t)) sm.p_part[e] = tid;
    }
    __syncthreads();
    lo = r.k_in ? min(lo, sm.p_part[0]) : sm.p_part[0];
    if (!r.k_in) hi = sm.p_part[1];
  }
  if (mine && tid == lo) {
    sm.cnt_before = ci - c;
    sm.mass_before = wi - w;
  }
  Race drawn = race;
  uint64_t weight = sum;
  for (int s = wave / 4; s < a.NS; s += kFinish / kThreads) {
    float x[16];
    load16<BF16>(a, ls.row, s * kSampleSlice, tid % kThreads, x);
    uint32_t in = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) in |= (x[k] >= r.least && x[k] < r.below ? 1u : 0u) << k;
    while (in != 0) {  // (every lane its own)
      const int k = __builtin_ctz(in);
      in &= in - 1;
      float l = x[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) l = k == e ? x[e] : l;
      int step;
      float rest;
      const int j = min(max(ls.grid.place(l, step, rest) - ls.lo, 0), ls.hi - ls.lo), part = listed_place(j, step) >> r.sub;
      if (part > hi) continue;
      const int id = token_of<BF16>(s * kSampleSlice, tid % kThreads, k);
      const uint64_t wl = listed_weight(sm.table, step, rest, sm.factor[j], ls.scale);
      if (part >= lo) {
        const uint32_t i = atomicAdd(&sm.count, 1u);
        if (i < kStaged) {
          sm.list[i] = make_uint2(key_of(l), (uint32_t)id);
          sm.weight[i] = wl;
        }
        continue;
      }
      const double d = ((double)r.max - (double)l) * r.inv_T;
      if (d <= q.min_d) {
        weight += wl;
        const uint32_t xn = noise_bits(z0 + (uint64_t)(id + 1) * kGolden);
        drawn.enter(id, d, __builtin_amdgcn_rcpf(fmaxf((float)((double)wl * unit), 1e-14f)), xn, noise_rest(xn));
      }
    }
    drawn.share();
  }
  __syncthreads();
  ls.n = sm.count;
  if (ls.n > kStaged) return;
  race = drawn;
  sum = weight;
  r.above += (int)sm.cnt_before;
  r.mass += (double)sm.mass_before * unit;
}

// The digit at which `target` (a count, or a weight) is reached, from the highest
// down (UP: from the lowest up), with what comes before it.  False: never.
template <bool MASS, bool UP>
__device__ __forceinline__ bool find_digit(FinishSmem& sm, int tid, int& turn, uint64_t target) {
  __syncthreads();
  const int now = turn;
  turn ^= 1;
  if (tid >= 64)
    for (int i = tid - 64; i < 256; i += kFinish - 64) {
      sm.cnt[turn][i] = 0;
      sm.mass[turn][i] = 0;
    }
  if (tid < 64) {
    uint64_t v[4], s = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int b = UP ? 4 * tid + e : 255 - 4 * tid - e;
      v[e] = MASS ? sm.mass[now][b] : (uint64_t)sm.cnt[now][b];
      s += v[e];
    }
    const uint64_t in = prefix_sum(s);
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
      sm.cnt_in = sm.cnt[now][b];
    }
  }
  __syncthreads();
  return sm.digit >= 0;
}

// Among the listed tokens that `in` allows, the key at which the target is reached
// in descending order: the key, what is before it and how many tokens have it.  The
// keys' differences from the lowest are cut into digits of 8 bits, the highest first
// (the keys of a bin agree in their upper bits: digits of the keys themselves would
// count all tokens in one place).
struct Border {
  uint32_t key, ties;
  uint64_t before;
  bool found;
};
template <bool MASS, typename L, typename In>
__device__ __forceinline__ Border find_key(const L& ls, FinishSmem& sm, int tid, int& turn, uint64_t target, In in) {
  Border b{0u, 0u, 0u, true};
  const uint32_t base = sm.key_lo, span = sm.key_hi - base;
  int shift = max(0, 32 - __clz((int)span) - 8), last = 32;
#pragma unroll 1
  for (;;) {
    ls.each([&](int id, uint32_t key, auto w) {
      const uint32_t v = key - base;
      if (!in(id, key) || (last < 32 && v >> last != b.key)) return;
      const uint32_t dg = last < 32 ? v >> shift & ((1u << (last - shift)) - 1) : v >> shift;
      atomicAdd(&sm.cnt[turn][dg], 1u);
      if (MASS) atomicAdd((unsigned long long*)&sm.mass[turn][dg], (unsigned long long)w());
    });
    if (!find_digit<MASS, false>(sm, tid, turn, target)) {
      b.found = false;
      return b;
    }
    b.key = last < 32 ? b.key << (last - shift) | (uint32_t)sm.digit : (uint32_t)sm.digit;
    b.before += sm.before;
    target -= sm.before;
    b.ties = sm.cnt_in;
    if (shift == 0) break;
    last = shift;
    shift = max(0, shift - 8);
  }
  b.key += base;
  return b;
}

// The n-th lowest id (from 1) of the listed tokens with this key.
template <typename L>
__device__ __forceinline__ uint32_t find_id(const L& ls, FinishSmem& sm, int tid, int& turn, uint32_t key, uint32_t n) {
  uint32_t found = 0;
  uint64_t target = n;
#pragma unroll 1
  for (int shift = 16; shift >= 0; shift -= 8) {
    ls.each([&](int id, uint32_t k, auto) {
      if (k == key && (shift == 16 || ((uint32_t)id ^ found) >> (shift + 8) == 0)) atomicAdd(&sm.cnt[turn][(uint32_t)id >> shift & 255u], 1u);
    });
    if (!find_digit<false, true>(sm, tid, turn, target)) return 0xffffffffu;
    found |= (uint32_t)sm.digit << shift;
    target -= sm.before;
  }
  return found;
}

// Both borders of a short list at once: kPer lanes per token add up the counts and
// weights of the tokens from the first to it (one row with top_k and top_p: 8 us; digit
// by digit 16).
constexpr int kFew = 256, kPer = kFinish / kFew;
__device__ __forceinline__ uint64_t quad_sum(uint64_t v) {
  v += (uint64_t)__shfl_xor((unsigned long long)v, 1);
  return v + (uint64_t)__shfl_xor((unsigned long long)v, 2);
}
static_assert(kPer == 4, "quad_sum");
__device__ __forceinline__ void border_of_few(FinishSmem& sm, int tid, uint32_t n, const Request& q, const SampleRow& r,
                                              double unit, uint32_t& key, uint32_t& id_to) {
  const uint32_t i = (uint32_t)tid / kPer;
  const bool mine = i < n;
  const uint2 e = sm.list[mine ? i : 0];
  uint64_t sum = 0;
  uint32_t count = 0;
  if (mine)
    for (uint32_t j = tid % kPer; j < n; j += kPer) {
      const uint2 o = sm.list[j];
      const uint64_t w = sm.weight[j];
      const bool before = o.x > e.x || (o.x == e.x && o.y <= e.y);
      count += before ? 1u : 0u;
      sum += before ? w : 0ull;
    }
  count = (uint32_t)quad_sum(count);
  sum = quad_sum(sum);
  const bool teller = mine && tid % kPer == 0;
  const uint32_t last = r.k_in ? min((uint32_t)(q.top_k - r.above), n) : n;
  if (teller && count == last) {
    sm.key_lo = e.x;
    sm.key_hi = e.y;
    sm.total = sum;
  }
  __syncthreads();
  if (r.k_in) {
    key = sm.key_lo;
    id_to = sm.key_hi;
  }
  if (!q.use_p) return;
  const double total = r.k_in ? r.mass + (double)sm.total * unit : r.total;
  const uint64_t target = (uint64_t)fmax(ceil(((q.top_p - kSlack) * total - r.mass) / unit), 1.0);
  const bool reached = sm.total >= target;
  __syncthreads();
  if (teller && count <= last && sum >= target && sum - sm.weight[i] < target) {
    sm.key_lo = e.x;
    sm.key_hi = e.y;
  }
  __syncthreads();
  if (reached) {
    key = sm.key_lo;
    id_to = sm.key_hi;
  }
}

// The same for more: digit by digit.
template <typename L>
__device__ __forceinline__ void border_of_many(const L& ls, FinishSmem& sm, int tid, const Request& q, const SampleRow& r,
                                               double unit, uint32_t& key, uint32_t& id_to) {
  uint32_t lo = 0xffffffffu, hi = 0u;
  ls.each([&](int, uint32_t k, auto) {
    lo = min(lo, k);
    hi = max(hi, k);
  });
  if (tid == 0) {
    sm.key_lo = 0xffffffffu;
    sm.key_hi = 0;
    sm.total = 0;
  }
  int turn = 0;
  if (tid < 256) {
    sm.cnt[0][tid] = 0;
    sm.mass[0][tid] = 0;
  }
  __syncthreads();
  lo = from_lane(all_lanes(lo, [](uint32_t x, uint32_t y) { return min(x, y); }), 63);
  hi = from_lane(all_lanes(hi, [](uint32_t x, uint32_t y) { return max(x, y); }), 63);
  if ((tid & 63) == 0 && lo <= hi) {
    atomicMin(&sm.key_lo, lo);
    atomicMax(&sm.key_hi, hi);
  }
  __syncthreads();
  if (sm.key_lo > sm.key_hi) return;  // nothing listed
  double total = r.total;
  if (r.k_in) {
    const uint32_t n = (uint32_t)(q.top_k - r.above);
    const Border b = find_key<false>(ls, sm, tid, turn, n, [](int, uint32_t) { return true; });
    if (b.found) {
      key = b.key;
      if (n - (uint32_t)b.before < b.ties) id_to = find_id(ls, sm, tid, turn, key, n - (uint32_t)b.before);
    }
    if (q.use_p) {  // the weight of the first top_k
      uint64_t mine = 0;
      ls.each([&](int id, uint32_t k, auto w) {
        if (k > key || (k == key && (uint32_t)id <= id_to)) mine += w();
      });
      atomicAdd((unsigned long long*)&sm.total, (unsigned long long)mine);
      __syncthreads();
      total = r.mass + (double)sm.total * unit;
    }
  }
  if (q.use_p) {
    const uint64_t target = (uint64_t)fmax(ceil(((q.top_p - kSlack) * total - r.mass) / unit), 1.0);
    const uint32_t k_key = key, k_id = id_to;
    const Border b = find_key<true>(ls, sm, tid, turn, target, [&](int id, uint32_t k) {
      return k > k_key || (k == k_key && (uint32_t)id <= k_id);
    });
    if (b.found) {
      key = b.key;
      // as many of the equal tokens as it takes, in their order
      const uint64_t w = ls.weight(logit_of(key));
      const uint64_t need = w > 0 ? (target - b.before + w - 1) / w : b.ties;
      const uint32_t n = (uint32_t)(need < 1 ? 1 : need > b.ties ? b.ties : need);
      if (b.key != k_key) id_to = 0xffffffffu;
      if (n < b.ties) id_to = find_id(ls, sm, tid, turn, key, n);
    }
  }
}

// The row's border (key, id) among its listed tokens, and their part in the draw.
template <typename L>
__device__ __forceinline__ void finish_list(const L& ls, FinishSmem& sm, int tid, const Request& q, const SampleRow& r,
                                            uint64_t z0, double unit, uint32_t& key, uint32_t& id_to, Race& race,
                                            uint64_t& sum) {
  if (ls.n == 0) return;
  if (ls.n <= kFew)
    border_of_few(sm, tid, ls.n, q, r, unit, key, id_to);
  else
    border_of_many(ls, sm, tid, q, r, unit, key, id_to);
  ls.each([&](int id, uint32_t k, auto weight) {
    if (!(k > key || (k == key && (uint32_t)id <= id_to))) return;
    const double d = ((double)r.max - (double)logit_of(k)) * r.inv_T;
    if (d > q.min_d) return;
    const uint64_t w = weight();
    sum += w;
    const uint32_t xn = noise_bits(z0 + (uint64_t)(id + 1) * kGolden);
    race.enter(id, d, __builtin_amdgcn_rcpf(fmaxf((float)((double)w * unit), 1e-14f)), xn, noise_rest(xn));
  });
}

template <bool BF16>
__global__ void __launch_bounds__(kFinish) sample_finish_kernel(SampleArgs a) {
  __shared__ FinishSmem sm;
  constexpr int W = kFinish / 64;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Request q = request_of(a, row);
  const SampleRow r0 = a.row[row];
  const uint32_t n = a.count[row];
  // (asked for before it is known whether they are used: the list holds kFinish entries, written or not)
  const uint2 entry = a.list[(int64_t)row * kSampleList + tid];
  const double step = kTables.step[tid & (kSteps - 1)], rel = kTables.rel[tid & (kSampleBins - 1)];
  // the row's maximum
  const float ms = tid < a.NS ? a.smax[(int64_t)row * a.NS + tid] : -INFINITY;
  const float m0 = wave_max(ms);
  if (lane == 0) sm.wm[wave] = m0;
  __syncthreads();
  float M = sm.wm[0];
  for (int w = 1; w < W; ++w) M = fmaxf(M, sm.wm[w]);
  if (M == -INFINITY || q.greedy) {
    int id = 0x7fffffff;
    if (q.greedy && ms == M && tid < a.NS) id = a.sarg[(int64_t)row * a.NS + tid];
    id = wave_min(id);
    if (lane == 0) sm.wi[wave] = id;
    __syncthreads();
    if (tid == 0) {
      for (int w = 0; w < W; ++w) id = min(id, sm.wi[w]);
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
  SampleRow r = r0;
  const uint64_t z0 = (uint64_t)__float_as_uint(a.u[row]);
  Race race;
  Draw best = kNoDraw;  // of the earlier passes
  // weights of the kept tokens: the earlier passes', and of the list, whose order changes from
  // call to call, as integers of `unit`
  double sum = 0.0, unit = 0.0;
  uint64_t in_list = 0;
  uint32_t key = 0, id_to = 0xffffffffu;
  if (q.listed()) {
    Tokens<BF16> ls{a, sm, row, tid, n, (double)M, r.inv_T, Grid(r.inv_T, M), r.lo, r.hi, power_of_2(r.bits)};
    ls.stage(entry, step, rel);
    unit = kTables.edge[min(r.lo, kSampleBins - 1)] * top_scale(ls.grid, sm.table, r.max) * power_of_2(-r.bits);
    if (r.tail) r.total += (double)a.tail[row] * 0x1p-38 * (kTables.edge[kLastBin] * top_scale(ls.grid, sm.table, r.max));
    if (r.sub >= 0) narrow(ls, sm, tid, q, r, z0, unit, race, in_list);
    finish_list(ls, sm, tid, q, r, z0, unit, key, id_to, race, in_list);
  }
  if (q.plain()) {
    // the slices' own draws, relative to their maxima
    r = SampleRow{};
    r.max = M;
    r.inv_T = row_inv_T(q.inv_T, M);
    const double d = ((double)M - (double)ms) * r.inv_T;
    if (tid < a.NS && ms > -INFINITY && d <= kSpan) {
      const int64_t at = (int64_t)row * a.NS + tid;
      best = a.best[at];
      best.s -= d;
      best.d += d;
      sum = a.sum[at] * exp(-d);
    }
  } else if (tid * a.spw < a.NS) {  // the second pass's
    const int64_t at = (int64_t)row * a.NS + tid;
    best = a.best[at];
    sum = a.sum[at];
  }
  best = better_draw(wave_draw(best), race.best());
  sum = wave_sum(sum);
  in_list = from_lane(prefix_sum(in_list), 63);
  if (lane == 0) {
    sm.wd[wave] = best;
    sm.ws[wave] = sum;
    sm.wl[wave] = in_list;
  }
  __syncthreads();
  if (wave != 0) return;
  best = wave_draw(lane < W ? sm.wd[lane] : kNoDraw);
  in_list = from_lane(prefix_sum(lane < W ? sm.wl[lane] : (uint64_t)0), 63);
  sum = wave_sum(lane < W ? sm.ws[lane] : 0.0) + (double)in_list * unit;
  if (lane == 0) {
    a.tokens[row] = min(best.id, a.V - 1);
    if (a.chosen != nullptr) a.chosen[row] = (float)(exp(-best.d) / sum);
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
  hipLaunchKernelGGL((sample_finish_kernel<BF16>), dim3((unsigned)a.rows), dim3(kFinish), 0, st, a);
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
  uint8_t* best = take(R * NS * sizeof(SampleDraw));
  uint8_t* sum = take(R * NS * 8);
  uint8_t* row = take(R * sizeof(SampleRow));
  uint8_t* count = take(R * 4);
  uint8_t* tail = take(R * 8);
  uint8_t* list = take(R * kSampleList * 8);
  uint8_t* sub_mass = take(R * kSampleSub * 8);
  uint8_t* sub_count = take(R * kSampleSub * 4);
  if (a != nullptr) {
    a->smax = (float*)smax;
    a->sarg = (int32_t*)sarg;
    a->hist = (uint64_t*)hist;
    a->best = (SampleDraw*)best;
    a->sum = (double*)sum;
    a->row = (SampleRow*)row;
    a->count = (uint32_t*)count;
    a->tail = (uint64_t*)tail;
    a->list = (uint2*)list;
    a->sub_mass = (uint64_t*)sub_mass;
    a->sub_count = (uint32_t*)sub_count;
  }
  return off;
}

hipError_t launch_sample(const SampleArgs& in, hipStream_t st) {
  SampleArgs a = in;
  a.NS = (a.V + kSampleSlice - 1) / kSampleSlice;
  // Every part reads the row's bins (1 KB a slice): few rows take many parts, many rows few.
  // 400 rows of 32 slices: 20 parts a row 51 us, 10 41, 5 55, 2 96.
  const int parts = std::max(1, std::min({kSampleParts, a.NS, 4096 / a.rows}));
  a.spw = (a.NS + parts - 1) / parts;
  a.NW = (a.NS + a.spw - 1) / a.spw;
  return a.bf16 ? sample_t<true>(a, st) : sample_t<false>(a, st);
}

}  // namespace spade
