// A token per row of logits by temperature, top-k, top-p and min-p (harli_sample).
//
// All three filters keep the first tokens in the order of (logit, then lower index), so what stays is a cut: a logit, and the last index
// among the tokens that have just this logit.  Two launches:
//   k_sample_stretch  reads the logits once, kStretch of a row per workgroup, all in registers: their maximum, the sum of their weights
//                     (relative to that maximum) and, where a filter asks for it, tokens and weights by bins of the logit;
//   k_sample_row      one workgroup per row: puts the stretches together, finds the bin that a cut falls into, fetches the tokens of that
//                     bin (only from stretches that have some) and settles the cut among them in LDS; then the stretch that the random
//                     number points at, and the token in it.
// Weights are exp in 64 bits rounded to fixed point, so sums by atomics are the same in any order; stretches are joined in 64-bit floating
// point in a fixed order.  A row's result depends neither on the batch nor on scheduling.
// What bounds it, 256 rows of 152064 logits: the first launch reads them in 25.3 us (6.2 TB/s) when it takes the maximum alone; the
// exponential in 64 bits makes that 40.7, the bins 49.  The second takes 42, most of it for the tokens of the cut's bin: nearly every
// stretch has some and is read again.  One row of 32000: 5.4 and 18 us, latency and a cold instruction cache.
#include <mutex>

#include "ctx.h"
#include "device_utils.h"
#include "scan_utils.h"

namespace harli {
namespace {

// tokens per workgroup of the first launch: 16 per thread (8192, half the bins to write and join: no gain there, the row's launch slower,
// 128 rows of 128256 28.2 us instead of 24.6)
constexpr int kStretch = 4096;
constexpr int kMostVocab = 1 << 20;
constexpr int kMostStretches = kMostVocab / kStretch;
constexpr int kLogitBins = 256;     // of a stretch, downwards from its maximum
constexpr int kCandidates = 8192;   // tokens of one bin that the second launch holds in LDS
constexpr int kDigits = 2048;       // bins of a search: 11 bits
constexpr int kRowThreads = 1024, kRowWaves = kRowThreads / 64;
constexpr double kOne = (double)(1ull << 50);  // weight 1 in fixed point: 2^13 of them fit 64 bits

// Order of the logits as unsigned integers; both zeros alike.
__device__ __forceinline__ unsigned order_key(float v) {
  const unsigned u = __float_as_uint(v + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float order_value(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ bool usable(float v) { return v > -INFINITY; }  // (not NaN either)

// 2^(j / 64), by the series of exp (constant expressions: the compiler's own doubles)
constexpr int kPowersN = 64;
constexpr double kLn2 = 0.693147180559945309417;
constexpr double exp_series(double x) {
  double sum = 1, term = 1;
  for (int i = 1; i < 24; ++i) term = term * x / i, sum += term;
  return sum;
}
struct Powers {
  double v[kPowersN], down[kPowersN];  // 2^(j / 64), 2^(-j / 64)
};
constexpr Powers make_powers() {
  Powers t{};
  for (int j = 0; j < kPowersN; ++j) t.v[j] = exp_series(kLn2 * j / kPowersN), t.down[j] = exp_series(-kLn2 * j / kPowersN);
  return t;
}
__constant__ Powers kPowers = make_powers();

// 2^((n + f) / 64), n a whole number, |f| <= 1/2: n = 64 e + j; the table's 2^(j / 64) times the series of exp(f ln 2 / 64) to the fourth
// power (what follows is below 2^-44).  The coefficients come as kernel arguments, that is as scalar operands: as immediates every one
// of them is moved into registers for every token.
struct Series {
  double c1, c2, c3, c4;
};
constexpr Series kSeries = {kLn2 / 64, kLn2 / 64 * (kLn2 / 64) / 2, kLn2 / 64 * (kLn2 / 64) * (kLn2 / 64) / 6,
                            kLn2 / 64 * (kLn2 / 64) * (kLn2 / 64) * (kLn2 / 64) / 24};
struct Exp {
  Series s;
  const double* powers;  // the table in LDS
  __device__ __forceinline__ double at(int n, double f) const {
    const double p = fma(fma(fma(fma(s.c4, f, s.c3), f, s.c2), f, s.c1), f, 1.0);
    return __builtin_amdgcn_ldexp(p * powers[n & (kPowersN - 1)], n >> 6);
  }
  __device__ __forceinline__ double at(double t) const {
    const double n = rint(t);
    return at((int)n, t - n);  // (far below the range it saturates: zero)
  }
  // weight of a usable logit relative to `top`, which is not infinite; per_t = 64 log2(e) / temperature
  __device__ __forceinline__ double weight(float v, float top, double per_t) const { return at(((double)v - (double)top) * per_t); }
  __device__ __forceinline__ u64 fixed(float v, float top, double per_t) const { return fixed_of(weight(v, top, per_t)); }
  // kOne stands for 1 (and w <= 1): beside 4 the last bit of a number is 2^-50
  static __device__ __forceinline__ u64 fixed_of(double w) { return (u64)__double_as_longlong(w + 4.0) & ((1ull << 52) - 1); }
};
// A row with logits of +inf is one of them alone, at zero.
__device__ __forceinline__ float finite_row(float v) { return v == INFINITY ? 0.f : -INFINITY; }
// Where a logit lies, in 64ths of a power of two of its weight: v * per_t, rounded to a whole number.  A bin is 2^shift of them, on a grid
// common to all stretches: an eighth to a sixteenth of the logit's unit, so that 256 bins span 16 units at least and one holds a
// few per cent of a vocabulary at most (bins are wider above a temperature of 5, and span less below one of 1/22).
__device__ __forceinline__ int bin_shift(float t) { return max(1, min(7, ilogbf(11.54f / t))); }  // 2^shift * t ln(2) / 64 <= 1/8
// Beside 3 * 2^51 the last bit of a number is 1, also with an even number added: what a sum there rounds to does not depend on the latter.
constexpr double kWholes = 3.0 * (double)(1ull << 51);
__device__ __forceinline__ double whole_of(float v, double per_t) { return fma((double)v, per_t, kWholes) - kWholes; }
// the border of the grid at or above it
__device__ __forceinline__ double ceiling_of(float top, double per_t, int shift) {
  return __builtin_amdgcn_ldexp(ceil(__builtin_amdgcn_ldexp(whole_of(top, per_t), -shift)), shift);
}
// Whole numbers are exact below 2^53.  A row whose largest logit is further away than 2^43 is searched and summed up by its differences
// from that logit; a stretch whose largest is further than 2^44 weighs nothing in any other row.
constexpr double kFarRow = (double)(1ull << 43), kFarStretch = (double)(1ull << 44);

constexpr double kPerT = 64 * 1.4426950408889634074;
struct RowSettings {
  float t, p;
  double min_p;
  int k;  // 0: off
  bool greedy, cut;
};
__device__ __forceinline__ RowSettings settings_of(const harli_sample_batch& a, int b) {
  RowSettings s;
  s.t = a.temperature ? a.temperature[b] : 1.f;
  s.greedy = !(s.t > 0.f);
  s.k = a.top_k ? a.top_k[b] : 0;
  if (s.k < 0 || s.k >= a.vocab) s.k = 0;
  s.p = a.top_p ? a.top_p[b] : 1.f;
  if (!(s.p < 1.f)) s.p = 1.f;
  const float m = a.min_p ? a.min_p[b] : 0.f;
  s.min_p = m > 1.f ? 1.0 : m > 0.f ? (double)m : 0.0;
  s.cut = !s.greedy && (s.k > 0 || s.p < 1.f || s.min_p > 0.0);
  return s;
}

// Workspace, by row and stretch.
struct SampleWs {
  float* top;        // largest logit
  unsigned* usable;  // tokens that can be drawn
  double* weight;      // sum of their weights, in fixed point relative to the largest
  double* upto_weight;         // [kLogitBins] weights of the bins up to each one
  unsigned short* upto_count;  // [kLogitBins] tokens of them
  int n;             // stretches per row
};

constexpr int kStretchThreads = 256, kPer = kStretch / kStretchThreads;

__global__ void __launch_bounds__(kStretchThreads) k_sample_stretch(harli_sample_batch a, SampleWs ws, Series series) {
  __shared__ float s_top[4];
  __shared__ u64 s_weight[4], bin_weight[kLogitBins];
  __shared__ double powers[kPowersN];
  __shared__ unsigned s_n[4], bin_count[kLogitBins];
  const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, first = blockIdx.x * kStretch;
  const float* z = a.logits + (size_t)b * a.ld + first;
  const int n = min(kStretch, a.vocab - first);
  float v[kPer];
  if (n == kStretch && (uintptr_t)z % 16 == 0) {  // which thread has which token does not matter here
#pragma unroll
    for (int i = 0; i < kPer / 4; ++i) {
      const float4 x = reinterpret_cast<const float4*>(z)[i * kStretchThreads + tid];
      v[4 * i] = x.x, v[4 * i + 1] = x.y, v[4 * i + 2] = x.z, v[4 * i + 3] = x.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = z[min(i * kStretchThreads + tid, n - 1)];
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = i * kStretchThreads + tid < n ? v[i] : -INFINITY;
  }
  const RowSettings s = settings_of(a, b);
  bin_weight[tid] = 0, bin_count[tid] = 0;
  if (tid < kPowersN) powers[tid] = kPowers.down[tid];
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < kPer; ++i) top = fmaxf(top, v[i]);  // (NaN is the other operand)
  top = wave_top(top);
  if (lane == 0) s_top[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
  const size_t at = (size_t)b * ws.n + blockIdx.x;
  if (tid == 0) ws.top[at] = top;
  if (s.greedy) return;
  const bool infinite = top == INFINITY;
  if (infinite) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = finite_row(v[i]);
    top = 0.f;
  }
  const double per_t = kPerT / (double)s.t;
  const int shift = bin_shift(s.t);
  const double ceiling = ceiling_of(top, per_t, shift);
  const bool far = !(fabs(ceiling) < kFarStretch);
  u64 sum = 0;
  unsigned count = 0;
  // Logits below the bins and below all weights (2^-60) are taken as the one at that border, or the next below it that is a float.
  // This is the loop that the launch's time goes into: conversions between 64-bit floating point and integers, and ldexp, are slow beside sums and products, hence the sums beside
  // kWholes and the exponent added as bits.
  const int deepest = max(60 * 64, kLogitBins << shift) + 64;  // wholes; 2^-513 at most
  const double border = (ceiling - (double)deepest) / per_t;
  const float nearest = (float)border, least = border > -3e38 ? ((double)nearest <= border ? nearest : nextafterf(nearest, -INFINITY)) : -INFINITY;
  const double wholes = kWholes + ceiling;
  double c3 = series.c3;
  asm("" : "+v"(c3));  // (one scalar operand per instruction)
  auto add = [&](float x, bool masked) {
    x = __builtin_amdgcn_fmed3f(x, least, INFINITY);  // (least for NaN too)
    const double d = (double)x, y = fma(d, -per_t, wholes), f = fma(d, per_t, y - wholes);
    const unsigned below = min((unsigned)(u64)__double_as_longlong(y), (unsigned)deepest);  // wholes below the ceiling
    const double p = fma(fma(fma(fma(series.c4, f, c3), f, series.c2), f, series.c1), f, 1.0) * powers[below & (kPowersN - 1)];
    u64 w = Exp::fixed_of(__hiloint2double(__double2hiint(p) - (int)((below << 14) & 0xfff00000u), __double2loint(p)));
    if (masked && x == -INFINITY) w = 0;
    sum += w;
    if (s.cut) {
      const unsigned bin = below >> shift;
      if (bin < kLogitBins && !(masked && x == -INFINITY)) {
        atomicAdd(&bin_weight[bin], w);
        if (s.k) atomicAdd(&bin_count[bin], 1u);
      }
    }
  };
  if (least > -INFINITY) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) add(v[i], false);
  } else {  // a temperature at which no logit is too small
#pragma unroll 1
    for (int i = 0; i < kStretch; i += kStretchThreads)
      if (i + tid < n) {
        const float x = z[i + tid];
        add(infinite ? finite_row(x) : x, true);
      }
  }
  if (s.k) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) count += usable(v[i]);
  }
  if (far) sum = 0;
  sum = wave_scan(sum);
  count = wave_scan(count);
  if (lane == 63) s_weight[wave] = sum, s_n[wave] = count;
  __syncthreads();
  if (tid == 0) {
    ws.weight[at] = (double)(s_weight[0] + s_weight[1] + s_weight[2] + s_weight[3]);
    ws.usable[at] = s_n[0] + s_n[1] + s_n[2] + s_n[3];
  }
  if (s.cut) {
    static_assert(kLogitBins == kStretchThreads, "a bin per thread");
    u64 w = wave_scan(far ? 0 : bin_weight[tid]);
    unsigned c = wave_scan(far ? 0 : bin_count[tid]);
    __syncthreads();
    if (lane == 63) s_weight[wave] = w, s_n[wave] = c;
    __syncthreads();
    for (int x = 0; x < wave; ++x) w += s_weight[x], c += s_n[x];
    ws.upto_weight[at * kLogitBins + tid] = (double)w;
    if (s.k) ws.upto_count[at * kLogitBins + tid] = (unsigned short)c;
  }
}

// ---- the second launch -----------------------------------------------------------------------------------------------------------
// Its steps are short and depend on one another, so what it costs is their latency, and its own code: a launch finds the instruction cache
// cold.  The three searches (for top-k, for top-p, for the last of equal logits) are therefore one loop around one search.
constexpr int kPart = 1024;                        // tokens that a wave looks through at a time for those of a bin
constexpr int kListed = kCandidates / kRowWaves;   // tokens of the bin a wave can hold: every wave has a list of its own

struct RowShared {
  u64 digit[kDigits];
  double powers[kPowersN];
  uint2 listed[kCandidates];      // (key, index)
  float top[kMostStretches];
  int below[kMostStretches];      // bins from the row's first to the stretch's
  double scale[kMostStretches];   // of the stretch's sums to the row's, which are relative to its largest logit
  double kept[kMostStretches];
  u64 inside[kMostStretches];     // kept weight of the cut's own bin, in the row's fixed point
  double upto_weight[kLogitBins];  // of the row's bins up to each one
  unsigned upto_count[kLogitBins];
  unsigned char some[kMostStretches];  // whether the stretch has tokens of the bin
  double part[kRowThreads / kLogitBins][kLogitBins];
  unsigned part_n[kRowThreads / kLogitBins][kLogitBins];
  u64 tmp[kRowWaves];
  float wave_f[kRowWaves];
  u64 found_above;
  unsigned found;
  int least;
  unsigned overflow;  // a wave's list did not hold its tokens
};

// Sum of v up to and with this thread's, and over all (whole workgroup); the order of the additions is fixed.
template <typename T>
__device__ __forceinline__ T block_scan(T v, RowShared& sh, int lane, int wave, T& all) {
  static_assert(kRowWaves <= 16, "the waves' sums in a row of lanes");
  v = wave_scan(v);
  __syncthreads();
  T* tmp = reinterpret_cast<T*>(sh.tmp);
  if (lane == 63) tmp[wave] = v;
  __syncthreads();
  const T t = row_scan(lane < kRowWaves ? tmp[lane] : T(0));
  all = lane_value(t, kRowWaves - 1);
  const T before = lane_value(t, wave ? wave - 1 : 0);
  return wave ? before + v : v;
}
template <typename T>
__device__ __forceinline__ T all_sum(T v, RowShared& sh, int lane, int wave) {
  T all;
  (void)block_scan(v, sh, lane, wave, all);
  return all;
}

// Among the items i = from, from + step, .. < end of every thread, key(i) and amount(i) (0: not looked at): the key at which the amounts of
// higher keys are less than `want` and with its own not; `want` becomes what is missing above it (a want beyond the whole counts as the
// whole).  Keys are below 2^bits.
template <typename Key, typename Amount>
__device__ __forceinline__ unsigned find_key(int from, int end, int step, int bits, Key key, Amount amount, u64& want, RowShared& sh,
                                             int tid, int lane, int wave) {
  unsigned prefix = 0;
#pragma unroll 1
  while (bits > 0) {
    const int width = min(bits, 11), shift = bits - width;
    constexpr int DPT = kDigits / kRowThreads;  // digits per thread
#pragma unroll
    for (int i = 0; i < DPT; ++i) sh.digit[tid * DPT + i] = 0;
    __syncthreads();
#pragma unroll 1
    for (int i = from; i < end; i += step) {
      const unsigned k = key(i);
      if (bits == 32 || (k >> bits) == (prefix >> bits)) {
        const u64 w = amount(i);
        if (w) atomicAdd(&sh.digit[kDigits - 1 - ((k >> shift) & ((1u << width) - 1))], w);  // the highest first
      }
    }
    __syncthreads();
    u64 h[DPT], sum = 0, all;
#pragma unroll
    for (int i = 0; i < DPT; ++i) h[i] = sh.digit[tid * DPT + i], sum += h[i];
    u64 above = block_scan(sum, sh, lane, wave, all) - sum;
    want = min(want, all);
    if (above < want && above + sum >= want) {
#pragma unroll
      for (int i = 0; i < DPT; ++i) {
        if (above < want && above + h[i] >= want) sh.found = kDigits - 1 - (tid * DPT + i), sh.found_above = above;
        above += h[i];
      }
    }
    if (tid == 0 && all == 0) sh.found = 0, sh.found_above = 0;
    __syncthreads();
    want -= sh.found_above;
    prefix |= sh.found << shift;
    bits = shift;
  }
  return prefix;
}

// The smallest key that `enough` holds for, which it does from some key up to `hi` (and not for keys of NaN): 64 keys at a time, first those
// around a guess.  A wave's work, the same in all of them.
template <typename Enough>
__device__ __forceinline__ unsigned smallest_key(Enough enough, float guess, unsigned hi, int lane) {
  unsigned lo = 0, step = 1, at = order_key(guess) - 33;  // keys at + step * (1, 2, .. 64)
#pragma unroll 1
  while (true) {
    const u64 k = (u64)at + (u64)step * (lane + 1);
    const u64 m = __ballot(k >= hi || enough((unsigned)k));
    const int i = m ? __ffsll(m) - 1 : 64;
    if (i < 64) hi = min(hi, at + step * (i + 1));
    if (i > 0) lo = max(lo, at + step * i);
    if (hi - lo <= 1) return hi;
    step = (hi - lo + 63) / 64, at = lo;
  }
}

__global__ void __launch_bounds__(kRowThreads) k_sample_row(harli_sample_batch a, SampleWs ws, Series series) {
  extern __shared__ __align__(16) char row_lds[];
  RowShared& sh = *reinterpret_cast<RowShared*>(row_lds);
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), V = a.vocab, NS = ws.n;
  const float* z = a.logits + (size_t)b * a.ld;
  const size_t at0 = (size_t)b * NS;
  const RowSettings s = settings_of(a, b);

  // ---- the stretches together ----------------------------------------------------------------------------------------------------
  float mine = tid < NS ? ws.top[at0 + tid] : -INFINITY;
  float top = wave_top(mine);
  if (lane == 0) sh.wave_f[wave] = top;
  if (tid < kPowersN) sh.powers[tid] = kPowers.v[tid];
  if (tid == 0) sh.found = 0xffffffffu, sh.least = NS;
  __syncthreads();
  top = wave_top(lane < kRowWaves ? sh.wave_f[lane] : -INFINITY);
  if (top == -INFINITY) {
    if (tid == 0) {
      a.token[b] = -1;
      if (a.logprob) a.logprob[b] = -INFINITY;
    }
    return;
  }
  if (s.greedy) {
    if (mine == top) atomicMin(&sh.least, tid);
    __syncthreads();
    const int first = sh.least * kStretch;
    for (int i = first + tid; i < min(V, first + kStretch); i += kRowThreads)
      if (z[i] == top) atomicMin(&sh.found, (unsigned)i);
    __syncthreads();
    if (tid == 0) {
      a.token[b] = (int)sh.found;
      if (a.logprob) a.logprob[b] = 0.f;
    }
    return;
  }
  const bool infinite = top == INFINITY;  // uniform
  auto logit = [&](int i) { return infinite ? finite_row(z[i]) : z[i]; };
  if (infinite) mine = finite_row(mine), top = 0.f;
  const double per_t = kPerT / (double)s.t;
  const Exp ex{series, sh.powers};
  const int shift = bin_shift(s.t);
  const double ceiling = ceiling_of(top, per_t, shift);
  const bool far = !(fabs(ceiling) < kFarRow);  // uniform
  auto bin_of = [&](unsigned key) {             // of the row
    const double n = __builtin_amdgcn_ldexp(ceiling - whole_of(order_value(key), per_t), -shift);
    return n < (double)kLogitBins ? (int)n : kLogitBins;  // (keys of NaN: none)
  };
  double whole_mine = 0;
  if (tid < NS) {
    const bool some = usable(mine) && !far;
    const double own = ceiling_of(mine, per_t, shift), steps = __builtin_amdgcn_ldexp(ceiling - own, -shift);
    const double scale = some ? ex.at(fma(-(double)top, per_t, own)) : 0.0;  // of the stretch's sums, which are relative to its ceiling
    sh.top[tid] = mine;
    sh.below[tid] = some && steps < (double)kLogitBins ? (int)steps : kLogitBins;
    sh.scale[tid] = scale;
    whole_mine = some ? ws.weight[at0 + tid] * scale : 0.0;
    sh.kept[tid] = whole_mine;
  }
  auto row_weight = [&](unsigned key) { return ex.fixed(order_value(key), top, per_t); };

  // ---- the cut: logits with keys above t_key stay, and of those equal to it the ones up to index last ----------------------------
  unsigned t_key = 0, last = 0xffffffffu;
  int held = -1;  // the bin whose tokens are in LDS, and this wave's number of them
  int listed = 0;
  unsigned bin_first = 0, bin_keys = 0;  // its smallest key, and how many there are to the next bin's
  bool in_lds = false;
  if (s.cut) {
    if (far) {
      for (int i = tid; i < V; i += kRowThreads)
        if (usable(logit(i))) whole_mine += (double)row_weight(order_key(logit(i)));
    }
    double among = all_sum(whole_mine, sh, lane, wave);  // weight of the tokens that top-k leaves, in the row's fixed point
    // Bits that a search of the whole row drops from every weight, so that the sum of all fits 63: none up to 2^13 times the largest weight,
    // 8 at most.  All tokens together lose less than 2^-42 of their sum by it (with 8 dropped from every row's, a tail of light tokens
    // behind a heavy one lost a part of itself, and top-p near 1 kept too many of it).
    const int wide = max(0, __builtin_amdgcn_frexp_exp(among) - 63);
    {  // bins of the row
      constexpr int NG = kRowThreads / kLogitBins;
      const int g = tid & (kLogitBins - 1), grp = tid / kLogitBins;
      double m = 0;
      unsigned c = 0;
      constexpr int U = 10;  // stretches of a thread in flight
#pragma unroll 1
      for (int i0 = grp; i0 < NS; i0 += U * NG) {
        double x[U];
        unsigned n[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = min(i0 + u * NG, NS - 1);
          const size_t e = (at0 + i) * kLogitBins + max(g - sh.below[i], 0);
          x[u] = ws.upto_weight[e];
          n[u] = s.k ? ws.upto_count[e] : 0;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = min(i0 + u * NG, NS - 1);
          const bool in = i0 + u * NG < NS && g >= sh.below[i];
          m += in ? x[u] * sh.scale[i] : 0.0;
          c += in ? n[u] : 0;
        }
      }
      sh.part[grp][g] = m, sh.part_n[grp][g] = c;
      __syncthreads();
      if (tid < kLogitBins) {
        m = 0, c = 0;
#pragma unroll
        for (int x = 0; x < NG; ++x) m += sh.part[x][tid], c += sh.part_n[x][tid];
        sh.upto_weight[tid] = m, sh.upto_count[tid] = c;
      }
      __syncthreads();
    }
    u64 ties = ~0ull;  // how many of the tokens equal to t_key stay
#pragma unroll 1
    for (int phase = 0; phase < 3; ++phase) {
      int bin = kLogitBins;  // that the phase looks into; kLogitBins: none of them, it looks through the row
      u64 want = 0;
      double want_d = 0;
      if (phase == 0) {  // top-k
        if (!s.k) continue;
        if ((u64)s.k >= all_sum((u64)(tid < NS && usable(mine) ? ws.usable[at0 + tid] : 0), sh, lane, wave)) continue;  // (as many as there are)
        want = s.k;
        if (tid < kLogitBins) {
          const unsigned upto = sh.upto_count[tid], before = tid ? sh.upto_count[tid - 1] : 0;
          if (before < want && upto >= want) sh.found = tid, sh.found_above = before;
        }
        __syncthreads();
        if (want <= sh.upto_count[kLogitBins - 1]) bin = sh.found;
      } else if (phase == 1) {  // top-p
        if (!(s.p < 1.f)) continue;
        want_d = fmax((double)s.p * among, 1.0);  // (the first token in any case)
        __syncthreads();
        if (tid == 0) sh.found = kLogitBins;
        __syncthreads();
        if (tid < kLogitBins && sh.upto_weight[tid] >= want_d) atomicMin(&sh.found, (unsigned)tid);
        __syncthreads();
        bin = sh.found;
      } else {  // the cut's own bin, for the last of equal logits and for the weights
        if (s.min_p > 0.0) {
          const unsigned hi = smallest_key([&](unsigned k) { return ex.weight(order_value(k), top, per_t) >= s.min_p; },
                                           top + s.t * logf((float)s.min_p), order_key(top), lane);
          if (hi > t_key) t_key = hi, ties = ~0ull;
        }
        if (!t_key) break;
        bin = bin_of(t_key);
      }
      if (far || infinite) bin = kLogitBins;

      // ---- the tokens of the bin, in LDS (their order there is of no account)
      if (bin < kLogitBins && bin != held) {
        held = bin;
        listed = 0;
        __syncthreads();
        if (tid == 0) sh.overflow = 0;
        if (tid < NS) {
          const int j = bin - sh.below[tid];
          const size_t e = (at0 + tid) * kLogitBins + max(j, 0);
          bool some = j >= 0;
          if (j > 0) some = s.k ? ws.upto_count[e] != ws.upto_count[e - 1] : ws.upto_weight[e] != ws.upto_weight[e - 1];
          sh.some[tid] = some;
        }
        __syncthreads();
        // the logits of the bin: from the smallest in it (or above) to the smallest above it
        float border[2];
        unsigned border_key[2];
#pragma unroll 1
        for (int above = 0; above < 2; ++above)
          border_key[above] = smallest_key([&](unsigned k) { return bin_of(k) <= bin - above; },
                                           (float)((ceiling + 0.5 - (double)((bin + 1 - above) << shift)) / per_t), order_key(INFINITY), lane);
        bin_first = border_key[0], bin_keys = border_key[1] - border_key[0];
        border[0] = order_value(border_key[0]), border[1] = order_value(border_key[1]);
        // the next part's tokens are in flight while this part's are looked at
        constexpr int R = kPart / 64;
        auto needed = [&](int lo) {
          while (lo < V && !__builtin_amdgcn_readfirstlane(sh.some[lo / kStretch])) lo += kRowWaves * kPart;
          return lo;
        };
        float v[R], ahead[R];
        int lo = needed(wave * kPart);
        auto fetch = [&] {
          const float* p = z + lo;  // (the same in all lanes)
          if (lo + kPart <= V) {
#pragma unroll
            for (int r = 0; r < R; ++r) ahead[r] = p[r * 64 + (unsigned)lane];
          } else if (lo < V) {
#pragma unroll
            for (int r = 0; r < R; ++r) ahead[r] = r * 64 + lane < V - lo ? p[r * 64 + lane] : NAN;
          }
        };
        fetch();
#pragma unroll 1
        while (lo < V && listed <= kListed) {
          const int now = lo;
          lo = needed(now + kRowWaves * kPart);
#pragma unroll
          for (int r = 0; r < R; ++r) v[r] = ahead[r];
          fetch();
          // a bit per token of the lane; then every lane lists its own
          unsigned hits = 0;
#pragma unroll
          for (int r = R - 1; r >= 0; --r) hits = hits + hits + (v[r] >= border[0] && v[r] < border[1]);
          const int n = __popc(hits), upto = wave_scan(n), all = lane_value(upto, 63);
          int at = wave * kListed + listed + upto - n;
          listed += all;
          if (listed <= kListed) {
#pragma unroll 1
            for (; hits; hits &= hits - 1, ++at) sh.listed[at].y = (unsigned)(now + lane + 64 * (__ffs((int)hits) - 1));
          }
        }
        if (listed > kListed && lane == 0) sh.overflow = 1;
        if (listed <= kListed) {  // their keys
          constexpr int U = 4;
#pragma unroll 1
          for (int i = lane; i < listed; i += U * 64) {
            float x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = z[sh.listed[wave * kListed + min(i + u * 64, listed - 1)].y];
#pragma unroll
            for (int u = 0; u < U; ++u)
              if (i + u * 64 < listed) sh.listed[wave * kListed + i + u * 64].x = order_key(x[u]);
          }
        }
        __syncthreads();
      }
      in_lds = bin < kLogitBins && sh.overflow == 0;
      // what the search looks at: the listed tokens, every wave its own, or all of the row
      const int from = in_lds ? wave * kListed + lane : tid, end = in_lds ? wave * kListed + listed : V, step = in_lds ? 64 : kRowThreads;
      auto key_at = [&](int i) {
        if (in_lds) return sh.listed[i].x;
        const float v = logit(i);
        return usable(v) ? order_key(v) : 0u;
      };
      const int wide_sum = in_lds ? 0 : wide;
      unsigned common = 0;
      int bits = 32;
      if (phase == 2) {
        u64 equal = 0;
        for (int i = from; i < end; i += step) equal += key_at(i) == t_key;
        if (ties >= all_sum(equal, sh, lane, wave)) break;  // all of them
        want = ties;
        bits = 20;
      } else if (in_lds) {  // keys of the bin count from its smallest
        common = bin_first;
        bits = bin_keys > 1 ? 32 - __clz((int)(bin_keys - 1)) : 0;
      }
      if (phase == 0 && in_lds) want -= sh.found_above;
      if (phase == 1) {
        const double x = in_lds ? ceil(want_d - (bin ? sh.upto_weight[bin - 1] : 0.0)) : ceil(__builtin_amdgcn_ldexp(want_d, -wide));
        want = x < 1.0 ? 1 : (u64)x;
      }
      const unsigned key = common + find_key(
          from, end, step, bits,
          [&](int i) { return phase == 2 ? (unsigned)(kMostVocab - 1) - (in_lds ? sh.listed[i].y : (unsigned)i) : key_at(i) - common; },
          [&](int i) -> u64 {
            const unsigned k = key_at(i);
            return phase == 2 ? k == t_key : k == 0 ? 0 : phase == 0 ? 1 : row_weight(k) >> wide_sum;
          },
          want, sh, tid, lane, wave);
      if (phase == 0) {
        t_key = key, ties = want;
        if (!(s.p < 1.f)) continue;
        // what the first k weigh: above the bin, and the listed tokens above the cut (or the row's tokens above it)
        double w = in_lds && tid == 0 && bin ? sh.upto_weight[bin - 1] : 0.0;
        for (int i = from; i < end; i += step) {
          const unsigned k = key_at(i);
          if (k > key) w += (double)row_weight(k);
        }
        among = all_sum(w, sh, lane, wave) + (double)ties * (double)row_weight(key);
      } else if (phase == 1) {
        const u64 w = row_weight(key) >> wide_sum, of_key = w ? (want + w - 1) / w : ~0ull;
        if (key > t_key) t_key = key, ties = of_key;
        else if (key == t_key && of_key < ties) ties = of_key;
      } else {
        last = (unsigned)(kMostVocab - 1) - key;
      }
    }
  }
  if (far && !t_key) t_key = 1;  // (below every key: nothing is cut off)
  // kept weight of every stretch
  {
    if (t_key) {
      __syncthreads();
      if (in_lds) {
        const int bin = held;
        for (int i = tid; i < NS; i += kRowThreads) sh.inside[i] = 0;
        __syncthreads();
        for (int i = wave * kListed + lane; i < wave * kListed + listed; i += 64) {
          const unsigned k = sh.listed[i].x, x = sh.listed[i].y;
          if (k > t_key || (k == t_key && x <= last)) atomicAdd(&sh.inside[x / kStretch], row_weight(k));
        }
        __syncthreads();
        if (tid < NS) {
          const int j = min(bin - sh.below[tid], kLogitBins) - 1;  // the last bin before it
          sh.kept[tid] = (j >= 0 ? ws.upto_weight[(at0 + tid) * kLogitBins + j] * sh.scale[tid] : 0.0) + (double)sh.inside[tid];
        }
      } else {
#pragma unroll 1
        for (int i = wave; i < NS; i += kRowWaves) {
          double m = 0;
          for (int x = i * kStretch + lane; x < min(V, (i + 1) * kStretch); x += 64) {
            const float v = logit(x);
            const unsigned k = usable(v) ? order_key(v) : 0;
            if (k > t_key || (k == t_key && (unsigned)x <= last)) m += (double)row_weight(k);
          }
          m = wave_scan(m);
          if (lane == 63) sh.kept[i] = m;
        }
      }
    }
  }
  __syncthreads();

  // ---- the draw ------------------------------------------------------------------------------------------------------------------
  // the stretch: four per lane, the same sums in every wave
  constexpr int SPL = kMostStretches / 64;
  double part[SPL], lane_sum = 0;
#pragma unroll
  for (int i = 0; i < SPL; ++i) part[i] = lane * SPL + i < NS ? sh.kept[lane * SPL + i] : 0.0, lane_sum += part[i];
  const double upto = wave_scan(lane_sum), all = lane_value(upto, 63);
  const float u = a.uniform[b];
  const double wanted = u > 0.f ? (double)fminf(u, 1.f) * all : 0.0;
  int pick = -1;       // of this lane: its first stretch that reaches past the number, else its last with any weight
  double start = 0, run = upto - lane_sum;
  bool reached = false;
#pragma unroll
  for (int i = 0; i < SPL; ++i) {
    if (part[i] > 0 && !reached) pick = lane * SPL + i, start = run, reached = run + part[i] > wanted;
    run += part[i];
  }
  const u64 past = __ballot(reached), some = __ballot(pick >= 0);
  const int from = past ? __ffsll(past) - 1 : 63 - __clzll((long long)some);
  pick = lane_value(pick, from);
  const double offset = wanted - lane_value(start, from);
  const int first = pick * kStretch;
  // the token: some in a row per thread
  constexpr int TPT = kStretch / kRowThreads;
  const float local = sh.top[pick];
  u64 w[TPT], sum = 0;
  float v[TPT];
#pragma unroll
  for (int i = 0; i < TPT; ++i) v[i] = first + tid * TPT + i < V ? logit(first + tid * TPT + i) : -INFINITY;
#pragma unroll
  for (int i = 0; i < TPT; ++i) {
    const unsigned k = usable(v[i]) ? order_key(v[i]) : 0;
    w[i] = k && (k > t_key || (k == t_key && (unsigned)(first + tid * TPT + i) <= last)) ? ex.fixed(v[i], local, per_t) : 0;
    sum += w[i];
  }
  u64 whole_stretch, before = block_scan(sum, sh, lane, wave, whole_stretch) - sum;
  const double x = offset / ex.weight(local, top, per_t);
  u64 target = x >= (double)whole_stretch ? whole_stretch - 1 : x > 0 ? (u64)x : 0;
  if (target >= whole_stretch) target = whole_stretch - 1;
  if (target < before || target >= before + sum) return;
#pragma unroll
  for (int i = 0; i < TPT; ++i) {
    if (target >= before && target < before + w[i]) {
      a.token[b] = first + tid * TPT + i;
      if (a.logprob) {
        // log of the sum: a logarithm in 32 bits and what the exponential in 64 leaves of it
        const double sum1 = all / kOne, y = (double)logf((float)sum1), r = sum1 * ex.at(-y * kPerT) - 1.0;
        a.logprob[b] = (float)(((double)v[i] - (double)top) * per_t / kPerT - y - (r - 0.5 * r * r));
      }
    }
    before += w[i];
  }
}

struct SampleLayout {
  SampleWs ws;
  size_t bytes;
};
SampleLayout sample_layout(int batch, int vocab, void* base) {
  auto al = [](size_t n) { return (n + 255) & ~size_t(255); };
  SampleLayout l{};
  l.ws.n = (vocab + kStretch - 1) / kStretch;
  const size_t n = (size_t)batch * l.ws.n;
  char* p = static_cast<char*>(base);
  auto take = [&](size_t bytes) {
    char* q = p + l.bytes;
    l.bytes += al(bytes);
    return q;
  };
  l.ws.upto_weight = reinterpret_cast<double*>(take(n * kLogitBins * 8));
  l.ws.weight = reinterpret_cast<double*>(take(n * 8));
  l.ws.top = reinterpret_cast<float*>(take(n * 4));
  l.ws.usable = reinterpret_cast<unsigned*>(take(n * 4));
  l.ws.upto_count = reinterpret_cast<unsigned short*>(take(n * kLogitBins * 2));
  return l;
}

// k_sample_row needs more dynamic LDS than the default limit; asked for once per device.
constexpr int kMaxDevices = 64;
bool g_row_lds[kMaxDevices] = {};
std::mutex g_row_lds_mu;

harli_status allow_row_lds() {
  int dev = -1;
  HARLI_HIP(hipGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices) return fail(HARLI_ERR_INVALID, "sample: device ordinal %d outside 0..%d", dev, kMaxDevices - 1);
  std::lock_guard<std::mutex> lk(g_row_lds_mu);
  if (!g_row_lds[dev]) {
    HARLI_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(&k_sample_row), hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(RowShared)));
    g_row_lds[dev] = true;
  }
  return HARLI_OK;
}

}  // namespace
}  // namespace harli

using namespace harli;

extern "C" size_t harli_sample_workspace_bytes(int32_t batch, int32_t vocab) {
  if (batch < 1 || batch > 65535 || vocab < 1 || vocab > kMostVocab) return 0;
  return sample_layout(batch, vocab, nullptr).bytes;
}

extern "C" harli_status harli_sample(const harli_sample_batch* b, void* hip_stream) {
  if (!b) return fail(HARLI_ERR_INVALID, "sample: null argument");
  if (b->batch < 1 || b->batch > 65535) return fail(HARLI_ERR_INVALID, "sample: batch %d outside 1..65535", b->batch);
  if (b->vocab < 1 || b->vocab > kMostVocab) return fail(HARLI_ERR_INVALID, "sample: vocabulary of %d outside 1..%d", b->vocab, kMostVocab);
  if (!b->logits || !b->uniform || !b->token) return fail(HARLI_ERR_INVALID, "sample: logits, uniform and token are required");
  if (b->ld < b->vocab) return fail(HARLI_ERR_INVALID, "sample: rows %lld apart hold %d logits", (long long)b->ld, b->vocab);
  const size_t need = harli_sample_workspace_bytes(b->batch, b->vocab);
  if (!b->workspace || (uintptr_t)b->workspace % 256 || b->workspace_bytes < need)
    return fail(HARLI_ERR_INVALID, "sample: a 256-byte aligned workspace of %zu bytes is needed, got %zu", need, b->workspace ? b->workspace_bytes : 0);
  harli_status rc = allow_row_lds();
  if (rc != HARLI_OK) return rc;
  const SampleWs ws = sample_layout(b->batch, b->vocab, b->workspace).ws;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  hipLaunchKernelGGL(k_sample_stretch, dim3(ws.n, b->batch), dim3(kStretchThreads), 0, st, *b, ws, kSeries);
  hipLaunchKernelGGL(k_sample_row, dim3(b->batch), dim3(kRowThreads), sizeof(RowShared), st, *b, ws, kSeries);
  HARLI_HIP(hipGetLastError());
  return HARLI_OK;
}
