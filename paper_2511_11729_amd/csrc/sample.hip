// A token per row of logits by temperature, top-k, top-p and min-p (harli_sample).
// All three filters keep the first tokens in the order of (logit, then lower index), so what stays is a cut: a logit and how many of
// the tokens that have just this logit.  The cut is found digit by digit on the logits' order-preserving integers, counting tokens
// for top-k and adding weights for top-p.  Weights are exp in 64 bits, rounded to fixed point: their sums are the same in any order.
#include "ctx.h"
#include "device_utils.h"

namespace harli {
namespace {

constexpr int kSampleThreads = 1024;
typedef unsigned long long u64;

__device__ __forceinline__ unsigned order_key(float v) {  // of a logit that is not NaN; both zeros alike
  const unsigned u = __float_as_uint(v + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float order_value(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// exp((v - max) / t) in fixed point (`one` stands for 1)
__device__ __forceinline__ double weight_of(float v, float max, double inv_t) {
  return v == max ? 1.0 : v == -INFINITY || max == INFINITY ? 0.0 : exp(((double)v - (double)max) * inv_t);
}
__device__ __forceinline__ u64 fixed_of(double w, double one) { return (u64)(w * one + 0.5); }

__device__ __forceinline__ u64 wave_sum64(u64 v) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

__global__ void __launch_bounds__(kSampleThreads) k_sample(harli_sample_batch a, double one) {
  constexpr int NW = kSampleThreads / 64;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.vocab;
  const float* z = a.logits + (size_t)b * a.ld;
  __shared__ float s_max[NW];
  __shared__ int s_bin, s_first;
  __shared__ u64 mass[256], s_part[NW], s_above;
  __shared__ u64 s_ties[NW];

  float mx = -INFINITY;
  for (int i = tid; i < V; i += kSampleThreads) {
    const float v = z[i];
    if (v > mx) mx = v;
  }
  for (int o = 1; o < 64; o <<= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
  if (lane == 0) s_max[wave] = mx;
  if (tid == 0) s_first = 0x7fffffff;
  __syncthreads();
  for (int w = 0; w < NW; ++w) mx = fmaxf(mx, s_max[w]);
  if (mx == -INFINITY) {
    if (tid == 0) {
      a.token[b] = -1;
      if (a.logprob) a.logprob[b] = -INFINITY;
    }
    return;
  }
  const float T = a.temperature ? a.temperature[b] : 1.f;
  if (!(T > 0.f)) {
    for (int i = tid; i < V; i += kSampleThreads)
      if (z[i] == mx) {
        atomicMin(&s_first, i);
        break;
      }
    __syncthreads();
    if (tid == 0) {
      a.token[b] = s_first;
      if (a.logprob) a.logprob[b] = 0.f;
    }
    return;
  }
  const double inv_t = 1.0 / (double)T;
  auto usable = [&](float v) { return v > -INFINITY; };  // (false for NaN)

  // the cut: keys above t_key stay, and the first `ties` of those equal to it
  unsigned t_key = 0;
  u64 ties = ~0ull, total = 0;
  // digit by digit: the key at which what lies above it is less than `want` and with it not; BY_MASS: weights, else tokens
  auto select = [&](bool by_mass, u64 want, unsigned& key, u64& rest) {
    unsigned prefix = 0, mask = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) mass[tid] = 0;
      __syncthreads();
      for (int i = tid; i < V; i += kSampleThreads) {
        const float v = z[i];
        if (!usable(v)) continue;
        const unsigned k = order_key(v);
        if ((k & mask) == prefix) atomicAdd(&mass[(k >> shift) & 255], by_mass ? fixed_of(weight_of(v, mx, inv_t), one) : 1ull);
      }
      __syncthreads();
      if (tid == 0) {
        u64 above = 0;
        int bin = 255;
        for (; bin > 0 && above + mass[bin] < want; --bin) above += mass[bin];
        s_bin = bin, s_above = above;
      }
      __syncthreads();
      want -= s_above;
      prefix |= (unsigned)s_bin << shift;
      mask |= 255u << shift;
      __syncthreads();
    }
    key = prefix, rest = want;
  };
  // weights above the key, and the number of tokens at it
  auto sums = [&](unsigned key, u64& above, u64& at) {
    u64 s = 0, n = 0;
    for (int i = tid; i < V; i += kSampleThreads) {
      const float v = z[i];
      if (!usable(v)) continue;
      const unsigned k = order_key(v);
      if (k > key) s += fixed_of(weight_of(v, mx, inv_t), one);
      else if (k == key) ++n;
    }
    s = wave_sum64(s), n = wave_sum64(n);
    if (lane == 0) s_part[wave] = s, s_ties[wave] = n;
    __syncthreads();
    above = at = 0;
    for (int w = 0; w < NW; ++w) above += s_part[w], at += s_ties[w];
    __syncthreads();
  };
  const int k_row = a.top_k ? a.top_k[b] : 0;
  const float p_row = a.top_p ? a.top_p[b] : 1.f;
  double floor_p = a.min_p ? (double)a.min_p[b] : 0.0;
  floor_p = floor_p > 1.0 ? 1.0 : floor_p > 0.0 ? floor_p : 0.0;
  u64 above, at;
  sums(0, above, at);  // (no finite logit and no infinity has key 0)
  u64 usable_n = 0;
  if (k_row > 0 && k_row < V) {
    // fewer usable tokens than k: all of them
    u64 n = 0;
    for (int i = tid; i < V; i += kSampleThreads) n += usable(z[i]);
    n = wave_sum64(n);
    if (lane == 0) s_part[wave] = n;
    __syncthreads();
    for (int w = 0; w < NW; ++w) usable_n += s_part[w];
    __syncthreads();
    if ((u64)k_row < usable_n) {
      select(false, k_row, t_key, ties);
      sums(t_key, above, at);
      above += ties * fixed_of(weight_of(order_value(t_key), mx, inv_t), one);
    }
  }
  total = above;
  if (p_row < 1.f) {
    const double x = (double)p_row * (double)total;
    u64 want = x < 1.0 ? 1 : (u64)ceil(x);
    if (want > total) want = total;
    unsigned key;
    u64 rest;
    select(true, want, key, rest);
    const u64 w = fixed_of(weight_of(order_value(key), mx, inv_t), one);
    const u64 n = w ? (rest + w - 1) / w : 1;
    if (key > t_key || n < ties) t_key = key, ties = n;
  }

  // ---- the draw: waves take stretches of the row, by index ---------------------------------------------------------------
  const int per = ((V + NW - 1) / NW + 63) / 64 * 64, lo = min(V, wave * per), hi = min(V, lo + per);
  u64 n_at = 0;
  for (int i = lo + lane; i < hi; i += 64) n_at += usable(z[i]) && order_key(z[i]) == t_key;
  n_at = wave_sum64(n_at);
  if (lane == 0) s_ties[wave] = n_at;
  __syncthreads();
  u64 before = 0;
  for (int w = 0; w < wave; ++w) before += s_ties[w];
  auto kept = [&](int i, u64& seen) -> u64 {  // weight of token i (0: not kept); wave collective
    const float v = i < hi ? z[i] : -INFINITY;
    const unsigned k = usable(v) ? order_key(v) : 0;
    const bool tie = usable(v) && k == t_key;
    const u64 m = __ballot(tie);
    const u64 r = seen + __popcll(m & ((1ull << lane) - 1));
    seen += __popcll(m);
    if (!usable(v) || k < t_key || (tie && r >= ties)) return 0;
    const double w = weight_of(v, mx, inv_t);
    return w >= floor_p ? fixed_of(w, one) : 0;
  };
  u64 mine = 0, seen = before;
  for (int i0 = lo; i0 < hi; i0 += 64) mine += kept(i0 + lane, seen);
  mine = wave_sum64(mine);
  if (lane == 0) s_part[wave] = mine;
  __syncthreads();
  u64 start = 0, all = 0;
  for (int w = 0; w < NW; ++w) {
    if (w < wave) start += s_part[w];
    all += s_part[w];
  }
  const float u = a.uniform[b];
  const double x = u > 0.f ? (double)u * (double)all : 0.0;
  u64 target = x >= (double)all ? all - 1 : (u64)x;
  if (target >= all) target = all - 1;
  if (target < start || target >= start + mine) return;
  seen = before;
  for (int i0 = lo; i0 < hi; i0 += 64) {
    const u64 w = kept(i0 + lane, seen);
    u64 c = w;
    for (int o = 1; o < 64; o <<= 1) {
      const u64 v = __shfl_up(c, o, 64);
      if (lane >= o) c += v;
    }
    const u64 hit = __ballot(start + c > target);
    if (hit) {
      if (lane == __ffsll(hit) - 1) {
        a.token[b] = i0 + lane;
        if (a.logprob) a.logprob[b] = (float)log((double)w / (double)all);
      }
      return;
    }
    start += __shfl(c, 63, 64);
  }
}

}  // namespace
}  // namespace harli

using namespace harli;

extern "C" size_t harli_sample_workspace_bytes(int32_t batch, int32_t vocab) {
  if (batch < 1 || vocab < 1 || vocab > (1 << 24)) return 0;
  return 256;
}

extern "C" harli_status harli_sample(const harli_sample_batch* b, void* hip_stream) {
  if (!b) return fail(HARLI_ERR_INVALID, "sample: null argument");
  if (b->batch < 1) return fail(HARLI_ERR_INVALID, "sample: batch %d", b->batch);
  if (b->vocab < 1 || b->vocab > (1 << 24)) return fail(HARLI_ERR_INVALID, "sample: vocabulary of %d outside 1..2^24", b->vocab);
  if (!b->logits || !b->uniform || !b->token) return fail(HARLI_ERR_INVALID, "sample: logits, uniform and token are required");
  if (b->ld < b->vocab) return fail(HARLI_ERR_INVALID, "sample: rows %lld apart hold %d logits", (long long)b->ld, b->vocab);
  const size_t need = harli_sample_workspace_bytes(b->batch, b->vocab);
  if (!b->workspace || (uintptr_t)b->workspace % 256 || b->workspace_bytes < need)
    return fail(HARLI_ERR_INVALID, "sample: a 256-byte aligned workspace of %zu bytes is needed, got %zu", need, b->workspace ? b->workspace_bytes : 0);
  int bits = 0;
  while ((1ll << bits) < b->vocab) ++bits;
  const double one = (double)(1ull << (62 - bits));
  hipLaunchKernelGGL(k_sample, dim3(b->batch), dim3(kSampleThreads), 0, static_cast<hipStream_t>(hip_stream), *b, one);
  HARLI_HIP(hipGetLastError());
  return HARLI_OK;
}
