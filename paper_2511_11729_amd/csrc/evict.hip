// Eviction from the paged KV cache by accumulated attention weight (harli_kv_evict).  Every (layer, sequence, KV head) ranks its
// own tokens, keeps the best and moves those of them that lie behind the kept length into the slots that fell free.
// Reads 8 bytes per token and moves whole rows of keys and values: bound by HBM.  Only rows behind the kept length move (not
// everything behind the first gap, as keeping the order would): a service that gives up one page of 16 tokens at a time moves at
// most 16 rows per head, and sources (slots >= keep) and targets (slots < keep) never meet, so rows move in any order.
#include "ctx.h"
#include "device_utils.h"

namespace harli {
namespace {

constexpr int kPageTokens = 16;
constexpr int kMostPages = 1 << 26;  // of a table row: token indexes stay in 32 bits
constexpr int kMoves = 1024;          // moves listed in LDS at a time
constexpr int kMostTokens = 1 << 18;  // of a sequence: a bit each in LDS
constexpr int kBins = 2048;           // of the search for the last weight that stays: 11, 11 and 10 bits

// Order of the weights as unsigned integers: NaN below every other, both zeros alike, protected tokens above.
__device__ __forceinline__ unsigned rank_key(uint2 rec, int sink, long long recent_from) {
  const int pos = (int)rec.y;
  if (pos < sink || (long long)pos >= recent_from) return 0xffffffffu;
  const unsigned u = __float_as_uint(__uint_as_float(rec.x) + 0.f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sum of v over the threads before this one, and of all of them in `all` (the whole workgroup calls it; `tmp`: one entry per wave).
template <int NW>
__device__ __forceinline__ int scan_before(int v, int* tmp, int lane, int wave, int& all) {
  int s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(s, o, 64);
    if (lane >= o) s += x;
  }
  __syncthreads();  // tmp is free
  if (lane == 63) tmp[wave] = s;
  __syncthreads();
  int before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    if (w < wave) before += tmp[w];
    all += tmp[w];
  }
  return before + s - v;
}

struct EvictArgs {
  harli_evict_batch b;
  int n_kv, row_bytes;
  char* slab;
  KvGeom geom;
  int* err_flag;
};

// NT threads with KR keys each in registers (KR = 0: keys are read again for every pass); rows move in words of VEC bytes.
// A wave's 64 keys of one round are 64 tokens in a row: their ballot is a word of the bitmap of those that stay.
template <int NT, int KR, int VEC>
__global__ void __launch_bounds__(NT) k_evict(EvictArgs args) {
  constexpr int NW = NT / 64, BPT = kBins / NT;
  static_assert(kBins % NT == 0, "whole bins per thread");
  const harli_evict_batch& a = args.b;
  const KvGeom& geom = args.geom;
  const int n_kv = args.n_kv;
  const int c = blockIdx.x, b = blockIdx.y, layer = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = a.n_tokens[b], keep = max(a.keep[b], 0);
  const bool first = c == 0 && layer == 0;
  if (n > a.max_kv_len || n > a.max_pages * kPageTokens) {
    if (first && tid == 0) {
      atomicOr(args.err_flag, 4);
      if (a.n_left) a.n_left[b] = n;
    }
    return;
  }
  if (first && tid == 0 && a.n_left) a.n_left[b] = min(n, keep);
  if (n <= keep) return;
  const long long recent_from = (long long)(a.position ? a.position[b] : n) - a.recent;
  const int* table = a.page_table + (size_t)b * a.max_pages;
  harli_kv_record* rec = a.records + ((size_t)layer * geom.n_pages_total * n_kv + c) * kPageTokens;
  const size_t page_recs = (size_t)n_kv * kPageTokens;
  auto good = [&](int page) { return page >= 0 && page < geom.n_pages_total; };
  auto load_key = [&](int t) -> unsigned {  // of a token of the sequence
    const int page = table[t / kPageTokens];
    if (!good(page)) {
      if (first) atomicOr(args.err_flag, 1);
      return 0;
    }
    return rank_key(*reinterpret_cast<const uint2*>(rec + page * page_recs + t % kPageTokens), a.sink, recent_from);
  };

  extern __shared__ unsigned long long stays[];  // a bit per token
  __shared__ int hist[kBins], tmp[NW], s_bin, s_above, s_count;
  __shared__ int from[kMoves], to[kMoves];

  unsigned key[KR ? KR : 1];
  const int rounds = (n + NT - 1) / NT;
  if constexpr (KR > 0) {
#pragma unroll
    for (int i = 0; i < KR; ++i) {
      const int t = i * NT + tid;
      key[i] = 0;
      if (i < rounds && t < n) key[i] = load_key(t);
    }
  }
  // f(round, token, key) for the rounds of this thread; token >= n: none (key 0)
  auto each = [&](auto&& f) {
    if constexpr (KR > 0) {
#pragma unroll
      for (int i = 0; i < KR; ++i)
        if (i < rounds) f(i * NT + tid, key[i]);
    } else {
#pragma unroll 4
      for (int i = 0; i < rounds; ++i) {
        const int t = i * NT + tid;
        f(t, t < n ? load_key(t) : 0u);
      }
    }
  };

  // ---- the keep-th largest key, digit by digit: a token stays if its key is above `prefix`, or equal to it (in the digits seen)
  // and among the first `want` of those ------------------------------------------------------------------------------------
  unsigned prefix = 0, mask = 0;
  int want = keep, count = n;
  for (int shift = 21; keep > 0 && want < count && shift >= 0; shift = shift == 21 ? 10 : shift == 10 ? 0 : -1) {
    const unsigned digits = shift ? 2047u : 1023u;
    for (int i = tid; i < kBins; i += NT) hist[i] = 0;
    __syncthreads();
    each([&](int t, unsigned k) {
      if (t < n && (k & mask) == prefix) atomicAdd(&hist[(k >> shift) & digits], 1);
    });
    __syncthreads();
    int h[BPT], sum = 0, all;  // thread 0 has the highest bins
#pragma unroll
    for (int i = 0; i < BPT; ++i) h[i] = hist[kBins - 1 - (tid * BPT + i)], sum += h[i];
    int above = scan_before<NW>(sum, tmp, lane, wave, all);
    if (above < want && above + sum >= want) {
#pragma unroll
      for (int i = 0; i < BPT; ++i) {
        if (above < want && above + h[i] >= want) s_bin = kBins - 1 - (tid * BPT + i), s_above = above, s_count = h[i];
        above += h[i];
      }
    }
    __syncthreads();
    want -= s_above;
    count = s_count;
    prefix |= (unsigned)s_bin << shift;
    mask |= digits << shift;
    __syncthreads();
  }

  // ---- who stays ---------------------------------------------------------------------------------------------------------
  if (keep == 0) {
    for (int i = tid; i < (n + 63) / 64; i += NT) stays[i] = 0;
  } else if (want == count) {  // all of the last ones
    each([&](int t, unsigned k) {
      const unsigned long long m = __ballot(t < n && (k & mask) >= prefix);
      if (lane == 0 && t < n) stays[t / 64] = m;
    });
  } else {  // equal keys: the first `want` of them, in order of the slots
    int seen = 0;
    each([&](int t, unsigned k) {
      const bool eq = t < n && k == prefix;
      const unsigned long long me = __ballot(eq);
      int all;
      __syncthreads();
      if (lane == 0) tmp[wave] = __popcll(me);
      __syncthreads();
      int r = seen + __popcll(me & ((1ull << lane) - 1));
      all = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        if (w < wave) r += tmp[w];
        all += tmp[w];
      }
      seen += all;
      const unsigned long long m = __ballot(t < n && (k > prefix || (eq && r < want)));
      if (lane == 0 && t < n) stays[t / 64] = m;
    });
  }
  __syncthreads();

  // ---- the moves: the i-th of those that stay behind the kept length goes to the i-th slot that fell free --------------------
  const int words = (n + 63) / 64, per = (words + NT - 1) / NT, w_lo = min(words, tid * per), w_hi = min(words, w_lo + per);
  auto below = [](int bits) { return bits >= 64 ? ~0ull : bits <= 0 ? 0ull : (1ull << bits) - 1; };
  auto holes_of = [&](int w) { return ~stays[w] & below(keep - 64 * w); };
  auto movers_of = [&](int w) { return stays[w] & ~below(keep - 64 * w); };
  int holes = 0, movers = 0, total, total_movers;
  for (int w = w_lo; w < w_hi; ++w) holes += __popcll(holes_of(w)), movers += __popcll(movers_of(w));
  const int h0 = scan_before<NW>(holes, tmp, lane, wave, total), m0 = scan_before<NW>(movers, tmp, lane, wave, total_movers);
  const int row_words = args.row_bytes / VEC;
  typedef unsigned int __attribute__((ext_vector_type(VEC / 4))) word;
  for (int first_move = 0; first_move < total; first_move += kMoves) {
    int h = h0 - first_move, m = m0 - first_move;
    for (int w = w_lo; w < w_hi; ++w) {
      for (unsigned long long x = holes_of(w); x; x &= x - 1, ++h)
        if (h >= 0 && h < kMoves) to[h] = 64 * w + __ffsll(x) - 1;
      for (unsigned long long x = movers_of(w); x; x &= x - 1, ++m)
        if (m >= 0 && m < kMoves) from[m] = 64 * w + __ffsll(x) - 1;
    }
    __syncthreads();
    const int moves = min(kMoves, total - first_move);
#pragma unroll 4
    for (int i = tid; i < moves * 2 * row_words; i += NT) {
      const int r = i / row_words, x = i - r * row_words, src = from[r >> 1], dst = to[r >> 1], ps = table[src / kPageTokens], pd = table[dst / kPageTokens];
      if (!good(ps) || !good(pd)) continue;
      const size_t head = (size_t)c * kPageTokens;
      const word v = *reinterpret_cast<const word*>(args.slab + kv_page_off(geom, ps, layer, r & 1) + (head + src % kPageTokens) * args.row_bytes + x * VEC);
      *reinterpret_cast<word*>(args.slab + kv_page_off(geom, pd, layer, r & 1) + (head + dst % kPageTokens) * args.row_bytes + x * VEC) = v;
    }
    for (int i = tid; i < moves; i += NT) {
      const int src = from[i], dst = to[i], ps = table[src / kPageTokens], pd = table[dst / kPageTokens];
      if (good(ps) && good(pd)) rec[pd * page_recs + dst % kPageTokens] = rec[ps * page_recs + src % kPageTokens];
    }
    __syncthreads();
  }
}

template <int VEC>
void launch_evict(const EvictArgs& a, int heads, int layers, hipStream_t st) {
  const dim3 grid(heads, a.b.batch, layers);
  const size_t bits = (size_t)(a.b.max_kv_len + 63) / 64 * 8;
  if (a.b.max_kv_len <= 256 * 32) hipLaunchKernelGGL((k_evict<256, 32, VEC>), grid, dim3(256), bits, st, a);
  else if (a.b.max_kv_len <= 1024 * 32) hipLaunchKernelGGL((k_evict<1024, 32, VEC>), grid, dim3(1024), bits, st, a);
  else hipLaunchKernelGGL((k_evict<1024, 0, VEC>), grid, dim3(1024), bits, st, a);
}

}  // namespace
}  // namespace harli

using namespace harli;

extern "C" harli_status harli_kv_evict(harli_ctx* c, const harli_evict_batch* b, void* hip_stream) {
  if (!c || !b) return fail(HARLI_ERR_INVALID, "kv_evict: null argument");
  const harli_model_cfg& m = c->cfg;
  if (b->batch < 1 || b->batch > m.max_batch) return fail(HARLI_ERR_INVALID, "kv_evict: batch %d outside 1..%d", b->batch, m.max_batch);
  if (!b->n_tokens || !b->keep || !b->page_table || !b->records)
    return fail(HARLI_ERR_INVALID, "kv_evict: n_tokens, keep, page_table and records are required");
  if ((uintptr_t)b->records % 16) return fail(HARLI_ERR_INVALID, "kv_evict: records are not 16-byte aligned");
  if (b->max_kv_len < 1 || b->max_kv_len > m.max_seq_len) return fail(HARLI_ERR_INVALID, "kv_evict: max_kv_len %d outside 1..%d", b->max_kv_len, m.max_seq_len);
  if (b->max_pages > kMostPages || b->max_pages * kPageTokens < b->max_kv_len)
    return fail(HARLI_ERR_INVALID, "kv_evict: page table rows of %d pages cannot hold %d tokens", b->max_pages, b->max_kv_len);
  if (b->sink < 0 || b->recent < 0) return fail(HARLI_ERR_INVALID, "kv_evict: sink %d, recent %d", b->sink, b->recent);
  if (b->n_left && (b->n_left == b->n_tokens || b->n_left == b->keep || b->n_left == b->position))
    return fail(HARLI_ERR_INVALID, "kv_evict: n_left is an input");
  if (b->max_kv_len > kMostTokens) return fail(HARLI_ERR_INVALID, "kv_evict: max_kv_len %d above %d", b->max_kv_len, kMostTokens);
  const int row_bytes = (int)(m.head_dim * esize(c));
  const EvictArgs a{*b, m.n_kv_heads, row_bytes, c->slab, c->geom, c->dw.err_flag};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  // pages start at multiples of 16 rows: rows of whole 16 bytes keep their words aligned, others (fp32, even head sizes) have 8
  if (row_bytes % 16 == 0) launch_evict<16>(a, m.n_kv_heads, m.n_layers, st);
  else launch_evict<8>(a, m.n_kv_heads, m.n_layers, st);
  HARLI_HIP(hipGetLastError());
  return HARLI_OK;
}
