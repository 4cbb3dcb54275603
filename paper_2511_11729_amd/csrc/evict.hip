// Eviction from the paged KV cache by accumulated attention weight (harli_kv_evict).  Every (layer, sequence, KV head) ranks its
// own tokens, keeps the best and moves those of them that lie behind the kept length into the slots that fell free.
// Reads 8 bytes per token and moves whole rows of keys and values: bound by HBM where many rows move (192 sequences of about 800 tokens
// cut to half, 736 MB in 168 us: 4.4 TB/s, a large copy reaches 4.7), by latency where few do (16 of 1040 tokens that give up a page,
// 64 heads each: 13.7 us for 26 MB).  Only rows behind the kept length move (not
// everything behind the first gap, as keeping the order would): a service that gives up one page of 16 tokens at a time moves at
// most 16 rows per head, and sources (slots >= keep) and targets (slots < keep) never meet, so rows move in any order.
#include <algorithm>
#include <mutex>

#include "ctx.h"
#include "device_utils.h"
#include "scan_utils.h"

namespace harli {
namespace {

constexpr int kPageTokens = 16;
constexpr int kMostPages = 1 << 26;  // of a table row: token indexes stay in 32 bits
constexpr int kMostTokens = 1 << 18;  // of a sequence: a bit each in LDS
constexpr int kBins = 2048;           // of the search for the last weight that stays: 11, 11 and 10 bits
// Tokens whose keys are read once and stay in LDS (128 KiB of a CU's 160); of longer sequences they are read again for every pass.  Two of
// 30003 in 128 heads, cut to an eighth / giving up 16 tokens: 143 / 34 us, read again 174 / 52.
constexpr int kKeysInLds = 32768;

// Order of the weights as unsigned integers: NaN below every other, both zeros alike, protected tokens above.
__device__ __forceinline__ unsigned rank_key(uint2 rec, int sink, long long recent_from) {
  const int pos = (int)rec.y;
  const unsigned u = __float_as_uint(__uint_as_float(rec.x) + 0.f);
  unsigned k = u & 0x80000000u ? ~u : u | 0x80000000u;
  k = (u & 0x7fffffffu) > 0x7f800000u ? 0 : k;
  const bool is_protected = (pos < sink) | ((long long)pos >= recent_from);
  return is_protected ? 0xffffffffu : k;
}

// Sum of v over the threads before this one, and of all of them in `all` (the whole workgroup calls it; `tmp`: one entry per wave).
template <int NW>
__device__ __forceinline__ int scan_before(int v, int* tmp, int lane, int wave, int& all) {
  const int s = wave_scan(v);
  __syncthreads();  // tmp is free
  if (lane == 63) tmp[wave] = s;
  __syncthreads();
  const int t = row_scan(lane < NW ? tmp[lane] : 0);
  all = lane_value(t, NW - 1);
  const int before = lane_value(t, wave ? wave - 1 : 0);
  return (wave ? before : 0) + s - v;
}

struct EvictArgs {
  harli_evict_batch b;
  int n_kv, row_bytes, row_lanes;  // row_lanes: the power of two of lanes that move a row, words of it each
  char* slab;
  KvGeom geom;
  int* err_flag;
};

// LDS: a bit per token that stays, then keys and bins of the search, whose place the moves' offsets take afterwards.
struct Move {
  u64 src, dst;  // of a key's row, from the slab's start
};
__host__ __device__ constexpr int moves_listed(int threads) { return 2 * threads; }  // at a time
__host__ __device__ inline size_t bitmap_bytes(int max_kv_len) { return ((size_t)max_kv_len + 127) / 128 * 2 * (8 + 8); }  // and two sums per word
size_t evict_lds(int max_kv_len, bool keys, int threads) {
  const size_t search = (keys ? ((size_t)max_kv_len + 3) / 4 * 16 : 0) + kBins * 4;
  return bitmap_bytes(max_kv_len) + std::max(search, (size_t)moves_listed(threads) * (sizeof(Move) + 8));
}

// NT threads; KEYS: the keys stay in LDS; rows move in words of VEC bytes.
// One workgroup per head, also for few long sequences: several of them that share a head's rows need a second launch for the records that
// all go by (two of 30003 cut to an eighth, 64 heads: 114 us instead of 127; but two of 12000 that give up 16 tokens 37 instead of 21).
// The time goes into the rows at large sizes, and into latencies and the kernel's own code at small ones, hence loops instead of unrolled
// rounds over keys in registers (39 KB of code: 21.6 us where the loops took 17.5, for 16 sequences of 1040 tokens that give up one page
// in eight layers).
template <int NT, bool KEYS, int VEC>
__global__ void __launch_bounds__(NT) k_evict(EvictArgs args) {
  constexpr int NW = NT / 64, BPT = kBins / NT, kMoves = moves_listed(NT);
  static_assert(kBins % NT == 0 && NW <= 16, "whole bins per thread; the waves' sums in a row of lanes");
  const harli_evict_batch& a = args.b;
  const KvGeom& geom = args.geom;
  const int n_kv = args.n_kv;
  const int c = blockIdx.x, b = blockIdx.y, layer = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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

  extern __shared__ __align__(16) char evict_lds_mem[];
  const int most_words = (a.max_kv_len + 127) / 128 * 2;
  u64* stays = reinterpret_cast<u64*>(evict_lds_mem);           // a bit per token
  int2* sums = reinterpret_cast<int2*>(stays + most_words);     // free slots and moving tokens before each word
  char* rest = evict_lds_mem + bitmap_bytes(a.max_kv_len);
  int* hist = reinterpret_cast<int*>(rest);
  unsigned* keys = reinterpret_cast<unsigned*>(rest + kBins * 4);
  Move* moves = reinterpret_cast<Move*>(rest);  // once the search is done
  int2* pairs = reinterpret_cast<int2*>(rest + kMoves * sizeof(Move));
  __shared__ int tmp[NW], s_bin, s_above, s_count;

  bool bad = false;
  // Keys of U tokens of the sequence, NT apart, from t on (the last one's for those behind it).  All page ids, then all records are in flight
  // together: the assembly has both come before anything that depends on one of them (left alone, the compiler branches around loads
  // and waits for each: 27 us instead of 10 for the keys of 30003 tokens).
  auto load_keys = [&](int t, auto& k) {
    constexpr int U = sizeof(k) / sizeof(k[0]);
    int pg[U];
    uint2 r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) pg[u] = table[min(t + u * NT, n - 1) / kPageTokens];
#pragma unroll
    for (int u = 0; u < U; ++u) asm volatile("" : "+v"(pg[u]));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool ok = good(pg[u]);
      bad |= !ok;
      r[u] = *reinterpret_cast<const uint2*>(rec + (ok ? pg[u] : 0) * page_recs + min(t + u * NT, n - 1) % kPageTokens);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) asm volatile("" : "+v"(r[u].x), "+v"(r[u].y));
#pragma unroll
    for (int u = 0; u < U; ++u) k[u] = good(pg[u]) ? rank_key(r[u], a.sink, recent_from) : 0;
  };
  // the first pass of the search counts while the keys come in
  constexpr int kTopDigit = 21;
  auto clear = [&] {
#pragma unroll
    for (int i = 0; i < BPT; ++i) hist[tid * BPT + i] = 0;
    __syncthreads();
  };
  clear();
  {
    constexpr int U = KEYS ? 8 : 4;
#pragma unroll 1
    for (int t0 = tid; t0 < n; t0 += U * NT) {
      unsigned k[U];
      load_keys(t0, k);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (t0 + u * NT < n) {
          if constexpr (KEYS) keys[t0 + u * NT] = k[u];
          atomicAdd(&hist[kBins - 1 - (k[u] >> kTopDigit)], 1);  // the highest first
        }
    }
  }
  // f(key) for the tokens of this thread
  auto each = [&](auto&& f) {
    if constexpr (KEYS) {
#pragma unroll 2
      for (int t = 4 * tid; t < n; t += 4 * NT) {
        const uint4 k = *reinterpret_cast<const uint4*>(keys + t);
        f(k.x);
        if (t + 1 < n) f(k.y);
        if (t + 2 < n) f(k.z);
        if (t + 3 < n) f(k.w);
      }
    } else {
      constexpr int U = 4;
#pragma unroll 1
      for (int t = tid; t < n; t += U * NT) {
        unsigned k[U];
        load_keys(t, k);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (t + u * NT < n) f(k[u]);
      }
    }
  };
  auto key_of = [&](int t) {
    if constexpr (KEYS) return keys[t];
    unsigned k[1];
    load_keys(t, k);
    return k[0];
  };

  // ---- the keep-th largest key, digit by digit: a token stays if its key is above `prefix`, or equal to it (in the digits seen)
  // and among the first `want` of those ------------------------------------------------------------------------------------
  unsigned prefix = 0, mask = 0;
  int want = keep, count = n;
#pragma unroll 1
  for (int shift = kTopDigit; keep > 0 && want < count && shift >= 0; shift = shift == kTopDigit ? 10 : shift == 10 ? 0 : -1) {
    const unsigned digits = shift ? 2047u : 1023u;
    if (shift < kTopDigit) {
      clear();
      each([&](unsigned k) {
        if ((k & mask) == prefix) atomicAdd(&hist[kBins - 1 - ((k >> shift) & digits)], 1);
      });
    }
    __syncthreads();
    int h[BPT], sum = 0, all;
#pragma unroll
    for (int i = 0; i < BPT; ++i) h[i] = hist[tid * BPT + i], sum += h[i];
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
  }
  if (bad && first) atomicOr(args.err_flag, 1);
  __syncthreads();

  // ---- who stays: 64 tokens in a row are a ballot ---------------------------------------------------------------------------
  const int n_up = (n + 63) / 64 * 64;
  if (keep == 0 || want == count) {  // nothing, or all of the last ones
    for (int t = tid; t < n_up; t += NT) {
      const u64 m = __ballot(t < n && keep > 0 && (key_of(min(t, n - 1)) & mask) >= prefix);
      if (lane == 0) stays[t / 64] = m;
    }
  } else {  // equal keys: the first `want` of them, in order of the slots
    int seen = 0;
#pragma unroll 1
    for (int t0 = 0; t0 < n; t0 += NT) {
      const int t = t0 + tid;
      const unsigned k = key_of(min(t, n - 1));
      const bool eq = t < n && k == prefix;
      const u64 me = __ballot(eq);
      __syncthreads();
      if (lane == 0) tmp[wave] = __popcll(me);
      __syncthreads();
      const int sums = row_scan(lane < NW ? tmp[lane] : 0), before = lane_value(sums, wave ? wave - 1 : 0);
      const int r = seen + (wave ? before : 0) + (int)__popcll(me & ((1ull << lane) - 1));
      const u64 m = __ballot(t < n && (k > prefix || (eq && r < want)));
      if (lane == 0 && t < n) stays[t / 64] = m;
      seen += lane_value(sums, NW - 1);
    }
  }
  __syncthreads();

  // ---- the moves: the i-th of those that stay behind the kept length goes to the i-th slot that fell free --------------------
  const int words = (n + 63) / 64, per = (words + NT - 1) / NT, w_lo = min(words, tid * per), w_hi = min(words, w_lo + per);
  auto below = [](int bits) { return bits >= 64 ? ~0ull : bits <= 0 ? 0ull : (1ull << bits) - 1; };
  auto holes_of = [&](int w) { return ~stays[w] & below(keep - 64 * w); };
  auto movers_of = [&](int w) { return stays[w] & ~below(keep - 64 * w); };
  int holes = 0, movers = 0, total, total_movers;
  for (int w = w_lo; w < w_hi; ++w) holes += __popcll(holes_of(w)), movers += __popcll(movers_of(w));
  holes = scan_before<NW>(holes, tmp, lane, wave, total), movers = scan_before<NW>(movers, tmp, lane, wave, total_movers);
  for (int w = w_lo; w < w_hi; ++w) {
    sums[w] = make_int2(holes, movers);
    holes += __popcll(holes_of(w)), movers += __popcll(movers_of(w));
  }
  typedef unsigned int __attribute__((ext_vector_type(VEC / 4))) word;
  const int row_words = args.row_bytes / VEC, row_lanes = args.row_lanes, per_pass = NT / row_lanes, x0 = tid & (row_lanes - 1), r0 = tid / row_lanes;
#pragma unroll 1
  for (int at = 0; at < total; at += kMoves) {
    __syncthreads();
    // an eighth of a word per thread
#pragma unroll 1
    for (int x = tid; x < 8 * words; x += NT) {
      const int w = x / 8, up = 8 * (x & 7);
      const u64 free = holes_of(w), moving = movers_of(w);
      const int2 before = sums[w];
      auto list = [&](u64 all, int i, auto&& put) {
        i += (int)__popcll(all & ((1ull << up) - 1)) - at;
        for (unsigned bits = (unsigned)(all >> up) & 255; bits; bits &= bits - 1, ++i)
          if (i >= 0 && i < kMoves) put(i, 64 * w + up + __ffs((int)bits) - 1);
      };
      list(free, before.x, [&](int i, int t) { pairs[i].y = t; });
      list(moving, before.y, [&](int i, int t) { pairs[i].x = t; });
    }
    __syncthreads();
    const int n_moves = min(kMoves, total - at);
#pragma unroll 1
    for (int i = tid; i < n_moves; i += NT) {
      const int src = pairs[i].x, dst = pairs[i].y;
      int ps = table[src / kPageTokens], pd = table[dst / kPageTokens];
      asm volatile("" : "+v"(ps), "+v"(pd));
      const bool ok = good(ps) && good(pd);
      auto row_off = [&](int page, int slot) {
        return kv_page_off(geom, page, layer, 0) + (size_t)(c * kPageTokens + slot % kPageTokens) * args.row_bytes;
      };
      moves[i] = ok ? Move{row_off(ps, src), row_off(pd, dst)} : Move{0, 0};  // (to itself)
      if (ok) rec[pd * page_recs + dst % kPageTokens] = rec[ps * page_recs + src % kPageTokens];
    }
    __syncthreads();
    // keys and values of several rows in flight: eight where a head has a CU to itself (two of 30003, 128 heads: 143.7 us, four 147.2)
    constexpr int U = NT == 1024 ? 8 : 4;
#pragma unroll 1
    for (int i = r0; i < n_moves; i += U * per_pass)
#pragma unroll 1
      for (int x = x0; x < row_words; x += row_lanes) {
        word k[U], v[U];
        Move mv[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          mv[u] = moves[min(i + u * per_pass, n_moves - 1)];
          const char* p = args.slab + mv[u].src + x * VEC;
          k[u] = *reinterpret_cast<const word*>(p), v[u] = *reinterpret_cast<const word*>(p + geom.block_bytes);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          char* p = args.slab + mv[u].dst + x * VEC;
          if (i + u * per_pass < n_moves && mv[u].src != mv[u].dst) *reinterpret_cast<word*>(p) = k[u], *reinterpret_cast<word*>(p + geom.block_bytes) = v[u];
        }
      }
  }
}

// Long sequences need more dynamic LDS than the default limit; asked for once per device.
constexpr int kMaxDevices = 64;
bool g_evict_lds[kMaxDevices] = {};
std::mutex g_evict_lds_mu;

harli_status allow_evict_lds() {
  int dev = -1;
  HARLI_HIP(hipGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices) return fail(HARLI_ERR_INVALID, "kv_evict: device ordinal %d outside 0..%d", dev, kMaxDevices - 1);
  std::lock_guard<std::mutex> lk(g_evict_lds_mu);
  if (!g_evict_lds[dev]) {
    const void* kernels[] = {reinterpret_cast<const void*>(&k_evict<512, true, 16>), reinterpret_cast<const void*>(&k_evict<512, true, 8>),
                             reinterpret_cast<const void*>(&k_evict<1024, true, 16>), reinterpret_cast<const void*>(&k_evict<1024, true, 8>),
                             reinterpret_cast<const void*>(&k_evict<1024, false, 16>), reinterpret_cast<const void*>(&k_evict<1024, false, 8>)};
    const size_t most = std::max(evict_lds(kKeysInLds, true, 1024), evict_lds(kMostTokens, false, 1024));
    for (const void* k : kernels) HARLI_HIP(hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)most));
    g_evict_lds[dev] = true;
  }
  return HARLI_OK;
}

template <int VEC>
harli_status launch_evict(EvictArgs a, int heads, int layers, int n_cu, hipStream_t st) {
  const int n = a.b.max_kv_len, words = a.row_bytes / VEC;
  for (a.row_lanes = 1; a.row_lanes < words && a.row_lanes < 64;) a.row_lanes *= 2;
  const bool keys = n <= kKeysInLds;
  // Threads of a workgroup: as many as let every head run at once (2048 threads per CU), not more than the length has work for, and
  // 1024 where the keys leave a CU's LDS to one workgroup.  256 / 512 / 1024 threads in us, 16 tokens leave: 1024 heads of 1000 tokens
  // 16.9 / 22.1 / 38.1, of 4000 35.3 / 38.4 / 53.9, of 8000 66.9 / 57.7 / 70.0 (16 each in 192 uneven sequences of about 800
  // tokens cut to half: 187 / 178 / -); 512 heads of 1000 13.6 / 14.1 / 21.4, of 16000
  // 62.2 / 53.1 / 58.8; 64 heads of 1000 10.3 / 10.3 / 11.5, of 4000 14.8 / 12.0 / 12.6, of 16000 35.9 / 23.7 / 19.6.
  const long long all = (long long)heads * layers * a.b.batch;
  const int threads = n > 16384 || (all <= n_cu && n > 4096) ? 1024 : all <= 2 * n_cu || n > 2048 ? 512 : 256;
  const size_t lds = evict_lds(n, keys, threads);
  if (lds > (48u << 10)) {  // (with the kernel's own)
    const harli_status rc = allow_evict_lds();
    if (rc != HARLI_OK) return rc;
  }
  const dim3 grid(heads, a.b.batch, layers);
  if (threads == 256) hipLaunchKernelGGL((k_evict<256, true, VEC>), grid, dim3(256), lds, st, a);
  else if (threads == 512) hipLaunchKernelGGL((k_evict<512, true, VEC>), grid, dim3(512), lds, st, a);
  else if (keys) hipLaunchKernelGGL((k_evict<1024, true, VEC>), grid, dim3(1024), lds, st, a);
  else hipLaunchKernelGGL((k_evict<1024, false, VEC>), grid, dim3(1024), lds, st, a);
  return HARLI_OK;
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
  if (b->max_pages > kMostPages || (long long)b->max_pages * kPageTokens < b->max_kv_len)
    return fail(HARLI_ERR_INVALID, "kv_evict: page table rows of %d pages cannot hold %d tokens", b->max_pages, b->max_kv_len);
  if (b->sink < 0 || b->recent < 0) return fail(HARLI_ERR_INVALID, "kv_evict: sink %d, recent %d", b->sink, b->recent);
  if (b->n_left && (b->n_left == b->n_tokens || b->n_left == b->keep || b->n_left == b->position))
    return fail(HARLI_ERR_INVALID, "kv_evict: n_left is an input");
  if (b->max_kv_len > kMostTokens) return fail(HARLI_ERR_INVALID, "kv_evict: max_kv_len %d above %d", b->max_kv_len, kMostTokens);
  const int row_bytes = (int)(m.head_dim * esize(c));
  EvictArgs a{};
  a.b = *b, a.n_kv = m.n_kv_heads, a.row_bytes = row_bytes, a.slab = c->slab, a.geom = c->geom, a.err_flag = c->dw.err_flag;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  // pages start at multiples of 16 rows: rows of whole 16 bytes keep their words aligned, others (fp32, even head sizes) have 8
  const harli_status rc = row_bytes % 16 == 0 ? launch_evict<16>(a, m.n_kv_heads, m.n_layers, c->n_cu, st) : launch_evict<8>(a, m.n_kv_heads, m.n_layers, c->n_cu, st);
  if (rc != HARLI_OK) return rc;
  HARLI_HIP(hipGetLastError());
  return HARLI_OK;
}
