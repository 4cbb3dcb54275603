// Attention of one new token per sequence that records the weight of every cached token (harli_kv_attend and tracked decode
// steps; Harli Sec. 2.1 decode, Sec. 4.1 index-based KV).  Two launches: the cache is read in chunks of tokens, each leaving
// (maximum, sum, output) and its scores; then k_attend_finish joins the chunks and turns the scores into weights, which it can
// only now that the maximum and the sum over all chunks are known:  P_j = exp2(s_j - M) / L.  On bf16 storage a workgroup has all query
// heads of its KV head and the cache is read once; on fp32 it has one query head, and a group's heads read the same keys and values.
// What bounds it: HBM, for keys and values (2 d e bytes per token and KV head).  The scores are 4 bytes per token and query head,
// written once and read back, and the records 8 + 8 bytes per token and KV head.  Of bf16 caches, first and second launch, and what the
// first reads and writes: 16 sequences of 1024 tokens, 32 KV heads 46.9 and 8.0 us (273 MB, 5.8 TB/s); one of 32001, 32 / 8 heads 31.2
// and 10.2 (140 MB, 4.5 TB/s: a launch that fills and drains the chip once); 192 uneven ones of about 800, 28 / 4 heads 90.1 and
// 26.5 (383 MB, 39 of them scores and outputs of chunks, 4.3 TB/s).
#include <algorithm>
#include <cmath>

#include "attend.h"
#include "decode_large.h"
#include "device_utils.h"
#include "scan_utils.h"

namespace harli {
namespace {

constexpr int kPageTokens = 16;
constexpr int kMostPages = 1 << 26;  // of a table row: token indexes stay in 32 bits
constexpr int kChunkF32 = 256;       // tokens per chunk on fp32 storage: one per thread
constexpr int kFinishTokens = 1024;  // tokens of a block of records: four per thread
constexpr int kPiece = 64;           // elements of an output row that are joined at a time
// up to here an output element is one thread's (64 sequences of 200 tokens, 28 / 4 heads: 19.8 us instead of 23.2; 16 of 4096, 32 chunks,
// 32 / 8 heads: 66 either way)
constexpr int kFewChunks = 16;

// fp32 storage: one chunk of one query head; a thread scores one token, then a wave adds up P.V of every fourth token with a lane
// per element.  EL: elements per lane; a head larger than 64 EL goes to several workgroups (blockIdx.z), which score it alike.
template <int EL>
__global__ void __launch_bounds__(256) k_attend_f32(const float* q, const int* kv_len, const int* page_table, int max_pages, int layer,
                                                    int n_q, int n_kv, int d, const char* slab, KvGeom geom, int* err_flag, AttendWs att) {
  __shared__ __align__(16) float qs[EL < 16 ? 64 * EL : 4];
  __shared__ float red[8], ps[kChunkF32], os[4][64 * EL];
  __shared__ long long at[kChunkF32];  // element offset of a token's value from the slab's start, -1: no such page
  const int ch = blockIdx.x / n_q, hq = blockIdx.x - ch * n_q, b = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int hk = hq / (n_q / n_kv);
  const int n_all = kv_len[b] + att.n_new, n = min(min(n_all, att.n_chunks * kChunkF32), max_pages * kPageTokens);
  if (n != n_all && blockIdx.x == 0 && blockIdx.z == 0 && tid == 0) atomicOr(err_flag, 4);
  if (ch * kChunkF32 >= n) return;
  const float* qv = q + ((size_t)b * n_q + hq) * d;
  const int e0 = blockIdx.z * (64 * EL);
  if (EL < 16 && tid < d) qs[tid] = qv[tid];
  const float* base = reinterpret_cast<const float*>(slab);
  __syncthreads();
  const int t = ch * kChunkF32 + tid, nt = min(kChunkF32, n - ch * kChunkF32);
  float s = -INFINITY;
  long long v_at = -1;
  if (t < n) {
    const int page = page_table[(size_t)b * max_pages + t / kPageTokens];
    if (page >= 0 && page < geom.n_pages_total) {
      const size_t in_page = ((size_t)hk * kPageTokens + t % kPageTokens) * d;
      const float* kp = base + kv_page_off(geom, page, layer, 0) / 4 + in_page;
      const float* qe = EL < 16 ? qs : qv;
      s = 0.f;
      int e = 0;
      for (; e + 64 <= d; e += 64) {  // a whole 256 bytes in flight
        float kv[64];
#pragma unroll
        for (int x = 0; x < 64; x += 4) __builtin_memcpy(kv + x, kp + e + x, 16);
#pragma unroll
        for (int x = 0; x < 64; x += 4) s += qe[e + x] * kv[x] + qe[e + x + 1] * kv[x + 1] + qe[e + x + 2] * kv[x + 2] + qe[e + x + 3] * kv[x + 3];
      }
#pragma unroll 4
      for (; e + 4 <= d; e += 4) {
        float kv[4];
        __builtin_memcpy(kv, kp + e, 16);
        s += qe[e] * kv[0] + qe[e + 1] * kv[1] + qe[e + 2] * kv[2] + qe[e + 3] * kv[3];
      }
      if (e < d) s += qe[e] * kp[e] + qe[e + 1] * kp[e + 1];  // (head sizes are even)
      s *= 1.4426950408889634f * rsqrtf((float)d);
      v_at = (long long)(kv_page_off(geom, page, layer, 1) / 4 + in_page);
    } else {
      atomicOr(err_flag, 1);
    }
  }
  if (att.scores && blockIdx.z == 0) att.scores[((size_t)b * n_q + hq) * att.score_ld + t] = s;
  float m = s;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  if (lane == 0) red[wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const float p = v_at < 0 ? 0.f : exp2f(s - (m == -INFINITY ? 0.f : m));
  ps[tid] = p;
  at[tid] = v_at;
  const float sum = wave_sum(p);
  if (lane == 0) red[4 + wave] = sum;
  __syncthreads();
  float acc[EL];
#pragma unroll
  for (int x = 0; x < EL; ++x) acc[x] = 0.f;
  constexpr int U = EL >= 16 ? 1 : 8;  // tokens of a wave in flight
  for (int u0 = wave; u0 < nt; u0 += 4 * U) {
    float v[U][EL];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int x = 0; x < EL; ++x) v[u][x] = base[max(at[min(u0 + 4 * u, nt - 1)], 0ll) + min(e0 + lane + 64 * x, d - 1)];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float pu = u0 + 4 * u < nt && at[min(u0 + 4 * u, nt - 1)] >= 0 ? ps[u0 + 4 * u] : 0.f;
#pragma unroll
      for (int x = 0; x < EL; ++x) acc[x] = pu != 0.f ? acc[x] + pu * v[u][x] : acc[x];
    }
  }
#pragma unroll
  for (int x = 0; x < EL; ++x) os[wave][lane + 64 * x] = acc[x];
  __syncthreads();
  const size_t out = ((size_t)b * n_q + hq) * att.n_chunks + ch;
  for (int e = tid; e < min(64 * EL, d - e0); e += 256) att.o[out * d + e0 + e] = (os[0][e] + os[1][e]) + (os[2][e] + os[3][e]);
  if (tid == 0 && blockIdx.z == 0) *reinterpret_cast<float2*>(att.ml + out * 2) = make_float2(m, (red[4] + red[5]) + (red[6] + red[7]));
}

struct FinishArgs {
  const int *kv_len, *page_table, *position;
  int max_pages, layer, n_q, n_kv, d, n_pages, parts;
  float* out;
  unsigned short* frag;
  harli_kv_record* records;
  float decay;
};

// A KV head of a sequence is `parts` workgroups.  Each finds the maximum and the sum of every query head over the chunks, and then takes its
// share of the blocks of records and of the pieces of output rows: VEC elements a lane, kPiece / VEC lanes a piece, chunks side by side.
// What it costs is the latency of its steps, so the first block's scores and records are on their way before the sums are needed.
template <int VEC>
__global__ void __launch_bounds__(256) k_attend_finish(FinishArgs a, AttendWs att) {
  extern __shared__ float s_ml[];  // [heads of the group][maximum, 1 / sum]
  __shared__ float red[256 * VEC];
  constexpr int HP = 8;  // query heads whose scores are fetched ahead
  const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // (turned from sequence to sequence: the first parts have the most to do, and every eighth workgroup goes to the same XCD)
  const int at_x = (blockIdx.x + b) % gridDim.x, part = at_x / a.n_kv, c = at_x - part * a.n_kv, G = a.n_q / a.n_kv;
  const int n = max(0, min(min(a.kv_len[b] + att.n_new, att.n_chunks * att.chunk), a.max_pages * kPageTokens));
  const int nch = (n + att.chunk - 1) / att.chunk;
  const size_t head0 = (size_t)b * a.n_q + c * G;
  const float* ml = att.ml + head0 * att.n_chunks * 2;
  int t = part * kFinishTokens + tid * 4;
  const bool record = att.scores != nullptr;

  float4 sc[HP];
  int page = -1;
  uint4 r[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
  auto fetch = [&](int tokens_at) {
    t = tokens_at;
    if (!record || t >= n) return;
    page = a.page_table[(size_t)b * a.max_pages + t / kPageTokens];
#pragma unroll
    for (int h = 0; h < HP; ++h)
      if (h < G) sc[h] = *reinterpret_cast<const float4*>(att.scores + (head0 + h) * att.score_ld + t);
  };
  auto record_at = [&] { return a.records + (((size_t)a.layer * a.n_pages + page) * a.n_kv + c) * kPageTokens + t % kPageTokens; };
  fetch(t);

  // ---- maximum and sum of every query head, a wave each
  for (int h = wave; h < G; h += 4) {
    const float2* p = reinterpret_cast<const float2*>(ml + (size_t)h * att.n_chunks * 2);
    const float2 mine = lane < nch ? p[lane] : make_float2(-INFINITY, 0.f);
    float m = mine.x;
    for (int i = lane + 64; i < nch; i += 64) m = fmaxf(m, p[i].x);
    m = wave_top(m);
    m = m == -INFINITY ? 0.f : m;
    float l = mine.y * exp2f(mine.x - m);
    for (int i = lane + 64; i < nch; i += 64) l += p[i].y * exp2f(p[i].x - m);
    l = lane_value(wave_scan(l), 63);
    if (lane == 0) s_ml[2 * h] = m, s_ml[2 * h + 1] = l == 0.f ? 0.f : 1.f / l;  // no token that counts: zeros
  }
  __syncthreads();

  // ---- records
#pragma unroll 1
  while (record && t - tid * 4 < n) {  // (fetch moves t)
    if (t < n && page >= 0 && page < a.n_pages) {  // (another page id is reported where its keys were asked for)
      harli_kv_record* rec = record_at();
      r[0] = reinterpret_cast<const uint4*>(rec)[0], r[1] = reinterpret_cast<const uint4*>(rec)[1];
      float got[4] = {0.f, 0.f, 0.f, 0.f};
      auto add = [&](int h, const float4& s) {
        const float M = s_ml[2 * h], inv = s_ml[2 * h + 1];
        got[0] += __builtin_amdgcn_exp2f(s.x - M) * inv;
        got[1] += __builtin_amdgcn_exp2f(s.y - M) * inv;
        got[2] += __builtin_amdgcn_exp2f(s.z - M) * inv;
        got[3] += __builtin_amdgcn_exp2f(s.w - M) * inv;
      };
#pragma unroll
      for (int h = 0; h < HP; ++h)
        if (h < G) add(h, sc[h]);
      for (int h = HP; h < G; ++h) add(h, *reinterpret_cast<const float4*>(att.scores + (head0 + h) * att.score_ld + t));
      unsigned* w[4] = {&r[0].x, &r[0].z, &r[1].x, &r[1].z};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool newest = t + i == n - 1;
        const float old = newest || a.decay == 0.f ? 0.f : a.decay * __uint_as_float(*w[i]);
        *w[i] = __float_as_uint(old + got[i]);
        if (newest) w[i][1] = (unsigned)(a.position ? a.position[b] : n - 1);
      }
      if (t + 4 <= n) {
        reinterpret_cast<uint4*>(rec)[0] = r[0], reinterpret_cast<uint4*>(rec)[1] = r[1];
      } else {
        for (int i = 0; i < n - t; ++i) reinterpret_cast<uint2*>(rec)[i] = make_uint2(w[i][0], w[i][1]);
      }
    }
    fetch(t + a.parts * kFinishTokens);
  }

  auto store = [&](int col, float v) {  // element col of the sequence's row
    if (a.frag) a.frag[xfrag_off(b, col, (a.n_q * a.d + 31) >> 5)] = f2bf(v);
    else a.out[(size_t)b * a.n_q * a.d + col] = v;
  };
  // ---- output rows of few chunks: an element per thread
  if (nch <= kFewChunks) {
#pragma unroll 1
    for (int i = part * 256 + tid; i < G * a.d; i += a.parts * 256) {
      const int h = i / a.d, e = i - h * a.d;
      const size_t at = (head0 + h) * att.n_chunks;
      const float M = s_ml[2 * h];
      float v = 0.f;
#pragma unroll 8
      for (int j = 0; j < nch; ++j) v += att.o[(at + j) * a.d + e] * exp2f(att.ml[(at + j) * 2] - M);
      store(c * G * a.d + i, v * s_ml[2 * h + 1]);
    }
    return;
  }
  // ---- of many
  constexpr int NL = kPiece / VEC, NG = 256 / NL;
  const int per_row = (a.d + kPiece - 1) / kPiece, gi = tid / NL;
#pragma unroll 1
  for (int piece = part; piece < G * per_row; piece += a.parts) {
    const int h = piece / per_row, e = (piece - h * per_row) * kPiece + (tid - gi * NL) * VEC;
    const size_t at = (head0 + h) * att.n_chunks;
    const float M = s_ml[2 * h];
    float acc[VEC];
#pragma unroll
    for (int x = 0; x < VEC; ++x) acc[x] = 0.f;
    if (e < a.d) {
#pragma unroll 8
      for (int i = gi; i < nch; i += NG) {
        const float f = exp2f(att.ml[(at + i) * 2] - M);
        float v[VEC];
        __builtin_memcpy(v, __builtin_assume_aligned(att.o + (at + i) * a.d + e, VEC * 4), VEC * 4);
#pragma unroll
        for (int x = 0; x < VEC; ++x) acc[x] += v[x] * f;
      }
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < VEC; ++x) red[(gi * NL + (tid - gi * NL)) * VEC + x] = acc[x];
    __syncthreads();
    for (int x = tid; x < kPiece; x += 256) {
      const int k = (piece - h * per_row) * kPiece + x;
      if (k >= a.d) continue;
      float v = 0.f;
#pragma unroll
      for (int g = 0; g < NG; ++g) v += red[g * kPiece + x];
      v *= s_ml[2 * h + 1];
      store((c * G + h) * a.d + k, v);
    }
  }
}

__global__ void __launch_bounds__(256) k_record_init(harli_record_batch r, int n_kv, int n_pages, int* err_flag) {
  const int b = blockIdx.y, layer = blockIdx.z;
  const int n = r.n_tokens[b], seen = min(n, r.max_pages * kPageTokens);
  if (n > seen && layer == 0 && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(err_flag, 4);
  const int per_page = n_kv * kPageTokens;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < (long long)((seen + kPageTokens - 1) / kPageTokens) * per_page; i += (long long)gridDim.x * 256) {
    const int lp = (int)(i / per_page), k = (int)(i - (long long)lp * per_page), t = lp * kPageTokens + k % kPageTokens;
    const int page = r.page_table[(size_t)b * r.max_pages + lp];
    if (page < 0 || page >= n_pages) {
      if (k == 0) atomicOr(err_flag, 1);
      continue;
    }
    if (t < seen) r.records[((size_t)layer * n_pages + page) * per_page + k] = harli_kv_record{0.f, t};
  }
}

}  // namespace

AttendWs attend_layout(const harli_ctx* c, int batch, int max_kv_len, void* base, bool scores, int n_new, size_t* bytes) {
  const harli_model_cfg& m = c->cfg;
  AttendWs w;
  w.chunk = m.dtype == HARLI_BF16 ? attend_chunk_bf16(m.head_dim, m.n_q_heads / m.n_kv_heads) : kChunkF32;
  w.n_chunks = (max_kv_len + w.chunk - 1) / w.chunk;
  w.score_ld = w.n_chunks * w.chunk;
  w.n_new = n_new;
  auto al = [](size_t n) { return (n + 255) & ~size_t(255); };
  const size_t heads = (size_t)batch * m.n_q_heads, ml = al(heads * w.n_chunks * 8), o = al(heads * w.n_chunks * m.head_dim * 4);
  char* p = static_cast<char*>(base);
  w.ml = reinterpret_cast<float*>(p);
  w.o = reinterpret_cast<float*>(p + ml);
  w.scores = scores ? reinterpret_cast<float*>(p + ml + o) : nullptr;
  if (bytes) *bytes = ml + o + al(heads * w.score_ld * 4);
  return w;
}

harli_status check_tracking(const harli_ctx* c, const harli_tracking* t, int batch, int max_kv_len, const char* who) {
  if (!(t->decay >= 0.f && t->decay <= 1.f)) return fail(HARLI_ERR_INVALID, "%s: decay %g outside 0..1", who, t->decay);
  if ((uintptr_t)t->records % 16) return fail(HARLI_ERR_INVALID, "%s: records are not 16-byte aligned", who);
  const size_t need = harli_kv_attend_workspace_bytes(c, batch, max_kv_len);
  if (!t->workspace || (uintptr_t)t->workspace % 256 || t->workspace_bytes < need)
    return fail(HARLI_ERR_INVALID, "%s: a 256-byte aligned workspace of %zu bytes is needed, got %zu", who, need, t->workspace ? t->workspace_bytes : 0);
  return HARLI_OK;
}

void attend_f32(harli_ctx* c, const float* q, const int* kv_len, const int* page_table, int batch, int max_pages, int layer,
                const AttendWs& att, hipStream_t st) {
  const harli_model_cfg& m = c->cfg;
  const int d = m.head_dim;
#define ATT_F32(EL_)                                                                                                              \
  hipLaunchKernelGGL(k_attend_f32<EL_>, dim3(m.n_q_heads * att.n_chunks, batch, (d + 64 * EL_ - 1) / (64 * EL_)), dim3(256), 0, st, q, kv_len, \
                     page_table, max_pages, layer, m.n_q_heads, m.n_kv_heads, d, c->slab, c->geom, c->dw.err_flag, att)
  if (d <= 64) ATT_F32(1);
  else if (d <= 128) ATT_F32(2);
  else if (d <= 256) ATT_F32(4);
  else ATT_F32(16);
#undef ATT_F32
}

void attend_finish(harli_ctx* c, const AttendWs& att, const int* kv_len, const int* page_table, int batch, int max_pages, int layer,
                   float* out, unsigned short* frag, const harli_tracking* t, hipStream_t st) {
  const harli_model_cfg& m = c->cfg;
  // Workgroups of a KV head: one per block of records as far as the chip holds them, and for the output rows two per CU.  In us for the
  // whole call, bf16, heads of 128: 32 sequences of about 3000 tokens, 28 / 4 heads, 1 / 4 / as many parts as there are blocks (8):
  // 66.3 / 61.4 / 58.9; 192 of about 800, the longest 3076, 1 / 2 / 4: 120 / 111 / 109; one of 32001, 32 / 8 heads, 8 (for the
  // output rows alone) / 32: 45.3 / 40.3.  Output rows with one / two / four / sixteen workgroups per CU: 16 of 1024, 32 / 8 heads, 24.4 /
  // 24.9 / 26.5 / 26.5; 64 of 200, 28 / 4 heads, 20.7 / 19.8 / 20.7 / 24.5.
  const int G = m.n_q_heads / m.n_kv_heads, blocks = att.scores ? (att.score_ld + kFinishTokens - 1) / kFinishTokens : 0;
  const int pieces = G * ((m.head_dim + kPiece - 1) / kPiece), heads = batch * m.n_kv_heads;
  const int parts = std::max({1, std::min(blocks, 16 * c->n_cu / heads), std::min(pieces, 2 * c->n_cu / heads)});
  const FinishArgs a{kv_len, page_table, t->position, max_pages, layer, m.n_q_heads, m.n_kv_heads, m.head_dim, c->geom.n_pages_total, parts,
                     out, frag, t->records, t->decay};
  const dim3 grid(m.n_kv_heads * parts, batch);
  const size_t lds = (size_t)G * 8;
  if (m.head_dim % 4 == 0) hipLaunchKernelGGL(k_attend_finish<4>, grid, dim3(256), lds, st, a, att);
  else hipLaunchKernelGGL(k_attend_finish<2>, grid, dim3(256), lds, st, a, att);
}

}  // namespace harli

using namespace harli;

extern "C" size_t harli_kv_attend_workspace_bytes(const harli_ctx* c, int32_t batch, int32_t max_kv_len) {
  if (!c || batch < 1 || batch > c->cfg.max_batch || max_kv_len < 1 || max_kv_len > c->cfg.max_seq_len) return 0;
  size_t n = 0;
  (void)attend_layout(c, batch, max_kv_len, nullptr, true, 0, &n);
  return n;
}

extern "C" harli_status harli_kv_attend(harli_ctx* c, const harli_attend_batch* b, void* hip_stream) {
  if (!c || !b) return fail(HARLI_ERR_INVALID, "kv_attend: null argument");
  const harli_model_cfg& m = c->cfg;
  if (b->batch < 1 || b->batch > m.max_batch) return fail(HARLI_ERR_INVALID, "kv_attend: batch %d outside 1..%d", b->batch, m.max_batch);
  if (b->layer < 0 || b->layer >= m.n_layers) return fail(HARLI_ERR_INVALID, "kv_attend: layer %d outside 0..%d", b->layer, m.n_layers - 1);
  if (!b->q || !b->out || !b->n_tokens || !b->page_table) return fail(HARLI_ERR_INVALID, "kv_attend: q, out, n_tokens and page_table are required");
  if (((uintptr_t)b->q | (uintptr_t)b->out) % 16) return fail(HARLI_ERR_INVALID, "kv_attend: q and out have to be 16-byte aligned");
  if (b->max_kv_len < 1 || b->max_kv_len > m.max_seq_len) return fail(HARLI_ERR_INVALID, "kv_attend: max_kv_len %d outside 1..%d", b->max_kv_len, m.max_seq_len);
  if (b->max_pages > kMostPages || (long long)b->max_pages * kPageTokens < b->max_kv_len)
    return fail(HARLI_ERR_INVALID, "kv_attend: page table rows of %d pages cannot hold %d tokens", b->max_pages, b->max_kv_len);
  harli_status s = check_tracking(c, &b->track, b->batch, b->max_kv_len, "kv_attend");
  if (s != HARLI_OK) return s;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const AttendWs att = attend_layout(c, b->batch, b->max_kv_len, b->track.workspace, b->track.records != nullptr, 0);
  if (m.dtype == HARLI_BF16) {
    s = attend_bf16(c, b, att, st);
    if (s != HARLI_OK) return s;
  } else {
    attend_f32(c, b->q, b->n_tokens, b->page_table, b->batch, b->max_pages, b->layer, att, st);
  }
  attend_finish(c, att, b->n_tokens, b->page_table, b->batch, b->max_pages, b->layer, b->out, nullptr, &b->track, st);
  HARLI_HIP(hipGetLastError());
  return HARLI_OK;
}

extern "C" harli_status harli_kv_record_init(harli_ctx* c, const harli_record_batch* b, void* hip_stream) {
  if (!c || !b) return fail(HARLI_ERR_INVALID, "kv_record_init: null argument");
  const harli_model_cfg& m = c->cfg;
  if (b->batch < 1 || b->batch > m.max_batch) return fail(HARLI_ERR_INVALID, "kv_record_init: batch %d outside 1..%d", b->batch, m.max_batch);
  if (!b->n_tokens || !b->page_table || !b->records) return fail(HARLI_ERR_INVALID, "kv_record_init: n_tokens, page_table and records are required");
  if ((uintptr_t)b->records % 16) return fail(HARLI_ERR_INVALID, "kv_record_init: records are not 16-byte aligned");
  if (b->max_kv_len < 1 || b->max_kv_len > m.max_seq_len) return fail(HARLI_ERR_INVALID, "kv_record_init: max_kv_len %d outside 1..%d", b->max_kv_len, m.max_seq_len);
  if (b->max_pages > kMostPages || (long long)b->max_pages * kPageTokens < b->max_kv_len)
    return fail(HARLI_ERR_INVALID, "kv_record_init: page table rows of %d pages cannot hold %d tokens", b->max_pages, b->max_kv_len);
  const long long most = (long long)((b->max_kv_len + kPageTokens - 1) / kPageTokens) * m.n_kv_heads * kPageTokens;
  const int blocks = (int)((most + 255) / 256);
  hipLaunchKernelGGL(k_record_init, dim3(blocks, b->batch, m.n_layers), dim3(256), 0, static_cast<hipStream_t>(hip_stream), *b, m.n_kv_heads,
                     c->geom.n_pages_total, c->dw.err_flag);
  HARLI_HIP(hipGetLastError());
  return HARLI_OK;
}
