// Attention that records weights: what its chunk kernels (decode.hip on bf16 storage, attend.hip on fp32) and the kernel that
// joins the chunks share.
#pragma once
#include "ctx.h"

namespace harli {

struct AttendWs {
  float* o = nullptr;       // [batch][n_q][n_chunks][d] outputs of the chunks, not normalised
  float* ml = nullptr;      // [batch][n_q][n_chunks][2] their (maximum, sum), the maximum in the log2 domain
  float* scores = nullptr;  // [batch][n_q][score_ld] q.k / sqrt(d) * log2(e), or null: nothing is recorded
  int score_ld = 0, n_chunks = 0, chunk = 0;
  int n_new = 0;            // tokens of a sequence beyond its count: 1 where the count is of the tokens before the step
};

// The workspace at `base` for a batch and length bound; with base null only *bytes is of use.
AttendWs attend_layout(const harli_ctx* c, int batch, int max_kv_len, void* base, bool scores, int n_new, size_t* bytes = nullptr);
// Checks of harli_tracking shared by the entry points (host only).
harli_status check_tracking(const harli_ctx* c, const harli_tracking* t, int batch, int max_kv_len, const char* who);

int attend_chunk_bf16(int d, int G);                                                                     // decode.hip
harli_status attend_bf16(harli_ctx* c, const harli_attend_batch* b, const AttendWs& att, hipStream_t st);  // decode.hip
void attend_f32(harli_ctx* c, const float* q, const int* kv_len, const int* page_table, int batch, int max_pages, int layer,
                const AttendWs& att, hipStream_t st);
// Joins the chunks: output rows in fp32 (out) or as the operand of the step's output projection (frag), records where t has some.
void attend_finish(harli_ctx* c, const AttendWs& att, const int* kv_len, const int* page_table, int batch, int max_pages, int layer,
                   float* out, unsigned short* frag, const harli_tracking* t, hipStream_t st);

}  // namespace harli
