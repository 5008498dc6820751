// C entry points of sampled speculative decoding: argument checks and launches.
#include "sample.cuh"

namespace {

using namespace dvi;

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
// Null, or an array of 4-byte elements.
bool words_ok(const void* p) { return aligned(p, 4); }
// Whether rows of the probabilities share memory with rows of the logits (n of each, ld bytes from row to
// row).  They may be the same numbers; rows that lie between the others' are found apart only for equal ld.
bool overlap(uintptr_t x, int64_t ld_x, int64_t row_x, uintptr_t out, int64_t ld_out, int64_t row_out, int64_t n) {
  if (x == out && row_x == row_out && (n == 1 || ld_x == ld_out)) return false;
  if (x + (n - 1) * ld_x + row_x <= out || out + (n - 1) * ld_out + row_out <= x) return false;
  if (n == 1 || ld_x != ld_out) return true;
  const int64_t d = static_cast<int64_t>(out - x) % ld_x, at = d < 0 ? d + ld_x : d;
  return at < row_x || at + row_out > ld_x;
}
// The launchers refuse grids past 31 bits.
dvi_status launched(cudaError_t e) {
  return e == cudaSuccess ? DVI_OK : e == cudaErrorInvalidConfiguration ? DVI_ERR_CAPACITY : DVI_ERR_CUDA;
}

}  // namespace

extern "C" dvi_status dvi_token_probs(int dtype, const void* d_logits, int64_t ld_logits, int n_rows, int vocab,
                                      const dvi_sampling* sampling, float* d_probs, int64_t ld_probs,
                                      int32_t* d_status, dvi_stream stream) {
  if (!sampling || (dtype != DVI_F32 && dtype != DVI_BF16) || n_rows < 0 || vocab < 1) return DVI_ERR_INVALID_ARG;
  if (vocab > kMaxVocab || n_rows > (1 << 30)) return DVI_ERR_CAPACITY;
  // (a setting that is not a number is refused here; one in a device array is flagged there)
  if (!sampling->temperature && !(sampling->temperature_all >= 0.f)) return DVI_ERR_INVALID_ARG;
  if (!sampling->top_k && sampling->top_k_all < 0) return DVI_ERR_INVALID_ARG;
  if (!sampling->top_p && !(sampling->top_p_all >= 0.f)) return DVI_ERR_INVALID_ARG;
  if (!words_ok(sampling->temperature) || !words_ok(sampling->top_k) || !words_ok(sampling->top_p) ||
      !words_ok(d_status))
    return DVI_ERR_INVALID_ARG;
  if (n_rows == 0) return DVI_OK;
  if (!d_logits || !d_probs || !aligned(d_logits, dtype == DVI_F32 ? 4 : 2) || !aligned(d_probs, 4) ||
      ld_logits < vocab || ld_probs < vocab)
    return DVI_ERR_INVALID_ARG;
  const int64_t e = dtype == DVI_F32 ? 4 : 2;
  if (overlap(reinterpret_cast<uintptr_t>(d_logits), ld_logits * e, vocab * e, reinterpret_cast<uintptr_t>(d_probs),
              ld_probs * 4, vocab * int64_t{4}, n_rows))
    return DVI_ERR_INVALID_ARG;
  TokenProbsArgs a{};
  a.x = d_logits;
  a.ld = ld_logits;
  a.out = d_probs;
  a.ld_out = ld_probs;
  a.n_rows = n_rows;
  a.vocab = vocab;
  a.temperature = sampling->temperature;
  a.top_k = sampling->top_k;
  a.top_p = sampling->top_p;
  a.temperature_all = sampling->temperature_all;
  a.top_k_all = sampling->top_k_all;
  a.top_p_all = sampling->top_p_all;
  a.status = d_status;
  cudaGetLastError();   // an error left pending by the caller is not this call's
  return launched(launch_token_probs(a, dtype, reinterpret_cast<cudaStream_t>(stream)));
}

extern "C" dvi_status dvi_verify_drafts(const dvi_draft_batch* batch, const float* d_target, int64_t ld_target,
                                        const float* d_draft, int64_t ld_draft, int32_t* d_out_ids,
                                        int32_t* d_n_committed, int32_t* d_n_accepted, dvi_stream stream) {
  const dvi_draft_batch* b = batch;
  if (!b || b->n_seqs < 0 || b->vocab < 1 || b->n_drafts < 0 || b->max_drafts < 0 || (b->bonus != 0 && b->bonus != 1))
    return DVI_ERR_INVALID_ARG;
  if (b->n_seqs > kMaxSampleSeqs || b->vocab > kMaxVocab || b->n_drafts > (1 << 30) || b->max_drafts > (1 << 20))
    return DVI_ERR_CAPACITY;
  if (b->n_seqs == 0) return b->n_drafts == 0 ? DVI_OK : DVI_ERR_INVALID_ARG;
  if (!b->draft_start && (b->n_drafts % b->n_seqs || b->max_drafts < b->n_drafts / b->n_seqs))
    return DVI_ERR_INVALID_ARG;
  if (!d_n_committed || !d_n_accepted || !words_ok(d_n_committed) || !words_ok(d_n_accepted) || !b->u_token ||
      !words_ok(b->u_token) || !words_ok(b->status) || !words_ok(b->draft_start))
    return DVI_ERR_INVALID_ARG;
  if (b->max_drafts + b->bonus > 0 && (!d_out_ids || !words_ok(d_out_ids))) return DVI_ERR_INVALID_ARG;
  if (b->n_drafts > 0 && (!b->draft_ids || !b->u_accept || !words_ok(b->draft_ids) || !words_ok(b->u_accept)))
    return DVI_ERR_INVALID_ARG;
  if (b->n_drafts + b->bonus > 0 && (!d_target || !words_ok(d_target) || ld_target < b->vocab))
    return DVI_ERR_INVALID_ARG;
  if (d_draft && (!words_ok(d_draft) || ld_draft < b->vocab)) return DVI_ERR_INVALID_ARG;
  VerifyArgs a{};
  a.p = d_target;
  a.ld_p = ld_target;
  a.q = d_draft;
  a.ld_q = ld_draft;
  a.ids = b->draft_ids;
  a.start = b->draft_start;
  a.u_accept = b->u_accept;
  a.u_token = b->u_token;
  a.out = d_out_ids;
  a.n_committed = d_n_committed;
  a.n_accepted = d_n_accepted;
  a.status = b->status;
  a.n_seqs = b->n_seqs;
  a.vocab = b->vocab;
  a.n_drafts = b->n_drafts;
  a.max_drafts = b->max_drafts;
  a.bonus = b->bonus;
  cudaGetLastError();
  return launched(launch_verify_drafts(a, reinterpret_cast<cudaStream_t>(stream)));
}

extern "C" dvi_status dvi_paged_plan(const dvi_page_pool* pool, const int32_t* d_lens, const int32_t* d_rows,
                                     int rows_each, int n_rows, int32_t* d_row_start, int64_t* d_slots,
                                     int32_t* d_positions, dvi_stream stream) {
  if (!pool || pool->n_pages < 1 || pool->n_seqs < 1 || pool->max_pages < 1 || n_rows < 0 || rows_each < 0)
    return DVI_ERR_INVALID_ARG;
  const int P = pool->page_tokens;
  if (P != 16 && P != 32 && P != 64 && P != 128) return DVI_ERR_INVALID_ARG;
  // positions and row counts are 32-bit numbers on the device
  if (pool->n_seqs > kPlanSeqs || static_cast<int64_t>(pool->max_pages) * P > (1ll << 30) || n_rows > (1 << 30) ||
      rows_each > (1 << 30))
    return DVI_ERR_CAPACITY;
  if (!pool->stack || !pool->n_free || !pool->table || !pool->held || !d_lens || !words_ok(pool->stack) ||
      !words_ok(pool->n_free) || !words_ok(pool->table) || !words_ok(pool->held) || !words_ok(pool->status) ||
      !words_ok(d_lens) || !words_ok(d_rows) || !words_ok(d_row_start) || !words_ok(d_positions) ||
      !aligned(d_slots, 8))
    return DVI_ERR_INVALID_ARG;
  PagePlanArgs a{};
  a.stack = pool->stack;
  a.n_free = pool->n_free;
  a.table = pool->table;
  a.held = pool->held;
  a.status = pool->status;
  a.lens = d_lens;
  a.rows = d_rows;
  a.rows_each = rows_each;
  a.n_pages = pool->n_pages;
  a.log_p = P == 16 ? 4 : P == 32 ? 5 : P == 64 ? 6 : 7;
  a.n_seqs = pool->n_seqs;
  a.max_pages = pool->max_pages;
  a.n_rows = d_slots || d_positions ? n_rows : 0;
  a.row_start = d_row_start;
  a.slots = d_slots;
  a.positions = d_positions;
  cudaGetLastError();
  return launched(launch_page_plan(a, reinterpret_cast<cudaStream_t>(stream)));
}
