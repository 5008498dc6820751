// Sampled speculative decoding: arguments and launchers of the token
// probabilities, the verification of drafts and the page plan.
#pragma once

#include "common.cuh"

namespace dvi {

constexpr int kMaxVocab = 1 << 18;        // tokens of a row (an index has 18 bits in the selection's keys)
constexpr int kMaxSampleSeqs = 1 << 16;   // sequences of a verification
constexpr int kPlanSeqs = 1024;           // slots of a page pool (as in a paged batch)

struct TokenProbsArgs {
  const void* x;            // logits [n_rows][vocab], ld elements from row to row
  int64_t ld;
  float* out;
  int64_t ld_out;
  int n_rows, vocab;
  const float* temperature; // [n_rows], or null: the same for all rows
  const int* top_k;
  const float* top_p;
  float temperature_all, top_p_all;
  int top_k_all;
  int* status;
};
cudaError_t launch_token_probs(const TokenProbsArgs& a, int dtype, cudaStream_t s);

struct VerifyArgs {
  const float* p;           // target rows: sequence b's first is its first draft's row + b * bonus
  int64_t ld_p;
  const float* q;           // drafter rows, or null: the one-hot rows of the drafted tokens
  int64_t ld_q;
  const int* ids;           // [n_drafts]
  const int* start;         // [n_seqs + 1], or null: n_drafts / n_seqs each
  const float* u_accept;    // [n_drafts]
  const float* u_token;     // [n_seqs]
  int* out;                 // [n_seqs][max_drafts + bonus]
  int* n_committed;
  int* n_accepted;
  int* status;
  int n_seqs, vocab, n_drafts, max_drafts, bonus;
};
cudaError_t launch_verify_drafts(const VerifyArgs& a, cudaStream_t s);

struct PagePlanArgs {
  int* stack;
  int* n_free;
  int* table;
  int* held;
  int* status;
  const int* lens;
  const int* rows;          // [n_seqs], or null: rows_each of every sequence
  int rows_each;
  int n_pages, log_p, n_seqs, max_pages, n_rows;
  int* row_start;           // [n_seqs + 1], or null
  int64_t* slots;           // [n_rows], or null
  int* positions;           // [n_rows], or null
};
cudaError_t launch_page_plan(const PagePlanArgs& a, cudaStream_t s);

}  // namespace dvi
