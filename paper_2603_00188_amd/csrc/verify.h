// Declarations shared by the host layer and the kernels of stlite_verify_drafts.
#pragma once

#include "stlite_internal.h"

namespace stlite {

struct VerifyArgs {
  int32_t n_seqs, vocab;
  int64_t total_new;
  const int32_t* cu_new;   // [n_seqs + 1]
  const void* target;      // [total_new] rows of vocab, target_stride apart
  const void* draft;       // the same, nullable
  int64_t target_stride, draft_stride;
  const int32_t* tokens;   // [total_new]
  const float* accept;     // [total_new]
  const float* pick;       // [n_seqs]
  int32_t* seq_lens;       // [n_seqs], nullable
  int32_t* out;            // [total_new]
  int32_t* n_out;          // [n_seqs]
  double2* sums;           // workspace [n_seqs][pieces]
  int32_t* stop;           // workspace [n_seqs]
  int32_t piece, pieces;   // entries of a row per wave, a multiple of 256; their number, of whole work-groups
};

constexpr int32_t kVerifyMinPiece = 256, kVerifyMaxPiece = 2048, kVerifyPieces = 4;  // (pieces of a work-group)

// type: 0 bf16, 1 fp16, 2 fp32
hipError_t launch_verify(const VerifyArgs& a, int type, hipStream_t stream);

}  // namespace stlite
