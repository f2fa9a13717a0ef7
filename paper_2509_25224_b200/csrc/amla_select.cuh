// What the launches of amla_select.cu take.
#pragma once

#include "amla_common.cuh"

namespace amla {

struct ScoreParams {
  const __nv_bfloat16* q;        // [B, Sq, H, 576]
  const __nv_bfloat16* means;    // [num_blocks, 576]
  const int32_t* block_table;    // [B, width]
  const int32_t* seqlens;        // [B]
  float scale_log2;
  int B, Sq, H, num_blocks, width;
  float* scores;                 // [B, Sq, width]
  int* status;
};

struct SelectParams {
  const float* scores;           // [B, Sq, width]; not read (may be null) where width <= keep
  const int32_t* block_table;
  const int32_t* seqlens;
  int B, Sq, width, keep, sink, recent;
  int32_t* table;                // [B * Sq, keep]
  int32_t* lens;                 // [B * Sq]
  int32_t* chosen;               // [B * Sq, keep] or null
  int* clear;                    // a status word that no scoring in front has set, or null
};

// The scores, and with `select` the choice by them in the same launch (where scores_select says that it can be).
bool scores_select(int width);
cudaError_t launch_page_scores(const ScoreParams& p, const SelectParams* select, int sms, cudaStream_t stream);
cudaError_t launch_pages_select(const SelectParams& p, cudaStream_t stream);

}  // namespace amla
