// Losses over a vocabulary (abl_xent_*, abl_distill_*): what the launchers take.
#pragma once

#include "block_store.h"

namespace abl {

constexpr int kTopEntries = 1024;   // of a row at most

// A call as the launchers see it: an xent call has T = 0, temperature 1, label_weight 1 and teacher_weight 0.
struct HeadCall {
  abl_head p;
  Rows h, W;
  const int64_t* labels;       // nullptr: none
  const int64_t* ids;          // [M][T]; nullptr: no teacher
  const float* logits;
  float *loss, *lse, *lse_t, *z_top;              // forward: written (lse may be nullptr, the last two are where there is no teacher)
  const float *in_lse, *in_lse_t, *in_z_top;      // backward: read
  const float* dloss;
  RowsOut dh;                  // p = nullptr: not wanted
  void* dW;
};

size_t head_layout_bytes(const abl_head& p, bool backward, bool copied);   // of one call's workspace; copied: whether the table is
size_t head_scratch_bytes(const abl_head& p, bool backward);               // of any call's
// (nothing is launched where the call's layout exceeds scratch_bytes)
int launch_head_forward(hipStream_t st, const HeadCall& c, void* scratch, size_t scratch_bytes);
int launch_head_backward(hipStream_t st, const HeadCall& c, void* scratch, size_t scratch_bytes);

}  // namespace abl
