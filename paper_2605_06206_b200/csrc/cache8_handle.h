// The handle behind include/foe_cache.h and what the layer's forward pass uses of it (internal to the library).
#pragma once

#include "../../include/foe_cache.h"
#include "cache8.h"

struct foe_cache {
  foe_cache_config cfg;
  int device, n_sms, rows_max;          // rows_max: most query rows of a call
  void* memory;                         // the workspace that the pointers below are parts of
  int* status;
  float *part_o, *part_ml, *lse, *logits;
  int* split_done;
  int4* division;
  size_t split_done_count;
  long long logits_stride;
  foe::Cache8Workspace ws;
  __nv_bfloat16 *k_stage, *v_stage;     // K and V rows of a layer's call, in pages of 64 consecutive tokens
  int *tok_pos, *tok_slot;
  cudaStream_t last_stream;
};

namespace foe {

// argument checks of a view (the pointers and sizes that every call needs); FOE_OK or the error.  `rows`: query rows.
foe_status cache8_check(const foe_cache* h, const foe_cache_view* v, bool need_q, int* rows);
foe_status cache8_check_weights(const foe_cache* h, const foe_cache_view* v, const float* in, const float* out, long long stride, int window);
Cache8Args cache8_args(const foe_cache* h, const foe_cache_view* v, int* status);
// the attention of checked arguments, with its weights: launches only.  Returns the number of kernels launched, -1 on error.
int cache8_attend(foe_cache* h, const foe_cache_view* v, const void* q, long long q_stride, int q_head_stride, void* out,
                  long long out_stride, const float* w_in, float* w_out, long long w_stride, int window, int* status, cudaStream_t st);
// staged rows (a layer's projection) into the cache
void cache8_append_staged(foe_cache* h, const foe_cache_view* v, int* status, cudaStream_t st);
// position and staging slot of every token of a layer's call
void launch_cache8_token_map(const int* q_lens, const int* positions, int n_seqs, int n_tokens, int max_context, int* tok_pos,
                             int* tok_slot, int* status, cudaStream_t st);

}  // namespace foe
