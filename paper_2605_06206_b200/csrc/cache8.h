// Host-callable launchers of the 8-bit cache kernels (internal to the library).
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace foe {

// One call's view of the cache (device pointers) and its shapes.
struct Cache8Args {
  uint8_t *k_pages, *v_pages;       // [num_pages][n_kv][64][dh] codes
  float *k_scales, *v_scales;       // [num_pages][n_kv]
  const int* block_table;           // [n_seqs][max_pages_per_seq]
  const int* context_lens;          // [n_seqs] tokens cached before the call
  const int* q_lens;                // [n_seqs] new tokens, or nullptr: one each
  int n_seqs, max_pages_per_seq, num_pages, n_tokens, max_q_len;
  int n_q, n_kv, dh;
  int few_q;                        // sequences of up to this many new tokens go the way of single tokens
  int max_len;                      // tokens a sequence may reach: min(64 * table width, the handle's max_context)
  int max_kv_pages;                 // pages of that many tokens
  int* status;
};

// where the row of (token t, head h) starts: (t / 64) * tile + (t % 64) * row + h * head elements
struct Cache8Rows { long long tile, row, head; };

struct Cache8AppendArgs {
  Cache8Args c;
  const __nv_bfloat16 *k, *v;
  Cache8Rows k_lay, v_lay;
};

struct Cache8AttendArgs {
  Cache8Args c;
  const __nv_bfloat16* q;           // [n_tokens] rows of n_q heads
  long long q_stride;               // elements between two tokens' rows
  int q_head_stride;                // elements between two heads of a row
  __nv_bfloat16* out;               // [n_tokens] rows of n_q * dh values
  long long out_stride;
  float scale_log2;                 // log2(e) / sqrt(dh)
  // partial results of a (sequence, KV head) whose keys are worked on by several CTAs
  float *part_o, *part_ml;
  int* split_done;
  int4* division;                   // chunks whose keys are split: every block's first CTA, CTAs, first token and rows
  // for the accumulated weights (nullptr without them)
  float* lse;                       // [n_tokens][n_q] log2 of the row's softmax denominator
  float* logits;                    // single tokens: [n_seqs][n_q][logits_stride] scores in the log2 domain
  long long logits_stride;
};

struct Cache8WeightsArgs {
  Cache8AttendArgs a;
  const float* weights_in;          // [n_seqs][n_kv][weights_stride]
  float* weights_out;
  long long weights_stride;
  int window;                       // the last `window` queries of a sequence count; 0: all
};

struct Cache8EvictArgs {
  Cache8Args c;                     // context_lens = tokens cached
  const float* weights;             // [n_seqs][n_kv][weights_stride]
  long long weights_stride;
  const int* to_table;              // [n_seqs][to_pages_per_seq]
  int to_pages_per_seq;
  int budget, sink, recent;
  int* new_lens;                    // [n_seqs]
  int* kept;                        // [n_seqs][n_kv][budget]
  float* weights_out;               // [n_seqs][n_kv][weights_out_stride], or nullptr
  long long weights_out_stride;
};

// fmt: kC8E4M3 or kC8Int8 (cache8.cuh)
void launch_cache8_append(int fmt, const Cache8AppendArgs& a, cudaStream_t st);
// single tokens: q_lens nullptr, or the sequences with 1 <= q_lens <= few_q
void launch_cache8_decode(int fmt, const CUtensorMap& tmK, const CUtensorMap& tmV, const Cache8AttendArgs& a, int n_sms,
                          cudaStream_t st);
size_t cache8_decode_part_rows(int n_sms);   // rows of part_o / part_ml
cudaError_t cache8_decode_configure();
// Operand tiles of long chunks' sequences: K bf16, V fp16 [pages][n_kv][64][dh padded to 64 or 128], with their scales and maps
// (64 x 64 boxes).  pages is at least what the longest sequence of a call needs.
struct Cache8Workspace {
  __nv_bfloat16* k;
  __half* v;
  float4* scales;
  long long pages;
  CUtensorMap tmK, tmV;
};
// chunks: q_lens given, n_tokens rows in all; tmQ maps q as [tokens][heads][dh] with boxes of 128 x 1 x 64.  part_o / part_ml hold cache8_chunk_part_rows(n_sms) rows; ws is used by calls
// with max_q_len >= cache8_expand_min_tokens(n_q / n_kv, dh).
// Sequences of fewer than min_q tokens are left out.  Returns the number of kernels launched.
int launch_cache8_chunk(int fmt, const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const Cache8AttendArgs& a,
                        const Cache8Workspace& ws, int min_q, int n_sms, cudaStream_t st);
int cache8_expand_min_tokens(int group, int dh);    // group: query heads per KV head
int cache8_chunk_max_split_blocks();
size_t cache8_chunk_part_rows(int n_sms);
cudaError_t cache8_chunk_configure();
void launch_cache8_weights(int fmt, const Cache8WeightsArgs& w, int n_sms, cudaStream_t st);
void launch_cache8_evict(int fmt, const Cache8EvictArgs& a, int n_sms, cudaStream_t st);
cudaError_t cache8_evict_configure();

}  // namespace foe
