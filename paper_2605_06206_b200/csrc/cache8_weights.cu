// Accumulated attention weights: weights_out[b][h][j] = weights_in[b][h][j] + sum of the probabilities that key j of KV
// head h received from the counted queries, over the query heads of the KV head.
//
// Single tokens: the decode kernel has left every score in the log2 domain and each row's denominator, so this is one pass
// over 4 bytes per (query head, key).  Chunks: the scores are formed again, S^T = K q^T with the keys as the M side, so
// that a thread's accumulators belong to two keys and the sum over query rows stays in the thread; a block owns a page of
// a KV head, so nothing is added atomically and the result does not depend on any order.
#include "cache8.cuh"
#include "cache8.h"

namespace foe {

// ------------------------------------------------------------------------------------------- single tokens
constexpr int kWtThreads = 128, kWtKeys = 4;     // keys of a thread (their loads are in flight together)
__global__ void __launch_bounds__(kWtThreads)
cache8_weights_token_kernel(const Cache8WeightsArgs w) {
  pdl_wait();
  pdl_launch_dependents();
  const Cache8AttendArgs& a = w.a;
  const Cache8Args& c = a.c;
  const int b = blockIdx.z, kvh = blockIdx.y;
  const int G = c.n_q / c.n_kv;
  const int len = min(max(c.context_lens[b], 0) + 1, c.max_len);
  const int j0 = blockIdx.x * (kWtThreads * kWtKeys) + threadIdx.x;
  if (j0 - int(threadIdx.x) >= len) return;
  const float* lse = a.lse + size_t(b) * c.n_q + kvh * G;
  const float* s = a.logits + (size_t(b) * c.n_q + kvh * G) * a.logits_stride;
  const size_t row = (size_t(b) * c.n_kv + kvh) * w.weights_stride;
  float p[kWtKeys];
#pragma unroll
  for (int i = 0; i < kWtKeys; ++i) p[i] = 0.f;
#pragma unroll 2
  for (int h = 0; h < G; ++h) {
    const float l = lse[h];
#pragma unroll
    for (int i = 0; i < kWtKeys; ++i) {
      const int j = j0 + i * kWtThreads;
      if (j < len) p[i] += fast_exp2(s[h * a.logits_stride + j] - l);
    }
  }
#pragma unroll
  for (int i = 0; i < kWtKeys; ++i) {
    const int j = j0 + i * kWtThreads;
    if (j < len) w.weights_out[row + j] = w.weights_in[row + j] + p[i];
  }
}

// ------------------------------------------------------------------------------------------- chunks
constexpr int kWcThreads = 128;                  // four warps, 16 keys of every page each
constexpr int kWcPages = 4;                      // pages of a block: what its query rows cost to bring in is spent once for them
constexpr int kWcRows = 64;                      // query rows in shared memory at a time
template <int FMT, int DH>
__global__ void __launch_bounds__(kWcThreads)
cache8_weights_chunk_kernel(const Cache8WeightsArgs w) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int NC = DH / 16;
  // Rows as B fragments: [row tile of 8][k-step][lane] two registers; factor, log2 of the denominator and position of every row
  __shared__ uint2 frag[kWcRows / 8][NC][32];
  __shared__ float row_f[kWcRows], row_lse[kWcRows];
  __shared__ int row_pos[kWcRows];
  __shared__ int red[kWcThreads / 32];
  const Cache8AttendArgs& a = w.a;
  const Cache8Args& c = a.c;
  const int page0 = blockIdx.x * kWcPages, kvh = blockIdx.y, b = blockIdx.z;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
  const int G = c.n_q / c.n_kv;
  const int ctx = c.context_lens[b], q_len = c.q_lens[b];
  if (q_len < 0 || q_len > c.max_q_len || ctx < 0 || (long long)ctx + q_len > c.max_len) return;   // (reported by the attention)
  const int len = ctx + q_len;
  if (page0 * 64 >= len) return;
  const int start = c8_block_prefix(c.q_lens, b, red);
  if ((long long)start + q_len > c.n_tokens) return;
  const int n_pages = min(kWcPages, (len + 63) / 64 - page0);
  // counted queries that see any key of the pages
  const int i_first = max(w.window > 0 ? max(q_len - w.window, 0) : 0, page0 * 64 - ctx);
  const int n_rows = (q_len - i_first) * G;
  float sum[kWcPages][2];                                           // keys g and g + 8 of the warp's 16 keys of every page
#pragma unroll
  for (int i = 0; i < kWcPages; ++i) sum[i][0] = sum[i][1] = 0.f;

  for (int base = 0; base < n_rows; base += kWcRows) {
    const int here = min(kWcRows, n_rows - base);
    __syncthreads();                                                // the rows before have been used
    for (int tile = warp; tile * 8 < here; tile += kWcThreads / 32) {
      const int r = base + tile * 8 + g;
      const bool there = r < n_rows;
      const int i = i_first + r / G, h = r % G;
      uint4 v[NC / 4][2];
      uint32_t mx = 0;
#pragma unroll
      for (int hh = 0; hh < NC / 4; ++hh) {
        const int d0 = (t4 + 4 * hh) * 16;
        v[hh][0] = v[hh][1] = make_uint4(0, 0, 0, 0);
        if (there && d0 < c.dh) {
          const uint4* p = reinterpret_cast<const uint4*>(a.q + (long long)(start + i) * a.q_stride + (kvh * G + h) * a.q_head_stride + d0);
          v[hh][0] = __ldg(p);
          v[hh][1] = __ldg(p + 1);
        }
        mx = max(mx, max(c8_absmax(v[hh][0]), c8_absmax(v[hh][1])));
      }
      mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      const int eq = c8_query_exp(mx);
      const float down = c8_pow2(-eq);
#pragma unroll
      for (int hh = 0; hh < NC / 4; ++hh) {
        const uint32_t x[8] = {v[hh][0].x, v[hh][0].y, v[hh][0].z, v[hh][0].w, v[hh][1].x, v[hh][1].y, v[hh][1].z, v[hh][1].w};
#pragma unroll
        for (int k = 0; k < 4; ++k)
          frag[tile][hh * 4 + k][lane] = make_uint2(pack_f16(bf16_lo(x[2 * k]) * down, bf16_hi(x[2 * k]) * down),
                                                    pack_f16(bf16_lo(x[2 * k + 1]) * down, bf16_hi(x[2 * k + 1]) * down));
      }
      if (t4 == 0) {
        row_f[tile * 8 + g] = c8_pow2(eq) * a.scale_log2;
        row_lse[tile * 8 + g] = there ? a.lse[size_t(start + i) * c.n_q + kvh * G + h] : 0.f;
        row_pos[tile * 8 + g] = there ? ctx + i : -1;               // (a row that is none sees no key)
      }
    }
    __syncthreads();
#pragma unroll
    for (int pi = 0; pi < kWcPages; ++pi) {
      if (pi >= n_pages) break;
      const int page = c.block_table[size_t(b) * c.max_pages_per_seq + page0 + pi];
      if (page < 0 || page >= c.num_pages) continue;
      const size_t ph = size_t(page) * c.n_kv + kvh;
      const int key0 = (page0 + pi) * 64 + warp * 16;
      // this warp's 16 keys as A fragments: row g is key key0 + g, row g + 8 key key0 + g + 8; a lane holds the codes of
      // chunks t4 and t4 + 4
      uint32_t ka[NC][4];
#pragma unroll
      for (int hh = 0; hh < NC / 4; ++hh) {
        const int d0 = (t4 + 4 * hh) * 16;
        uint4 x = make_uint4(0, 0, 0, 0), y = x;
        if (d0 < c.dh) {
          const uint8_t* p = c.k_pages + (ph * 64 + warp * 16 + g) * c.dh + d0;
          x = *reinterpret_cast<const uint4*>(p);
          y = *reinterpret_cast<const uint4*>(p + 8 * c.dh);
        }
        const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          c8_decode_natural<FMT>(xs[i], ka[hh * 4 + i][0], ka[hh * 4 + i][2]);
          c8_decode_natural<FMT>(ys[i], ka[hh * 4 + i][1], ka[hh * 4 + i][3]);
        }
      }
      const float sk = c.k_scales[ph];
      for (int tile = 0; tile * 8 < here; ++tile) {
        float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NC; ++k) {
          const uint2 q = frag[tile][k][lane];
          mma_f16_16816(s, ka[k][0], ka[k][1], ka[k][2], ka[k][3], q.x, q.y);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {                               // columns 2 t4, 2 t4 + 1
          const int r = tile * 8 + t4 * 2 + e;
          const float f = row_f[r] * sk, l = row_lse[r];
          const int pos = row_pos[r];
          if (key0 + g <= pos) sum[pi][0] += fast_exp2(fmaf(s[e], f, -l));
          if (key0 + g + 8 <= pos) sum[pi][1] += fast_exp2(fmaf(s[e + 2], f, -l));
        }
      }
    }
  }
  const size_t row = (size_t(b) * c.n_kv + kvh) * w.weights_stride;
#pragma unroll
  for (int pi = 0; pi < kWcPages; ++pi) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float v = sum[pi][e];
      v += __shfl_xor_sync(0xffffffffu, v, 1);
      v += __shfl_xor_sync(0xffffffffu, v, 2);
      const int key = (page0 + pi) * 64 + warp * 16 + g + 8 * e;
      if (t4 == 0 && pi < n_pages && key < len) w.weights_out[row + key] = w.weights_in[row + key] + v;
    }
  }
}

void launch_cache8_weights(int fmt, const Cache8WeightsArgs& w, cudaStream_t st) {
  const Cache8Args& c = w.a.c;
  if (c.n_seqs <= 0) return;
  if (!c.q_lens) {
    const dim3 grid(unsigned((c.max_len + kWtThreads * kWtKeys - 1) / (kWtThreads * kWtKeys)), c.n_kv, c.n_seqs);
    launch_pdl(cache8_weights_token_kernel, grid, dim3(kWtThreads), 0, st, w);
    return;
  }
  const dim3 grid((c.max_kv_pages + kWcPages - 1) / kWcPages, c.n_kv, c.n_seqs);
  if (fmt == kC8E4M3) {
    if (c.dh > 64) launch_pdl(cache8_weights_chunk_kernel<kC8E4M3, 128>, grid, dim3(kWcThreads), 0, st, w);
    else launch_pdl(cache8_weights_chunk_kernel<kC8E4M3, 64>, grid, dim3(kWcThreads), 0, st, w);
  } else {
    if (c.dh > 64) launch_pdl(cache8_weights_chunk_kernel<kC8Int8, 128>, grid, dim3(kWcThreads), 0, st, w);
    else launch_pdl(cache8_weights_chunk_kernel<kC8Int8, 64>, grid, dim3(kWcThreads), 0, st, w);
  }
}

}  // namespace foe
