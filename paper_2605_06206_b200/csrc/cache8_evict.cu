// Eviction from the 8-bit cache by accumulated attention weight: every (sequence, KV head) keeps its first `sink`
// tokens, its last `recent` ones and the heaviest of the rest, budget tokens in all, in their order.
//
// Two launches.  The first chooses: one block per (sequence, KV head) finds the k-th largest weight by a radix search
// over the weights as ordered integers (three passes of 11, 11 and 10 bits, then one pass that writes the kept positions
// with a running prefix sum; ties go to the lower position).  The second copies: one block per (destination page, KV
// head, K or V) gathers its 64 rows, takes their largest magnitude and encodes them at a scale made for them.  Source and
// destination pages are disjoint, so all destination pages are built at once, and a source page that several sequences
// share (a common prompt prefix) is left as it is for the others.
// Bound: memory (4 bytes per weight, once per pass through L2; 2 bytes read and 2 written per kept K/V element pair).
#include "cache8.cuh"
#include "cache8.h"

namespace foe {

constexpr int kEvThreads = 512;
constexpr int kEvBins = 2048;

// order of the weights as unsigned integers: larger weight, larger key; -0 = +0; a NaN below everything
__device__ __forceinline__ uint32_t weight_key(float x) {
  uint32_t u = __float_as_uint(x);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;
  if (u == 0x80000000u) u = 0u;
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__global__ void __launch_bounds__(kEvThreads)
cache8_select_kernel(const Cache8EvictArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ uint32_t hist[kEvBins];
  __shared__ uint32_t warp_sum_s[kEvThreads / 32];
  __shared__ uint32_t found[2];
  const Cache8Args& c = a.c;
  const int b = blockIdx.y, kvh = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int len = c.context_lens[b];
  if (len < 0 || len > c.max_len) {
    if (tid == 0) atomicExch(c.status, kStatusBounds);
    len = 0;
  }
  const size_t row = size_t(b) * c.n_kv + kvh;
  const float* wt = a.weights + row * a.weights_stride;
  int* kept = a.kept + row * a.budget;
  float* wout = a.weights_out ? a.weights_out + row * a.weights_out_stride : nullptr;
  const int n_new = min(len, a.budget);
  if (kvh == 0 && tid == 0) a.new_lens[b] = n_new;
  if (len <= a.budget) {
    for (int j = tid; j < len; j += kEvThreads) {
      kept[j] = j;
      if (wout) wout[j] = wt[j];
    }
    return;
  }
  const int lo = a.sink, hi = len - a.recent;              // the candidates
  int k = a.budget - a.sink - a.recent;                    // how many of them stay; 0 <= k < hi - lo
  uint32_t prefix = 0, mask = 0;                           // digits of the k-th largest key found so far
  if (k > 0) {
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0);
      const uint32_t dmask = pass == 2 ? 1023u : 2047u;
      for (int i = tid; i < kEvBins; i += kEvThreads) hist[i] = 0;
      __syncthreads();
      for (int j = lo + tid; j < hi; j += kEvThreads) {
        const uint32_t u = weight_key(wt[j]);
        if ((u & mask) == prefix) atomicAdd(&hist[(u >> shift) & dmask], 1u);
      }
      __syncthreads();
      // the digit whose bin holds the k-th largest: thread t sums the 4 bins from the top down
      constexpr int PER = kEvBins / kEvThreads;
      uint32_t mine = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) mine += hist[kEvBins - 1 - (tid * PER + i)];
      uint32_t incl = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      if (lane == 31) warp_sum_s[warp] = incl;
      __syncthreads();
      uint32_t before = 0;
      for (int w = 0; w < warp; ++w) before += warp_sum_s[w];
      uint32_t above = before + incl - mine;               // keys in higher bins
      if (above < uint32_t(k) && above + mine >= uint32_t(k)) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int bin = kEvBins - 1 - (tid * PER + i);
          const uint32_t n = hist[bin];
          if (above < uint32_t(k) && above + n >= uint32_t(k)) { found[0] = uint32_t(bin); found[1] = above; break; }
          above += n;
        }
      }
      __syncthreads();
      prefix |= found[0] << shift;
      mask |= dmask << shift;
      k -= int(found[1]);
      __syncthreads();
    }
  }
  // keys above `prefix` stay, and the first k of those equal to it (k == 0 from the start: none of either)
  const bool any = a.budget - a.sink - a.recent > 0;
  uint32_t base = 0;                                       // kept so far
  uint32_t base_eq = 0;                                    // equal to the k-th largest so far
#pragma unroll 1
  for (int j0 = 0; j0 < len; j0 += kEvThreads) {
    const int j = j0 + tid;
    const bool in = j < len;
    const bool forced = in && (j < lo || j >= hi);
    const float x = in ? wt[j] : 0.f;
    const uint32_t u = weight_key(x);
    const bool eq = in && !forced && any && u == prefix;
    const bool gt = in && !forced && any && u > prefix;
    // rank among the equal ones first, then the position among the kept
    const uint32_t beq = __ballot_sync(0xffffffffu, eq), lt = (1u << lane) - 1;
    if (lane == 0) warp_sum_s[warp] = __popc(beq);
    __syncthreads();
    uint32_t eq_before = base_eq, eq_all = 0;
    for (int w = 0; w < kEvThreads / 32; ++w) {
      if (w < warp) eq_before += warp_sum_s[w];
      eq_all += warp_sum_s[w];
    }
    __syncthreads();
    const bool keep = forced || gt || (eq && eq_before + __popc(beq & lt) < uint32_t(k));
    const uint32_t bk = __ballot_sync(0xffffffffu, keep);
    if (lane == 0) warp_sum_s[warp] = __popc(bk);
    __syncthreads();
    uint32_t at = base, all = 0;
    for (int w = 0; w < kEvThreads / 32; ++w) {
      if (w < warp) at += warp_sum_s[w];
      all += warp_sum_s[w];
    }
    __syncthreads();
    if (keep) {
      at += __popc(bk & lt);
      kept[at] = j;
      if (wout) wout[at] = x;
    }
    base += all;
    base_eq += eq_all;
  }
}

constexpr int kGaThreads = 128;
template <int FMT, int DH>
__global__ void __launch_bounds__(kGaThreads)
cache8_gather_kernel(const Cache8EvictArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int CH = DH / 16;                              // 16-code pieces of a row
  constexpr int PER = 64 * CH / kGaThreads;
  __shared__ long long src_s[64];                          // (page, head) index and row of every source row
  __shared__ float scale_s[64];
  __shared__ uint32_t red[kGaThreads / 32];
  const Cache8Args& c = a.c;
  const int b = blockIdx.x / a.to_pages_per_seq, blk = blockIdx.x - b * a.to_pages_per_seq;
  const int kvh = blockIdx.y;
  const bool is_v = blockIdx.z != 0;
  const int rows = min(a.new_lens[b] - blk * 64, 64);
  if (rows <= 0) return;
  const int to_page = a.to_table[size_t(b) * a.to_pages_per_seq + blk];
  if (to_page < 0 || to_page >= c.num_pages) {
    if (threadIdx.x == 0) atomicExch(c.status, kStatusBounds);
    return;
  }
  const uint8_t* pages = is_v ? c.v_pages : c.k_pages;
  const float* scales = is_v ? c.v_scales : c.k_scales;
  if (threadIdx.x < 64) {
    long long src = -1;
    float s = 0.f;
    if (int(threadIdx.x) < rows) {
      const int pos = a.kept[(size_t(b) * c.n_kv + kvh) * a.budget + blk * 64 + threadIdx.x];
      const int page = c.block_table[size_t(b) * c.max_pages_per_seq + (pos >> 6)];
      if (page < 0 || page >= c.num_pages) {
        atomicExch(c.status, kStatusBounds);
      } else {
        const long long ph = (long long)page * c.n_kv + kvh;
        src = ph * 64 + (pos & 63);
        s = scales[ph];
      }
    }
    src_s[threadIdx.x] = src;
    scale_s[threadIdx.x] = s;
  }
  __syncthreads();
  uint4 x[PER];
  uint32_t amax = 0;                                       // fp32 bits of the largest magnitude; a NaN scale wins
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int p = i * kGaThreads + threadIdx.x, row = p / CH, ch = p - row * CH;
    const long long src = src_s[row];
    x[i] = make_uint4(0, 0, 0, 0);
    if (src >= 0) x[i] = *reinterpret_cast<const uint4*>(pages + src * DH + ch * 16);
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const float s = scale_s[(i * kGaThreads + threadIdx.x) / CH];
    const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float v[4];
      c8_decode4<FMT>(w[q], v);
#pragma unroll
      for (int e = 0; e < 4; ++e) amax = max(amax, __float_as_uint(v[e] * s) & 0x7fffffffu);
    }
  }
  amax = __reduce_max_sync(0xffffffffu, amax);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = amax;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kGaThreads / 32; ++w) amax = max(amax, red[w]);
  const int e = c8_exponent<FMT>(amax >> 16);              // (values held in 8 bits have at most 8 significant ones)
  const bool nan = e == 0x7fffffff;
  const size_t to = size_t(to_page) * c.n_kv + kvh;
  uint4* dst = reinterpret_cast<uint4*>((is_v ? c.v_pages : c.k_pages) + to * 64 * DH);
  const float inv = nan ? 0.f : c8_pow2(-e);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int p = i * kGaThreads + threadIdx.x, row = p / CH;
    if (row >= rows) continue;                             // rows behind the last kept one stay as they were
    const float f = scale_s[row] * inv;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (!nan) v = make_uint4(c8_rescale4<FMT>(x[i].x, f), c8_rescale4<FMT>(x[i].y, f), c8_rescale4<FMT>(x[i].z, f), c8_rescale4<FMT>(x[i].w, f));
    dst[p] = v;
  }
  if (threadIdx.x == 0) (is_v ? c.v_scales : c.k_scales)[to] = nan ? __int_as_float(0x7fc00000) : c8_pow2(e);
}

template <int FMT>
static void launch_evict_t(const Cache8EvictArgs& a, cudaStream_t st) {
  const Cache8Args& c = a.c;
  launch_pdl(cache8_select_kernel, dim3(c.n_kv, c.n_seqs), dim3(kEvThreads), 0, st, a);
  const dim3 grid(unsigned(c.n_seqs) * a.to_pages_per_seq, c.n_kv, 2);
  if (c.dh == 64) launch_pdl(cache8_gather_kernel<FMT, 64>, grid, dim3(kGaThreads), 0, st, a);
  else if (c.dh == 96) launch_pdl(cache8_gather_kernel<FMT, 96>, grid, dim3(kGaThreads), 0, st, a);
  else launch_pdl(cache8_gather_kernel<FMT, 128>, grid, dim3(kGaThreads), 0, st, a);
}

void launch_cache8_evict(int fmt, const Cache8EvictArgs& a, cudaStream_t st) {
  if (a.c.n_seqs <= 0) return;
  if (fmt == kC8E4M3) launch_evict_t<kC8E4M3>(a, st);
  else launch_evict_t<kC8Int8>(a, st);
}

}  // namespace foe
