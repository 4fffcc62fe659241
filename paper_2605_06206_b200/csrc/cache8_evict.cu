// Eviction from the 8-bit cache by accumulated attention weight: every (sequence, KV head) keeps its first `sink`
// tokens, its last `recent` ones and the heaviest of the rest, budget tokens in all, in their order.
//
// Two launches.  The first chooses: one block per (sequence, KV head) finds the k-th largest weight by a radix search
// over the weights as ordered integers (three passes of 11, 11 and 10 bits over keys in shared memory), then writes the
// kept positions, each thread those of a run whose place a prefix sum gives; ties go to the lower position.  The second copies: one block per (destination page, KV
// head, K or V) gathers its 64 rows, takes their largest magnitude and encodes them at a scale made for them.  Source and
// destination pages are disjoint, so all destination pages are built at once, and a source page that several sequences
// share (a common prompt prefix) is left as it is for the others.
// Bound: memory (4 bytes per weight; 2 bytes read and 2 written per kept K/V element pair).  Measured (B200): 32 sequences of
// 4k to 9k tokens, 8 KV heads of 128, cut to 2048: 69 us, 19 for the choice and 50 for the copy (5.3 TB/s); one sequence of
// 1500 tokens 9.6 us.  Reading the weights again in every pass and scanning tile by tile took 34 us for the choice, decoding
// every code to find the largest 73 us for the copy.
#include "cache8.cuh"
#include "cache8.h"

namespace foe {

constexpr int kEvThreads = 1024;
constexpr int kEvBins = 2048;
constexpr int kEvKeysMax = 48 * 1024;            // keys that fit the shared memory of one block, beside the bins

// order of the weights as unsigned integers: larger weight, larger key; -0 = +0; a NaN below everything
__device__ __forceinline__ uint32_t weight_key(float x) {
  uint32_t u = __float_as_uint(x);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;
  if (u == 0x80000000u) u = 0u;
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// the weight a key stands for (a NaN or -0 comes back as some NaN or +0)
__device__ __forceinline__ float key_weight(uint32_t u) {
  return __uint_as_float(u == 0u ? 0x7fc00000u : ((u & 0x80000000u) ? (u & 0x7fffffffu) : ~u));
}

// sum of v over the threads before this one (every warp adds up the other warps' sums by itself)
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* warp_sums) {
  static_assert(kEvThreads == 1024, "one warp sum per lane");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  auto scan = [lane](uint32_t x) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t u = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += u;
    }
    return x;
  };
  const uint32_t incl = scan(v);
  __syncthreads();                                         // (the sums of an earlier scan have been read)
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  const uint32_t mine = warp_sums[lane];
  const uint32_t before = scan(mine) - mine;
  return __shfl_sync(0xffffffffu, before, warp) + incl - v;
}

// STAGED: the row's keys are read once into shared memory (rows of up to kEvKeysMax tokens); otherwise every pass reads the
// weights again.
template <bool STAGED>
__global__ void __launch_bounds__(kEvThreads)
cache8_select_kernel(const Cache8EvictArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  extern __shared__ uint32_t keys[];
  __shared__ uint32_t hist[kEvBins];
  __shared__ uint32_t warp_sums[kEvThreads / 32];
  __shared__ uint32_t found[2];
  const Cache8Args& c = a.c;
  const int b = blockIdx.y, kvh = blockIdx.x, tid = threadIdx.x, lane = tid & 31;
  int len = c.context_lens[b];
  if (len < 0 || len > c.max_len) {
    if (tid == 0) atomicExch(c.status, kStatusBounds);
    len = 0;
  }
  const size_t row = size_t(b) * c.n_kv + kvh;
  const float* wt = a.weights + row * a.weights_stride;
  int* kept = a.kept + row * a.budget;
  float* wout = a.weights_out ? a.weights_out + row * a.weights_out_stride : nullptr;
  if (kvh == 0 && tid == 0) a.new_lens[b] = min(len, a.budget);
  if (len <= a.budget) {
    for (int j = tid; j < len; j += kEvThreads) {
      kept[j] = j;
      if (wout) wout[j] = wt[j];
    }
    return;
  }
  const int lo = a.sink, hi = len - a.recent;              // the candidates
  const int want = a.budget - a.sink - a.recent;           // how many of them stay; 0 <= want < hi - lo
  auto key = [&](int j) { return STAGED ? keys[j] : weight_key(wt[j]); };
  if (STAGED) {
    constexpr int AHEAD = 8;                               // loads in flight
    for (int j0 = tid; j0 < len; j0 += AHEAD * kEvThreads) {
      float x[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) x[i] = j0 + i * kEvThreads < len ? __ldg(wt + j0 + i * kEvThreads) : 0.f;
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        if (j0 + i * kEvThreads < len) keys[j0 + i * kEvThreads] = weight_key(x[i]);
    }
  }
  uint32_t prefix = 0, mask = 0;                           // digits of the want-th largest key found so far
  int k = want;                                            // how many keys with these digits stay
#pragma unroll 1
  for (int pass = 0; pass < 3 && want > 0; ++pass) {
    const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0);
    const uint32_t dmask = pass == 2 ? 1023u : 2047u;
    for (int i = tid; i < kEvBins; i += kEvThreads) hist[i] = 0;
    __syncthreads();
    for (int j = lo + tid; j < hi; j += kEvThreads) {
      const uint32_t u = key(j);
      // (adding up a warp's equal bins first, by match or by ballot, measured slower than the plain additions)
      if ((u & mask) == prefix) atomicAdd(&hist[(u >> shift) & dmask], 1u);
    }
    __syncthreads();
    // the digit whose bin holds the k-th largest: thread t sums its bins from the top down
    constexpr int PER = kEvBins / kEvThreads;
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) mine += hist[kEvBins - 1 - (tid * PER + i)];
    uint32_t above = block_scan(mine, warp_sums);     // keys in higher bins
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
  }
  __syncthreads();                                         // (with want == 0: the staged keys are there)
  // Keys above `prefix` stay, and the first k of those equal to it.  A thread takes a run of consecutive positions, its
  // length odd so that the threads of a warp read different banks; one scan gives every run its place.
  const int run = ((len + kEvThreads - 1) / kEvThreads) | 1;
  const int j0 = min(tid * run, len), j1 = min(j0 + run, len);
  if constexpr (STAGED) {
    static_assert(kEvKeysMax / kEvThreads < 64, "a run's positions are the bits of one word");
    unsigned long long keep = 0, eq = 0;                   // kept whatever the ties do; equal to the last one kept
    for (int j = j0; j < j1; ++j) {
      const uint32_t u = keys[j];
      const bool forced = j < lo || j >= hi;
      keep |= (unsigned long long)(forced || (want > 0 && u > prefix)) << (j - j0);
      eq |= (unsigned long long)(!forced && want > 0 && u == prefix) << (j - j0);
    }
    uint32_t at = block_scan(__popcll(keep), warp_sums);
    const uint32_t eq_before = block_scan(__popcll(eq), warp_sums);
    at += min(eq_before, uint32_t(k));
    for (uint32_t n = eq_before; eq && n < uint32_t(k); ++n, eq &= eq - 1) keep |= eq & -eq;      // the lowest ties that still fit
    for (; keep; keep &= keep - 1, ++at) {
      const int j = j0 + __ffsll(keep) - 1;
      kept[at] = j;
      if (wout) wout[at] = key_weight(keys[j]);
    }
    return;
  }
  uint32_t n_keep = 0, n_eq = 0;
  for (int j = j0; j < j1; ++j) {
    if (j < lo || j >= hi) { ++n_keep; continue; }
    const uint32_t u = key(j);
    n_keep += want > 0 && u > prefix;
    n_eq += want > 0 && u == prefix;
  }
  uint32_t at = block_scan(n_keep, warp_sums);
  uint32_t eq = block_scan(n_eq, warp_sums);
  at += min(eq, uint32_t(k));
  for (int j = j0; j < j1; ++j) {
    bool keep = j < lo || j >= hi;
    if (!keep && want > 0) {
      const uint32_t u = key(j);
      keep = u > prefix;
      if (u == prefix) keep = eq++ < uint32_t(k);
    }
    if (keep) {
      kept[at] = j;
      if (wout) wout[at] = wt[j];
      ++at;
    }
  }
}

// Largest magnitude of 16 codes, as a number.  e4m3 magnitudes are ordered like their codes without the sign; int8 codes
// are looked at with an offset of 128, whose largest and smallest give the magnitude.
template <int FMT>
__device__ __forceinline__ float largest_of(uint4 x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t hi = 0, lo = 0xffffffffu;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (FMT == kC8E4M3) {
      hi = __vmaxu2(hi, __vmaxu2(w[i] & 0x007f007fu, (w[i] >> 8) & 0x007f007fu));
    } else {
      const uint32_t u = w[i] ^ 0x80808080u, e = u & 0x00ff00ffu, o = (u >> 8) & 0x00ff00ffu;
      hi = __vmaxu2(hi, __vmaxu2(e, o));
      lo = __vminu2(lo, __vminu2(e, o));
    }
  }
  const int m = int(max(hi & 0xffffu, hi >> 16));
  if constexpr (FMT == kC8E4M3) {
    float v[4];
    c8_decode4<FMT>(uint32_t(m), v);
    return v[0];
  } else {
    return float(max(m - 128, 128 - int(min(lo & 0xffffu, lo >> 16))));
  }
}

constexpr int kGaThreads = 128;
template <int FMT, int DH>
__global__ void __launch_bounds__(kGaThreads, 12)
cache8_gather_kernel(const Cache8EvictArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int CH = DH / 16;                              // 16-code pieces of a row
  constexpr int PER = 64 * CH / kGaThreads;
  __shared__ int src_s[64];                                // row of codes in the pool (fewer than 2^31), or -1
  __shared__ float scale_s[64];
  __shared__ uint32_t red[kGaThreads / 32];
  const Cache8Args& c = a.c;
  const int blocks = (a.budget + 63) / 64;
  const int b = blockIdx.x / blocks, blk = blockIdx.x - b * blocks;
  const int kvh = blockIdx.y;
  const bool is_v = blockIdx.z != 0;
  // (the position is loaded beside the length that says whether it is one)
  const int at = blk * 64 + threadIdx.x;
  int pos = 0;
  if (threadIdx.x < 64 && at < a.budget) pos = a.kept[(size_t(b) * c.n_kv + kvh) * a.budget + at];
  const int rows = min(a.new_lens[b] - blk * 64, 64);
  if (rows <= 0) return;
  const int to_page = a.to_table[size_t(b) * a.to_pages_per_seq + blk];
  if (to_page < 0 || to_page >= c.num_pages) {
    if (threadIdx.x == 0) atomicExch(c.status, kStatusBounds);
    return;
  }
  const uint8_t* pages = is_v ? c.v_pages : c.k_pages;
  if (threadIdx.x < 64) {
    int src = -1;
    float s = 0.f;
    if (int(threadIdx.x) < rows) {
      const int page = c.block_table[size_t(b) * c.max_pages_per_seq + (pos >> 6)];
      if (page < 0 || page >= c.num_pages) {
        atomicExch(c.status, kStatusBounds);
      } else {
        const int ph = page * c.n_kv + kvh;
        src = ph * 64 + (pos & 63);
        s = (is_v ? c.v_scales : c.k_scales)[ph];
      }
    }
    src_s[threadIdx.x] = src;
    scale_s[threadIdx.x] = s;
  }
  __syncthreads();
  uint4 x[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int p = i * kGaThreads + threadIdx.x, row = p / CH, ch = p - row * CH;
    const int src = src_s[row];
    x[i] = make_uint4(0, 0, 0, 0);
    if (src >= 0) x[i] = *reinterpret_cast<const uint4*>(pages + size_t(src) * DH + ch * 16);
  }
  uint32_t amax = 0;                                       // fp32 bits of the largest magnitude; a NaN scale wins
#pragma unroll
  for (int i = 0; i < PER; ++i)
    amax = max(amax, __float_as_uint(largest_of<FMT>(x[i]) * scale_s[(i * kGaThreads + threadIdx.x) / CH]) & 0x7fffffffu);
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
    uint4 v = x[i];
    if (nan) v = make_uint4(0, 0, 0, 0);
    else if (f != 1.f) v = make_uint4(c8_rescale4<FMT>(v.x, f), c8_rescale4<FMT>(v.y, f), c8_rescale4<FMT>(v.z, f), c8_rescale4<FMT>(v.w, f));
    dst[p] = v;
  }
  if (threadIdx.x == 0) (is_v ? c.v_scales : c.k_scales)[to] = nan ? __int_as_float(0x7fc00000) : c8_pow2(e);
}

template <int FMT>
static void launch_evict_t(const Cache8EvictArgs& a, cudaStream_t st) {
  const Cache8Args& c = a.c;
  if (c.max_len <= kEvKeysMax) launch_pdl(cache8_select_kernel<true>, dim3(c.n_kv, c.n_seqs), dim3(kEvThreads), size_t(c.max_len) * 4, st, a);
  else launch_pdl(cache8_select_kernel<false>, dim3(c.n_kv, c.n_seqs), dim3(kEvThreads), 0, st, a);
  const dim3 grid(unsigned(c.n_seqs) * ((a.budget + 63) / 64), c.n_kv, 2);
  if (c.dh == 64) launch_pdl(cache8_gather_kernel<FMT, 64>, grid, dim3(kGaThreads), 0, st, a);
  else if (c.dh == 96) launch_pdl(cache8_gather_kernel<FMT, 96>, grid, dim3(kGaThreads), 0, st, a);
  else launch_pdl(cache8_gather_kernel<FMT, 128>, grid, dim3(kGaThreads), 0, st, a);
}

cudaError_t cache8_evict_configure() {
  return cudaFuncSetAttribute(cache8_select_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kEvKeysMax * 4);
}

void launch_cache8_evict(int fmt, const Cache8EvictArgs& a, cudaStream_t st) {
  if (a.c.n_seqs <= 0) return;
  if (fmt == kC8E4M3) launch_evict_t<kC8E4M3>(a, st);
  else launch_evict_t<kC8Int8>(a, st);
}

}  // namespace foe
