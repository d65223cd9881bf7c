// Logits to tokens: penalties for repeated tokens, bias, temperature and grammar mask over
// the vocabulary, the best token and the log of the sum of exponentials, in one pass.
//
// Per row and token v, seen c times in the row's list:
//   c > 0:  z = (z > 0 ? z / repetition : z repetition) - presence - frequency c
//   z = (z + bias) (1 / temperature),  -infinity where the mask says no
// each operation rounded to fp32 as it stands here.  Bound by bytes: logits in, results
// out.  A row is a cluster's: every CTA counts the list's tokens of its share of the
// vocabulary in shared memory, walks its logits once with a running maximum and sum, and
// the first CTA joins what they found in the order of the tokens.  Lanes take neighbouring
// tokens, so no row needs an alignment, and a word of the mask is a warp's (one lane loads
// it for all).  The next kItems logits of a thread are on their way while these are worked
// on, and go past the caches as what is not read again (22.3 -> 20.4 us at the size below).
//
// [64, 128001] fp32 with 3000 tokens seen a row, a bias and masks, all of it from memory:
// 20.4 us, 3.3 TB/s (a plain copy of the size 11.7); 18.0 without lists, of which a CTA's
// count is 2 us before its walk; 14 where the L2 has the logits.  In four CTAs an SM there
// are two batches in flight at most: the rest is the walk's instructions, 25 a token.
// Tried: the share into the L2 at first (24.1), 4 or 16 logits at once (23.6, 29.5), 512
// threads (27.7), three CTAs an SM with more registers (29.9), no exponentials (20.1).
#include <cfloat>

#include "sparoa_kernels.h"

namespace sparoa {

namespace {

constexpr int kThreads = 256;
constexpr int kItems = 8;            // tokens of a thread at once
constexpr int kStep = kItems * kThreads;
constexpr int kAhead = 16;           // tokens of the list that a thread loads at once
constexpr int kMaxChunk = 80 << 10;  // tokens counted at once, two bytes each

// The best token and the sum of exp(z - clamp(best)) of some tokens.
struct Found {
  float top;
  int token;  // INT_MAX: none above -infinity
  float sum;
};
// what sums go by: infinities would give differences that are no numbers
__device__ __forceinline__ float ref_of(float top) { return fminf(fmaxf(top, -FLT_MAX), FLT_MAX); }
constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float weight(float z) {
  float w;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(w) : "f"(z * kLog2e));
  return w;
}
__device__ __forceinline__ Found join(const Found& a, const Found& b) {
  Found f;
  const bool second = b.top > a.top || (b.top == a.top && b.token < a.token);
  f.top = second ? b.top : a.top;
  f.token = second ? b.token : a.token;
  const float r = ref_of(f.top);
  f.sum = a.sum * weight(ref_of(a.top) - r) + b.sum * weight(ref_of(b.top) - r);
  return f;
}
__device__ __forceinline__ Found from_lane(const Found& f, int d) {
  Found o;
  o.top = __shfl_xor_sync(0xffffffffu, f.top, d);
  o.token = __shfl_xor_sync(0xffffffffu, f.token, d);
  o.sum = __shfl_xor_sync(0xffffffffu, f.sum, d);
  return o;
}

__device__ __forceinline__ float load_logit(const float* p) { return __ldcs(p); }
__device__ __forceinline__ float load_logit(const __nv_bfloat16* p) { return __bfloat162float(__ldcs(p)); }

enum Parts : int { kSeen = 1, kBiased = 2, kMasked = 4, kStored = 8 };  // what a kernel does besides

// A row's rules, and where a thread's tokens of the CTA's share are.
template <typename XT>
struct Share {
  const XT* x;
  const float* bias;
  const uint32_t* allowed;
  float* y;
  const unsigned* count;  // two counts in each, or one (wide)
  // inv_rep = 1 / rep rounded: a quotient q = z inv_rep, corrected by the rest z - q rep times
  // inv_rep, is the rounded z / rep (Markstein, 1990)
  float rep, inv_rep, presence, frequency, inv;
  int lo, len;
  bool wide;
};

// kItems tokens of a thread, kThreads apart, from token v0 of the share on.  FULL: all are there.
template <int PARTS, bool FULL, typename XT>
struct Batch {
  float b[kItems];
  uint32_t open;  // lane u: the word of token u

  static __device__ __forceinline__ bool there(const Share<XT>& s, int v) { return FULL || v + (int)threadIdx.x < s.len; }
  static __device__ __forceinline__ void fetch(const Share<XT>& s, int v0, float (&z)[kItems]) {
#pragma unroll
    for (int u = 0; u < kItems; ++u) {
      const int v = v0 + u * kThreads;
      z[u] = there(s, v) ? load_logit(s.x + v) : -INFINITY;
    }
  }
  __device__ __forceinline__ void rules(const Share<XT>& s, int v0) {
    const int lane = threadIdx.x & 31, v1 = v0 + lane * kThreads;
    if ((PARTS & kMasked) != 0) open = lane < kItems && (FULL || v1 + (int)(threadIdx.x & ~31u) < s.len) ? s.allowed[v1 >> 5] : 0u;
#pragma unroll
    for (int u = 0; u < kItems; ++u) {
      const int v = v0 + u * kThreads;
      if ((PARTS & kBiased) != 0) b[u] = there(s, v) ? s.bias[v] : 0.f;
    }
  }
  __device__ __forceinline__ void penalise(const Share<XT>& s, int v0, float (&z)[kItems]) {
    unsigned c[kItems], any = 0u;
#pragma unroll
    for (int u = 0; u < kItems; ++u) {
      const int v = v0 + u * kThreads;
      c[u] = !there(s, v) ? 0u : s.wide ? s.count[v + threadIdx.x] : reinterpret_cast<const uint16_t*>(s.count)[v + threadIdx.x];
      any |= c[u];
    }
    if (!any) return;
    // without a branch for each (a division's own cost the share with most of the list's tokens
    // as much again as its bytes)
#pragma unroll
    for (int u = 0; u < kItems; ++u) {
      const float q = __fmul_rn(z[u], s.inv_rep), rest = fmaf(-q, s.rep, z[u]);
      const float ratio = fabsf(q) < INFINITY ? fmaf(rest, s.inv_rep, q) : q;
      const float less = __fsub_rn(__fsub_rn(z[u] > 0.f ? ratio : __fmul_rn(z[u], s.rep), s.presence), __fmul_rn(s.frequency, (float)c[u]));
      z[u] = c[u] ? less : z[u];
    }
  }
  __device__ __forceinline__ void finish(const Share<XT>& s, int v0, float (&z)[kItems], Found& f) {
    const uint32_t bit = 1u << (threadIdx.x & 31);
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < kItems; u += 2) {
      f2_t p = f2(z[u], z[u + 1]);
      if ((PARTS & kBiased) != 0) p = fadd2(p, f2(b[u], b[u + 1]));
      f2_split(fmul2(p, f2(s.inv, s.inv)), z[u], z[u + 1]);
    }
#pragma unroll
    for (int u = 0; u < kItems; ++u) {
      const int v = v0 + u * kThreads;
      if ((PARTS & kMasked) != 0) z[u] = __shfl_sync(0xffffffffu, open, u) & bit ? z[u] : -INFINITY;
      if ((PARTS & kStored) != 0 && there(s, v)) s.y[v] = z[u];
      top = fmaxf(top, z[u]);  // (a number that is none is never the largest)
    }
    if (top > f.top) {
      const float ref = ref_of(top);
      f.sum *= weight(ref_of(f.top) - ref);
      f.top = top;
#pragma unroll
      for (int u = kItems - 1; u >= 0; --u)
        if (z[u] == top) f.token = s.lo + v0 + u * kThreads + (int)threadIdx.x;
    }
    const float ref = -ref_of(f.top);
    f2_t sum = f2(f.sum, 0.f);
#pragma unroll
    for (int u = 0; u < kItems; u += 2) {
      float x, y;
      f2_split(fmul2(fadd2(f2(z[u], z[u + 1]), f2(ref, ref)), f2(kLog2e, kLog2e)), x, y);
      asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(x));
      asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(y));
      sum = fadd2(sum, f2(x, y));
    }
    float x, y;
    f2_split(sum, x, y);
    f.sum = x + y;
  }
};

// zero counts of `chunk` tokens, or of half as many that have 32 bits
__device__ __forceinline__ void no_counts(unsigned* count, int chunk) {
  for (int i = threadIdx.x; i < chunk / 8; i += kThreads) reinterpret_cast<uint4*>(count)[i] = make_uint4(0u, 0u, 0u, 0u);
}

// Counts have 16 bits, which a list below 2^16 tokens cannot pass; the vocabulary of a row with a
// longer one is walked in shares of half the size, with 32 bits.
template <typename XT, int PARTS>
__global__ void __launch_bounds__(kThreads, 4) logits_kernel(const __grid_constant__ LogitArgs a) {
  extern __shared__ __align__(16) unsigned s_count[];
  __shared__ Found s_found[kThreads / 32], s_cta;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rank = (int)(blockIdx.x % a.split);
  const int64_t r = blockIdx.x / a.split;
  Share<XT> s;
  s.rep = s.inv_rep = s.inv = 1.f;
  s.presence = s.frequency = 0.f;
  s.count = s_count;
  if constexpr ((PARTS & kSeen) != 0) no_counts(s_count, a.chunk);
  pdl_wait();
  pdl_trigger();
  if (a.penalties) {
    const float* p = a.penalties + r * 4;
    s.rep = p[0];
    s.inv_rep = __frcp_rn(p[0]);
    s.presence = p[1];
    s.frequency = p[2];
    s.inv = __frcp_rn(p[3]);
  }
  int64_t s0 = 0, s1 = 0;
  if constexpr ((PARTS & kSeen) != 0) {
    s0 = a.seen_start[r];
    s1 = a.seen_start[r + 1];
    if (s0 < 0 || s1 < s0 || s1 > a.n_seen) {
      if (threadIdx.x == 0 && rank == 0) atomicOr(a.err, kErrBadIndex);
      s0 = s1 = 0;
    }
  }
  const bool seen = (PARTS & kSeen) && s1 > s0;
  s.wide = seen && s1 - s0 > 65535;
  const int chunk = s.wide ? a.chunk / 2 : a.chunk;
  Found f{-INFINITY, 0x7FFFFFFF, 0.f};
  for (int64_t lo = (int64_t)rank * chunk; lo < a.V; lo += (int64_t)a.split * chunk) {
    s.lo = (int)lo;
    s.len = min(chunk, a.V - s.lo);
    const int64_t at = lo + threadIdx.x;
    s.x = static_cast<const XT*>(a.x) + r * a.ld_x + at;
    if ((PARTS & kBiased) != 0) s.bias = a.bias + r * a.ld_bias + at;
    if ((PARTS & kMasked) != 0) s.allowed = a.allowed + r * a.ld_allowed + (at >> 5);
    if ((PARTS & kStored) != 0) s.y = a.y + r * a.ld_y + at;
    float z[kItems];
    Batch<PARTS, false, XT>::fetch(s, 0, z);  // on its way while the tokens are counted
    if (seen) {
      if (lo >= (int64_t)a.split * chunk) {  // (the first share's counts are zero already)
        __syncthreads();                     // (the counts before were read)
        no_counts(s_count, a.chunk);
      }
      __syncthreads();
      // (kAhead loads of a thread are on their way at once; what is no token counts nowhere)
      for (int64_t i0 = s0 + threadIdx.x; i0 < s1; i0 += kAhead * kThreads) {
        unsigned t[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) t[k] = i0 + k * kThreads < s1 ? (unsigned)a.seen[i0 + k * kThreads] - (unsigned)s.lo : 0xFFFFFFFFu;
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if (t[k] < (unsigned)s.len) atomicAdd(s_count + (s.wide ? t[k] : t[k] >> 1), !s.wide && (t[k] & 1u) ? 0x10000u : 1u);
      }
      __syncthreads();
    }
    int v0 = 0;
    for (; v0 + kStep <= s.len; v0 += kStep) {
      Batch<PARTS, true, XT> batch;
      batch.rules(s, v0);
      float next[kItems];
      if (v0 + 2 * kStep <= s.len)
        Batch<PARTS, true, XT>::fetch(s, v0 + kStep, next);
      else
        Batch<PARTS, false, XT>::fetch(s, v0 + kStep, next);
      if (seen) batch.penalise(s, v0, z);
      batch.finish(s, v0, z, f);
#pragma unroll
      for (int u = 0; u < kItems; ++u) z[u] = next[u];
    }
    if (v0 < s.len) {
      Batch<PARTS, false, XT> batch;
      batch.rules(s, v0);
      if (seen) batch.penalise(s, v0, z);
      batch.finish(s, v0, z, f);
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) f = join(f, from_lane(f, d));
  if (lane == 0) s_found[warp] = f;
  __syncthreads();
  if (warp == 0) {
    f = lane < kThreads / 32 ? s_found[lane] : Found{-INFINITY, 0x7FFFFFFF, 0.f};
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) f = join(f, from_lane(f, d));
    if (lane == 0) s_cta = f;
  }
  cluster_arrive();
  cluster_wait();
  if (rank == 0 && warp == 0) {
    f = Found{-INFINITY, 0x7FFFFFFF, 0.f};
    if (lane < a.split) {
      const uint32_t from = cluster_map(smem_u32(&s_cta), (uint32_t)lane);
      f.top = __uint_as_float(ld_cluster_u32(from));
      f.token = (int)ld_cluster_u32(from + 4);
      f.sum = __uint_as_float(ld_cluster_u32(from + 8));
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) f = join(f, from_lane(f, d));
    if (lane == 0) {
      if (a.best) a.best[r] = f.top > -INFINITY ? f.token : -1;
      if (a.lse) a.lse[r] = f.sum == 0.f ? -INFINITY : ref_of(f.top) + logf(f.sum);  // (a sum of NaN stays one)
    }
  }
  cluster_arrive();  // what the CTAs found is read until here
  cluster_wait();
}

template <typename XT, int PARTS>
cudaError_t launch_logits_t(LogitArgs a, cudaStream_t s) {
  constexpr bool SEEN = (PARTS & kSeen) != 0;
  // CTAs of a row until there are four an SM, each with two rounds of tokens at least, and until
  // four CTAs' counts fit an SM
  const int64_t want = 4ll * device_sm_count();
  a.split = 1;
  while (a.split < 8 && ((a.R * a.split * 2 <= want && a.V > a.split * 2 * kStep) || (SEEN && a.V > a.split * (24 << 10))))
    a.split *= 2;
  a.chunk = ((a.V + a.split - 1) / a.split + 63) / 64 * 64;
  if (SEEN && a.chunk > kMaxChunk) a.chunk = kMaxChunk;
  const size_t smem = SEEN ? (size_t)a.chunk * 2 : 0;
  const cudaError_t e = smem_optin(reinterpret_cast<const void*>(logits_kernel<XT, PARTS>), smem);
  if (e != cudaSuccess) return e;
  return launch_cluster_kernel(logits_kernel<XT, PARTS>, dim3((unsigned)(a.R * a.split)), dim3(kThreads), (unsigned)a.split, smem, s, a);
}

template <typename XT, int PARTS = 0>
cudaError_t launch_by_parts(int parts, const LogitArgs& a, cudaStream_t s) {
  if (parts == PARTS) return launch_logits_t<XT, PARTS>(a, s);
  if constexpr (PARTS < 15) return launch_by_parts<XT, PARTS + 1>(parts, a, s);
  return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_logits(const LogitArgs& a, cudaStream_t s) {
  if (a.R <= 0) return cudaSuccess;
  const int parts = (a.seen_start ? kSeen : 0) | (a.bias ? kBiased : 0) | (a.allowed ? kMasked : 0) | (a.y ? kStored : 0);
  return a.x_bf16 ? launch_by_parts<__nv_bfloat16>(parts, a, s) : launch_by_parts<float>(parts, a, s);
}

}  // namespace sparoa
