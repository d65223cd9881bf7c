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
// tokens, so no row needs an alignment, and a word of the mask is a warp's.
#include <cfloat>

#include "sparoa_kernels.h"

namespace sparoa {

namespace {

constexpr int kThreads = 512;
constexpr int kItems = 8;               // tokens of a thread at once
constexpr int kMaxChunk = 48 * 1024;    // tokens counted at once, 4 bytes each

// The best token and the sum of exp(z - clamp(best)) of some tokens.
struct Found {
  float top;
  int token;  // INT_MAX: none above -infinity
  float sum;
};
// what sums go by: infinities would give differences that are no numbers
__device__ __forceinline__ float ref_of(float top) { return fminf(fmaxf(top, -FLT_MAX), FLT_MAX); }
__device__ __forceinline__ float weight(float z) { return exp2f(z * 1.4426950408889634f); }
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

__device__ __forceinline__ float load_logit(const float* p) { return *p; }
__device__ __forceinline__ float load_logit(const __nv_bfloat16* p) { return __bfloat162float(*p); }

template <typename XT, bool SEEN>
__global__ void __launch_bounds__(kThreads) logits_kernel(const __grid_constant__ LogitArgs a) {
  extern __shared__ __align__(16) unsigned s_count[];  // [chunk]
  __shared__ Found s_found[kThreads / 32], s_cta;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rank = (int)(blockIdx.x % a.split);
  const int64_t r = blockIdx.x / a.split;
  pdl_wait();
  pdl_trigger();
  float rep = 1.f, presence = 0.f, frequency = 0.f, inv = 1.f;
  if (a.penalties) {
    const float* p = a.penalties + r * 4;
    rep = p[0];
    presence = p[1];
    frequency = p[2];
    inv = __frcp_rn(p[3]);
  }
  int64_t s0 = 0, s1 = 0;
  if constexpr (SEEN) {
    s0 = a.seen_start[r];
    s1 = a.seen_start[r + 1];
    if (s0 < 0 || s1 < s0 || s1 > a.n_seen) {
      if (threadIdx.x == 0 && rank == 0) atomicOr(a.err, kErrBadIndex);
      s0 = s1 = 0;
    }
  }
  const XT* x = static_cast<const XT*>(a.x) + r * a.ld_x;
  const float* bias = a.bias ? a.bias + r * a.ld_bias : nullptr;
  const uint32_t* allowed = a.allowed ? a.allowed + r * a.ld_allowed : nullptr;
  float* y = a.y ? a.y + r * a.ld_y : nullptr;
  Found f{-INFINITY, 0x7FFFFFFF, 0.f};
  for (int64_t lo64 = (int64_t)rank * a.chunk; lo64 < a.V; lo64 += (int64_t)a.split * a.chunk) {
    const int lo = (int)lo64, len = min(a.chunk, a.V - lo);
    if constexpr (SEEN) {
      if (s1 > s0) {
        __syncthreads();  // (the counts before were read)
        for (int i = threadIdx.x * 4; i < len; i += kThreads * 4) *reinterpret_cast<uint4*>(s_count + i) = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
        for (int64_t i = s0 + threadIdx.x; i < s1; i += kThreads) {
          const int64_t t = (int64_t)a.seen[i] - lo;  // (what is no token of the vocabulary counts nowhere)
          if (t >= 0 && t < len) atomicAdd(s_count + t, 1u);
        }
        __syncthreads();
      }
    }
    for (int v0 = 0; v0 < len; v0 += kItems * kThreads) {
      float z[kItems], b[kItems];
      uint32_t ok[kItems];
#pragma unroll
      for (int u = 0; u < kItems; ++u) {
        const int v = v0 + u * kThreads + (int)threadIdx.x;
        const bool there = v < len;
        z[u] = there ? load_logit(x + lo + v) : 0.f;
        b[u] = there && bias ? bias[lo + v] : 0.f;
        ok[u] = there ? (allowed ? allowed[(lo + v) >> 5] >> lane : 1u) : 0u;
      }
      float top = f.top;
#pragma unroll
      for (int u = 0; u < kItems; ++u) {
        const int v = v0 + u * kThreads + (int)threadIdx.x;
        if constexpr (SEEN) {
          const unsigned c = s1 > s0 && v < len ? s_count[v] : 0u;
          if (c) z[u] = __fsub_rn(__fsub_rn(z[u] > 0.f ? __fdiv_rn(z[u], rep) : __fmul_rn(z[u], rep), presence), __fmul_rn(frequency, (float)c));
        }
        if (bias) z[u] = __fadd_rn(z[u], b[u]);
        z[u] = ok[u] & 1u ? __fmul_rn(z[u], inv) : -INFINITY;
        if (y && v < len) y[lo + v] = z[u];
        if (z[u] > top) {
          top = z[u];
          f.token = lo + v;
        }
      }
      const float ref = ref_of(top);
      f.sum *= weight(ref_of(f.top) - ref);
      f.top = top;
#pragma unroll
      for (int u = 0; u < kItems; ++u) f.sum += weight(z[u] - ref);
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

template <typename XT, bool SEEN>
cudaError_t launch_logits_t(LogitArgs a, cudaStream_t s) {
  const int64_t want = 3ll * device_sm_count();
  a.split = 1;
  while (a.split < 8 && (a.R * a.split < want || (SEEN && (a.V + a.split - 1) / a.split > 16384)) && a.V > a.split * 4096) a.split *= 2;
  a.chunk = ((a.V + a.split - 1) / a.split + 31) / 32 * 32;
  if (SEEN && a.chunk > kMaxChunk) a.chunk = kMaxChunk;
  const size_t smem = SEEN ? (size_t)a.chunk * sizeof(unsigned) : 0;
  const cudaError_t e = smem_optin(reinterpret_cast<const void*>(logits_kernel<XT, SEEN>), smem);
  if (e != cudaSuccess) return e;
  return launch_cluster_kernel(logits_kernel<XT, SEEN>, dim3((unsigned)(a.R * a.split)), dim3(kThreads), (unsigned)a.split, smem, s, a);
}

}  // namespace

cudaError_t launch_logits(const LogitArgs& a, cudaStream_t s) {
  if (a.R <= 0) return cudaSuccess;
  if (a.x_bf16) return a.seen_start ? launch_logits_t<__nv_bfloat16, true>(a, s) : launch_logits_t<__nv_bfloat16, false>(a, s);
  return a.seen_start ? launch_logits_t<float, true>(a, s) : launch_logits_t<float, false>(a, s);
}

}  // namespace sparoa
