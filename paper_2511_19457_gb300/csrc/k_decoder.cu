// Operators around the GEMMs of a decoder layer: the residual step between two
// blocks (norm after a block, gate, residual, norm before the next one), and
// rotary positions of new tokens on their way into a paged key/value cache.
#include "sparoa_kernels.h"

namespace sparoa {

namespace {

// ---------------------------------------------------------------------------
// Residual step: r = x + scale g N_post(h), y = N_pre(r), rows of C values.
//
// Bound by bytes: h and x are read once, r and y written once.  A row is held in
// registers between the reductions (8-value chunks, NCH a thread): by a warp where
// C <= 1024, else by a CTA of its own.  Sums are fp32; a layer norm's variance is
// the mean square of the deviations from the mean, not a difference of two sums.
// y comes from the fp32 r, not from the r that is stored.
template <typename RT>
__device__ __forceinline__ void load8(const RT* p, float (&f)[8]);
template <>
__device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16* p, float (&f)[8]) {
  unpack8(*reinterpret_cast<const uint4*>(p), f);
}
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&f)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&f)[8]) {
  *reinterpret_cast<uint4*>(p) = pack8(f);
}
__device__ __forceinline__ void store8(float* p, const float (&f)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
}

constexpr int kNormWarps = 4;  // warps of a CTA whose rows take a warp each

template <typename RT, int NCH, bool WARP>
__global__ void __launch_bounds__(WARP ? 32 * kNormWarps : 512) add_norm_kernel(const __grid_constant__ AddNormArgs a) {
  __shared__ float s_sum[2][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int T = WARP ? 32 : (int)blockDim.x, at = WARP ? lane : (int)threadIdx.x;
  const int C = a.C, chunks = C / 8;
  const float inv_c = 1.f / (float)C;
  int slot = 0;
  auto sum = [&](float v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if constexpr (!WARP) {
      // (two slots in turn: a slot is written again only after another slot's barrier)
      if (lane == 0) s_sum[slot][warp] = v;
      __syncthreads();
      v = lane < (T >> 5) ? s_sum[slot][lane] : 0.f;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
      slot ^= 1;
    }
    return v;
  };
  float f[NCH][8];
  // f = N(f); chunks past the row stay zero until the affine part, which they skip
  auto normalise = [&](const NormDev& n) {
    if (n.kind == 0) return;
    if (n.kind == 2) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < NCH; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) s += f[i][k];
      const float mean = sum(s) * inv_c;
#pragma unroll
      for (int i = 0; i < NCH; ++i)
        if (at + T * i < chunks)
#pragma unroll
          for (int k = 0; k < 8; ++k) f[i][k] -= mean;
    }
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) q = fmaf(f[i][k], f[i][k], q);
    const float rs = rsqrtf(sum(q) * inv_c + n.eps);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = at + T * i;
      if (c >= chunks) continue;
      float w[8], b[8];
      if (n.weight) load8<float>(n.weight + c * 8, w);
      if (n.bias) load8<float>(n.bias + c * 8, b);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float v = f[i][k] * rs;
        if (n.weight) v *= w[k];
        if (n.bias) v += b[k];
        f[i][k] = v;
      }
    }
  };
  pdl_wait();
  pdl_trigger();
  const int64_t step = (int64_t)gridDim.x * (WARP ? kNormWarps : 1);
  for (int64_t r = WARP ? (int64_t)blockIdx.x * kNormWarps + warp : (int64_t)blockIdx.x; r < a.R; r += step) {
    const RT* xr = static_cast<const RT*>(a.x) + r * C;
    float x[NCH][8];
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = at + T * i;
#pragma unroll
      for (int k = 0; k < 8; ++k) f[i][k] = x[i][k] = 0.f;
      if (c < chunks) {
        if (a.h) load8<__nv_bfloat16>(a.h + r * C + c * 8, f[i]);
        if (a.x) load8<RT>(xr + c * 8, x[i]);
      }
    }
    normalise(a.post);
    const float* gr = a.gate ? a.gate + (a.per ? r / a.per : 0) * C : nullptr;
    RT* rr = static_cast<RT*>(a.r) + r * C;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = at + T * i;
      if (c >= chunks) continue;
      float g[8];
      if (gr) load8<float>(gr + c * 8, g);
#pragma unroll
      for (int k = 0; k < 8; ++k) f[i][k] = fmaf(f[i][k], gr ? a.scale * g[k] : a.scale, x[i][k]);
      if (a.r) store8(rr + c * 8, f[i]);
    }
    if (!a.y) continue;
    normalise(a.pre);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = at + T * i;
      if (c < chunks) store8(a.y + r * C + c * 8, f[i]);
    }
  }
}

// ---------------------------------------------------------------------------
// Rotary positions and the cache's append: a CTA per token.
//
// Bound by bytes: a token's row is read once and written once.  The angle of pair i
// at position p is p f_i; turns[i] is f_i / (2 pi) in units of 2^-64, so p turns[i]
// modulo 2^64 is the angle's fraction of a turn, exactly, however far the position
// (a product of floats is off by 2^-25 of the angle itself: half a degree at 131072).
// Every value of 16 a head is one item: two 16-byte chunks read, two written.
__global__ void __launch_bounds__(kRopeThreads) rope_append_kernel(const __grid_constant__ RopeArgs a) {
  __shared__ float2 s_cs[64];
  const int64_t t = blockIdx.x;
  pdl_wait();
  pdl_trigger();
  // the token's sequence: how many of them end at or before it
  int b = 0;
  for (int i0 = 0; i0 < a.batch; i0 += kRopeThreads) {
    const int i = i0 + (int)threadIdx.x;
    b += __syncthreads_count(i < a.batch && (int64_t)a.q_start[i + 1] <= t);
  }
  if (b >= a.batch || t < a.q_start[0]) return;  // a row of no sequence
  const int64_t place = (int64_t)a.kv_len[b] - a.q_start[b + 1] + t;
  const uint64_t pos = (uint64_t)(a.positions ? (int64_t)a.positions[t] : place);
  for (int i = threadIdx.x; i < a.rot / 2; i += kRopeThreads) {
    const int32_t turn = (int32_t)((pos * a.turns[i]) >> 32);  // signed fraction of a turn, 2^-32
    float sn, cs;
    sincospif((float)turn * 4.656612873077393e-10f, &sn, &cs);  // 2^-31: half turns
    s_cs[i] = make_float2(cs * a.scale, sn * a.scale);
  }
  // the page of the token's place; -1: not cached
  int64_t base = -1;
  if (place >= 0) {
    const int64_t col = place >> a.page_log2;
    const int page = col < a.max_pages ? a.table[b * a.table_stride + col] : -1;
    if (page >= 0 && page < a.pages)
      base = (((int64_t)page * a.kv_heads) << a.page_log2) + (place & ((1 << a.page_log2) - 1));
    else if (threadIdx.x == 0)
      atomicOr(a.err, kErrBadIndex);
  }
  __syncthreads();
  const int D = a.D, sl = D == 128 ? 3 : 2, items = (a.heads + 2 * a.kv_heads) << sl;
  const __nv_bfloat16* src = a.qkv + t * a.ld_qkv;
  for (int it = threadIdx.x; it < items; it += kRopeThreads) {
    const int head = it >> sl, s = it & ((1 << sl) - 1);
    const bool turned = head < a.heads + a.kv_heads && s < a.rot / 16;
    const bool half = turned && !a.interleaved;
    const int c0 = half ? s * 8 : s * 16, c1 = half ? a.rot / 2 + s * 8 : c0 + 8;
    __nv_bfloat16* dst;
    if (head < a.heads) {
      dst = a.q_out + t * a.ld_q + head * D;
    } else {
      if (base < 0) continue;
      const bool key = head < a.heads + a.kv_heads;
      const int kh = key ? head - a.heads : head - a.heads - a.kv_heads;
      dst = (key ? a.k : a.v) + (base + ((int64_t)kh << a.page_log2)) * D;
    }
    uint4 u = *reinterpret_cast<const uint4*>(src + head * D + c0);
    uint4 w = *reinterpret_cast<const uint4*>(src + head * D + c1);
    if (turned) {
      float p[8], q[8];
      unpack8(u, p);
      unpack8(w, q);
      if (half) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float2 cs = s_cs[s * 8 + k];
          const float lo = p[k], hi = q[k];
          p[k] = lo * cs.x - hi * cs.y;
          q[k] = hi * cs.x + lo * cs.y;
        }
      } else {
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
          const float2 c = s_cs[s * 8 + k / 2], e = s_cs[s * 8 + 4 + k / 2];
          const float p0 = p[k], p1 = p[k + 1], q0 = q[k], q1 = q[k + 1];
          p[k] = p0 * c.x - p1 * c.y;
          p[k + 1] = p1 * c.x + p0 * c.y;
          q[k] = q0 * e.x - q1 * e.y;
          q[k + 1] = q1 * e.x + q0 * e.y;
        }
      }
      u = pack8(p);
      w = pack8(q);
    }
    *reinterpret_cast<uint4*>(dst + c0) = u;
    *reinterpret_cast<uint4*>(dst + c1) = w;
  }
}

template <typename RT>
cudaError_t launch_add_norm_t(const AddNormArgs& a, cudaStream_t s) {
  const int chunks = a.C / 8;
  const int64_t most = (int64_t)1 << 30;
  auto go = [&](auto kernel, int threads, int64_t grid) {
    return launch_kernel(kernel, dim3((unsigned)(grid < most ? grid : most)), dim3((unsigned)threads), 0, s, a);
  };
  const int64_t wgrid = (a.R + kNormWarps - 1) / kNormWarps;
  if (chunks <= 32) return go(add_norm_kernel<RT, 1, true>, 32 * kNormWarps, wgrid);
  if (chunks <= 64) return go(add_norm_kernel<RT, 2, true>, 32 * kNormWarps, wgrid);
  if (chunks <= 128) return go(add_norm_kernel<RT, 4, true>, 32 * kNormWarps, wgrid);
  if (chunks <= 1024) return go(add_norm_kernel<RT, 2, false>, ((chunks + 1) / 2 + 31) / 32 * 32, a.R);
  return go(add_norm_kernel<RT, 4, false>, ((chunks + 3) / 4 + 31) / 32 * 32, a.R);
}

}  // namespace

cudaError_t launch_add_norm(const AddNormArgs& a, cudaStream_t s) {
  if (a.R <= 0) return cudaSuccess;
  return a.res_f32 ? launch_add_norm_t<float>(a, s) : launch_add_norm_t<__nv_bfloat16>(a, s);
}

cudaError_t launch_rope_append(const RopeArgs& a, cudaStream_t s) {
  if (a.T <= 0) return cudaSuccess;
  return launch_kernel(rope_append_kernel, dim3((unsigned)a.T), dim3(kRopeThreads), 0, s, a);
}

}  // namespace sparoa
