// Operators around the GEMMs of a decoder layer: the residual step between two
// blocks (norm after a block, gate, residual, norm before the next one), and
// rotary positions of new tokens on their way into a paged key/value cache.
#include "sparoa_kernels.h"

namespace sparoa {

namespace {

// ---------------------------------------------------------------------------
// Residual step: r = x + scale g N_post(h), y = N_pre(r), rows of C values.
//
// Bound by bytes: h and x are read once, r and y written once.  A CTA takes every
// gridDim-th row, 8 values of it a thread (16 of rows beyond 8192): rows are on their way
// into shared memory by bulk copies, up to kNormStages of them, while one is in registers between
// its reductions, and the norms' parameters, which are a thread's for all its rows, stay in
// registers.  (Rows loaded into registers by the CTA that reduces them, without any ahead:
// [8192, 4096] with both norms 102 us.)  Sums are fp32; a layer norm's variance is the mean
// square of the deviations from the mean, not a difference of two sums.  y comes from the
// fp32 r, not from the r that is stored.
// V values at p as floats, 4 or 8: 16 bytes or fewer at once
__device__ __forceinline__ void load_v(const float* p, float (&f)[4]) {
  const float4 a = *reinterpret_cast<const float4*>(p);
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
}
__device__ __forceinline__ void load_v(const float* p, float (&f)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void load_v(const __nv_bfloat16* p, float (&f)[8]) {
  unpack8(*reinterpret_cast<const uint4*>(p), f);
}
__device__ __forceinline__ void load_v(const __nv_bfloat16* p, float (&f)[4]) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  f[0] = __uint_as_float(u.x << 16);
  f[1] = __uint_as_float(u.x & 0xFFFF0000u);
  f[2] = __uint_as_float(u.y << 16);
  f[3] = __uint_as_float(u.y & 0xFFFF0000u);
}
__device__ __forceinline__ void store_v(__nv_bfloat16* p, const float (&f)[8]) {
  *reinterpret_cast<uint4*>(p) = pack8(f);
}
__device__ __forceinline__ void store_v(__nv_bfloat16* p, const float (&f)[4]) {
  *reinterpret_cast<uint2*>(p) = make_uint2(act_pack2<0>(f[0], f[1]), act_pack2<0>(f[2], f[3]));
}
__device__ __forceinline__ void store_v(float* p, const float (&f)[4]) {
  *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
}

constexpr int kNormStages = 3;

// A norm's parameters of a thread's NCH pieces of V columns: in registers, or read again
// for every row (from L1) where there are too many.
template <int V, int NCH, bool KEEP>
struct NormCols {
  float w[KEEP ? NCH : 1][V], b[KEEP ? NCH : 1][V];
  __device__ __forceinline__ void load(const NormDev& n, int i, int col, bool live) {
    float (&ww)[V] = w[KEEP ? i : 0], (&bb)[V] = b[KEEP ? i : 0];
#pragma unroll
    for (int k = 0; k < V; ++k) {
      ww[k] = 1.f;
      bb[k] = 0.f;
    }
    if (live && n.weight) load_v(n.weight + col, ww);
    if (live && n.bias) load_v(n.bias + col, bb);
  }
};

// VALUES a thread in pieces of 16 bytes of the residual stream, so that a warp's accesses
// are whole lines (fp32 in pieces of 8 values, two halves of a sector in turn: 83 us).
template <typename RT, int VALUES>
__global__ void __launch_bounds__(1024, 1) add_norm_kernel(const __grid_constant__ AddNormArgs a) {
  constexpr int V = 16 / sizeof(RT), NCH = VALUES / V;
  constexpr bool KEEP = VALUES == 8;
  extern __shared__ __align__(128) uint8_t norm_smem[];  // stages: a row of x, a row of h
  __shared__ float s_sum[2][32];
  __shared__ __align__(8) unsigned long long s_full[kNormStages];
  __shared__ int s_abort;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, T = (int)blockDim.x, at = (int)threadIdx.x;
  const int C = a.C, chunks = C / V;
  const float inv_c = 1.f / (float)C;
  const uint32_t xbytes = a.x ? (uint32_t)C * sizeof(RT) : 0u, hbytes = a.h ? (uint32_t)C * 2u : 0u;
  const long long limit = a.wait_limit ? a.wait_limit : kWaitLimitCycles;
  const unsigned S = (unsigned)a.stages;
  if (at == 0) {
    for (int i = 0; i < kNormStages; ++i) mbar_init(smem_u32(&s_full[i]), 1u);
    fence_mbar_init();
    s_abort = 0;
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  int slot = 0;
  auto sum = [&](float v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if (T > 32) {
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
  unsigned fills = 0;
  auto fill = [&](int64_t r) {  // by one thread: row r into the next stage
    if (r >= a.R) return;
    const unsigned n = fills++;
    const uint32_t bar = smem_u32(&s_full[n % S]);
    const uint32_t dst = smem_u32(norm_smem) + (n % S) * (xbytes + hbytes);
    mbar_arrive_expect_tx(bar, xbytes + hbytes);
    if (xbytes) bulk_load(dst, static_cast<const RT*>(a.x) + r * C, xbytes, bar);
    if (hbytes) bulk_load(dst + xbytes, a.h + r * C, hbytes, bar);
  };
  const int64_t step = gridDim.x;
  if (at == 0)
    for (unsigned i = 0; i < S; ++i) fill(blockIdx.x + i * step);
  NormCols<V, NCH, KEEP> post, pre;
  if constexpr (KEEP) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      post.load(a.post, i, (at + T * i) * V, at + T * i < chunks);
      pre.load(a.pre, i, (at + T * i) * V, at + T * i < chunks);
    }
  }
  float f[NCH][V];
  // f = N(f); columns past the row are zero, and stay zero until the affine part
  auto normalise = [&](const NormDev& n, NormCols<V, NCH, KEEP>& p) {
    if (n.kind == 0) return;
    if (n.kind == 2) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < NCH; ++i)
#pragma unroll
        for (int k = 0; k < V; ++k) s += f[i][k];
      const float mean = sum(s) * inv_c;
#pragma unroll
      for (int i = 0; i < NCH; ++i)
#pragma unroll
        for (int k = 0; k < V; ++k) f[i][k] = at + T * i < chunks ? f[i][k] - mean : 0.f;
    }
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int k = 0; k < V; ++k) q = fmaf(f[i][k], f[i][k], q);
    const float rs = rsqrtf(sum(q) * inv_c + n.eps);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      if constexpr (!KEEP) p.load(n, i, (at + T * i) * V, at + T * i < chunks);
#pragma unroll
      for (int k = 0; k < V; ++k) f[i][k] = fmaf(f[i][k] * rs, p.w[KEEP ? i : 0][k], p.b[KEEP ? i : 0][k]);
    }
  };
  bool ok = true;
  unsigned n = 0;
  for (int64_t r = blockIdx.x; r < a.R; r += step, ++n) {
    const uint8_t* stage = norm_smem + (n % S) * (xbytes + hbytes);
    float g[KEEP ? NCH : 1][V], x[NCH][V];
    const float* gr = a.gate ? a.gate + (a.per == 0u ? 0ll : (int64_t)((uint32_t)r / a.per) * C) : nullptr;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
#pragma unroll
      for (int k = 0; k < V; ++k) {
        g[KEEP ? i : 0][k] = 1.f;
        f[i][k] = x[i][k] = 0.f;
      }
      if (KEEP && gr && at + T * i < chunks) load_v(gr + (at + T * i) * V, g[KEEP ? i : 0]);
    }
    ok = mbar_wait(smem_u32(&s_full[n % S]), (n / S) & 1u, a.err, &s_abort, kErrTimeoutFull, limit) && ok;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = at + T * i;
      if (c < chunks) {
        if (xbytes) load_v(reinterpret_cast<const RT*>(stage) + c * V, x[i]);
        if (hbytes) load_v(reinterpret_cast<const __nv_bfloat16*>(stage + xbytes) + c * V, f[i]);
      }
    }
    __syncthreads();  // everyone has read the stage
    if (at == 0 && ok) fill(r + S * step);
    normalise(a.post, post);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = at + T * i;
      if (!KEEP && gr && c < chunks) load_v(gr + c * V, g[0]);
#pragma unroll
      for (int k = 0; k < V; ++k) f[i][k] = c < chunks ? fmaf(f[i][k], a.scale * g[KEEP ? i : 0][k], x[i][k]) : 0.f;
      if (a.r && c < chunks && ok) store_v(static_cast<RT*>(a.r) + r * C + c * V, f[i]);
    }
    if (!a.y) continue;
    normalise(a.pre, pre);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = at + T * i;
      if (c < chunks && ok) store_v(a.y + r * C + c * V, f[i]);
    }
  }
  // after a timeout: no copy is in flight into shared memory that is given back
  if (!ok && at == 0)
    for (unsigned i = fills > S ? fills - S : 0u; i < fills; ++i) mbar_drain(smem_u32(&s_full[i % S]), (i / S) & 1u, limit);
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
  const int values = a.C <= 8192 ? 8 : 16;  // a thread
  const int threads = ((a.C + values - 1) / values + 31) / 32 * 32;
  const size_t row = (size_t)a.C * ((a.x ? sizeof(RT) : 0) + (a.h ? 2 : 0)), most = 220 << 10;
  AddNormArgs args = a;
  args.stages = most / row < (size_t)kNormStages ? (int)(most / row) : kNormStages;  // (16384 fp32 values and their h: 2)
  const size_t smem = args.stages * row;
  // CTAs that fit an SM at once: 64 registers a thread, 2048 threads, 32 CTAs, shared memory
  int fit = 1024 / threads;
  if (fit > 32) fit = 32;
  const int by_smem = (int)(most / (smem + 2048));
  if (fit > by_smem) fit = by_smem;
  if (fit < 1) fit = 1;
  const int64_t grid = (int64_t)fit * device_sm_count();
  auto go = [&](auto kernel) {
    const cudaError_t e = smem_optin(reinterpret_cast<const void*>(kernel), smem);
    if (e != cudaSuccess) return e;
    return launch_kernel(kernel, dim3((unsigned)(grid < a.R ? grid : a.R)), dim3((unsigned)threads), smem, s, args);
  };
  return values == 8 ? go(add_norm_kernel<RT, 8>) : go(add_norm_kernel<RT, 16>);
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
