// Operators around the GEMMs of a decoder layer: the residual step between two
// blocks (norm after a block, gate, residual, norm before the next one), and
// rotary positions of new tokens on their way into a paged key/value cache.
#include "sparoa_kernels.h"

namespace sparoa {

namespace {

// ---------------------------------------------------------------------------
// Residual step: r = x + scale g N_post(h), y = N_pre(r), rows of C values.
//
// Bound by bytes: h and x are read once, r and y written once.  Of long rows a CTA takes every
// gridDim-th row, 8 to 32 values of it a thread.  While a row is in registers the next
// ones are on their way into shared memory by bulk copies, `stages` of them.  What is left
// above the bytes is instructions, hence packed fp32 pairs and two 16-byte pieces of the
// stream a thread: [8192, 4096] bf16 with a norm before the next block 106 us without rows
// ahead, 58 with 8 values a thread unpacked, 46 so (5.9 TB/s); 59 with 32 values a thread
// and a warp per 1024, for want of warps.  Requesting parameters into L1 ahead of their
// use made every size slower.
// Sums are fp32; a layer norm's variance is the mean square of the deviations from the
// mean, not a difference of two sums.  y comes from the fp32 r, not from the r that is
// stored.
// 16 bytes of a row or, with 4 values, 8 (bf16) as packed fp32 pairs; zeros unless `live`
__device__ __forceinline__ f2_t pair_of(uint32_t u) {
  return f2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
}
__device__ __forceinline__ void load_p(const float* p, bool live, f2_t (&f)[2]) {
  const float4 a = live ? *reinterpret_cast<const float4*>(p) : make_float4(0.f, 0.f, 0.f, 0.f);
  f[0] = f2(a.x, a.y);
  f[1] = f2(a.z, a.w);
}
__device__ __forceinline__ void load_p(const float* p, bool live, f2_t (&f)[4]) {
  f2_t a[2], b[2];
  load_p(p, live, a);
  load_p(p + 4, live, b);
  f[0] = a[0]; f[1] = a[1]; f[2] = b[0]; f[3] = b[1];
}
__device__ __forceinline__ void load_p(const __nv_bfloat16* p, bool live, f2_t (&f)[4]) {
  const uint4 u = live ? *reinterpret_cast<const uint4*>(p) : make_uint4(0u, 0u, 0u, 0u);
  f[0] = pair_of(u.x); f[1] = pair_of(u.y); f[2] = pair_of(u.z); f[3] = pair_of(u.w);
}
__device__ __forceinline__ void load_p(const __nv_bfloat16* p, bool live, f2_t (&f)[2]) {
  const uint2 u = live ? *reinterpret_cast<const uint2*>(p) : make_uint2(0u, 0u);
  f[0] = pair_of(u.x);
  f[1] = pair_of(u.y);
}
__device__ __forceinline__ uint32_t rounded(f2_t v) {
  float lo, hi;
  f2_split(v, lo, hi);
  return act_pack2<0>(lo, hi);
}
__device__ __forceinline__ void store_p(__nv_bfloat16* p, const f2_t (&f)[4]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(rounded(f[0]), rounded(f[1]), rounded(f[2]), rounded(f[3]));
}
__device__ __forceinline__ void store_p(__nv_bfloat16* p, const f2_t (&f)[2]) {
  *reinterpret_cast<uint2*>(p) = make_uint2(rounded(f[0]), rounded(f[1]));
}
__device__ __forceinline__ void store_p(float* p, const f2_t (&f)[2]) {
  float4 v;
  f2_split(f[0], v.x, v.y);
  f2_split(f[1], v.z, v.w);
  *reinterpret_cast<float4*>(p) = v;
}

// A row in registers, NCH 16-byte pieces of the stream a thread, the thread's T pieces apart.
template <typename RT, int NCH>
struct NormRow {
  static constexpr int V = 16 / sizeof(RT), P = V / 2;
  using Values = f2_t[NCH][P];

  static __device__ __forceinline__ void load_weights(const NormDev& n, Values& w, int at, int T, int C) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
#pragma unroll
      for (int k = 0; k < P; ++k) w[i][k] = f2(1.f, 1.f);
      if (n.weight) load_p(n.weight + (at + T * i) * V, at + T * i < C / V, w[i]);
    }
  }
  // f = N(f); columns past the row are zero, and stay zero until the affine part.  `kept`:
  // the weights of the thread's columns, or null to read them (from L1).
  template <typename Sum>
  static __device__ __forceinline__ void normalise(const NormDev& n, Values& f, const Values* kept, int at, int T, int C,
                                                   const Sum& sum) {
    const int chunks = C / V;
    const float inv_c = 1.f / (float)C;
    if (n.kind == 0) return;
    float lo, hi;
    if (n.kind == 2) {
      f2_t s = f[0][0];
#pragma unroll
      for (int i = 0; i < NCH; ++i)
#pragma unroll
        for (int k = 0; k < P; ++k)
          if (i + k > 0) s = fadd2(s, f[i][k]);
      f2_split(s, lo, hi);
      const float mean = sum(lo + hi) * -inv_c;
#pragma unroll
      for (int i = 0; i < NCH; ++i)
        if (at + T * i < chunks)
#pragma unroll
          for (int k = 0; k < P; ++k) f[i][k] = fadd2(f[i][k], f2(mean, mean));
    }
    f2_t q = fmul2(f[0][0], f[0][0]);
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int k = 0; k < P; ++k)
        if (i + k > 0) q = ffma2(f[i][k], f[i][k], q);
    f2_split(q, lo, hi);
    const float rs = rsqrtf(sum(lo + hi) * inv_c + n.eps);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = at + T * i;
      const bool live = c < chunks;
      f2_t w[P];
#pragma unroll
      for (int k = 0; k < P; ++k) {
        f[i][k] = fmul2(f[i][k], f2(rs, rs));
        if (kept) f[i][k] = fmul2(f[i][k], (*kept)[i][k]);
      }
      if (!kept && n.weight) {
        load_p(n.weight + c * V, live, w);
#pragma unroll
        for (int k = 0; k < P; ++k) f[i][k] = fmul2(f[i][k], w[k]);
      }
      if (n.bias) {
        load_p(n.bias + c * V, live, w);
#pragma unroll
        for (int k = 0; k < P; ++k) f[i][k] = fadd2(f[i][k], w[k]);
      }
    }
  }

  // Row r from its x and h (in f) to r and y; `store`: whether they are written.
  template <typename Sum>
  static __device__ __forceinline__ void finish(const AddNormArgs& a, int64_t r, Values& f, const Values& x,
                                                const Values* post_w, const Values* pre_w, int at, int T, bool store,
                                                const Sum& sum) {
    const int C = a.C, chunks = C / V;
    normalise(a.post, f, post_w, at, T, C, sum);
    if (a.gate) {
      const float* gr = a.gate + (a.per == 0u ? 0ll : (int64_t)((uint32_t)r / a.per) * C);
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int c = at + T * i;
        f2_t g[P];
        load_p(gr + c * V, c < chunks, g);
#pragma unroll
        for (int k = 0; k < P; ++k) f[i][k] = fmul2(f[i][k], g[k]);
      }
    }
    const int64_t row = r * C;
    const f2_t scale = f2(a.scale, a.scale);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = at + T * i;
#pragma unroll
      for (int k = 0; k < P; ++k) f[i][k] = ffma2(f[i][k], scale, x[i][k]);
      if (a.r && c < chunks && store) store_p(static_cast<RT*>(a.r) + row + c * V, f[i]);
    }
    if (!a.y) return;
    normalise(a.pre, f, pre_w, at, T, C, sum);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = at + T * i;
      if (c < chunks && store) store_p(a.y + row + c * V, f[i]);
    }
  }
};

template <int VALUES>
constexpr int kNormThreads = VALUES == 8 ? 1024 : 512;  // at most
constexpr int kNormStages = 4;  // at most

// VALUES a thread in pieces of 16 bytes of the residual stream, so that a warp's accesses
// are whole lines (fp32 in pieces of 8 values, two halves of a sector in turn, was slower
// by a sixth).
template <typename RT, int VALUES>
__global__ void __launch_bounds__(kNormThreads<VALUES>, VALUES <= 16 ? 1024 / kNormThreads<VALUES> : 1) add_norm_kernel(const __grid_constant__ AddNormArgs a) {
  constexpr int V = 16 / sizeof(RT), NCH = VALUES / V, P = V / 2;
  using Row = NormRow<RT, NCH>;
  constexpr bool KEEP = VALUES == 8;
  extern __shared__ __align__(128) uint8_t norm_smem[];  // stages: a row of x, a row of h
  __shared__ float s_sum[2][32];
  __shared__ __align__(8) unsigned long long s_full[kNormStages];
  __shared__ int s_abort;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, T = (int)blockDim.x, at = (int)threadIdx.x;
  const int C = a.C, chunks = C / V;
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
  const int64_t step = gridDim.x;
  unsigned fills = 0;
  auto fill = [&](int64_t r) {  // by one thread: row r into the next stage
    if (r >= a.R) return;
    const uint32_t bar = smem_u32(&s_full[fills % S]);
    const uint32_t dst = smem_u32(norm_smem) + (fills % S) * (xbytes + hbytes);
    ++fills;
    mbar_arrive_expect_tx(bar, xbytes + hbytes);
    if (xbytes) bulk_load(dst, static_cast<const RT*>(a.x) + r * C, xbytes, bar);
    if (hbytes) bulk_load(dst + xbytes, a.h + r * C, hbytes, bar);
  };
  if (at == 0)
    for (unsigned i = 0; i < S; ++i) fill(blockIdx.x + i * step);
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
  // the norms' weights of the thread's columns: in registers, or read again for every row
  // (from L1) where there are too many
  typename Row::Values post_w, pre_w;
  if constexpr (KEEP) {
    Row::load_weights(a.post, post_w, at, T, C);
    Row::load_weights(a.pre, pre_w, at, T, C);
  }
  bool ok = true;
  unsigned st = 0, phase = 0;
#pragma unroll 1
  for (int64_t r = blockIdx.x; r < a.R; r += step) {
    const uint8_t* stage = norm_smem + st * (xbytes + hbytes);
    typename Row::Values x, f;
    ok = mbar_wait(smem_u32(&s_full[st]), phase, a.err, &s_abort, kErrTimeoutFull, limit) && ok;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = at + T * i;
      load_p(reinterpret_cast<const RT*>(stage) + c * V, c < chunks && xbytes, x[i]);
      load_p(reinterpret_cast<const __nv_bfloat16*>(stage + xbytes) + c * V, c < chunks && hbytes, f[i]);
    }
    if (T > 32)
      __syncthreads();  // everyone has read the stage
    else
      __syncwarp();
    if (at == 0 && ok) fill(r + S * step);
    if (++st == S) {
      st = 0;
      phase ^= 1u;
    }
    Row::finish(a, r, f, x, KEEP ? &post_w : nullptr, KEEP ? &pre_w : nullptr, at, T, ok, sum);
  }
  // after a timeout: no copy is in flight into shared memory that is given back
  if (!ok && at == 0)
    for (unsigned i = fills > S ? fills - S : 0u; i < fills; ++i) mbar_drain(smem_u32(&s_full[i % S]), (i / S) & 1u, limit);
}

// Short rows: a warp for each, which needs no barrier and no shared memory, and a CTA for
// every two or four (rows of 512 bytes: 5.8 us for 12000 with four, 6.6 with two).  The next
// norm's weights are on their way with the row where a lane has 24 values of it ([6304, 768]
// bf16 9.8 us so, 10.6 without; with 16 values 6.6 and 6.1, with 32 12.1 and 11.6: the
// registers that they take cost warps).
template <typename RT, int NCH>
constexpr int kShortWarps = NCH * 16 / sizeof(RT) <= 8 ? 4 : 2;
template <typename RT, int NCH>
__global__ void __launch_bounds__(32 * kShortWarps<RT, NCH>) short_norm_kernel(const __grid_constant__ AddNormArgs a) {
  using Row = NormRow<RT, NCH>;
  const int lane = threadIdx.x & 31, C = a.C, chunks = C / Row::V;
  const int64_t r = (int64_t)blockIdx.x * kShortWarps<RT, NCH> + (threadIdx.x >> 5);
  pdl_wait();
  pdl_trigger();
  if (r >= a.R) return;
  typename Row::Values x, f;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = lane + 32 * i;
    load_p(static_cast<const RT*>(a.x) + r * C + c * Row::V, a.x && c < chunks, x[i]);
    load_p(a.h + r * C + c * Row::V, a.h && c < chunks, f[i]);
  }
  typename Row::Values pre_w;
  constexpr bool EARLY = NCH * Row::V == 24;
  if constexpr (EARLY) Row::load_weights(a.pre, pre_w, lane, 32, C);
  Row::finish(a, r, f, x, nullptr, EARLY ? &pre_w : nullptr, lane, 32, true, [](float v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
  });
}

// ---------------------------------------------------------------------------
// Rotary positions and the cache's append: a CTA per token.
//
// Bound by bytes: a token's row is read once and written once.  The angle of pair i
// at position p is p f_i; turns[i] is f_i / (2 pi) in units of 2^-64, so p turns[i]
// modulo 2^64 is the angle's fraction of a turn, exactly, however far the position
// (a product of floats is off by 2^-25 of the angle itself: half a degree at 131072).
// 16 values of a head are one item: two 16-byte chunks read, two written.  A thread's items
// are the same 16 of every kRopeThreads / 8th (or / 4th) head, so their cosines and sines
// are read from shared memory once (for every item again, in pairs: 70 % of the L1's
// bandwidth), and its first items are on their way while the place is looked up.
// [8191 tokens, 48 heads of 128] 33 us so, 30 the bytes.
constexpr int kRopeItems = 4;  // of a thread at once
static_assert(kRopeThreads > 64, "a thread without an angle");
__global__ void __launch_bounds__(kRopeThreads) rope_append_kernel(const __grid_constant__ RopeArgs a) {
  __shared__ __align__(16) float s_cos[64], s_sin[64];
  __shared__ int64_t s_base;
  const int64_t t = blockIdx.x;
  const int D = a.D, sl = D == 128 ? 3 : 2, items = (a.heads + 2 * a.kv_heads) << sl;
  const int s = threadIdx.x & ((1 << sl) - 1);
  const bool turns = s < a.rot / 16, half = turns && !a.interleaved;  // of a rotated head
  const int h0 = half ? s * 8 : s * 16, h1 = half ? a.rot / 2 + s * 8 : h0 + 8;
  const __nv_bfloat16* src = a.qkv + t * a.ld_qkv;
  pdl_wait();
  pdl_trigger();
  uint4 u[kRopeItems], w[kRopeItems];
  auto fetch = [&](int it0) {
#pragma unroll
    for (int i = 0; i < kRopeItems; ++i) {
      const int it = it0 + i * kRopeThreads, head = it >> sl;
      if (it >= items) break;
      const bool value = head >= a.heads + a.kv_heads;
      u[i] = *reinterpret_cast<const uint4*>(src + head * D + (value ? s * 16 : h0));
      w[i] = *reinterpret_cast<const uint4*>(src + head * D + (value ? s * 16 + 8 : h1));
    }
  };
  fetch(threadIdx.x);
  // the token's sequence: how many of them end at or before it
  int b = 0;
  const int64_t room = (int64_t)a.max_pages << a.page_log2;
  for (int i0 = 0; i0 < a.batch; i0 += kRopeThreads) {
    const int i = i0 + (int)threadIdx.x;
    const int64_t end = i < a.batch ? a.q_start[i + 1] : 0;
    b += __syncthreads_count(i < a.batch && end <= t);
  }
  if (t == 0) {  // the first CTA looks the lists over
    for (int i = threadIdx.x; i < a.batch; i += kRopeThreads) {
      const int64_t begin = a.q_start[i], end = a.q_start[i + 1], len = a.kv_len[i];
      if (begin < 0 || end < begin || end > a.T || len < 0 || len > room) atomicOr(a.err, kErrBadIndex);
    }
  }
  if (b >= a.batch || t < a.q_start[0]) return;  // a row of no sequence
  const int64_t end = a.q_start[b + 1], len = a.kv_len[b], place = len - end + t;
  // by a thread that has no angle to do: the row of the place's first key head, -1: not cached.
  // A sequence that its lists give rows it cannot have caches none of them: they would take the
  // places of others.
  if (threadIdx.x == kRopeThreads - 1) {
    int64_t base = -1;
    const int64_t begin = a.q_start[b];
    if (place >= 0 && begin >= 0 && begin <= t && end > t && end <= a.T && len <= room) {
      const int page = a.table[b * a.table_stride + (place >> a.page_log2)];
      if (page >= 0 && page < a.pages)
        base = (((int64_t)page * a.kv_heads) << a.page_log2) + (place & ((1 << a.page_log2) - 1));
      else
        atomicOr(a.err, kErrBadIndex);
    }
    s_base = base;
  }
  const uint64_t pos = (uint64_t)(a.positions ? (int64_t)a.positions[t] : place);
  for (int i = threadIdx.x; i < a.rot / 2; i += kRopeThreads) {
    const int32_t turn = (int32_t)((pos * a.turns[i]) >> 32);  // signed fraction of a turn, 2^-32
    float sn, cs;
    sincospif((float)turn * 4.656612873077393e-10f, &sn, &cs);  // 2^-31: half turns
    s_cos[i] = cs * a.scale;
    s_sin[i] = sn * a.scale;
  }
  __syncthreads();
  const int64_t base = s_base;
  float cs[8], sn[8];
  if (turns) {
#pragma unroll
    for (int k = 0; k < 8; k += 4) {
      const float4 c4 = *reinterpret_cast<const float4*>(s_cos + s * 8 + k), s4 = *reinterpret_cast<const float4*>(s_sin + s * 8 + k);
      cs[k] = c4.x; cs[k + 1] = c4.y; cs[k + 2] = c4.z; cs[k + 3] = c4.w;
      sn[k] = s4.x; sn[k + 1] = s4.y; sn[k + 2] = s4.z; sn[k + 3] = s4.w;
    }
  }
  for (int it0 = threadIdx.x; it0 < items; it0 += kRopeItems * kRopeThreads) {
    if (it0 != (int)threadIdx.x) fetch(it0);
#pragma unroll
    for (int i = 0; i < kRopeItems; ++i) {
      const int it = it0 + i * kRopeThreads, head = it >> sl;
      if (it >= items) break;
      const bool value = head >= a.heads + a.kv_heads;
      __nv_bfloat16* dst = a.q_out + t * a.ld_q + head * D;
      if (head >= a.heads) {
        if (base < 0) continue;
        const int kh = value ? head - a.heads - a.kv_heads : head - a.heads;
        dst = (value ? a.v : a.k) + (base + ((int64_t)kh << a.page_log2)) * D;
      }
      if (turns && !value) {
        float p[8], q[8];
        unpack8(u[i], p);
        unpack8(w[i], q);
        if (half) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float lo = p[k], hi = q[k];
            p[k] = lo * cs[k] - hi * sn[k];
            q[k] = hi * cs[k] + lo * sn[k];
          }
        } else {
#pragma unroll
          for (int k = 0; k < 8; k += 2) {
            const int c = k / 2, e = 4 + k / 2;
            const float p0 = p[k], p1 = p[k + 1], q0 = q[k], q1 = q[k + 1];
            p[k] = p0 * cs[c] - p1 * sn[c];
            p[k + 1] = p1 * cs[c] + p0 * sn[c];
            q[k] = q0 * cs[e] - q1 * sn[e];
            q[k + 1] = q1 * cs[e] + q0 * sn[e];
          }
        }
        u[i] = make_uint4(act_pack2<0>(p[0], p[1]), act_pack2<0>(p[2], p[3]), act_pack2<0>(p[4], p[5]), act_pack2<0>(p[6], p[7]));
        w[i] = make_uint4(act_pack2<0>(q[0], q[1]), act_pack2<0>(q[2], q[3]), act_pack2<0>(q[4], q[5]), act_pack2<0>(q[6], q[7]));
      }
      *reinterpret_cast<uint4*>(dst + (value ? s * 16 : h0)) = u[i];
      *reinterpret_cast<uint4*>(dst + (value ? s * 16 + 8 : h1)) = w[i];
    }
  }
}

template <typename RT, int VALUES>
cudaError_t launch_add_norm_v(AddNormArgs a, cudaStream_t s) {
  const void* kernel = reinterpret_cast<const void*>(add_norm_kernel<RT, VALUES>);
  static const int regs = [&] {  // (the same on every device)
    cudaFuncAttributes at;
    return cudaFuncGetAttributes(&at, kernel) == cudaSuccess ? (at.numRegs + 7) / 8 * 8 : 128;
  }();
  const int threads = ((a.C + VALUES - 1) / VALUES + 31) / 32 * 32;
  // CTAs that fit an SM at once (by their registers, with two rows each in shared memory),
  // and the rows that each has on its way
  const size_t row = (size_t)a.C * ((a.x ? sizeof(RT) : 0) + (a.h ? 2 : 0)), most = 216 << 10;
  int fit = 65536 / (regs * threads);
  if (fit > 2048 / threads) fit = 2048 / threads;
  if (fit > 32) fit = 32;
  const int by_smem = (int)(most / (2 * row + 1536));
  if (fit > by_smem) fit = by_smem;
  if (fit < 1) fit = 1;
  a.stages = (int)((most / fit - 1536) / row);
  if (a.stages > kNormStages) a.stages = kNormStages;
  const size_t smem = a.stages * row;
  const int64_t grid = (int64_t)fit * device_sm_count();
  const cudaError_t e = smem_optin(kernel, smem);
  if (e != cudaSuccess) return e;
  return launch_kernel(add_norm_kernel<RT, VALUES>, dim3((unsigned)(grid < a.R ? grid : a.R)), dim3((unsigned)threads), smem,
                       s, a);
}

template <typename RT, int NCH>
cudaError_t launch_short_norm(const AddNormArgs& a, cudaStream_t s) {
  constexpr int W = kShortWarps<RT, NCH>;
  return launch_kernel(short_norm_kernel<RT, NCH>, dim3((unsigned)((a.R + W - 1) / W)), dim3(32 * W), 0, s, a);
}

// A warp a row where it has two 16-byte pieces of the stream a lane at most ([6304, 64] bf16
// 2.4 us, by CTAs 5.3; [300, 512] 2.6 and 2.5) and, up to 1024 values, where there are 8 rows
// an SM ([6304, 768] bf16 with a gate 9.9, 12.7; [2500, 768] fp32 5.6, 6.2; 1200 rows equal;
// [300, 768] 3.1, 2.6: CTAs begin on a row with more loads), or 16 with more than 6 pieces
// ([2500, 1024] fp32 7.8, 8.5; 1200 rows 6.0, 4.9).  Else by CTAs:
// two pieces a thread ([8192, 4096] bf16 46 us, one 48; fp32 75, four 78), one of a bf16 row
// of up to 1024 values, whose weights then stay in registers ([6304, 768] 12.9, two 14.2),
// and four or eight where threads run out.
template <typename RT>
cudaError_t launch_add_norm_t(const AddNormArgs& a, cudaStream_t s) {
  const int pieces = (a.C * (int)sizeof(RT) + 511) / 512;
  if (pieces == 1) return launch_short_norm<RT, 1>(a, s);
  if (pieces == 2) return launch_short_norm<RT, 2>(a, s);
  if (a.C <= 1024 && a.R >= (pieces <= 6 ? 8ll : 16ll) * device_sm_count()) {
    if constexpr (sizeof(RT) == 2)
      return pieces == 3 ? launch_short_norm<RT, 3>(a, s) : launch_short_norm<RT, 4>(a, s);
    else
      return pieces <= 4   ? launch_short_norm<RT, 4>(a, s)
             : pieces <= 6 ? launch_short_norm<RT, 6>(a, s)
                           : launch_short_norm<RT, 8>(a, s);
  }
  if (a.C > 8192) return launch_add_norm_v<RT, 32>(a, s);
  if constexpr (sizeof(RT) == 2)
    if (a.C > 1024) return launch_add_norm_v<RT, 16>(a, s);
  return launch_add_norm_v<RT, 8>(a, s);
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
