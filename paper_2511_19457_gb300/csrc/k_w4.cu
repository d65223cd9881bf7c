// Products of a few tokens' rows with weights of 4 bits: y = epilogue(x W^T),
// W[n][k] = scale[n][k / group] (code[n][k] - zero[n][k / group]).
//
// Bound by the bytes of the weights, half a byte each and read once.  They are laid out
// once (w4_pack_kernel) in tiles of 16 rows x 128 columns that a warp copies whole: the
// codes as the lanes of an mma.sync m16n8k16 take them, then the tile's scales and zeros.
// A code becomes the bf16 number 128 + code by one logic operation (its four bits are the
// low bits of the mantissa), and 128 + zero is taken away, which is exact; the products
// with x are summed in fp32 over a group, and only that sum is multiplied by the scale.
// So nothing is rounded before the result but the fp32 sums.
#include "sparoa_kernels.h"

namespace sparoa {

namespace {

constexpr int kTileK = 128;
constexpr int kWarps = 8;             // each with R tiles of 16 rows, all over the same columns
constexpr int kThreads = 32 * (kWarps + 1);  // and a warp that copies x
constexpr int kXTiles = 2;            // tiles of columns in a stage of x
constexpr int kXPitch = kXTiles * kTileK * 2 + 64;  // of a token's row: two tokens' 64 bytes in different banks
constexpr int kXStages = 3;

__host__ __device__ constexpr int tile_bytes(int groups, bool zeros) { return 1024 + groups * (zeros ? 48 : 32); }

template <int R, int NT>
struct Cfg {
  static constexpr int kStages = R == 1 ? 6 : 4;      // tiles of columns on their way, a warp
  static constexpr int kRows = 16 * R * kWarps;       // of a CTA
  static constexpr int kTokens = 8 * NT;
  static constexpr int kPitch = kRows + 4;            // floats: a fragment's stores are free of bank conflicts
  static size_t smem(int tile) {
    const size_t ring = (size_t)kWarps * kStages * R * tile + (size_t)kXStages * kTokens * kXPitch;
    const size_t part = (size_t)kTokens * kPitch * sizeof(float);
    return (ring > part ? ring : part) + 128;
  }
};

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 lds_u4(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds_u16(uint32_t addr) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds_u8(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(addr)
               : "memory");
  return v;
}
// codes 2 m and 2 m + 1 of a word, less the zero: a pair of bf16 whole numbers
__device__ __forceinline__ uint32_t pair_of(uint32_t word, int m, uint32_t zero) {
  const uint32_t v = ((word >> (4 * m)) & 0x000F000Fu) | 0x43004300u;
  const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), *reinterpret_cast<const __nv_bfloat162*>(&zero));
  return *reinterpret_cast<const uint32_t*>(&d);
}

// GROUPS: of a tile's columns (128 / group)
template <int GROUPS, int R, int NT>
__global__ void __launch_bounds__(kThreads) w4_kernel(const __grid_constant__ W4Args a) {
  using C = Cfg<R, NT>;
  constexpr int S = C::kStages;
  extern __shared__ __align__(128) uint8_t smem_raw[];
  __shared__ __align__(8) unsigned long long s_full[kWarps][S], s_xfull[kXStages], s_xempty[kXStages];
  __shared__ int s_abort;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, tq = lane & 3;
  const int tile = tile_bytes(GROUPS, a.zeros);
  const uint32_t base = (smem_u32(smem_raw) + 127u) & ~127u, xring = base + kWarps * S * R * tile;
  const uint32_t ring = base + warp * S * R * tile;
  const int rank = (int)(blockIdx.x % a.split), block = (int)(blockIdx.x / a.split), tok0 = blockIdx.y * C::kTokens;
  const int tokens = min(C::kTokens, a.M - tok0);
  const int t0 = (int)((int64_t)rank * a.tiles / a.split), t1 = (int)((int64_t)(rank + 1) * a.tiles / a.split), count = t1 - t0;
  const int rt0 = (block * kWarps + warp) * R;  // the warp's first tile of rows
  const long long limit = a.wait_limit ? a.wait_limit : kWaitLimitCycles;
  if (threadIdx.x == 0) {
    for (int w = 0; w < kWarps; ++w)
      for (int i = 0; i < S; ++i) mbar_init(smem_u32(&s_full[w][i]), 1u);
    for (int i = 0; i < kXStages; ++i) {
      mbar_init(smem_u32(&s_xfull[i]), 1u);
      mbar_init(smem_u32(&s_xempty[i]), kWarps);
    }
    fence_mbar_init();
    s_abort = 0;
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  float acc[R][NT][4];
#pragma unroll
  for (int j = 0; j < R; ++j)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[j][n][0] = acc[j][n][1] = acc[j][n][2] = acc[j][n][3] = 0.f;
  bool ok = true;
  if (warp == kWarps) {
    // x: 256 columns of every token a stage
    const int stages = (count + kXTiles - 1) / kXTiles;
    int s = 0;
    for (; s < stages; ++s) {
      const int st = s % kXStages;
      if (!(ok = mbar_wait_warp(smem_u32(&s_xempty[st]), ((s / kXStages) & 1u) ^ 1u, a.err, &s_abort, kErrTimeoutEmpty, limit))) break;
      const int k0 = (t0 + s * kXTiles) * kTileK, cols = min((t0 + min(count, (s + 1) * kXTiles)) * kTileK, a.K) - k0;
      const int pad = min(kXTiles, count - s * kXTiles) * kTileK - cols;  // columns past K: zeros
      const uint32_t dst = xring + st * C::kTokens * kXPitch, bar = smem_u32(&s_xfull[st]);
      for (int e = lane; e < tokens * (pad >> 3); e += 32)
        sts_u4(dst + (e / (pad >> 3)) * kXPitch + (cols + e % (pad >> 3) * 8) * 2, make_uint4(0u, 0u, 0u, 0u));
      __syncwarp();
      if (lane == 0) mbar_arrive_expect_tx(bar, (uint32_t)(tokens * cols * 2));
      __syncwarp();
      for (int t = lane; t < tokens; t += 32) bulk_load(dst + t * kXPitch, a.x + (int64_t)(tok0 + t) * a.K + k0, (uint32_t)cols * 2u, bar);
    }
    // after a timeout: no copy is in flight into shared memory that is given back
    if (!ok)
      for (int i = s > kXStages ? s - kXStages : 0; i < s; ++i) mbar_drain(smem_u32(&s_xfull[i % kXStages]), (i / kXStages) & 1u, limit);
  } else {
    const int mine = min(R, a.row_tiles - rt0);  // tiles of rows that there are; none: 0 or less
    int issued = 0;
    auto fill = [&](int t) {  // by lane 0
      const uint32_t dst = ring + (t % S) * R * tile, bar = smem_u32(&s_full[warp][t % S]);
      mbar_arrive_expect_tx(bar, (uint32_t)(mine * tile));
      for (int j = 0; j < mine; ++j) bulk_load(dst + j * tile, a.w + ((int64_t)(rt0 + j) * a.tiles + t0 + t) * tile, (uint32_t)tile, bar);
    };
    if (mine > 0) {
      issued = min(S, count);
      if (lane == 0)
        for (int t = 0; t < issued; ++t) fill(t);
      __syncwarp();
    }
    int t = 0;
    for (; t < count; ++t) {
      const int xs = t / kXTiles, xst = xs % kXStages;
      if (t % kXTiles == 0 && !(ok = mbar_wait_warp(smem_u32(&s_xfull[xst]), (xs / kXStages) & 1u, a.err, &s_abort, kErrTimeoutFull, limit))) break;
      if (mine > 0) {
        if (!(ok = mbar_wait_warp(smem_u32(&s_full[warp][t % S]), (t / S) & 1u, a.err, &s_abort, kErrTimeoutFull, limit))) break;
        const uint32_t st = ring + (t % S) * R * tile;
        const uint32_t xrow = xring + xst * C::kTokens * kXPitch + g * kXPitch + (t % kXTiles) * kTileK * 2 + tq * 16;
        uint32_t code[R][2][4];
#pragma unroll
        for (int j = 0; j < R; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint4 v = lds_u4(st + j * tile + h * 512 + lane * 16);
            code[j][h][0] = v.x; code[j][h][1] = v.y; code[j][h][2] = v.z; code[j][h][3] = v.w;
          }
#pragma unroll
        for (int gi = 0; gi < GROUPS; ++gi) {
          float part[R][NT][4];
          uint32_t zero[R][2];
#pragma unroll
          for (int j = 0; j < R; ++j) {
#pragma unroll
            for (int n = 0; n < NT; ++n) part[j][n][0] = part[j][n][1] = part[j][n][2] = part[j][n][3] = 0.f;
#pragma unroll
            for (int h = 0; h < 2; ++h)
              zero[j][h] = a.zeros ? 0x43004300u + lds_u8(st + j * tile + 1024 + GROUPS * 32 + gi * 16 + h * 8 + g) * 0x00010001u : 0x43084308u;
          }
#pragma unroll
          for (int i = gi * 4 / GROUPS; i < (gi + 1) * 4 / GROUPS; ++i) {
            uint32_t fr[R][2][4];
#pragma unroll
            for (int j = 0; j < R; ++j)
#pragma unroll
              for (int m = 0; m < 4; ++m) {
                fr[j][m >> 1][(m & 1) * 2] = pair_of(code[j][0][i], m, zero[j][0]);
                fr[j][m >> 1][(m & 1) * 2 + 1] = pair_of(code[j][1][i], m, zero[j][1]);
              }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const uint4 b = lds_u4(xrow + n * 8 * kXPitch + i * 64);
#pragma unroll
              for (int j = 0; j < R; ++j) {
                mma16816(part[j][n], fr[j][0], b.x, b.y);
                mma16816(part[j][n], fr[j][1], b.z, b.w);
              }
            }
          }
#pragma unroll
          for (int j = 0; j < R; ++j) {
            const uint32_t at = st + j * tile + 1024 + gi * 32 + g * 2;
            const float s0 = __uint_as_float(lds_u16(at) << 16), s1 = __uint_as_float(lds_u16(at + 16) << 16);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              acc[j][n][0] = fmaf(s0, part[j][n][0], acc[j][n][0]);
              acc[j][n][1] = fmaf(s0, part[j][n][1], acc[j][n][1]);
              acc[j][n][2] = fmaf(s1, part[j][n][2], acc[j][n][2]);
              acc[j][n][3] = fmaf(s1, part[j][n][3], acc[j][n][3]);
            }
          }
        }
        __syncwarp();  // the stage may be filled again
        if (t + S < count) {
          if (lane == 0) fill(t + S);
          issued = t + S + 1;
        }
      }
      __syncwarp();
      if (lane == 0 && (t % kXTiles == kXTiles - 1 || t + 1 == count)) mbar_arrive(smem_u32(&s_xempty[xst]));
    }
    if (!ok)
      for (int i = t; i < issued; ++i) mbar_drain(smem_u32(&s_full[warp][i % S]), (i / S) & 1u, limit);
  }
  // the CTA's sums [tokens][rows], over the rings (every copy has arrived)
  __syncthreads();
  if (warp < kWarps) {
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = (warp * R + j) * 16 + g + (e >> 1) * 8, token = n * 8 + 2 * tq + (e & 1);
          asm volatile("st.shared.f32 [%0], %1;" ::"r"(base + (token * C::kPitch + row) * 4), "f"(acc[j][n][e]) : "memory");
        }
  }
  // every CTA of the cluster adds up its share of the rows, in the order of the columns
  cluster_arrive();
  cluster_wait();
  const int share = C::kRows / a.split, pieces = share / 8;
  if (!*(volatile int*)&s_abort) {
    for (int e = threadIdx.x; e < tokens * pieces; e += kThreads) {
      const int token = e / pieces, row = rank * share + e % pieces * 8, n = block * C::kRows + row;
      if (n >= a.N) continue;
      float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      for (int q = 0; q < a.split; ++q) {
        const uint32_t from = cluster_map(base + (token * C::kPitch + row) * 4, q);
        const float4 p = ld_cluster_f4(from), r = ld_cluster_f4(from + 16);
        v[0] += p.x; v[1] += p.y; v[2] += p.z; v[3] += p.w;
        v[4] += r.x; v[5] += r.y; v[6] += r.z; v[7] += r.w;
      }
      const int64_t at = (int64_t)(tok0 + token) * a.N + n;
      float res[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (a.ep.residual) unpack8(*reinterpret_cast<const uint4*>(a.ep.residual + at), res);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float scale, shift;
        epi_affine(a.ep, a.N, n + k, scale, shift);
        v[k] = epi_act(fmaf(v[k], scale, shift) + res[k], a.ep.act);
      }
      if (a.y_f32) {
        float4* to = reinterpret_cast<float4*>(static_cast<float*>(a.y) + at);
        to[0] = make_float4(v[0], v[1], v[2], v[3]);
        to[1] = make_float4(v[4], v[5], v[6], v[7]);
      } else {
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.y) + at) = pack8(v);
      }
    }
  }
  cluster_arrive();  // the sums are read until here
  cluster_wait();
}

// A CTA a tile: its codes in the order of the lanes (row g of the tile's first or second
// half, columns 32 i + 8 tq onwards, whose pairs lie 16 bits apart), scales, zeros.
__global__ void __launch_bounds__(256) w4_pack_kernel(const __grid_constant__ W4PackArgs a) {
  pdl_wait();
  pdl_trigger();
  const int groups = kTileK / a.group, tiles = (a.K + kTileK - 1) / kTileK, tile = tile_bytes(groups, a.zeros != nullptr);
  const int rt = (int)(blockIdx.x / tiles), tk = (int)(blockIdx.x % tiles), all = a.K / a.group;
  uint8_t* out = a.out + (int64_t)blockIdx.x * tile;
  const int t = threadIdx.x, lane = (t >> 2) & 31;
  const int row = rt * 16 + (t >> 7) * 8 + (lane >> 2), k = tk * kTileK + 32 * (t & 3) + 8 * (lane & 3);
  uint32_t word = 0u;
  if (row < a.N && k < a.K) {
    const uint32_t v = *reinterpret_cast<const uint32_t*>(a.codes + (int64_t)row * (a.K / 2) + k / 2);
#pragma unroll
    for (int e = 0; e < 8; ++e) word |= ((v >> (4 * e)) & 15u) << (4 * ((e >> 1) + 4 * (e & 1)));
  }
  reinterpret_cast<uint32_t*>(out)[t] = word;
  if (t < groups * 16) {
    const int n = rt * 16 + (t & 15), gi = tk * groups + (t >> 4);
    const bool there = n < a.N && gi < all;
    reinterpret_cast<uint16_t*>(out + 1024)[t] = there ? a.scales[(int64_t)n * all + gi] : (uint16_t)0;
    if (a.zeros) out[1024 + groups * 32 + t] = there ? (uint8_t)(a.zeros[(int64_t)n * all + gi] & 15) : (uint8_t)0;
  }
}

template <int GROUPS, int R, int NT>
cudaError_t launch_w4_t(W4Args a, cudaStream_t s) {
  using C = Cfg<R, NT>;
  const int blocks = (a.row_tiles + kWarps * R - 1) / (kWarps * R), toks = (a.M + C::kTokens - 1) / C::kTokens;
  // columns split over a cluster until every SM has two CTAs
  const int64_t want = 2ll * device_sm_count();
  a.split = 1;
  while (a.split < 8 && (int64_t)blocks * toks * a.split < want && a.tiles >= 4 * a.split) a.split *= 2;
  const size_t smem = C::smem(tile_bytes(GROUPS, a.zeros));
  const cudaError_t e = smem_optin(reinterpret_cast<const void*>(w4_kernel<GROUPS, R, NT>), smem);
  if (e != cudaSuccess) return e;
  return launch_cluster_kernel(w4_kernel<GROUPS, R, NT>, dim3((unsigned)(blocks * a.split), (unsigned)toks), dim3(kThreads),
                               (unsigned)a.split, smem, s, a);
}

template <int GROUPS>
cudaError_t launch_w4_g(const W4Args& a, cudaStream_t s) {
  if (a.M <= 8) return launch_w4_t<GROUPS, 1, 1>(a, s);
  if (a.M <= 16) return launch_w4_t<GROUPS, 1, 2>(a, s);
  if (a.M <= 32) return launch_w4_t<GROUPS, 2, 4>(a, s);
  return launch_w4_t<GROUPS, 2, 8>(a, s);
}

}  // namespace

uint64_t w4_packed_bytes(int64_t N, int64_t K, int group, bool zeros) {
  return (uint64_t)((N + 15) / 16) * (uint64_t)((K + kTileK - 1) / kTileK) * (uint64_t)tile_bytes(kTileK / group, zeros);
}

cudaError_t launch_w4_pack(const W4PackArgs& a, cudaStream_t s) {
  const int64_t tiles = (int64_t)((a.N + 15) / 16) * ((a.K + kTileK - 1) / kTileK);
  return launch_kernel(w4_pack_kernel, dim3((unsigned)tiles), dim3(256), 0, s, a);
}

cudaError_t launch_w4(W4Args a, cudaStream_t s) {
  a.row_tiles = (a.N + 15) / 16;
  a.tiles = (a.K + kTileK - 1) / kTileK;
  if (a.group == 128) return launch_w4_g<1>(a, s);
  if (a.group == 64) return launch_w4_g<2>(a, s);
  return launch_w4_g<4>(a, s);
}

}  // namespace sparoa
