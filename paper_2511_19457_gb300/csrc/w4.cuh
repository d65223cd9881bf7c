// 4-bit weights as their kernels take them, and what the kernels share.
//
// A tile is 16 rows x 128 columns: the codes, then the bf16 scales of its 128 / group groups (16 each) and,
// with zero points, the zeros (a byte each).  Row r's 64 bytes of codes are at 64 r: four pieces of 16
// bytes, piece q at place q ^ (r / 2 % 4) (rows side by side are then in different banks), word i of it the
// columns 32 i + 8 q onwards, whose pairs lie 16 bits apart.  The (up to) eight tiles of 128 rows and the same
// columns follow one another, then those of the next columns, then the next 128 rows.
#pragma once

#include "sparoa_kernels.h"

namespace sparoa {

constexpr int kW4TileK = 128;
__host__ __device__ constexpr int w4_tile_bytes(int groups, bool zeros) { return 1024 + groups * (zeros ? 48 : 32); }
// byte of a tile at which piece q of row r's codes is
__host__ __device__ __forceinline__ int w4_piece(int r, int q) { return r * 64 + ((q ^ ((r >> 1) & 3)) << 4); }

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
// number of tile (rt, tk) of row_tiles x tiles
__host__ __device__ __forceinline__ int64_t w4_tile_at(int rt, int tk, int row_tiles, int tiles) {
  const int first = rt / 8 * 8, rows = row_tiles - first < 8 ? row_tiles - first : 8;
  return (int64_t)first * tiles + (int64_t)tk * rows + rt % 8;
}
// 128 + zero, twice
__device__ __forceinline__ uint32_t w4_zero_pair(uint32_t zero) { return 0x43004300u + zero * 0x00010001u; }
// Codes 2 m and 2 m + 1 of a word, less the zero: a pair of bf16 whole numbers, exactly (a code's bits
// are the low bits of the mantissa of 128 + code).
__device__ __forceinline__ uint32_t w4_pair(uint32_t word, int m, uint32_t zero) {
  const uint32_t v = ((word >> (4 * m)) & 0x000F000Fu) | 0x43004300u;
  const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), *reinterpret_cast<const __nv_bfloat162*>(&zero));
  return *reinterpret_cast<const uint32_t*>(&d);
}

// The sums [teams][all][pitch >= rows] that each CTA of a cluster has at `part` in its shared memory, of
// one block of rows and `tokens` <= all tokens: every CTA adds up its share of the rows, in one order,
// and finishes it.  Between two cluster barriers.
__device__ __forceinline__ void w4_finish(const W4Args& a, uint32_t part, int pitch, int rows, int block, int rank, int tok0,
                                          int tokens, int teams, int all) {
  const int share = rows / 8 / a.split * 8, begin = rank * share, pieces = (rank + 1 == a.split ? rows - begin : share) / 8;
  for (int e = threadIdx.x; e < tokens * pieces; e += blockDim.x) {
    const int token = e / pieces, row = begin + e % pieces * 8, n = block * rows + row;
    if (n >= a.N) continue;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int q = 0; q < a.split; ++q) {
      const uint32_t from = cluster_map(part + (token * pitch + row) * 4, q);
      for (int i = 0; i < teams; ++i) {
        const float4 p = ld_cluster_f4(from + i * all * pitch * 4), r = ld_cluster_f4(from + i * all * pitch * 4 + 16);
        v[0] += p.x; v[1] += p.y; v[2] += p.z; v[3] += p.w;
        v[4] += r.x; v[5] += r.y; v[6] += r.z; v[7] += r.w;
      }
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

// CTAs (a cluster) that the columns of each of `blocks` blocks are split over, by the time that the rounds
// of clusters take: a CTA's is its tiles, each of `weight` eighths, and `start` more for its beginning and
// end (kW4Start: 3 us of 0.3 each).  14336 columns, 32 blocks of 128 rows, one token: 1 CTA each 38.8 us, 2 21.4, 4 13, 8
// 24.0 (the GPU does not hold 32 clusters of 8 at once).
constexpr int kW4Start = 10;
struct W4Split {
  int split = 1;
  int64_t time = INT64_MAX;
};
template <typename... KArgs>
W4Split w4_split(void (*kernel)(KArgs...), int64_t blocks, int tiles, int weight, int threads, size_t smem, int start = kW4Start) {
  W4Split best;
  for (int s = 1; s <= 8 && s <= tiles; s *= 2) {
    const int fit = cluster_fit(reinterpret_cast<const void*>(kernel), s, threads, smem);
    if (fit <= 0) continue;
    const int64_t time = (blocks + fit - 1) / fit * ((tiles + s - 1) / s * weight + 8 * start);
    if (time < best.time) {
      best.time = time;
      best.split = s;
    }
  }
  return best;
}
// x for TMA, in boxes of `tokens` rows: of 64 columns, or where a row is whole 64s (a->x_boxed) of
// `halves` times 64 at once, which lie in shared memory as that many boxes would.
bool w4_x_map(CUtensorMap* m, W4Args* a, int tokens, int halves);
cudaError_t launch_w4_tc(const W4Args& a, cudaStream_t s);  // (k_w4tc.cu)

}  // namespace sparoa
