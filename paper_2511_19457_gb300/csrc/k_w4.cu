// Products of a few tokens' rows with weights of 4 bits: y = epilogue(x W^T),
// W[n][k] = scale[n][k / group] (code[n][k] - zero[n][k / group]).
//
// Bound by the bytes of the weights, half a byte each and read once, and nearly as much by the instructions
// that make numbers of the codes (11 for 8 codes, 2 cycles each).  A CTA has 64, 96 or 128 rows of W over
// its share of the columns, 16 a warp, as they fill the GPU best (w4_split); a warp's teammate has the same
// rows of every other tile of columns.  The rows' tiles of two tiles of columns come in one copy (w4.cuh; a
// copy each took 44 cycles more of the copy unit, and there would be sixteen), kStages of them on their way,
// with x beside them by TMA.  A code becomes the bf16 number 128 + code by one logic operation, 128 + zero is
// taken away, which is exact, and mma.sync m16n8k16 sums the products with x in fp32 over a group; only that
// sum is multiplied by the scale.  So nothing is rounded before the result but fp32 sums.
//
// 16 tokens x 4096 columns x 14336 rows, groups of 128, from memory: 14.0 us, 2.2 TB/s.  The copies alone
// (no product, no numbers made of codes) 10.5, without the numbers of codes 13: a third of it is a launch, the
// first bytes' way and the cluster's sum (4.5 us for 2048 x 2048), and the rest waits on issue slots (46 %
// busy) and the logic pipe (47 %).  Tried: weights straight from memory to registers,
// without copies (slower), 24 warps of three teams (slower), shifts as multiplications (slower), the weights
// into the L2 before the kernel before ends (16.4), no teams (24.6).
#include "w4.cuh"

namespace sparoa {

namespace {

constexpr int kTileK = kW4TileK;
constexpr int kWarps = 8;                             // of 16 rows each, a team: every other tile of columns
constexpr int kTeams = 2;
constexpr int kThreads = 32 * (kTeams * kWarps + 2);  // and a warp that loads codes, one that loads x
constexpr int kPitch = 16 * kWarps + 4;      // floats of a token's sums
constexpr int kStages = 4;                   // of kTeams tiles of columns, on their way

template <int NT>
struct Cfg {
  static constexpr int kTokens = 8 * NT;
  static constexpr int kHalf = kTokens * 128;  // 64 columns of x
  static size_t smem(int tile) { return (size_t)kStages * kTeams * (2 * kHalf + 8 * tile) + 1024; }
};

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// the same onto zero
__device__ __forceinline__ void mma16816_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
// GROUPS: of a tile's columns (128 / group).  Column g of a fragment is token g / 2 + g % 2 * 4 of its
// eight: lanes side by side then read different banks of x in its 128-byte swizzle.
template <int GROUPS, int NT>
__global__ void __launch_bounds__(kThreads, 1) w4_kernel(const __grid_constant__ CUtensorMap tx, const __grid_constant__ W4Args a) {
  using C = Cfg<NT>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) unsigned long long s_full[kStages], s_empty[kStages];
  __shared__ int s_abort;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, tq = lane & 3;
  const int tile = w4_tile_bytes(GROUPS, a.zeros);
  const uint32_t xring = (smem_u32(smem_raw) + 1023u) & ~1023u, ring = xring + kStages * kTeams * 2 * C::kHalf;
  const int rank = (int)(blockIdx.x % a.split), block = (int)(blockIdx.x / a.split), tok0 = blockIdx.y * C::kTokens;
  const int tokens = min(C::kTokens, a.M - tok0);
  const int t0 = (int)((int64_t)rank * a.tiles / a.split), count = (int)((int64_t)(rank + 1) * a.tiles / a.split) - t0;
  // (as many warps as there are tiles of rows, the teams' one after the other: a scheduler has every
  // fourth warp)
  const int team = warp / a.block_tiles, mine = warp % a.block_tiles;
  constexpr int kLoadWarp = kTeams * kWarps;
  const int first = block * a.block_tiles, rows = min(a.block_tiles, a.row_tiles - first);  // the CTA's tiles of rows
  const long long limit = a.wait_limit ? a.wait_limit : kWaitLimitCycles;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(smem_u32(&s_full[i]), 2u);
      mbar_init(smem_u32(&s_empty[i]), (uint32_t)(kTeams * rows));
    }
    fence_mbar_init();
    s_abort = 0;
    prefetch_tmap(&tx);
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  float acc[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f;
  const int stages = (count + kTeams - 1) / kTeams;
  const int in_block = first % 8 ? 0 : min(8, a.row_tiles - first);  // of the layout's block from there
  if (warp >= kLoadWarp) {
    // A copy takes 200 cycles and more to give out, so there are as few as can be, by two warps: one has the
    // first tile's codes (all tiles', where they lie side by side), the other x and the second tile's.  One
    // lane of each, asleep while it waits.
    if (lane == 0) {
      const bool whole = rows == in_block, codes = warp == kLoadWarp;
      const int head = min(rows, 8 - first % 8);  // rows up to the layout's next block
      const uint32_t head_bytes = (uint32_t)(head * tile), tail_bytes = (uint32_t)((rows - head) * tile);
      const int64_t step = (int64_t)min(8, a.row_tiles - first / 8 * 8) * tile, step2 = (int64_t)min(8, a.row_tiles - first - head) * tile;
      const uint8_t* from = a.w + w4_tile_at(first, t0, a.row_tiles, a.tiles) * tile;
      const uint8_t* from2 = head < rows ? a.w + w4_tile_at(first + head, t0, a.row_tiles, a.tiles) * tile : from;
      int s = 0;
      for (; s < stages; ++s, from += kTeams * step, from2 += kTeams * step2) {
        const int st = s % kStages, t = s * kTeams, there = min(kTeams, count - t);
        if (!mbar_wait(smem_u32(&s_empty[st]), (s / kStages + 1) & 1u, a.err, &s_abort, kErrTimeoutEmpty, limit)) break;
        const uint32_t bar = smem_u32(&s_full[st]), to = ring + st * kTeams * kWarps * tile;
        auto tile_codes = [&](int i) {
          bulk_load(to + i * rows * tile, from + i * step, head_bytes, bar);
          if (tail_bytes) bulk_load(to + i * rows * tile + head_bytes, from2 + i * step2, tail_bytes, bar);
        };
        if (codes) {
          const uint32_t bytes = (uint32_t)((whole ? there : 1) * rows * tile);
          mbar_arrive_expect_tx(bar, bytes);
          if (whole)
            bulk_load(to, from, bytes, bar);
          else
            tile_codes(0);
        } else {
          const bool second = !whole && there > 1;
          const int boxes = a.x_boxed ? 2 * kTeams : 2 * there;  // of 64 columns
          mbar_arrive_expect_tx(bar, (uint32_t)(boxes * C::kHalf + (second ? rows * tile : 0)));
          const uint32_t xto = xring + st * kTeams * 2 * C::kHalf;
          if (a.x_boxed)
            tma_load_3d(xto, &tx, bar, 0, tok0, 2 * (t0 + t));
          else
            for (int i = 0; i < boxes; ++i) tma_load_2d(xto + i * C::kHalf, &tx, bar, (t0 + t) * kTileK + i * 64, tok0);
          if (second) tile_codes(1);
        }
      }
      // no copy is in flight into shared memory that is given back, whichever wait of the CTA ran out and
      // when (where the other warp gave out none, this waits its limit)
      for (int i = s > kStages ? s - kStages : 0; i < s; ++i) mbar_drain(smem_u32(&s_full[i % kStages]), (i / kStages) & 1u, limit);
    }
    __syncwarp();
  } else if (team < kTeams && mine < rows) {
    // byte of the lane's 16 of x in columns 0 to 31 of 64 (64 further, by the swizzle, in the others), and of
    // its piece of row g
    const uint32_t token = (g >> 1) + (g & 1) * 4, x_at = swz_offset<64>(token, tq), w_at = w4_piece(g, tq);
    for (int s = 0; s < stages; ++s) {
      const int st = s % kStages;
      if (!mbar_wait_warp(smem_u32(&s_full[st]), (s / kStages) & 1u, a.err, &s_abort, kErrTimeoutFull, limit)) break;
      if (s * kTeams + team < count) {  // (but for the last stage's other tiles)
        const uint32_t x = xring + (st * kTeams + team) * 2 * C::kHalf + x_at, x_odd = x ^ 64u;
        const uint32_t w = ring + (st * kTeams * kWarps + team * rows + mine) * tile;
        const uint32_t meta = w + 1024 + g * 2;
        const uint4 c0 = lds_u4(w + w_at), c1 = lds_u4(w + w_at + 512);
#pragma unroll
        for (int gi = 0; gi < GROUPS; ++gi) {
          float part[NT][4];
          uint32_t z0 = 8u, z1 = 8u;
          if (a.zeros) {
            z0 = lds_u8(w + 1024 + GROUPS * 32 + gi * 16 + g);
            z1 = lds_u8(w + 1024 + GROUPS * 32 + gi * 16 + g + 8);
          }
          z0 = w4_zero_pair(z0);
          z1 = w4_zero_pair(z1);
#pragma unroll
          for (int j = gi * 4 / GROUPS; j < (gi + 1) * 4 / GROUPS; ++j) {
            const uint32_t w0 = j == 0 ? c0.x : j == 1 ? c0.y : j == 2 ? c0.z : c0.w, w1 = j == 0 ? c1.x : j == 1 ? c1.y : j == 2 ? c1.z : c1.w;
            const uint32_t f0[4] = {w4_pair(w0, 0, z0), w4_pair(w1, 0, z1), w4_pair(w0, 1, z0), w4_pair(w1, 1, z1)};
            const uint32_t f1[4] = {w4_pair(w0, 2, z0), w4_pair(w1, 2, z1), w4_pair(w0, 3, z0), w4_pair(w1, 3, z1)};
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const uint4 v = lds_u4((j & 1 ? x_odd : x) + (j >> 1) * C::kHalf + n * 1024);
              if (j == gi * 4 / GROUPS)
                mma16816_first(part[n], f0, v.x, v.y);
              else
                mma16816(part[n], f0, v.x, v.y);
              mma16816(part[n], f1, v.z, v.w);
            }
          }
          const float s0 = __uint_as_float(lds_u16(meta + gi * 32) << 16), s1 = __uint_as_float(lds_u16(meta + gi * 32 + 16) << 16);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            acc[n][0] = fmaf(s0, part[n][0], acc[n][0]);
            acc[n][1] = fmaf(s0, part[n][1], acc[n][1]);
            acc[n][2] = fmaf(s1, part[n][2], acc[n][2]);
            acc[n][3] = fmaf(s1, part[n][3], acc[n][3]);
          }
        }
      }
      __syncwarp();
      if (lane == 0 && !a.fault) mbar_arrive(smem_u32(&s_empty[st]));
    }
  }
  // the CTA's sums [tokens][rows], where x was (every copy has arrived)
  __syncthreads();
  if (warp < kLoadWarp && team < kTeams && mine < rows) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int col = 2 * tq + (e & 1), row = mine * 16 + g + (e >> 1) * 8, token = n * 8 + (col >> 1) + (col & 1) * 4;
        asm volatile("st.shared.f32 [%0], %1;" ::"r"(xring + ((team * C::kTokens + token) * kPitch + row) * 4), "f"(acc[n][e]) : "memory");
      }
  }
  cluster_arrive();
  cluster_wait();
  if (!*(volatile int*)&s_abort) w4_finish(a, xring, kPitch, 16 * a.block_tiles, block, rank, tok0, tokens, kTeams, C::kTokens);
  cluster_arrive();  // the sums are read until here
  cluster_wait();
}

// A CTA a tile (w4.cuh).
__global__ void __launch_bounds__(256) w4_pack_kernel(const __grid_constant__ W4PackArgs a) {
  pdl_wait();
  pdl_trigger();
  const int groups = kTileK / a.group, tiles = (a.K + kTileK - 1) / kTileK, tile = w4_tile_bytes(groups, a.zeros != nullptr);
  const int rt = (int)(blockIdx.x / tiles), tk = (int)(blockIdx.x % tiles), all = a.K / a.group;
  uint8_t* out = a.out + w4_tile_at(rt, tk, (a.N + 15) / 16, tiles) * tile;
  const int t = threadIdx.x, r = t >> 4, q = (t >> 2) & 3, i = t & 3;
  const int row = rt * 16 + r, k = tk * kTileK + 32 * i + 8 * q;
  uint32_t word = 0u;
  if (row < a.N && k < a.K) {
    const uint32_t v = *reinterpret_cast<const uint32_t*>(a.codes + (int64_t)row * (a.K / 2) + k / 2);
#pragma unroll
    for (int e = 0; e < 8; ++e) word |= ((v >> (4 * e)) & 15u) << (4 * ((e >> 1) + 4 * (e & 1)));
  }
  *reinterpret_cast<uint32_t*>(out + w4_piece(r, q) + 4 * i) = word;
  if (t < groups * 16) {
    const int n = rt * 16 + (t & 15), gi = tk * groups + (t >> 4);
    const bool there = n < a.N && gi < all;
    reinterpret_cast<uint16_t*>(out + 1024)[t] = there ? a.scales[(int64_t)n * all + gi] : (uint16_t)0;
    if (a.zeros) out[1024 + groups * 32 + t] = there ? (uint8_t)(a.zeros[(int64_t)n * all + gi] & 15) : (uint8_t)0;
  }
}

template <int GROUPS, int NT>
cudaError_t launch_w4_t(W4Args a, cudaStream_t s) {
  using C = Cfg<NT>;
  const auto kernel = w4_kernel<GROUPS, NT>;
  static_assert(kTeams * C::kTokens * kPitch * 4 <= kStages * (2 * C::kHalf + 8 * 1024), "sums over the rings");
  const size_t smem = C::smem(w4_tile_bytes(GROUPS, true));
  const cudaError_t e = smem_optin(reinterpret_cast<const void*>(kernel), smem);
  if (e != cudaSuccess) return e;
  CUtensorMap tx;
  if (!w4_x_map(&tx, &a, C::kTokens, 2 * kTeams)) return cudaErrorInvalidValue;
  // (rows that fill the GPU: 896 tiles of rows as 150 blocks of 6 instead of 112 of 8)
  const int toks = (a.M + C::kTokens - 1) / C::kTokens;
  W4Split best;
  for (const int rows : {8, 6, 4}) {
    const int64_t blocks = (int64_t)((a.row_tiles + rows - 1) / rows) * toks;
    const W4Split s = w4_split(kernel, blocks, a.tiles, rows, kThreads, smem);
    if (s.time < best.time) {
      best = s;
      a.block_tiles = rows;
    }
  }
  a.split = best.split;
  const int blocks = (a.row_tiles + a.block_tiles - 1) / a.block_tiles;
  return launch_cluster_kernel(kernel, dim3((unsigned)(blocks * a.split), (unsigned)toks), dim3(kThreads), (unsigned)a.split, smem, s, tx, a);
}

template <int GROUPS>
cudaError_t launch_w4_g(const W4Args& a, cudaStream_t s) {
  return a.M <= 8 ? launch_w4_t<GROUPS, 1>(a, s) : launch_w4_t<GROUPS, 2>(a, s);
}

}  // namespace

uint64_t w4_packed_bytes(int64_t N, int64_t K, int group, bool zeros) {
  return (uint64_t)((N + 15) / 16) * (uint64_t)((K + kTileK - 1) / kTileK) * (uint64_t)w4_tile_bytes(kTileK / group, zeros);
}

cudaError_t launch_w4_pack(const W4PackArgs& a, cudaStream_t s) {
  const int64_t tiles = (int64_t)((a.N + 15) / 16) * ((a.K + kTileK - 1) / kTileK);
  return launch_kernel(w4_pack_kernel, dim3((unsigned)tiles), dim3(256), 0, s, a);
}

bool w4_x_map(CUtensorMap* m, W4Args* a, int tokens, int halves) {
  a->x_boxed = a->K % 64 == 0;
  if (!a->x_boxed) return make_tmap_2d(m, a->x, (uint64_t)a->M, (uint64_t)a->K, 64, (uint32_t)tokens);
  return make_tmap_3d(m, a->x, 64, (uint64_t)a->M, (uint64_t)(a->K / 64), (uint64_t)a->K, 64, 64, (uint32_t)tokens, (uint32_t)halves);
}

cudaError_t launch_w4(W4Args a, cudaStream_t s) {
  a.row_tiles = (a.N + 15) / 16;
  a.tiles = (a.K + kTileK - 1) / kTileK;
  // up to 16 tokens as columns of mma.sync: 16 tokens x 4096 x 14336 14.0 us, on tcgen05 17.8; x 14336 x 4096
  // 15.8 and 16.2, x 2048 x 2048 5.2 and 5.9, in groups of 32 x 4096 x 14336 15.2 and 22.9; but 24 tokens 18.9
  // and 15.1, 64 38.5 and 17.1
  if (a.M > 16) return launch_w4_tc(a, s);
  if (a.group == 128) return launch_w4_g<1>(a, s);
  return a.group == 64 ? launch_w4_g<2>(a, s) : launch_w4_g<4>(a, s);
}

}  // namespace sparoa
