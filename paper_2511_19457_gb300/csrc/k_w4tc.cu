// Products with 4-bit weights on tcgen05, for more tokens than mma.sync takes in time.
//
// A CTA has 128 rows of W and up to 64 tokens, or 128 where there are more (launch_g).  Eight warps, in two groups that take turns, make bf16 whole
// numbers of a tile of columns' codes (a thread a row) and put them into tensor memory, where they are the A
// operand; x is the B operand, by TMA in shared memory.  Another four take each group's sums out of tensor
// memory, and multiply and add them in fp32 in registers (a thread a row).  Codes less zeros are exact, and
// only the fp32 sums of a group are multiplied by its scale: nothing is rounded but fp32 sums.
//
// Bound by the bytes of the weights, read once for 64 tokens; beside them x comes from the L2 for every
// block of rows.  61 tokens x 14336 columns x 4096 rows, groups of 128, from memory: 17.0 us.  Its products
// with A from tensor memory take 64 to 70 cycles each, whatever the number of tokens: 600 a tile of
// 128 x 128, 28 tiles a CTA in clusters of 4, 9 us; the rest is the start, the first tile and the cluster's
// sum.  On mma.sync the products alone cannot take less than 12.6 us (0.5 an SM and cycle), and with the codes'
// instructions beside them took 38.5.  Tried: two CTAs an SM with half the tensor memory each (20.2), two
// warps that issue products (no faster), the weights into the L2 before the kernel before ends (18.2).
#include "w4.cuh"

namespace sparoa {

namespace {

constexpr int kTileK = kW4TileK;
constexpr int kRows = 128;
constexpr int kBufs = 4;  // of A in tensor memory
constexpr int kCodeWarps = 8;
constexpr int kPitch = kRows + 4;  // floats of a token's sums
constexpr uint32_t kCols = 512, kA = 256;

template <int NTOK>
struct Cfg {
  static constexpr int kStages = NTOK > 64 ? 4 : 8;      // tiles of columns on their way
  static constexpr int kSums = NTOK > 64 ? 2 : kBufs;    // of sums in tensor memory
  static constexpr int kSumWarps = NTOK > 64 ? 8 : 4;    // four for 64 tokens
  static constexpr int kLoadWarp = kCodeWarps + kSumWarps, kXWarp = kLoadWarp + 1, kMmaWarp = kLoadWarp + 2;
  static constexpr int kThreads = 32 * (kMmaWarp + 1);
  static constexpr int kHalf = NTOK * 128;  // 64 columns of x
  static size_t smem(int tile) { return (size_t)kStages * (2 * kHalf + 8 * tile) + 1024; }
};

template <int NTOK>
struct Bars {
  unsigned long long full[Cfg<NTOK>::kStages], empty[Cfg<NTOK>::kStages];  // codes and x
  unsigned long long a[kBufs], a_free[kBufs], d[Cfg<NTOK>::kSums], d_free[Cfg<NTOK>::kSums], drain;
};

__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t bd, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(bd), "r"(idesc), "r"(acc));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0],"
      " {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

// GROUPS: of a tile's columns (128 / group)
template <int GROUPS, int NTOK>
__global__ void __launch_bounds__(Cfg<NTOK>::kThreads, 1) w4_tc_kernel(const __grid_constant__ CUtensorMap tx, const __grid_constant__ W4Args a) {
  using C = Cfg<NTOK>;
  constexpr int kStages = C::kStages, kSums = C::kSums, kSumWarps = C::kSumWarps, kLoadWarp = C::kLoadWarp, kXWarp = C::kXWarp, kMmaWarp = C::kMmaWarp;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) Bars<NTOK> bars;
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int tile = w4_tile_bytes(GROUPS, a.zeros);
  const uint32_t xring = (smem_u32(smem_raw) + 1023u) & ~1023u, ring = xring + kStages * 2 * C::kHalf;
  const int rank = (int)(blockIdx.x % a.split), block = (int)(blockIdx.x / a.split), tok0 = blockIdx.y * NTOK;
  const int tokens = min(NTOK, a.M - tok0);
  const int t0 = (int)((int64_t)rank * a.tiles / a.split), count = (int)((int64_t)(rank + 1) * a.tiles / a.split) - t0;
  const long long limit = a.wait_limit ? a.wait_limit : kWaitLimitCycles;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(smem_u32(&bars.full[i]), 2u);
      mbar_init(smem_u32(&bars.empty[i]), kCodeWarps / 2 + kSumWarps);
    }
    for (int i = 0; i < kBufs; ++i) {
      mbar_init(smem_u32(&bars.a[i]), kCodeWarps / 2);
      mbar_init(smem_u32(&bars.a_free[i]), 1u);
    }
    for (int i = 0; i < kSums; ++i) {
      mbar_init(smem_u32(&bars.d[i]), 1u);
      mbar_init(smem_u32(&bars.d_free[i]), kSumWarps);
    }
    mbar_init(smem_u32(&bars.drain), 1u);
    fence_mbar_init();
    s_abort = 0;
    prefetch_tmap(&tx);
  }
  if (warp == kMmaWarp) tmem_alloc(smem_u32(&s_tmem), kCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_wait();
  pdl_trigger();
  const uint32_t tmem = s_tmem, lanes = (uint32_t)(warp & 3) << 21;  // the warp's 32 lanes of tensor memory
  // waits for up to three barriers at once: asked for one after the other they cost a warp 90 cycles each
  // when they are there already
  auto wait = [&](uint32_t bit, unsigned long long& b0, unsigned p0, unsigned long long& b1, unsigned p1, unsigned long long& b2,
                  unsigned p2) {
    const uint32_t x = smem_u32(&b0), y = smem_u32(&b1), z = smem_u32(&b2);
    const bool there = (int)mbar_try_wait(x, p0 & 1u) & (int)mbar_try_wait(y, p1 & 1u) & (int)mbar_try_wait(z, p2 & 1u);
    if (__all_sync(0xffffffffu, there)) return true;
    return mbar_wait_warp(x, p0 & 1u, a.err, &s_abort, bit, limit) && mbar_wait_warp(y, p1 & 1u, a.err, &s_abort, bit, limit) &&
           mbar_wait_warp(z, p2 & 1u, a.err, &s_abort, bit, limit);
  };
  auto wait2 = [&](uint32_t bit, unsigned long long& b0, unsigned p0, unsigned long long& b1, unsigned p1) {
    const uint32_t x = smem_u32(&b0), y = smem_u32(&b1);
    const bool there = (int)mbar_try_wait(x, p0 & 1u) & (int)mbar_try_wait(y, p1 & 1u);
    if (__all_sync(0xffffffffu, there)) return true;
    return mbar_wait_warp(x, p0 & 1u, a.err, &s_abort, bit, limit) && mbar_wait_warp(y, p1 & 1u, a.err, &s_abort, bit, limit);
  };
  auto arrive = [&](unsigned long long& bar) {
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&bar));
  };
  if (warp < kCodeWarps) {
    // every other tile, a row a thread
    const int row = threadIdx.x & 127;
    for (int t = warp >> 2; t < count; t += 2) {
      const int st = t % kStages;
      if (!wait2(kErrTimeoutFull, bars.full[st], t / kStages, bars.a_free[t % kBufs], t / kBufs + 1)) break;
      tc_fence_after();
      const uint32_t from = ring + (st * 8 + (row >> 4)) * tile;
      uint4 piece[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) piece[q] = lds_u4(from + w4_piece(row & 15, q));
#pragma unroll
      for (int gi = 0; gi < GROUPS; ++gi) {
        const uint32_t zero = w4_zero_pair(a.zeros ? lds_u8(from + 1024 + GROUPS * 32 + gi * 16 + (row & 15)) : 8u);
#pragma unroll
        for (int i = gi * 4 / GROUPS; i < (gi + 1) * 4 / GROUPS; ++i) {
          uint32_t r[16];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const uint32_t word = i == 0 ? piece[q].x : i == 1 ? piece[q].y : i == 2 ? piece[q].z : piece[q].w;
#pragma unroll
            for (int m = 0; m < 4; ++m) r[4 * q + m] = w4_pair(word, m, zero);
          }
          tmem_st16(tmem + lanes + kA + (t % kBufs) * 64 + i * 16, r);
        }
      }
      tmem_wait_st();
      tc_fence_before();
      arrive(bars.a[t % kBufs]);
      if (lane == 0) mbar_arrive(smem_u32(&bars.empty[st]));
    }
  } else if (warp < kCodeWarps + kSumWarps) {
    // a row a thread, and of 128 tokens half
    constexpr int kMine = NTOK > 64 ? 64 : NTOK, kOnce = NTOK > 64 ? 16 : 32;
    const int row = threadIdx.x & 127, col0 = kMine * ((warp - kCodeWarps) >> 2);
    f2_t acc[kMine / 2];
#pragma unroll
    for (int i = 0; i < kMine / 2; ++i) acc[i] = f2(0.f, 0.f);
    int n = 0;  // groups so far
    for (int t = 0; t < count; ++t) {
      const int st = t % kStages;
      bool ok = true;
      const uint32_t from = ring + (st * 8 + (row >> 4)) * tile + 1024 + (row & 15) * 2;
#pragma unroll(NTOK > 64 ? 1 : GROUPS)  // (four groups' registers would not do)
      for (int gi = 0; gi < GROUPS; ++gi, ++n) {
        if (!(ok = ok && wait2(kErrTimeoutAcc, bars.d[n % kSums], n / kSums, bars.full[st], t / kStages))) break;
        const float s = __uint_as_float(lds_u16(from + gi * 32) << 16);
        const f2_t scale = f2(s, s);
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < kMine; c += kOnce) {
          uint32_t v[kOnce];
          if constexpr (kOnce == 16) {
            float w[16];
            tmem_ld16(tmem + lanes + (n % kSums) * NTOK + col0 + c, w);
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = __float_as_uint(w[k]);
          } else {
            tmem_ld32_nowait(tmem + lanes + (n % kSums) * NTOK + c, v);
            tmem_wait_ld32(v);
          }
          if (c + kOnce == kMine) {
            tc_fence_before();
            arrive(bars.d_free[n % kSums]);
          }
#pragma unroll
          for (int k = 0; k < kOnce; k += 2)
            acc[(c + k) / 2] = ffma2(f2(__uint_as_float(v[k]), __uint_as_float(v[k + 1])), scale, acc[(c + k) / 2]);
        }
      }
      if (!ok) break;
      arrive(bars.empty[st]);
    }
    // the CTA's sums [tokens][rows], where x was: its last product is done
    static_assert(NTOK * kPitch * 4 <= kStages * 2 * C::kHalf, "sums over x alone");
#pragma unroll
    for (int i = 0; i < kMine / 2; ++i) {
      float x, y;
      f2_split(acc[i], x, y);
      const uint32_t to = xring + ((col0 + 2 * i) * kPitch + row) * 4;
      asm volatile("st.shared.f32 [%0], %1;" ::"r"(to), "f"(x) : "memory");
      asm volatile("st.shared.f32 [%0], %1;" ::"r"(to + kPitch * 4), "f"(y) : "memory");
    }
  } else {
    if (warp == kLoadWarp || warp == kXWarp) {
      const int mine = min(8, a.row_tiles - block * 8);  // tiles of rows that there are
      const uint32_t bytes = (uint32_t)(mine * tile);
      const uint8_t* from = a.w + w4_tile_at(block * 8, t0, a.row_tiles, a.tiles) * tile;
      if (lane == 0) {  // (asleep while it waits)
        int t = 0;
        for (; t < count; ++t, from += bytes) {
          const int st = t % kStages;
          if (!mbar_wait(smem_u32(&bars.empty[st]), (t / kStages + 1) & 1u, a.err, &s_abort, kErrTimeoutEmpty, limit)) break;
          const uint32_t bar = smem_u32(&bars.full[st]);
          if (warp == kLoadWarp) {
            mbar_arrive_expect_tx(bar, bytes);
            bulk_load(ring + st * 8 * tile, from, bytes, bar);
          } else {
            mbar_arrive_expect_tx(bar, 2u * C::kHalf);
            if (a.x_boxed) {
              tma_load_3d(xring + st * 2 * C::kHalf, &tx, bar, 0, tok0, 2 * (t0 + t));
            } else {
              tma_load_2d(xring + st * 2 * C::kHalf, &tx, bar, (t0 + t) * kTileK, tok0);
              tma_load_2d(xring + (st * 2 + 1) * C::kHalf, &tx, bar, (t0 + t) * kTileK + 64, tok0);
            }
          }
        }
        // no copy is in flight into shared memory that is given back, whichever wait of the CTA ran out and
        // when (the other warp's copies of a stage may be missing: then this waits its limit)
        for (int i = t > kStages ? t - kStages : 0; i < t; ++i) mbar_drain(smem_u32(&bars.full[i % kStages]), (i / kStages) & 1u, limit);
      }
      __syncwarp();
    } else if (warp == kMmaWarp) {
      const bool leader = elect_one();
      constexpr uint32_t id = idesc_bf16_f32(kRows, NTOK);
      int n = 0;
      bool ok = true;
      for (int t = 0; t < count && ok; ++t) {
        const int st = t % kStages;
        const uint64_t xd = smem_desc_kmajor<64>(xring + st * 2 * C::kHalf);
#pragma unroll
        for (int gi = 0; gi < GROUPS; ++gi, ++n) {
          if (!(ok = ok && wait(kErrTimeoutAcc, bars.a[t % kBufs], t / kBufs, bars.d_free[n % kSums], n / kSums + 1, bars.full[st], t / kStages))) break;
          tc_fence_after();
          if (leader) {
#pragma unroll
            for (int k = 0; k < 8 / GROUPS; ++k) {
              const int kk = gi * (8 / GROUPS) + k;
              mma_ts(tmem + (n % kSums) * NTOK, tmem + kA + (t % kBufs) * 64 + kk * 8, xd + (((kk >> 2) * C::kHalf + (kk & 3) * 32) >> 4), id, k > 0);
            }
            if (!a.fault) tc_commit(smem_u32(&bars.d[n % kSums]));
          }
          __syncwarp();
        }
        if (!ok) break;
        if (leader) tc_commit(smem_u32(&bars.a_free[t % kBufs]));
        __syncwarp();
      }
      // the MMAs end before tensor memory is given back (waits for them may run out after this warp's)
      if (leader) tc_commit(smem_u32(&bars.drain));
      __syncwarp();
      mbar_drain(smem_u32(&bars.drain), 0u, limit);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_dealloc(tmem, kCols);
  cluster_arrive();
  cluster_wait();
  if (!*(volatile int*)&s_abort) w4_finish(a, xring, kPitch, kRows, block, rank, tok0, tokens, 1, NTOK);
  cluster_arrive();  // the sums are read until here
  cluster_wait();
}

// The split of a's columns with NTOK tokens a CTA, and its time.  With 128 a tile takes half as long again
// as with 64, and beginning and end two fifths.
template <int GROUPS, int NTOK>
cudaError_t plan(const W4Args& a, W4Split* best) {
  const auto kernel = w4_tc_kernel<GROUPS, NTOK>;
  const size_t smem = Cfg<NTOK>::smem(w4_tile_bytes(GROUPS, true));
  const cudaError_t e = smem_optin(reinterpret_cast<const void*>(kernel), smem);
  if (e != cudaSuccess) return e;
  const int64_t blocks = (int64_t)((a.N + kRows - 1) / kRows) * ((a.M + NTOK - 1) / NTOK);
  *best = w4_split(kernel, blocks, a.tiles, NTOK > 64 ? 12 : 8, Cfg<NTOK>::kThreads, smem, NTOK > 64 ? 14 : kW4Start);
  return cudaSuccess;
}

template <int GROUPS, int NTOK>
cudaError_t launch_t(W4Args a, const W4Split& best, cudaStream_t s) {
  CUtensorMap tx;
  if (!w4_x_map(&tx, &a, NTOK, 2)) return cudaErrorInvalidValue;
  const int blocks = (a.N + kRows - 1) / kRows, toks = (a.M + NTOK - 1) / NTOK;
  a.split = best.split;
  return launch_cluster_kernel(w4_tc_kernel<GROUPS, NTOK>, dim3((unsigned)(blocks * a.split), (unsigned)toks), dim3(Cfg<NTOK>::kThreads),
                               (unsigned)a.split, Cfg<NTOK>::smem(w4_tile_bytes(GROUPS, true)), s, tx, a);
}

// Tokens a CTA: 32 or 64 where that is all, above it what takes less time by the plan.  4096 columns x 14336 rows,
// 128 tokens: 64 a CTA 35.6 us, 128 23.5; 256 tokens 50.7 and 46, 512 100 and 67; but 4096 x 4096, 128 tokens 11.7 and
// 12.9.
template <int GROUPS>
cudaError_t launch_g(const W4Args& a, cudaStream_t s) {
  W4Split best, wide;
  cudaError_t e = a.M <= 32 ? plan<GROUPS, 32>(a, &best) : plan<GROUPS, 64>(a, &best);
  if (e == cudaSuccess && a.M > 64) e = plan<GROUPS, 128>(a, &wide);
  if (e != cudaSuccess) return e;
  if (a.M <= 32) return launch_t<GROUPS, 32>(a, best, s);
  return wide.time < best.time ? launch_t<GROUPS, 128>(a, wide, s) : launch_t<GROUPS, 64>(a, best, s);
}

}  // namespace

cudaError_t launch_w4_tc(const W4Args& a, cudaStream_t s) {
  if (a.group == 128) return launch_g<1>(a, s);
  return a.group == 64 ? launch_g<2>(a, s) : launch_g<4>(a, s);
}

}  // namespace sparoa
