// Attention of chunks of new tokens over a paged key/value cache on tcgen05.
#include <cfloat>
#include <cstring>

#include "paged.cuh"

namespace sparoa {

namespace {

// ---------------------------------------------------------------------------
// An item is 256 query rows: two tiles of 128, whose scores and sums live in tensor
// memory side by side: S (128 x 128 fp32, later overwritten by the weights P in
// bf16) and O (128 x D fp32) of each.  Twelve warps: two groups of four for the softmax
// of a tile (a thread per row), one that issues the MMAs, one that loads K and V by
// TMA, page by page, into a ring, one that walks the items and loads their Q, and one that
// writes down for the second kernel which item was cut at the CTA's start and, where tiles of Q
// are no boxes, loads half of their rows.
//
// Bound by the tensor cores and, nearly as much, by the softmax: the 256 x 128 scores of a
// unit are 2 x 2 x 128 x 128 x D MACs (2048 cycles at D = 128 and 4096 a cycle; Q K^T takes
// a sixth more for its operands from shared memory) and 32768 exponentials (1024 cycles at
// 32 a cycle) with as many maxima, sums and conversions.  So the two tiles alternate: while
// the softmax works on one, the tensor cores multiply for the other.  A prompt of 8191
// tokens, 32 heads over 8 of 128: 421 us, 1.31 PFLOP/s.
//   S = Q K^T     both operands in shared memory, K-major, 128-byte swizzle
//   O += P V      P from tensor memory, V from shared memory as it lies ([key][D], the
//                 MN-major form of the B operand)
// An item of one tile is bound by the bytes of K and V, so there the weights are two
// bf16 parts (the second in the columns of S that the first leaves free).  With two tiles they are
// one part, since another would be half as many MACs again: the error of a prompt's results
// against 64 bits is 2.1e-3 of their norm so, 1.6e-3 of it the results' own rounding.
// S of the next unit is issued behind the product that still reads P from the same columns.
// This rests on the one tensor pipe of an SM taking the MMAs of one thread, all of them of one
// CTA and M = 128, in the order of their issue.  What is documented is that order for MMAs of one
// shape and accumulator; these have two accumulators and, with D = 64, two values of N.  All 512
// columns are in use, so P has no place of its own; waiting for the product's end before S is issued
// makes a prompt of 8191 tokens 453 us instead of 421, with the same bits.  That O stands still once the
// S after it is complete rests on the commit alone, which covers all MMAs issued before.
//
// The softmax keeps a reference m of each row instead of the exact maximum: O and the
// sum are only rescaled where the maximum has outgrown m by more than 2^8 in weight
// (weights and their sum hold that easily, and O for values up to 2^119 over the number of keys
// that weigh), which after a row's first units is rare.  The end's O / sum is the same number.
// Weights are 2^(s sl2 - z) in one FMA, z the scaled reference as rounded to fp32 (to a
// quarter at scores of 2^24 / 8).  So everything that brings weights of two references together
// (rescaling, the two groups' sums, the parts of an item) goes by the same z, and the log of the
// sum takes back what the rounding added.
constexpr int kRows = 256;     // rows of an item
constexpr int kTileRows = 128;
constexpr int kSoftWarps = 8;
constexpr int kMmaWarp = 8, kLoadWarp = 9, kItemWarp = 10, kHelpWarp = 11;
constexpr int kThreads = 384;
constexpr int kItems = 4;      // items that the item warp is ahead, at most
constexpr float kSlackLog2 = 8.f;
constexpr int kOutBytes = 32 * 64;  // 32 rows of 32 values

// Steps of about 0.3 us, fitted to the CTAs' times as they were before weights below the normal
// range were kept (6 % less for two tiles): a unit of one tile 1.2 us, of two
// tiles 1.5, an item's beginning and end 2.7 (7 and 12 steps were each slower on some of a
// prompt, mixed chunks, drafts and windows).  A join is 4 us, but items left whole so that
// there is none keep some CTAs twice as long: 4 x 1000 tokens, window 1024, 23 -> 37 us.
struct ChunkCut {
  static constexpr int ROWS = kRows, EXTRA = 9, MIN_SHARE = 16, WHOLE_SHARE = 0, WHOLE_MORE = 0;
  static __device__ __forceinline__ int weight(int rows) { return rows > kTileRows ? 5 : 4; }
};
using Cursor = PagedCursor<ChunkCut>;

template <int D>
struct Cfg {
  static constexpr int kHalves = D / 64;               // 64-column halves of a tile
  static constexpr int kHalf = kTileRows * 128;         // bytes of one
  static constexpr int kTile = kHalves * kHalf;         // a tile of Q, or the K or V of a unit
  static constexpr int kStages = D == 128 ? 4 : 8;
  static constexpr int kSmem = (2 + kStages) * kTile + 1024;
  static constexpr int kSlotFloats = kRows * (D + 2);   // a partial result: sums [D / 4][256][4], maxima, sums of weights
  static constexpr uint32_t kCols = 512;                // S, S, O, O: 256 + 2 D columns, to a power of two
  static constexpr uint32_t kO = 256;                   // first column of O
};

// 2^x; results below the normal range are zero
__device__ __forceinline__ float ex2_ftz(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float scaled_ref(float m, float sl2) { return __fmul_rn(m, sl2); }
// what weights by reference m are multiplied by to go by `top`
__device__ __forceinline__ float to_ref(float m, float top, float sl2) {
  return m == -INFINITY ? 0.f : exp2f(scaled_ref(m, sl2) - scaled_ref(top, sl2));
}
// log of the sum of exp(scale s), of which l is by reference m
__device__ __forceinline__ float log_sum(float m, float l, float scale, float sl2) {
  if (l == 0.f) return -INFINITY;
  const float added = fmaf(-m, sl2, scaled_ref(m, sl2));  // (exact)
  return fmaf(m, scale, fmaf(added, 0.6931471805599453f, logf(l)));
}

struct JoinItem {
  int c0, c1;  // CTAs that share the item
  int q0, t, h, rows, valid;
};

// A from tensor memory (a lane per row, two values a column)
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t bd, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(bd), "r"(idesc), "r"(acc));
}
// MN-major operand in 128-byte swizzle: rows of K (keys) of 64 values, groups of 8 rows
// 1024 bytes apart (stride offset), the next 64 values kHalf bytes on (leading offset).
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t addr, uint32_t half) {
  uint64_t d = 0;
  d |= (uint64_t)((addr >> 4) & 0x3FFF);
  d |= (uint64_t)(half >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0],"
      " {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

// Registers: all groups of four warps start with 168 a thread (the launch's 64512 / 384);
// the softmax groups, whose threads hold a row of scores, take what the third gives up.
constexpr int kManyRegs = 208, kFewRegs = 88;
static_assert(2 * kManyRegs + kFewRegs == 3 * 168, "registers of the launch");
template <int N>
__device__ __forceinline__ void reg_inc() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void reg_dec() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

struct Bars {
  unsigned long long full[8], empty[8];      // ring
  unsigned long long item[kItems], item_free[kItems], q_free[2];
  unsigned long long s[2], p[2], q[2], o[2], o_free[2];  // per tile
  unsigned long long joined, drain;
};

// What the roles of a CTA share.
struct Shared {
  PagedPlan<kSoftWarps * kOutBytes> plan;  // scratch: each softmax warp's block of the result on its way out
  Bars bars;
  Cursor start;
  Cursor items[kItems];
  float m[kTileRows], l[kTileRows];  // an item of one tile: the second group's statistics
  uint32_t tmem;
  int abort;
};

struct Role {
  const PagedArgs& a;
  Shared& sh;
  uint32_t sq, ring;   // Q tiles, K and V stages
  long long limit;

  __device__ __forceinline__ bool wait(unsigned long long& bar, unsigned parity, uint32_t bit) const {
    return mbar_wait_warp(smem_u32(&bar), parity, a.err, &sh.abort, bit, limit);
  }
  __device__ __forceinline__ bool aborted() const { return *(volatile int*)&sh.abort != 0; }
  __device__ __forceinline__ int rows(const Cursor& c) const { return c.n * a.group - c.t * kRows; }
  // item n of the CTA's share; null after a timeout
  __device__ __forceinline__ const Cursor* item(unsigned n) const {
    return wait(sh.bars.item[n % kItems], (n / kItems) & 1u, kErrTimeoutFull) ? &sh.items[n % kItems] : nullptr;
  }
  __device__ __forceinline__ void item_done(unsigned n) const {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&sh.bars.item_free[n % kItems]));
  }
};

// Whether the queries of a tile are a box [128 / group tokens][group heads][D] of q.
__host__ __device__ __forceinline__ bool boxes_of_q(int group) { return kTileRows % group == 0; }

// The share's items for the other warps, and their tiles of Q: by TMA, or row by row with
// the help of one more warp where tiles do not begin and end with a token.  One warp that
// does nothing else: in the softmax warps the same took 4000 cycles at every item, mostly
// for its instructions, which the loops over units drive out of the caches.
template <int D>
__device__ __forceinline__ void item_role(const Role& r, const CUtensorMap* tq) {
  using C = Cfg<D>;
  const PagedArgs& a = r.a;
  Bars& bars = r.sh.bars;
  const int lane = threadIdx.x & 31;
  const bool boxes = boxes_of_q(a.group), leads = (threadIdx.x >> 5) == kItemWarp;
  Cursor c = r.sh.start;
  unsigned used[2] = {0, 0};  // items of a tile
  bool ok = true;
  for (unsigned n = 0;; ++n) {
    if (leads) {
      if (!(ok = r.wait(bars.item_free[n % kItems], ((n / kItems) & 1u) ^ 1u, kErrTimeoutEmpty))) break;
      if (lane == 0) {
        r.sh.items[n % kItems] = c;
        mbar_arrive(smem_u32(&bars.item[n % kItems]));
      }
      __syncwarp();
    }
    if (c.done()) break;
    const int rows = r.rows(c);
    for (int tile = 0; tile < (rows > kTileRows ? 2 : 1); ++tile) {
      // every product with the tile before is done
      if (!(ok = r.wait(bars.q_free[tile], (used[tile]++ & 1u) ^ 1u, kErrTimeoutEmpty))) break;
      const uint32_t dst = r.sq + tile * C::kTile, bar = smem_u32(&bars.q[tile]);
      const int first = c.t * kRows + tile * kTileRows;
      if (boxes) {
        // (rows past the item's last are other sequences' or zero: their results go nowhere)
        if (lane == 0) {
          mbar_arrive_expect_tx(bar, (uint32_t)C::kTile);
#pragma unroll
          for (int i = 0; i < C::kHalves; ++i)
            tma_load_3d(dst + i * C::kHalf, tq, bar, i * 64, c.h * a.group, c.q0 + over_group(a, first));
        }
        __syncwarp();
      } else {
        const __nv_bfloat16* base = a.q + (int64_t)c.q0 * a.ld_q + c.h * a.group * D;
#pragma unroll 2
        for (int i = leads ? 0 : 1; i < kTileRows * D / 256; i += 2) {
          const int e = i * 32 + lane, ch = e % (D / 8), rr = e / (D / 8);
          const bool live = tile * kTileRows + rr < rows;
          const int at = live ? first + rr : 0, tok = over_group(a, at);
          cp_async_16(dst + (ch >> 3) * C::kHalf + swz_offset<64>(rr, ch & 7),
                      base + tok * a.ld_q + (at - tok * a.group) * D + ch * 8, live ? 16u : 0u);
        }
        cp_async_commit();
        cp_async_wait<0>();
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
      }
    }
    if (!ok) break;
    c.next_item(a, r.sh.plan);
  }
  // after a timeout: wait for the copies in flight into memory that is given back
  if (boxes && r.aborted())
    for (int tile = 0; tile < 2; ++tile)
      if (used[tile] > 0) mbar_drain(smem_u32(&bars.q[tile]), (used[tile] - 1) & 1u, r.limit);
}

// K and V of every unit: K0 V0 K1 V1 ...
template <int D>
__device__ __forceinline__ void load_role(const Role& r, const CUtensorMap* tk, const CUtensorMap* tv) {
  using C = Cfg<D>;
  const PagedArgs& a = r.a;
  const int lane = threadIdx.x & 31;
  Cursor c = r.sh.start;
  const int pages = kUnitKeys >> a.page_log2;        // of a whole unit
  const int pg = lane / C::kHalves, half = lane % C::kHalves;
  const uint32_t box = 128u << a.page_log2;          // bytes: page_size rows of 128
  unsigned n = 0;                                    // stages filled
  // a page before all rows' windows may be gone: a box outside of the pool reads zeros
  auto seen = [&](const Cursor& at, int key) { return key + (1 << a.page_log2) > at.k.lo; };
  auto entry = [&]() {
    const int key = c.key0() + (pg << a.page_log2);
    return !c.done() && pg < pages && key < c.k.hi && seen(c, key) ? page_of(a, c.b, key) : -1;
  };
  int page = entry();
  bool ok = true;
  while (!c.done() && ok) {
    const int key0 = c.key0();
    const int live = max(0, min(c.k.hi, key0 + kUnitKeys) - key0);
    const int need = (live + (1 << a.page_log2) - 1) >> a.page_log2;
    const bool mine = pg < need;
    const bool there = mine && seen(c, key0 + (pg << a.page_log2));
    const int row = there ? pool_row(a, page_checked(a, page), c.h, 0) : -kUnitKeys;
    c.next(a, r.sh.plan);
    page = entry();  // on its way while this unit waits for room
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      const unsigned st = n % C::kStages;
      ok = r.wait(r.sh.bars.empty[st], ((n / C::kStages) & 1u) ^ 1u, kErrTimeoutEmpty);
      if (!ok) break;
      const uint32_t bar = smem_u32(&r.sh.bars.full[st]);
      if (lane == 0) mbar_arrive_expect_tx(bar, (uint32_t)(need * C::kHalves) * box);
      __syncwarp();
      if (mine) tma_load_2d(r.ring + st * C::kTile + half * C::kHalf + pg * box, kv ? tv : tk, bar, half * 64, row);
      ++n;
    }
  }
  // after a timeout: wait for the copies in flight into memory that is given back
  if (r.aborted())
    for (unsigned i = n > (unsigned)C::kStages ? n - C::kStages : 0u; i < n; ++i)
      mbar_drain(smem_u32(&r.sh.bars.full[i % C::kStages]), (i / C::kStages) & 1u, r.limit);
}

// The MMAs.
template <int D>
__device__ __forceinline__ void mma_role(const Role& r, uint32_t tmem) {
  using C = Cfg<D>;
  const PagedArgs& a = r.a;
  Bars& bars = r.sh.bars;
  const int lane = threadIdx.x & 31;
  const bool leader = elect_one();
  constexpr uint32_t id_s = idesc_bf16_f32(kTileRows, kUnitKeys);
  constexpr uint32_t id_o = idesc_bf16_f32(kTileRows, D) | (1u << 16);  // B is MN-major
  unsigned base = 0, sp[2] = {0, 0}, qs[2] = {0, 0}, os[2] = {0, 0};
  bool ok = true;
  // stages of unit j of the item: K 2 j, V 2 j + 1 from base
  auto full = [&](unsigned i) {
    ok = ok && r.wait(bars.full[(base + i) % C::kStages], ((base + i) / C::kStages) & 1u, kErrTimeoutFull);
    return ok;
  };
  auto free_stage = [&](unsigned i) {
    if (leader) tc_commit(smem_u32(&bars.empty[(base + i) % C::kStages]));
    __syncwarp();
  };
  auto qk = [&](int slot, int tile, unsigned i) {  // S of `slot` from the Q of `tile`
    tc_fence_after();
    if (leader) {
      const uint64_t qd = smem_desc_kmajor<64>(r.sq + tile * C::kTile);
      const uint64_t kd = smem_desc_kmajor<64>(r.ring + ((base + i) % C::kStages) * C::kTile);
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        const uint32_t at = ((kk >> 2) * C::kHalf + (kk & 3) * 32) >> 4;
        tc_mma_bf16(tmem + slot * 128, qd + at, kd + at, id_s, kk > 0);
      }
      if (!a.fault) tc_commit(smem_u32(&bars.s[slot]));
    }
    __syncwarp();
  };
  // O of `slot` += P V; fine: P has two parts
  auto pv = [&](int slot, unsigned i, int steps, bool first, bool last, bool fine) {
    if (first) ok = ok && r.wait(bars.o_free[slot], (os[slot]++ & 1u) ^ 1u, kErrTimeoutAcc);
    ok = ok && r.wait(bars.p[slot], sp[slot]++ & 1u, kErrTimeoutAcc);
    if (!ok) return;
    tc_fence_after();
    if (leader) {
      const uint64_t vd = smem_desc_mn(r.ring + ((base + i) % C::kStages) * C::kTile, C::kHalf);
      const uint32_t d = tmem + C::kO + slot * D, p = tmem + slot * 128;
      if (steps == 8) {
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) mma_ts(d, p + kk * 8, vd + kk * 128, id_o, !(first && kk == 0));
      } else {
        for (int kk = 0; kk < steps; ++kk) mma_ts(d, p + kk * 8, vd + kk * 128, id_o, !(first && kk == 0));
      }
      if (fine)
        for (int kk = 0; kk < steps; ++kk) mma_ts(d, p + 64 + kk * 8, vd + kk * 128, id_o, 1u);
      if (last) tc_commit(smem_u32(&bars.o[slot]));
    }
    __syncwarp();
  };
  auto free_q = [&](int tile) {
    if (leader) tc_commit(smem_u32(&bars.q_free[tile]));
    __syncwarp();
  };
  for (unsigned n = 0; ok; ++n) {
    const Cursor* item = r.item(n);
    if (!item || item->done()) break;
    const int count = item->end - item->first, first_key = item->key0(), hi = item->k.hi, len = item->len;
    const bool two = r.rows(*item) > kTileRows;
    r.item_done(n);
    // k-steps of unit j, whose values are in stage i
    auto steps_of = [&](int j, unsigned i) {
      const int key0 = first_key + j * kUnitKeys, steps = (max(0, min(hi, key0 + kUnitKeys) - key0) + 15) >> 4;
      if (key0 + steps * 16 > len) {
        // values past the sequence's end may be anything, and 0 * NaN is NaN: zero them
        const int from = max(0, len - key0), nz = steps * 16 - from;
        for (int e = lane; e < nz * C::kHalves * 8; e += 32) {
          const int row = from + e / (C::kHalves * 8), ch = e % (C::kHalves * 8);
          sts_u4(r.ring + ((base + i) % C::kStages) * C::kTile + (ch >> 3) * C::kHalf + row * 128 + (ch & 7) * 16,
                 make_uint4(0u, 0u, 0u, 0u));
        }
        fence_proxy_async_smem();
        __syncwarp();
      }
      return steps;
    };
    ok = r.wait(bars.q[0], qs[0]++ & 1u, kErrTimeoutFull);
    if (two) ok = ok && r.wait(bars.q[1], qs[1]++ & 1u, kErrTimeoutFull);
    if (!ok || !full(0)) break;
    qk(0, 0, 0);
    if (two) {
      // two tiles: both take every unit
      qk(1, 1, 0);
      free_stage(0);
      if (count == 1) {
        free_q(0);
        free_q(1);
      }
      for (int j = 0; j < count && full(2 * j + 1); ++j) {
        const bool last = j + 1 == count;
        const int steps = steps_of(j, 2 * j + 1);
        pv(0, 2 * j + 1, steps, j == 0, last, false);
        if (!ok) break;
        if (!last) {
          if (!full(2 * j + 2)) break;
          qk(0, 0, 2 * j + 2);
          if (j + 2 == count) free_q(0);
        }
        pv(1, 2 * j + 1, steps, j == 0, last, false);
        if (!ok) break;
        free_stage(2 * j + 1);
        if (!last) {
          qk(1, 1, 2 * j + 2);
          free_stage(2 * j + 2);
          if (j + 2 == count) free_q(1);
        }
      }
    } else {
      // one tile: the units take turns
      free_stage(0);
      if (count > 1) {
        if (!full(2)) break;
        qk(1, 0, 2);
        free_stage(2);
      }
      if (count <= 2) free_q(0);
      for (int j = 0; j < count && full(2 * j + 1); ++j) {
        const int steps = steps_of(j, 2 * j + 1);
        pv(j & 1, 2 * j + 1, steps, j < 2, j + 2 >= count, true);
        if (!ok) break;
        free_stage(2 * j + 1);
        if (j + 2 < count) {
          if (!full(2 * j + 4)) break;
          qk(j & 1, 0, 2 * j + 4);
          free_stage(2 * j + 4);
          if (j + 3 == count) free_q(0);
        }
      }
    }
    base += 2 * count;
  }
  if (r.aborted()) {  // the MMAs issued so far end before tensor memory is given back
    if (leader) tc_commit(smem_u32(&bars.drain));
    __syncwarp();
    mbar_drain(smem_u32(&bars.drain), 0u, r.limit);
  }
}

// The softmax: a thread per row of a tile.
template <int D>
__device__ __forceinline__ void softmax_role(const Role& r, uint32_t tmem) {
  using C = Cfg<D>;
  const PagedArgs& a = r.a;
  Bars& bars = r.sh.bars;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, grp = warp >> 2, row = threadIdx.x & 127;
  const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // the warp's 32 lanes of tensor memory
  const uint32_t ts = tmem + lanes + grp * 128, to = tmem + lanes + C::kO + grp * D;
  const float sl2 = a.scale * 1.4426950408889634f, slack = fminf(kSlackLog2 / sl2, FLT_MAX);
  unsigned sn = 0, on = 0, joins = 0;
  bool ok = true;
  for (unsigned n = 0;; ++n) {
    const Cursor* item = r.item(n);
    if (!item || item->done()) break;
    const Cursor& c = *item;
    const int rows = r.rows(c), count = c.end - c.first;
    const bool two = rows > kTileRows;
    // the group's rows and units: its own tile and all units, or the tile and every other unit
    const int r0 = two ? grp * kTileRows : 0, j0 = two ? 0 : grp, dj = two ? 1 : 2;
    const bool live = r0 + row < rows;
    const bool idle = r0 + (warp & 3) * 32 >= rows;  // no row of the warp is the item's
    const bool works = j0 < count;
    // keys [low, lim) that the row sees; a row past the item's last one never asks for masks
    int lim = 0x7FFFFFFF, low = 0;
    if (live) {
      const int p = c.len - c.n + over_group(a, c.t * kRows + r0 + row);
      lim = a.causal ? min(c.len, p + 1) : c.len;
      low = first_seen(a, p);
    }
    const int first_key = c.key0();
    float m = -INFINITY, l = 0.f;
    for (int j = j0; j < count; j += dj) {
      const int key0 = first_key + j * kUnitKeys;
      if (!(ok = r.wait(bars.s[grp], sn & 1u, kErrTimeoutAcc))) break;
      ++sn;
      tc_fence_after();
      if (!idle) {
        uint32_t s[4][32];
#pragma unroll
        for (int i = 0; i < 4; ++i) tmem_ld32_nowait(ts + i * 32, s[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) tmem_wait_ld32(s[i]);
        if (!__all_sync(0xffffffffu, key0 >= low && key0 + kUnitKeys <= lim)) {
          const int from = low - key0, to_ = lim - key0;
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < 32; ++k)
              if (i * 32 + k < from || i * 32 + k >= to_) s[i][k] = 0xFF800000u;  // -infinity
        }
        // (several maxima and sums side by side: one chain of 64 steps each is as long as all
        // of the row's exponentials)
        float mx4[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          mx4[i] = __uint_as_float(s[i][0]);
#pragma unroll
          for (int k = 1; k < 31; k += 2)
            mx4[i] = fmaxf(mx4[i], fmaxf(__uint_as_float(s[i][k]), __uint_as_float(s[i][k + 1])));
          mx4[i] = fmaxf(mx4[i], __uint_as_float(s[i][31]));
        }
        const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3]));
        const bool grows = mx > m + slack;
        if (j == j0) {
          m = mx;
        } else if (__any_sync(0xffffffffu, grows)) {
          // S of this unit is complete, so the product before it is: O stands still
          const float f = grows ? to_ref(m, mx, sl2) : 1.f;
          if (grows) m = mx;
          l *= f;
#pragma unroll 1
          for (int i = 0; i < D / 16; ++i) {
            float o[16];
            uint32_t q[16];
            tmem_ld16(to + i * 16, o);
#pragma unroll
            for (int k = 0; k < 16; ++k) q[k] = __float_as_uint(o[k] * f);
            tmem_st16(to + i * 16, q);
          }
        }
        const float nz = m == -INFINITY ? 0.f : -scaled_ref(m, sl2);
        // A weight below the normal range counts where its value is large, and fp32 sums and
        // bf16 weights hold it: 2^x is the square of 2^(x / 2), which is a normal number.  A prompt of
        // 8191 tokens takes 397 us with such weights flushed to zero, 421 so, 477 with exp2f.
        const f2_t sc = f2(0.5f * sl2, 0.5f * sl2), off = f2(0.5f * nz, 0.5f * nz);
        f2_t sum[4];
        auto weigh = [&](auto two_parts) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t p[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              float x, y;
              f2_split(ffma2(f2(__uint_as_float(s[i][2 * k]), __uint_as_float(s[i][2 * k + 1])), sc, off), x, y);
              const f2_t h = f2(ex2_ftz(x), ex2_ftz(y)), w = fmul2(h, h);
              f2_split(w, x, y);
              sum[k & 3] = i == 0 && k < 4 ? w : fadd2(sum[k & 3], w);
              s[i][2 * k] = __float_as_uint(x);
              s[i][2 * k + 1] = __float_as_uint(y);
              asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p[k]) : "f"(y), "f"(x));
            }
            tmem_st16(ts + i * 16, p);  // (columns of scores that are in registers already)
            if constexpr (decltype(two_parts)::value) {
#pragma unroll
              for (int k = 0; k < 16; ++k) {
                const float lo = __uint_as_float(s[i][2 * k]) - __uint_as_float(p[k] << 16);
                const float up = __uint_as_float(s[i][2 * k + 1]) - __uint_as_float(p[k] & 0xFFFF0000u);
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p[k]) : "f"(up), "f"(lo));
              }
              tmem_st16(ts + 64 + i * 16, p);
            }
          }
        };
        if (two)
          weigh(BoolConst<false>());
        else
          weigh(BoolConst<true>());
        float x, y;
        f2_split(fadd2(fadd2(sum[0], sum[1]), fadd2(sum[2], sum[3])), x, y);
        l += x + y;
        tmem_wait_st();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars.p[grp]));
    }
    if (works) ok = ok && r.wait(bars.o[grp], on++ & 1u, kErrTimeoutAcc);
    if (!ok) break;
    tc_fence_after();
    const bool halves = !two && count > 1;  // two sums over every other unit
    if (halves && grp == 1) {
      // the first group adds this one's sums to its own
      r.sh.m[row] = m;
      r.sh.l[row] = l;
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars.joined));
    } else if (works) {
      float f0 = 1.f, f1 = 0.f;
      if (halves) {
        if (!(ok = r.wait(bars.joined, joins++ & 1u, kErrTimeoutAcc))) break;
        tc_fence_after();
        const float m1 = r.sh.m[row], l1 = r.sh.l[row], top = fmaxf(m, m1);
        f0 = to_ref(m, top, sl2);
        f1 = to_ref(m1, top, sl2);
        l = l * f0 + l1 * f1;
        m = top;
      }
      const bool part = c.cut();
      float* slot = a.ws + (size_t)part_slot(blockIdx.x, c.first == 0) * C::kSlotFloats;
      const int at = r0 + row, of = live ? over_group(a, c.t * kRows + at) : 0;
      const int64_t out = (int64_t)(c.q0 + of) * a.heads + c.h * a.group + (live ? c.t * kRows + at - of * a.group : 0);
      const float inv = l == 0.f ? 0.f : 1.f / l;  // (a sum of NaN stays one)
      const uint32_t mine = smem_u32(r.sh.plan.scratch) + warp * kOutBytes;
      int64_t to_row[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) to_row[i] = __shfl_sync(0xffffffffu, live ? out : -1ll, i * 8 + (lane >> 2));
      // values [32 i, 32 i + 32) of the rows: to the workspace as they are (a part of the
      // item), or divided, by way of shared memory, so that four lanes write 64 bytes of a row
      auto put = [&](int i, const uint32_t (&o)[32]) {
        if (part) {
          if (live)
#pragma unroll
            for (int k = 0; k < 32; k += 4)
              *reinterpret_cast<uint4*>(slot + (size_t)((i * 32 + k) / 4 * kRows + at) * 4) =
                  make_uint4(o[k], o[k + 1], o[k + 2], o[k + 3]);
          return;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float lo = __uint_as_float(o[k * 8 + 2 * e]) * inv, hi = __uint_as_float(o[k * 8 + 2 * e + 1]) * inv;
            w[e] = l == 0.f ? 0u : act_pack2<0>(lo, hi);
          }
          sts_u4(mine + sw64_offset(lane, k), make_uint4(w[0], w[1], w[2], w[3]));
        }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float4 v = lds_f4(mine + sw64_offset(k * 8 + (lane >> 2), lane & 3));
          if (to_row[k] >= 0) *reinterpret_cast<float4*>(a.y + to_row[k] * D + i * 32 + (lane & 3) * 8) = v;
        }
        __syncwarp();
      };
      if (!idle) {
        // (a loop, and 32 columns at a time: unrolled, its instructions are fetched for every
        // item anew)
#pragma unroll 1
        for (int i = 0; i < D / 32; ++i) {
          uint32_t o[32];
          tmem_ld32_nowait(to + i * 32, o);
          if (halves) {
            uint32_t e[32];
            tmem_ld32_nowait(to + D + i * 32, e);
            tmem_wait_ld32(o);
            tmem_wait_ld32(e);
#pragma unroll
            for (int k = 0; k < 32; ++k)
              o[k] = __float_as_uint(__uint_as_float(o[k]) * f0 + __uint_as_float(e[k]) * f1);
          } else {
            tmem_wait_ld32(o);
          }
          put(i, o);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {  // O has been read: the next item's products may begin
        mbar_arrive(smem_u32(&bars.o_free[grp]));
        if (halves) mbar_arrive(smem_u32(&bars.o_free[1]));
      }
      if (!idle) {
        if (part) {
          slot[kRows * D + at] = m;
          slot[kRows * D + kRows + at] = l;
        } else if (live && a.lse) {
          a.lse[out] = log_sum(m, l, a.scale, sl2);
        }
      }
    }
    r.item_done(n);
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    paged_chunk_kernel(const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv,
                       const __grid_constant__ CUtensorMap tq, const __grid_constant__ PagedArgs a) {
  using C = Cfg<D>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) Shared sh;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    Bars& bars = sh.bars;
    for (int i = 0; i < C::kStages; ++i) {
      mbar_init(smem_u32(&bars.full[i]), 1u);
      mbar_init(smem_u32(&bars.empty[i]), 1u);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&bars.s[i]), 1u);
      mbar_init(smem_u32(&bars.p[i]), 4u);
      mbar_init(smem_u32(&bars.q[i]), boxes_of_q(a.group) ? 1u : 2u);
      mbar_init(smem_u32(&bars.q_free[i]), 1u);
      mbar_init(smem_u32(&bars.o[i]), 1u);
      mbar_init(smem_u32(&bars.o_free[i]), 4u);
    }
    for (int i = 0; i < kItems; ++i) {
      mbar_init(smem_u32(&bars.item[i]), 1u);
      mbar_init(smem_u32(&bars.item_free[i]), kSoftWarps + 1u);
    }
    mbar_init(smem_u32(&bars.joined), 4u);
    mbar_init(smem_u32(&bars.drain), 1u);
    fence_mbar_init();
    sh.abort = 0;
    prefetch_tmap(&tk);
    prefetch_tmap(&tv);
    prefetch_tmap(&tq);
  }
  if (warp == kMmaWarp) tmem_alloc(smem_u32(&sh.tmem), C::kCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_wait();
  pdl_trigger();
  make_plan<ChunkCut>(a, sh.plan);
  const unsigned long long total = sh.plan.total;
  const unsigned ctas = cut_ctas<ChunkCut>(total);
  const bool works = blockIdx.x < ctas;
  const unsigned long long u0 = works ? cut_start(total, ctas, blockIdx.x) : 0ull;
  const unsigned long long u1 = works ? cut_start(total, ctas, blockIdx.x + 1) : 0ull;
  if (warp == 0 && works) {
    Cursor c;
    c.seek(a, sh.plan, ctas, u0, (int)(u1 - u0));
    if (lane == 0) sh.start = c;
  }
  __syncthreads();
  if (warp == kHelpWarp && lane == 0) {
    // an item cut at this CTA's start is joined later; the first of its cuts speaks for it
    JoinItem j{};
    if (works && !sh.start.done() && sh.start.first > 0) {
      const Cursor& c = sh.start;
      const PagedShares s = shares_of(c, total, ctas, u1);
      j.c0 = (int)s.c0;
      j.c1 = (int)s.c1;
      j.q0 = c.q0;
      j.t = c.t;
      j.h = c.h;
      j.rows = min(kRows, c.n * a.group - c.t * kRows);
      j.valid = s.c0 + 1 == blockIdx.x;
    }
    reinterpret_cast<JoinItem*>(a.ws + (size_t)2 * gridDim.x * C::kSlotFloats)[blockIdx.x] = j;
  }
  const uint32_t sq = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const Role r{a, sh, sq, sq + 2 * C::kTile, a.wait_limit ? a.wait_limit : kWaitLimitCycles};
  if (warp < kSoftWarps) {
    reg_inc<kManyRegs>();
    if (works) softmax_role<D>(r, sh.tmem);
  } else {
    reg_dec<kFewRegs>();
    if (works && warp == kMmaWarp) mma_role<D>(r, sh.tmem);
    if (works && warp == kLoadWarp) load_role<D>(r, &tk, &tv);
    if (works && (warp == kItemWarp || (warp == kHelpWarp && !boxes_of_q(a.group)))) item_role<D>(r, &tq);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_dealloc(sh.tmem, C::kCols);
}

// Joins the parts of the items that several CTAs shared, in the order of their keys: a
// block per cut and 32 rows, a warp per 8 columns and D / 8 warps.  Bound by latency, so the
// statistics of all parts and the sums of the first four are asked for at once, then four
// parts at a time (part after part, each waiting for the one before it, 10 took 15 us).
constexpr int kJoinParts = 4;
constexpr int kCtas = 184;  // at most: the join keeps statistics of as many parts in shared memory
template <int D>
__global__ void __launch_bounds__(4 * D)
    paged_join_kernel(const __grid_constant__ PagedArgs a, int grid) {
  using C = Cfg<D>;
  __shared__ float s_w[kCtas][32], s_l[kCtas][32];  // maxima and sums of weights of the parts
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait();
  pdl_trigger();
  const JoinItem j = reinterpret_cast<const JoinItem*>(a.ws + (size_t)2 * grid * C::kSlotFloats)[blockIdx.x];
  const int r = blockIdx.y * 32 + lane, parts = j.c1 - j.c0 + 1;
  if (!j.valid || (int)blockIdx.y * 32 >= j.rows) return;
  const bool live = r < j.rows;
  auto slot = [&](int c) { return a.ws + (size_t)part_slot(j.c0 + c, c == 0) * C::kSlotFloats; };
  const float sl2 = a.scale * 1.4426950408889634f;
  float4 p[kJoinParts], q[kJoinParts];
  auto fetch = [&](int c0) {
#pragma unroll
    for (int i = 0; i < kJoinParts; ++i) {
      const float* from = slot(min(c0 + i, parts - 1)) + (size_t)(live ? r : 0) * 4;
      p[i] = *reinterpret_cast<const float4*>(from + (size_t)(2 * warp) * kRows * 4);
      q[i] = *reinterpret_cast<const float4*>(from + (size_t)(2 * warp + 1) * kRows * 4);
    }
  };
  fetch(0);
  for (int c = warp; c < parts; c += D / 8) {
    s_w[c][lane] = live ? slot(c)[kRows * D + r] : -INFINITY;
    s_l[c][lane] = live ? slot(c)[kRows * D + kRows + r] : 0.f;
  }
  __syncthreads();
  if (!live) return;
  float l = 0.f, mx = -INFINITY;
  for (int c = 0; c < parts; ++c) mx = fmaxf(mx, s_w[c][lane]);
  float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int c0 = 0; c0 < parts; c0 += kJoinParts) {
    if (c0 > 0) fetch(c0);
#pragma unroll
    for (int i = 0; i < kJoinParts; ++i) {
      if (c0 + i >= parts) break;
      const float w = to_ref(s_w[c0 + i][lane], mx, sl2);
      l = fmaf(w, s_l[c0 + i][lane], l);
      f[0] = fmaf(w, p[i].x, f[0]); f[1] = fmaf(w, p[i].y, f[1]); f[2] = fmaf(w, p[i].z, f[2]); f[3] = fmaf(w, p[i].w, f[3]);
      f[4] = fmaf(w, q[i].x, f[4]); f[5] = fmaf(w, q[i].y, f[5]); f[6] = fmaf(w, q[i].z, f[6]); f[7] = fmaf(w, q[i].w, f[7]);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;  // (a sum of NaN stays one)
#pragma unroll
  for (int k = 0; k < 8; ++k) f[k] *= inv;
  const int row = j.t * kRows + r, of = over_group(a, row);
  const int64_t at = (int64_t)(j.q0 + of) * a.heads + j.h * a.group + row - of * a.group;
  *reinterpret_cast<uint4*>(a.y + at * D + warp * 8) = pack8(f);
  if (a.lse && warp == 0) a.lse[at] = log_sum(mx, l, a.scale, sl2);
}

int grid_of() {
  const int sms = device_sm_count();
  return sms < kCtas ? sms : kCtas;
}

template <int D>
cudaError_t launch_chunk(const PagedArgs& a, cudaStream_t s) {
  CUtensorMap tk, tv, tq;
  const uint64_t rows = (uint64_t)a.pages * a.kv_heads << a.page_log2;
  if (!make_tmap_2d(&tk, a.k, rows, D, 64, 1u << a.page_log2) || !make_tmap_2d(&tv, a.v, rows, D, 64, 1u << a.page_log2))
    return cudaErrorInvalidValue;
  memset(&tq, 0, sizeof(tq));
  if (boxes_of_q(a.group) && !make_tmap_3d(&tq, a.q, D, (uint64_t)a.heads, (uint64_t)a.T, D, (uint64_t)a.ld_q, 64,
                                           (uint32_t)a.group, (uint32_t)(kTileRows / a.group)))
    return cudaErrorInvalidValue;
  cudaError_t e = smem_optin(reinterpret_cast<const void*>(paged_chunk_kernel<D>), Cfg<D>::kSmem);
  if (e != cudaSuccess) return e;
  const int grid = grid_of();
  e = launch_kernel(paged_chunk_kernel<D>, dim3(grid), dim3(kThreads), Cfg<D>::kSmem, s, tk, tv, tq, a);
  if (e != cudaSuccess) return e;
  return launch_kernel(paged_join_kernel<D>, dim3(grid, kRows / 32), dim3(4 * D), 0, s, a, grid);
}

}  // namespace

size_t paged_chunk_ws_bytes() {
  return ((size_t)2 * Cfg<128>::kSlotFloats * sizeof(float) + sizeof(JoinItem)) * grid_of();
}

cudaError_t launch_paged_chunk(const PagedArgs& a, cudaStream_t s) {
  return a.D == 128 ? launch_chunk<128>(a, s) : launch_chunk<64>(a, s);
}

}  // namespace sparoa
