// Attention over a paged key/value cache: the kernel for few query rows per key
// head (one new token, or a few drafted ones, of each sequence), right for any
// number, and the choice between it and the kernel for chunks of tokens.
#include "paged.cuh"

namespace sparoa {

namespace {

// ---------------------------------------------------------------------------
// Few rows.  Bound by the bytes of the cache, read once.
//
// A CTA of 8 warps walks its share of the units; of a unit's 128 keys each warp has
// 16 of its own, whose K and V rows it fetches itself by TMA (boxes of 16 rows x 64
// values, 128-byte swizzle, so that the fragment loads are free of bank conflicts)
// into a ring of its own, kStages - 1 ahead, across the ends of items: no barrier
// stands between loads and products.  S = Q K^T and O += P V on mma.sync m16n8k16 with
// the item's (up to 16) rows as M, an online softmax per warp; when an item ends the
// 8 partial results are joined in shared memory, in the ring's one free stage.  An
// item that several CTAs share leaves fp32 partial results in the workspace, and the
// CTA that arrives last joins them in the order of the keys, so that results do not
// depend on timing.
//
// Score rules change and mask the 16 x 16 scores of a warp where they lie, in registers: a kernel for
// each set of rules that occurs, so that none pays for another's.  One token of each of 48 contexts of
// 400 to 12000, 32 heads over 8 of 128, scores capped: 107 us, 106 without a cap (138 with exponentials for
// every cap).
constexpr int kRows = 16;     // rows of an item
constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kKeys = 16;     // a warp's keys of a unit

// An item's beginning and end take as long as one unit to three (64 contexts of 500 to
// 16000 tokens: 188 us with 1 and with 3, 185 with 2); joining parts of an item as eight
// units of a CTA that has few.
template <int WALK>
struct SmallCut {
  static constexpr bool RULED = WALK != kPlainWalk, REVERSED = WALK == kReversedWalk;
  static constexpr int ROWS = kRows, EXTRA = 2, MIN_SHARE = 2, WHOLE_SHARE = 8, WHOLE_MORE = 8;
  static __device__ __forceinline__ int weight(int) { return 1; }
};
static_assert(kKeys * kWarps == kUnitKeys, "unit");

template <int D>
struct Cfg {
  static constexpr int kHalf = kKeys * 128;             // bytes of a box
  static constexpr int kBoxes = D / 64;
  static constexpr int kStageBytes = 2 * kBoxes * kHalf;  // K and V; also [16][D] fp32
  static constexpr int kStages = D == 128 ? 3 : 5;
  static constexpr int kSmem = kWarps * kStages * kStageBytes + 1024;
};

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

// the bf16 pair of what `hi` (a rounded pair) leaves of lo and up
__device__ __forceinline__ uint32_t rest2(uint32_t hi, float lo, float up) {
  return pack2(lo - __uint_as_float(hi << 16), up - __uint_as_float(hi & 0xFFFF0000u));
}

// Floats of a partial result: [16][D] sums, then [16] maxima and [16] sums of weights.
template <int D>
constexpr int kSlotFloats = kRows * (D + 2);

template <int D, int RULES>
__global__ void __launch_bounds__(kThreads, 1)
    paged_small_kernel(const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv,
                       const __grid_constant__ PagedArgs a) {
  using C = Cfg<D>;
  using Cut = SmallCut<walk_of(RULES)>;
  using Cursor = PagedCursor<Cut>;
  constexpr int S = C::kStages;
  extern __shared__ uint8_t smem_raw[];
  __shared__ PagedPlan<> plan;
  __shared__ Cursor s_start;
  __shared__ __align__(8) unsigned long long s_bar[kWarps][S];
  __shared__ float s_m[kWarps][kRows], s_l[kWarps][kRows];
  __shared__ uint32_t s_at[kWarps];
  __shared__ int s_abort, s_last;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, tq = lane & 3;
  const uint32_t ring = ((smem_u32(smem_raw) + 1023u) & ~1023u) + (uint32_t)(warp * S * C::kStageBytes);
  if (lane == 0) {
    for (int s = 0; s < S; ++s) mbar_init(smem_u32(&s_bar[warp][s]), 1u);
    fence_mbar_init();
    if (warp == 0) {
      s_abort = 0;
      prefetch_tmap(&tk);
      prefetch_tmap(&tv);
    }
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  make_plan<Cut>(a, plan);
  const unsigned long long total = plan.total;
  const unsigned ctas = cut_ctas<Cut>(total);
  if (blockIdx.x >= ctas) return;
  const unsigned long long u0 = cut_start(total, ctas, blockIdx.x), u1 = cut_start(total, ctas, blockIdx.x + 1);
  if (warp == 0) {
    Cursor c;
    c.seek(a, plan, ctas, u0, (int)(u1 - u0));
    if (lane == 0) s_start = c;
  }
  __syncthreads();

  const long long limit = a.wait_limit ? a.wait_limit : kWaitLimitCycles;
  Cursor pc = s_start, cc = pc;   // the next unit to fetch, and the one being used
  unsigned issued = 0, used = 0;  // stages filled and consumed
  bool dead = false;              // a wait ran out: no more loads or products
  auto live = [&](const Cursor& c) {
    const int key = c.key0() + warp * kKeys;
    return key < c.k.hi && key + kKeys > c.k.lo;
  };
  int page = 0;  // of the next unit to fetch, loaded a step ahead
  auto look_up = [&]() {
    if (!pc.done() && live(pc)) page = page_of(a, pc.b, pc.key0() + warp * kKeys);
  };
  auto fetch = [&]() {
    if (pc.done()) return;
    if (live(pc) && !dead) {
      if (lane == 0) {
        const int row = pool_row(a, page_checked(a, page), pc.h, pc.key0() + warp * kKeys);
        const uint32_t bar = smem_u32(&s_bar[warp][issued % S]), dst = ring + (issued % S) * C::kStageBytes;
        mbar_arrive_expect_tx(bar, C::kStageBytes);
#pragma unroll
        for (int i = 0; i < C::kBoxes; ++i) tma_load_2d(dst + i * C::kHalf, &tk, bar, i * 64, row);
#pragma unroll
        for (int i = 0; i < C::kBoxes; ++i) tma_load_2d(dst + (C::kBoxes + i) * C::kHalf, &tv, bar, i * 64, row);
      }
      ++issued;
    }
    pc.next(a, plan);
    look_up();
  };
  look_up();
  for (int i = 0; i < S - 1; ++i) fetch();

  uint32_t qa[D / 16][4];
  float o[D / 8][4], m0, m1, l0, l1;
  int lim0 = 0, lim1 = 0, low0 = 0, low1 = 0;  // keys that rows g and g + 8 see: [low, lim)
  bool fresh = true, any = false;
  const float sl2 = a.log2_unit;
  RowRules rule[2];
  // lane's rows within the ldmatrix blocks: K (n = key, k = value), V transposed
  const int krow = ((lane >> 4) << 3) + (lane & 7), kch = (lane >> 3) & 1;
  const int vrow = (((lane >> 3) & 1) << 3) + (lane & 7), vch = lane >> 4;

  for (; !cc.done(); cc.next(a, plan)) {
    fetch();
    const int rows = cc.n * a.group - cc.t * kRows;  // rows of the item (16 at most count)
    if (fresh) {
      fresh = false;
      any = false;
      m0 = m1 = -INFINITY;
      l0 = l1 = 0.f;
#pragma unroll
      for (int j = 0; j < D / 8; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
      const __nv_bfloat16* p[2] = {nullptr, nullptr};
      int lim[2] = {0, 0}, low[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (g + 8 * i < rows) {
          const int row = cc.t * kRows + g + 8 * i, tok = over_group(a, row), head = cc.h * a.group + row - tok * a.group;
          const int pos = cc.len - cc.n + tok;
          p[i] = a.q + (int64_t)(cc.q0 + tok) * a.ld_q + head * D;
          if constexpr (RULES != kPlain) {
            rule[i].load<RULES>(a, cc.q0, cc.n, cc.len, cc.prefix, tok, head);
          } else {
            lim[i] = a.causal ? min(cc.len, pos + 1) : cc.len;
            low[i] = first_seen(a, pos);
          }
        } else if constexpr (RULES != kPlain) {
          rule[i].none();
        }
      }
      lim0 = lim[0]; lim1 = lim[1]; low0 = low[0]; low1 = low[1];
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        const int c = kk * 16 + 2 * tq;
        qa[kk][0] = p[0] ? *reinterpret_cast<const uint32_t*>(p[0] + c) : 0u;
        qa[kk][1] = p[1] ? *reinterpret_cast<const uint32_t*>(p[1] + c) : 0u;
        qa[kk][2] = p[0] ? *reinterpret_cast<const uint32_t*>(p[0] + c + 8) : 0u;
        qa[kk][3] = p[1] ? *reinterpret_cast<const uint32_t*>(p[1] + c + 8) : 0u;
      }
    }
    if (live(cc) && !dead) {
      const uint32_t st = used % S, sk = ring + st * C::kStageBytes, sv = sk + C::kBoxes * C::kHalf;
      if (!mbar_wait_warp(smem_u32(&s_bar[warp][st]), (used / S) & 1u, a.err, &s_abort, kErrTimeoutFull, limit)) {
        dead = true;
      } else {
        ++used;
        any = true;
        const int key0 = cc.key0() + warp * kKeys;
        // values past the sequence's end may be anything, and 0 * NaN is NaN: zero them
        if (key0 + kKeys > cc.len) {
          const int from = cc.len - key0;  // 1 to 15
          for (int i = lane; i < (kKeys - from) * C::kBoxes * 8; i += 32) {
            const int r = from + i / (C::kBoxes * 8), c = i % (C::kBoxes * 8);
            sts_u4(sv + (c >> 3) * C::kHalf + r * 128 + (c & 7) * 16, make_uint4(0u, 0u, 0u, 0u));
          }
          fence_proxy_async_smem();  // before the stage is filled again by TMA
          __syncwarp();
        }
        float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          uint32_t r[4];
          const int ch = kk * 2 + kch;
          ldsm4(sk + (ch >> 3) * C::kHalf + krow * 128 + (((ch & 7) ^ (krow & 7)) << 4), r);
          mma16816(s[0], qa[kk], r[0], r[1]);
          mma16816(s[1], qa[kk], r[2], r[3]);
        }
        if constexpr (RULES != kPlain) {
          // (kernels for trees are for all that they may come with)
          if ((RULES & kCap) && (!(RULES & kTree) || a.cap > 0.f)) {
            const Capped cap(a);
            float top = 0.f;
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
#pragma unroll
              for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(s[nt][e]));
            if (__all_sync(0xffffffffu, cap.near(top))) {
#pragma unroll
              for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                for (int e = 0; e < 4; e += 2) f2_split(cap.near(f2(s[nt][e], s[nt][e + 1])), s[nt][e], s[nt][e + 1]);
            } else {
#pragma unroll
              for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                for (int e = 0; e < 4; e += 2) f2_split(cap.far(f2(s[nt][e], s[nt][e + 1])), s[nt][e], s[nt][e + 1]);
            }
          }
          if ((RULES & kBias) && (!(RULES & kTree) || a.slopes)) {
            const float far[2] = {(float)(rule[0].pos - key0), (float)(rule[1].pos - key0)}, one = a.cap > 0.f ? 1.f : a.score_log2;
            const bool drafted = (RULES & kTree) && key0 + kKeys > rule[0].base;
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const RowRules& u = rule[e >> 1];
                const int k = nt * 8 + 2 * tq + (e & 1);
                float d = fabsf(far[e >> 1] - (float)k);
                if (drafted) d = u.distance(key0 + k, d);
                s[nt][e] = fmaf(-u.slope, d, s[nt][e] * one);
              }
          }
          const uint32_t seen[2] = {rule[0].seen32<(RULES & kTree) != 0>(key0), rule[1].seen32<(RULES & kTree) != 0>(key0)};
#pragma unroll
          for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (!(seen[e >> 1] >> (nt * 8 + 2 * tq + (e & 1)) & 1u)) s[nt][e] = -INFINITY;
        } else {
#pragma unroll
          for (int nt = 0; nt < 2; ++nt) {
            const int key = key0 + nt * 8 + 2 * tq;
            if (key < low0 || key >= lim0) s[nt][0] = -INFINITY;
            if (key + 1 < low0 || key + 1 >= lim0) s[nt][1] = -INFINITY;
            if (key < low1 || key >= lim1) s[nt][2] = -INFINITY;
            if (key + 1 < low1 || key + 1 >= lim1) s[nt][3] = -INFINITY;
          }
        }
        float x0 = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1]));
        float x1 = fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3]));
        x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 1));
        x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 1));
        x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 2));
        x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 2));
        const bool grows = x0 > m0 || x1 > m1;
        if (__any_sync(0xffffffffu, grows)) {
          const float n0 = fmaxf(m0, x0), n1 = fmaxf(m1, x1);
          // (a row that has seen no key yet: nothing to rescale)
          const float c0 = m0 == -INFINITY ? 0.f : exp2f((m0 - n0) * sl2), c1 = m1 == -INFINITY ? 0.f : exp2f((m1 - n1) * sl2);
          m0 = n0;
          m1 = n1;
          l0 *= c0;
          l1 *= c1;
#pragma unroll
          for (int j = 0; j < D / 8; ++j) {
            o[j][0] *= c0; o[j][1] *= c0;
            o[j][2] *= c1; o[j][3] *= c1;
          }
        }
        // (exp2f: weights below the normal range count where their values are large)
        const float z0 = m0 == -INFINITY ? 0.f : m0, z1 = m1 == -INFINITY ? 0.f : m1;
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
          s[nt][0] = exp2f((s[nt][0] - z0) * sl2);
          s[nt][1] = exp2f((s[nt][1] - z0) * sl2);
          s[nt][2] = exp2f((s[nt][2] - z1) * sl2);
          s[nt][3] = exp2f((s[nt][3] - z1) * sl2);
          l0 += s[nt][0] + s[nt][1];
          l1 += s[nt][2] + s[nt][3];
        }
        // weights as two bf16 parts, high and what is left of them: 16 bits of each,
        // where one part alone would be off by as much as the result's own rounding
        const uint32_t pa[4] = {pack2(s[0][0], s[0][1]), pack2(s[0][2], s[0][3]), pack2(s[1][0], s[1][1]),
                                pack2(s[1][2], s[1][3])};
        const uint32_t pb[4] = {rest2(pa[0], s[0][0], s[0][1]), rest2(pa[1], s[0][2], s[0][3]),
                                rest2(pa[2], s[1][0], s[1][1]), rest2(pa[3], s[1][2], s[1][3])};
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
          uint32_t r[4];
          const int ch = j * 2 + vch;
          ldsm4_trans(sv + (ch >> 3) * C::kHalf + vrow * 128 + (((ch & 7) ^ (vrow & 7)) << 4), r);
          mma16816(o[2 * j], pa, r[0], r[1]);
          mma16816(o[2 * j + 1], pa, r[2], r[3]);
          mma16816(o[2 * j], pb, r[0], r[1]);
          mma16816(o[2 * j + 1], pb, r[2], r[3]);
        }
        __syncwarp();  // the stage may be filled again
      }
    }
    if (cc.blk + 1 == cc.end) {
      // the item, or this CTA's share of it, ends: join the warps
      const int valid = rows < kRows ? rows : kRows;
      l0 += __shfl_xor_sync(0xffffffffu, l0, 1);
      l1 += __shfl_xor_sync(0xffffffffu, l1, 1);
      l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
      l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
      if (tq == 0) {
        s_m[warp][g] = m0;
        s_m[warp][g + 8] = m1;
        s_l[warp][g] = l0;
        s_l[warp][g + 8] = l1;
      }
      // sums [16][D] fp32 into the free stage, 32-byte pieces swizzled by the row
      const uint32_t mine = ring + (issued % S) * C::kStageBytes;
      if (any) {
#pragma unroll
        for (int j = 0; j < D / 8; ++j) {
          const uint32_t at = mine + g * (D * 4) + ((j ^ g) << 5) + tq * 8;
          if (g < valid) asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(o[j][0]), "f"(o[j][1]) : "memory");
          if (g + 8 < valid)
            asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(at + 8 * D * 4), "f"(o[j][2]), "f"(o[j][3]) : "memory");
        }
      }
      // where the other warps' sums are: their free stages
      if (lane == 0) s_at[warp] = mine;
      __syncthreads();
      const int row = threadIdx.x >> 4, piece = threadIdx.x & 15;
      const bool mine_out = row < valid && piece < D / 8;
      float acc[8], mx = -INFINITY, ls = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) acc[k] = 0.f;
      if (mine_out) {
#pragma unroll
        for (int w = 0; w < kWarps; ++w) mx = fmaxf(mx, s_m[w][row]);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float mw = s_m[w][row];
          if (mw == -INFINITY && s_l[w][row] == 0.f) continue;  // saw no key: its sums may not be there
          const float f = exp2f((mw - mx) * sl2);
          ls += f * s_l[w][row];
          const uint32_t at = s_at[w] + row * (D * 4) + ((piece ^ (row & 7)) << 5);
          const float4 p = lds_f4(at), q = lds_f4(at + 16);
          acc[0] += f * p.x; acc[1] += f * p.y; acc[2] += f * p.z; acc[3] += f * p.w;
          acc[4] += f * q.x; acc[5] += f * q.y; acc[6] += f * q.z; acc[7] += f * q.w;
        }
      }
      fence_proxy_async_smem();
      bool write = true;
      if (cc.cut()) {
        // shared with other CTAs: leave the partial result; the last to arrive joins them
        const PagedShares sh = shares_of(cc, total, ctas, u1);
        float* slot = a.ws + (size_t)part_slot(blockIdx.x, cc.first == 0) * kSlotFloats<D>;
        if (mine_out) {
          float4* d = reinterpret_cast<float4*>(slot + row * D + piece * 8);
          d[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
          d[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
          if (piece == 0) {
            slot[kRows * D + row] = mx;
            slot[kRows * D + kRows + row] = ls;
          }
        }
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) s_last = atomicAdd(&a.cnt[sh.c0], 1u) == sh.c1 - sh.c0;
        __syncthreads();
        write = s_last != 0;
        if (write) {
          __threadfence();
          if (threadIdx.x == 0) a.cnt[sh.c0] = 0u;  // ready for the next call
          if (mine_out) {
            // kParts parts' loads are on their way at once (one after the other, 19 parts
            // of a sequence over the whole GPU took 15 us, now 4)
            constexpr int kParts = 8;
            mx = -INFINITY;
            ls = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) acc[k] = 0.f;
            for (unsigned c = sh.c0; c <= sh.c1; c += kParts) {
              float pm[kParts], pl[kParts];
              float4 v[kParts], w[kParts];
#pragma unroll
              for (int i = 0; i < kParts; ++i) {
                const unsigned ci = min(c + i, sh.c1);
                const float* p = a.ws + (size_t)part_slot(ci, ci == sh.c0) * kSlotFloats<D>;
                pm[i] = __ldcg(p + kRows * D + row);
                pl[i] = __ldcg(p + kRows * D + kRows + row);
                v[i] = __ldcg(reinterpret_cast<const float4*>(p + row * D + piece * 8));
                w[i] = __ldcg(reinterpret_cast<const float4*>(p + row * D + piece * 8 + 4));
              }
#pragma unroll
              for (int i = 0; i < kParts; ++i) {
                if (c + i > sh.c1 || (pm[i] == -INFINITY && pl[i] == 0.f)) continue;
                const float nm = fmaxf(mx, pm[i]), f = mx == -INFINITY ? 0.f : exp2f((mx - nm) * sl2), e = exp2f((pm[i] - nm) * sl2);
                mx = nm;
                ls = ls * f + pl[i] * e;
                acc[0] = acc[0] * f + v[i].x * e; acc[1] = acc[1] * f + v[i].y * e;
                acc[2] = acc[2] * f + v[i].z * e; acc[3] = acc[3] * f + v[i].w * e;
                acc[4] = acc[4] * f + w[i].x * e; acc[5] = acc[5] * f + w[i].y * e;
                acc[6] = acc[6] * f + w[i].z * e; acc[7] = acc[7] * f + w[i].w * e;
              }
            }
          }
        }
      }
      if (write && mine_out) {
        const int r = cc.t * kRows + row, of = over_group(a, r);
        const int64_t tok = cc.q0 + of;
        const int head = cc.h * a.group + r - of * a.group;
        const float inv = ls == 0.f ? 0.f : 1.f / ls;  // (a sum of NaN stays one)
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[k] *= inv;
        *reinterpret_cast<uint4*>(a.y + (tok * a.heads + head) * D + piece * 8) = pack8(acc);
        if (a.lse && piece == 0)
          a.lse[tok * a.heads + head] = ls == 0.f ? -INFINITY : fmaf(mx, a.unit, logf(ls));
      }
      __syncthreads();  // the free stages may be filled, s_m, s_l and s_at written again
      fresh = true;
    }
  }
  // after a timeout: no copy is in flight into shared memory that is given back
  if (dead)
    for (unsigned i = used; i < issued; ++i) mbar_drain(smem_u32(&s_bar[warp][i % S]), (i / S) & 1u, limit);
}

bool few_rows(const PagedArgs& a) { return (int64_t)a.max_q * a.group <= kRows; }

int grid_of() {
  const int sms = device_sm_count();
  return sms < kPagedCounters ? sms : kPagedCounters;
}
size_t small_ws_bytes() { return (size_t)2 * kPagedCounters * kSlotFloats<128> * sizeof(float); }

template <int D, int RULES>
cudaError_t launch_small(const PagedArgs& a, cudaStream_t s) {
  CUtensorMap tk, tv;
  const uint64_t rows = (uint64_t)a.pages * a.kv_heads << a.page_log2;
  if (!make_tmap_2d(&tk, a.k, rows, D, 64, kKeys) || !make_tmap_2d(&tv, a.v, rows, D, 64, kKeys))
    return cudaErrorInvalidValue;
  const cudaError_t e = smem_optin(reinterpret_cast<const void*>(paged_small_kernel<D, RULES>), Cfg<D>::kSmem);
  if (e != cudaSuccess) return e;
  return launch_kernel(paged_small_kernel<D, RULES>, dim3(grid_of()), dim3(kThreads), Cfg<D>::kSmem, s, tk, tv, a);
}

template <int D>
cudaError_t launch_by_rules(const PagedArgs& a, cudaStream_t s) {
  switch (rules_of(a)) {
    case kPlain: return launch_small<D, kPlain>(a, s);
    case kRuled: return launch_small<D, kRuled>(a, s);
    case kRuled | kCap: return launch_small<D, kRuled | kCap>(a, s);
    case kRuled | kBias: return launch_small<D, kRuled | kBias>(a, s);
    case kRuled | kCap | kBias: return launch_small<D, kRuled | kCap | kBias>(a, s);
    case kRuled | kTree: return launch_small<D, kRuled | kTree>(a, s);
  }
  return launch_small<D, kRuled | kCap | kBias | kTree>(a, s);
}

}  // namespace

int rules_of(const PagedArgs& a) {
  if (!a.ruled) return kPlain;
  const int changes = (a.cap > 0.f ? kCap : 0) | (a.slopes ? kBias : 0);
  if (!a.tree) return kRuled | changes;
  return kRuled | kTree | (changes ? kCap | kBias : 0);
}

size_t paged_ws_bytes() {
  const size_t small = small_ws_bytes(), chunk = paged_chunk_ws_bytes();
  return small > chunk ? small : chunk;
}
size_t paged_ws_bytes(const PagedArgs& a) { return few_rows(a) ? small_ws_bytes() : paged_chunk_ws_bytes(); }

cudaError_t launch_paged_attention(const PagedArgs& a, cudaStream_t s) {
  if (!few_rows(a)) return launch_paged_chunk(a, s);
  return a.D == 128 ? launch_by_rules<128>(a, s) : launch_by_rules<64>(a, s);
}

}  // namespace sparoa
