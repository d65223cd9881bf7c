// Work plan of attention over a paged cache, shared by its kernels.
//
// An item is one tile of ROWS query rows of one sequence and key head (row r of a
// sequence: token r / group, query head key_head * group + r % group).  Its keys are
// walked in units of 128; its cost is a weight for each and EXTRA for its beginning and
// end, in steps that a kernel's Cut states as measured.  The costs of all items, in the
// order (sequence, key head, tile), form one line that the CTAs cut into equal shares:
// every CTA has as much to do as any other, however ragged the batch, and at most its
// first and last item are shared with other CTAs.  Shares are MIN_SHARE at least, which is
// no less than a unit, so that no CTA between two others of an item has none of it.  Where
// the shares are shorter than
// WHOLE_SHARE, an item not much longer than one is not cut but goes to the CTA in whose
// share it begins: joining its parts would take longer than they do.  Lengths are on the
// device, so every CTA makes the plan itself (a load per sequence and a scan).
#pragma once

#include "sparoa_kernels.h"

namespace sparoa {

constexpr int kUnitKeys = 128;

// The batch in shared memory: first row, new tokens and cached tokens of each sequence,
// and until the CTAs have found their shares its cost per key head (SCRATCH bytes to use
// afterwards).
template <int SCRATCH = 16>
struct PagedPlan {
  int q0[kPagedMaxBatch], n[kPagedMaxBatch], len[kPagedMaxBatch];
  unsigned long long total;
  union alignas(16) {
    unsigned long long cost[kPagedMaxBatch];
    uint8_t scratch[SCRATCH];
  };
};

// Keys [lo, hi) that some row of tile t may see; hi <= lo: none.  units >= 1, so that
// rows without keys are still written.
struct TileKeys {
  int lo, hi, blk0, units;
};

// row / group for rows below 2^31 (the host's multiplier, see PagedArgs)
__device__ __forceinline__ int over_group(const PagedArgs& a, int row) {
  return a.group == 1 ? row : (int)(__umulhi((unsigned)row, a.group_mul) >> a.group_shift);
}

template <typename Cut>
__device__ __forceinline__ int tiles_of(int n, int group) {
  return (n * group + Cut::ROWS - 1) / Cut::ROWS;  // (n * group is at most 2^30)
}

// First key that the token at position p sees (no overflow: windows reach 2^31 - 1, and
// tokens before the sequence's first position are negative).
__device__ __forceinline__ int first_seen(const PagedArgs& a, int p) {
  return a.window > 0 && p + 1 > a.window ? p + 1 - a.window : 0;
}

template <typename Cut>
__device__ __forceinline__ TileKeys tile_keys(const PagedArgs& a, int n, int len, int t) {
  constexpr int RT = Cut::ROWS;
  TileKeys k;
  k.hi = len;
  if (a.causal) {
    const int last = over_group(a, min(n * a.group, (t + 1) * RT) - 1);
    k.hi = max(0, min(len, len - n + last + 1));
  }
  k.lo = first_seen(a, len - n + over_group(a, t * RT));
  k.blk0 = k.lo / kUnitKeys;
  k.units = max(1, (k.hi + kUnitKeys - 1) / kUnitKeys - k.blk0);
  return k;
}

// Cost of tile t.
template <typename Cut>
__device__ __forceinline__ int tile_cost(const PagedArgs& a, int n, int len, int t) {
  return tile_keys<Cut>(a, n, len, t).units * Cut::weight(n * a.group - t * Cut::ROWS) + Cut::EXTRA;
}

// Fills the plan (all threads of the CTA; ends with a block barrier).  What the lists
// say is brought into the tensors' bounds; where it is not there already, the error
// bit is set.
template <typename Cut, typename Plan>
__device__ __forceinline__ void make_plan(const PagedArgs& a, Plan& p) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  if (threadIdx.x == 0) p.total = 0ull;
  __syncthreads();
  bool many = false;
  const long long room = (long long)a.max_pages << a.page_log2;
  unsigned long long sum = 0ull;
  for (int b = threadIdx.x; b < a.batch; b += blockDim.x) {
    long long q0 = a.q_start[b], n = (long long)a.q_start[b + 1] - q0, len = a.kv_len[b];
    const bool bad_rows = q0 < 0 || n < 0 || q0 + n > a.T || n * a.group > 0x3FFFFFFF;
    if (bad_rows || len < 0 || len > room) {
      atomicOr(a.err, kErrBadIndex);
      if (bad_rows) n = 0;
      len = len < 0 ? 0 : min(len, room);
    }
    const int tiles = tiles_of<Cut>((int)n, a.group);
    p.q0[b] = (int)q0;
    p.n[b] = (int)n;
    p.len[b] = (int)len;
    p.cost[b] = tiles == 1 ? (unsigned long long)tile_cost<Cut>(a, (int)n, (int)len, 0) : 0ull;
    many |= tiles > 1;
    sum += p.cost[b] * a.kv_heads;
  }
  if (__syncthreads_or(many)) {
    for (int b = warp; b < a.batch; b += warps) {
      const int n = p.n[b], len = p.len[b], tiles = tiles_of<Cut>(n, a.group);
      if (tiles <= 1) continue;
      unsigned long long u = 0ull;
      for (int t = lane; t < tiles; t += 32) u += (unsigned long long)tile_cost<Cut>(a, n, len, t);
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) u += __shfl_xor_sync(0xffffffffu, u, d);
      if (lane == 0) {
        p.cost[b] = u;
        sum += u * a.kv_heads;
      }
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (lane == 0 && sum) atomicAdd(&p.total, sum);
  __syncthreads();
}

// a / b, by a 32-bit division where they allow it (a 64-bit one takes 200 cycles)
__device__ __forceinline__ unsigned long long quotient(unsigned long long a, unsigned long long b) {
  return (a >> 32) == 0ull && (b >> 32) == 0ull ? (unsigned)a / (unsigned)b : a / b;
}
// A walk over one CTA's share of the line, the same in all lanes of a warp.
template <typename Cut>
struct PagedCursor {
  int b, h, t, tiles;
  int q0, n, len;
  TileKeys k;
  int weight;        // of a unit of the item
  int pos, left;     // where the share enters the item's cost, and the share's cost from there
  int whole;         // items of at most this cost are not cut
  int first, end;    // the share's units of the item
  int blk;           // unit, first to end - 1; at `end`: nothing left

  __device__ __forceinline__ bool done() const { return blk >= end; }
  __device__ __forceinline__ int key0() const { return (k.blk0 + blk) * kUnitKeys; }
  // whether other CTAs have units of the item
  __device__ __forceinline__ bool cut() const { return first > 0 || end < k.units; }

  template <typename Plan>
  __device__ __forceinline__ void load_seq(const PagedArgs& a, const Plan& p) {
    q0 = p.q0[b];
    n = p.n[b];
    len = p.len[b];
    tiles = tiles_of<Cut>(n, a.group);
  }
  // a unit belongs to the share that has the first step of its cost
  __device__ __forceinline__ int unit_at(int at) const { return max(0, at - Cut::EXTRA + weight - 1) / weight; }
  __device__ __forceinline__ void enter(const PagedArgs& a) {
    k = tile_keys<Cut>(a, n, len, t);
    weight = Cut::weight(n * a.group - t * Cut::ROWS);
    if (cost() <= whole) {
      first = pos == 0 ? 0 : k.units;
      end = k.units;
    } else {
      first = unit_at(pos);
      end = min(k.units, unit_at(pos + left));
    }
    blk = first;
  }
  __device__ __forceinline__ int cost() const { return k.units * weight + Cut::EXTRA; }
  // to position u < total of the line, `steps` of which are to be walked (a converged warp)
  template <typename Plan>
  __device__ __forceinline__ void seek(const PagedArgs& a, const Plan& p, unsigned ctas, unsigned long long u, int steps) {
    const int lane = threadIdx.x & 31;
    unsigned long long before = 0ull;  // cost of the sequences before b0
    int b0 = 0;
    for (;; b0 += 32) {
      const unsigned long long mine = b0 + lane < a.batch ? p.cost[b0 + lane] * a.kv_heads : 0ull;
      unsigned long long incl = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const unsigned long long o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
      }
      const unsigned hit = __ballot_sync(0xffffffffu, before + incl > u);
      if (hit || b0 + 32 >= a.batch) {
        const int l = hit ? __ffs(hit) - 1 : 31;
        b = b0 + l;
        before += __shfl_sync(0xffffffffu, incl - mine, l);
        break;
      }
      before += __shfl_sync(0xffffffffu, incl, 31);
    }
    load_seq(a, p);
    const unsigned long long per = p.cost[b];
    unsigned long long rem = u - before;
    h = (int)quotient(rem, per);
    rem -= h * per;
    t = 0;
    if (tiles > 1) {
      for (int t0 = 0;; t0 += 32) {
        const unsigned mine = t0 + lane < tiles ? (unsigned)tile_cost<Cut>(a, n, len, t0 + lane) : 0u;
        unsigned incl = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const unsigned o = __shfl_up_sync(0xffffffffu, incl, d);
          if (lane >= d) incl += o;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, incl > rem);
        if (hit || t0 + 32 >= tiles) {
          const int l = hit ? __ffs(hit) - 1 : 31;
          t = t0 + l;
          rem -= __shfl_sync(0xffffffffu, incl - mine, l);
          break;
        }
        rem -= __shfl_sync(0xffffffffu, incl, 31);
      }
    }
    pos = (int)rem;
    left = steps;
    whole = p.total < (unsigned long long)Cut::WHOLE_SHARE * ctas ? (int)quotient(p.total, ctas) + Cut::WHOLE_MORE : 0;
    enter(a);
    if (done()) next_item(a, p);
  }
  // to the share's next item that has units of it, if any (done() afterwards: none)
  template <typename Plan>
  __device__ __forceinline__ void next_item(const PagedArgs& a, const Plan& p) {
    for (;;) {
      left -= cost() - pos;
      if (left <= 0) {
        blk = end;
        return;
      }
      if (++t == tiles) {
        t = 0;
        if (++h == a.kv_heads) {
          h = 0;
          do ++b; while (p.n[b] == 0);  // (the line goes on: there is such a sequence)
          load_seq(a, p);
        }
      }
      pos = 0;
      enter(a);
      if (!done()) return;
    }
  }
  template <typename Plan>
  __device__ __forceinline__ void next(const PagedArgs& a, const Plan& p) {
    if (++blk >= end) next_item(a, p);
  }
};

// CTAs that get a share.
template <typename Cut>
__device__ __forceinline__ unsigned cut_ctas(unsigned long long total) {
  return total < Cut::MIN_SHARE ? (unsigned)(total > 0) : (unsigned)min((unsigned long long)gridDim.x, quotient(total, Cut::MIN_SHARE));
}
// The line's cut: CTA c of `ctas` has positions [c total / ctas, (c + 1) total / ctas).
__device__ __forceinline__ unsigned long long cut_start(unsigned long long total, unsigned ctas, unsigned c) {
  return quotient(total * c, ctas);
}
// the CTA that has position u
__device__ __forceinline__ unsigned cut_owner(unsigned long long total, unsigned ctas, unsigned long long u) {
  return (unsigned)quotient((u + 1) * ctas - 1, total);
}
// The CTAs that have the first and the last unit of the item of place c, whose share ends
// at position `until`.
struct PagedShares {
  unsigned c0, c1;
};
template <typename Cut>
__device__ __forceinline__ PagedShares shares_of(const PagedCursor<Cut>& c, unsigned long long total, unsigned ctas,
                                                 unsigned long long until) {
  const unsigned long long first = until - c.left - c.pos + Cut::EXTRA;
  PagedShares s;
  s.c0 = cut_owner(total, ctas, first);
  s.c1 = cut_owner(total, ctas, first + (unsigned long long)(c.k.units - 1) * c.weight);
  return s;
}
// Where CTA c leaves its part of an item: a CTA has at most one part that another began
// (its first item's end) and one that another ends (its last item's beginning).
__device__ __forceinline__ unsigned part_slot(unsigned c, bool begins) { return 2u * c + (begins ? 1u : 0u); }

// The table's entry for key `key` of sequence b, as it is (loaded ahead of its use).
__device__ __forceinline__ int page_of(const PagedArgs& a, int b, int key) {
  return a.table[b * a.table_stride + (key >> a.page_log2)];
}
// The page of an entry, brought into the pool's bounds.
__device__ __forceinline__ int page_checked(const PagedArgs& a, int page) {
  if (page >= 0 && page < a.pages) return page;
  atomicOr(a.err, kErrBadIndex);
  return 0;
}
// Row of the pool [pages * kv_heads * page_size][D] that holds key `key` of key head h.
__device__ __forceinline__ int pool_row(const PagedArgs& a, int page, int h, int key) {
  return (int)(((long long)page * a.kv_heads + h) << a.page_log2) + (key & ((1 << a.page_log2) - 1));
}

}  // namespace sparoa
