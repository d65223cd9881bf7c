// Trees of drafted tokens after the model has judged them: the path that its own choices
// confirm, and the path's keys and values in the places that follow one another.
//
// Bound by latency: the kept tokens' rows are a few KB a layer.  One launch for all layers: a
// CTA per sequence, cache and 256 pieces of 16 bytes of a token's row finds the path itself (a
// warp, two tokens a lane, a vote per step) and then moves its pieces of every kept token.
// A kept token never moves up, and the path is walked in its order, so a place is written
// only after what it held was read: a thread moves the same piece of all tokens.
//
// 64 trees of 25 tokens in four layers' caches, 8 key heads of 128: 3.6 us on the device,
// one tree of 7 in two layers 2.5, of which a launch is 2; a call from Python takes 7.
#include "sparoa_kernels.h"

namespace sparoa {

namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 8;  // tokens that a thread has on their way

// CACHES: pools that the arguments have room for.  Two KB of arguments take the host and the GPU a
// microsecond and more of a call: with room for 8 caches 7.1 us, for 128 8.4 (two caches).
template <int CACHES>
struct Pools {
  void *k[CACHES], *v[CACHES];
};

template <int CACHES>
__global__ void __launch_bounds__(kThreads) tree_accept_kernel(const __grid_constant__ TreeArgs a, const __grid_constant__ Pools<CACHES> pools) {
  __shared__ int s_from[kTreeTokens], s_to[kTreeTokens];  // rows of the pool (key head 0), -1: not there
  __shared__ int s_path[kTreeTokens], s_best[kTreeTokens];
  __shared__ int s_count;
  const int b = blockIdx.x, lane = threadIdx.x & 31;
  pdl_wait();
  pdl_trigger();
  const long long q0 = a.q_start[b], n = (long long)a.q_start[b + 1] - q0, len = a.kv_len[b];
  const long long room = (long long)a.max_pages << a.page_log2;
  const bool bad = q0 < 0 || n < 0 || n > kTreeTokens || q0 + n > a.T || len < 0 || len > room;
  const bool tells = blockIdx.y == 0 && blockIdx.z == 0;  // the one of the sequence's CTAs that writes the lists
  if (threadIdx.x < 32) {
    int count = 0;
    if (bad) {
      if (lane == 0) atomicOr(a.err, kErrBadIndex);
    } else if (n > 0) {
      unsigned long long all[2], above[2];
      int token[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int node = lane + 32 * i;
        const bool there = node < n;
        const unsigned long long own = 1ull << node;
        above[i] = there ? a.tree[q0 + node] & (own - 1ull) : 0ull;
        all[i] = above[i] | own;
        token[i] = there ? a.tokens[q0 + node] : -1;
        s_best[node] = there ? a.best[q0 + node] : -1;
      }
      __syncwarp();
      int at = 0;
      for (;;) {
        if (lane == 0) s_path[count] = at;
        ++count;
        const unsigned long long way = __shfl_sync(0xffffffffu, at < 32 ? all[0] : all[1], at & 31);
        const int best = s_best[at];
        const unsigned lo = __ballot_sync(0xffffffffu, best >= 0 && above[0] == way && token[0] == best);
        const unsigned hi = __ballot_sync(0xffffffffu, best >= 0 && above[1] == way && token[1] == best);
        if (!(lo | hi)) break;
        at = lo ? __ffs(lo) - 1 : 31 + __ffs(hi);  // (behind the token before: its ancestors have lower numbers)
      }
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int k = lane + 32 * i;
        if (k < count) {
          const long long base = len - n;
          auto row_of = [&](long long place) {
            if (place < 0) return -1;  // (a token before its sequence's first position was not cached)
            const int page = a.table[b * a.table_stride + (place >> a.page_log2)];
            if (page >= 0 && page < a.pages) return (int)((((long long)page * a.kv_heads) << a.page_log2) + (place & ((1 << a.page_log2) - 1)));
            atomicOr(a.err, kErrBadIndex);
            return -1;
          };
          s_from[k] = s_path[k] == k ? -1 : row_of(base + s_path[k]);
          s_to[k] = s_path[k] == k ? -1 : row_of(base + k);
        }
      }
    }
    if (lane == 0) s_count = count;
  }
  __syncthreads();
  const int count = s_count;
  if (tells) {
    if (!bad)
      for (int i = threadIdx.x; i < n; i += kThreads) a.path[q0 + i] = i < count ? s_path[i] : -1;
    if (threadIdx.x == 0) {
      a.count[b] = count;
      a.following[b] = count ? s_best[s_path[count - 1]] : -1;
      a.new_len[b] = bad ? a.kv_len[b] : (int)(len - n + count > 0 ? len - n + count : 0);
    }
  }
  const int c = blockIdx.z * kThreads + threadIdx.x, pieces = a.D / 8, each = a.kv_heads * pieces;
  if (c >= 2 * each) return;
  const int head = c % each / pieces;
  uint4* pool = reinterpret_cast<uint4*>(c < each ? pools.k[blockIdx.y] : pools.v[blockIdx.y]) +
                ((int64_t)head << a.page_log2) * pieces + c % pieces;
  for (int k0 = 0; k0 < count; k0 += kAhead) {
    uint4 u[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (k0 + i < count && s_from[k0 + i] >= 0) u[i] = pool[(int64_t)s_from[k0 + i] * pieces];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (k0 + i < count && s_from[k0 + i] >= 0 && s_to[k0 + i] >= 0) pool[(int64_t)s_to[k0 + i] * pieces] = u[i];
  }
}

template <int CACHES>
cudaError_t launch(const TreeArgs& a, void* const* k, void* const* v, cudaStream_t s) {
  Pools<CACHES> pools;
  for (int i = 0; i < CACHES; ++i) {
    pools.k[i] = i < a.caches ? k[i] : nullptr;
    pools.v[i] = i < a.caches ? v[i] : nullptr;
  }
  const int parts = (2 * a.kv_heads * a.D / 8 + kThreads - 1) / kThreads;
  return launch_kernel(tree_accept_kernel<CACHES>, dim3((unsigned)a.batch, (unsigned)a.caches, (unsigned)parts), dim3(kThreads), 0, s, a, pools);
}

}  // namespace

cudaError_t launch_tree_accept(const TreeArgs& a, void* const* k, void* const* v, cudaStream_t s) {
  if (a.caches <= 8) return launch<8>(a, k, v, s);
  return a.caches <= 32 ? launch<32>(a, k, v, s) : launch<kTreeCaches>(a, k, v, s);
}

}  // namespace sparoa
