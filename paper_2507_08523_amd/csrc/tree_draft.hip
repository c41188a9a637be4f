// Trees of drafted tokens, for gfx950: ancestor masks (what the attention of a tree
// reads), the accepted path, and the K/V rows of that path moved to the front.
//
// A request of P context tokens has n drafted ones, node 0 .. n-1, appended to its
// cache at the positions P + i (InferLog section 2.1.2: the newest tokens attend to
// the cached KV of their context).  Node i continues node parent[i] < i, or the
// context (-1):
//   m_i = 2^i | m_parent(i),   depth_i = |m_i| - 1,
// bit j of m_i set where node i sees node j.  The target model picks a token behind
// every node; from the root on, a node is accepted whose token is the pick behind its
// parent.  A path p_0 < p_1 < ... of accepted nodes has p_i >= i, so its rows go to
// the positions P + i one after the other without a row being overwritten that is
// still to be read.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/ilpc.h"
#include "ilpc_internal.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 16;
constexpr int kMaxWords = 16;  // words of 64 nodes: a wave each
constexpr int kMaxRequests = 1 << 20;

// Rows of request r, [*q0, *q0 + n): n = 0 where they are not all in the buffers.
__device__ __forceinline__ int rows_of(const int32_t* cu_q, int r, int n_rows, int* q0) {
  const int a = cu_q[r], b = cu_q[r + 1];
  *q0 = a;
  return a >= 0 && b <= n_rows && b > a ? b - a : 0;
}

// One workgroup a request, a wave for each 64 nodes.  Within a wave's nodes ancestors
// are gathered by doubling (each node takes over the bits of the node it points at, and
// then that node's pointer: 6 steps for 64 generations); `top` is the first ancestor
// outside of them, from which a node goes on in the words below.  Bound by the launch
// and one round trip: 1.5 us for a tree of 64, 3.1 for 512 of 90 to 160 nodes in 3 words.
__global__ void tree_masks_kernel(const int32_t* __restrict__ parents, const int32_t* __restrict__ cu_q,
                                  const int32_t* __restrict__ start_pos, int n_rows, int words,
                                  uint64_t* __restrict__ masks, int32_t* __restrict__ positions) {
  __shared__ uint64_t s_bits[64 * kMaxWords];
  __shared__ int s_top[64 * kMaxWords];
  const int r = blockIdx.x, i = threadIdx.x, lane = i & 63, base = i & ~63, cap = words * 64;
  int q0;
  const int n = rows_of(cu_q, r, n_rows, &q0);
  const int start = positions && start_pos ? start_pos[r] : 0;
  const int given = i < n ? parents[q0 + i] : -1;
  const int p = given >= 0 && given < i ? given : -1;  // (anything else sees itself alone)
  uint64_t bits = 1ull << lane;
  int jump = p >= base ? p - base : lane;
#pragma unroll
  for (int k = 0; k < 6; ++k) {
    bits |= __shfl(bits, jump);
    jump = __shfl(jump, jump);
  }
  const int top = __shfl(p, jump);
  int depth = -1;
  uint64_t* row = masks + size_t(q0 + i) * words;
  if (words == 1) {
    if (i < n) *row = bits;
    depth += __popcll(bits);
  } else {
    s_bits[i] = bits;
    s_top[i] = top;
    __syncthreads();
    int u = i;
    for (int w = words - 1; w >= 0; --w) {
      uint64_t x = 0;
      if (u >= 0 && u >> 6 == w) {
        x = s_bits[u];
        u = s_top[u];
        depth += __popcll(x);
      }
      if (i < n) row[w] = x;
    }
  }
  if (positions && i < n) positions[q0 + i] = start + depth;
  // nodes that the words have no bits for see no node
  for (int k = cap + i; k < n; k += cap) {
    for (int w = 0; w < words; ++w) masks[size_t(q0 + k) * words + w] = 0;
    if (positions) positions[q0 + k] = start;
  }
}

// One wave a request: the nodes of kAhead * 64 at a time in registers, and a ballot a
// step for the first child of the last accepted node that has the token wanted.  Later
// nodes are looked at once the ones before hold no such child: children follow their
// parents.  Bound by round trips, to the lengths and then to the nodes (all of a chunk's at once):
// 3.2 us for 4 trees of 48 to 64, 4.7 for 512 of 12 to 32; a step of the path is registers only.
constexpr int kAhead = 4;

__global__ __launch_bounds__(64) void tree_accept_kernel(
    const int32_t* __restrict__ parents, const int32_t* __restrict__ tokens, const int32_t* __restrict__ targets,
    const int32_t* __restrict__ root_targets, const int32_t* __restrict__ cu_q, const int32_t* __restrict__ start_pos,
    int n_rows, int32_t* __restrict__ path, int32_t* __restrict__ n_accepted, int32_t* __restrict__ next_tokens,
    int32_t* __restrict__ kept_lens, int32_t* __restrict__ kept_blocks) {
  const int r = blockIdx.x, lane = threadIdx.x;
  int q0;
  const int rows = rows_of(cu_q, r, n_rows, &q0), start = start_pos[r];
  const int n = start < 0 ? 0 : rows;  // (no draft: nothing is accepted, and nothing cut)
  int want = root_targets ? root_targets[r] : -1, cur = -1, count = 0;
  bool any_token = !root_targets;  // of the root: node 0, whatever its token
  for (int b0 = 0; b0 < n; b0 += 64 * kAhead) {
    int par[kAhead], tok[kAhead], pick[kAhead];
#pragma unroll
    for (int c = 0; c < kAhead; ++c) {
      const int i = b0 + c * 64 + lane, at = q0 + min(i, n - 1);
      par[c] = parents[at], tok[c] = tokens[at], pick[c] = targets[at];
      if (i >= n || par[c] < -1 || par[c] >= i) par[c] = -2;
    }
    while (true) {
      int found = -1, behind = 0;
#pragma unroll
      for (int c = kAhead - 1; c >= 0; --c) {
        const int i = b0 + c * 64 + lane;
        const uint64_t m = __ballot(par[c] == cur && (any_token ? i == 0 : tok[c] == want));
        if (m) {
          const int l = __builtin_ctzll(m);
          found = b0 + c * 64 + l;
          behind = __builtin_amdgcn_readlane(pick[c], l);
        }
      }
      if (found < 0) break;
      if (lane == 0) path[q0 + count] = found;
      ++count;
      cur = found;
      want = behind;
      any_token = false;
    }
    if (any_token) break;
  }
  for (int i = count + lane; i < rows; i += 64) path[q0 + i] = -1;
  if (lane == 0) {
    n_accepted[r] = count;
    next_tokens[r] = want;
    kept_lens[r] = start < 0 ? INT32_MAX : start + count;
    kept_blocks[r] = start < 0 ? INT32_MAX : (start + count + kBlock - 1) / kBlock;
  }
}

// One wave a (request, kv head), so that all of a batch's are resident at once; 64 rows of the path
// at a time, one a lane, with the block table's entries behind the start, one a lane as well; and of
// the rows that move kMoved at a time read into registers, then written: the K row in 16-byte
// pieces, the V row one dimension a lane (V blocks are dimension-major).  Bound by V, of which a
// row's 2 bytes a dimension move whole lines: 512 requests of 12 to 32 nodes, 8 kv heads of D 128 10.7 us; few
// requests 3.9, three dependent round trips (count and path, table, rows) and a launch.
constexpr int kMoved = 8;

template <int D>
__global__ __launch_bounds__(64) void compact_kernel(uint16_t* k_pool, uint16_t* v_pool, int num_blocks,
                                                     const int32_t* __restrict__ block_tables, int max_blocks,
                                                     const int32_t* __restrict__ cu_q,
                                                     const int32_t* __restrict__ start_pos, int n_rows,
                                                     const int32_t* __restrict__ path,
                                                     const int32_t* __restrict__ n_accepted, int Hkv) {
  constexpr int kPieces = D / 8, kAtOnce = 64 / kPieces;  // pieces of a K row, rows of K that the lanes take at once
  const int r = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
  int q0;
  const int n = rows_of(cu_q, r, n_rows, &q0), start = start_pos[r], count = min(n_accepted[r], n);
  if (start < 0) return;
  const int32_t* bt = block_tables + size_t(r) * max_blocks;
  const int lb0 = start / kBlock;
  const int window = bt[min(lb0 + lane, max_blocks - 1)];
  auto place = [&](int64_t pos) -> int64_t {  // block * 16 + offset, or -1
    const int64_t lb = pos / kBlock, w = lb - lb0;
    const int near = __shfl(window, int(w & 63));
    const int id = lb >= max_blocks ? -1 : w < 64 ? near : bt[lb];
    return id >= 0 && id < num_blocks ? int64_t(id) * kBlock + pos % kBlock : -1;
  };
  for (int i0 = 0; i0 < count; i0 += 64) {
    const int i = i0 + lane, p = i < count ? path[q0 + i] : -1;
    const int64_t src = place(int64_t(start) + max(p, 0)), dst = place(int64_t(start) + i);
    uint64_t moves = __ballot(p > i && p < n && src >= 0 && dst >= 0);
    while (moves) {
      const int rows = min(__popcll(moves), kMoved);
      int row[kMoved];  // lanes of the rows that move now
#pragma unroll
      for (int k = 0; k < kMoved; ++k) {
        row[k] = moves ? __builtin_ctzll(moves) : 0;
        moves &= moves - 1;
      }
      u32x4 kv[kMoved / kAtOnce];
      int64_t to[kMoved / kAtOnce];
#pragma unroll
      for (int k = 0; k < kMoved / kAtOnce; ++k) {
        int l = row[k * kAtOnce];
#pragma unroll
        for (int e = 1; e < kAtOnce; ++e) l = lane / kPieces == e ? row[k * kAtOnce + e] : l;
        const int64_t s = __shfl(src, l);
        to[k] = __shfl(dst, l);
        if (k * kAtOnce + lane / kPieces < rows)
          kv[k] = *(const u32x4*)(k_pool + ((s / kBlock * Hkv + h) * kBlock + s % kBlock) * D + lane % kPieces * 8);
      }
      uint16_t v[kMoved][D / 64];
#pragma unroll
      for (int k = 0; k < kMoved; ++k)
        if (k < rows) {
          const int64_t s = __shfl(src, row[k]);
#pragma unroll
          for (int e = 0; e < D / 64; ++e)
            v[k][e] = v_pool[((s / kBlock * Hkv + h) * D + e * 64 + lane) * kBlock + s % kBlock];
        }
      // all rows have arrived before the first one is written (by other lanes than read it)
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
      for (int k = 0; k < kMoved / kAtOnce; ++k)
        if (k * kAtOnce + lane / kPieces < rows)
          *(u32x4*)(k_pool + ((to[k] / kBlock * Hkv + h) * kBlock + to[k] % kBlock) * D + lane % kPieces * 8) = kv[k];
#pragma unroll
      for (int k = 0; k < kMoved; ++k)
        if (k < rows) {
          const int64_t t = __shfl(dst, row[k]);
#pragma unroll
          for (int e = 0; e < D / 64; ++e)
            v_pool[((t / kBlock * Hkv + h) * D + e * 64 + lane) * kBlock + t % kBlock] = v[k][e];
        }
      asm volatile("" ::: "memory");
    }
  }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int launch_status(const char* fn) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ILPC_OK : ilpc::set_error(ILPC_EHIP, "%s: launch failed: %s", fn, hipGetErrorString(e));
}

}  // namespace

extern "C" int ilpc_tree_masks(const int32_t* parents, const int32_t* cu_q, const int32_t* start_pos, int32_t B,
                               int32_t n_rows, int32_t mask_words, uint64_t* masks, int32_t* positions, void* stream) {
  static const char* fn = "ilpc_tree_masks";
  using ilpc::set_error;
  if (B < 0 || n_rows < 0 || mask_words < 1) return set_error(ILPC_EINVAL, "%s: negative or zero size", fn);
  if (B > kMaxRequests || mask_words > kMaxWords)
    return set_error(ILPC_EUNSUP, "%s: B %d or mask_words %d too large", fn, B, mask_words);
  if (B == 0 || n_rows == 0) return ILPC_OK;
  if (!parents || !cu_q || !masks) return set_error(ILPC_EINVAL, "%s: NULL pointer", fn);
  if (reinterpret_cast<uintptr_t>(masks) & 7u) return set_error(ILPC_EINVAL, "%s: masks must be 8-byte aligned", fn);
  hipLaunchKernelGGL(tree_masks_kernel, dim3(B), dim3(64 * mask_words), 0, static_cast<hipStream_t>(stream), parents,
                     cu_q, start_pos, n_rows, mask_words, masks, positions);
  return launch_status(fn);
}

extern "C" int ilpc_tree_accept(const int32_t* parents, const int32_t* tokens, const int32_t* targets,
                                const int32_t* root_targets, const int32_t* cu_q, const int32_t* start_pos, int32_t B,
                                int32_t n_rows, int32_t* path, int32_t* n_accepted, int32_t* next_tokens,
                                int32_t* kept_lens, int32_t* kept_blocks, void* stream) {
  static const char* fn = "ilpc_tree_accept";
  using ilpc::set_error;
  if (B < 0 || n_rows < 0) return set_error(ILPC_EINVAL, "%s: negative size", fn);
  if (B > kMaxRequests) return set_error(ILPC_EUNSUP, "%s: B %d too large", fn, B);
  if (B == 0) return ILPC_OK;
  if (!cu_q || !start_pos || !n_accepted || !next_tokens || !kept_lens || !kept_blocks ||
      (n_rows && (!parents || !tokens || !targets || !path)))
    return set_error(ILPC_EINVAL, "%s: NULL pointer", fn);
  hipLaunchKernelGGL(tree_accept_kernel, dim3(B), dim3(64), 0, static_cast<hipStream_t>(stream), parents, tokens,
                     targets, root_targets, cu_q, start_pos, n_rows, path, n_accepted, next_tokens, kept_lens,
                     kept_blocks);
  return launch_status(fn);
}

extern "C" int ilpc_kv_compact(uint16_t* k_pool, uint16_t* v_pool, int32_t num_blocks, const int32_t* block_tables,
                               int32_t max_blocks, const int32_t* cu_q, const int32_t* start_pos, int32_t B,
                               int32_t n_rows, const int32_t* path, const int32_t* n_accepted, int32_t Hkv, int32_t D,
                               int32_t block_size, void* stream) {
  static const char* fn = "ilpc_kv_compact";
  using ilpc::set_error;
  if (B < 0 || n_rows < 0 || num_blocks < 0 || max_blocks < 1 || Hkv < 1)
    return set_error(ILPC_EINVAL, "%s: negative or zero size", fn);
  if (block_size != kBlock) return set_error(ILPC_EUNSUP, "%s: block_size must be 16", fn);
  if (D != 64 && D != 128) return set_error(ILPC_EUNSUP, "%s: head_dim %d unsupported", fn, D);
  if (B > kMaxRequests || Hkv > 65535 || max_blocks > (1 << 24))
    return set_error(ILPC_EUNSUP, "%s: B %d, Hkv %d or max_blocks %d too large", fn, B, Hkv, max_blocks);
  if (B == 0 || n_rows == 0) return ILPC_OK;
  if (!k_pool || !v_pool || !block_tables || !cu_q || !start_pos || !path || !n_accepted)
    return set_error(ILPC_EINVAL, "%s: NULL pointer", fn);
  if (!aligned16(k_pool) || !aligned16(v_pool))
    return set_error(ILPC_EINVAL, "%s: the pools must be 16-byte aligned", fn);
  const dim3 grid{unsigned(B), unsigned(Hkv)};
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(64), 0, s, k_pool, v_pool, num_blocks, block_tables, max_blocks, cu_q,
                       start_pos, n_rows, path, n_accepted, Hkv);
  };
  if (D == 128) launch(compact_kernel<128>);
  else launch(compact_kernel<64>);
  return launch_status(fn);
}
