// Forked requests on the paged cache, for gfx950: rows of a batch that go on from
// another row's tokens (several answers sampled from one prompt, beams), the block
// copies that this takes, and the release of blocks that more than one row may hold.
//
// InferLog section 2.1.2: KV blocks are shared where prompts share a prefix, and freed
// when no request holds them.  A fork holds its source's full blocks with it and a copy
// of the last, partly filled one, which both go on writing.  holds[b] counts the
// holders of block first_id + b beyond the first, so that ilpc_extend_tables' blocks,
// held once, need no count set.  Blocks below first_id are not counted (the prefix
// cache's own).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "../../include/ilpc.h"
#include "ilpc_internal.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 16;
constexpr int kThreads = 1024;
constexpr int kMaxRequests = 1 << 20;

// What is refused on the device (bits of *status).
enum { kNoBlocks = 1, kTooLong = 2, kBadValue = 8, kNotHeld = 16 };

__device__ __forceinline__ int blocks_of(int64_t tokens) { return int((tokens + kBlock - 1) / kBlock); }

// Exclusive sum of a over the threads of the workgroup, its total, and the bits of all flags.
struct Sum {
  int before, total, flags;
};

__device__ __forceinline__ Sum scan(int a, int flags) {
  __shared__ int sa[kThreads / 64], sf[kThreads / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int inc = a;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int u = __shfl_up(inc, off);
    if (lane >= off) inc += u;
  }
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) flags |= __shfl_xor(flags, off);
  if (lane == 63) sa[wave] = inc, sf[wave] = flags;
  __syncthreads();
  Sum s{inc - a, 0, 0};
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < wave) s.before += sa[w];
    s.total += sa[w];
    s.flags |= sf[w];
  }
  __syncthreads();
  return s;
}

// One entry of a fork's row: a shared block of the source, its own copy of the last one, or none.
__device__ __forceinline__ void fork_entry(int r, int j, int src, int len, int own_id, int32_t* block_tables,
                                           int max_blocks, int32_t* holds, int first_id, int num_blocks) {
  const int full = len / kBlock;
  int id = -1;
  if (j < full) {
    id = block_tables[size_t(src) * max_blocks + j];
    if (id >= first_id && id < num_blocks) atomicAdd(holds + (id - first_id), 1);
  } else if (j == full && len % kBlock) {
    id = own_id;
  }
  block_tables[size_t(r) * max_blocks + j] = id;
}

// Checks, lengths and copies, by one workgroup: a thread takes a run of rows.  The batch
// is forked whole or not at all, so that nothing is written before all rows are known
// to be right.  FILL: the same workgroup writes the rows.  Bound by its round trips (sources,
// lengths, ids): 3.9 us for 512 rows; 4.2 with FILL for 16 rows of up to 38 blocks.  draft_start (or NULL): -1, no
// draft, for rows forked from or over, by whichever of their forks comes last.
template <bool FILL>
__global__ __launch_bounds__(kThreads) void fork_scan_kernel(
    int32_t* block_tables, int max_blocks, int B, int32_t* seq_lens, const int32_t* __restrict__ sources,
    int32_t* holds, int first_id, const int32_t* __restrict__ free_ids, int n_free, const int32_t* taken,
    int num_blocks, int32_t* __restrict__ copy_src, int32_t* __restrict__ copy_dst, int32_t* draft_start,
    int32_t* taken_out, int32_t* __restrict__ status) {
  const int per = (B + kThreads - 1) / kThreads;
  const int r0 = min(int(threadIdx.x) * per, B), r1 = min(r0 + per, B);
  const int64_t had = *taken;
  int copies = 0, bad = 0;
  for (int r = r0; r < r1; ++r) {
    const int s = sources[r];
    if (s < 0 || s >= B) {
      bad |= kBadValue;
      continue;
    }
    const int len = seq_lens[s];
    if (sources[s] != s || len < 0) bad |= kBadValue;
    if (len > int64_t(max_blocks) * kBlock) bad |= kTooLong;
    copies += s != r && len % kBlock;
  }
  const Sum t = scan(copies, bad);
  int refused = t.flags;
  if (had < 0 || had > n_free) refused |= kBadValue;
  if (had + t.total > n_free) refused |= kNoBlocks;
  int64_t at = had + t.before;
  for (int r = r0; r < r1; ++r) {
    int from = -1, to = -1;
    if (!refused) {
      const int s = sources[r], len = seq_lens[s];
      if (s != r) {
        if (len % kBlock) {
          from = block_tables[size_t(s) * max_blocks + len / kBlock];
          to = free_ids[at++];
        }
        seq_lens[r] = len;  // (sources stay: no other row's length comes from here)
        if (draft_start) draft_start[r] = draft_start[s] = -1;
      }
    }
    copy_src[r] = from;
    copy_dst[r] = to;
  }
  if (threadIdx.x == 0) {
    *taken_out = int32_t(refused ? had : had + t.total);
    *status = refused;
  }
  if constexpr (FILL) {
    if (refused) return;
    __syncthreads();
    for (int e = threadIdx.x; e < B * max_blocks; e += kThreads) {
      const int r = e / max_blocks, s = sources[r];
      if (s != r)
        fork_entry(r, e - r * max_blocks, s, seq_lens[s], copy_dst[r], block_tables, max_blocks, holds, first_id,
                   num_blocks);
    }
  }
}

// A fork's entries, 256 of a row a workgroup: 448 forks of 64 to 138 blocks 4.4 us, most of it
// the launch and two round trips; holds are counted by atomics, whose sums have no order.
constexpr int kFillThreads = 256;

__global__ __launch_bounds__(kFillThreads) void fork_fill_kernel(
    int32_t* block_tables, int max_blocks, const int32_t* __restrict__ seq_lens, const int32_t* __restrict__ sources,
    int32_t* __restrict__ holds, int first_id, int num_blocks, const int32_t* __restrict__ copy_dst,
    const int32_t* __restrict__ status) {
  const int r = blockIdx.x, s = sources[r];
  if (*status != 0 || s == r) return;
  const int len = seq_lens[s], own_id = copy_dst[r];
  for (int64_t j = int64_t(blockIdx.y) * kFillThreads + threadIdx.x; j < max_blocks;
       j += int64_t(gridDim.y) * kFillThreads)
    fork_entry(r, int(j), s, len, own_id, block_tables, max_blocks, holds, first_id, num_blocks);
}

// -- release ------------------------------------------------------------------
// First every entry's hold is dropped; the one that drops a block's last hold marks the
// block (one dropped below that shows that it was given back too often).  Then the marked
// blocks go back in the order of their ids, which does not depend on the order of the drops.
// Marks are the bits of the words behind the counts, zero between calls.  448 rows of 64 to
// 138 blocks that end together: 5.2 to 5.8 us to drop, by atomics on the same blocks' counts, and 5.2 to
// collect; 12 rows of up to 38 blocks in one launch 4.7.

struct Release {
  const int32_t* block_tables;
  int max_blocks, B;
  const int32_t* seq_lens;
  int32_t* holds;
  int first_id, n_held;  // blocks counted: first_id .. first_id + n_held - 1
  __device__ __forceinline__ uint32_t* marks() const { return reinterpret_cast<uint32_t*>(holds + n_held); }
  // the counted block of an entry, or -1
  __device__ __forceinline__ int block(int r, int j) const {
    const int b = block_tables[size_t(r) * max_blocks + j] - first_id;
    return b >= 0 && b < n_held ? b : -1;
  }
  __device__ __forceinline__ void drop(int b) const {
    if (b >= 0 && atomicSub(holds + b, 1) == 0) atomicOr(marks() + (b >> 5), 1u << (b & 31));
  }
  // entries of row r that drop a hold
  __device__ __forceinline__ int entries(int r) const { return min(blocks_of(max(seq_lens[r], 0)), max_blocks); }
  __device__ __forceinline__ int bad_len(int r) const {
    const int len = seq_lens[r];
    return len < 0 ? kBadValue : len > int64_t(max_blocks) * kBlock ? kTooLong : 0;
  }
};

// The lengths' faults, by the whole workgroup.
__device__ __forceinline__ int check_lens(const Release& a, int64_t had, int n_free) {
  int bad = had < 0 || had > n_free ? kBadValue : 0;
  for (int r = threadIdx.x; r < a.B; r += blockDim.x) bad |= a.bad_len(r);
  return bad;
}

// Lengths and taken are checked behind it, by the workgroup that collects (which gives the holds back where they are
// refused), so that a row's length and its first entries are asked for at once.
__global__ __launch_bounds__(kFillThreads) void drop_kernel(Release a) {
  for (int r = blockIdx.x; r < a.B; r += gridDim.x) {
    const int first = a.block(r, min(int(threadIdx.x), a.max_blocks - 1)), n = a.entries(r);
    if (threadIdx.x < n) a.drop(first);
    for (int j = threadIdx.x + kFillThreads; j < n; j += kFillThreads) a.drop(a.block(r, j));
  }
}

// The marked blocks in ascending order, by one workgroup: kChunk words of marks at a time in LDS with the
// marks before each, so that every thread places one bit.  DROP: the same workgroup has dropped
// the holds, and marked the blocks in LDS alone (so they fit one chunk).
constexpr int kChunk = 4096;

template <bool DROP>
__global__ __launch_bounds__(kThreads) void collect_kernel(Release a, const int32_t* taken, int32_t* __restrict__ free_ids,
                                                           int n_free, int32_t* taken_out,
                                                           int32_t* __restrict__ status) {
  __shared__ uint32_t s_marks[kChunk];
  __shared__ int s_before[kChunk];
  const int tid = threadIdx.x, words = (a.n_held + 31) / 32, chunks = (words + kChunk - 1) / kChunk;
  const int64_t had = *taken;
  int over = 0;
  if (DROP)
    for (int w = tid; w < words; w += kThreads) s_marks[w] = 0;
  const int bad = scan(0, check_lens(a, had, n_free)).flags;
  if (DROP && !bad) {
    for (int e = tid; e < a.B * a.max_blocks; e += kThreads) {
      const int r = e / a.max_blocks, j = e - r * a.max_blocks, b = a.block(r, j);
      if (j >= blocks_of(a.seq_lens[r]) || b < 0) continue;
      const int left = atomicSub(a.holds + b, 1);
      if (left == 0) atomicOr(&s_marks[b >> 5], 1u << (b & 31));
      if (left < 0) over = kNotHeld;
    }
    __syncthreads();
  }
  // Marks of chunk c in LDS, with the number before each word; their number.
  auto take = [&](int c) -> int {
    const int n = min(words - c * kChunk, kChunk), per = (n + kThreads - 1) / kThreads;
    if (!DROP) {
      for (int w = tid; w < n; w += kThreads) s_marks[w] = a.marks()[c * kChunk + w];
      __syncthreads();
    }
    const int w0 = min(tid * per, n), w1 = min(w0 + per, n);
    int count = 0;
    for (int w = w0; w < w1; ++w) count += __popc(s_marks[w]);
    const Sum t = scan(count, 0);
    int at = t.before;
    for (int w = w0; w < w1; ++w) s_before[w] = at, at += __popc(s_marks[w]);
    __syncthreads();
    return t.total;
  };
  // Every mark of the chunk: f(block, its place).
  auto each = [&](int c, auto f) {
    const int n = min(words - c * kChunk, kChunk);
#pragma unroll 4
    for (int e = tid; e < n * 32; e += kThreads) {
      const int w = e >> 5, bit = e & 31;
      const uint32_t m = s_marks[w];
      if (m >> bit & 1u) f((c * kChunk + w) * 32 + bit, s_before[w] + __popc(m & ((1u << bit) - 1)));
    }
  };
  int total = 0;
  for (int c = 0; c < chunks; ++c) {
    total += take(c);
    if (!DROP) {
      each(c, [&](int b, int) { over |= a.holds[b] < -1 ? int(kNotHeld) : 0; });
      __syncthreads();
    }
  }
  int refused = scan(0, over).flags;
  if (total > had) refused |= kNoBlocks;
  if (bad) refused = bad;  // (what was dropped by such lengths says nothing)
  int64_t at = had - total;
  for (int c = 0; c < chunks; ++c) {
    const int n = chunks > 1 ? take(c) : total;
    if (!refused)
      each(c, [&](int b, int k) {
        a.holds[b] = 0;
        free_ids[at + k] = a.first_id + b;
      });
    at += n;
    if (!DROP) {
      for (int w = tid; w < min(words - c * kChunk, kChunk); w += kThreads)
        if (s_marks[w]) a.marks()[c * kChunk + w] = 0;
      __syncthreads();
    }
  }
  if (tid == 0) {
    *taken_out = int32_t(refused ? had : had - total);
    *status = refused;
  }
  if (refused && !(DROP && bad))  // every hold as it was
    for (int r = 0; r < a.B; ++r) {
      const int n = a.entries(r);
      for (int j = tid; j < n; j += kThreads) {
        const int b = a.block(r, j);
        if (b >= 0) atomicAdd(a.holds + b, 1);
      }
    }
}

// -- copies ---------------------------------------------------------------------
// 16 KiB of a block's K or V slab a workgroup, all of it on its way before the first store.  Bound
// by the bytes: 64 blocks of 8 heads, D 128 to 448 places (29 MB written) 8.6 us; a large copy's 5.0
// TB/s would take 6.7.
constexpr int kCopyThreads = 256, kCopyEach = 4, kCopyBytes = kCopyThreads * kCopyEach * 16;

__global__ __launch_bounds__(kCopyThreads) void copy_blocks_kernel(u32x4* __restrict__ k_pool, u32x4* __restrict__ v_pool,
                                                                   int num_blocks, int slab, int pieces,
                                                                   const int32_t* __restrict__ src,
                                                                   const int32_t* __restrict__ dst) {
  const int i = blockIdx.x / (2 * pieces), piece = blockIdx.x % (2 * pieces);
  const int s = src[i], d = dst[i];
  if (s < 0 || s >= num_blocks || d < 0 || d >= num_blocks || s == d) return;
  u32x4* pool = piece & 1 ? v_pool : k_pool;
  const int first = (piece >> 1) * kCopyThreads * kCopyEach + threadIdx.x;
  u32x4 x[kCopyEach];
#pragma unroll
  for (int e = 0; e < kCopyEach; ++e)
    if (first + e * kCopyThreads < slab) x[e] = pool[size_t(s) * slab + first + e * kCopyThreads];
#pragma unroll
  for (int e = 0; e < kCopyEach; ++e)
    if (first + e * kCopyThreads < slab) pool[size_t(d) * slab + first + e * kCopyThreads] = x[e];
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int launch_status(const char* fn) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ILPC_OK : ilpc::set_error(ILPC_EHIP, "%s: launch failed: %s", fn, hipGetErrorString(e));
}

int check_sizes(const char* fn, int32_t B, int32_t max_blocks, int32_t n_free, int32_t num_blocks, int32_t first_id) {
  using ilpc::set_error;
  if (B < 0 || max_blocks < 1 || n_free < 0 || num_blocks < 0 || first_id < 0 || first_id > num_blocks)
    return set_error(ILPC_EINVAL, "%s: negative or zero size, or first_id past num_blocks", fn);
  if (B > kMaxRequests || max_blocks > (1 << 24) || num_blocks > INT32_MAX / kBlock)
    return set_error(ILPC_EUNSUP, "%s: B %d, max_blocks %d or num_blocks %d too large", fn, B, max_blocks, num_blocks);
  return ILPC_OK;
}

// Most table entries that one workgroup fills, or drops, by itself.  us in one launch, in two (a call
// alone; forks, releases): 368 entries 8, 11 and 7, 11; 2048 8, 11 and 8, 12; 4096 9 to 10, 11 and 9 to 10,
// 12; 8192 15, 11 and 13, 12 to 13; 16384 22 to 26, 11 and 20, 14; 70656 82, 11 and 69, 25.
constexpr int kOneFork = 4096, kOneRelease = 4096;

}  // namespace

extern "C" int ilpc_fork_tables_drafts(int32_t* block_tables, int32_t max_blocks, int32_t B, int32_t* seq_lens,
                                       const int32_t* sources, int32_t* holds, int32_t first_id,
                                       const int32_t* free_ids, int32_t n_free, const int32_t* taken,
                                       int32_t num_blocks, int32_t* copy_src, int32_t* copy_dst, int32_t* start_pos,
                                       int32_t* taken_out, int32_t* status, void* stream) {
  static const char* fn = "ilpc_fork_tables";
  using ilpc::set_error;
  const int rc = check_sizes(fn, B, max_blocks, n_free, num_blocks, first_id);
  if (rc != ILPC_OK) return rc;
  if ((B && (!block_tables || !seq_lens || !sources || !copy_src || !copy_dst)) || (n_free && !free_ids) ||
      (num_blocks > first_id && !holds) || !taken || !taken_out || !status)
    return set_error(ILPC_EINVAL, "%s: NULL pointer", fn);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool one = int64_t(B) * max_blocks <= kOneFork;
  auto launch_scan = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(1), dim3(kThreads), 0, s, block_tables, max_blocks, B, seq_lens, sources, holds,
                       first_id, free_ids, n_free, taken, num_blocks, copy_src, copy_dst, start_pos, taken_out, status);
  };
  if (one) launch_scan(fork_scan_kernel<true>);
  else launch_scan(fork_scan_kernel<false>);
  const int rc1 = launch_status(fn);
  if (rc1 != ILPC_OK || one) return rc1;
  const unsigned parts = unsigned(std::min<int64_t>((int64_t(max_blocks) + kFillThreads - 1) / kFillThreads, 64));
  hipLaunchKernelGGL(fork_fill_kernel, dim3(unsigned(B), parts), dim3(kFillThreads), 0, s, block_tables, max_blocks,
                     seq_lens, sources, holds, first_id, num_blocks, copy_dst, status);
  return launch_status(fn);
}

extern "C" int ilpc_fork_tables(int32_t* block_tables, int32_t max_blocks, int32_t B, int32_t* seq_lens,
                                const int32_t* sources, int32_t* holds, int32_t first_id, const int32_t* free_ids,
                                int32_t n_free, const int32_t* taken, int32_t num_blocks, int32_t* copy_src,
                                int32_t* copy_dst, int32_t* taken_out, int32_t* status, void* stream) {
  return ilpc_fork_tables_drafts(block_tables, max_blocks, B, seq_lens, sources, holds, first_id, free_ids, n_free,
                                 taken, num_blocks, copy_src, copy_dst, nullptr, taken_out, status, stream);
}

extern "C" int ilpc_release_shared(const int32_t* block_tables, int32_t max_blocks, int32_t B, const int32_t* seq_lens,
                                   int32_t* holds, int32_t first_id, int32_t* free_ids, int32_t n_free,
                                   const int32_t* taken, int32_t num_blocks, int32_t* taken_out, int32_t* status,
                                   void* stream) {
  static const char* fn = "ilpc_release_shared";
  using ilpc::set_error;
  const int rc = check_sizes(fn, B, max_blocks, n_free, num_blocks, first_id);
  if (rc != ILPC_OK) return rc;
  if ((B && (!block_tables || !seq_lens)) || (n_free && !free_ids) || (num_blocks > first_id && !holds) || !taken ||
      !taken_out || !status)
    return set_error(ILPC_EINVAL, "%s: NULL pointer", fn);
  hipStream_t s = static_cast<hipStream_t>(stream);
  // (without rows there is no block to look at, however many there are)
  const Release a{block_tables, max_blocks, B, seq_lens, holds, first_id, B ? num_blocks - first_id : 0};
  if (B == 0 || (int64_t(B) * max_blocks <= kOneRelease && a.n_held <= kChunk * 32)) {
    hipLaunchKernelGGL(collect_kernel<true>, dim3(1), dim3(kThreads), 0, s, a, taken, free_ids, n_free, taken_out,
                       status);
    return launch_status(fn);
  }
  hipLaunchKernelGGL(drop_kernel, dim3(unsigned(std::min(B, 1024))), dim3(kFillThreads), 0, s, a);
  const int rc1 = launch_status(fn);
  if (rc1 != ILPC_OK) return rc1;
  hipLaunchKernelGGL(collect_kernel<false>, dim3(1), dim3(kThreads), 0, s, a, taken, free_ids, n_free, taken_out,
                     status);
  return launch_status(fn);
}

extern "C" int ilpc_holds_words(int32_t n_blocks, int32_t* words) {
  static const char* fn = "ilpc_holds_words";
  if (!words || n_blocks < 0) return ilpc::set_error(ILPC_EINVAL, "%s: n_blocks %d, or words is NULL", fn, n_blocks);
  if (n_blocks > INT32_MAX / kBlock) return ilpc::set_error(ILPC_EUNSUP, "%s: n_blocks %d too large", fn, n_blocks);
  *words = n_blocks + (n_blocks + 31) / 32;
  return ILPC_OK;
}

extern "C" int ilpc_copy_blocks(uint16_t* k_pool, uint16_t* v_pool, int32_t num_blocks, const int32_t* src,
                                const int32_t* dst, int32_t n, int32_t Hkv, int32_t D, int32_t block_size,
                                void* stream) {
  static const char* fn = "ilpc_copy_blocks";
  using ilpc::set_error;
  if (n < 0 || num_blocks < 0 || Hkv < 1) return set_error(ILPC_EINVAL, "%s: negative or zero size", fn);
  if (block_size != kBlock) return set_error(ILPC_EUNSUP, "%s: block_size must be 16", fn);
  if (D != 64 && D != 128) return set_error(ILPC_EUNSUP, "%s: head_dim %d unsupported", fn, D);
  if (Hkv > 65535) return set_error(ILPC_EUNSUP, "%s: Hkv %d too large", fn, Hkv);
  const int slab = Hkv * D * 2;  // 16-byte pieces of a block's K, or V
  const int pieces = (slab * 16 + kCopyBytes - 1) / kCopyBytes;
  if (int64_t(n) * 2 * pieces >= (1 << 24)) return set_error(ILPC_EUNSUP, "%s: too many blocks", fn);
  if (n == 0) return ILPC_OK;
  if (!k_pool || !v_pool || !src || !dst) return set_error(ILPC_EINVAL, "%s: NULL pointer", fn);
  if (!aligned16(k_pool) || !aligned16(v_pool))
    return set_error(ILPC_EINVAL, "%s: the pools must be 16-byte aligned", fn);
  hipLaunchKernelGGL(copy_blocks_kernel, dim3(unsigned(n) * 2 * pieces), dim3(kCopyThreads), 0,
                     static_cast<hipStream_t>(stream), reinterpret_cast<u32x4*>(k_pool),
                     reinterpret_cast<u32x4*>(v_pool), num_blocks, slab, pieces, src, dst);
  return launch_status(fn);
}
