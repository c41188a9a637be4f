// A growing batch's metadata on the device, for gfx950: block tables, row
// offsets, context lengths and slot map from the requests' lengths
// (extend), blocks given back (release), and the K/V append that goes by the
// slot map.
//
// InferLog section 2.1.2: the KV cache is held in fixed-size blocks that are
// allocated as a request's tokens come and freed when it ends.  Request r holds
// s_r tokens and gets n_r new ones:
//   c_r = sum_{q<r} n_q,   h_r = ceil(s_r / 16),   d_r = ceil((s_r + n_r) / 16) - h_r,
//   b_r = sum_{q<r} d_q,   table[r][h_r + k] = free[taken + b_r + k]   (k < d_r),
//   slot[c_r + i] = 16 * table[r][(s_r + i) / 16] + (s_r + i) % 16     (i < n_r).
// Both sums run over the requests in order, so ids come out as from an
// allocator that serves request after request, whatever runs in parallel.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/ilpc.h"
#include "ilpc_internal.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 16;
constexpr int kScanThreads = 1024;
constexpr int kMaxRequests = 1 << 20;
// Most rows (of extend; blocks that there can be, of release) that the workgroup of
// the sums fills in itself.  us in one launch, in two: 512 requests of a row 5.5, 8.6;
// one request of 4096 rows 5.9, 7.3, of 8192 7.6, 7.7; 64 requests of 96 rows 9.3, 9.9,
// of 128 11.0, 9.6; 512 of 12 10.9, 12.4, of 16 13.1, 11.4.  Released ids (of a table of
// as many or more): 512 3.7, 5.8; 4096 5.4, 5.9; 8192 8.1, 6.0.
constexpr int kOneFill = 6144, kOneRelease = 8192;

// What is refused on the device (bits of *status).
enum { kNoBlocks = 1, kTooLong = 2, kTooManyRows = 4, kBadValue = 8 };

__device__ __forceinline__ int blocks_of(int64_t tokens) { return int((tokens + kBlock - 1) / kBlock); }

// Exclusive sums of (a, b) over the threads of the workgroup, their totals in
// ta, tb, and the bits of all flags in `flags`.
struct Sums {
  int64_t a, b, ta, tb;
  int flags;
};

__device__ __forceinline__ Sums scan(int64_t a, int64_t b, int flags) {
  constexpr int kW = kScanThreads / 64;
  __shared__ int64_t sa[kW], sb[kW];
  __shared__ int sf[kW];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t ia = a, ib = b;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int64_t ua = __shfl_up(ia, off), ub = __shfl_up(ib, off);
    if (lane >= off) ia += ua, ib += ub;
  }
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) flags |= __shfl_xor(flags, off);
  if (lane == 63) sa[wave] = ia, sb[wave] = ib, sf[wave] = flags;
  __syncthreads();
  Sums s{ia - a, ib - b, 0, 0, 0};
  for (int w = 0; w < kW; ++w) {
    if (w < wave) s.a += sa[w], s.b += sb[w];
    s.ta += sa[w], s.tb += sb[w], s.flags |= sf[w];
  }
  return s;
}

// The last r in [lo, hi) with sums[r] <= x (sums ascending, sums[lo] <= x).
__device__ __forceinline__ int owner(const int32_t* sums, int lo, int hi, int x) {
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// What the fill needs of a request: start, first row, first new block.
struct Growth {
  const int32_t *seq_lens, *cu_q, *cu_blocks;  // B, B + 1, B + 1
  __device__ __forceinline__ int start(int r) const { return seq_lens[r] - (cu_q[r + 1] - cu_q[r]); }
};

// Slot of row i, a row of request r.  A block that is taken holds a new token at its
// offset 0 (it starts at or behind the tokens held), so that the rows whose position is
// a multiple of 16 are the blocks taken, one by one: each writes its table entry.
__device__ __forceinline__ int place_row(int i, int r, const Growth& g, int32_t* block_tables, int max_blocks,
                                         const int32_t* free_ids, int first_id, int num_blocks) {
  const int start = g.start(r), pos = start + (i - g.cu_q[r]), lb = pos / kBlock, had = blocks_of(start);
  int32_t* entry = block_tables + size_t(r) * max_blocks + lb;
  const int id = lb < had ? *entry : free_ids[first_id + g.cu_blocks[r] + lb - had];
  if (pos % kBlock == 0) *entry = id;
  return id >= 0 && id < num_blocks ? id * kBlock + pos % kBlock : -1;
}

// Lengths and sums, by one workgroup: a thread takes a run of requests, adds it
// up, and behind the sum over the threads before it writes the run's results.
// Reads of a request's lengths come before the same thread's write, so seq_lens
// may be start_pos.  FILL: the same workgroup then writes the table entries and
// slots, from sums that it keeps in LDS: a decode step's tables are one launch.
constexpr int kFillRequests = 2048;  // FILL: at most

template <bool FILL>
__global__ __launch_bounds__(kScanThreads) void extend_scan_kernel(
    int32_t* block_tables, const int32_t* start_pos, const int32_t* __restrict__ new_lens, int B,
    const int32_t* __restrict__ free_ids, int n_free, const int32_t* taken, int num_blocks, int max_blocks,
    int max_rows, int32_t* seq_lens, int32_t* __restrict__ cu_q, int32_t* __restrict__ cu_blocks,
    int32_t* __restrict__ slot_map, int32_t* taken_out, int32_t* __restrict__ status) {
  constexpr int kKeep = FILL ? kFillRequests : 1;
  __shared__ int32_t k_seq[kKeep], k_cu[kKeep + 1], k_cb[kKeep + 1];
  const int per = (B + kScanThreads - 1) / kScanThreads;
  const int r0 = min(int(threadIdx.x) * per, B), r1 = min(r0 + per, B);
  const int64_t had = *taken;
  int64_t rows = 0, blocks = 0;
  int bad = 0;
#pragma unroll 4
  for (int r = r0; r < r1; ++r) {
    const int64_t s = start_pos[r], n = new_lens[r];
    if (s < 0 || n < 0) bad |= kBadValue;
    if (s + n > int64_t(max_blocks) * kBlock) bad |= kTooLong;
    rows += n;
    blocks += blocks_of(s + n) - blocks_of(s);
  }
  const Sums t = scan(rows, blocks, bad);
  int refused = t.flags;
  if (had < 0 || had > n_free) refused |= kBadValue;
  if (had + t.tb > n_free) refused |= kNoBlocks;
  if (t.ta > max_rows) refused |= kTooManyRows;
  int64_t a = t.a, b = t.b;
#pragma unroll 4
  for (int r = r0; r < r1; ++r) {
    const int64_t s = start_pos[r], n = new_lens[r];
    const int32_t row = refused ? 0 : int32_t(a), block = refused ? 0 : int32_t(b), len = int32_t(refused ? s : s + n);
    cu_q[r] = row;
    cu_blocks[r] = block;
    seq_lens[r] = len;
    if (FILL) k_cu[r] = row, k_cb[r] = block, k_seq[r] = len;
    a += n;
    b += blocks_of(s + n) - blocks_of(s);
  }
  const int n_rows = refused ? 0 : int(t.ta), n_new = refused ? 0 : int(t.tb);
  if (threadIdx.x == 0) {
    cu_q[B] = n_rows;
    cu_blocks[B] = n_new;
    if (FILL) k_cu[B] = n_rows, k_cb[B] = n_new;
    *taken_out = int32_t(had + n_new);
    *status = refused;
  }
  if constexpr (FILL) {
    __syncthreads();
    const Growth g{k_seq, k_cu, k_cb};
    for (int i = threadIdx.x; i < max_rows; i += kScanThreads)
      slot_map[i] = i < n_rows ? place_row(i, owner(k_cu, 0, B, i), g, block_tables, max_blocks, free_ids, int(had),
                                           num_blocks)
                               : -1;
  }
}

// Table entries and slots from the sums, for many rows: 1024 rows a workgroup, whose
// requests it looks up once, 64 probes a round trip (512 requests, 1.0 M rows: 8.4 us by
// halves and with the blocks taken looked up on their own, 5.5 to 6.8 so).
constexpr int kFillThreads = 256, kFillRows = 1024;

// owner() by a wave, sums[0] <= x.
__device__ __forceinline__ int wave_owner(const int32_t* sums, int n, int x) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, at = lo + lane * step;
    // (the lanes that hold are the first ones)
    const uint64_t holds = __ballot(at < hi && (lane == 0 || sums[at] <= x));
    lo += (63 - __builtin_clzll(holds)) * step;
    hi = min(lo + step, hi);
  }
  return lo;
}

__global__ __launch_bounds__(kFillThreads) void extend_fill_kernel(
    int32_t* __restrict__ block_tables, int B, int max_blocks, const int32_t* __restrict__ free_ids,
    const int32_t* __restrict__ taken_out, int num_blocks, const int32_t* __restrict__ seq_lens,
    const int32_t* __restrict__ cu_q, const int32_t* __restrict__ cu_blocks, int32_t* __restrict__ slot_map,
    int max_rows) {
  __shared__ int s_of[2];
  const int n_rows = cu_q[B], first_id = *taken_out - cu_blocks[B];
  const Growth g{seq_lens, cu_q, cu_blocks};
  const int64_t i0 = int64_t(blockIdx.x) * kFillRows, i1 = min(i0 + kFillRows, int64_t(max_rows));
  const int wave = threadIdx.x >> 6;
  if (wave < 2 && i0 < n_rows) {
    const int r = wave_owner(cu_q, B, int(wave ? min(i1, int64_t(n_rows)) - 1 : i0));
    if ((threadIdx.x & 63) == 0) s_of[wave] = r;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kFillRows / kFillThreads; ++u) {
    const int64_t i = i0 + u * kFillThreads + threadIdx.x;
    if (i < i1)
      slot_map[i] = i < n_rows ? place_row(int(i), owner(cu_q, s_of[0], s_of[1] + 1, int(i)), g, block_tables,
                                           max_blocks, free_ids, first_id, num_blocks)
                               : -1;
  }
}

template <bool FILL>
__global__ __launch_bounds__(kScanThreads) void release_scan_kernel(
    const int32_t* __restrict__ block_tables, const int32_t* __restrict__ first_block,
    const int32_t* __restrict__ seq_lens, int B, int max_blocks, int n_free, const int32_t* taken,
    int32_t* __restrict__ free_ids, int32_t* __restrict__ cu_blocks, int32_t* taken_out,
    int32_t* __restrict__ status) {
  __shared__ int32_t k_cb[FILL ? kFillRequests + 1 : 1];
  const int per = (B + kScanThreads - 1) / kScanThreads;
  const int r0 = min(int(threadIdx.x) * per, B), r1 = min(r0 + per, B);
  const int64_t had = *taken;
  auto count = [&](int r) { return max(blocks_of(seq_lens[r]) - max(first_block[r], 0), 0); };
  int64_t blocks = 0;
  int bad = 0;
#pragma unroll 4
  for (int r = r0; r < r1; ++r) {
    if (first_block[r] < 0 || seq_lens[r] < 0) bad |= kBadValue;
    if (seq_lens[r] > int64_t(max_blocks) * kBlock) bad |= kTooLong;
    blocks += count(r);
  }
  const Sums t = scan(0, blocks, bad);
  int refused = t.flags;
  if (had < 0 || had > n_free) refused |= kBadValue;
  if (t.tb > had) refused |= kNoBlocks;
  int64_t b = t.b;
#pragma unroll 4
  for (int r = r0; r < r1; ++r) {
    cu_blocks[r] = refused ? 0 : int32_t(b);
    if (FILL) k_cb[r] = cu_blocks[r];
    b += count(r);
  }
  const int n = refused ? 0 : int(t.tb);
  if (threadIdx.x == 0) {
    cu_blocks[B] = n;
    if (FILL) k_cb[B] = n;
    *taken_out = int32_t(had - n);
    *status = refused;
  }
  if constexpr (FILL) {
    __syncthreads();
    for (int e = threadIdx.x; e < n; e += kScanThreads) {
      const int r = owner(k_cb, 0, B, e);
      free_ids[had - n + e] = block_tables[size_t(r) * max_blocks + first_block[r] + (e - k_cb[r])];
    }
  }
}

__global__ __launch_bounds__(kFillThreads) void release_fill_kernel(
    const int32_t* __restrict__ block_tables, int B, int max_blocks, const int32_t* __restrict__ first_block,
    const int32_t* __restrict__ cu_blocks, const int32_t* __restrict__ taken_out, int32_t* __restrict__ free_ids) {
  __shared__ int s_of[2];
  const int n = cu_blocks[B], at = *taken_out, wave = threadIdx.x >> 6;
  for (int64_t e0 = int64_t(blockIdx.x) * kFillThreads; e0 < n; e0 += int64_t(gridDim.x) * kFillThreads) {
    __syncthreads();
    if (wave < 2) {
      const int r = wave_owner(cu_blocks, B, int(wave ? min(e0 + kFillThreads, int64_t(n)) - 1 : e0));
      if ((threadIdx.x & 63) == 0) s_of[wave] = r;
    }
    __syncthreads();
    const int64_t e = e0 + threadIdx.x;
    if (e < n) {
      const int r = owner(cu_blocks, s_of[0], s_of[1] + 1, int(e));
      free_ids[at + e] = block_tables[size_t(r) * max_blocks + first_block[r] + (e - cu_blocks[r])];
    }
  }
}

// ---------------------------------------------------------------------------
// K/V append by slots: one workgroup per 16 rows and kv head.  Rows that take
// consecutive slots of one block (a prompt's) are a run, at most 16 rows; the
// workgroup in whose 16 rows a run starts stores all of it, so that whole
// 16-byte pieces of the dimension-major V block are written at once and not
// two bytes a row.
template <int D>
__global__ __launch_bounds__(256) void append_slots_kernel(
    const uint16_t* __restrict__ k_new, const uint16_t* __restrict__ v_new, int64_t k_stride, int64_t v_stride,
    uint16_t* __restrict__ k_pool, uint16_t* __restrict__ v_pool, int num_blocks,
    const int32_t* __restrict__ slot_map, int n_rows, int Hkv) {
  constexpr int kChunks = D / 8, kSpan = 2 * kBlock;  // rows looked at: 16, and the rest of the last run
  __shared__ __attribute__((aligned(16))) uint16_t sv[kSpan][D + 8];
  __shared__ int s_slot[kSpan];
  __shared__ uint32_t s_cont;
  const int h = blockIdx.y, tid = threadIdx.x;
  const int64_t base = int64_t(blockIdx.x) * kBlock;
  if (tid < 64) {
    auto at = [&](int64_t i) {
      const int s = i >= 0 && i < n_rows ? slot_map[i] : -1;
      return s >= 0 && s / kBlock < num_blocks ? s : -1;
    };
    const int i = tid & (kSpan - 1);
    const int s = at(base + i), before = at(base + i - 1);
    // the row goes on with the run of the one before it
    const bool cont = s >= 0 && before == s - 1 && before >= 0 && s % kBlock != 0;
    const uint64_t m = __ballot(cont);
    if (tid < kSpan) s_slot[i] = s;
    if (tid == 0) s_cont = uint32_t(m);
  }
  __syncthreads();
  const uint32_t cont = s_cont;
  // rows of runs that start here: from the first start to the end of the last
  // run (16 rows cannot all go on with a run from before: it would be longer)
  const uint32_t starts = ~cont & 0xFFFFu, ends = ~cont & 0xFFFF0000u;
  if (starts == 0) return;
  const int a = __builtin_ctz(starts), b = ends ? __builtin_ctz(ends) : kSpan;
  for (int idx = tid; idx < (b - a) * kChunks; idx += 256) {
    const int i = a + idx / kChunks, c = idx % kChunks, s = s_slot[i];
    if (s < 0) continue;
    const size_t to = ((size_t(s / kBlock) * Hkv + h) * kBlock + s % kBlock) * D + c * 8;
    *(u32x4*)(k_pool + to) = *(const u32x4*)(k_new + (base + i) * k_stride + size_t(h) * D + c * 8);
    *(u32x4*)(&sv[i][c * 8]) = *(const u32x4*)(v_new + (base + i) * v_stride + size_t(h) * D + c * 8);
  }
  __syncthreads();
  for (int idx = tid; idx < (b - a) * D; idx += 256) {
    const int i = a + idx / D, d = idx % D, s = s_slot[i];
    if (s < 0) continue;
    // rows of this half of the block (8 slots) that the run covers: all of them?
    const int j = i - s % 8;  // row of the half's first slot
    const bool whole = j >= a && j + 8 <= b && ((cont >> (j + 1)) & 0x7Fu) == 0x7Fu;
    uint16_t* dst = v_pool + ((size_t(s / kBlock) * Hkv + h) * D + d) * kBlock + s % kBlock;
    if (!whole) {
      *dst = sv[i][d];
    } else if (i == j) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = uint32_t(sv[i + 2 * e][d]) | uint32_t(sv[i + 2 * e + 1][d]) << 16;
      *(u32x4*)dst = w;
    }
  }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int launch_status(const char* fn) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ILPC_OK : ilpc::set_error(ILPC_EHIP, "%s: launch failed: %s", fn, hipGetErrorString(e));
}

}  // namespace

extern "C" int ilpc_extend_tables(int32_t* block_tables, int32_t max_blocks, int32_t B, const int32_t* start_pos,
                                  const int32_t* new_lens, const int32_t* free_ids, int32_t n_free,
                                  const int32_t* taken, int32_t num_blocks, int32_t* seq_lens, int32_t* cu_q,
                                  int32_t* cu_blocks, int32_t* slot_map, int32_t max_rows, int32_t* taken_out,
                                  int32_t* status, void* stream) {
  static const char* fn = "ilpc_extend_tables";
  using ilpc::set_error;
  if (B < 0 || max_blocks < 1 || n_free < 0 || num_blocks < 0 || max_rows < 0)
    return set_error(ILPC_EINVAL, "%s: negative or zero size", fn);
  if (B > kMaxRequests || max_blocks > (1 << 24) || num_blocks > INT32_MAX / kBlock)
    return set_error(ILPC_EUNSUP, "%s: B %d, max_blocks %d or num_blocks %d too large", fn, B, max_blocks, num_blocks);
  if ((B && (!block_tables || !start_pos || !new_lens || !seq_lens)) || (n_free && !free_ids) || !taken || !cu_q ||
      !cu_blocks || (max_rows && !slot_map) || !taken_out || !status)
    return set_error(ILPC_EINVAL, "%s: NULL pointer", fn);
  hipStream_t s = static_cast<hipStream_t>(stream);
  // One launch as long as one workgroup's fill costs less than the second launch.
  const bool one = B <= kFillRequests && max_rows <= kOneFill;
  auto launch_scan = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(1), dim3(kScanThreads), 0, s, block_tables, start_pos, new_lens, B, free_ids,
                       n_free, taken, num_blocks, max_blocks, max_rows, seq_lens, cu_q, cu_blocks, slot_map, taken_out,
                       status);
  };
  if (one) launch_scan(extend_scan_kernel<true>);
  else launch_scan(extend_scan_kernel<false>);
  const int rc = launch_status(fn);
  if (rc != ILPC_OK || one) return rc;
  if (max_rows == 0) return rc;
  const unsigned grid = unsigned((int64_t(max_rows) + kFillRows - 1) / kFillRows);
  hipLaunchKernelGGL(extend_fill_kernel, dim3(grid), dim3(kFillThreads), 0, s, block_tables, B, max_blocks, free_ids,
                     taken_out, num_blocks, seq_lens, cu_q, cu_blocks, slot_map, max_rows);
  return launch_status(fn);
}

extern "C" int ilpc_release_tables(const int32_t* block_tables, int32_t max_blocks, int32_t B,
                                   const int32_t* first_block, const int32_t* seq_lens, int32_t* free_ids,
                                   int32_t n_free, const int32_t* taken, int32_t* cu_blocks, int32_t* taken_out,
                                   int32_t* status, void* stream) {
  static const char* fn = "ilpc_release_tables";
  using ilpc::set_error;
  if (B < 0 || max_blocks < 1 || n_free < 0) return set_error(ILPC_EINVAL, "%s: negative or zero size", fn);
  if (B > kMaxRequests || max_blocks > (1 << 24))
    return set_error(ILPC_EUNSUP, "%s: B %d or max_blocks %d too large", fn, B, max_blocks);
  if ((B && (!block_tables || !first_block || !seq_lens)) || (n_free && !free_ids) || !taken || !cu_blocks ||
      !taken_out || !status)
    return set_error(ILPC_EINVAL, "%s: NULL pointer", fn);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t most = int64_t(B) * max_blocks;  // blocks there can be
  const bool one = B <= kFillRequests && most <= kOneRelease;
  auto launch_scan = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(1), dim3(kScanThreads), 0, s, block_tables, first_block, seq_lens, B, max_blocks,
                       n_free, taken, free_ids, cu_blocks, taken_out, status);
  };
  if (one) launch_scan(release_scan_kernel<true>);
  else launch_scan(release_scan_kernel<false>);
  const int rc = launch_status(fn);
  if (rc != ILPC_OK || one) return rc;
  const unsigned grid = unsigned(most < 256 * kFillThreads ? (most + kFillThreads - 1) / kFillThreads : 256);
  hipLaunchKernelGGL(release_fill_kernel, dim3(grid), dim3(kFillThreads), 0, s, block_tables, B, max_blocks,
                     first_block, cu_blocks, taken_out, free_ids);
  return launch_status(fn);
}

extern "C" int ilpc_kv_append_slots(const uint16_t* k_new, int64_t k_stride, const uint16_t* v_new, int64_t v_stride,
                                    uint16_t* k_pool, uint16_t* v_pool, int32_t num_blocks, const int32_t* slot_map,
                                    int32_t n_rows, int32_t Hkv, int32_t D, int32_t block_size, void* stream) {
  static const char* fn = "ilpc_kv_append_slots";
  using ilpc::set_error;
  if (n_rows < 0 || num_blocks < 0 || Hkv < 1) return set_error(ILPC_EINVAL, "%s: negative or zero size", fn);
  if (block_size != kBlock) return set_error(ILPC_EUNSUP, "%s: block_size must be 16", fn);
  if (D != 64 && D != 128) return set_error(ILPC_EUNSUP, "%s: head_dim %d unsupported", fn, D);
  if (Hkv > 65535 || n_rows > (1 << 28) - kBlock) return set_error(ILPC_EUNSUP, "%s: grid too large", fn);
  if (n_rows == 0) return ILPC_OK;
  if (!k_new || !v_new || !k_pool || !v_pool || !slot_map) return set_error(ILPC_EINVAL, "%s: NULL pointer", fn);
  const int64_t row = int64_t(Hkv) * D;
  if (k_stride < row || v_stride < row || k_stride % 8 != 0 || v_stride % 8 != 0)
    return set_error(ILPC_EINVAL, "%s: row strides must be multiples of 8 elements, at least Hkv * D", fn);
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(k_pool) || !aligned16(v_pool))
    return set_error(ILPC_EINVAL, "%s: K/V buffers must be 16-byte aligned", fn);
  const dim3 grid(unsigned((int64_t(n_rows) + kBlock - 1) / kBlock), unsigned(Hkv));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (D == 128)
    hipLaunchKernelGGL(append_slots_kernel<128>, grid, dim3(256), 0, s, k_new, v_new, k_stride, v_stride, k_pool,
                       v_pool, num_blocks, slot_map, n_rows, Hkv);
  else
    hipLaunchKernelGGL(append_slots_kernel<64>, grid, dim3(256), 0, s, k_new, v_new, k_stride, v_stride, k_pool,
                       v_pool, num_blocks, slot_map, n_rows, Hkv);
  return launch_status(fn);
}
