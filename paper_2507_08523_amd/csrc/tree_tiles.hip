// Attention of drafted trees with many query columns, for gfx950 (the mathematics and
// the kernel for few columns are in tree_attn.hip).
//
// A workgroup of four waves works 128 columns -- (node, head of the group) pairs of one
// (request, kv head) -- against 64-key tiles of K and V in LDS, each wave 32 columns.
// Per 32 keys and wave, on v_mfma_f32_32x32x16_bf16:
//   S^T = K Q^T   D/16 products,   O^T += V^T P^T   2 * D/32 products,
// the products with V of a step and the scores of the next one in one run, behind them
// the exponentials; what overlaps a wave's exponentials with products is the other
// wave of its SIMD.  Exponentials are taken against the running maximum; where a
// lane's sum of 16 of them leaves [0, 2^8] the step's maximum is taken and they are
// taken again (the first step always).  Weights enter the products with V rounded to
// bf16 (half a step, 2^-8 of each), the sums add the fp32 values.
//
// Why 128 columns and LDS: a wave that streams K and V into its registers reads them once for
// every 32 columns, and the largest batches then wait for the path from L2 (128 requests of
// 64 nodes behind 2050 keys, 64 heads on 8 of D 128: 873 us; here 584 to 610, 0.91 PFLOP/s).
// What bounds it there: of the SIMDs' cycles 54% have matrix products and 45% other vector
// instructions, 23% both, and under that load the clock falls to 1.5 to 1.7 GHz, so that the
// products alone, without exponentials and with operands that stay in registers, still take
// 530 us (a large library product reaches 1.23 PFLOP/s).  The order of the operands' reads,
// how far ahead they are taken (3, 4, 6) and priorities of waves change nothing (606 to
// 613); 64 columns a wave, which halve the reads from LDS, do not fit the registers beside O
// (740 to 890), nor with O in accumulation registers (657).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "../../include/ilpc.h"
#include "ilpc_internal.h"
#include "tree_attn.h"

namespace {

using namespace ilpc;

constexpr int kBlock = 16;
constexpr int kWaves = 4;
constexpr int kCols = 32 * kWaves;  // columns of a workgroup
constexpr int kKeys = 64;           // keys of a tile: two steps of 32
constexpr int kTileBlocks = kKeys / kBlock;
constexpr int kMaxHalfWords = 32;   // mask words of 32 nodes
// Largest sum of a lane's exponentials of a step accepted without taking the
// step's maximum.
constexpr float kSumLimit = 256.f;

// 16-byte slot of chunk c in LDS K row m: XOR-swizzled so that the lanes an LDS
// cycle serves (consecutive rows, one chunk each) hit distinct banks.
template <int D>
__device__ __forceinline__ int k_slot(int m, int c) {
  return D == 128 ? (c ^ (m & 15)) : (c ^ ((m >> 1) & 7));
}
// 16-byte half (keys 0-7 or 8-15) of V row d of a [D][16] block in LDS.
__device__ __forceinline__ int v_slot(int d, int hf) { return hf ^ ((d >> 2) & 1) ^ ((d >> 3) & 1); }

// One (block, kv head) slab of a pool straight into LDS: instruction i moves 16
// bytes a lane from base + off[i] + i KiB (base wave-uniform) to lds + i KiB + 16
// * lane.  Inline assembly, so that the compiler does not wait for such loads
// before every LDS read; callers wait with an explicit vmcnt.  M0 carries the LDS
// address; nothing else in these kernels uses it.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_slab4(uint32_t o0, uint32_t o1, uint32_t o2, uint32_t o3, uint64_t base,
                                           uint32_t lds) {
  asm volatile("s_mov_b32 m0, %5\n\ts_nop 0\n\t"
               "global_load_lds_dwordx4 %0, %4\n\t"
               "global_load_lds_dwordx4 %1, %4 offset:1024\n\t"
               "global_load_lds_dwordx4 %2, %4 offset:2048\n\t"
               "global_load_lds_dwordx4 %3, %4 offset:%6"
               :
               : "v"(o0), "v"(o1), "v"(o2), "v"(o3), "s"(base), "s"(lds), "n"(3 * 1024)
               : "memory", "m0");
}
__device__ __forceinline__ void load_slab2(uint32_t o0, uint32_t o1, uint64_t base, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\t"
               "global_load_lds_dwordx4 %0, %2\n\t"
               "global_load_lds_dwordx4 %1, %2 offset:1024"
               :
               : "v"(o0), "v"(o1), "s"(base), "s"(lds)
               : "memory", "m0");
}
// (outside the kernel templates: the cast in their host pass would drop the stubs)
__device__ __forceinline__ uint32_t lds_offset(uint8_t* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)p));
}
#pragma clang diagnostic pop
__device__ __forceinline__ uint32_t scalar(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint64_t scalar(uint64_t x) {
  return uint64_t(scalar(uint32_t(x >> 32))) << 32 | scalar(uint32_t(x));
}
// A word that no kernel writes meanwhile, at a wave-uniform address, through the
// scalar cache.
__device__ __forceinline__ int32_t scalar_load(const int32_t* p) {
  return *(const __attribute__((address_space(4))) int32_t*)scalar(reinterpret_cast<uint64_t>(p));
}
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }  // vmcnt(0)
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(0xC07F); }    // lgkmcnt(0)
// Barrier without the fence of __syncthreads: the caller has waited for what it needs.
__device__ __forceinline__ void bare_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

constexpr int wgs_per_cu(int D) { return D == 64 ? 3 : 2; }

// R groups of four waves work the same columns, each its range of the tiles in buffers of
// its own, and the first joins their states: where a compute unit has one workgroup, a group's
// barriers and loads are waited for while the other works (32 requests of 12 to 32 nodes behind
// 570 to 1050 keys, 32 heads on 8: 23.3 us, with 48% of the wave-cycles still waiting; one group
// 24.5; ranges over workgroups, joined by a kernel of their own, 36).
template <int D, int R>
__global__ __launch_bounds__(64 * kWaves * R, R == 1 ? wgs_per_cu(D) : 1) void tree_tile_kernel(TreeArgs a, int n_ct,
                                                                                              int recip) {
  constexpr int kDch = D / 16, kDt = D / 32;  // 16-dimension chunks of a row, 32-row tiles of O^T
  constexpr int kRowBytes = D * 2, kKch = D / 8;
  constexpr int kSlabBytes = kBlock * D * 2, kTileBytes = kTileBlocks * kSlabBytes;
  constexpr int kInsts = kSlabBytes / 1024;
  __shared__ __attribute__((aligned(16))) uint8_t rings[R][4 * kTileBytes];  // two K tiles, two V tiles
  __shared__ uint32_t s_any[kMaxHalfWords];  // nodes that some row of the tile sees
  __shared__ float s_ml[kWaves][2][32];      // maxima and sums of the second group

  const int tid = threadIdx.x, lane = tid & 63;
  const int group = __builtin_amdgcn_readfirstlane(tid >> 8), wave = __builtin_amdgcn_readfirstlane(tid >> 6) & (kWaves - 1);
  uint8_t* ring = rings[group];
  const int n = lane & 31, hh = lane >> 5;
  const int G = a.Hq / a.Hkv;

  // Workgroup b runs on XCD b % 8; each XCD takes a contiguous range of items, so that a pair's
  // column tiles read its keys through one L2: item = (kv head * B + request) * n_ct + column tile
  const unsigned nb = gridDim.x, per_x = nb >> 3, extra = nb & 7u, x = blockIdx.x & 7u;
  const unsigned item = x * per_x + min(x, extra) + (blockIdx.x >> 3);
  const unsigned pair = item / unsigned(n_ct);
  const int ct = int(item - pair * unsigned(n_ct));
  const int h = int(pair / unsigned(a.B)), r = int(pair % unsigned(a.B));
  const int32_t* bt = a.block_tables + size_t(r) * a.max_blocks;
  auto raw_id = [&](int blk) { return scalar_load(bt + min(blk, a.max_blocks - 1)); };
  // Lengths, and where the range is the whole context the block ids of its first tiles, in one round trip.
  int q0 = scalar_load(a.cu_q + r), q_end = scalar_load(a.cu_q + r + 1), L_in = scalar_load(a.seq_lens + r);
  int first_k, id_k0, next_k, next_v;  // unchecked; the last two of tile 1
  auto ask_ids = [&](int blk0) {
    first_k = raw_id(blk0 + max(wave - 2, 0)), id_k0 = raw_id(blk0 + 2 + wave);
    next_k = raw_id(blk0 + kTileBlocks + 2 + wave), next_v = id_k0;
    __builtin_amdgcn_sched_barrier(0);  // (all on their way before the first is looked at)
  };
  if constexpr (R == 1) ask_ids(0);
  asm volatile("" : "+s"(q0), "+s"(q_end), "+s"(L_in));
  const int L = min(L_in, a.max_blocks * kBlock), q_len = q_end - q0;
  const int first_col = ct * kCols, n_valid = min(min(q_len, a.max_q_len) * G - first_col, kCols);
  if (q0 < 0 || q_end > a.n_rows || q_len <= 0 || q_len > L || n_valid <= 0) return;
  const int start = L - q_len;  // the nodes' first key
  const int n_blk = (L + kBlock - 1) / kBlock;
  const int all_tiles = (L + kKeys - 1) / kKeys, range = (all_tiles + R - 1) / R;
  const int j0 = min(group * range, all_tiles);  // the range's first tile
  const int blk0 = j0 * kTileBlocks;

  // Columns are split into (node, head of the group) by a 16-bit reciprocal of G, exact for the
  // offsets met here, below G + kCols <= 192.
  auto div_g = [&](int u) { return int((unsigned(u) * unsigned(recip)) >> 16); };
  const int t0 = first_col / G, rem0 = first_col - t0 * G;
  const int wave_first = wave * 32;
  const bool active = wave_first < n_valid;
  // This lane's column (padding columns repeat the last valid one).
  const int co = rem0 + min(wave_first + n, n_valid - 1), t = t0 + div_g(co), head = h * G + (co - div_g(co) * G);
  const uint32_t* mask_row = a.masks + size_t(q0 + t) * a.half_words;

  // A wave loads one pool block of every K tile and of every V tile.  In step u the
  // scores of step u + 1 and the products with V of step u - 1 are taken, so K runs half a
  // tile ahead and V half a tile behind: K tile j holds the range's blocks 4j+2 .. 4j+5, V tile j
  // its blocks 4j-2 .. 4j+1, and both are free at the same barrier; K tile -1 holds the
  // first two blocks.
  uint32_t koff[kInsts];
#pragma unroll
  for (int i = 0; i < kInsts; ++i) {
    const int m = i * (1024 / kRowBytes) + lane / kKch;
    koff[i] = uint32_t(diff_key_of_row(m) * kRowBytes + k_slot<D>(m, lane % kKch) * 16 + 1024 - i * 1024);
  }
  const uint32_t voff = uint32_t((lane >> 1) * 32 + v_slot(lane >> 1, lane & 1) * 16);
  const uint32_t ring0 = lds_offset(ring) + wave * kSlabBytes;
  const size_t slab_stride = size_t(a.Hkv) * kSlabBytes;
  const uint64_t kbase = reinterpret_cast<uint64_t>(a.k_pool) - 1024 + size_t(h) * kSlabBytes;
  const uint64_t vbase = reinterpret_cast<uint64_t>(a.v_pool) + size_t(h) * kSlabBytes;
  // (ids past the last block, or outside the pool, read block 0: hidden keys)
  auto usable = [&](int blk, int id) { return (blk < n_blk && id >= 0 && id < a.num_blocks) ? id : 0; };
  auto k_buf = [&](int j) { return unsigned(j & 1) * kTileBytes; };
  auto v_buf = [&](int j) { return unsigned(2 + (j & 1)) * kTileBytes; };
  auto issue_k = [&](int j, int id) {
    const uint64_t base = scalar(kbase + size_t(id) * slab_stride);
    const uint32_t to = scalar(ring0 + k_buf(j));
    if constexpr (kInsts == 4) load_slab4(koff[0], koff[1], koff[2], koff[3], base, to);
    else load_slab2(koff[0], koff[1], base, to);
  };
  auto issue_v = [&](int j, int id) {
    const uint64_t base = scalar(vbase + size_t(id) * slab_stride);
    const uint32_t to = scalar(ring0 + v_buf(j));
    if constexpr (kInsts == 4) load_slab4(voff, voff, voff, voff, base, to);
    else load_slab2(voff, voff, base, to);
  };

  if constexpr (R > 1) ask_ids(blk0);
  bf16x8 qf[kDch];  // Q operand
  {
    const uint16_t* qr = a.q + int64_t(q0 + t) * a.q_stride + size_t(head) * D;
#pragma unroll
    for (int kc = 0; kc < kDch; ++kc) qf[kc] = as_bf16x8(*(const u32x4*)(qr + kc * 16 + hh * 8));
  }
  // Which nodes some row of the tile sees: V of the others is zeroed, and keys behind the last are left out (below).
  if (tid < kMaxHalfWords) s_any[tid] = 0;
  if (wave >= 2) {
    issue_k(-1, usable(blk0 + wave - 2, first_k));
    issue_v(0, usable(blk0 + wave - 2, first_k));
  } else {
#pragma unroll
    for (int i = 0; i < kInsts; ++i) *(u32x4*)(ring + v_buf(0) + wave * kSlabBytes + i * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
  }
  issue_k(0, usable(blk0 + 2 + wave, id_k0));
  // (a thread takes words of one column of the masks, and adds them to LDS once)
  const int n_words = (div_g(rem0 + n_valid - 1) + 1) * a.half_words;
  const int word_step = 64 * kWaves * R / a.half_words * a.half_words;
  const uint32_t* tile_masks = a.masks + size_t(q0 + t0) * a.half_words;
  uint32_t any = tid < min(n_words, word_step) ? tile_masks[tid] : 0u;
  wait_lds();
  bare_barrier();
  if (tid < word_step)
    for (int e = tid + word_step; e < n_words; e += word_step) any |= tile_masks[e];
  if (any) atomicOr(&s_any[tid % a.half_words], any);

  f32x16 sA, sB;          // scores of this step and of the next, in turn
  bf16x8 pA[2], pB[2];    // weights of this step and of the one before, in turn
  pB[0] = pB[1] = as_bf16x8(u32x4{0, 0, 0, 0});
  f32x16 o[kDt];
  float m = -FLT_MAX, l = 0.f;  // l: this lane half's share
#pragma unroll
  for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dt][e] = 0.f;

  // The products of a step: O += V P of the step before (the two V blocks at sV, weights pp), and the scores
  // sn of the next (the 32 K rows at sK); and, independent of both, the exponentials pc of this step's scores
  // sc, one or two behind each product.  LDS operands are read kPrefetch ahead.
  constexpr int kPv = 2 * kDt, kQk = kDch, kPrefetch = 4;
  static_assert(kPv == kQk, "operands alternate");
  float sum;
  auto products = [&](auto with_pv, auto with_exp, auto with_qk, const uint8_t* sV, const uint8_t* sK, f32x16& sc, f32x16& sn,
                      bf16x8(&pp)[2], bf16x8(&pc)[2]) __attribute__((always_inline)) {
    constexpr bool pv = decltype(with_pv)::value, qk = decltype(with_qk)::value;
    constexpr int total = (pv ? kPv : 0) + (qk ? kQk : 0), kEach = decltype(with_exp)::value ? 16 / total : 0;
    // operand i of the sequence: K and V in turn where both are wanted
    auto is_v = [](int i) { return pv && (!qk || (i & 1)); };
    auto index = [](int i) { return pv && qk ? i >> 1 : i; };
    auto operand = [&](int i) -> bf16x8 {
      const int u = index(i);
      if (is_v(i)) {
        const int b = u / kDt, d = (u % kDt) * 32 + n;
        return *(const bf16x8*)(sV + b * kSlabBytes + d * 32 + (v_slot(d, hh) << 4));
      }
      return *(const bf16x8*)(sK + n * kRowBytes + (k_slot<D>(n, u * 2 + hh) << 4));
    };
    if constexpr (qk) {
#pragma unroll
      for (int e = 0; e < 16; ++e) sn[e] = 0.f;
    }
    __builtin_amdgcn_sched_barrier(0);
    bf16x8 buf[kPrefetch + 1];
#pragma unroll
    for (int i = 0; i < kPrefetch && i < total; ++i) buf[i] = operand(i);
    __builtin_amdgcn_sched_barrier(0);
    float t[2], w[2];
#pragma unroll
    for (int i = 0; i < total; ++i) {
      if (i + kPrefetch < total) buf[(i + kPrefetch) % (kPrefetch + 1)] = operand(i + kPrefetch);
      const bf16x8 op = buf[i % (kPrefetch + 1)];
      const int u = index(i);
      if (is_v(i)) o[u % kDt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op, pp[u / kDt], o[u % kDt], 0, 0, 0);
      else sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op, qf[u], sn, 0, 0, 0);
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        const int e = i * kEach + k;
        w[e & 1] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], a.scale_log2, -m));
        t[e & 1] = e < 2 ? w[e & 1] : t[e & 1] + w[e & 1];
        if (e & 1) pc[e >> 3][(e & 7) - 1] = (__bf16)w[0], pc[e >> 3][e & 7] = (__bf16)w[1];
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (kEach > 0) sum = t[0] + t[1];
  };
  // After a step's exponentials: the sum, or where one left [0, 2^8] the maximum anew, O and the
  // sum so far brought to it, and the exponentials again.
  auto settle = [&](f32x16& sc, bf16x8(&pc)[2]) __attribute__((always_inline)) {
    if (__ballot(!(sum <= kSumLimit))) {
      float mx = sc[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, sc[e]);
      const float m_new = fmaxf(m, max_across_halves(mx) * a.scale_log2), alpha = __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] *= alpha;
      sum = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], a.scale_log2, -m));
        pc[e >> 3][e & 7] = (__bf16)w;
        sum += w;
      }
    }
    l += sum;
  };
  using yes = std::true_type;
  using no = std::false_type;

  // Zero V of the keys of this wave's block of tile j that no row sees (its own loads of it have
  // landed; others read it behind the next barrier): slots that hold no token may have any bits, and
  // a weight of 0 does not hide a NaN.
  auto zero_hidden_v = [&](int j) {
    const int k0 = (j0 + j) * kKeys + (wave - 2) * kBlock;
    if (k0 + kBlock <= start || (j == 0 && wave < 2)) return;
    uint32_t lo, hi;
    tree_words(s_any, a.half_words, k0, start, &lo, &hi);
    const uint32_t seen = tree_window(k0, start, L, lo, hi) & 0xFFFFu;
    if (seen == 0xFFFFu) return;
    const uint32_t mine = seen >> (8 * v_slot(lane >> 1, lane & 1));
    uint8_t* sV = ring + v_buf(j) + wave * kSlabBytes;
#pragma unroll
    for (int i = 0; i < kInsts; ++i) {
      u32x4* q = (u32x4*)(sV + i * 1024 + lane * 16);
      u32x4 v = *q;
#pragma unroll
      for (int w = 0; w < 4; ++w)
        v[w] &= (mine >> (2 * w) & 1u ? 0x0000FFFFu : 0u) | (mine >> (2 * w + 1) & 1u ? 0xFFFF0000u : 0u);
      *q = v;
    }
    wait_lds();
  };

  // One step (the first one multiplies weights of 0 with zeros).
  auto body = [&](int u, f32x16& sc, f32x16& sn, bf16x8(&pp)[2], bf16x8(&pc)[2]) __attribute__((always_inline)) {
    const int j = u >> 1, k0 = j0 * kKeys + u * 32;
    if (k0 + 32 > start) {
      uint32_t lo, hi;
      tree_words(mask_row, a.half_words, k0, start, &lo, &hi);
      const uint32_t mine = tree_window(k0, start, L, lo, hi) >> (8 * hh);
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (!(mine >> ((e >> 3) * 16 + (e & 7)) & 1u)) sc[e] = -INFINITY;
    }
    const uint8_t *sV = ring + v_buf(j) + (u & 1) * 2 * kSlabBytes, *sK = ring + k_buf(j) + (u & 1) * 32 * kRowBytes;
    products(yes(), yes(), yes(), sV, sK, sc, sn, pp, pc);
    settle(sc, pc);
  };
  // Two steps a tile.  Before the first of tile j: wait for this wave's loads of K(j) and V(j);
  // barrier; issue K(j+1) and V(j+1) into the buffers of tile j-1, which every wave has
  // left behind.  The scores of the step behind the last are computed from whatever is there, and ignored.
  auto turn = [&](int j) __attribute__((always_inline)) {
    wait_loads();
    zero_hidden_v(j);
    bare_barrier();
  };
  wait_loads();
  wait_lds();
  bare_barrier();
  // The range's tiles are those up to the last node that these columns' rows see, and a tree's rows see none behind
  // their own (4 requests of 1000 nodes, 500 keys before them, 32 heads on 8: 180 us with all keys, 115 so; 32 of 198
  // to 238 behind 370 to 500: 120, 110; the 128 of above: 591, 584).
  const uint32_t seen = lane < a.half_words ? s_any[lane] : 0u;
  const uint64_t some = __ballot(seen != 0);
  const int top = some ? 63 - __builtin_clzll(some) : 0;
  const uint32_t top_bits = __builtin_amdgcn_readlane(seen, top);
  const int n_seen = top_bits ? min(top * 32 + 32 - __builtin_clz(top_bits), q_len) : 0;
  const int seen_tiles = (start + n_seen + kKeys - 1) / kKeys, turns = min(range, seen_tiles);
  const int n_tiles = max(min(j0 + range, seen_tiles) - j0, 0);
  if (active) products(no(), no(), yes(), ring, ring + k_buf(-1) + 32 * kRowBytes, sB, sA, pB, pA);
  for (int j = 0; j < n_tiles; ++j) {
    turn(j);
    const int kb = blk0 + (j + 1) * kTileBlocks + 2 + wave, vb = kb - 4;
    if (j + 1 < n_tiles) issue_k(j + 1, usable(kb, next_k));
    issue_v(j + 1, usable(vb, next_v));
    next_k = raw_id(kb + kTileBlocks);
    next_v = raw_id(vb + kTileBlocks);
    if (active) {
      // (the ids' scalar loads are waited for here, and not with the first LDS operands of the products)
      asm volatile("" : "+s"(next_k), "+s"(next_v));
      body(2 * j, sA, sB, pB, pA);
      body(2 * j + 1, sB, sA, pA, pB);
    }
  }
  if constexpr (R > 1)  // (the second range may have fewer tiles than the first)
    for (int j = n_tiles; j < turns; ++j) bare_barrier();
  turn(n_tiles);
  if (active && n_tiles > 0) products(yes(), no(), no(), ring + v_buf(n_tiles), ring, sA, sB, pB, pA);
  float total = add_across_halves(l);
  if constexpr (R == 2) {
    // O as it lies in the lanes, by way of the second group's buffers (behind a barrier: its waves have all left them)
    __syncthreads();
    f32x4* so = reinterpret_cast<f32x4*>(rings[1]) + wave * (kDt * 4 * 64) + lane;
    if (group == 1 && active) {
#pragma unroll
      for (int i = 0; i < kDt * 4; ++i) {
        const f32x16& x = o[i >> 2];
        so[i * 64] = f32x4{x[(i & 3) * 4], x[(i & 3) * 4 + 1], x[(i & 3) * 4 + 2], x[(i & 3) * 4 + 3]};
      }
      if (hh == 0) s_ml[wave][0][n] = m, s_ml[wave][1][n] = total;
    }
    __syncthreads();
    if (group == 1 || !active) return;
    const float m1 = s_ml[wave][0][n], top = fmaxf(m, m1);
    const float w0 = __builtin_amdgcn_exp2f(m - top), w1 = __builtin_amdgcn_exp2f(m1 - top);
    total = total * w0 + s_ml[wave][1][n] * w1;
#pragma unroll
    for (int i = 0; i < kDt * 4; ++i) {
      const f32x4 v = so[i * 64];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i >> 2][(i & 3) * 4 + e] = o[i >> 2][(i & 3) * 4 + e] * w0 + v[e] * w1;
    }
  }
  if (!active) return;

  const float inv = total > 0.f ? 1.f / total : 0.f;
  // The rows leave through LDS, so that whole 128-byte half rows are stored (a lane
  // holds 8-byte pieces of one row).  4 KiB a wave, where K was, which every wave has left
  // behind: 32 rows of 64 dimensions a pass, 16-byte chunks XOR-swizzled by row.
  uint8_t* tb = ring + wave * 4096;
  size_t orow[4];
  bool ok[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = wave_first + i * 8 + (lane >> 3), u = rem0 + min(c, n_valid - 1), tt = div_g(u);
    ok[i] = c < n_valid;
    orow[i] = (size_t(q0 + t0 + tt) * a.Hq + h * G + (u - tt * G)) * D + (lane & 7) * 8;
  }
#pragma unroll
  for (int half = 0; half < kDt / 2; ++half) {
#pragma unroll
    for (int dl = 0; dl < 2; ++dl)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4) {
        bf16x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (__bf16)(o[2 * half + dl][g4 * 4 + e] * inv);
        *(bf16x4*)(tb + n * 128 + (((dl * 4 + g4) ^ (n & 7)) << 4) + hh * 8) = v;
      }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = i * 8 + (lane >> 3);
      const u32x4 v = *(const u32x4*)(tb + row * 128 + (((lane & 7) ^ (row & 7)) << 4));
      if (ok[i]) *(u32x4*)(a.out + orow[i] + half * 64) = v;
    }
  }
}

}  // namespace

namespace ilpc {

hipError_t launch_tree_tiles(const TreeArgs& a, int groups, int n_ct, hipStream_t stream) {
  const dim3 grid{unsigned(int64_t(a.B) * a.Hkv * n_ct)}, block{unsigned(64 * kWaves * groups)};
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, n_ct, 65536 / (a.Hq / a.Hkv) + 1);
  };
  if (a.D == 128) {
    if (groups == 1) launch(tree_tile_kernel<128, 1>);
    else launch(tree_tile_kernel<128, 2>);
  } else {
    if (groups == 1) launch(tree_tile_kernel<64, 1>);
    else launch(tree_tile_kernel<64, 2>);
  }
  return hipGetLastError();
}

}  // namespace ilpc
