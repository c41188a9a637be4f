// Differential attention of many query columns, for gfx950 (the mathematics and
// the kernel for few columns are in diff_attn.hip).
//
// A workgroup of four waves works 128 columns -- (token, head of the group) pairs
// of one (request, kv head) -- against 64-key tiles of K and V in LDS, each wave
// 32 columns with both of their maps.  Per 32 keys and wave, on
// v_mfma_f32_32x32x16_bf16:
//   S_m^T = K_m Q_m^T            D/32 products a map,
//   O^T += V^T P^T               2 * D/32 products,
// in two passes over the keys.
//
// Precision.  y = (A_1 - lambda A_2) V is a difference, and where the maps nearly
// agree it is much smaller than its terms; weights of one map rounded to bf16 would
// leave an error of up to 2^-8 of the terms.  The difference of the weights is therefore
// taken in fp32 and then rounded, which needs both maps' sums beforehand:
//   pass 1, K alone:   m_m, l_m = sum 2^(s log2(e) q_m.k_m - m_m),
//   pass 2, K and V:   y = sum (p_1 - (lambda l_1 / l_2) p_2) v / l_1.
// The rounding to bf16, half a step of the combined weight, is a choice: the products with V
// then take half the time that two bf16 numbers a weight would, as the kernel for few
// columns has.  Error against 64 bits (2-norm; the output's own rounding is 0.0017 of it): q of
// standard deviation 0.09, 0.3, 1, 2, 4, 30: 0.0023, 0.0023, 0.0023, 0.0021, 0.0020, 0.0018;
// scores of one map rising by 0.5 every 32 of 3000 keys 0.0023; maps that nearly agree,
// everywhere or behind some first keys, 0.0017 to 0.0024.
// One pass with the ratio of the sums so far, sum (p_1 - beta p_2) v and sum p_2 v set
// right at the end, is as many products (six D-wide ones a column and key: 2 + 4, here
// 2 + 2 + 2), took 0.72 to 0.87 of the time and was not kept: weights rounded against a ratio that the
// first keys have and the others do not left 0.006 to 0.026 of nearly agreeing maps.
//
// What bounds it: vector instructions.  242 a step and wave in both passes, 64 of them
// exponentials of 8 cycles, keep a SIMD busy 66% of the time, the products 38%, 16% both at
// once (a product also holds up the vector instructions beside it, 12 to 25 cycles each): 64
// prompts of 1.9 K tokens (64/8 heads) 8.2 to 9.1 ms (box to box), 0.73 to 0.83 PFLOP/s of
// products.  Tried, within 1% of this: the next step's scores in a second set of registers,
// their products placed between the exponentials; 3 or 6 LDS operands in flight instead of 4;
// the products' raised priority left out.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "../../include/ilpc.h"
#include "diff_attn.h"
#include "ilpc_internal.h"

namespace {

using namespace ilpc;

constexpr int kBlock = 16;
constexpr int kWaves = 4;
constexpr int kCols = 32 * kWaves;  // columns of a workgroup
constexpr int kKeys = 64;           // keys of a tile: two steps of 32
constexpr int kTileBlocks = kKeys / kBlock;
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

// 16-byte chunk of a K or Q row in memory that is logical chunk c, in an order in
// which map 1's dimensions come first: the same, or in the pair layout quarters
// 0, 2, 1, 3 of the row.
template <int D>
__device__ __forceinline__ int source_chunk(int c, int pairs) {
  constexpr int kQuarter = D / 32;  // 16-byte chunks of a quarter row
  const int quarter = c / kQuarter;
  return pairs && (quarter == 1 || quarter == 2) ? c + (quarter == 1 ? kQuarter : -kQuarter) : c;
}

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
               "global_load_lds_dwordx4 %3, %4 offset:3072"
               :
               : "v"(o0), "v"(o1), "v"(o2), "v"(o3), "s"(base), "s"(lds)
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

enum { kByPair, kByRows };  // how workgroups find their column tile

constexpr int wgs_per_cu(int D) { return D == 64 ? 3 : 2; }

template <int D>
__global__ __launch_bounds__(64 * kWaves, wgs_per_cu(D)) void diff_prefill_kernel(DiffArgs a, int recip, int numbering) {
  constexpr int kDch = D / 16;                          // 16-dimension chunks of a row: half of them map 1's
  constexpr int kDt = D / 32;                           // 32-row tiles of O^T
  constexpr int kRowBytes = D * 2, kKch = D / 8;
  constexpr int kSlabBytes = kBlock * D * 2;
  constexpr int kTileBytes = kTileBlocks * kSlabBytes;
  constexpr int kInsts = kSlabBytes / 1024;
  __shared__ __attribute__((aligned(16))) uint8_t ring[4 * kTileBytes];  // two K tiles, two V tiles
  __shared__ __attribute__((aligned(16))) float s_norm[D];               // norm weight, or ones

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, hh = lane >> 5;
  const int G = a.Hq / a.Hkv;

  int r, h, place;  // request, kv head, which of the request's column tiles (the heaviest first)
  if (numbering == kByPair) {
    // Grid: 8 (XCDs: workgroup b runs on XCD b % 8) x column tiles x pairs / 8.  An XCD
    // takes every eighth (request, kv head), its column tiles one after the other: they
    // read the same keys through one L2.
    const unsigned pair = blockIdx.z * 8u + blockIdx.x;
    if (pair >= unsigned(a.B) * unsigned(a.Hkv)) return;
    r = int(pair / unsigned(a.Hkv)), h = int(pair % unsigned(a.Hkv));
    place = int(blockIdx.y);
  } else {
    // Grid: 8 x numbers / 8 x kv heads.  Request r has the numbers from (columns before
    // it) / 128 + r on, which is room for its tiles whatever the lengths; found eight
    // probes a round trip.
    const unsigned e = blockIdx.y * 8u + blockIdx.x;
    auto first = [&](int row, int i) {
      return unsigned(uint64_t(unsigned(max(row, 0))) * unsigned(G) / kCols) + unsigned(i);
    };
    int lo = 0, hi = a.B;  // first(lo) <= e < first(hi)
    unsigned base = 0;
    while (hi - lo > 1) {
      const int st = (hi - lo + 7) >> 3;
      int row[7];
      unsigned f[7];
#pragma unroll
      for (int k = 0; k < 7; ++k) row[k] = scalar_load(a.cu_q + min(lo + st * (k + 1), a.B));
      __builtin_amdgcn_sched_barrier(0);  // (all on their way before the first is looked at)
#pragma unroll
      for (int k = 0; k < 7; ++k) f[k] = first(row[k], min(lo + st * (k + 1), a.B));
      int next = lo;
#pragma unroll
      for (int k = 0; k < 7; ++k)
        if (lo + st * (k + 1) < hi && f[k] <= e) next = lo + st * (k + 1), base = f[k];
      hi = min(next + st, hi);
      lo = next;
    }
    r = lo, h = int(blockIdx.z), place = int(e - base);
  }
  const int32_t* bt = a.block_tables + size_t(r) * a.max_blocks;
  auto raw_id = [&](int blk) { return scalar_load(bt + min(blk, a.max_blocks - 1)); };
  // Lengths and the block ids of the first tiles in one round trip.
  const int q0 = scalar_load(a.cu_q + r), q_end = scalar_load(a.cu_q + r + 1), L_in = scalar_load(a.seq_lens + r);
  const int first_k = raw_id(max(wave - 2, 0)), k0 = raw_id(2 + wave), v0 = raw_id(wave);
  int next_k = raw_id(kTileBlocks + 2 + wave), next_v = v0;  // of the next tile, unchecked
  __builtin_amdgcn_sched_barrier(0);  // (no test of one ahead of the last load)
  asm volatile("" : : "s"(q0), "s"(q_end), "s"(L_in), "s"(first_k), "s"(k0), "s"(v0), "s"(next_k));
  const int L = min(L_in, a.max_blocks * kBlock);
  const int q_len = q_end - q0;
  const int64_t all_cols = int64_t(min(q_len, a.max_q_len)) * G;
  const int tile = int((all_cols + kCols - 1) / kCols) - 1 - place;
  if (q0 < 0 || q_end > a.n_rows || q_len <= 0 || q_len > L || tile < 0) return;
  const unsigned col0 = unsigned(tile) * kCols;
  // Columns are split into (row, head of the group) by a 16-bit reciprocal of G,
  // exact for the offsets met here, below G + kCols <= 192.
  auto div_g = [&](int u) { return int((unsigned(u) * unsigned(recip)) >> 16); };
  const int row_a = int(col0 / unsigned(G)), rem0 = int(col0 - unsigned(row_a) * unsigned(G));
  const int n_valid = int(min(all_cols - col0, int64_t(kCols)));
  const int wave_first = wave * 32;
  const bool active = wave_first < n_valid;
  // This lane's column (padding columns repeat the last valid one).
  const int co = min(wave_first + n, n_valid - 1);
  const int t_off = div_g(rem0 + co), head = h * G + (rem0 + co - t_off * G);
  const int pos0 = L - q_len + row_a;
  const int pos = pos0 + t_off;
  const int wave_pos_min = pos0 + div_g(rem0 + min(wave_first, n_valid - 1));
  const int wave_pos_max = pos0 + div_g(rem0 + min(wave_first + 32, n_valid) - 1);
  const int key_lim = pos0 + div_g(rem0 + n_valid - 1) + 1;  // keys from here on are hidden from all columns
  const int n_tiles = (key_lim + kKeys - 1) / kKeys;
  const int n_blk = (key_lim + kBlock - 1) / kBlock;
  const int last_step = active ? wave_pos_max / 32 : -1;  // last step with a key that some column of the wave sees

  // A wave loads one pool block of every K tile and of every V tile.  K runs half
  // a tile ahead: tile j holds the blocks 4j+2 .. 4j+5, whose scores are taken
  // while V blocks 4j .. 4j+3 are multiplied, so that both are free at the same
  // barrier; tile -1 holds the first two blocks.
  uint32_t koff[kInsts];
#pragma unroll
  for (int i = 0; i < kInsts; ++i) {
    const int m = i * (1024 / kRowBytes) + lane / kKch;
    const int c = source_chunk<D>(k_slot<D>(m, lane % kKch), a.pairs);
    koff[i] = uint32_t(diff_key_of_row(m) * kRowBytes + c * 16 + 1024 - i * 1024);
  }
  const uint32_t voff = uint32_t((lane >> 1) * 32 + v_slot(lane >> 1, lane & 1) * 16);
  const uint32_t ring0 = lds_offset(ring) + wave * kSlabBytes;
  const size_t slab_stride = size_t(a.Hkv) * kSlabBytes;
  const uint64_t kbase = reinterpret_cast<uint64_t>(a.k_pool) - 1024 + size_t(h) * kSlabBytes;
  const uint64_t vbase = reinterpret_cast<uint64_t>(a.v_pool) + size_t(h) * kSlabBytes;
  // (ids past the last block, or outside the pool, read block 0: masked keys)
  auto usable = [&](int blk, int id) { return (blk < n_blk && id >= 0 && id < a.num_blocks) ? id : 0; };
  // Tile j of K in the first pass (0) and the second (1), and of V.  The second pass's
  // first tiles have buffers that the first pass's last tile does not hold.
  auto k_buf = [&](int pass, int j) { return unsigned(2 * pass + (j & 1)) * kTileBytes; };
  auto v_buf = [&](int j) { return unsigned((n_tiles + j) & 1) * kTileBytes; };
  auto issue_k = [&](int pass, int j, int id) {
    const uint64_t base = scalar(kbase + size_t(id) * slab_stride);
    const uint32_t to = scalar(ring0 + k_buf(pass, j));
    if constexpr (kInsts == 4) load_slab4(koff[0], koff[1], koff[2], koff[3], base, to);
    else load_slab2(koff[0], koff[1], base, to);
  };
  auto issue_v = [&](int j, int id) {
    const uint64_t base = scalar(vbase + size_t(id) * slab_stride);
    const uint32_t to = scalar(ring0 + v_buf(j));
    if constexpr (kInsts == 4) load_slab4(voff, voff, voff, voff, base, to);
    else load_slab2(voff, voff, base, to);
  };

  if (wave >= 2) issue_k(0, -1, usable(wave - 2, first_k));
  issue_k(0, 0, usable(2 + wave, k0));
  bf16x8 qf[kDch];  // Q operand, map 1's chunks first
  {
    const uint16_t* qr = a.q + int64_t(q0 + row_a + t_off) * a.q_stride + size_t(head) * D;
#pragma unroll
    for (int kc = 0; kc < kDch; ++kc)
      qf[kc] = as_bf16x8(*(const u32x4*)(qr + source_chunk<D>(kc * 2, a.pairs) * 8 + hh * 8));
  }
  const float lam = a.ep.lambda[head];
  if (tid < D) s_norm[tid] = a.ep.norm_w ? a.ep.norm_w[tid] : 1.f;

  f32x16 s1, s2;  // scores of the next step
  float m1 = -FLT_MAX, m2 = -FLT_MAX, l1 = 0.f, l2 = 0.f;  // l: this lane half's share

  auto mask = [&](int step) {
    const int j0 = step * 32;
    if (j0 + 31 <= wave_pos_min) return;
    const int rel = pos - j0 - hh * 8;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const bool hide = (e >> 3) * 16 + (e & 7) > rel;
      s1[e] = hide ? -INFINITY : s1[e];
      s2[e] = hide ? -INFINITY : s2[e];
    }
  };

  // Sums of a masked step's exponentials against the running maxima, which are taken
  // anew where a lane's sum leaves [0, 2^8], the first step among them.
  auto add_step = [&]() __attribute__((always_inline)) {
    float t1, t2;
    auto exps = [&]() __attribute__((always_inline)) {
      float u1[2], u2[2];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float a1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s1[e], a.scale_log2, -m1));
        const float a2 = __builtin_amdgcn_exp2f(__builtin_fmaf(s2[e], a.scale_log2, -m2));
        u1[e & 1] = e < 2 ? a1 : u1[e & 1] + a1;
        u2[e & 1] = e < 2 ? a2 : u2[e & 1] + a2;
      }
      t1 = u1[0] + u1[1];
      t2 = u2[0] + u2[1];
    };
    exps();
    if (__ballot(!(t1 <= kSumLimit) || !(t2 <= kSumLimit))) {
      float x1 = s1[0], x2 = s2[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) x1 = fmaxf(x1, s1[e]), x2 = fmaxf(x2, s2[e]);
      const float n1 = fmaxf(m1, max_across_halves(x1) * a.scale_log2);
      const float n2 = fmaxf(m2, max_across_halves(x2) * a.scale_log2);
      l1 *= __builtin_amdgcn_exp2f(m1 - n1), l2 *= __builtin_amdgcn_exp2f(m2 - n2);
      m1 = n1, m2 = n2;
      exps();
    }
    l1 += t1;
    l2 += t2;
  };

  f32x16 o[kDt];       // sum of (p_1 - beta p_2) v
  bf16x8 pc[2];        // p_1 - beta p_2 of the step whose products with V are due

  // Products: O += V P of a step (the two V blocks at sV), then the scores of the
  // next (the 32 K rows at sK), the LDS operands read kPrefetch ahead.
  constexpr int kPv = 2 * kDt, kQk = kDch, kPrefetch = 4;
  auto products = [&](auto with_pv, auto with_qk, const uint8_t* sV, const uint8_t* sK)
                      __attribute__((always_inline)) {
    constexpr int first = decltype(with_pv)::value ? 0 : kPv;
    constexpr int last = decltype(with_qk)::value ? kPv + kQk : kPv;
    // score products alternate between the maps, which are independent chains
    auto chunk_of = [](int u) { return (u & 1) * (kDch / 2) + (u >> 1); };
    auto operand = [&](int st) -> bf16x8 {
      if (st < kPv) {
        const int b = st / kDt, d = (st % kDt) * 32 + n;
        return *(const bf16x8*)(sV + b * kSlabBytes + d * 32 + (v_slot(d, hh) << 4));
      }
      return *(const bf16x8*)(sK + n * kRowBytes + (k_slot<D>(n, chunk_of(st - kPv) * 2 + hh) << 4));
    };
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (decltype(with_qk)::value) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s1[e] = 0.f, s2[e] = 0.f;
    }
    bf16x8 buf[kPrefetch];
#pragma unroll
    for (int st = first; st < first + kPrefetch && st < last; ++st) buf[st % kPrefetch] = operand(st);
#pragma unroll
    for (int st = first; st < last; ++st) {
      const bf16x8 op = buf[st % kPrefetch];
      if (st + kPrefetch < last) buf[st % kPrefetch] = operand(st + kPrefetch);
      if (st < kPv) {
        o[st % kDt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op, pc[st / kDt], o[st % kDt], 0, 0, 0);
      } else {
        const int u = st - kPv;
        if (u & 1) s2 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op, qf[chunk_of(u)], s2, 0, 0, 0);
        else s1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op, qf[chunk_of(u)], s1, 0, 0, 0);
      }
    }
    // pin that order: kPrefetch reads, then the product of one operand a read
    constexpr int steps = last - first, lead = steps < kPrefetch ? steps : kPrefetch;
    __builtin_amdgcn_sched_group_barrier(0x100, lead, 0);
#pragma unroll
    for (int st = 0; st < steps; ++st) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if (st < steps - lead) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
  };
  using yes = std::true_type;
  using no = std::false_type;

  // Zero the V rows of keys >= key_lim in this wave's block of V tile j (its own
  // loads of it have landed; others read it behind the next barrier): unwritten
  // slots may hold any bits, and a weight of 0 does not hide a NaN.
  auto zero_v_tail = [&](int j) {
    const int nv = key_lim - (j * kKeys + wave * kBlock);
    if (nv >= kBlock) return;
    uint8_t* sV = ring + v_buf(j) + wave * kSlabBytes;
    const int keep = nv - v_slot(lane >> 1, lane & 1) * 8;
#pragma unroll
    for (int i = 0; i < kInsts; ++i) {
      u32x4* p = (u32x4*)(sV + i * 1024 + lane * 16);
      u32x4 v = *p;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] &= (2 * e < keep ? 0x0000FFFFu : 0u) | (2 * e + 1 < keep ? 0xFFFF0000u : 0u);
      *p = v;
    }
    wait_lds();
  };

  // First pass, the sums of both maps.  Two steps a tile.  Before the first of tile j:
  // wait for this wave's loads of K(j); barrier; issue K(j+1) into the buffer of tile j-1,
  // which every wave has left behind, or behind the last tile the second pass's first
  // ones.  The scores of a step past the wave's last one are computed and ignored.
  wait_loads();
  wait_lds();
  bare_barrier();
  if (active) products(no(), yes(), ring, ring + k_buf(0, -1) + 32 * kRowBytes);
  for (int u = 0; u < 2 * n_tiles; ++u) {
    const int j = u >> 1;
    if (!(u & 1)) {
      if (j > 0) wait_loads();
      bare_barrier();
      if (j + 1 < n_tiles) {
        const int kb = (j + 1) * kTileBlocks + 2 + wave;
        issue_k(0, j + 1, usable(kb, next_k));
        next_k = raw_id(kb + kTileBlocks);
      } else {
        if (wave >= 2) issue_k(1, -1, usable(wave - 2, first_k));
        issue_k(1, 0, usable(2 + wave, k0));
        issue_v(0, usable(wave, v0));
        next_k = raw_id(kTileBlocks + 2 + wave);
        next_v = raw_id(kTileBlocks + wave);
      }
    }
    if (u <= last_step) {
      mask(u);
      add_step();
      // (the ids' scalar loads are waited for here, and not with the first LDS operands of the products)
      asm volatile("" : "+s"(next_k), "+s"(next_v));
      products(no(), yes(), ring, ring + k_buf(0, j) + (u & 1) * 32 * kRowBytes);
    }
  }
  const float sum1 = add_across_halves(l1), sum2 = add_across_halves(l2);
  const float beta = lam * sum1 / sum2, inv = 1.f / sum1;

  // Second pass, the products with V: the same over K and V.
#pragma unroll
  for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dt][e] = 0.f;
  wait_loads();
  bare_barrier();
  if (active) products(no(), yes(), ring, ring + k_buf(1, -1) + 32 * kRowBytes);
  for (int u = 0; u < 2 * n_tiles; ++u) {
    const int j = u >> 1;
    if (!(u & 1)) {
      if (j > 0) wait_loads();
      zero_v_tail(j);
      bare_barrier();
      if (j + 1 < n_tiles) {
        const int kb = (j + 1) * kTileBlocks + 2 + wave, vb = kb - 2;
        issue_k(1, j + 1, usable(kb, next_k));
        issue_v(j + 1, usable(vb, next_v));
        next_k = raw_id(kb + kTileBlocks);
        next_v = raw_id(vb + kTileBlocks);
      }
    }
    if (u <= last_step) {
      mask(u);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float a1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s1[e], a.scale_log2, -m1));
        const float a2 = __builtin_amdgcn_exp2f(__builtin_fmaf(s2[e], a.scale_log2, -m2));
        pc[e >> 3][e & 7] = (__bf16)__builtin_fmaf(-beta, a2, a1);
      }
      asm volatile("" : "+s"(next_k), "+s"(next_v));
      products(yes(), yes(), ring + v_buf(j) + (u & 1) * 2 * kSlabBytes, ring + k_buf(1, j) + (u & 1) * 32 * kRowBytes);
    }
  }
  if (!active) return;

  float sq = 0.f;
#pragma unroll
  for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      o[dt][e] *= inv;
      sq += o[dt][e] * o[dt][e];
    }
  float fac = a.ep.scale;
  if (a.ep.norm_w) fac *= rsqrtf(add_across_halves(sq) * (1.f / D) + a.ep.eps);
  // The rows leave through LDS, so that whole 128-byte half rows are stored (a lane
  // holds 8-byte pieces of one row).  4 KiB a wave, in the buffers of the tile
  // before the last, which every wave has left behind: 32 rows of 64 dimensions a
  // pass, 16-byte chunks XOR-swizzled by row.
  uint8_t* tb = ring + (wave < 2 ? k_buf(1, n_tiles) : v_buf(n_tiles)) + (wave & 1) * 4096;
  size_t orow[4];
  bool ok[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = wave_first + i * 8 + (lane >> 3), u = rem0 + min(c, n_valid - 1), t = div_g(u);
    ok[i] = c < n_valid;
    orow[i] = (size_t(q0 + row_a + t) * a.Hq + h * G + (u - t * G)) * D + (lane & 7) * 8;
  }
#pragma unroll
  for (int p = 0; p < kDt / 2; ++p) {
#pragma unroll
    for (int dl = 0; dl < 2; ++dl)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4) {
        const f32x4 w = *(const f32x4*)&s_norm[(2 * p + dl) * 32 + g4 * 8 + hh * 4];
        bf16x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (__bf16)(o[2 * p + dl][g4 * 4 + e] * (fac * w[e]));
        *(bf16x4*)(tb + n * 128 + (((dl * 4 + g4) ^ (n & 7)) << 4) + hh * 8) = v;
      }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = i * 8 + (lane >> 3);
      const u32x4 v = *(const u32x4*)(tb + row * 128 + (((lane & 7) ^ (row & 7)) << 4));
      if (ok[i]) *(u32x4*)(a.out + orow[i] + p * 64) = v;
    }
  }
}

}  // namespace

namespace ilpc {

int launch_diff_prefill(const DiffArgs& a, hipStream_t stream) {
  // By pair where that fills all XCDs evenly and most numbers hold rows (the host knows
  // the longest request and the sum of all); else by rows, as far as that grid goes; past
  // that by pair again, up to 2^25 workgroups, most of which may be idle.
  const int64_t G = a.Hq / a.Hkv, n_ct = (a.max_q_len * G + kCols - 1) / kCols, pairs = int64_t(a.B) * a.Hkv;
  const int64_t numbers = a.n_rows * G / kCols + a.B;
  const bool even = (pairs % 8 == 0 || pairs >= 64) && 2 * a.B * n_ct <= 3 * numbers;
  const bool by_pair = even || numbers > 8 * 65535 || a.Hkv > 65535;
  if (by_pair && !even && pairs * n_ct > (1 << 25)) return ILPC_EUNSUP;
  if (device_cus() <= 0) return ILPC_EHIP;
  const dim3 grid(8, unsigned(by_pair ? n_ct : (numbers + 7) / 8), unsigned(by_pair ? (pairs + 7) / 8 : a.Hkv));
  const dim3 block(64 * kWaves);
  const int recip = 65536 / int(G) + 1, numbering = by_pair ? kByPair : kByRows;
  if (a.D == 128) hipLaunchKernelGGL(diff_prefill_kernel<128>, grid, block, 0, stream, a, recip, numbering);
  else hipLaunchKernelGGL(diff_prefill_kernel<64>, grid, block, 0, stream, a, recip, numbering);
  return hipGetLastError() == hipSuccess ? ILPC_OK : ILPC_EHIP;
}

}  // namespace ilpc
