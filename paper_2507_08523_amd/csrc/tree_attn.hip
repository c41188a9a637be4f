// Attention of drafted tokens over the paged cache, for gfx950: each request's newest
// tokens are a tree, of which a token sees what its mask names, and all keys before it.
//
// Request r has L_r keys, the last n_r of them its nodes (InferLog section 2.1.2: the
// newest tokens attend to the cached KV of their context and to their own).  With P =
// L_r - n_r and mask m_i of node i,
//   out_i = sum_j p_j v_j / sum_j p_j,  p_j = 2^(s log2(e) q_i.k_j - max),
// over the keys j < P and the keys P + b for the bits b of m_i.  A row that sees no key
// gives 0.  Columns are (node, head of the group) pairs of a (request, kv head), so all
// heads of a group share every K/V read.
//
// 32 columns a wave, on v_mfma_f32_32x32x16_bf16:
//   S^T = K Q^T,  O^T += V^T P^T,
// with the softmax in fp32; weights enter the products with V rounded to bf16 (half a
// step, 2^-8 of each; the sums add the fp32 values).  Every wave streams its range of
// the keys from the pools into registers, two pool blocks (32 keys) a step, the next
// step's loads in flight; W waves of a workgroup and n_split workgroups share a column
// tile's keys where there are too few tiles to fill the chip, and their states are
// joined at the end.
//
// What bounds it: with few tiles the chain of one wave's steps, each about 1 us of loads,
// LDS, products and exponentials one after the other, and the joins (64 nodes of one
// request behind 4096 keys, 32 heads on 8, D 128: 17 us and 4 for the join, 18.6 in a row of calls;
// its 18 MB would take 3.6; 43% of the wave-cycles wait for loads, 41% issue).  Two steps of
// loads ahead cost 1 us more, no maximum at all saves nothing.  4 requests of 8
// nodes, 4 heads of D 64 on one: 4.4 us, little more than a launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/ilpc.h"
#include "ilpc_internal.h"
#include "tree_attn.h"

namespace {

using namespace ilpc;

constexpr int kBlock = 16;
constexpr int kStepKeys = 32;        // keys a step (two pool blocks)
constexpr int kTileCols = 32;        // query columns of a wave
constexpr int kMaxGroups = 64;       // most workgroups to a tile's keys (a lane of the join each)
constexpr int kMaxNodes = 1024;      // of a request
constexpr float kLazyRescale = 8.f;  // log2 growth of a column max tolerated before rescaling O

template <int D>
struct StepRegs {
  u32x4 k[D / 16];     // K rows of the step, in the order of memory
  u32x4 v[2][D / 32];  // V^T operand, [pool block of the step][32-dimension tile]
  uint32_t lo, hi;     // mask words of a step that reaches into the tree
};

// Orders a wave's LDS stores and reads across its lanes (the hardware keeps a wave's
// LDS operations in order; the compiler has to as well).
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

constexpr int group_waves(int W) { return W > 4 ? W : 4; }  // waves of a workgroup, W of them to a tile

template <int D, int W>
__global__ __launch_bounds__(64 * group_waves(W), 2) void tree_stream_kernel(TreeArgs a, int n_ct, int n_split) {
  constexpr int kDch = D / 16, kDt = D / 32, kWavesPerGroup = group_waves(W);
  // Q^T of each wave and the K rows of its step in LDS; for the join the same space
  // holds every wave's O, a row of kRow floats a column.
  constexpr int kRow = D + 4, kCols = kTileCols;
  constexpr int kQBytes = kWavesPerGroup * kDch * 64 * 16, kOBytes = kWavesPerGroup * kCols * kRow * 4;
  constexpr int kRowPieces = D / 8 + 1;  // 16-byte pieces of a K row in LDS: one more than it has
  constexpr int kKBytes = kWavesPerGroup * kStepKeys * kRowPieces * 16;
  static_assert(kOBytes >= kQBytes + kKBytes, "the join's rows are the larger");
  __shared__ __attribute__((aligned(16))) uint8_t lds[kOBytes];
  __shared__ float s_m[kWavesPerGroup][kCols], s_l[kWavesPerGroup][kCols];
  u32x4(*q_lds)[kDch][64] = reinterpret_cast<u32x4(*)[kDch][64]>(lds);
  u32x4(*k_lds)[kStepKeys][kRowPieces] = reinterpret_cast<u32x4(*)[kStepKeys][kRowPieces]>(lds + kQBytes);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, hh = lane >> 5;

  // Workgroup b runs on XCD b % 8; each XCD takes a contiguous range of items, numbered
  // head-major, so that the keys that requests share, of one head or few, stay in its L2.
  const unsigned nb = gridDim.x, per = nb >> 3, extra = nb & 7u;
  const unsigned x = blockIdx.x & 7u, i = blockIdx.x >> 3;
  const unsigned group = x * per + min(x, extra) + i;
  const unsigned item = group * (kWavesPerGroup / W) + wave / W;  // (fewer than 2^31 of them)
  const bool in_grid = item < unsigned(a.B) * unsigned(a.Hkv) * unsigned(n_split) * unsigned(n_ct);
  // item = ((kv head * B + request) * n_ct + column tile) * n_split + range of the keys
  const unsigned all = in_grid ? item : 0u, unit = all / unsigned(n_split), pair = unit / unsigned(n_ct);
  const int sp = int(all - unit * unsigned(n_split)), ct = int(unit - pair * unsigned(n_ct));
  const int h = int(pair / unsigned(a.B)), r = int(pair % unsigned(a.B));
  const int G = a.Hq / a.Hkv;

  const int32_t* bt = a.block_tables + size_t(r) * a.max_blocks;
  auto load_ids = [&](int window) { return bt[min(window * 64 + lane, a.max_blocks - 1)]; };
  const int q0 = a.cu_q[r], q_end = a.cu_q[r + 1], q_len = q_end - q0, L_in = a.seq_lens[r];
  // The first 4096 keys' block ids come with the lengths, which say where a range begins.
  constexpr int kFirst = 5;
  int first_ids[kFirst];
#pragma unroll
  for (int i = 0; i < kFirst; ++i) first_ids[i] = load_ids(i);
  asm volatile("" : "+v"(first_ids[0]), "+v"(first_ids[1]), "+v"(first_ids[2]), "+v"(first_ids[3]), "+v"(first_ids[4]));
  const int L = min(L_in, a.max_blocks * kBlock);
  const int col0 = ct * kTileCols, n_cols = min(min(q_len, a.max_q_len) * G - col0, kTileCols);
  const bool valid = in_grid && q0 >= 0 && q_end <= a.n_rows && q_len > 0 && q_len <= L && n_cols > 0;

  f32x16 o[kDt];
#pragma unroll
  for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dt][e] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  // This lane's column (padding columns repeat the last valid one).
  const bool col_valid = valid && n < n_cols;
  const int colc = col0 + (col_valid ? n : max(n_cols, 1) - 1);
  const int t = colc / G, head = h * G + (colc - t * G);
  if (valid) {
    const uint16_t* qr = a.q + int64_t(q0 + t) * a.q_stride + size_t(head) * D;
    const uint32_t* mask_row = a.masks + size_t(q0 + t) * a.half_words;
    u32x4 qc[kDch];
#pragma unroll
    for (int kc = 0; kc < kDch; ++kc) qc[kc] = *(const u32x4*)(qr + kc * 16 + hh * 8);
    const int start = L - q_len;  // the nodes' first key
    const int n_blk = (L + kBlock - 1) / kBlock;
    const int n_steps_all = (L + kStepKeys - 1) / kStepKeys;
    const int n_ranges = n_split * W, range = sp * W + wave % W;
    const int steps_per = (n_steps_all + n_ranges - 1) / n_ranges;
    const int s_begin = min(range * steps_per, n_steps_all);
    const int n_steps = min(s_begin + steps_per, n_steps_all);
    const size_t head_off = size_t(h) * kBlock * D;
    const size_t slab = size_t(a.Hkv) * kBlock * D;

    // Block ids come 64 at a time, one a lane, a window ahead of use; a step
    // picks its two with readlane.  Ids past the request's blocks or outside the
    // pool read block 0 (those keys are masked and their V rows zeroed, or the
    // request's output is unspecified).
    const int s_first = min(s_begin, n_steps_all - 1);  // (an empty range reads a step that is there, and leaves it)
    int win = (2 * s_first) >> 6;
    int ids0 = first_ids[0], ids1 = first_ids[1];  // of the even and the odd one of windows win, win + 1
#pragma unroll
    for (int i = 1; i < kFirst - 1; ++i)
      if (win == i) (i & 1 ? ids1 : ids0) = first_ids[i], (i & 1 ? ids0 : ids1) = first_ids[i + 1];
    if (win >= kFirst - 1) {
      const int x0 = load_ids(win), x1 = load_ids(win + 1);
      ids0 = win & 1 ? x1 : x0;
      ids1 = win & 1 ? x0 : x1;
    }
    auto block_id = [&](int lb) {
      const int id = (win & 1) ? __builtin_amdgcn_readlane(ids1, lb & 63) : __builtin_amdgcn_readlane(ids0, lb & 63);
      return (lb < n_blk && id >= 0 && id < a.num_blocks) ? id : 0;
    };
    auto load = [&](int s, StepRegs<D>& R) {
      if ((2 * s) >> 6 != win) {
        if (win & 1) ids1 = load_ids(win + 2);
        else ids0 = load_ids(win + 2);
        ++win;
      }
      const int id0 = block_id(2 * s), id1 = block_id(2 * s + 1);
#pragma unroll
      for (int kc = 0; kc < kDch; ++kc)
        R.k[kc] = *(const u32x4*)(a.k_pool + size_t(kc < kDch / 2 ? id0 : id1) * slab + head_off +
                                  kc % (kDch / 2) * 512 + lane * 8);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint16_t* vs = a.v_pool + size_t(b ? id1 : id0) * slab + head_off + size_t(n) * kBlock + hh * 8;
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt) R.v[b][dt] = *(const u32x4*)(vs + dt * 32 * kBlock);
      }
      R.lo = R.hi = 0;
      if ((s + 1) * kStepKeys > start) tree_words(mask_row, a.half_words, s * kStepKeys, start, &R.lo, &R.hi);
    };

    // A block's K rows are one contiguous piece of memory and are read as such, 1 KB an
    // instruction; the operand's layout (a row a lane) comes from LDS, whose rows
    // are 16 bytes longer, so that neither the stores nor the reads meet in a bank.
    u32x4* k_st = &k_lds[wave][lane / (D / 8)][lane % (D / 8)];
    const u32x4* k_ld = &k_lds[wave][diff_key_of_row(n)][hh];

    auto compute = [&](int s, StepRegs<D>& R) {
      const int j0 = s * kStepKeys;
#pragma unroll
      for (int kc = 0; kc < kDch; ++kc) k_st[kc * (512 / D) * kRowPieces] = R.k[kc];
      wave_lds_fence();
      f32x16 sc;
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[e] = 0.f;
#pragma unroll
      for (int kc = 0; kc < kDch; ++kc)
        sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(k_ld[kc * 2]), as_bf16x8(q_lds[wave][kc][lane]), sc, 0, 0, 0);
      wave_lds_fence();
      if (j0 + kStepKeys > start) {
        // the mask, and zeroed V rows of keys that no column of the tile sees: slots
        // that hold no token may have any bits, and a weight of 0 does not hide a NaN
        const uint32_t seen = tree_window(j0, start, L, R.lo, R.hi);
        const uint32_t mine = seen >> (8 * hh);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!(mine >> ((e >> 3) * 16 + (e & 7)) & 1u)) sc[e] = -INFINITY;
        uint32_t any = seen;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) any |= __shfl_xor(any, off);
        any >>= 8 * hh;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t keep = (any >> (b * 16 + 2 * w) & 1u ? 0x0000FFFFu : 0u) |
                                  (any >> (b * 16 + 2 * w + 1) & 1u ? 0xFFFF0000u : 0u);
#pragma unroll
            for (int dt = 0; dt < kDt; ++dt) R.v[b][dt][w] &= keep;
          }
      }
      float mx = sc[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, sc[e]);
      mx = max_across_halves(mx) * a.scale_log2;
      // O and the sum are rescaled only when a column max has grown by more than 2^8
      if (__ballot(mx > m_run + kLazyRescale)) {
        const float m_new = fmaxf(m_run, mx);
        const float alpha = m_new == m_run ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[dt][e] *= alpha;
      }
      // (a column that has seen no key yet has scores and maximum -inf: exp2(-inf - 0) = 0)
      const float m_sub = m_run == -INFINITY ? 0.f : m_run;
      bf16x8 pb[2];
      float ls = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], a.scale_log2, -m_sub));
        pb[e >> 3][e & 7] = (__bf16)p;
        ls += p;
      }
      l_run += ls;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt)
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(R.v[b][dt]), pb[b], o[dt], 0, 0, 0);
    };

    // Two register sets; the scheduling barriers keep a step's loads behind the
    // computation that frees their registers.
    StepRegs<D> ra, rb;
    int s = s_begin;
    load(s_first, ra);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kc = 0; kc < kDch; ++kc) q_lds[wave][kc][lane] = qc[kc];
    for (; s + 1 < n_steps; s += 2) {
      load(s + 1, rb);
      __builtin_amdgcn_sched_barrier(0);
      compute(s, ra);
      __builtin_amdgcn_sched_barrier(0);
      if (s + 2 < n_steps) load(s + 2, ra);
      __builtin_amdgcn_sched_barrier(0);
      compute(s + 1, rb);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (s < n_steps) compute(s, ra);
  }

  const float l_tot = add_across_halves(l_run);
  // Join of the W ranges: every wave's O, max and sum to LDS (behind a barrier:
  // no wave reads Q from there any more), then a thread sums 4 dimensions of a
  // column over the waves, with weights 2^(m_k - M).
  float(*so)[kCols][kRow] = reinterpret_cast<float(*)[kCols][kRow]>(lds);
  constexpr int kPer = D / 4;  // threads to a column
  const int d = lane % kPer * 4;
  __syncthreads();
  if (col_valid) {
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4) {
        const f32x4 v = {o[dt][g4 * 4], o[dt][g4 * 4 + 1], o[dt][g4 * 4 + 2], o[dt][g4 * 4 + 3]};
        *(f32x4*)&so[wave][n][dt * 32 + g4 * 8 + hh * 4] = v;
      }
    if (hh == 0) {
      s_m[wave][n] = m_run;
      s_l[wave][n] = l_tot;
    }
  }
  __syncthreads();
  if (!valid) return;
  const int w0 = wave / W * W;  // first wave of the tile
  for (int u = (wave - w0) * 64 + lane; u < n_cols * kPer; u += W * 64) {
    const int c = u / kPer;
    float mx = s_m[w0][c];
#pragma unroll
    for (int k = 1; k < W; ++k) mx = fmaxf(mx, s_m[w0 + k][c]);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float den = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const float m = s_m[w0 + k][c];
      // (a range that saw no key of this column has weight 0)
      const float wg = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mx);
      den += wg * s_l[w0 + k][c];
      const f32x4 v = *(const f32x4*)&so[w0 + k][c][d];
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += wg * v[e];
    }
    if (n_split > 1) {
      const size_t slot = (size_t(unit) * n_split + sp) * kCols + c;
      *(f32x4*)(a.part_o + slot * D + d) = acc;
      if (d == 0) {
        a.part_ml[slot * 2] = mx;
        a.part_ml[slot * 2 + 1] = den;
      }
      continue;
    }
    const int tt = (col0 + c) / G, hd = h * G + (col0 + c - tt * G);
    const float inv = den > 0.f ? 1.f / den : 0.f;
    bf16x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (__bf16)(acc[e] * inv);
    *(bf16x4*)(a.out + (size_t(q0 + tt) * a.Hq + hd) * D + d) = v;
  }
}

// Join of the n_split states of a (request, kv head, column), a wave each: lane
// k reads split k's (max, sum), M = max m_k, w_k = 2^(m_k - M),
// O = sum w_k O_k / sum w_k l_k.  A split that saw no key has m = -inf and weight 0;
// where none saw any the sum is 0 and so is the row.  (2048 rows of 4 splits: 4.0 us, one
// round trip and a launch.)
constexpr int kJoinWaves = 4;

template <int D>
__global__ __launch_bounds__(64 * kJoinWaves) void tree_join_kernel(TreeArgs a, int n_ct, int n_split, int cols_cap) {
  constexpr int kPer = D / 64;  // dimensions of a lane
  typedef float vec_t __attribute__((ext_vector_type(kPer)));
  const int lane = threadIdx.x & 63;
  const unsigned w = __builtin_amdgcn_readfirstlane(blockIdx.x * kJoinWaves + (threadIdx.x >> 6));
  const unsigned unit = w / unsigned(cols_cap), pair = unit / unsigned(n_ct);
  const int c = int(w - unit * unsigned(cols_cap)), ct = int(unit - pair * unsigned(n_ct));
  if (pair >= unsigned(a.B) * unsigned(a.Hkv)) return;
  const int h = int(pair / unsigned(a.B)), r = int(pair % unsigned(a.B));
  const int G = a.Hq / a.Hkv, col = ct * kTileCols + c;
  const int t = col / G, head = h * G + (col - t * G);
  // Everything that the lengths do not decide is asked for with them, in one round trip:
  // the splits' maxima and sums, the first kAhead of their rows.  (Slots of columns that
  // the batch does not have hold nothing of use, and nothing comes of it.)
  const size_t slot0 = size_t(unit) * n_split * kTileCols + c;  // of split 0
  constexpr int kAhead = 8;
  const float* po = a.part_o + slot0 * D + lane * kPer;
  vec_t v[kAhead];
  auto load = [&](int k) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) v[u] = *(const vec_t*)(po + size_t(min(k + u, n_split - 1)) * kTileCols * D);
  };
  int q0 = a.cu_q[r], q_end = a.cu_q[r + 1], L_in = a.seq_lens[r];
  float2 ml = *(const float2*)(a.part_ml + (slot0 + size_t(min(lane, n_split - 1)) * kTileCols) * 2);
  load(0);
  // (pinned here: they would sink behind the test of the lengths)
  asm volatile("" : "+s"(q0), "+s"(q_end), "+s"(L_in));
  asm volatile("" : "+v"(ml.x), "+v"(ml.y));
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    if constexpr (kPer == 2) {
      asm volatile("" : "+v"(v[u]));
    } else {
      float x = v[u][0];
      asm volatile("" : "+v"(x));
      v[u][0] = x;
    }
  }
  const int q_len = q_end - q0, L = min(L_in, a.max_blocks * kBlock);
  if (q0 < 0 || q_end > a.n_rows || q_len <= 0 || q_len > L || col >= min(q_len, a.max_q_len) * G) return;
  const float m = lane < n_split ? ml.x : -INFINITY;
  float mx = m;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off));
  const float wgt = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mx);
  float den = wgt * ml.y;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) den += __shfl_xor(den, off);
  const float inv = den > 0.f ? 1.f / den : 0.f;
  vec_t y = {};
  for (int k = 0; k < n_split; k += kAhead) {
    if (k > 0) load(k);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (k + u < n_split) y += v[u] * __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wgt), k + u));
  }
  uint16_t* orow = a.out + (size_t(q0 + t) * a.Hq + head) * D + lane * kPer;
#pragma unroll
  for (int e = 0; e < kPer; ++e) orow[e] = __builtin_bit_cast(uint16_t, (__bf16)(y[e] * inv));
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// How a launch cuts its work: columns of a tile (32: the kernel above, `waves` of a workgroup to
// a tile and `groups` workgroups to its keys; kTreeTileCols: tree_tiles.hip, four waves or eight), and how
// many tiles.
struct Plan {
  int cols, waves, groups;
  int64_t n_ct, units;  // column tiles of a (request, kv head), of the batch
};

// What few tiles wait for is a wave's steps, about 1 us each one after the other: four waves to a tile,
// and more workgroups while there are compute units without one; but their states' join is
// a launch more (3 us, and more for many columns), so that tables of up to about 1.2 K
// keys are not cut, and a tile's range count goes as the root of its steps: the steps fall as 1 / ranges
// and the join's reads grow with them.  us (waves x groups; 8 kv heads, D 128 where not said):
//   tiles, keys       8, 300    4x1 8.6, 4x4 10.4             8, 1000    4x8 10.6, 4x4 11.7, 8x1 12.3
//   8, 4000           4x8 13.0, 4x16 13.3, 4x4 16.1           8, 16000   4x16 21.4, 4x24 23.9, 4x8 24.7
//   32, 500           4x1 10.2, 4x4 10.8                      32, 1500   4x6 13.1, 4x4 13.3, 4x1 15.9
//   64, 1000          4x1 13.8, 4x3 14.6                      64, 2000   4x4 16.9, 4x2 18.0, 4x1 20.5
//   64, 4096          4x4 20.3, 8x3 19.6, 4x8 21.4            128, 1000  4x1 13.8, 8x1 14.0, 4x2 16.7
//   128, 3000         8x2 22.3, 4x2 23.5, 4x1 27.5            128, 6000  8x2 30.2, 4x2 33.3, 4x1 47.7
//   256, 2000         4x1 22.9, 4x2 27.9                      D 64: 32, 1000  8x1 9.0, 4x8 9.8, 4x1 10.0
//   D 64: 128, 2500   8x1 14.5, 4x4 16.1, 4x1 18.2            D 64: 32, 3000  4x8 10.8, 8x1 14.9
// A compute unit holds two workgroups of the kernel above.  From more than two tiles of 32 to a unit on, and in
// tables of up to 320 keys from more than one (D 128), columns are taken 128 at a time on LDS tiles, where a pair has
// more than one tile of 32 (here, there):
//   280, 150    10.1, 9.8       384, 110    8.9, 7.6         400, 290    11.9, 11.8     400, 490    14.6, 14.5
//   512, 230    11.9, 10.7      512, 320    12.6, 13.2       512, 2000   32.6, 36.2     400, 2000   30.5, 34.0
//   520, 70     13.2, 8.8       520, 290    18.4, 12.1       520, 1000   29.7, 23.1     520, 4000   81.5, 59.2
//   640, 2000   67.6, 61.0      1024, 300   18.0, 14.8       2048, 2000  124, 76.5      16384, 2050 873, 584
//   D 64: 384, 110  6.2, 6.3     500, 290   8.3, 9.4         768, 110    7.4, 6.5       768, 490    12.1, 11.4
//   D 64: 520, 740  14.1, 14.8   768, 2000  26.7, 24.8       2048, 1500  51.6, 37.6     2816, 1000  50.6, 36.7
// and by two groups of waves where no compute unit has two of those (one group, two): 192 tiles of 128, 1200 keys
// 29.5, 27.1; 256, 2000 46.2, 42.2; 256, 800 23.3, 23.8; 384, 2000 62.5, 75.7; D 64: 256, 1500 26.7, 22.5.
// One tile a pair stays here: 1024 of 500 keys 48.2, 51.7, of 1000 95.4, 95.9; 2400 of 100 34.0, 39.2.  Its waves go by
// how many of its workgroups a unit gets (1, 2, 4 waves):
//   280, 150    12.4, 9.1, 9.6    280, 1000  37.3, 26.9, 31.3    512, 30    10.6, 7.9, 9.2     512, 1000  44.4, 44.6, 43.7
//   520, 300    20.0, 23.1, 21.3  520, 2000  107, 127, 112       768, 30    11.1, 10.7, 13.7   768, 1000  76.4, 78.8, 75.0
//   904, 150    19.1, 18.0, 19.5  904, 2000  165, 167, 171       1024, 500  51.2, 49.1, 48.2   2400, 100  34.0, 34.5, 38.5
//   D 64: 400, 150  8.7, 6.4, 6.8     520, 1000  28.9, 29.6, 27.5     900, 150  9.9, 9.3, 10.4
// Where a pair has more tiles, they share its keys from L2: 384 of 500 keys 23.3, 15.4, 14.0.
// Between half as many tiles as compute units and as many, no rule cuts the keys (waves x groups):
//   one tile of 32 a pair   136, 2000   4x1 24.5, 8x1 25.7, 4x2 35.0    136, 8000   4x1 101, 8x1 102, 4x2 134
//                           192, 4000   4x1 70.5, 8x1 71.5, 4x2 84.1    256, 8000   4x1 180, 8x1 179, 4x2 193
//   eight tiles a pair      192, 1000   4x1 13.3, 8x1 14.7, 4x2 20.2    192, 4000   4x1 33.5, 8x1 28.5, 4x2 33.6
//                           192, 16000  4x1 116, 8x1 88.3, 4x2 94.1     256, 8000   4x1 65.2, 8x1 55.9, 4x2 61.2
//   D 64, one tile          136, 4000   4x1 27.1, 8x1 25.1, 4x2 33.1    192, 2000   4x1 18.5, 8x1 18.8, 4x2 23.1
// so that what the rules leave there is eight waves for pairs of several tiles from 2 K keys on.  At 128 tiles, one
// a pair, the cut that several tiles gain by costs: 2000 keys 4x1 23.5, 8x2 28.6 (taken); 8000 98.7, 98.6.
// `steps` goes by the table's width, which bounds the contexts (their lengths are on the device), and the sides
// above had tables as wide as their contexts.  In wider ones short contexts get workgroups and a join that they do
// not need; us by the width in blocks: 4 requests of 72 to 80 keys, 4 heads of D 64 on one: 6 5.5, 128 8.9, 512 9.9,
// 2048 14.0; one request of 308 keys, 32 heads on 8: 21 7.6, 256 10.1, 1024 14.1, 2048 18.5; 64 of 216 to 266, 64 on
// 8: 18 25.9, 128 23.6, from 256 on 21.3.  Longer or more ones do not depend on it: one of 4160 keys 261 19.6, 2048
// 18.7; 32 of 570 to 1050 23.3 to 23.9.
Plan make_plan(int64_t B, int64_t max_q_len, int Hq, int Hkv, int D, int64_t max_blocks) {
  const int64_t cus = ilpc::device_cus(), cols = max_q_len * (Hq / Hkv), pairs = B * Hkv;
  const int64_t steps = (max_blocks * kBlock + kStepKeys - 1) / kStepKeys;
  auto cut = [&](int c) -> Plan { return {c, 4, 1, (cols + c - 1) / c, pairs * ((cols + c - 1) / c)}; };
  Plan p = cut(kTileCols);
  const int64_t u = p.units;
  if (p.n_ct > 1 && (u > 2 * cus || (D == 128 && u > cus && steps <= 10))) {
    p = cut(kTreeTileCols);
    if (p.units <= cus && steps >= 32) p.waves = 8;
    return p;
  }
  if (u > 3 * cus) {
    p.waves = 2;
  } else if (u > 2 * cus) {
    p.waves = D == 64 ? 4 : 1;
  } else if (u > cus) {
    p.waves = p.n_ct == 1 ? 2 : 4;
  } else if (2 * u <= cus) {
    const int64_t room = std::min<int64_t>(cus / u, kMaxGroups);
    if (room >= 3 && (steps >= 40 || (room >= 16 && steps >= 28)))
      p.groups = int(std::min<int64_t>(room, int64_t(std::sqrt(double(steps)))));
    else if (D == 64 ? steps >= 20 : room == 2 && steps >= 64)
      p.waves = 8, p.groups = D == 64 ? 1 : 2;
  }
  return p;
}

size_t part_bytes(const Plan& p, int D) {
  return p.groups > 1 ? size_t(p.units) * p.groups * kTileCols * (D + 2) * sizeof(float) : 0;
}

int64_t column_tiles(int64_t max_q_len, int Hq, int Hkv) {
  return (max_q_len * (Hq / Hkv) + kTileCols - 1) / kTileCols;
}

int check_sizes(const char* fn, int32_t B, int32_t max_q_len, int32_t Hq, int32_t Hkv, int32_t D, int32_t max_blocks) {
  using ilpc::set_error;
  if (B < 0 || max_q_len < 0 || max_blocks < 1 || Hq < 1 || Hkv < 1)
    return set_error(ILPC_EINVAL, "%s: negative or zero size", fn);
  if (D != 64 && D != 128) return set_error(ILPC_EUNSUP, "%s: head_dim %d unsupported", fn, D);
  if (Hq % Hkv != 0 || Hq / Hkv > 64) return set_error(ILPC_EUNSUP, "%s: Hq %d / Hkv %d unsupported", fn, Hq, Hkv);
  if (max_blocks > (1 << 24)) return set_error(ILPC_EUNSUP, "%s: max_blocks %d > %d", fn, max_blocks, 1 << 24);
  if (max_q_len > kMaxNodes) return set_error(ILPC_EUNSUP, "%s: max_q_len %d > %d", fn, max_q_len, kMaxNodes);
  if (int64_t(B) * Hkv * std::max<int64_t>(column_tiles(max_q_len, Hq, Hkv), 1) > (1 << 23))
    return set_error(ILPC_EUNSUP, "%s: batch too large", fn);
  return ILPC_OK;
}

}  // namespace

extern "C" int ilpc_tree_attn_workspace_bytes(int32_t B, int32_t max_q_len, int32_t Hq, int32_t Hkv, int32_t D,
                                              int32_t max_blocks, size_t* bytes) {
  static const char* fn = "ilpc_tree_attn_workspace_bytes";
  if (!bytes) return ilpc::set_error(ILPC_EINVAL, "%s: bytes is NULL", fn);
  const int rc = check_sizes(fn, B, max_q_len, Hq, Hkv, D, max_blocks);
  if (rc != ILPC_OK) return rc;
  *bytes = 0;
  if (B == 0 || max_q_len == 0) return ILPC_OK;
  if (ilpc::device_cus() <= 0) return ilpc::set_error(ILPC_EHIP, "%s: cannot query the device", fn);
  *bytes = part_bytes(make_plan(B, max_q_len, Hq, Hkv, D, max_blocks), D);
  return ILPC_OK;
}

extern "C" int ilpc_paged_tree_attn(const uint16_t* q, int64_t q_stride, int32_t n_rows, const uint16_t* k_pool,
                                    const uint16_t* v_pool, int32_t num_blocks, const int32_t* block_tables,
                                    int32_t max_blocks, const int32_t* cu_q, const int32_t* seq_lens, int32_t B,
                                    int32_t max_q_len, int32_t Hq, int32_t Hkv, int32_t D, int32_t block_size,
                                    float softmax_scale, const uint64_t* masks, int32_t mask_words, uint16_t* out,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  static const char* fn = "ilpc_paged_tree_attn";
  using ilpc::set_error;
  const int rc = check_sizes(fn, B, max_q_len, Hq, Hkv, D, max_blocks);
  if (rc != ILPC_OK) return rc;
  if (num_blocks < 1 || n_rows < 0) return set_error(ILPC_EINVAL, "%s: num_blocks %d, n_rows %d", fn, num_blocks, n_rows);
  if (block_size != kBlock) return set_error(ILPC_EUNSUP, "%s: block_size must be 16", fn);
  if (!(std::isfinite(softmax_scale) && softmax_scale > 0.f))
    return set_error(ILPC_EINVAL, "%s: softmax_scale must be finite and positive", fn);
  if (mask_words < 1 || int64_t(mask_words) * 64 < max_q_len || mask_words > kMaxNodes / 64)
    return set_error(ILPC_EINVAL, "%s: mask_words %d of 64 nodes for max_q_len %d", fn, mask_words, max_q_len);
  if (B == 0 || max_q_len == 0 || n_rows == 0) return ILPC_OK;
  if (!q || !k_pool || !v_pool || !block_tables || !cu_q || !seq_lens || !masks || !out)
    return set_error(ILPC_EINVAL, "%s: NULL pointer", fn);
  if (!aligned16(q) || !aligned16(k_pool) || !aligned16(v_pool) || !aligned16(out) ||
      (reinterpret_cast<uintptr_t>(masks) & 7u))
    return set_error(ILPC_EINVAL, "%s: Q/K/V/out must be 16-byte aligned, masks 8-byte", fn);
  if (q_stride < int64_t(Hq) * D || q_stride % 8 != 0)
    return set_error(ILPC_EINVAL, "%s: q_stride must be a multiple of 8 elements, at least Hq * D", fn);
  const uint16_t *q_end = q + int64_t(n_rows - 1) * q_stride + int64_t(Hq) * D, *out_end = out + int64_t(n_rows) * Hq * D;
  if (q < out_end && out < q_end) return set_error(ILPC_EINVAL, "%s: q and out overlap", fn);
  if (ilpc::device_cus() <= 0) return set_error(ILPC_EHIP, "%s: cannot query the device", fn);
  const Plan plan = make_plan(B, max_q_len, Hq, Hkv, D, max_blocks);
  const size_t need = part_bytes(plan, D);
  if (need && (!workspace || workspace_bytes < need || !aligned16(workspace)))
    return set_error(ILPC_EINVAL, "%s: workspace must be %zu bytes, 16-byte aligned", fn, need);
  float* part_o = need ? static_cast<float*>(workspace) : nullptr;
  float* part_ml = need ? part_o + size_t(plan.units) * plan.groups * kTileCols * D : nullptr;
  const TreeArgs a{q, q_stride, n_rows, k_pool, v_pool, num_blocks, block_tables, max_blocks, cu_q, seq_lens, B,
                   max_q_len, Hq, Hkv, D, softmax_scale * 1.4426950408889634f,
                   reinterpret_cast<const uint32_t*>(masks), mask_words * 2, out, part_o, part_ml};
  const int n_ct = int(plan.n_ct);
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (plan.cols > kTileCols) {
    e = launch_tree_tiles(a, plan.waves / 4, n_ct, s);
  } else {
    const int waves = group_waves(plan.waves), per_group = waves / plan.waves;
    const dim3 grid{unsigned((plan.units * plan.groups + per_group - 1) / per_group)}, block{unsigned(64 * waves)};
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a, n_ct, plan.groups); };
    if (D == 128) {
      if (plan.waves == 1) launch(tree_stream_kernel<128, 1>);
      else if (plan.waves == 2) launch(tree_stream_kernel<128, 2>);
      else if (plan.waves == 4) launch(tree_stream_kernel<128, 4>);
      else launch(tree_stream_kernel<128, 8>);
    } else {
      if (plan.waves == 2) launch(tree_stream_kernel<64, 2>);
      else if (plan.waves == 4) launch(tree_stream_kernel<64, 4>);
      else launch(tree_stream_kernel<64, 8>);
    }
    e = hipGetLastError();
  }
  if (e == hipSuccess && plan.groups > 1) {
    const int cols_cap = int(std::min<int64_t>(int64_t(max_q_len) * (Hq / Hkv), kTileCols));
    const dim3 grid{unsigned((plan.units * cols_cap + kJoinWaves - 1) / kJoinWaves)}, block{64 * kJoinWaves};
    auto join = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a, n_ct, plan.groups, cols_cap); };
    if (D == 128) join(tree_join_kernel<128>);
    else join(tree_join_kernel<64>);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return set_error(ILPC_EHIP, "%s: launch failed: %s", fn, hipGetErrorString(e));
  return ILPC_OK;
}
