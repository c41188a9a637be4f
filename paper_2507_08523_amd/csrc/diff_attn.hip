// Differential attention over the paged cache, for gfx950: each head is the
// difference of two softmax maps over one set of values.
//
// With the halves q = [q1 | q2] and k = [k1 | k2] of a head's D dimensions,
//   A_m = softmax(s q_m k_m^T)  (causal),   y = (A_1 - lambda_h A_2) V,
//   out = out_scale * w * y / sqrt(mean(y^2) + eps)   (w: optional norm weight).
// A K row of the pool holds [k1 | k2], a V row all D values, so the pools, the
// block tables and the appends are those of ordinary attention (InferLog
// section 2.1.2: the suffix queries attend to the reused KV of the cached prefix
// and to their own).  In one pass over the keys a head keeps per map a running
// maximum m_m, a sum l_m and O_m = sum 2^(s log2(e) q_m.k_m - m_m) v; at the end
//   y = O_1 / l_1 - lambda_h O_2 / l_2.
//
// Kernel for few columns: 16 (token, head of the group) columns a wave.  The two
// maps are the two 16-column halves of the N side of one
// v_mfma_f32_32x32x16_bf16 stream: column c holds [q1 | 0], column 16 + c
// [0 | q2], so one product over all D dimensions of a K row gives both scores.
// Half of those products multiply zeros, which costs nothing here: the kernel is
// bound by reading K and V from HBM.  Each wave streams its range of a
// request's keys from the pools into registers, two pool blocks (32 keys) a
// step, the next step's loads in flight (K then takes the operand's layout by
// way of LDS); W waves of a workgroup and n_split workgroups share a (request, kv
// head, column tile) where there are too few of them to fill the chip, and their
// states are joined at the end.
//   Precision: y is a difference, and where the two maps nearly agree (the case
// the method is made for) it is much smaller than its terms, so that a weight
// rounded to bf16 (up to 2^-8 relative) would leave an error of several bf16
// roundings of y.  Each weight p therefore enters as two bf16 numbers, hi = bf16(p) and
// lo = bf16(p - hi), 16 bits in all: 8 more products a step, on matrix cores
// that wait for HBM.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/ilpc.h"
#include "diff_attn.h"
#include "ilpc_internal.h"

namespace {

using namespace ilpc;

constexpr int kBlock = 16;
constexpr int kStepKeys = 32;        // keys a step (two pool blocks)
constexpr int kTileCols = 16;        // query columns of a wave (each one twice, once a map)
constexpr int kMaxGroups = 64;       // most workgroups to a pair (a lane of the join each)
constexpr float kLazyRescale = 8.f;  // log2 growth of a column max tolerated before rescaling O

template <int D>
struct StepRegs {
  u32x4 k[D / 16];      // K rows of the step, in the order of memory
  u32x4 v[2][D / 32];   // V^T operand, [pool block of the step][32-dimension tile]
};

// Orders a wave's LDS stores and reads across its lanes (the hardware keeps a wave's
// LDS operations in order; the compiler has to as well).
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

constexpr int group_waves(int W) { return W > 4 ? W : 4; }  // waves of a workgroup, W of them to a pair

template <int D, int W>
__global__ __launch_bounds__(64 * group_waves(W), 2) void diff_stream_kernel(
    const uint16_t* __restrict__ q, int64_t q_stride, int n_rows, const uint16_t* __restrict__ k_pool,
    const uint16_t* __restrict__ v_pool, int num_blocks, const int32_t* __restrict__ block_tables, int max_blocks,
    const int32_t* __restrict__ cu_q, const int32_t* __restrict__ seq_lens, int n_req, int max_q_len, int Hq, int Hkv,
    float scale_log2, int pairs_layout, DiffEpilogue ep, uint16_t* __restrict__ out, int n_ct, int n_split,
    float* __restrict__ part_o, float* __restrict__ part_ml) {
  constexpr int kDch = D / 16, kDt = D / 32, kWavesPerGroup = group_waves(W);
  // Q^T of each wave and the K rows of its step in LDS; for the join the same space
  // holds every wave's O, a row of kRow floats a column.
  constexpr int kRow = D + 4, kCols = 2 * kTileCols;
  constexpr int kQBytes = kWavesPerGroup * kDch * 64 * 16, kOBytes = kWavesPerGroup * kCols * kRow * 4;
  constexpr int kRowPieces = D / 8 + 1;  // 16-byte pieces of a K row in LDS: one more than it has
  constexpr int kKBytes = kWavesPerGroup * kStepKeys * kRowPieces * 16;
  static_assert(kOBytes >= kQBytes + kKBytes, "the join's rows are the larger");
  __shared__ __attribute__((aligned(16))) uint8_t lds[kOBytes];
  __shared__ float s_m[kWavesPerGroup][kCols], s_l[kWavesPerGroup][kCols], s_lambda[kWavesPerGroup][kCols];
  u32x4(*q_lds)[kDch][64] = reinterpret_cast<u32x4(*)[kDch][64]>(lds);
  u32x4(*k_lds)[kStepKeys][kRowPieces] = reinterpret_cast<u32x4(*)[kStepKeys][kRowPieces]>(lds + kQBytes);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, hh = lane >> 5;
  const int map = n >> 4, nc = n & 15;  // this lane's map, and its column of the tile

  // Workgroup b runs on XCD b % 8; each XCD takes a contiguous range of items,
  // numbered head-major: requests of every length fall to each XCD, and the keys that
  // requests share, of one head or few, stay in its L2 (512 requests, 8 kv heads, 1100
  // to 2140 keys, 1024 shared: 354 us, numbered by requests 373; none shared 750, 744).
  const unsigned nb = gridDim.x, per = nb >> 3, extra = nb & 7u;
  const unsigned x = blockIdx.x & 7u, i = blockIdx.x >> 3;
  const unsigned group = x * per + min(x, extra) + i;
  const unsigned item = group * (kWavesPerGroup / W) + wave / W;  // (fewer than 2^31 of them)
  const bool in_grid = item < unsigned(n_req) * unsigned(Hkv) * unsigned(n_split) * unsigned(n_ct);
  // item = ((kv head * n_req + request) * n_ct + column tile) * n_split + range of the keys
  const unsigned all = in_grid ? item : 0u, unit = all / unsigned(n_split), pair = unit / unsigned(n_ct);
  const int sp = int(all - unit * unsigned(n_split)), ct = int(unit - pair * unsigned(n_ct));
  const int h = int(pair / unsigned(n_req)), r = int(pair % unsigned(n_req));
  const int G = Hq / Hkv;

  const int32_t* bt = block_tables + size_t(r) * max_blocks;
  auto load_ids = [&](int window) { return bt[min(window * 64 + lane, max_blocks - 1)]; };
  const int q0 = cu_q[r], q_end = cu_q[r + 1], q_len = q_end - q0, L_in = seq_lens[r];
  // The first 4096 keys' block ids come with the lengths, which say where a range begins.
  constexpr int kFirst = 5;
  int first_ids[kFirst];
#pragma unroll
  for (int i = 0; i < kFirst; ++i) first_ids[i] = load_ids(i);
  asm volatile("" : "+v"(first_ids[0]), "+v"(first_ids[1]), "+v"(first_ids[2]), "+v"(first_ids[3]), "+v"(first_ids[4]));
  const int L = min(L_in, max_blocks * kBlock);
  const int col0 = ct * kTileCols, n_cols = min(min(q_len, max_q_len) * G - col0, kTileCols);
  const bool valid = in_grid && q0 >= 0 && q_end <= n_rows && q_len > 0 && q_len <= L && n_cols > 0;

  f32x16 o[kDt];
#pragma unroll
  for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dt][e] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  // This lane's column (padding columns repeat the last valid one).
  const bool col_valid = valid && nc < n_cols;
  const int colc = col0 + (col_valid ? nc : max(n_cols, 1) - 1);
  const int t = colc / G, head = h * G + (colc - t * G);
  float lambda = 0.f;
  if (valid) {
    lambda = ep.lambda[head];
    const int pos = L - q_len + t;  // keys 0 .. pos are visible to this column
    // (all loads of Q at once: a load under the test of each chunk's map is a round trip each)
    const uint16_t* qr = q + int64_t(q0 + t) * q_stride + size_t(head) * D;
    u32x4 qc[kDch / 2];
#pragma unroll
    for (int i = 0; i < kDch / 2; ++i)
      qc[i] = *(const u32x4*)(qr + diff_chunk_of_map<D>(map, i, pairs_layout) * 16 + hh * 8);
    const int n_blk = (L + kBlock - 1) / kBlock;
    // keys past the last column's position are not visited (and their V rows zeroed)
    const int key_end = L - q_len + (col0 + n_cols - 1) / G + 1;
    const int n_steps_all = (key_end + kStepKeys - 1) / kStepKeys;
    const int n_ranges = n_split * W, range = sp * W + wave % W;
    const int steps_per = (n_steps_all + n_ranges - 1) / n_ranges;
    const int s_begin = min(range * steps_per, n_steps_all);
    const int n_steps = min(s_begin + steps_per, n_steps_all);
    const size_t head_off = size_t(h) * kBlock * D;
    const size_t slab = size_t(Hkv) * kBlock * D;

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
      const int a = load_ids(win), b = load_ids(win + 1);
      ids0 = win & 1 ? b : a;
      ids1 = win & 1 ? a : b;
    }
    auto block_id = [&](int lb) {
      const int id = (win & 1) ? __builtin_amdgcn_readlane(ids1, lb & 63) : __builtin_amdgcn_readlane(ids0, lb & 63);
      return (lb < n_blk && id >= 0 && id < num_blocks) ? id : 0;
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
        R.k[kc] = *(const u32x4*)(k_pool + size_t(kc < kDch / 2 ? id0 : id1) * slab + head_off + kc % (kDch / 2) * 512 +
                                  lane * 8);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint16_t* vs = v_pool + size_t(b ? id1 : id0) * slab + head_off + size_t(n) * kBlock + hh * 8;
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt) R.v[b][dt] = *(const u32x4*)(vs + dt * 32 * kBlock);
      }
    };

    const int mask_from = L - q_len + col0 / G;  // steps reaching past this key need the causal mask

    // A block's K rows are one contiguous piece of memory and are read as such, 1 KB an
    // instruction; the operand's layout (a row a lane) comes from LDS, whose rows
    // are 16 bytes longer, so that neither the stores nor the reads meet in a bank.
    // Reading rows straight into the operand, 32 bytes of 32 rows an instruction, keeps
    // the address path busy: 128 requests of 8 kv heads with 812 keys, 512 of them
    // shared, 48.3 us and 37.6 this way; without shared keys HBM hides most of it.
    u32x4* k_st = &k_lds[wave][lane / (D / 8)][lane % (D / 8)];
    const u32x4* k_ld = &k_lds[wave][diff_key_of_row(n)][hh];

    auto compute = [&](int s, StepRegs<D>& R) {
      const int j0 = s * kStepKeys;
#pragma unroll
      for (int kc = 0; kc < kDch; ++kc) k_st[kc * (512 / D) * kRowPieces] = R.k[kc];
      wave_lds_fence();
      // (one chain of products: a second one's sums cost the register that a third wave of a
      // SIMD has at D = 64, and there is none left at D = 128)
      f32x16 sc;
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[e] = 0.f;
#pragma unroll
      for (int kc = 0; kc < kDch; ++kc)
        sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(k_ld[kc * 2]), as_bf16x8(q_lds[wave][kc][lane]), sc, 0, 0, 0);
      wave_lds_fence();
      if (j0 + kStepKeys - 1 > mask_from) {
        // causal mask (which also covers keys >= L), and the V rows of keys >=
        // key_end zeroed: unwritten pool slots may hold any bits
        const int rel = pos - j0 - hh * 8;
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if ((e >> 3) * 16 + (e & 7) > rel) sc[e] = -INFINITY;
        const int lim = key_end - j0 - hh * 8;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const int k0 = b * 16 + 2 * w;
              R.v[b][dt][w] &= (k0 < lim ? 0x0000FFFFu : 0u) | (k0 + 1 < lim ? 0xFFFF0000u : 0u);
            }
      }
      float mx = sc[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, sc[e]);
      mx = max_across_halves(mx) * scale_log2;
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
      // (a column that has seen no key yet, in a range that starts past key 0,
      // has scores and maximum -inf: exp2(-inf - 0) = 0)
      const float m_sub = m_run == -INFINITY ? 0.f : m_run;
      bf16x8 ph[2], pl[2];
      float ls = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], scale_log2, -m_sub));
        const __bf16 hi = (__bf16)p;
        ph[e >> 3][e & 7] = hi;
        pl[e >> 3][e & 7] = (__bf16)(p - (float)hi);
        ls += p;
      }
      l_run += ls;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt)
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(R.v[b][dt]), ph[b], o[dt], 0, 0, 0);
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt)
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(R.v[b][dt]), pl[b], o[dt], 0, 0, 0);
    };

    // Two register sets; the scheduling barriers keep a step's loads behind the
    // computation that frees their registers.
    StepRegs<D> ra, rb;
    int s = s_begin;
    load(s_first, ra);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kDch / 2; ++i) {
      q_lds[wave][diff_chunk_of_map<D>(map, i, pairs_layout)][lane] = qc[i];
      q_lds[wave][diff_chunk_of_map<D>(1 - map, i, pairs_layout)][lane] = u32x4{0, 0, 0, 0};
    }
    asm volatile("" : "+v"(lambda));  // (asked for with Q, and not at the end)
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
  // column over the waves, both maps, with weights 2^(m_k - M).
  float(*so)[kCols][kRow] = reinterpret_cast<float(*)[kCols][kRow]>(lds);
  constexpr int kPer = D / 4;  // threads to a column
  const int d = lane % kPer * 4;
  f32x4 nw = {1.f, 1.f, 1.f, 1.f};
  if (ep.norm_w && n_split == 1) nw = *(const f32x4*)(ep.norm_w + d);
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
      s_lambda[wave][n] = lambda;
    }
  }
  asm volatile("" : "+v"(nw));  // (on its way since before the barrier)
  __syncthreads();
  if (!valid) return;
  const int w0 = wave / W * W;     // first wave of the pair
  for (int u = (wave - w0) * 64 + lane; u < n_cols * kPer; u += W * 64) {
    const int c = u / kPer;
    f32x4 acc[2];
    float mx[2], den[2];
#pragma unroll
    for (int mp = 0; mp < 2; ++mp) {
      const int vc = mp * kTileCols + c;
      mx[mp] = s_m[w0][vc];
#pragma unroll
      for (int k = 1; k < W; ++k) mx[mp] = fmaxf(mx[mp], s_m[w0 + k][vc]);
      acc[mp] = f32x4{0.f, 0.f, 0.f, 0.f};
      den[mp] = 0.f;
#pragma unroll
      for (int k = 0; k < W; ++k) {
        const float m = s_m[w0 + k][vc];
        // (a range that saw no key of this column has weight 0)
        const float wg = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mx[mp]);
        den[mp] += wg * s_l[w0 + k][vc];
        const f32x4 v = *(const f32x4*)&so[w0 + k][vc][d];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[mp][e] += wg * v[e];
      }
      if (n_split > 1) {
        const size_t slot = (size_t(unit) * n_split + sp) * kCols + vc;
        *(f32x4*)(part_o + slot * D + d) = acc[mp];
        if (d == 0) {
          part_ml[slot * 2] = mx[mp];
          part_ml[slot * 2 + 1] = den[mp];
        }
      }
    }
    if (n_split > 1) continue;
    const int tt = (col0 + c) / G, hd = h * G + (col0 + c - tt * G);
    const float w1 = 1.f / den[0], w2 = s_lambda[w0][c] / den[1];
    f32x4 y;
    float sq = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      y[e] = acc[0][e] * w1 - acc[1][e] * w2;
      sq += y[e] * y[e];
    }
    f32x4 f = {ep.scale, ep.scale, ep.scale, ep.scale};
    if (ep.norm_w) {
#pragma unroll
      for (int off = 1; off < kPer; off <<= 1) sq += __shfl_xor(sq, off);
      const float inv = rsqrtf(sq * (1.f / D) + ep.eps);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] *= inv * nw[e];
    }
    bf16x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (__bf16)(y[e] * f[e]);
    *(bf16x4*)(out + (size_t(q0 + tt) * Hq + hd) * D + d) = v;
  }
}

// Join of the n_split states of a (request, kv head, column), a wave each: lane
// k reads split k's (max, sum) of each map, M = max m_k, w_k = 2^(m_k - M),
// O = sum w_k O_k / sum w_k l_k.  Split 0 holds key 0, which every column sees,
// so M is finite; a split that saw none has m = -inf and weight 0.
constexpr int kJoinWaves = 4;

template <int D>
__global__ __launch_bounds__(64 * kJoinWaves) void diff_join_kernel(
    const float* __restrict__ part_o, const float* __restrict__ part_ml, const int32_t* __restrict__ cu_q,
    const int32_t* __restrict__ seq_lens, int n_rows, int max_blocks, int n_req, int max_q_len, int Hq, int Hkv,
    int n_ct, int n_split, int cols_cap, DiffEpilogue ep, uint16_t* __restrict__ out) {
  constexpr int kPer = D / 64;  // dimensions of a lane
  typedef float vec_t __attribute__((ext_vector_type(kPer)));
  const int lane = threadIdx.x & 63;
  const unsigned w = __builtin_amdgcn_readfirstlane(blockIdx.x * kJoinWaves + (threadIdx.x >> 6));
  const unsigned unit = w / unsigned(cols_cap), pair = unit / unsigned(n_ct);
  const int c = int(w - unit * unsigned(cols_cap)), ct = int(unit - pair * unsigned(n_ct));
  if (pair >= unsigned(n_req) * unsigned(Hkv)) return;
  const int h = int(pair / unsigned(n_req)), r = int(pair % unsigned(n_req));
  const int G = Hq / Hkv, col = ct * kTileCols + c;
  const int t = col / G, head = h * G + (col - t * G);

  // Everything that the lengths do not decide is asked for with them, in one round trip:
  // the splits' maxima and sums, the first kAhead of their rows.  (Slots of columns that
  // the batch does not have hold nothing of use, and nothing comes of it.)
  const size_t slot0 = size_t(unit) * n_split * (2 * kTileCols) + c;  // of split 0
  constexpr size_t kNext = 2 * kTileCols;                              // from one split to the next
  constexpr int kAhead = 8;
  const float* po = part_o + slot0 * D + lane * kPer;
  vec_t v[kAhead][2];
  auto load = [&](int k) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int mp = 0; mp < 2; ++mp)
        v[u][mp] = *(const vec_t*)(po + (size_t(min(k + u, n_split - 1)) * kNext + mp * kTileCols) * D);
  };
  int q0 = cu_q[r], q_end = cu_q[r + 1], L_in = seq_lens[r];
  float lam = ep.lambda[head];
  float2 ml[2];
#pragma unroll
  for (int mp = 0; mp < 2; ++mp)
    ml[mp] = *(const float2*)(part_ml + (slot0 + mp * kTileCols + size_t(min(lane, n_split - 1)) * kNext) * 2);
  load(0);
  // (pinned here: they would sink behind the test of the lengths)
  asm volatile("" : "+s"(q0), "+s"(q_end), "+s"(L_in), "+s"(lam));
  asm volatile("" : "+v"(ml[0].x), "+v"(ml[0].y), "+v"(ml[1].x), "+v"(ml[1].y));
#pragma unroll
  for (int u = 0; u < kAhead; ++u)
#pragma unroll
    for (int mp = 0; mp < 2; ++mp) {
      if constexpr (kPer == 2) {
        asm volatile("" : "+v"(v[u][mp]));
      } else {
        float x = v[u][mp][0];
        asm volatile("" : "+v"(x));
        v[u][mp][0] = x;
      }
    }
  const int q_len = q_end - q0, L = min(L_in, max_blocks * kBlock);
  if (q0 < 0 || q_end > n_rows || q_len <= 0 || q_len > L || col >= min(q_len, max_q_len) * G) return;

  float wgt[2], den[2];
#pragma unroll
  for (int mp = 0; mp < 2; ++mp) {
    const float m = lane < n_split ? ml[mp].x : -INFINITY;
    float mx = m;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off));
    wgt[mp] = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mx);
    den[mp] = wgt[mp] * ml[mp].y;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) den[mp] += __shfl_xor(den[mp], off);
  }
  const float f1 = 1.f / den[0], f2 = -lam / den[1];
  vec_t y = {};
  for (int k = 0; k < n_split; k += kAhead) {
    if (k > 0) load(k);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (k + u < n_split)
        y += v[u][0] * (f1 * __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wgt[0]), k + u))) +
             v[u][1] * (f2 * __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wgt[1]), k + u)));
  }
  float fac = ep.scale;
  if (ep.norm_w) {
    float sq = 0.f;
#pragma unroll
    for (int e = 0; e < kPer; ++e) sq += y[e] * y[e];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sq += __shfl_xor(sq, off);
    fac *= rsqrtf(sq * (1.f / D) + ep.eps);
  }
  uint16_t* orow = out + (size_t(q0 + t) * Hq + head) * D + lane * kPer;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const float f = ep.norm_w ? fac * ep.norm_w[lane * kPer + e] : fac;
    orow[e] = __builtin_bit_cast(uint16_t, (__bf16)(y[e] * f));
  }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Waves of a workgroup, and workgroups, to a (request, kv head, column tile).
struct Plan {
  int waves, groups;
};

int64_t column_tiles(int64_t max_q_len, int Hq, int Hkv) {
  return (max_q_len * (Hq / Hkv) + kTileCols - 1) / kTileCols;
}

// How a launch cuts its units (column tiles of the (request, kv head) pairs).  What a
// launch waits for is the compute unit with most to do, and a wave's steps follow each
// other at about 1 us: four waves to a unit, and several workgroups (whose states a
// second launch joins, 2 us), while every workgroup has a CU to itself; else two;
// and four again, quarters of the load, where twos leave some CUs twice the work of
// others.  One wave to a unit is better than two only for a few steps of very many units,
// all starts.  8 kv heads, D 128, us:
//   units, keys       waves x workgroups
//   8, 600            4x1 9.4, 4x5 8.6       8, 1000     4x1 12.2, 4x4 9.8, 4x8 8.7
//   8, 4000           4x6 13.3, 4x11 12.0 (taken), 4x16 11.1
//   32, 500           4x1 8.7, 4x4 9.3
//   32, 800           4x4 10.5, 4x7 9.6      32, 2100    4x4 14.1, 4x8 12.3
//   64, 800           4x1 11.6, 4x4 10.9     64, 2100    4x1 22.8, 4x4 18.5
//   96, 2100          4x1 23.2, 4x2 23.0     96, 4000    4x1 37.8, 4x2 34.1
//   128, 2100         4x1 24.7, 4x2 27.9     128, 8000   4x1 96.3, 4x2 91.5
//   264, 1000         2x1 24.4, 4x1 29.4
//   576, 1000         2x1 56.6, 4x1 47.8; of 300 21.3 (taken), 20.3
//   1024, 1000        2x1 88.6, 4x1 87.8 (60% of the keys shared by all 39.0, 41.8)
//   1248, 1000        2x1 111, 4x1 107       4096, 2100  2x1 684, 4x1 682 (324, 350)
// D 64, whose steps and join are shorter: 512 of 2100 2x1 41.4, 4x1 41.8 (shared 31.4,
// 28.1); 1024 of 1000 39.9, 39.1 (25.1, 28.4); 128 of 2100 4x1 18.2, 8x1 15.9; 256 of 2100
// 23.5, 24.6; 16 of 600 4x1 7.4, 4x6 7.9, of 1000 4x1 9.6, 8x1 9.0, 4x4 8.5, 4x8 8.0.
// Short contexts, 1x1 and 2x1: 2048 units of 32 keys 11.4, 15.3, of 96 22.4, 24.0, 4096 22.0,
// 28.1 and 39.4, 40.5, 1536 9.8, 11.5 and 19.1, 20.8, 1024 9.7, 8.6; D 64, 2048 of 96 13.7,
// 15.1, 1536 11.9, 10.3.
// A workgroup's steps go as 1 / workgroups and the join's reads as their number, so the
// best number goes as the root of the steps: 16, 32, 64 workgroups to 1 unit of 8000 keys
// 15.7, 17.0, -; of 16000 19.6, 18.7, 22.8; of 32000 26.7, 22.7, 25.0; of 128000 72.8, 46.7,
// 39.0.
// A pair's tiles find each other's keys in L2, and four waves are better up to two units to
// a CU: 320 units of 2600 keys, 2 tiles a pair 2x1 52.4, 4x1 43.2, 8 tiles 50.5, 38.6; 512
// of 1300 32.8, 34.6 and 31.8, 28.9; but 576 of 600 24.9, 26.1.
Plan stream_plan(int64_t units, int64_t n_ct, int64_t max_blocks, int D) {
  const int64_t cus = ilpc::device_cus(), steps = (max_blocks * kBlock + kStepKeys - 1) / kStepKeys;
  const bool four = units <= cus || (D == 64 && units <= 3 * cus) || (n_ct > 1 && units <= 2 * cus) ||
                    (steps >= 32 && ((units > 2 * cus && units <= 3 * cus) || (units > 4 * cus && units <= 5 * cus)));
  if (!four) return {steps <= 4 && units > (D == 64 ? 7 : 5) * cus ? 1 : 2, 1};
  const int64_t room = std::min<int64_t>(cus / units, kMaxGroups);
  const int64_t ones = (steps + 3) / 4;  // workgroups that leave a wave one step
  if (steps >= (D == 64 ? 24 : 17) && ones <= std::min<int64_t>(room, 10)) return {4, int(ones)};
  if (room >= 3 && steps >= (room >= 4 ? 24 : D == 64 ? 40 : 32))
    return {4, int(std::min({room, (steps + 7) / 8, int64_t(std::sqrt(double(steps)))}))};
  if (room == 2 && (steps > 128 || (D == 128 && steps >= 64 && 5 * units <= 2 * cus))) return {4, 2};
  return {D == 64 && 2 * units <= cus && steps >= 32 ? 8 : 4, 1};
}

// Whether the kernel for many columns takes a batch: of more than one column tile a
// pair, where there are more than four units to a CU (at D = 64, whose exponentials it
// takes twice as well, eleven).  us here, there: D 128, contexts of 2100 keys, 768 units 60,
// 88; 1056 85, 88; 1280 91, 89; 2176 160, 120; of 600 keys, 768 25, 31; 1056 36, 31; 2176 56,
// 43; of 100, 768 11, 12; 1056 17, 12.  D 64, 2100 keys, 1056 units 52, 74; 1792 76, 74; 2560
// 95, 103; 3584 129, 106; of 600, 1056 21, 25; 1792 28, 26; 2560 36, 36; 3584 46, 37; of 100,
// 1056 11, 11; 2176 13, 12.
// (Its grid holds 2^22 columns a request and 2^18 pairs.)
bool many_columns(int64_t B, int64_t max_q_len, int Hq, int Hkv, int D) {
  const int64_t n_ct = column_tiles(max_q_len, Hq, Hkv);
  if (max_q_len * (Hq / Hkv) > (1 << 22) || B * Hkv > (1 << 18)) return false;
  return n_ct > 1 && B * Hkv * n_ct > (D == 64 ? 11 : 4) * int64_t(ilpc::device_cus());
}

// Workgroups of a launch.
int64_t stream_grid(int64_t units, const Plan& plan) {
  const int64_t per_group = group_waves(plan.waves) / plan.waves;
  return (units * plan.groups + per_group - 1) / per_group;
}

size_t part_bytes(int64_t units, int D, int n) {
  return n > 1 ? size_t(units) * n * (2 * kTileCols) * (D + 2) * sizeof(float) : 0;
}

int check_sizes(const char* fn, int32_t B, int32_t max_q_len, int32_t Hq, int32_t Hkv, int32_t D, int32_t max_blocks) {
  using ilpc::set_error;
  if (B < 0 || max_q_len < 0 || max_blocks < 1 || Hq < 1 || Hkv < 1)
    return set_error(ILPC_EINVAL, "%s: negative or zero size", fn);
  if (D != 64 && D != 128) return set_error(ILPC_EUNSUP, "%s: head_dim %d unsupported", fn, D);
  if (Hq % Hkv != 0 || Hq / Hkv > 64) return set_error(ILPC_EUNSUP, "%s: Hq %d / Hkv %d unsupported", fn, Hq, Hkv);
  if (max_blocks > (1 << 24)) return set_error(ILPC_EUNSUP, "%s: max_blocks %d > %d", fn, max_blocks, 1 << 24);
  if (int64_t(B) * Hkv > INT32_MAX / 16 || int64_t(max_q_len) * (Hq / Hkv) > (1 << 30))
    return set_error(ILPC_EUNSUP, "%s: batch too large", fn);
  // The kernel for few columns: fewer than 2^32 threads (and 2^31 items).  So many units
  // are one or two waves each whatever the device.
  const int64_t n_ct = column_tiles(max_q_len, Hq, Hkv), units = int64_t(B) * Hkv * n_ct;
  if (units > (1 << 24) && !many_columns(B, max_q_len, Hq, Hkv, D) &&
      stream_grid(units, stream_plan(units, n_ct, max_blocks, D)) * (64 * 4) > UINT32_MAX)
    return set_error(ILPC_EUNSUP, "%s: batch too large", fn);
  return ILPC_OK;
}

}  // namespace

extern "C" int ilpc_diff_attn_workspace_bytes(int32_t B, int32_t max_q_len, int32_t Hq, int32_t Hkv, int32_t D,
                                              int32_t max_blocks, size_t* bytes) {
  static const char* fn = "ilpc_diff_attn_workspace_bytes";
  if (!bytes) return ilpc::set_error(ILPC_EINVAL, "%s: bytes is NULL", fn);
  const int rc = check_sizes(fn, B, max_q_len, Hq, Hkv, D, max_blocks);
  if (rc != ILPC_OK) return rc;
  *bytes = 0;
  if (B == 0 || max_q_len == 0) return ILPC_OK;
  if (ilpc::device_cus() <= 0) return ilpc::set_error(ILPC_EHIP, "%s: cannot query the device", fn);
  if (many_columns(B, max_q_len, Hq, Hkv, D)) return ILPC_OK;
  const int64_t units = int64_t(B) * Hkv * column_tiles(max_q_len, Hq, Hkv);
  *bytes = part_bytes(units, D, stream_plan(units, column_tiles(max_q_len, Hq, Hkv), max_blocks, D).groups);
  return ILPC_OK;
}

extern "C" int ilpc_paged_diff_attn(const uint16_t* q, int64_t q_stride, int32_t n_rows, const uint16_t* k_pool,
                                    const uint16_t* v_pool, int32_t num_blocks, const int32_t* block_tables,
                                    int32_t max_blocks, const int32_t* cu_q, const int32_t* seq_lens, int32_t B,
                                    int32_t max_q_len, int32_t Hq, int32_t Hkv, int32_t D, int32_t block_size,
                                    float softmax_scale, int32_t layout, const float* lambda,
                                    const float* norm_weight, float norm_eps, float out_scale, uint16_t* out,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  static const char* fn = "ilpc_paged_diff_attn";
  using ilpc::set_error;
  const int rc = check_sizes(fn, B, max_q_len, Hq, Hkv, D, max_blocks);
  if (rc != ILPC_OK) return rc;
  if (num_blocks < 1 || n_rows < 0) return set_error(ILPC_EINVAL, "%s: num_blocks %d, n_rows %d", fn, num_blocks, n_rows);
  if (block_size != kBlock) return set_error(ILPC_EUNSUP, "%s: block_size must be 16", fn);
  if (layout != ILPC_DIFF_HALVES && layout != ILPC_DIFF_ROPE)
    return set_error(ILPC_EINVAL, "%s: layout %d", fn, layout);
  if (!(std::isfinite(softmax_scale) && softmax_scale > 0.f) || !std::isfinite(out_scale))
    return set_error(ILPC_EINVAL, "%s: scales must be finite, and softmax_scale positive", fn);
  if (norm_weight && !(std::isfinite(norm_eps) && norm_eps >= 0.f))
    return set_error(ILPC_EINVAL, "%s: norm_eps must be finite and not negative", fn);
  if (B == 0 || max_q_len == 0 || n_rows == 0) return ILPC_OK;
  if (!q || !k_pool || !v_pool || !block_tables || !cu_q || !seq_lens || !lambda || !out)
    return set_error(ILPC_EINVAL, "%s: NULL pointer", fn);
  if (!aligned16(q) || !aligned16(k_pool) || !aligned16(v_pool) || !aligned16(out) || !aligned16(norm_weight))
    return set_error(ILPC_EINVAL, "%s: Q/K/V/out/norm_weight must be 16-byte aligned", fn);
  if (q_stride < int64_t(Hq) * D || q_stride % 8 != 0)
    return set_error(ILPC_EINVAL, "%s: q_stride must be a multiple of 8 elements, at least Hq * D", fn);
  const uint16_t *q_end = q + int64_t(n_rows - 1) * q_stride + int64_t(Hq) * D, *out_end = out + int64_t(n_rows) * Hq * D;
  if (q < out_end && out < q_end) return set_error(ILPC_EINVAL, "%s: q and out overlap", fn);
  if (many_columns(B, max_q_len, Hq, Hkv, D)) {
    const DiffArgs a{q, q_stride, n_rows, k_pool, v_pool, num_blocks, block_tables, max_blocks, cu_q, seq_lens, B,
                     max_q_len, Hq, Hkv, D, softmax_scale * 1.4426950408889634f, int(layout == ILPC_DIFF_ROPE),
                     DiffEpilogue{lambda, norm_weight, norm_eps, out_scale}, out};
    const int rc = launch_diff_prefill(a, static_cast<hipStream_t>(stream));
    if (rc == ILPC_EUNSUP) return set_error(rc, "%s: batch too large", fn);
    if (rc != ILPC_OK) return set_error(rc, "%s: no device, or the launch failed", fn);
    return ILPC_OK;
  }
  if (ilpc::device_cus() <= 0) return set_error(ILPC_EHIP, "%s: cannot query the device", fn);
  const int64_t n_ct = column_tiles(max_q_len, Hq, Hkv), units = int64_t(B) * Hkv * n_ct;
  const Plan plan = stream_plan(units, n_ct, max_blocks, D);
  const size_t need = part_bytes(units, D, plan.groups);
  if (need && (!workspace || workspace_bytes < need || !aligned16(workspace)))
    return set_error(ILPC_EINVAL, "%s: workspace must be %zu bytes, 16-byte aligned", fn, need);
  const DiffEpilogue ep{lambda, norm_weight, norm_eps, out_scale};
  float* part_o = need ? static_cast<float*>(workspace) : nullptr;
  float* part_ml = need ? part_o + size_t(units) * plan.groups * (2 * kTileCols) * D : nullptr;
  const dim3 grid{unsigned(stream_grid(units, plan))}, block{unsigned(64 * group_waves(plan.waves))};
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, block, 0, s, q, q_stride, n_rows, k_pool, v_pool, num_blocks, block_tables, max_blocks,
                       cu_q, seq_lens, B, max_q_len, Hq, Hkv, softmax_scale * 1.4426950408889634f,
                       int(layout == ILPC_DIFF_ROPE), ep, out, int(n_ct), plan.groups, part_o, part_ml);
  };
  if (D == 128) {
    if (plan.waves == 1) launch(diff_stream_kernel<128, 1>);
    else if (plan.waves == 2) launch(diff_stream_kernel<128, 2>);
    else launch(diff_stream_kernel<128, 4>);
  } else {
    if (plan.waves == 1) launch(diff_stream_kernel<64, 1>);
    else if (plan.waves == 2) launch(diff_stream_kernel<64, 2>);
    else if (plan.waves == 4) launch(diff_stream_kernel<64, 4>);
    else launch(diff_stream_kernel<64, 8>);
  }
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && plan.groups > 1) {
    const int cols_cap = int(std::min<int64_t>(int64_t(max_q_len) * (Hq / Hkv), kTileCols));
    const dim3 jgrid{unsigned((units * cols_cap + kJoinWaves - 1) / kJoinWaves)}, jblock{64 * kJoinWaves};
    auto join = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, jgrid, jblock, 0, s, part_o, part_ml, cu_q, seq_lens, n_rows, max_blocks, B, max_q_len,
                         Hq, Hkv, int(n_ct), plan.groups, cols_cap, ep, out);
    };
    if (D == 128) join(diff_join_kernel<128>);
    else join(diff_join_kernel<64>);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return set_error(ILPC_EHIP, "%s: launch failed: %s", fn, hipGetErrorString(e));
  return ILPC_OK;
}
