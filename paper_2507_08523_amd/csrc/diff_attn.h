// What the differential attention kernels share (not part of the ABI; the
// mathematics is in diff_attn.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace ilpc {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// What the last step of every kernel needs.
struct DiffEpilogue {
  const float* lambda;  // [Hq]
  const float* norm_w;  // [D] or nullptr: no norm
  float eps, scale;
};

// Key held by MFMA row m: the groups [4,8) and [8,12) of every 16 keys trade
// places, which makes accumulator register e of lane half hh the key
// (e >> 3) * 16 + 8 * hh + (e & 7): the layout of the P^T operand.
__device__ __forceinline__ int diff_key_of_row(int m) {
  const int grp = (m >> 2) & 3;
  return m + (grp == 1 ? 4 : (grp == 2 ? -4 : 0));
}

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

__device__ __forceinline__ float max_across_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float add_across_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The i-th 16-dimension chunk of a head that belongs to a map: of its half of D, or in
// the pair layout of its half of each half of D.
template <int D>
__device__ __forceinline__ int diff_chunk_of_map(int map, int i, int pairs) {
  constexpr int kQuarter = D / 64;  // chunks of a quarter
  return pairs ? (i / kQuarter * 2 + map) * kQuarter + i % kQuarter : map * (2 * kQuarter) + i;
}

// Arguments of a launch, already checked.
struct DiffArgs {
  const uint16_t* q;
  int64_t q_stride;
  int n_rows;
  const uint16_t *k_pool, *v_pool;
  int num_blocks;
  const int32_t* block_tables;
  int max_blocks;
  const int32_t *cu_q, *seq_lens;
  int B, max_q_len, Hq, Hkv, D;
  float scale_log2;  // softmax scale * log2(e)
  int pairs;         // pair layout
  DiffEpilogue ep;
  uint16_t* out;
};

// The kernel for many columns (diff_prefill.hip); ILPC_EUNSUP: its grid does not hold the
// batch, ILPC_EHIP: no device, or the launch failed.
int launch_diff_prefill(const DiffArgs& a, hipStream_t stream);

}  // namespace ilpc
