// What the kernels of attention over a tree of drafted tokens share (not part of the
// ABI; the mathematics is in tree_attn.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "diff_attn.h"

namespace ilpc {

// Arguments of a launch, already checked.
struct TreeArgs {
  const uint16_t* q;
  int64_t q_stride;
  int n_rows;
  const uint16_t *k_pool, *v_pool;
  int num_blocks;
  const int32_t* block_tables;
  int max_blocks;
  const int32_t *cu_q, *seq_lens;
  int B, max_q_len, Hq, Hkv, D;
  float scale_log2;       // softmax scale * log2(e)
  const uint32_t* masks;  // [n_rows][half_words], 32 nodes a word
  int half_words;
  uint16_t* out;
  // partial states of ranges of the keys, where there are several
  float *part_o, *part_ml;
};

// The 32 keys from j0 on that a row of the tree sees, bit k for key j0 + k: of the
// context (the keys before `start`) all, of the nodes those of its mask's words lo
// and hi (tree_words), none from key_end on.
__device__ __forceinline__ uint32_t tree_window(int j0, int start, int key_end, uint32_t lo, uint32_t hi) {
  const int off = j0 - start;  // node of key j0
  uint32_t w = off >= 0 ? __builtin_amdgcn_alignbit(hi, lo, off & 31) : off > -32 ? (lo << -off) | ((1u << -off) - 1) : ~0u;
  const int left = key_end - j0;
  return left >= 32 ? w : left > 0 ? w & ((1u << left) - 1) : 0u;
}
// The two mask words that the window of key j0 needs.
__device__ __forceinline__ void tree_words(const uint32_t* row, int half_words, int j0, int start, uint32_t* lo,
                                           uint32_t* hi) {
  const int w = (j0 > start ? j0 - start : 0) >> 5;
  *lo = w < half_words ? row[w] : 0u;
  *hi = w + 1 < half_words ? row[w + 1] : 0u;
}

// The kernel for many columns (tree_tiles.hip): kTreeTileCols to a workgroup, a (request, kv
// head)'s in n_ct tiles; one or two groups of four waves share a tile's keys.
constexpr int kTreeTileCols = 128;
hipError_t launch_tree_tiles(const TreeArgs& a, int groups, int n_ct, hipStream_t stream);

}  // namespace ilpc
