// What the decodes share: sums over the lanes of a row, and the lists' splits over workgroups with the workspace they take.
#pragma once
#include <hip/hip_bf16.h>
#include <hip/hip_runtime.h>

#include <algorithm>

#include "dam_internal.h"

namespace dam {

constexpr int kXcd = 8;

#ifdef __HIPCC__
// Sum over the LPR adjacent lanes that share a row (LPR = 4, 8, 16 or 32), on the DPP network.
template <int CTRL>
__device__ __forceinline__ float dpp_move(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false));
}

template <int LPR>
__device__ __forceinline__ float row_sum(float d) {
  d += dpp_move<0xB1>(d);   // quad_perm [1,0,3,2]
  d += dpp_move<0x4E>(d);   // quad_perm [2,3,0,1]
  if (LPR >= 8) d += dpp_move<0x141>(d);   // row_half_mirror: the other quad of the 8
  if (LPR >= 16) d += dpp_move<0x140>(d);  // row_mirror: the other half of the 16
  if (LPR >= 32) d += __shfl_xor(d, 16);
  return d;
}

// A listed key outside the cache is pulled to its nearest row: the result is then wrong, but no
// address leaves the head's rows. Applied where the row address is formed, not where the index is
// fetched: there it would make the pass wait for the index load (and, the counter being in order,
// for the rows in flight before it).
__device__ __forceinline__ int in_cache(int row, int cap) { return min(max(row, 0), cap - 1); }

__device__ __forceinline__ void store_out(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_out(__hip_bfloat16 *p, float v) { *p = __float2bfloat16(v); }
#endif

inline int pick_splits(int64_t items, int64_t max_kept) {
  // Enough workgroups to put two on every CU (512), each with at least 256 keys; one split (and nothing
  // to merge) when the batch alone provides them.
  int64_t s = (512 + items - 1) / items;
  s = std::min<int64_t>(s, std::max<int64_t>(1, max_kept / 256));
  return (int)std::min<int64_t>(std::max<int64_t>(s, 1), 64);
}

// Workspace of a call whose lists are split over `splits` workgroups: partial O, (reference, sum), flags.
struct Partials {
  float *o, *ml;
  uint64_t *flags;
  size_t bytes, flag_bytes;
  Partials(void *ws, const dam_decode_params *p, int splits, int64_t lists) {
    Carver c(ws);
    o = c.take<float>((size_t)p->batch * p->hq * splits * p->head_dim);
    ml = c.take<float>((size_t)p->batch * p->hq * splits * 2);
    const size_t before = c.off;
    flags = splits > 1 ? c.take<uint64_t>((size_t)lists * splits) : nullptr;
    bytes = c.off;
    flag_bytes = c.off - before;
  }
};

// The workspace queries' answer: a workspace for a batch takes any smaller one too, which is split further and may need
// more (a batch that sequences leave). Beyond kSplitBatch sequences no list is split, and the need grows with the batch.
constexpr int kSplitBatch = 1024;
template <typename F>
size_t bytes_up_to_batch(const dam_decode_params *p, F partials) {
  size_t most = partials(p).bytes;
  dam_decode_params fewer = *p;
  for (fewer.batch = std::min(p->batch, kSplitBatch); fewer.batch >= 1; --fewer.batch)
    most = std::max(most, partials(&fewer).bytes);
  return most;
}

}  // namespace dam
