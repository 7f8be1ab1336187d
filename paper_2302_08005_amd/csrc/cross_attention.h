// What the cross attention kernels of both files share.
#pragma once
#include "common.h"
#include "kernels.h"

namespace slapo {

// Rows of one (sample, key head): of q, out and their gradients, and of lse and delta. Query heads that share a key head are one array of
// rows for it, token after token and head after head, so the gradients of a key head add up over its query heads inside a block.
struct CrossRows {
  int group, q_len;
  uint32_t mul, shift;
  __device__ __forceinline__ CrossRows(const CrossShape& s) : group(s.group), q_len(s.q_len), mul(s.div_mul), shift(s.div_shift) {}
  __device__ __forceinline__ int count() const { return q_len * group; }
  __device__ __forceinline__ int token(int r) const { return (int)((__umulhi((uint32_t)r, mul) + (uint32_t)r) >> shift); }
  // elements from the sample's first token and the group's first head
  __device__ __forceinline__ int64_t at(int r, int64_t stride, int width) const {
    const int t = token(r);
    return t * stride + (int64_t)(r - t * group) * width;
  }
  __device__ __forceinline__ int64_t stat(int r) const {   // in [group][q_len]
    const int t = token(r);
    return (int64_t)(r - t * group) * q_len + t;
  }
};

__device__ __forceinline__ int visible(const CrossShape& s, const int32_t* lens, int b) {
  if (!lens) return s.kv_len;
  const int n = lens[b];
  return n < 0 ? 0 : n < s.kv_len ? n : s.kv_len;
}

// 16-bit types (cross_tiles.hip)
size_t cross_tiles_fwd_ws_bytes(int head_dim, const CrossShape& s);
size_t cross_tiles_bwd_ws_bytes(int head_dim, const CrossShape& s);
void launch_cross_tiles_fwd(bool f16, int head_dim, const CrossShape& s, const CrossOperands& p, hipStream_t st);
void launch_cross_tiles_bwd(bool f16, int head_dim, const CrossShape& s, const CrossOperands& p, hipStream_t st);

}  // namespace slapo
