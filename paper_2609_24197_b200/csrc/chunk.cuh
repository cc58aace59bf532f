// A ragged chunk of new tokens over a paged cache, as the kernels of the target's side see it: request b owns rows cu_q[b] .. cu_q[b + 1] - 1 of
// the chunk; its cache holds kv_lens[b] tokens, the chunk's own among them, so row i of its n rows stands at position kv_lens[b] - n + i.
#pragma once
#include "common.cuh"
#include "kernels.h"

namespace hspec {

struct ChunkRequest {
  int q0, n;      // first row, rows
  int len;        // cached tokens
};

// The arrays' values, held inside what the host knows: rows inside the chunk, lengths inside the page-table row.  Every kernel sees the same.
__device__ __forceinline__ ChunkRequest chunk_request(int cu0, int cu1, int len, int T, int max_len) {
  ChunkRequest r;
  r.q0 = min(max(cu0, 0), T);
  r.n = min(max(cu1, r.q0), T) - r.q0;
  r.len = min(max(len, 0), max_len);
  return r;
}
__device__ __forceinline__ bool chunk_request_bad(int cu0, int cu1, int len, int T, int max_len) {
  return cu0 < 0 || cu1 < cu0 || cu1 > T || len < 0 || len > max_len || cu1 - cu0 > len;
}

// The number of requests that end at or before row t: the request of the row, or B behind the last one.  One warp; needs cu_q[1 .. B] to ascend.
__device__ __forceinline__ int chunk_request_of(const int32_t* cu_q, int B, int t, int lane) {
  int n = 0;
  for (int base = 0; base < B; base += 32) {
    const bool before = base + lane < B && cu_q[base + lane + 1] <= t;
    n += __popc(__ballot_sync(0xffffffffu, before));
  }
  return n;
}

// Item `item` of a chunk whose requests are cut into items of `rows` rows: its request (-1: behind the last item), that request's first row and number of rows,
// and the item's first row among them.  rows_of(b): {first row, rows} of request b; one without rows has `least` items, one with -1 none.  There are at most
// T / rows + B items (T / rows + min(B, T) with least = 0).  One warp.
struct ChunkItem { int b, q0, n, first; };
struct ChunkRows { int q0, n; };
template <typename F>
__device__ __forceinline__ ChunkItem chunk_item(int B, int rows, int least, int item, int lane, F rows_of) {
  int before = 0;
  for (int base = 0; base < B; base += 32) {
    ChunkRows r{0, 0};
    if (base + lane < B) r = rows_of(base + lane);
    const int items = base + lane < B ? (r.n > 0 ? (r.n + rows - 1) / rows : r.n < 0 ? 0 : least) : 0;
    int upto = items;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, upto, off);
      if (lane >= off) upto += up;
    }
    const uint32_t mine = __ballot_sync(0xffffffffu, before + upto > item);
    if (mine) {
      const int l = __ffs(mine) - 1;
      return {base + l, __shfl_sync(0xffffffffu, r.q0, l), __shfl_sync(0xffffffffu, r.n, l),
              (item - before - __shfl_sync(0xffffffffu, upto - items, l)) * rows};
    }
    before += __shfl_sync(0xffffffffu, upto, 31);
  }
  return {-1, 0, 0, 0};
}

__device__ __forceinline__ uint32_t pack_f16_sat(float lo, float hi, uint32_t* status) {
  const __half2 h = __halves2half2(f16_sat(lo, status), f16_sat(hi, status));
  return *reinterpret_cast<const uint32_t*>(&h);
}

}  // namespace hspec
