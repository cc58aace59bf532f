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

__device__ __forceinline__ uint32_t pack_f16_sat(float lo, float hi, uint32_t* status) {
  const __half2 h = __halves2half2(f16_sat(lo, status), f16_sat(hi, status));
  return *reinterpret_cast<const uint32_t*>(&h);
}

}  // namespace hspec
