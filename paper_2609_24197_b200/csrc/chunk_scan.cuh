// What the kernels of a ragged chunk's scan share: a request's part in it, and the row types.
#pragma once
#include "chunk.cuh"

namespace hspec {

struct ScanRequest {
  int q0, n;       // first row, rows
  int keep;        // rows whose state is stored
  int slot;        // the state's place, or -1: none
  bool fresh;      // starts from zeros
  __device__ __forceinline__ bool stores() const { return slot >= 0 && (keep > 0 || fresh); }
};
__device__ __forceinline__ ScanRequest scan_request(const ChunkScanCall& c, int b) {
  const ChunkRequest q = chunk_request(c.cu_q[b], c.cu_q[b + 1], 0, c.T, 0);
  ScanRequest r{q.q0, q.n, q.n, c.slots ? c.slots[b] : b, c.fresh && c.fresh[b] != 0};
  if (c.keep) r.keep = int(min(max((long long)(c.keep[b]) + c.keep_more, 0ll), (long long)(q.n)));
  if (r.slot < 0 || r.slot >= c.num_slots) { r.slot = -1; r.fresh = true; }
  return r;
}

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32(float v) { return v; }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

template <typename T, int N> struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Word { T v[N]; };

__device__ __forceinline__ void store_row(void* y, int dtype, size_t at, float v, uint32_t* status) {
  if (dtype == CHUNK_F32) reinterpret_cast<float*>(y)[at] = v;
  else store_act16(y, at, v, dtype == CHUNK_BF16, status);
}

// ln(1 + e^v) without a loss at either end
__device__ __forceinline__ float softplus_f32(float v) { return v > 20.f ? v : log1pf(expf(v)); }
__device__ __forceinline__ float silu_f32(float v) { return v / (1.f + __expf(-v)); }

__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

}  // namespace hspec
