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

// rows that have to be gone through: all of them for outputs, the kept ones for the states alone
__device__ __forceinline__ int scan_upto(const ChunkScanCall& c, const ScanRequest& r) { return c.y ? r.n : r.keep; }

// Requests with more than SCAN_FEW such rows go through the tensor cores in chunks of SCAN_CHUNK rows (chunk_scan_tc.cu), where the shape allows it.
constexpr int SCAN_FEW = 32, SCAN_CHUNK = 128, SCAN_IMAGE_BYTES = 131072 + 40960;
struct LongArgs {
  ChunkScanCall c;
  const int32_t* plan;               // [0] requests with many rows, [1] their chunks
  const int32_t* list;               // [.., 2] request and its first chunk, longest requests first
  const int32_t* chunks;             // [.., 2] request and the chunk's index in it
  uint8_t* images;
  int y_vec, z_vec;                  // rows of y, and of x, start on 32-byte boundaries
};
inline long long scan_max_long(long long T, int B) { return T / (SCAN_FEW + 1) < B ? T / (SCAN_FEW + 1) : B; }
// (a request's chunks end where its kept rows do: up to two of them are not full)
inline long long scan_max_chunks(long long T, int B) { return T / SCAN_CHUNK + 2 * scan_max_long(T, B); }
cudaError_t scan_long_launch(const LongArgs& a, cudaStream_t stream);

struct ScanScratch {
  float* xbc;                        // [.., pitch] convolved rows
  float2* step;                      // [.., H] dt and the decay exp(dt A)
  // blocks of rows (scan_block_kernel) have their C apart, split into two bf16 parts, and the products C_t . B_s of a request's rows
  uint16_t* c_parts;                 // [.., G, 2, N]; null: requests with few rows go through scan_state_kernel
  float* cb;                         // [B, G, SCAN_FEW, SCAN_FEW]
  int pitch;
  int few;                           // requests with more rows than this go another way
  int apart;                         // 0: row t of the chunk lies at t; else row i of request b at b * apart + i
  __device__ __forceinline__ size_t row(int b, int q0, int i) const { return apart ? size_t(b) * apart + i : size_t(q0) + i; }
};

struct StateArgs {
  ChunkScanCall c;
  ScanScratch s;
  int p_blocks, p_block;             // blocks of a head, rows of its state in each
  int np;                            // padded N: row pitch of B and C in shared memory
  int y_vec;                         // four outputs start on their boundary
};
cudaError_t scan_block_launch(const StateArgs& a, cudaStream_t stream);

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
