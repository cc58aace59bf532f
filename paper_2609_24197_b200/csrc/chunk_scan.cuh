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
__device__ __forceinline__ int chunk_count(int keep, int upto) {
  const int k = min(keep, upto);
  return (k + SCAN_CHUNK - 1) / SCAN_CHUNK + (upto - k + SCAN_CHUNK - 1) / SCAN_CHUNK;
}
cudaError_t scan_long_launch(const LongArgs& a, cudaStream_t stream);
cudaError_t scan_long_wide_launch(const LongArgs& a, cudaStream_t stream);

// Whether products take their operands in three bf16 parts (what they leave is below 2^-24), not two (2^-16): for outputs that are not rounded to 16 bits.
__host__ __device__ inline bool scan_wide(const ChunkScanCall& c) { return c.y && c.y_dtype == CHUNK_F32; }
constexpr int SCAN_C_PARTS = 3;

struct ScanScratch {
  float* xbc;                        // [.., pitch] convolved rows
  float4* step;                      // [.., H] dt, and the decay exp(dt A) with what its rounding left out
  // blocks of rows (scan_block_kernel) have their C apart, split into bf16 parts, and the products C_t . B_s of a request's rows
  float4* sums;                      // [.., H] dt, e^c, and c, the sum of the log-decays so far, in two parts
  uint16_t* c_parts;                 // [.., G, SCAN_C_PARTS, N]; null: requests with few rows go through scan_state_kernel
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
  int y_vec;                         // two outputs start on their boundary
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

template <bool VEC, int N, typename TI>
__device__ __forceinline__ Word<TI, N> load_word(const TI* p) {
  Word<TI, N> w;
  if (VEC) w = *reinterpret_cast<const Word<TI, N>*>(p);
  else {
#pragma unroll
    for (int e = 0; e < N; ++e) w.v[e] = p[e];
  }
  return w;
}

// Two values at a time.
__device__ __forceinline__ uint64_t dup2(float v) { return pack_f32x2(v, v); }
__device__ __forceinline__ uint64_t silu2(uint64_t v) {
  float a, b;
  unpack_f32x2(mul_f32x2(v, dup2(-1.4426950408889634f)), a, b);
  unpack_f32x2(add_f32x2(pack_f32x2(ex2_ftz(a), ex2_ftz(b)), dup2(1.f)), a, b);
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(a));
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(b));
  return mul_f32x2(v, pack_f32x2(a, b));
}
// v = head + remainder, both bf16; packed with the first value in the low half
__device__ __forceinline__ void split2(uint64_t v, uint32_t& hi, uint32_t& lo) {
  float a, b;
  unpack_f32x2(v, a, b);
  hi = pack_bf16(a, b);
  unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(hi << 16), __uint_as_float(hi & 0xffff0000u)), dup2(-1.f), v), a, b);
  lo = pack_bf16(a, b);
}
// v in PARTS bf16 parts, each what those in front of it leave
template <int PARTS>
__device__ __forceinline__ void split_parts(uint64_t v, uint32_t (&part)[PARTS]) {
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    float a, b;
    unpack_f32x2(v, a, b);
    const uint32_t bits = part[p] = pack_bf16(a, b);
    v = fma_f32x2(pack_f32x2(__uint_as_float(bits << 16), __uint_as_float(bits & 0xffff0000u)), dup2(-1.f), v);
  }
}
template <typename TI, int N>
__device__ __forceinline__ void widen(const Word<TI, N>& w, uint64_t (&v)[N / 2]) {
#pragma unroll
  for (int i = 0; i < N / 2; ++i) v[i] = pack_f32x2(to_f32(w.v[2 * i]), to_f32(w.v[2 * i + 1]));
}

// N raw channels (from `ch` on) of a request's rows; below row zero the carried ones, or nothing.  Addresses are chosen and no loads skipped, so
// that those of several rows are under way together.
template <bool VEC, int N, typename TI>
struct RawRows {
  const TI* x;                       // the request's first row
  const TI* carried;                 // row -(d_conv - 1); null: nothing is carried
  long long ld;
  int d_xBC, K1;
  __device__ __forceinline__ RawRows(const ChunkScanCall& c, const ScanRequest& r, int ch)
      : x(reinterpret_cast<const TI*>(c.x) + size_t(r.q0) * c.ld_x + c.Di + ch),
        carried(r.fresh || c.d_conv == 1 ? nullptr : reinterpret_cast<const TI*>(c.conv_state) + size_t(r.slot) * (c.d_conv - 1) * c.d_xBC + ch),
        ld(c.ld_x), d_xBC(c.d_xBC), K1(c.d_conv - 1) {}
  // row i; behind `last` row `last` again
  __device__ __forceinline__ Word<TI, N> row(int i, int last) const { return load_word<VEC, N>(x + size_t(min(i, last)) * ld); }
  // rows i - 3 .. i - 1 (front_value: those that are not there are zero)
  __device__ __forceinline__ void front(Word<TI, N> (&w)[3], int i, int last) const {
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      const int row = i - 3 + j;
      w[j] = load_word<VEC, N>(row < 0 && there(row) ? carried + size_t(row + K1) * d_xBC : x + size_t(max(min(row, last), 0)) * ld);
    }
  }
  __device__ __forceinline__ bool there(int row) const { return row >= 0 || (carried && row + K1 >= 0); }
  __device__ __forceinline__ void front_value(const Word<TI, N> (&w)[3], int i, uint64_t (&before)[3][N / 2]) const {
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      widen(w[j], before[j]);
#pragma unroll
      for (int h = 0; h < N / 2; ++h)
        if (!there(i - 3 + j)) before[j][h] = 0ull;
    }
  }
};

// The convolution of 2 H channels.  A narrower one has the last of four taps; the rows in front of these are left out, not taken times zero: they may be
// no numbers.  K: its width, or 0: the call's.  (In the kernels of long requests the questions cost registers: those for rows on word boundaries are for K = 4.)
template <int H, int K>
struct Taps {
  uint64_t w[4][H], b[H];            // [tap][channels]
  int width;
  __device__ __forceinline__ void load(const ChunkScanCall& c, int ch) {
    const int taps = width = K ? K : c.d_conv;
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const float* f = c.conv_w + size_t(ch + 2 * h) * taps;
      b[h] = pack_f32x2(c.conv_b[ch + 2 * h], c.conv_b[ch + 2 * h + 1]);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j][h] = j >= 4 - taps ? pack_f32x2(f[j - (4 - taps)], f[j - (4 - taps) + taps]) : 0ull;
    }
  }
  // SiLU of the convolution at the row behind `before` (oldest first), which moves on by that row
  __device__ __forceinline__ void next(uint64_t (&before)[3][H], const uint64_t (&now)[H], uint64_t (&v)[H]) const {
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int taps = K ? K : width;
      uint64_t sum = b[h];
      if (taps > 3) sum = fma_f32x2(w[0][h], before[0][h], sum);
      if (taps > 2) sum = fma_f32x2(w[1][h], before[1][h], sum);
      if (taps > 1) sum = fma_f32x2(w[2][h], before[2][h], sum);
      v[h] = silu2(fma_f32x2(w[3][h], now[h], sum));
      before[0][h] = before[1][h]; before[1][h] = before[2][h]; before[2][h] = now[h];
    }
  }
};

}  // namespace hspec
