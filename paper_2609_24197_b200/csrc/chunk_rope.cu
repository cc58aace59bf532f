// Norm, rotary positions on several axes and the cache write of a ragged chunk's queries, keys and values.
//
// Pair j of a head (elements j and j + rot of its first 2 rot elements) turns by pos[axis(j)][t] * theta^(-j / rot).  The rates come from the
// host in 64 bits, the product and its reduction modulo 2 pi are 64-bit as well (at position 10^6 a 32-bit product is off by 0.06), and only
// the remainder, at most pi, goes to sincosf: off by 2^-23 there, which no 16-bit result shows.
//
// Bound by memory: every value is read and written once.  A thread takes 16 elements of a head, the 8 lower and the 8 upper partners of its
// pairs, so that norm, rotation and stores need no exchange but the sum of squares over the head's threads.  A block takes several rows;
// the loads of its first heads are under way while it looks up the rows' requests, pages and angles (one per row, shared by all heads).
#include "chunk.cuh"

#include <cmath>
#include <type_traits>

namespace hspec {

namespace {

constexpr int ROPE_ROWS = 4;       // most rows of a block
constexpr int ROPE_UNROLL = 2;     // heads of a thread that are loaded together, one such load ahead of their use

struct RopeArgs {
  ChunkRopeCall c;
  double rate[64];
  uint8_t axis[64];
  int rows;                        // rows of a block
  int step_rows, step_heads;       // the groups of threads of a block, in rows and heads
  int vec;                         // qkv rows start on 16-byte boundaries
};

template <typename T> struct Raw16;                       // 16 values as they lie in memory: two groups of 8
template <> struct Raw16<float> { uint4 v[4]; };
template <> struct Raw16<__nv_bfloat16> { uint4 v[2]; };
template <> struct Raw16<__half> { uint4 v[2]; };

__device__ __forceinline__ void widen(const Raw16<float>& r, float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[4 * i] = __uint_as_float(r.v[i].x); x[4 * i + 1] = __uint_as_float(r.v[i].y);
    x[4 * i + 2] = __uint_as_float(r.v[i].z); x[4 * i + 3] = __uint_as_float(r.v[i].w);
  }
}
template <typename T>
__device__ __forceinline__ void widen(const Raw16<T>& r, float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t w[4] = {r.v[i].x, r.v[i].y, r.v[i].z, r.v[i].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (sizeof(T) == 2 && std::is_same<T, __half>::value) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
        x[8 * i + 2 * j] = f.x; x[8 * i + 2 * j + 1] = f.y;
      } else {
        x[8 * i + 2 * j] = bf16_bits_to_float(uint16_t(w[j] & 0xffffu)); x[8 * i + 2 * j + 1] = bf16_bits_to_float(uint16_t(w[j] >> 16));
      }
    }
  }
}

template <typename TI>
__device__ __forceinline__ void load16(const TI* lo, const TI* hi, bool vec, Raw16<TI>& r) {
  constexpr int W = sizeof(r.v) / 32;                     // 16-byte words of a group of 8
  if (vec) {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      r.v[i] = __ldcs(reinterpret_cast<const uint4*>(lo) + i);
      r.v[W + i] = __ldcs(reinterpret_cast<const uint4*>(hi) + i);
    }
  } else {
    TI* x = reinterpret_cast<TI*>(r.v);
    for (int i = 0; i < 8; ++i) { x[i] = lo[i]; x[8 + i] = hi[i]; }
  }
}

template <bool F16>
__device__ __forceinline__ uint4 narrow8(const float* x, uint32_t* status) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = F16 ? pack_f16_sat(x[2 * i], x[2 * i + 1], status) : pack_bf16(x[2 * i], x[2 * i + 1]);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename TI, bool F16>
__global__ void __launch_bounds__(256, 3) chunk_rope_kernel(const __grid_constant__ RopeArgs a) {
  pdl_wait();
  pdl_trigger();
  const ChunkRopeCall& c = a.c;
  __shared__ __align__(16) float s_cos[ROPE_ROWS][64], s_sin[ROPE_ROWS][64];
  __shared__ long long s_slot[ROPE_ROWS];                 // place in the pools in rows of one head; -1: none (the row's queries are still turned)
  __shared__ int s_at[ROPE_ROWS];
  __shared__ int s_used[ROPE_ROWS];                       // the row belongs to a request
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int t0 = blockIdx.x * a.rows, rows = min(a.rows, c.T - t0);
  const int lanes = c.dh >> 4, sub = threadIdx.x % lanes, group = threadIdx.x / lanes, groups = 256 / lanes;
  const int heads = c.Hq + 2 * c.Hkv, rot = c.rot_pairs;
  // this thread's 16 elements of a head: a pair group of the rotated part, or 16 elements behind it
  const bool turns = sub * 8 < rot;
  const int lo = turns ? sub * 8 : 2 * rot + (sub - rot / 8) * 16, hi = turns ? lo + rot : lo + 8;
  // This thread's heads: every groups-th of the block's, row by row.  (The place is counted along: a division for every head, twice, was a third of
  // all instructions.)
  struct Place { int r, h; };
  auto next_of = [&](Place& x) {
    x.r += a.step_rows;
    x.h += a.step_heads;
    if (x.h >= heads) { x.h -= heads; ++x.r; }
  };
  Raw16<TI> raw[ROPE_UNROLL];
  Place to_fetch{group / heads, group % heads}, at = to_fetch;
  auto fetch = [&]() {
#pragma unroll
    for (int u = 0; u < ROPE_UNROLL; ++u) {
      if (to_fetch.r < rows) {
        const TI* src = reinterpret_cast<const TI*>(c.qkv) + size_t(t0 + to_fetch.r) * c.ld_qkv + to_fetch.h * c.dh;
        load16<TI>(src + lo, src + hi, a.vec, raw[u]);
      }
      next_of(to_fetch);
    }
  };
  fetch();                                                // (under way while the rows are looked up)
  // every request once, with rows or without, by threads that no row's look-up waits for where there are any
  for (int b = int(blockIdx.x) * 256 + 255 - int(threadIdx.x); b < c.B; b += int(gridDim.x) * 256)
    if (chunk_request_bad(c.cu_q[b], c.cu_q[b + 1], c.kv_lens[b], c.T, c.max_len)) atomicAdd(c.status + STATUS_WORD_BAD_INPUT, 1u);
  for (int r = warp; r < rows; r += 8) {
    const int t = t0 + r, b = chunk_request_of(c.cu_q, c.B, t, lane);
    if (lane == 0) {
      long long slot = -1;
      int at = 0, used = 0;
      if (b < c.B) {
        const int cu0 = c.cu_q[b], cu1 = c.cu_q[b + 1], len = c.kv_lens[b];
        const ChunkRequest q = chunk_request(cu0, cu1, len, c.T, c.max_len);
        used = t >= q.q0 && t < q.q0 + q.n;               // (a cu_q that does not ascend may have counted t to a request that does not own it)
        at = q.len - q.n + (t - q.q0);
        if (used && at >= 0) {
          const int page = c.page_table[size_t(b) * c.page_table_stride + at / c.page_size];
          if (page >= 0 && page < c.num_pages) slot = ((long long)page * c.page_size + at % c.page_size) * c.Hkv;
          else atomicAdd(c.status + STATUS_WORD_BAD_INPUT, 1u);
        }
      }
      s_slot[r] = slot; s_at[r] = at; s_used[r] = used;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < rows * rot; i += 256) {
    const int r = i / rot, j = i % rot;
    const int p = c.pos ? c.pos[size_t(a.axis[j]) * c.T + t0 + r] : s_at[r];
    const double ang = double(p) * a.rate[j];
    // modulo 2 pi, which is taken as the sum of two 64-bit numbers
    const double n = rint(ang * 0.15915494309189535);
    const double rem = fma(-n, 2.4492935982947064e-16, fma(-n, 6.283185307179586, ang));
    sincosf(float(rem), &s_sin[r][j], &s_cos[r][j]);
  }
  __syncthreads();
  const int items = rows * heads;
  for (int first = 0; first < items; first += ROPE_UNROLL * groups) {
    Raw16<TI> now[ROPE_UNROLL];
#pragma unroll
    for (int u = 0; u < ROPE_UNROLL; ++u) now[u] = raw[u];
    if (first + ROPE_UNROLL * groups < items) fetch();
#pragma unroll
    for (int u = 0; u < ROPE_UNROLL; ++u) {
      const int r = at.r, h = at.h;
      const bool on = r < rows;
      next_of(at);
      float x[16];
      if (on) widen(now[u], x);
      const float* w = h < c.Hq ? c.q_norm_w : c.k_norm_w;
      if (c.q_norm_w) {                                   // (uniform: both norms or none)
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) ss += on ? x[e] * x[e] : 0.f;
        for (int off = lanes >> 1; off > 0; off >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
        if (on && h < c.Hq + c.Hkv) {
          const float inv = rsqrtf(ss / float(c.dh) + c.eps);
#pragma unroll
          for (int e = 0; e < 8; ++e) { x[e] *= inv * w[lo + e]; x[8 + e] *= inv * w[hi + e]; }
        }
      }
      if (!on || !s_used[r]) continue;
      if (turns && h < c.Hq + c.Hkv) {
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const float4 c4 = *reinterpret_cast<const float4*>(&s_cos[r][sub * 8 + v * 4]), s4 = *reinterpret_cast<const float4*>(&s_sin[r][sub * 8 + v * 4]);
          const float cs[4] = {c4.x, c4.y, c4.z, c4.w}, sn[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = x[v * 4 + e], q = x[8 + v * 4 + e];
            x[v * 4 + e] = p * cs[e] - q * sn[e];
            x[8 + v * 4 + e] = q * cs[e] + p * sn[e];
          }
        }
      }
      uint16_t* dst;
      if (h < c.Hq) {
        dst = reinterpret_cast<uint16_t*>(c.q) + (size_t(t0 + r) * c.Hq + h) * c.dh;
      } else {
        if (s_slot[r] < 0) continue;
        const bool v = h >= c.Hq + c.Hkv;
        dst = reinterpret_cast<uint16_t*>(v ? c.v_pool : c.k_pool) + (size_t(s_slot[r]) + (h - c.Hq - (v ? c.Hkv : 0))) * c.dh;
      }
      *reinterpret_cast<uint4*>(dst + lo) = narrow8<F16>(x, c.status);
      *reinterpret_cast<uint4*>(dst + hi) = narrow8<F16>(x + 8, c.status);
    }
  }
}

template <typename TI>
cudaError_t launch_for(const RopeArgs& a, int blocks, cudaStream_t stream) {
  return launch_pdl(a.c.f16 ? chunk_rope_kernel<TI, true> : chunk_rope_kernel<TI, false>, dim3(blocks), dim3(256), 0, stream, a);
}

}  // namespace

cudaError_t chunk_rope_launch(const ChunkRopeCall& c, cudaStream_t stream) {
  RopeArgs a{};
  a.c = c;
  // (64 powers cost the host 3 us: a thread keeps the last base's)
  thread_local float theta = 0.f;
  thread_local int pairs = 0;
  thread_local double rate[64];
  if (theta != c.theta || pairs != c.rot_pairs) {
    for (int j = 0; j < c.rot_pairs; ++j) rate[j] = pow(double(c.theta), -double(j) / double(c.rot_pairs));
    theta = c.theta; pairs = c.rot_pairs;
  }
  for (int j = 0; j < c.rot_pairs; ++j) {
    a.rate[j] = rate[j];
    a.axis[j] = c.pair_axis ? c.pair_axis[j] : 0;
  }
  const size_t item = c.in_dtype == CHUNK_F32 ? 4 : 2;
  a.vec = (reinterpret_cast<uintptr_t>(c.qkv) % 16 == 0 && size_t(c.ld_qkv) * item % 16 == 0) ? 1 : 0;
  // The look-up of a row (three loads that wait for one another, then its angles) takes longer than the row itself: a block has up to ROPE_ROWS of
  // them, as long as four blocks are left for every SM.  8200 rows of 80 heads, bf16, three axes, 333 MB: 61 us (5.4 TB/s); 63 with 3, 65 with 5 and
  // 82 with 16 of them, 79 without a load ahead.
  const int spread = (c.T + 4 * 148 - 1) / (4 * 148);
  a.rows = spread < ROPE_ROWS ? spread : ROPE_ROWS;
  a.step_rows = 256 / (c.dh / 16) / (c.Hq + 2 * c.Hkv);
  a.step_heads = 256 / (c.dh / 16) % (c.Hq + 2 * c.Hkv);
  const int blocks = (c.T + a.rows - 1) / a.rows;
  if (c.in_dtype == CHUNK_F32) return launch_for<float>(a, blocks, stream);
  return c.in_dtype == CHUNK_F16 ? launch_for<__half>(a, blocks, stream) : launch_for<__nv_bfloat16>(a, blocks, stream);
}

}  // namespace hspec
