// The scan of requests with up to 32 rows (heads of 64 channels with 128 state elements: the serving shapes): single tokens and drafted blocks.
//
// With c_t the running sum of the rows' log-decays and S the state in front of them,
//   y_t = e^{c_t} (S C_t)  +  sum_{s <= t} e^{c_t - c_s} dt_s (C_t . B_s) x_s  +  D x_t,      S' = e^{c_m} S + sum_{s < m} (e^{c_m - c_s} dt_s x_s) B_s^T
// for m kept rows.  Bound by the state, which is read once and, where rows are kept, written once: a block has a head's state in registers, 16 channels
// a warp, from its first instruction on.  S C for all rows and what the rows give one another are products of 16 x 8 x 16 on the warp's tensor fragments
// (32 channels x rows are too few for the other tensor path): S comes from memory in the order of a fragment, four elements of its 128 a thread and step,
// and C in the same one.  Operands are split into a bf16 head and a bf16 remainder, three products for one (a relative error of about 2^-18 a term).
// The kept rows are added to the state in 32 bits.  (Row after row through the state, 17 rows of 32 requests take 182 us: three operations an element and row.)
#include "chunk_scan.cuh"

#include <atomic>
#include <climits>

namespace hspec {

namespace {

constexpr int NH = 64, NS = 128, FEW = SCAN_FEW;
constexpr int X_PITCH = NH + 4, W_PITCH = FEW + 4, C_PITCH = NS + 16;            // of rows in shared memory, in their own elements
struct BlockShared {
  float x[FEW][X_PITCH];
  float w[FEW][W_PITCH];                     // e^{c_t - c_s} dt_s (C_t . B_s), with D on the diagonal
  union {
    uint16_t c[2][FEW][C_PITCH];             // C's head and remainder
    float y[FEW][X_PITCH];                   // later the outputs, before the gate
  };
  float b[FEW][NS];
  double sum[FEW];                           // c_t
  float dt[FEW], ec[FEW], kept[FEW];         // dt, e^{c_t}, e^{c_m - c_s} dt_s
};

__device__ __forceinline__ void split_pair(float a, float b, uint32_t& hi, uint32_t& lo) {
  hi = pack_bf16(a, b);
  lo = pack_bf16(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xffff0000u));
}

template <typename TI, bool Y, bool VEC>
__global__ void __launch_bounds__(128, 4) scan_block_kernel(StateArgs a) {
  const ChunkScanCall& c = a.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gl = lane >> 2, q = lane & 3;
  const int h = blockIdx.x, b = blockIdx.y, g = h / (c.H / c.G);
  // (before the wait only what is at least two kernels back is read: the arrays that describe the chunk, and the states)
  const ScanRequest r = scan_request(c, b);
  const int n = scan_upto(c, r);
  if (n > a.s.few || (n == 0 && !r.stores())) { pdl_wait(); return; }
  // rows 16 warp + gl and + 8 of the state, of each elements 16 k + 4 q .. + 3
  float4 S[2][8];
  float* state = c.ssm_state + ((size_t(r.slot < 0 ? 0 : r.slot) * c.H + h) * NH + warp * 16 + gl) * NS + q * 4;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) S[i][k] = r.fresh ? make_float4(0.f, 0.f, 0.f, 0.f) : __ldcs(reinterpret_cast<const float4*>(state + i * 8 * NS + k * 16));
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) uint8_t block_sm[];
  BlockShared& s = *reinterpret_cast<BlockShared*>(block_sm);
  const size_t at0 = a.s.row(b, r.q0, 0);
  if (n > 0) {
    // ---- the rows: x, B, C; their steps
    for (int i = tid; i < n * (NH / 4); i += 128) {
      const int row = i >> 4, e = (i & 15) * 4;
      cp_async16(smem_u32(&s.x[row][e]), a.s.xbc + (at0 + row) * a.s.pitch + h * NH + e, true);
    }
    if (Y)
      for (int i = tid; i < n * 32; i += 128) {
        const int row = i >> 5, part = (i >> 4) & 1, e = (i & 15) * 8;
        cp_async16(smem_u32(&s.c[part][row][e]), a.s.c_parts + ((at0 + row) * c.G + g) * 2 * NS + part * NS + e, true);
      }
    if (r.keep > 0)
      for (int i = tid; i < r.keep * (NS / 4); i += 128) {
        const int row = i >> 5, e = (i & 31) * 4;
        cp_async16(smem_u32(&s.b[row][e]), a.s.xbc + (at0 + row) * a.s.pitch + c.Di + g * NS + e, true);
      }
    cp_async_commit();
    if (tid < 32) {
      const float dt = tid < n ? a.s.step[(at0 + tid) * c.H + h].x : 0.f;
      double sum = double(dt) * double(-expf(c.A_log[h]));
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const double up = __shfl_up_sync(0xffffffffu, sum, off);
        if (tid >= off) sum += up;
      }
      const double end = r.keep > 0 ? __shfl_sync(0xffffffffu, sum, max(r.keep - 1, 0)) : 0.0;
      s.sum[tid] = sum;
      s.dt[tid] = dt;
      s.ec[tid] = __expf(float(sum));
      s.kept[tid] = tid < r.keep ? dt * __expf(float(end - sum)) : 0.f;
    }
  }
  Word<TI, 4> z[FEW * NH / 4 / 128];
  const TI* gates = reinterpret_cast<const TI*>(c.x) + size_t(r.q0) * c.ld_x + h * NH;
  if (Y) {
#pragma unroll
    for (int i = 0; i < FEW * NH / 4 / 128; ++i) {
      const int row = (tid + i * 128) >> 4, e = (tid & 15) * 4;
      if (row >= n) continue;
      if (VEC) z[i] = *reinterpret_cast<const Word<TI, 4>*>(gates + size_t(row) * c.ld_x + e);
      else {
#pragma unroll
        for (int j = 0; j < 4; ++j) z[i].v[j] = gates[size_t(row) * c.ld_x + e + j];
      }
    }
  }
  __syncthreads();
  if (Y && n > 0) {
    const float D = c.Dskip[h];
    const int padded = (n + 15) / 16 * 16;                   // (what lies behind the last row is read as zeros, never as what happens to be there)
    for (int i = tid; i < padded * padded; i += 128) {
      const int t = i / padded, u = i % padded;
      float w = 0.f;
      if (u <= t && t < n) {
        w = a.s.cb[((size_t(b) * c.G + g) * FEW + t) * FEW + u] * s.dt[u] * __expf(float(s.sum[t] - s.sum[u]));
        if (u == t) w += D;
      }
      s.w[t][u] = w;
    }
    for (int i = tid; i < (padded - n) * NH; i += 128) s.x[n + i / NH][i % NH] = 0.f;
    for (int i = tid; i < (padded - n) * NS; i += 128) s.c[0][n + i / NS][i % NS] = s.c[1][n + i / NS][i % NS] = 0;
  }
  cp_async_wait<0>();
  bool odd = false;                                          // x is not finite (a thread looks at what it has copied)
  if (Y)
    for (int i = tid; i < n * (NH / 4); i += 128) {
      const float4 v = *reinterpret_cast<const float4*>(&s.x[i >> 4][(i & 15) * 4]);
      odd |= fmaf(v.x, 0.f, fmaf(v.y, 0.f, fmaf(v.z, 0.f, v.w * 0.f))) != 0.f;
    }
  odd = __syncthreads_or(odd);
  if (Y && n > 0) {
    float acc[4][4] = {};
    // ---- with the state
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      uint32_t hi[4], lo[4];
      split_pair(S[0][k].x, S[0][k].y, hi[0], lo[0]);
      split_pair(S[1][k].x, S[1][k].y, hi[1], lo[1]);
      split_pair(S[0][k].z, S[0][k].w, hi[2], lo[2]);
      split_pair(S[1][k].z, S[1][k].w, hi[3], lo[3]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (j * 8 >= n) break;
        const uint2 ch = *reinterpret_cast<const uint2*>(&s.c[0][j * 8 + gl][k * 16 + q * 4]), cl = *reinterpret_cast<const uint2*>(&s.c[1][j * 8 + gl][k * 16 + q * 4]);
        mma_bf16_16816(acc[j], hi, ch.x, ch.y);
        mma_bf16_16816(acc[j], hi, cl.x, cl.y);
        mma_bf16_16816(acc[j], lo, ch.x, ch.y);
      }
    }
    // (a lane has channels gl and gl + 8 of its warp's, of rows 8 j + 2 q and + 1)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j * 8 >= n) break;
      const float e0 = s.ec[j * 8 + 2 * q], e1 = s.ec[j * 8 + 2 * q + 1];
      acc[j][0] *= e0; acc[j][1] *= e1; acc[j][2] *= e0; acc[j][3] *= e1;
    }
    // ---- among the rows
    if (odd) {
      // (in a product a value that is not finite would reach the rows in front of it too, as zero times itself)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = j * 8 + 2 * q + (i & 1);
#pragma unroll 1
          for (int u = 0; u <= t && t < n; ++u) acc[j][i] = fmaf(s.w[t][u], s.x[u][warp * 16 + gl + (i >> 1) * 8], acc[j][i]);
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (odd || k * 16 >= n) break;
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {                          // channel gl (+ 8), rows 16 k + 2 q (+ 8) and the one behind it
        const int p = warp * 16 + gl + (i & 1) * 8, u = k * 16 + 2 * q + (i >> 1) * 8;
        split_pair(s.x[u][p], s.x[u + 1][p], hi[i], lo[i]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (j * 8 >= n) break;
        if (j * 8 + 7 < k * 16) continue;                    // (rows in front of the terms: nothing)
        const float2 w0 = *reinterpret_cast<const float2*>(&s.w[j * 8 + gl][k * 16 + 2 * q]), w1 = *reinterpret_cast<const float2*>(&s.w[j * 8 + gl][k * 16 + 2 * q + 8]);
        uint32_t wh[2], wl[2];
        split_pair(w0.x, w0.y, wh[0], wl[0]);
        split_pair(w1.x, w1.y, wh[1], wl[1]);
        mma_bf16_16816(acc[j], hi, wh[0], wh[1]);
        mma_bf16_16816(acc[j], hi, wl[0], wl[1]);
        mma_bf16_16816(acc[j], lo, wh[0], wh[1]);
      }
    }
    __syncthreads();                                         // (C has been read: the outputs take its place)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j * 8 >= n) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) s.y[j * 8 + 2 * q + (i & 1)][warp * 16 + gl + (i >> 1) * 8] = acc[j][i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < FEW * NH / 4 / 128; ++i) {
      const int row = (tid + i * 128) >> 4, e = (tid & 15) * 4;
      if (row >= n) continue;
      const float4 y = *reinterpret_cast<const float4*>(&s.y[row][e]);
      const float v[4] = {y.x * silu_f(to_f32(z[i].v[0])), y.y * silu_f(to_f32(z[i].v[1])), y.z * silu_f(to_f32(z[i].v[2])), y.w * silu_f(to_f32(z[i].v[3]))};
      const size_t to = (size_t(r.q0) + row) * c.ld_y + h * NH + e;
      if (!a.y_vec) {
#pragma unroll
        for (int j = 0; j < 4; ++j) store_row(c.y, c.y_dtype, to + j, v[j], c.status);
      } else if (c.y_dtype == CHUNK_F32) {
        *reinterpret_cast<float4*>(reinterpret_cast<float*>(c.y) + to) = make_float4(v[0], v[1], v[2], v[3]);
      } else {
        *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(c.y) + to) =
            c.y_dtype == CHUNK_BF16 ? make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])) : make_uint2(pack_f16_sat(v[0], v[1], c.status), pack_f16_sat(v[2], v[3], c.status));
      }
    }
  }
  if (!r.stores()) return;
  // ---- the state behind the kept rows
  if (r.keep > 0) {
    const float end = s.ec[r.keep - 1];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) S[i][k] = make_float4(S[i][k].x * end, S[i][k].y * end, S[i][k].z * end, S[i][k].w * end);
#pragma unroll 1
    for (int u = 0; u < r.keep; ++u) {
      const float kept = s.kept[u], x0 = kept * s.x[u][warp * 16 + gl], x1 = kept * s.x[u][warp * 16 + gl + 8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float4 v = *reinterpret_cast<const float4*>(&s.b[u][k * 16 + q * 4]);
        S[0][k].x = fmaf(x0, v.x, S[0][k].x); S[0][k].y = fmaf(x0, v.y, S[0][k].y); S[0][k].z = fmaf(x0, v.z, S[0][k].z); S[0][k].w = fmaf(x0, v.w, S[0][k].w);
        S[1][k].x = fmaf(x1, v.x, S[1][k].x); S[1][k].y = fmaf(x1, v.y, S[1][k].y); S[1][k].z = fmaf(x1, v.z, S[1][k].z); S[1][k].w = fmaf(x1, v.w, S[1][k].w);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) __stcs(reinterpret_cast<float4*>(state + i * 8 * NS + k * 16), S[i][k]);
}

template <typename TI, bool Y, bool VEC>
cudaError_t launch_vec(const StateArgs& a, cudaStream_t stream) {
  static std::atomic<uint32_t> ready{0};                     // devices on which the kernel has been told its shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev >= 32 || !(ready.load() >> dev & 1u)))
    e = cudaFuncSetAttribute(scan_block_kernel<TI, Y, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(sizeof(BlockShared)));
  if (e != cudaSuccess) return e;
  if (dev < 32) ready.fetch_or(1u << dev);
  return launch_pdl(scan_block_kernel<TI, Y, VEC>, dim3(unsigned(a.c.H), unsigned(a.c.B)), dim3(128), sizeof(BlockShared), stream, a);
}

template <typename TI>
cudaError_t launch_for(StateArgs a, cudaStream_t stream) {
  const ChunkScanCall& c = a.c;
  const int item = c.y_dtype == CHUNK_F32 ? 4 : 2;
  a.y_vec = c.y && reinterpret_cast<uintptr_t>(c.y) % (4 * item) == 0 && c.ld_y % 4 == 0 ? 1 : 0;
  if (!c.y) return launch_vec<TI, false, true>(a, stream);
  const bool vec = c.ld_x % 4 == 0 && reinterpret_cast<uintptr_t>(c.x) % (4 * sizeof(TI)) == 0;
  return vec ? launch_vec<TI, true, true>(a, stream) : launch_vec<TI, true, false>(a, stream);
}

}  // namespace

cudaError_t scan_block_launch(const StateArgs& a, cudaStream_t stream) {
  if (a.c.in_dtype == CHUNK_F32) return launch_for<float>(a, stream);
  return a.c.in_dtype == CHUNK_F16 ? launch_for<__half>(a, stream) : launch_for<__nv_bfloat16>(a, stream);
}

}  // namespace hspec
