// The scan of requests with up to 32 rows (heads of 64 channels with 128 state elements: the serving shapes): single tokens and drafted blocks.
//
// With c_t the running sum of the rows' log-decays and S the state in front of them,
//   y_t = e^{c_t} (S C_t)  +  sum_{s <= t} e^{c_t - c_s} dt_s (C_t . B_s) x_s  +  D x_t,      S' = e^{c_m} S + sum_{s < m} (e^{c_m - c_s} dt_s x_s) B_s^T
// for m kept rows.  Bound by the state, which is read once and, where rows are kept, written once: a block has a head's state in registers, 16 channels
// a warp, from its first instruction on.  S C for all rows and what the rows give one another are products of 16 x 8 x 16 on the warp's tensor fragments
// (32 channels x rows are too few for the other tensor path): S comes from memory in the order of a fragment, four elements of its 128 a thread and step,
// and C in the same one.  Operands are split into a bf16 head and a bf16 remainder, three products for one (a
// relative error of some 2^-18 a term, 3 x 2^-16 at most, where outputs are rounded to 16 bits), or into three parts and six products for 32-bit outputs.
// The kept rows are added to the state in 32 bits.  (Row after row through the state, 17 rows of 32 requests of 128 heads take 182 us, three operations an element
// and row; so they take 80, 2 TB/s: 13 to 18 for the kernel in front, 70 here for 150 MB of states and rows with 2 x 10^9 multiply-adds of the fragments.)
#include "chunk_scan.cuh"

#include <atomic>
#include <climits>

namespace hspec {

namespace {

constexpr int NH = 64, NS = 128, FEW = SCAN_FEW;
constexpr int X_PITCH = NH + 4, W_PITCH = FEW + 4, C_PITCH = NS + 16;            // of rows in shared memory, in their own elements
template <int PARTS>
struct BlockShared {
  float x[FEW][X_PITCH];
  float cb[FEW][W_PITCH];                    // C_t . B_s, up to the diagonal
  uint16_t c[PARTS][FEW][C_PITCH];           // C in bf16 parts
  float b[FEW][NS];
  float4 sums[FEW];                          // dt_t, e^{c_t}, c_t in two parts
};

// a and b in PARTS bf16 parts, each what those in front of it leave
template <int PARTS>
__device__ __forceinline__ void split_pair(float a, float b, uint32_t (&part)[PARTS][4], int i) {
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    const uint32_t v = part[p][i] = pack_bf16(a, b);
    a -= __uint_as_float(v << 16);
    b -= __uint_as_float(v & 0xffff0000u);
  }
}
// The products of two operands' parts down to those of the size of what the last part leaves.  The tensor cores cut the bits that do not fit their sums: of three
// parts the smallest products come first, and what a step gives is added outside, so that a sum is cut once a step and not six times (outputs off by 1.1e-6
// that way).
template <int PARTS>
__device__ __forceinline__ void mma_parts(float (&acc)[4], const uint32_t (&a)[PARTS][4], const uint2 (&b)[PARTS]) {
  if constexpr (PARTS == 2) {
    mma_bf16_16816(acc, a[0], b[0].x, b[0].y);
    mma_bf16_16816(acc, a[0], b[1].x, b[1].y);
    mma_bf16_16816(acc, a[1], b[0].x, b[0].y);
  } else {
    float step[4] = {};
#pragma unroll
    for (int size = PARTS - 1; size >= 0; --size)
#pragma unroll
      for (int i = 0; i <= size; ++i) mma_bf16_16816(step, a[i], b[size - i].x, b[size - i].y);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] += step[i];
  }
}

template <typename TI, int PARTS, bool Y, bool VEC>
__global__ void __launch_bounds__(128, PARTS == 2 ? 4 : 3) scan_block_kernel(StateArgs a) {
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
  BlockShared<PARTS>& s = *reinterpret_cast<BlockShared<PARTS>*>(block_sm);
  const size_t at0 = a.s.row(b, r.q0, 0);
  // ---- the rows: steps, x, C, B and their products
  if (tid < n) cp_async16(smem_u32(&s.sums[tid]), a.s.sums + (at0 + tid) * c.H + h, true);
  for (int i = tid; i < n * (NH / 4); i += 128) cp_async16(smem_u32(&s.x[i >> 4][(i & 15) * 4]), a.s.xbc + (at0 + (i >> 4)) * a.s.pitch + h * NH + (i & 15) * 4, true);
  for (int i = tid; i < r.keep * (NS / 4); i += 128)
    cp_async16(smem_u32(&s.b[i >> 5][(i & 31) * 4]), a.s.xbc + (at0 + (i >> 5)) * a.s.pitch + c.Di + g * NS + (i & 31) * 4, true);
  if (Y) {
    for (int i = tid; i < n * 16; i += 128) {
      const int row = i >> 4, e = (i & 15) * 8;
#pragma unroll
      for (int p = 0; p < PARTS; ++p) cp_async16(smem_u32(&s.c[p][row][e]), a.s.c_parts + (((at0 + row) * c.G + g) * SCAN_C_PARTS + p) * NS + e, true);
    }
    for (int i = tid; i < n * (FEW / 4); i += 128)
      if ((i & 7) * 4 <= i >> 3) cp_async16(smem_u32(&s.cb[i >> 3][(i & 7) * 4]), a.s.cb + ((size_t(b) * c.G + g) * FEW + (i >> 3)) * FEW + (i & 7) * 4, true);
  }
  cp_async_commit();
  // (what lies behind the last row is read as zeros, never as what happens to be there)
  const int padded = (n + 15) / 16 * 16;
  for (int i = tid; i < (padded - n) * NH; i += 128) s.x[n + i / NH][i % NH] = 0.f;
  for (int i = tid; i < padded - n; i += 128) s.sums[n + i] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (Y)
    for (int i = tid; i < (padded - n) * (NS / 8); i += 128)
#pragma unroll
      for (int p = 0; p < PARTS; ++p) *reinterpret_cast<uint4*>(&s.c[p][n + i / (NS / 8)][i % (NS / 8) * 8]) = make_uint4(0, 0, 0, 0);
  // A lane has channels p and p + 8 of rows 8 j + 2 q and + 1; after a swap with the lane four on (or back) two adjacent channels of one of the rows.
  const int odd_lane = gl & 1, out_row = 2 * q + odd_lane, out_ch = warp * 16 + (gl & ~1);
  const TI* gates = reinterpret_cast<const TI*>(c.x) + size_t(r.q0) * c.ld_x + h * NH + out_ch;
  Word<TI, 2> z[4][2];
  if (Y) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j * 8 + out_row < n) {
        z[j][0] = load_word<VEC, 2>(gates + size_t(j * 8 + out_row) * c.ld_x);
        z[j][1] = load_word<VEC, 2>(gates + size_t(j * 8 + out_row) * c.ld_x + 8);
      }
  }
  const float D = c.Dskip[h];
  cp_async_wait<0>();
  __syncthreads();
  if (Y && n > 0) {
    float acc[4][4] = {};
    // ---- with the state
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      uint32_t sp[PARTS][4];
      split_pair<PARTS>(S[0][k].x, S[0][k].y, sp, 0);
      split_pair<PARTS>(S[1][k].x, S[1][k].y, sp, 1);
      split_pair<PARTS>(S[0][k].z, S[0][k].w, sp, 2);
      split_pair<PARTS>(S[1][k].z, S[1][k].w, sp, 3);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (j * 8 >= n) break;
        uint2 cp[PARTS];
#pragma unroll
        for (int p = 0; p < PARTS; ++p) cp[p] = *reinterpret_cast<const uint2*>(&s.c[p][j * 8 + gl][k * 16 + q * 4]);
        mma_parts<PARTS>(acc[j], sp, cp);
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j * 8 >= n) break;
      const float e0 = s.sums[j * 8 + 2 * q].y, e1 = s.sums[j * 8 + 2 * q + 1].y;
      acc[j][0] *= e0; acc[j][1] *= e1; acc[j][2] *= e0; acc[j][3] *= e1;
    }
    // ---- among the rows: weight e^{c_t - c_u} dt_u (C_t . B_u) of row u for row t, with D on the diagonal
    auto weight = [&](int t, int u) {
      const float4 st = s.sums[t], su = s.sums[u];
      const float w = s.cb[t][u] * su.x * __expf((st.z - su.z) + (st.w - su.w));
      return u < t ? w : u == t ? w + D : 0.f;               // (behind the diagonal anything may be there)
    };
    bool odd = false;                                        // x is not finite
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (k * 16 >= n) break;
      uint32_t xp[PARTS][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {                          // channel gl (+ 8), rows 16 k + 2 q (+ 8) and the one behind it
        const int p = warp * 16 + gl + (i & 1) * 8, u = k * 16 + 2 * q + (i >> 1) * 8;
        const float x0 = s.x[u][p], x1 = s.x[u + 1][p];
        odd |= fmaf(x0, 0.f, x1 * 0.f) != 0.f;
        split_pair<PARTS>(x0, x1, xp, i);
      }
      if (__any_sync(0xffffffffu, odd)) break;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (j * 8 >= n) break;
        if (j * 8 + 7 < k * 16) continue;                    // (rows in front of the terms: nothing)
        const int t = j * 8 + gl, u = k * 16 + 2 * q;
        uint32_t w[PARTS][4];
        split_pair<PARTS>(weight(t, u), weight(t, u + 1), w, 0);
        split_pair<PARTS>(weight(t, u + 8), weight(t, u + 9), w, 1);
        uint2 wp[PARTS];
#pragma unroll
        for (int p = 0; p < PARTS; ++p) wp[p] = make_uint2(w[p][0], w[p][1]);
        mma_parts<PARTS>(acc[j], xp, wp);
      }
    }
    if (__any_sync(0xffffffffu, odd)) {
      // In a product a value that is not finite would reach the rows in front of it too, as zero times itself.  (Where the first sixteen rows have gone
      // into the products before one was found, those stay, and the others are added here.)
      bool early = false;
      for (int u = 0; u < min(n, 16); ++u) {
        const float x0 = s.x[u][warp * 16 + gl], x1 = s.x[u][warp * 16 + gl + 8];
        early |= fmaf(x0, 0.f, x1 * 0.f) != 0.f;
      }
      const int from = __any_sync(0xffffffffu, early) ? 0 : 16;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = j * 8 + 2 * q + (i & 1);
#pragma unroll 1
          for (int u = from; u <= t && t < n; ++u) acc[j][i] = fmaf(weight(t, u), s.x[u][warp * 16 + gl + (i >> 1) * 8], acc[j][i]);
        }
    }
    // ---- outputs
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j * 8 >= n) break;
      const int row = j * 8 + out_row;
#pragma unroll
      for (int i = 0; i < 2; ++i) {                          // channels out_ch and + 1, then both + 8
        const float mine = odd_lane ? acc[j][2 * i + 1] : acc[j][2 * i];
        const float got = __shfl_xor_sync(0xffffffffu, odd_lane ? acc[j][2 * i] : acc[j][2 * i + 1], 4);
        if (row >= n) continue;
        const float v0 = (odd_lane ? got : mine) * silu_f(to_f32(z[j][i].v[0])), v1 = (odd_lane ? mine : got) * silu_f(to_f32(z[j][i].v[1]));
        const size_t to = (size_t(r.q0) + row) * c.ld_y + h * NH + out_ch + i * 8;
        if (!a.y_vec) {
          store_row(c.y, c.y_dtype, to, v0, c.status);
          store_row(c.y, c.y_dtype, to + 1, v1, c.status);
        } else if (c.y_dtype == CHUNK_F32) {
          *reinterpret_cast<float2*>(reinterpret_cast<float*>(c.y) + to) = make_float2(v0, v1);
        } else {
          *reinterpret_cast<uint32_t*>(reinterpret_cast<uint16_t*>(c.y) + to) = c.y_dtype == CHUNK_BF16 ? pack_bf16(v0, v1) : pack_f16_sat(v0, v1, c.status);
        }
      }
    }
  }
  if (!r.stores()) return;
  // ---- the state behind the kept rows
  if (r.keep > 0) {
    const float4 last = s.sums[r.keep - 1];
    const float end = last.y;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) S[i][k] = make_float4(S[i][k].x * end, S[i][k].y * end, S[i][k].z * end, S[i][k].w * end);
#pragma unroll 1
    for (int u = 0; u < r.keep; ++u) {
      const float4 su = s.sums[u];
      const float kept = su.x * __expf((last.z - su.z) + (last.w - su.w)), x0 = kept * s.x[u][warp * 16 + gl], x1 = kept * s.x[u][warp * 16 + gl + 8];
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

template <typename TI, int PARTS, bool Y, bool VEC>
cudaError_t launch_vec(const StateArgs& a, cudaStream_t stream) {
  constexpr size_t smem = sizeof(BlockShared<PARTS>);
  static std::atomic<uint32_t> ready{0};                     // devices on which the kernel has been told its shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev >= 32 || !(ready.load() >> dev & 1u)))
    e = cudaFuncSetAttribute(scan_block_kernel<TI, PARTS, Y, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem));
  if (e != cudaSuccess) return e;
  if (dev < 32) ready.fetch_or(1u << dev);
  return launch_pdl(scan_block_kernel<TI, PARTS, Y, VEC>, dim3(unsigned(a.c.H), unsigned(a.c.B)), dim3(128), smem, stream, a);
}

template <typename TI>
cudaError_t launch_for(StateArgs a, cudaStream_t stream) {
  const ChunkScanCall& c = a.c;
  const int item = c.y_dtype == CHUNK_F32 ? 4 : 2;
  a.y_vec = c.y && reinterpret_cast<uintptr_t>(c.y) % (2 * item) == 0 && c.ld_y % 2 == 0 ? 1 : 0;
  const bool vec = c.ld_x % 2 == 0 && reinterpret_cast<uintptr_t>(c.x) % (2 * sizeof(TI)) == 0;
  if (!c.y) return vec ? launch_vec<TI, 2, false, true>(a, stream) : launch_vec<TI, 2, false, false>(a, stream);
  if (scan_wide(c)) return vec ? launch_vec<TI, 3, true, true>(a, stream) : launch_vec<TI, 3, true, false>(a, stream);
  return vec ? launch_vec<TI, 2, true, true>(a, stream) : launch_vec<TI, 2, true, false>(a, stream);
}

}  // namespace

cudaError_t scan_block_launch(const StateArgs& a, cudaStream_t stream) {
  if (a.c.in_dtype == CHUNK_F32) return launch_for<float>(a, stream);
  return a.c.in_dtype == CHUNK_F16 ? launch_for<__half>(a, stream) : launch_for<__nv_bfloat16>(a, stream);
}

}  // namespace hspec
