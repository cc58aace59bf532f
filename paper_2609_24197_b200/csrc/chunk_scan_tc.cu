// The scan of requests with many rows (heads of 64 channels with 128 state elements: the serving shapes) as products on the tensor cores.
//
// A request's rows are cut into chunks of 128.  With c_t the running sum of the steps' log-decays inside a chunk and S the state in front of it,
//   y_t = e^{c_t} (S C_t)  +  sum_{s <= t} e^{c_t - c_s} dt_s (C_t . B_s) x_s  +  D x_t,      S' = e^{c_last} S + sum_s (e^{c_last - c_s} dt_s x_s) B_s^T:
// three products a chunk and head (with the state, inside the chunk, of the next state), 128 x 64 results each over 128 terms.  The states go through a
// chunk one after another, the heads of a request side by side.
//
// The tensor cores take 16-bit operands, the states want more: every operand is split into a bf16 head and a bf16 remainder (16 bits together, any
// exponent of 32 bits), and three products, head x head + head x remainder + remainder x head, leave a relative error of about 2^-18 a term.
//
//   scan_prep_kernel   a block a chunk and group: convolves B and C, writes both split in the layouts in which the next kernel's products take them,
//                      and the scores C_t . B_s below the diagonal (mma.sync: the heads of a group share them, so they are little work)
//   scan_long_kernel   one block an SM over (request, head) items, longest requests first: a warp each to fetch B, to issue the products and to sum up the
//                      steps; and four warps each for scores (times decays, into tensor memory), x (convolved and split), state, and outputs
#include "chunk_scan.cuh"

#include <atomic>
#include <climits>

namespace hspec {

namespace {

constexpr int Q = SCAN_CHUNK, NH = 64, NS = 128;             // rows of a chunk; head width; state elements

// ---------------------------------------------------------------------------------------------------
// Images: what scan_prep_kernel leaves for a chunk and group.
//   B   head, remainder: [2 halves of 64 state elements][128 rows][64] bf16, each row's 16-byte pieces exchanged by the row's low three bits
//   C   head, remainder: [16 groups of 8 state elements][128 rows][8] bf16
//   G   C_t . B_s fp32, four column blocks of 32, of each the rows from 32 times its index on: [8 groups of 4 columns][rows][4]
constexpr int IMG_B = 0, IMG_C = 65536, IMG_G = 131072, IMG_BYTES = IMG_G + 40960;
static_assert(IMG_BYTES == SCAN_IMAGE_BYTES, "the scratch is sized by it");
__host__ __device__ constexpr int g_block(int cb) { return IMG_G + (cb == 0 ? 0 : cb == 1 ? 16384 : cb == 2 ? 28672 : 36864); }

// rows of chunk `ci` of a request: chunks end where the kept rows do
struct ChunkRange { int start, len; };
__device__ __forceinline__ ChunkRange chunk_range(int keep, int upto, int ci) {
  const int k = min(keep, upto), first = (k + Q - 1) / Q;
  ChunkRange r;
  if (ci < first) {
    r.start = ci * Q;
    r.len = min(Q, k - r.start);
  } else {
    r.start = k + (ci - first) * Q;
    r.len = min(Q, upto - r.start);
  }
  return r;
}
__device__ __forceinline__ int chunk_count(int keep, int upto) {
  const int k = min(keep, upto);
  return (k + Q - 1) / Q + (upto - k + Q - 1) / Q;
}

// v = head + remainder, both bf16, for two values; packed with the first in the low half
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo) {
  hi = pack_bf16(a, b);
  const float ra = a - __uint_as_float(hi << 16), rb = b - __uint_as_float(hi & 0xffff0000u);
  lo = pack_bf16(ra, rb);
}

// Row i of the request (raw, four channels from ch on); below zero a carried one, or nothing.
template <typename TI>
__device__ __forceinline__ void raw4(const LongArgs& a, const ScanRequest& r, int ch, int i, int end, float (&x)[4]) {
  const ChunkScanCall& c = a.c;
  const TI* p = nullptr;
  if (i >= 0) {
    if (i < end) p = reinterpret_cast<const TI*>(c.x) + size_t(r.q0 + i) * c.ld_x + c.Di + ch;
  } else if (!r.fresh && i + c.d_conv - 1 >= 0) {
    p = reinterpret_cast<const TI*>(c.conv_state) + (size_t(r.slot) * (c.d_conv - 1) + i + c.d_conv - 1) * c.d_xBC + ch;
  }
  if (!p) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = 0.f;
  } else if (a.vec) {
    const Word<TI, 4> w = *reinterpret_cast<const Word<TI, 4>*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = to_f32(w.v[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = to_f32(p[e]);
  }
}

// Weights of four channels: taps in front of a narrower convolution are zero.
struct Taps {
  float w[4][4], b[4];               // [tap][channel]
  __device__ __forceinline__ void load(const ChunkScanCall& c, int ch) {
    const int K = c.d_conv;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      b[e] = c.conv_b[ch + e];
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j][e] = j >= 4 - K ? c.conv_w[size_t(ch + e) * K + j - (4 - K)] : 0.f;
    }
  }
};

constexpr int PREP_PITCH = NS + 8;   // bf16 of a staged row: the rows of an ldmatrix spread over the banks
constexpr int PREP_SMEM = 4 * Q * PREP_PITCH * 2;

template <typename TI>
__global__ void __launch_bounds__(256) scan_prep_kernel(LongArgs a) {
  const ChunkScanCall& c = a.c;
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) uint16_t staged[];         // B head, B remainder, C head, C remainder
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int items = reinterpret_cast<volatile const int*>(a.plan)[1] * c.G;
  for (int item = blockIdx.x; item < items; item += gridDim.x) {
    const int g = item % c.G;
    const int2 at = *reinterpret_cast<const int2*>(a.chunks + 2 * (item / c.G));
    const ScanRequest r = scan_request(c, at.x);
    const ChunkRange range = chunk_range(r.keep, scan_upto(c, r), at.y);
    uint8_t* img = a.images + size_t(item) * IMG_BYTES;
    // ---- convolution: a thread has four channels of 32 rows
    {
      const int cg = tid & 63, first = (tid >> 6) * 32;
      const bool isC = cg >= 32;
      const int n = (cg & 31) * 4, ch = c.Di + ((isC ? c.G : 0) + g) * NS + n, end = range.start + range.len;
      Taps t;
      t.load(c, ch);
      float w0[4], w1[4], w2[4];
      raw4<TI>(a, r, ch, range.start + first - 3, end, w0);
      raw4<TI>(a, r, ch, range.start + first - 2, end, w1);
      raw4<TI>(a, r, ch, range.start + first - 1, end, w2);
      for (int i0 = 0; i0 < 32; i0 += 8) {
        float x[8][4];
#pragma unroll
        for (int i = 0; i < 8; ++i) raw4<TI>(a, r, ch, range.start + first + i0 + i, end, x[i]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int row = first + i0 + i;
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float s = fmaf(t.w[3][e], x[i][e], fmaf(t.w[2][e], w2[e], fmaf(t.w[1][e], w1[e], fmaf(t.w[0][e], w0[e], t.b[e]))));
            v[e] = row < range.len ? silu_f32(s) : 0.f;
            w0[e] = w1[e]; w1[e] = w2[e]; w2[e] = x[i][e];
          }
          uint2 hi, lo;
          split2(v[0], v[1], hi.x, lo.x);
          split2(v[2], v[3], hi.y, lo.y);
          uint16_t* s = staged + (isC ? 2 : 0) * Q * PREP_PITCH + row * PREP_PITCH + n;
          *reinterpret_cast<uint2*>(s) = hi;
          *reinterpret_cast<uint2*>(s + Q * PREP_PITCH) = lo;
          uint8_t* d;
          if (isC) d = img + IMG_C + ((n >> 3) * Q + row) * 16 + (n & 4) * 2;
          else d = img + IMG_B + (n >> 6) * 16384 + (row >> 3) * 1024 + (row & 7) * 128 + ((((n & 63) >> 3) ^ (row & 7)) << 4) + (n & 4) * 2;
          *reinterpret_cast<uint2*>(d) = hi;
          *reinterpret_cast<uint2*>(d + 32768) = lo;
        }
      }
    }
    __syncthreads();
    if (!c.y) { __syncthreads(); continue; }
    // ---- scores: warp w has rows 16 w .. + 15 against the columns up to the end of their block of 32
    {
      const uint32_t base = smem_u32(staged);
      const int row0 = warp * 16, cols = (warp / 2 + 1) * 32;
      // (ldmatrix: lane l names row l % 16 of the tile, its half of the 16 terms by l / 16; of B two tiles of 8 columns)
      const uint32_t a_at = base + ((2 * Q + row0 + (lane & 15)) * PREP_PITCH + (lane >> 4) * 8) * 2;
      const uint32_t b_at = base + (((lane & 7) + (lane >> 4) * 8) * PREP_PITCH + ((lane >> 3) & 1) * 8) * 2;
      constexpr uint32_t REST = Q * PREP_PITCH * 2;
      for (int c0 = 0; c0 < cols; c0 += 32) {
        float acc[4][4] = {};
#pragma unroll
        for (int ks = 0; ks < NS / 16; ++ks) {
          uint32_t ah[4], al[4];
          ldmatrix_x4(ah, a_at + ks * 32);
          ldmatrix_x4(al, a_at + REST + ks * 32);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            uint32_t bh[4], bl[4];
            ldmatrix_x4(bh, b_at + (c0 + j * 16) * PREP_PITCH * 2 + ks * 32);
            ldmatrix_x4(bl, b_at + REST + (c0 + j * 16) * PREP_PITCH * 2 + ks * 32);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              mma_bf16_16816(acc[2 * j + h], ah, bh[2 * h], bh[2 * h + 1]);
              mma_bf16_16816(acc[2 * j + h], ah, bl[2 * h], bl[2 * h + 1]);
              mma_bf16_16816(acc[2 * j + h], al, bh[2 * h], bh[2 * h + 1]);
            }
          }
        }
        const int cb = c0 / 32;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const int row = row0 + (lane >> 2) + half * 8, col = c0 + j * 8 + (lane & 3) * 2;
            float2 v = make_float2(col <= row ? acc[j][2 * half] : 0.f, col + 1 <= row ? acc[j][2 * half + 1] : 0.f);
            *reinterpret_cast<float2*>(img + g_block(cb) + (((col & 31) >> 2) * (Q - 32 * cb) + row - 32 * cb) * 16 + (col & 2) * 4) = v;
          }
        }
      }
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------------
constexpr int LONG_THREADS = 640;    // four warps for control, then scores, x, state and outputs
constexpr int SM_B = 0, SM_X = 65536, SM_XW = SM_X + 32768, SM_S = SM_XW + 32768, SM_STEPS = SM_S + 32768;    // head, remainder each
struct LongSteps {
  float n_hi[Q], n_lo[Q];            // log2 of dt_s e^{-c_s}, in two parts
  float c_hi[Q], c_lo[Q];            // log2 of e^{c_t}
  float ec[Q];                       // e^{c_t}
  float w[Q];                        // e^{c_last - c_s} dt_s
  float total;                       // e^{c_last}
  float pad[31];
};
struct __align__(8) LongBars {
  uint64_t b_full, x_full, c_full, g_full, s_full;           // operands in place
  uint64_t m_state, m_next, m_near;                          // products done: with the state, of the next state, inside the chunk
  uint64_t next_free, out_free;                              // their results read
  uint64_t x_read;                                           // the carried rows read
  uint64_t steps_full[2], steps_free[2];
  uint32_t tmem;
  uint32_t stop;
};
constexpr int LONG_SMEM = SM_STEPS + 2 * int(sizeof(LongSteps)) + int(sizeof(LongBars));
// tensor memory, columns
constexpr uint32_t TM_C = 0, TM_G = 128, TM_NEAR = 256, TM_STATE = 320, TM_NEXT = 384;

// Waits with a limit of about two seconds; false ends the block's work (the status word says so).
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, LongBars* bars, uint32_t* status, uint32_t code) {
  const uint32_t at = smem_u32(bar);
  uint64_t t0 = 0;
  for (uint32_t i = 0;; ++i) {
    if (mbar_try_wait(at, parity)) return true;
    if ((i & 255u) == 255u) {
      if (*reinterpret_cast<volatile uint32_t*>(&bars->stop)) return false;
      const uint64_t now = global_timer_ns();
      if (t0 == 0) t0 = now;
      else if (now - t0 > 2000000000ull) {
        atomicExch(status, code);
        *reinterpret_cast<volatile uint32_t*>(&bars->stop) = 1;
        return false;
      }
    }
  }
}

__device__ __forceinline__ uint64_t desc_mn(uint32_t addr) {             // rows of 64 values, 16-byte pieces exchanged; halves of 64 16 KB apart
  uint64_t d = 0;
  d |= uint64_t((addr & 0x3FFFF) >> 4);
  d |= uint64_t(16384 >> 4) << 16;
  d |= uint64_t(1024 >> 4) << 32;
  d |= uint64_t(1) << 46;
  d |= uint64_t(2) << 61;
  return d;
}
// fp32 results, bf16 operands, 128 x 64; B (and A, where it is in shared memory) with its rows along the terms
__device__ __forceinline__ constexpr uint32_t long_idesc(bool a_rows) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((a_rows ? 1u : 0u) << 15) | (1u << 16) | ((64u >> 3) << 17) | ((128u >> 4) << 24);
}

// The block's n-th item; the list is sorted longest first, and the rounds run through the blocks forth and back.
__device__ __forceinline__ int long_item(int n) { return n * int(gridDim.x) + ((n & 1) ? int(gridDim.x) - 1 - int(blockIdx.x) : int(blockIdx.x)); }

struct LongItem {
  ScanRequest r;
  int h, g, upto, chunks, base;      // base: the request's first chunk among all
};
__device__ __forceinline__ LongItem long_load(const LongArgs& a, int item) {
  const int2 at = *reinterpret_cast<const int2*>(a.list + 2 * (item / a.c.H));
  LongItem i;
  i.r = scan_request(a.c, at.x);
  i.h = item % a.c.H;
  i.g = i.h / (a.c.H / a.c.G);
  i.upto = scan_upto(a.c, i.r);
  i.chunks = chunk_count(i.r.keep, i.upto);
  i.base = at.y;
  return i;
}

template <typename TI, bool Y>
__global__ void __launch_bounds__(LONG_THREADS, 1) scan_long_kernel(LongArgs a) {
  const ChunkScanCall& c = a.c;
  pdl_wait();
  pdl_trigger();
  const int items = reinterpret_cast<volatile const int*>(a.plan)[0] * c.H;
  if (long_item(0) >= items) return;
  extern __shared__ __align__(1024) uint8_t smem[];
  LongSteps* steps = reinterpret_cast<LongSteps*>(smem + SM_STEPS);
  LongBars* bars = reinterpret_cast<LongBars*>(smem + SM_STEPS + 2 * sizeof(LongSteps));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (warp == 0) {
    if (lane == 0) {
      mbar_init(smem_u32(&bars->b_full), 1);
      mbar_init(smem_u32(&bars->x_full), 128);
      mbar_init(smem_u32(&bars->c_full), 128);
      mbar_init(smem_u32(&bars->g_full), 128);
      mbar_init(smem_u32(&bars->s_full), 128);
      mbar_init(smem_u32(&bars->m_state), 1);
      mbar_init(smem_u32(&bars->m_next), 1);
      mbar_init(smem_u32(&bars->m_near), 1);
      mbar_init(smem_u32(&bars->next_free), 128);
      mbar_init(smem_u32(&bars->out_free), 128);
      mbar_init(smem_u32(&bars->x_read), 128);
      for (int i = 0; i < 2; ++i) {
        mbar_init(smem_u32(&bars->steps_full[i]), 32);
        mbar_init(smem_u32(&bars->steps_free[i]), Y ? 512 : 256);
      }
      bars->stop = (smem_u32(smem) & 1023) ? 1u : 0u;
      if (bars->stop) atomicExch(c.status, STATUS_BAD_SMEM_BASE);
      fence_mbar_init();
    }
    __syncwarp();
    tmem_alloc(smem_u32(&bars->tmem), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars->tmem;
  const bool broken = bars->stop != 0;
  // (a role of whole warps goes on or gives up as a warp)
#define WAIT_ONE(bar, parity, code) \
  if (!wait_for(&bars->bar, parity, bars, c.status, code)) goto done
#define WAIT(bar, parity, code) \
  if (!__all_sync(0xffffffffu, wait_for(&bars->bar, parity, bars, c.status, code))) goto done

  if (broken) goto done;
  if (warp == 0) {
    // ---- B's image, a chunk at a time
    if (lane == 0) {
      uint32_t k = 0;
      bool ok = true;
      for (int n = 0; ok && long_item(n) < items; ++n) {
        const LongItem it = long_load(a, long_item(n));
        for (int ci = 0; ci < it.chunks; ++ci, ++k) {
          ok = !k || wait_for(&bars->m_next, (k - 1) & 1, bars, c.status, STATUS_TIMEOUT_PRODUCER);
          if (!ok) break;
          const uint8_t* src = a.images + (size_t(it.base + ci) * c.G + it.g) * IMG_BYTES + IMG_B;
          const uint32_t bar = smem_u32(&bars->b_full);
          mbar_expect_tx(bar, 65536);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(smem + SM_B + i * 16384)),
                         "l"(src + i * 16384), "r"(16384), "r"(bar) : "memory");
        }
      }
      if (k) mbar_wait(smem_u32(&bars->b_full), (k - 1) & 1);       // (no copy is under way when the block ends)
    }
  } else if (warp == 1) {
    // ---- products
    if (elect_one()) {
      uint32_t k = 0;
      const uint32_t b_hi = smem_u32(smem + SM_B), b_lo = b_hi + 32768, x_hi = smem_u32(smem + SM_X), x_lo = x_hi + 16384;
      const uint32_t w_hi = smem_u32(smem + SM_XW), w_lo = w_hi + 16384, s_hi = smem_u32(smem + SM_S), s_lo = s_hi + 16384;
      for (int n = 0; long_item(n) < items; ++n) {
        const LongItem it = long_load(a, long_item(n));
        for (int ci = 0; ci < it.chunks; ++ci, ++k) {
          const uint32_t now = k & 1, before = now ^ 1;
          // the next state's: B^T (x w)
          WAIT_ONE(b_full, now, STATUS_TIMEOUT_MMA);
          WAIT_ONE(x_full, now, STATUS_TIMEOUT_MMA);
          if (k) WAIT_ONE(next_free, before, STATUS_TIMEOUT_MMA);
          tc_fence_after();
#pragma unroll
          for (int p = 0; p < 3; ++p)
#pragma unroll
            for (int ks = 0; ks < Q / 16; ++ks)
              umma_bf16(tmem + TM_NEXT, desc_mn((p == 2 ? b_lo : b_hi) + ks * 2048), desc_mn((p == 1 ? w_lo : w_hi) + ks * 2048), long_idesc(true), p || ks);
          umma_commit(smem_u32(&bars->m_next));
          if (Y) {
            // with the state: C S
            WAIT_ONE(c_full, now, STATUS_TIMEOUT_MMA);
            WAIT_ONE(s_full, now, STATUS_TIMEOUT_MMA);
            if (k) WAIT_ONE(out_free, before, STATUS_TIMEOUT_MMA);
            tc_fence_after();
#pragma unroll
            for (int p = 0; p < 3; ++p)
#pragma unroll
              for (int ks = 0; ks < NS / 16; ++ks)
                umma_bf16_ts(tmem + TM_STATE, tmem + TM_C + (p == 2 ? 64 : 0) + ks * 8, desc_mn((p == 1 ? s_lo : s_hi) + ks * 2048), long_idesc(false), p || ks);
            umma_commit(smem_u32(&bars->m_state));
            // inside the chunk
            WAIT_ONE(g_full, now, STATUS_TIMEOUT_MMA);
            tc_fence_after();
#pragma unroll
            for (int p = 0; p < 3; ++p)
#pragma unroll
              for (int ks = 0; ks < Q / 16; ++ks)
                umma_bf16_ts(tmem + TM_NEAR, tmem + TM_G + (p == 2 ? 64 : 0) + ks * 8, desc_mn((p == 1 ? x_lo : x_hi) + ks * 2048), long_idesc(false), p || ks);
            umma_commit(smem_u32(&bars->m_near));
          }
        }
      }
    }
  } else if (warp == 2) {
    // ---- steps: a lane has four rows.  The sums are 64-bit: at a sum of 100 a 32-bit one is off by 4e-6, and so would be every weight.
    uint32_t k = 0;
    for (int n = 0; long_item(n) < items; ++n) {
      const LongItem it = long_load(a, long_item(n));
      const double rate = -exp(double(c.A_log[it.h])) * 1.4426950408889634;
      const float bias = c.dt_bias[it.h];
      for (int ci = 0; ci < it.chunks; ++ci, ++k) {
        const ChunkRange range = chunk_range(it.r.keep, it.upto, ci);
        float dt[4];
        double sum[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = lane * 4 + e;
          float raw = 0.f;
          const size_t t = size_t(it.r.q0 + range.start + i);
          if (i < range.len) raw = c.dt_raw ? c.dt_raw[t * c.H + it.h] : to_f32(reinterpret_cast<const TI*>(c.x)[t * c.ld_x + c.Di + c.d_xBC + it.h]);
          dt[e] = i < range.len ? softplus_f32(raw + bias) : 0.f;
          sum[e] = (e ? sum[e - 1] : 0.0) + double(dt[e]) * rate;
        }
        double upto = sum[3];
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
          const double up = __shfl_up_sync(0xffffffffu, upto, off);
          if (lane >= off) upto += up;
        }
        const double all = __shfl_sync(0xffffffffu, upto, 31), front = upto - sum[3];
        if (k >= 2) WAIT(steps_free[k & 1], ((k >> 1) - 1) & 1, STATUS_TIMEOUT_PRODUCER);
        LongSteps& s = steps[k & 1];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = lane * 4 + e;
          const double ct = front + sum[e];
          const float hi = float(ct);
          s.c_hi[i] = hi;
          s.c_lo[i] = float(ct - double(hi));
          s.ec[i] = exp2f(hi);
          s.w[i] = dt[e] * exp2f(float(all - ct));
          const double nd = dt[e] > 0.f ? double(log2f(dt[e])) - ct : -INFINITY;
          const float nh = float(nd);
          s.n_hi[i] = nh;
          s.n_lo[i] = dt[e] > 0.f ? float(nd - double(nh)) : 0.f;
        }
        if (lane == 0) s.total = exp2f(float(all));
        mbar_arrive(smem_u32(&bars->steps_full[k & 1]));
      }
    }
  } else if (warp >= 4 && warp < 8) {
    // ---- scores: C into tensor memory, then the scores times the decays
    if (Y) {
      const int row = tid - 128;
      const uint32_t lanes = tmem + (uint32_t(warp & 3) << 21);
      uint32_t k = 0;
      {
        uint32_t zero[16] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i) tmem_st16(lanes + TM_G + i * 16, zero);      // above the diagonal it stays so
        tmem_st_wait();
      }
      for (int n = 0; long_item(n) < items; ++n) {
        const LongItem it = long_load(a, long_item(n));
        const float D = c.Dskip[it.h];
        for (int ci = 0; ci < it.chunks; ++ci, ++k) {
          const uint8_t* img = a.images + (size_t(it.base + ci) * c.G + it.g) * IMG_BYTES;
          if (k) WAIT(m_state, (k - 1) & 1, STATUS_TIMEOUT_EPILOGUE);
          tc_fence_after();
#pragma unroll
          for (int part = 0; part < 4; ++part) {             // head, head, remainder, remainder
            uint32_t v[32];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const uint4 x = __ldg(reinterpret_cast<const uint4*>(img + IMG_C + part * 16384 + (i * Q + row) * 16));
              v[4 * i] = x.x; v[4 * i + 1] = x.y; v[4 * i + 2] = x.z; v[4 * i + 3] = x.w;
            }
            tmem_st32(lanes + TM_C + part * 32, v);
          }
          tmem_st_wait();
          tc_fence_before();
          mbar_arrive(smem_u32(&bars->c_full));
          WAIT(steps_full[k & 1], (k >> 1) & 1, STATUS_TIMEOUT_EPILOGUE);
          const LongSteps& s = steps[k & 1];
          const uint64_t chi = pack_f32x2(s.c_hi[row], s.c_hi[row]), clo = pack_f32x2(s.c_lo[row], s.c_lo[row]);
          if (k) WAIT(m_near, (k - 1) & 1, STATUS_TIMEOUT_EPILOGUE);
          tc_fence_after();
          for (int cb = 0; cb <= (warp & 3); ++cb) {
            const uint8_t* gsrc = img + g_block(cb) + (row - 32 * cb) * 16;
            const int pitch = (Q - 32 * cb) * 16;
            const bool diag = cb == (warp & 3);
            float4 g4[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) g4[i] = __ldg(reinterpret_cast<const float4*>(gsrc + i * pitch));
            uint32_t hi[16], lo[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int col = cb * 32 + 2 * i;
              const uint64_t e2 = add_f32x2(add_f32x2(chi, *reinterpret_cast<const uint64_t*>(&s.n_hi[col])),
                                            add_f32x2(clo, *reinterpret_cast<const uint64_t*>(&s.n_lo[col])));
              float e0, e1;
              unpack_f32x2(e2, e0, e1);
              if (diag) { e0 = fminf(e0, 126.f); e1 = fminf(e1, 126.f); }      // (above the diagonal: times zero)
              const float4 gg = g4[i >> 1];
              float v0 = ex2_ftz(e0) * ((i & 1) ? gg.z : gg.x), v1 = ex2_ftz(e1) * ((i & 1) ? gg.w : gg.y);
              if (diag) {
                if (2 * i == lane) v0 += D;
                if (2 * i + 1 == lane) v1 += D;
              }
              split2(v0, v1, hi[i], lo[i]);
            }
            tmem_st16(lanes + TM_G + cb * 16, hi);
            tmem_st16(lanes + TM_G + 64 + cb * 16, lo);
          }
          tmem_st_wait();
          tc_fence_before();
          mbar_arrive(smem_u32(&bars->g_full));
          mbar_arrive(smem_u32(&bars->steps_free[k & 1]));
        }
      }
    }
  } else if (warp >= 8 && warp < 12) {
    // ---- x: a thread has four channels of 16 rows
    const int t = tid - 256, cg = t & 15, first = (t >> 4) * 16;
    uint32_t k = 0, reads = 0;
    for (int n = 0; long_item(n) < items; ++n) {
      const LongItem it = long_load(a, long_item(n));
      const int ch = it.h * NH + cg * 4;
      Taps taps;
      taps.load(c, ch);
      for (int ci = 0; ci < it.chunks; ++ci, ++k) {
        const ChunkRange range = chunk_range(it.r.keep, it.upto, ci);
        const int end = range.start + range.len;
        float w0[4], w1[4], w2[4], x[8][4];
        raw4<TI>(a, it.r, ch, range.start + first - 3, end, w0);
        raw4<TI>(a, it.r, ch, range.start + first - 2, end, w1);
        raw4<TI>(a, it.r, ch, range.start + first - 1, end, w2);
#pragma unroll
        for (int i = 0; i < 8; ++i) raw4<TI>(a, it.r, ch, range.start + first + i, end, x[i]);
        WAIT(steps_full[k & 1], (k >> 1) & 1, STATUS_TIMEOUT_EPILOGUE);
        const LongSteps& s = steps[k & 1];
        if (k) {
          WAIT(m_next, (k - 1) & 1, STATUS_TIMEOUT_EPILOGUE);
          if (Y) WAIT(m_near, (k - 1) & 1, STATUS_TIMEOUT_EPILOGUE);
        }
#pragma unroll
        for (int i0 = 0; i0 < 16; i0 += 8) {
          if (i0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) raw4<TI>(a, it.r, ch, range.start + first + i0 + i, end, x[i]);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int row = first + i0 + i;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float u = fmaf(taps.w[3][e], x[i][e], fmaf(taps.w[2][e], w2[e], fmaf(taps.w[1][e], w1[e], fmaf(taps.w[0][e], w0[e], taps.b[e]))));
              v[e] = row < range.len ? silu_f32(u) : 0.f;
              w0[e] = w1[e]; w1[e] = w2[e]; w2[e] = x[i][e];
            }
            uint8_t* d = smem + SM_X + (row >> 3) * 1024 + (row & 7) * 128 + (((cg >> 1) ^ (row & 7)) << 4) + (cg & 1) * 8;
            uint2 hi, lo;
            if (Y) {
              split2(v[0], v[1], hi.x, lo.x);
              split2(v[2], v[3], hi.y, lo.y);
              *reinterpret_cast<uint2*>(d) = hi;
              *reinterpret_cast<uint2*>(d + 16384) = lo;
            }
            const float w = s.w[row];
            split2(v[0] * w, v[1] * w, hi.x, lo.x);
            split2(v[2] * w, v[3] * w, hi.y, lo.y);
            *reinterpret_cast<uint2*>(d + SM_XW - SM_X) = hi;
            *reinterpret_cast<uint2*>(d + SM_XW - SM_X + 16384) = lo;
          }
        }
        fence_proxy_async();
        mbar_arrive(smem_u32(&bars->x_full));
        mbar_arrive(smem_u32(&bars->steps_free[k & 1]));
      }
      // ---- the carried rows of this head's channels, and of its group's B and C for the group's first head: all of it read before any is written
      const int K1 = c.d_conv - 1;
      if (it.r.stores() && K1 > 0) {
        const bool all = it.h % (c.H / c.G) == 0;
        const int width = NH + (all ? 2 * NS : 0);
        TI* carried = reinterpret_cast<TI*>(c.conv_state) + size_t(it.r.slot) * K1 * c.d_xBC;
        auto place = [&](int i, int& j) {
          const int e = i % width;
          j = i / width;
          return e < NH ? it.h * NH + e : e < NH + NS ? c.Di + it.g * NS + e - NH : c.Di + (c.G + it.g) * NS + e - NH - NS;
        };
        TI v[8];                                             // 3 (64 + 256) values over 128 threads
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int i = t + q * 128;
          if (i >= K1 * width) continue;
          int j;
          const int at = place(i, j), from = it.r.keep + j - K1;
          if (from >= 0) v[q] = reinterpret_cast<const TI*>(c.x)[size_t(it.r.q0 + from) * c.ld_x + c.Di + at];
          else if (it.r.fresh) v[q] = TI(0.f);
          else v[q] = carried[size_t(from + K1) * c.d_xBC + at];
        }
        mbar_arrive(smem_u32(&bars->x_read));
        WAIT(x_read, reads & 1, STATUS_TIMEOUT_EPILOGUE);
        ++reads;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int i = t + q * 128;
          if (i >= K1 * width) continue;
          int j;
          const int at = place(i, j);
          carried[size_t(j) * c.d_xBC + at] = v[q];
        }
      }
    }
  } else if (warp >= 12 && warp < 16) {
    // ---- state: a thread has one state element of all 64 channels
    const int e = tid - 384;
    const uint32_t lanes = tmem + (uint32_t(warp & 3) << 21);
    uint32_t k = 0;
    for (int n = 0; long_item(n) < items; ++n) {
      const LongItem it = long_load(a, long_item(n));
      float* mem = c.ssm_state + ((size_t(it.r.slot < 0 ? 0 : it.r.slot) * c.H + it.h) * NH) * NS + e;
      float S[NH];
#pragma unroll
      for (int p = 0; p < NH; ++p) S[p] = it.r.fresh ? 0.f : __ldcs(mem + p * NS);
      if (it.r.keep == 0 && it.r.stores()) {
#pragma unroll
        for (int p = 0; p < NH; ++p) __stcs(mem + p * NS, 0.f);
      }
      for (int ci = 0; ci < it.chunks; ++ci, ++k) {
        if (Y) {
          if (k) WAIT(m_state, (k - 1) & 1, STATUS_TIMEOUT_EPILOGUE);
          uint8_t* d = smem + SM_S + (e >> 3) * 1024 + (e & 7) * 128;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            uint4 hi, lo;
            split2(S[8 * i], S[8 * i + 1], hi.x, lo.x);
            split2(S[8 * i + 2], S[8 * i + 3], hi.y, lo.y);
            split2(S[8 * i + 4], S[8 * i + 5], hi.z, lo.z);
            split2(S[8 * i + 6], S[8 * i + 7], hi.w, lo.w);
            const int at = (i ^ (e & 7)) << 4;
            *reinterpret_cast<uint4*>(d + at) = hi;
            *reinterpret_cast<uint4*>(d + 16384 + at) = lo;
          }
          fence_proxy_async();
          mbar_arrive(smem_u32(&bars->s_full));
        }
        WAIT(steps_full[k & 1], (k >> 1) & 1, STATUS_TIMEOUT_EPILOGUE);
        const float total = steps[k & 1].total;
        mbar_arrive(smem_u32(&bars->steps_free[k & 1]));
        WAIT(m_next, k & 1, STATUS_TIMEOUT_EPILOGUE);
        tc_fence_after();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t v[16];
          tmem_ld16(lanes + TM_NEXT + q * 16, v);
          tmem_wait_ld16(v);
#pragma unroll
          for (int i = 0; i < 16; ++i) S[q * 16 + i] = fmaf(total, S[q * 16 + i], __uint_as_float(v[i]));
        }
        tc_fence_before();
        mbar_arrive(smem_u32(&bars->next_free));
        const ChunkRange range = chunk_range(it.r.keep, it.upto, ci);
        if (range.start + range.len == it.r.keep && it.r.stores()) {
#pragma unroll
          for (int p = 0; p < NH; ++p) __stcs(mem + p * NS, S[p]);
        }
      }
    }
  } else if (warp >= 16) {
    // ---- outputs: a thread has one row's 64 channels
    if (Y) {
      const int row = tid - 512;
      const uint32_t lanes = tmem + (uint32_t(warp & 3) << 21);
      uint32_t k = 0;
      for (int n = 0; long_item(n) < items; ++n) {
        const LongItem it = long_load(a, long_item(n));
        for (int ci = 0; ci < it.chunks; ++ci, ++k) {
          const ChunkRange range = chunk_range(it.r.keep, it.upto, ci);
          const bool on = row < range.len;
          const size_t t = size_t(it.r.q0 + range.start + row);
          const TI* z = reinterpret_cast<const TI*>(c.x) + t * c.ld_x + it.h * NH;
          WAIT(steps_full[k & 1], (k >> 1) & 1, STATUS_TIMEOUT_EPILOGUE);
          const float ec = steps[k & 1].ec[row];
          mbar_arrive(smem_u32(&bars->steps_free[k & 1]));
          WAIT(m_near, k & 1, STATUS_TIMEOUT_EPILOGUE);
          tc_fence_after();
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float zz[16];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (on && a.vec) {
                const Word<TI, 4> w = *reinterpret_cast<const Word<TI, 4>*>(z + q * 16 + i * 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) zz[4 * i + j] = to_f32(w.v[j]);
              } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) zz[4 * i + j] = on ? to_f32(z[q * 16 + i * 4 + j]) : 0.f;
              }
            }
            uint32_t near[16], state[16];
            tmem_ld16(lanes + TM_NEAR + q * 16, near);
            tmem_ld16(lanes + TM_STATE + q * 16, state);
            tmem_wait_ld16(near);
            tmem_wait_ld16(state);
            if (q == 3) {
              tc_fence_before();
              mbar_arrive(smem_u32(&bars->out_free));
            }
            float y[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = fmaf(ec, __uint_as_float(state[i]), __uint_as_float(near[i])) * silu_f32(zz[i]);
            if (!on) continue;
            const size_t at = t * c.ld_y + it.h * NH + q * 16;
            if (!a.y_vec) {
#pragma unroll
              for (int i = 0; i < 16; ++i) store_row(c.y, c.y_dtype, at + i, y[i], c.status);
            } else if (c.y_dtype == CHUNK_F32) {
#pragma unroll
              for (int i = 0; i < 4; ++i) reinterpret_cast<float4*>(reinterpret_cast<float*>(c.y) + at)[i] = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
            } else {
              uint32_t o[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) o[i] = c.y_dtype == CHUNK_BF16 ? pack_bf16(y[2 * i], y[2 * i + 1]) : pack_f16_sat(y[2 * i], y[2 * i + 1], c.status);
              uint4* d = reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(c.y) + at);
              d[0] = make_uint4(o[0], o[1], o[2], o[3]);
              d[1] = make_uint4(o[4], o[5], o[6], o[7]);
            }
          }
        }
      }
    }
  }
done:
#undef WAIT
#undef WAIT_ONE
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, 512);
}

template <typename TI>
cudaError_t launch_for(LongArgs a, cudaStream_t stream) {
  const ChunkScanCall& c = a.c;
  auto on = [](const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; };
  a.vec = c.Di % 4 == 0 && c.ld_x % 4 == 0 && on(c.x, 4 * sizeof(TI)) && on(c.conv_state, 4 * sizeof(TI)) ? 1 : 0;
  const int item = c.y_dtype == CHUNK_F32 ? 4 : 2;
  a.y_vec = c.y && on(c.y, 16) && c.ld_y % (16 / item) == 0 ? 1 : 0;
  static std::atomic<uint32_t> ready{0};                     // devices on which the kernels have been told their shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 32 || !(ready.load() >> dev & 1u)) {
    e = cudaFuncSetAttribute(scan_prep_kernel<TI>, cudaFuncAttributeMaxDynamicSharedMemorySize, PREP_SMEM);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(scan_long_kernel<TI, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, LONG_SMEM);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(scan_long_kernel<TI, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, LONG_SMEM);
    if (e != cudaSuccess) return e;
    if (dev < 32) ready.fetch_or(1u << dev);
  }
  const long long chunks = (long long)(scan_max_chunks(c.T, c.B)) * c.G, heads = (long long)(scan_max_long(c.T, c.B)) * c.H;
  e = launch_pdl(scan_prep_kernel<TI>, dim3(unsigned(chunks < 148 ? chunks : 148)), dim3(256), PREP_SMEM, stream, a);
  if (e != cudaSuccess) return e;
  return launch_pdl(c.y ? scan_long_kernel<TI, true> : scan_long_kernel<TI, false>, dim3(unsigned(heads < 148 ? heads : 148)), dim3(LONG_THREADS), LONG_SMEM,
                    stream, a);
}

}  // namespace

cudaError_t scan_long_launch(const LongArgs& a, cudaStream_t stream) {
  if (a.c.in_dtype == CHUNK_F32) return launch_for<float>(a, stream);
  return a.c.in_dtype == CHUNK_F16 ? launch_for<__half>(a, stream) : launch_for<__nv_bfloat16>(a, stream);
}

}  // namespace hspec
