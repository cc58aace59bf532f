// The scan of requests with many rows (heads of 64 channels with 128 state elements: the serving shapes) as products on the tensor cores.
//
// A request's rows are cut into chunks of 128.  With c_t the running sum of the steps' log-decays inside a chunk and S the state in front of it,
//   y_t = e^{c_t} (S C_t)  +  sum_{s <= t} e^{c_t - c_s} dt_s (C_t . B_s) x_s  +  D x_t,      S' = e^{c_last} S + sum_s (e^{c_last - c_s} dt_s x_s) B_s^T:
// three products a chunk and head (with the state, inside the chunk, of the next state), 128 x 64 results each over 128 terms.  The states go through a
// chunk one after another, the heads of a request side by side.
//
// The tensor cores take 16-bit operands, the states want more: every operand is split into a bf16 head and a bf16 remainder (16 bits together, any
// exponent of 32 bits), and three products, head x head + head x remainder + remainder x head, leave a relative error of some 2^-18 a term, 3 x 2^-16 at
// most (outputs would be off by 4.6e-6 of their 2-norm, below what 16 bits round away; states are, by 3e-7 where a few hundred rows count in them, and by up
// to 5e-6 where some twenty do).  Outputs of 32 bits take three parts and six products (WIDE: off by 4e-7, in 860 us where two parts took 600): shared memory
// holds them because the scores come from the images, and tensor memory because both products of an output add up in one place.  The next state has two
// parts there too: a third one of B would not fit.
//
//   scan_prep_kernel   a block a chunk and group: convolves B and C, writes both split in the layouts in which the next kernel's products take them,
//                      and the scores C_t . B_s below the diagonal (mma.sync: the heads of a group share them, so they are little work)
//   scan_long_kernel   one block an SM over (request, head) items, longest requests first; all its warps go through a chunk's work together
//
// A prompt of 8192 rows, 128 heads: 536 us, of them 505 in the second kernel and 31 in the first (they overlap at their ends).  A chunk and head takes 15 000
// clocks: 4800 are instructions to issue, the tensor pipe is busy for a sixth, the rest is the latency of one phase after another with 16 warps on the SM.
#pragma once
#include "chunk_scan.cuh"

#include <atomic>
#include <climits>
#include <cstddef>

namespace hspec {

namespace {

constexpr int Q = SCAN_CHUNK, NH = 64, NS = 128;             // rows of a chunk; head width; state elements

// ---------------------------------------------------------------------------------------------------
// Images: what scan_prep_kernel leaves for a chunk and group.
//   B   head, remainder: [2 halves of 64 state elements][128 rows][64] bf16, each row's 16-byte pieces exchanged by the row's low three bits
//   C   head, remainder: [16 groups of 8 state elements][128 rows][8] bf16; WIDE: [32 groups of 4 state elements][128 rows][4] fp32
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

constexpr int PREP_PITCH = NS + 8;   // bf16 of a staged row: the rows of an ldmatrix spread over the banks
constexpr int prep_smem(bool wide) { return (wide ? 6 : 4) * Q * PREP_PITCH * 2; }

template <typename TI, bool VEC, bool WIDE>
__global__ void __launch_bounds__(256) scan_prep_kernel(LongArgs a) {
  constexpr int PARTS = WIDE ? 3 : 2;
  const ChunkScanCall& c = a.c;
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) uint16_t staged[];         // B's parts, then C's
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
      Taps<2, VEC ? 4 : 0> t;
      t.load(c, ch);
      const RawRows<VEC, 4, TI> raw(c, r, ch);
      Word<TI, 4> next[8], front[3];
#pragma unroll
      for (int i = 0; i < 8; ++i) next[i] = raw.row(range.start + first + i, end - 1);
      raw.front(front, range.start + first, end - 1);
      uint64_t before[3][2];
      raw.front_value(front, range.start + first, before);
      for (int i0 = 0; i0 < 32; i0 += 8) {
        Word<TI, 4> x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = next[i];
        if (i0 < 24) {
#pragma unroll
          for (int i = 0; i < 8; ++i) next[i] = raw.row(range.start + first + i0 + 8 + i, end - 1);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int row = first + i0 + i;
          uint64_t now[2], v[2];
          widen(x[i], now);
          t.next(before, now, v);
          if (row >= range.len) v[0] = v[1] = 0ull;
          uint32_t part[2][PARTS];
          split_parts(v[0], part[0]);
          split_parts(v[1], part[1]);
          uint16_t* s = staged + (isC ? PARTS : 0) * Q * PREP_PITCH + row * PREP_PITCH + n;
#pragma unroll
          for (int p = 0; p < PARTS; ++p) *reinterpret_cast<uint2*>(s + p * Q * PREP_PITCH) = make_uint2(part[0][p], part[1][p]);
          uint8_t* d;
          if (WIDE && isC) {
            *reinterpret_cast<ulonglong2*>(img + IMG_C + ((n >> 2) * Q + row) * 16) = make_ulonglong2(v[0], v[1]);
            continue;
          }
          if (isC) d = img + IMG_C + ((n >> 3) * Q + row) * 16 + (n & 4) * 2;
          else d = img + IMG_B + (n >> 6) * 16384 + (row >> 3) * 1024 + (row & 7) * 128 + ((((n & 63) >> 3) ^ (row & 7)) << 4) + (n & 4) * 2;
          *reinterpret_cast<uint2*>(d) = make_uint2(part[0][0], part[1][0]);
          *reinterpret_cast<uint2*>(d + 32768) = make_uint2(part[0][1], part[1][1]);
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
      const uint32_t a_at = base + ((PARTS * Q + row0 + (lane & 15)) * PREP_PITCH + (lane >> 4) * 8) * 2;
      const uint32_t b_at = base + (((lane & 7) + (lane >> 4) * 8) * PREP_PITCH + ((lane >> 3) & 1) * 8) * 2;
      constexpr uint32_t REST = Q * PREP_PITCH * 2;
      for (int c0 = 0; c0 < cols; c0 += 32) {
        float acc[4][4] = {};
#pragma unroll
        for (int ks = 0; ks < NS / 16; ++ks) {
          uint32_t cp[PARTS][4];
#pragma unroll
          for (int p = 0; p < PARTS; ++p) ldmatrix_x4(cp[p], a_at + p * REST + ks * 32);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            uint32_t bp[PARTS][4];
#pragma unroll
            for (int p = 0; p < PARTS; ++p) ldmatrix_x4(bp[p], b_at + p * REST + (c0 + j * 16) * PREP_PITCH * 2 + ks * 32);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int x = 0; x < PARTS; ++x)
#pragma unroll
                for (int y = 0; x + y < PARTS; ++y) mma_bf16_16816(acc[2 * j + h], cp[x], bp[y][2 * h], bp[y][2 * h + 1]);
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
// All warps go through a chunk's work together, two block barriers a chunk: what the products need (x split and the scores into place), then, under the
// products, what can be done ahead (the next chunk's convolution and steps, this one's gates), then what the products gave (outputs, state).  (With a
// role for every four to eight warps and barriers in shared memory between them the 8192 rows took 1514 us, then 560 without: a warp alone on its scheduler runs at its
// instructions' latency, and those that wait take the others' issue slots with their polling.)
constexpr int LONG_THREADS = 512;
// Shared memory: B's two parts, x's, weighted x's two, the state's; scores (WIDE: these come from the image) and steps.
template <bool WIDE>
struct LongLayout {
  static constexpr int PARTS = WIDE ? 3 : 2, B = 0, X = 65536, XW = X + PARTS * 16384, S = XW + 32768, G = S + PARTS * 16384,
                       STEPS = G + (WIDE ? 0 : IMG_BYTES - IMG_G);
  // tensor memory, columns.  WIDE: C has e^{c_t} in it, so that both products of an output add up in one place (NEAR), and the next state's in 64 columns.
  static constexpr uint32_t TM_C = 0, TM_G = WIDE ? 192 : 128, TM_NEAR = WIDE ? 384 : 256, TM_STATE = WIDE ? 384 : 320, TM_NEXT = WIDE ? 448 : 384;
};
struct LongSteps {
  float n_hi[Q], n_lo[Q];            // log2 of dt_s e^{-c_s}, in two parts
  float c_hi[Q], c_lo[Q];            // log2 of e^{c_t}
  float ec[Q];                       // e^{c_t}
  float w[Q];                        // e^{c_last - c_s} dt_s
  float total;                       // e^{c_last}
  float pad[31];
};
struct __align__(8) LongBars {
  uint64_t b_full, scores_full;      // copies landed
  uint64_t products;                 // done
  double sums[4];                    // of 32 steps each
  uint32_t tmem;
  uint32_t stop;                     // a wait gave up
  int any_odd[2], first_odd[2][NH];  // of a chunk (by its parity): whether x is finite, each channel's first row where not
};
template <bool WIDE> constexpr int LONG_SMEM = LongLayout<WIDE>::STEPS + 2 * int(sizeof(LongSteps)) + int(sizeof(LongBars));
static_assert(LONG_SMEM<false> <= 227 * 1024 && LONG_SMEM<true> <= 227 * 1024 && prep_smem(true) <= 227 * 1024, "a block's shared memory");

// Waits for a phase, with a limit (four million polls, some 0.1 to 4 s), after which the block's work ends (the status word says so).
__device__ __forceinline__ void wait_for(uint64_t* bar, uint32_t parity, LongBars* bars, uint32_t* status, uint32_t code) {
  const uint32_t at = smem_u32(bar);
  uint32_t left = 1u << 22;
  while (!mbar_try_wait(at, parity))
    if (--left == 0) {
      atomicExch(status, code);
      *reinterpret_cast<volatile uint32_t*>(&bars->stop) = 1;
      return;
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
// fp32 results, bf16 operands, 128 x n; B (and A, where it is in shared memory) with its rows along the terms
__device__ __forceinline__ constexpr uint32_t long_idesc(bool a_rows, uint32_t n) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((a_rows ? 1u : 0u) << 15) | (1u << 16) | ((n >> 3) << 17) | ((128u >> 4) << 24);
}

__device__ __forceinline__ void tmem_st4(uint32_t taddr, const uint32_t (&r)[4]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}

// Shared memory by its own address.
__device__ __forceinline__ uint4 lds16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}
__device__ __forceinline__ void sts4(uint32_t at, uint32_t v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(at), "r"(v) : "memory"); }
__device__ __forceinline__ void sts16(uint32_t at, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// One copy of a multiple of 16 bytes from and to 16-byte boundaries, counted by the barrier.
__device__ __forceinline__ void bulk_load(uint8_t* dst, const uint8_t* src, uint32_t bytes, uint64_t* bar) {
  mbar_expect_tx(smem_u32(bar), bytes);
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)), "l"(src), "r"(bytes),
               "r"(smem_u32(bar)) : "memory");
}

// The block's n-th item; the list is sorted longest first, and the rounds run through the blocks forth and back.
__device__ __forceinline__ int long_item(int n) { return n * int(gridDim.x) + ((n & 1) ? int(gridDim.x) - 1 - int(blockIdx.x) : int(blockIdx.x)); }

template <typename TI> __device__ __forceinline__ TI from_bits(uint32_t v);
template <> __device__ __forceinline__ float from_bits(uint32_t v) { return __uint_as_float(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_bits(uint32_t v) { return __ushort_as_bfloat16(uint16_t(v)); }
template <> __device__ __forceinline__ __half from_bits(uint32_t v) { return __ushort_as_half(uint16_t(v)); }

template <typename TI, bool Y, bool VEC, bool WIDE>
__global__ void __launch_bounds__(LONG_THREADS, 1) scan_long_kernel(LongArgs a) {
  using At = LongLayout<WIDE>;
  constexpr int PARTS = At::PARTS, SM_B = At::B, SM_X = At::X, SM_XW = At::XW, SM_S = At::S, SM_G = At::G, SM_STEPS = At::STEPS;
  constexpr uint32_t TM_C = At::TM_C, TM_G = At::TM_G, TM_NEAR = At::TM_NEAR, TM_STATE = At::TM_STATE, TM_NEXT = At::TM_NEXT;
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
      mbar_init(smem_u32(&bars->scores_full), 1);
      mbar_init(smem_u32(&bars->products), 1);
      for (int i = 0; i < 2 * NH; ++i) bars->first_odd[i / NH][i % NH] = Q;
      bars->any_odd[0] = bars->any_odd[1] = 0;
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
  // a thread's lane of tensor memory (a row of the chunk, or a state element), and its quarter of the columns
  const int row = (warp & 3) * 32 + lane, quarter = warp >> 2;
  const uint32_t lanes = tmem + (uint32_t(warp & 3) << 21);
  if (Y) {
    uint32_t zero[16] = {};
#pragma unroll
    for (int i = 0; i < PARTS; ++i) tmem_st16(lanes + TM_G + (quarter * PARTS + i) * 16, zero);        // above the diagonal it stays so
    tmem_st_wait();
  }
  const int cp = lane * 2, first = warp * 8;                 // its two channels of x and its eight rows of them
  uint32_t k = 0;                                            // chunks so far
  volatile uint32_t* stop = &bars->stop;
  for (int n = 0; long_item(n) < items && !*stop; ++n) {
    const int item = long_item(n);
    const int2 at = *reinterpret_cast<const int2*>(a.list + 2 * (item / c.H));
    const int h = item % c.H, g = h / (c.H / c.G);
    const ScanRequest r = scan_request(c, at.x);
    const int upto = scan_upto(c, r), chunks = chunk_count(r.keep, upto);
    const uint8_t* img = a.images + (size_t(at.y) * c.G + g) * IMG_BYTES;
    const TI* rows0 = reinterpret_cast<const TI*>(c.x) + size_t(r.q0) * c.ld_x + h * NH;             // the request's gates; x stands Di behind them
    float* mem = c.ssm_state + (((size_t(r.slot < 0 ? 0 : r.slot) * c.H + h) * NH) + quarter * 16) * NS + row;
    if (tid == 0) {
      bulk_load(smem + SM_B, img + IMG_B, 65536, &bars->b_full);
      if (Y && !WIDE) bulk_load(smem + SM_G, img + IMG_G, IMG_BYTES - IMG_G, &bars->scores_full);
    }
    Taps<1, VEC ? 4 : 0> taps;
    taps.load(c, h * NH + cp);
    const RawRows<VEC, 2, TI> raw(c, r, h * NH + cp);
    const double rate = -exp(double(c.A_log[h])) * 1.4426950408889634;
    const float dt_bias = c.dt_bias[h], D = c.Dskip[h];
    // the raw value that a row's step comes from (a row each for the second four warps: the first warp issues the products)
    auto raw_step = [&](const ChunkRange& range) {
      const size_t t = size_t(r.q0 + range.start + row);
      return quarter != 1 || row >= range.len ? 0.f
             : c.dt_raw ? c.dt_raw[t * c.H + h] : to_f32(reinterpret_cast<const TI*>(c.x)[t * c.ld_x + c.Di + c.d_xBC + h]);
    };
    // The steps of a chunk.  Their sums are 64-bit: at a sum of 100 a 32-bit one is off by 4e-6, and so would be every weight.
    auto make_steps = [&](LongSteps& s, float raw, int len) {
      const float dt = row < len ? softplus_f32(raw + dt_bias) : 0.f;
      double ct = double(dt) * rate;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const double up = __shfl_up_sync(0xffffffffu, ct, off);
        if (lane >= off) ct += up;
      }
      if (lane == 31) bars->sums[warp & 3] = ct;
      asm volatile("bar.sync 1, 128;" ::: "memory");
      double all = 0.0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const double part = bars->sums[i];
        if (i < (warp & 3)) ct += part;
        all += part;
      }
      asm volatile("bar.sync 1, 128;" ::: "memory");
      const float hi = float(ct);
      s.c_hi[row] = hi;
      s.c_lo[row] = float(ct - double(hi));
      s.ec[row] = ex2_ftz(hi);
      s.w[row] = dt * ex2_ftz(float(all - ct));
      const double nd = dt > 0.f ? double(__log2f(dt)) - ct : dt == 0.f ? -INFINITY : double(dt);
      const float nh = float(nd);
      s.n_hi[row] = nh;
      s.n_lo[row] = dt > 0.f ? float(nd - double(nh)) : 0.f;
      if (row == 0) s.total = ex2_ftz(float(all));
    };
    // x: eight raw rows become v, and `odd`: zero times every value, NaN where one is not finite
    Word<TI, 2> held[8], front[3];
    uint64_t v[8], odd;
    auto fetch_x = [&](const ChunkRange& range) {
      const int last = range.start + range.len - 1;
      if (range.len == Q && range.start >= 3) {
        const TI* p = raw.x + size_t(range.start + first - 3) * raw.ld;
#pragma unroll
        for (int i = 0; i < 3; ++i, p += raw.ld) front[i] = load_word<VEC, 2>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i, p += raw.ld) held[i] = load_word<VEC, 2>(p);
        return;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) held[i] = raw.row(range.start + first + i, last);
      raw.front(front, range.start + first, last);
    };
    auto convolve = [&](const ChunkRange& range) {
      uint64_t before[3][1];
      raw.front_value(front, range.start + first, before);
      odd = 0ull;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint64_t now[1], u[1];
        widen(held[i], now);
        taps.next(before, now, u);
        odd = fma_f32x2(u[0], 0ull, odd);
        v[i] = u[0];
      }
    };
    // state: one element of 16 channels
    float S[16];
    auto put_state = [&] {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t to = smem_u32(smem + SM_S) + (row >> 3) * 1024 + (row & 7) * 128 + (((quarter * 2 + i) ^ (row & 7)) << 4);
        uint32_t part[4][PARTS];
#pragma unroll
        for (int e = 0; e < 4; ++e) split_parts(pack_f32x2(S[8 * i + 2 * e], S[8 * i + 2 * e + 1]), part[e]);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) sts16(to + p * 16384, make_uint4(part[0][p], part[1][p], part[2][p], part[3][p]));
      }
    };
    ChunkRange range = chunk_range(r.keep, upto, 0);
    fetch_x(range);
    float step = raw_step(range);
#pragma unroll
    for (int p = 0; p < 16; ++p) S[p] = r.fresh ? 0.f : __ldcs(mem + p * NS);
    if (r.keep == 0 && r.stores()) {
#pragma unroll
      for (int p = 0; p < 16; ++p) __stcs(mem + p * NS, 0.f);
    }
    if (Y) put_state();
    if (quarter == 1) make_steps(steps[k & 1], step, range.len);
    convolve(range);
    if (chunks > 1) {
      const ChunkRange next = chunk_range(r.keep, upto, 1);
      fetch_x(next);
      step = raw_step(next);
    }
    __syncthreads();
    for (int ci = 0; ci < chunks; ++ci, ++k) {
      const LongSteps& s = steps[k & 1];
      const uint32_t s_at = smem_u32(&s);
      // ---- operands of the products: C
      uint32_t cw[32];
      if (Y) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint4 x = __ldg(reinterpret_cast<const uint4*>(img + IMG_C + ((quarter * 8 + i) * Q + row) * 16));
          cw[4 * i] = x.x; cw[4 * i + 1] = x.y; cw[4 * i + 2] = x.z; cw[4 * i + 3] = x.w;
        }
      }
      // ---- x
      {
        const uint32_t to = smem_u32(smem + SM_X) + warp * 1024 + (lane & 3) * 4;
        const uint4 wa = lds16(s_at + offsetof(LongSteps, w) + first * 4), wb = lds16(s_at + offsetof(LongSteps, w) + first * 4 + 16);
        const uint32_t w[8] = {wa.x, wa.y, wa.z, wa.w, wb.x, wb.y, wb.z, wb.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t at = to + i * 128 + (((lane >> 2) ^ i) << 4);
          uint32_t hi, lo;
          if (Y) {
            uint32_t part[PARTS];
            split_parts(v[i], part);
#pragma unroll
            for (int p = 0; p < PARTS; ++p) sts4(at + p * 16384, part[p]);
          }
          split2(mul_f32x2(v[i], dup2(__uint_as_float(w[i]))), hi, lo);
          sts4(at + SM_XW - SM_X, hi);
          sts4(at + SM_XW - SM_X + 16384, lo);
        }
        // A value that is not finite would reach the rows in front of it too, as zero times itself: it leaves the operands, and what it reaches is made
        // NaN where the products are read.  (Rows behind the last one repeat it, with weight zero: they are cleared as well.)
        float odd0, odd1;
        unpack_f32x2(odd, odd0, odd1);
        if (odd0 + odd1 != 0.f) {
          // (x alone decides: its weighted form is NaN in every row of a chunk that has a step without a number, and stays so for the state)
          uint32_t bad = Y ? 0xffff : 0;
          if (!Y) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float x0, x1;
              unpack_f32x2(v[i], x0, x1);
              bad |= (fabsf(x0) < INFINITY ? 0u : 1u << 2 * i) | (fabsf(x1) < INFINITY ? 0u : 2u << 2 * i);
            }
          }
#pragma unroll 1
          for (; bad; bad &= bad - 1) {
            const int i = (__ffs(bad) - 1) >> 1, e = (__ffs(bad) - 1) & 1;
            uint16_t* x = reinterpret_cast<uint16_t*>(smem + SM_X + warp * 1024 + i * 128 + (((lane >> 2) ^ i) << 4) + (lane & 3) * 4) + e;
            uint16_t* w = x + (SM_XW - SM_X) / 2;
            if (Y) {
              if ((x[0] & 0x7f80) != 0x7f80) continue;
#pragma unroll
              for (int p = 0; p < PARTS; ++p) x[p * 8192] = 0;
            }
            w[0] = w[8192] = 0;
            if (first + i < range.len) {
              atomicMin(&bars->first_odd[k & 1][cp + e], first + i);
              *reinterpret_cast<volatile int*>(&bars->any_odd[k & 1]) = 1;
            }
          }
        }
      }
      // ---- scores times decays: every fourth block of 8 columns up to the diagonal's
      if (Y) {
        if constexpr (WIDE) {
          const uint64_t ec = dup2(s.ec[row]);
          uint32_t part[PARTS][16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            uint32_t one[PARTS];
            split_parts(mul_f32x2(ec, pack_f32x2(__uint_as_float(cw[2 * i]), __uint_as_float(cw[2 * i + 1]))), one);
#pragma unroll
            for (int p = 0; p < PARTS; ++p) part[p][i] = one[p];
          }
#pragma unroll
          for (int p = 0; p < PARTS; ++p) tmem_st16(lanes + TM_C + p * 64 + quarter * 16, part[p]);
        } else {
          wait_for(&bars->scores_full, k & 1, bars, c.status, STATUS_TIMEOUT_EPILOGUE);
          tmem_st32(lanes + TM_C + quarter * 32, cw);
        }
        const uint64_t chi = dup2(s.c_hi[row]), clo = dup2(s.c_lo[row]);
        auto two = [](uint32_t a, uint32_t b) { return pack_f32x2(__uint_as_float(a), __uint_as_float(b)); };
        uint4 gg[2], nh[2], nl[2];
        auto fetch = [&](int cb) {
          const int pitch = (Q - 32 * cb) * 16, o = cb * 4 + quarter;
          const int from = g_block(cb) + (row - 32 * cb) * 16 + quarter * 2 * pitch;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if constexpr (WIDE) gg[i] = __ldg(reinterpret_cast<const uint4*>(img + from + i * pitch));
            else gg[i] = lds16(smem_u32(smem + SM_G) - IMG_G + from + i * pitch);
            nh[i] = lds16(s_at + (o * 8 + 4 * i) * 4);
            nl[i] = lds16(s_at + (Q + o * 8 + 4 * i) * 4);
          }
        };
        fetch(0);
#pragma unroll
        for (int cb = 0; cb < 4; ++cb) {
          if (cb > (warp & 3)) break;
          const int o = cb * 4 + quarter;
          uint64_t u[4];
          float e[8];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            unpack_f32x2(add_f32x2(add_f32x2(chi, two(nh[i].x, nh[i].y)), add_f32x2(clo, two(nl[i].x, nl[i].y))), e[4 * i], e[4 * i + 1]);
            unpack_f32x2(add_f32x2(add_f32x2(chi, two(nh[i].z, nh[i].w)), add_f32x2(clo, two(nl[i].z, nl[i].w))), e[4 * i + 2], e[4 * i + 3]);
            u[2 * i] = mul_f32x2(pack_f32x2(ex2_ftz(e[4 * i]), ex2_ftz(e[4 * i + 1])), two(gg[i].x, gg[i].y));
            u[2 * i + 1] = mul_f32x2(pack_f32x2(ex2_ftz(e[4 * i + 2]), ex2_ftz(e[4 * i + 3])), two(gg[i].z, gg[i].w));
          }
          if (cb < (warp & 3)) {
            fetch(cb + 1);
          } else {                                             // (above the diagonal the weights may be anything)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int col = o * 8 + 2 * i;
              float u0, u1;
              unpack_f32x2(u[i], u0, u1);
              u[i] = pack_f32x2(col < row ? u0 : col == row ? u0 + D : 0.f, col + 1 < row ? u1 : col + 1 == row ? u1 + D : 0.f);
            }
          }
          uint32_t part[PARTS][4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t one[PARTS];
            split_parts(u[i], one);
#pragma unroll
            for (int p = 0; p < PARTS; ++p) part[p][i] = one[p];
          }
#pragma unroll
          for (int p = 0; p < PARTS; ++p) tmem_st4(lanes + TM_G + p * 64 + o * 4, part[p]);
        }
        tmem_st_wait();
      }
      fence_proxy_async();
      tc_fence_before();
      __syncthreads();
      // ---- the products, in parts that the first warp issues between its own work: it would wait for the tensor core otherwise
      img += size_t(c.G) * IMG_BYTES;
      constexpr int NEXTS = WIDE ? 3 : 2, EACH = WIDE ? 6 : 3, ALL = Y ? NEXTS + 2 * EACH : NEXTS;        // of the next state; of each of an output's two; all
      auto issue = [&](int part) {
        if (warp == 0) {
          if (elect_one()) {
            constexpr uint64_t REST = 16384 >> 4;            // from an operand's part to the next (B: twice that)
            if (part == 0) {
              tc_fence_after();
              wait_for(&bars->b_full, k & 1, bars, c.status, STATUS_TIMEOUT_MMA);
            }
            if (part < NEXTS) {
              // the next state's: B's head times the head and the remainder of x at once (their places are as far apart as the halves of a 128-column
              // operand), next to one another, then its remainder times the head: A comes from shared memory, which is what bounds this one.  WIDE: one
              // after another, for want of columns.
              const int b_part = WIDE ? part == 2 : part, w_part = WIDE && part == 1;
              const uint64_t b_at = desc_mn(smem_u32(smem + SM_B)) + b_part * 2 * REST, w_at = desc_mn(smem_u32(smem + SM_XW)) + w_part * REST;
              const uint32_t shape = WIDE || part ? long_idesc(true, 64) : long_idesc(true, 128);
#pragma unroll
              for (int ks = 0; ks < Q / 16; ++ks) umma_bf16(tmem + TM_NEXT, b_at + ks * 128, w_at + ks * 128, shape, part || ks);
            } else {
              // inside the chunk, then with the state: head x head, head x remainder, remainder x head.  WIDE: of parts h, m and l the smallest products
              // first, lh, hl, mm, mh, hm for both, then hh for both: the tensor cores cut the bits that do not fit a sum, at its size then.
              const int n = part - NEXTS, one = EACH - 1;
              const bool far = WIDE ? (n < 2 * one ? n >= one : n == 2 * one + 1) : n >= EACH;
              const int p = !WIDE ? n - (far ? EACH : 0) : n < 2 * one ? n - (far ? one : 0) : one;
              const int left = WIDE ? (p == 0 ? 2 : p == 2 || p == 3) : p == 2, right = WIDE ? (p == 1 ? 2 : p == 2 || p == 4) : p == 1;
              const uint32_t a_at = tmem + (far ? TM_C : TM_G) + left * 64, to = tmem + (far ? TM_STATE : TM_NEAR);
              const uint64_t o_at = desc_mn(smem_u32(smem + (far ? SM_S : SM_X))) + right * REST;
#pragma unroll
              for (int ks = 0; ks < Q / 16; ++ks) umma_bf16_ts(to, a_at + ks * 8, o_at + ks * 128, long_idesc(false, 64), (WIDE ? n : p) || ks);
            }
            if (part == ALL - 1) umma_commit(smem_u32(&bars->products));
            if (!WIDE && part == 2 && ci + 1 < chunks) bulk_load(smem + SM_G, img + IMG_G, IMG_BYTES - IMG_G, &bars->scores_full);
          }
          __syncwarp();
        }
      };
      // (a part has 8 instructions of 128 x 64 x 16: parts `from` to `to`)
      auto issue_to = [&](int from, int to) {
#pragma unroll 1
        for (int p = from; p < to; ++p) issue(p);
      };
      constexpr int FIRST = WIDE ? 6 : 3, SECOND = WIDE ? 8 : 4, THIRD = WIDE ? 10 : 5;
      if (WIDE) issue_to(0, Y ? FIRST : NEXTS);
      else { issue(0); issue(1); if (Y) issue(2); }
      // ---- meanwhile: gates of this chunk, steps and convolution of the next one, raw rows of the one behind that
      const bool on = row < range.len, keeps = range.start + range.len == r.keep && r.stores();
      const size_t t = size_t(range.start + (on ? row : 0));
      uint64_t gate[8];
      if (Y) {
        // (a thread's 16 values in one load where they lie on a 32-byte boundary: every load of a warp goes to 32 rows, and takes its time for that)
        const TI* z = rows0 + t * c.ld_x + quarter * 16;
        Word<TI, 2> w[8];
        if (sizeof(TI) == 2 && a.z_vec) {
          uint4 lo, hi;
          ldg_nc_32B(z, lo, hi);
          const uint32_t bits[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
          for (int i = 0; i < 8; ++i) { w[i].v[0] = from_bits<TI>(bits[i]); w[i].v[1] = from_bits<TI>(bits[i] >> 16); }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const Word<TI, 4> four = load_word<VEC, 4>(z + 4 * i);
            w[2 * i].v[0] = four.v[0]; w[2 * i].v[1] = four.v[1];
            w[2 * i + 1].v[0] = four.v[2]; w[2 * i + 1].v[1] = four.v[3];
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          uint64_t one[1];
          widen(w[i], one);
          gate[i] = one[0];
        }
      }
      const int len = range.len;
      if (ci + 1 < chunks) {
        range = chunk_range(r.keep, upto, ci + 1);
        const float now = step;
        convolve(range);
        if (Y) { if (WIDE) issue_to(FIRST, SECOND); else issue(3); }
        if (ci + 2 < chunks) {
          const ChunkRange next = chunk_range(r.keep, upto, ci + 2);
          fetch_x(next);
          step = raw_step(next);
        }
        if (Y) { if (WIDE) issue_to(SECOND, THIRD); else issue(4); }
        if (quarter == 1) make_steps(steps[(k + 1) & 1], now, range.len);
      } else if (Y) {
        if (WIDE) issue_to(FIRST, THIRD);
        else { issue(3); issue(4); }
      }
      if (Y) {
#pragma unroll
        for (int i = 0; i < 8; ++i) gate[i] = silu2(gate[i]);
        if (WIDE) issue_to(THIRD, ALL);
        else { issue(5); issue(6); issue(7); }
      }
      if (warp == 1 && bars->any_odd[(k + 1) & 1]) {           // (the chunk in front of this one has been read)
        bars->first_odd[(k + 1) & 1][lane] = bars->first_odd[(k + 1) & 1][lane + 32] = Q;
        __syncwarp();
        if (lane == 0) bars->any_odd[(k + 1) & 1] = 0;
      }
      if (tid == 0) wait_for(&bars->products, k & 1, bars, c.status, STATUS_TIMEOUT_MMA);
      __syncthreads();
      if (*stop) break;
      if (tid == 0 && ci + 1 < chunks) bulk_load(smem + SM_B, img + IMG_B, 65536, &bars->b_full);
      // ---- what the products gave: outputs
      tc_fence_after();
      const bool any_odd = bars->any_odd[k & 1] != 0;
      const int* first_odd = bars->first_odd[k & 1] + quarter * 16;
      if (Y) {
        uint32_t near[16], state[16];
        tmem_ld16(lanes + TM_NEAR + quarter * 16, near);
        if (!WIDE) tmem_ld16(lanes + TM_STATE + quarter * 16, state);
        const uint64_t ec = dup2(s.ec[row]);
        tmem_wait_ld16(near);
        if (!WIDE) tmem_wait_ld16(state);
        float y[16];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          uint64_t sum = pack_f32x2(__uint_as_float(near[2 * i]), __uint_as_float(near[2 * i + 1]));
          if (!WIDE) sum = fma_f32x2(ec, pack_f32x2(__uint_as_float(state[2 * i]), __uint_as_float(state[2 * i + 1])), sum);
          unpack_f32x2(mul_f32x2(sum, gate[i]), y[2 * i], y[2 * i + 1]);
        }
        if (any_odd) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (row >= first_odd[i]) y[i] = NAN;
        }
        if (on) {
          const size_t to = (size_t(r.q0) + t) * c.ld_y + h * NH + quarter * 16;
          if (!a.y_vec) {                                      // (no 32-byte boundary)
            for (int i = 0; i < 16; ++i) store_row(c.y, c.y_dtype, to + i, y[i], c.status);
          } else if (c.y_dtype == CHUNK_F32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) reinterpret_cast<float4*>(reinterpret_cast<float*>(c.y) + to)[i] = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
          } else {
            uint32_t o[8];
            if (c.y_dtype == CHUNK_BF16) {
#pragma unroll
              for (int i = 0; i < 8; ++i) o[i] = pack_bf16(y[2 * i], y[2 * i + 1]);
            } else {
#pragma unroll
              for (int i = 0; i < 8; ++i) o[i] = pack_f16_sat(y[2 * i], y[2 * i + 1], c.status);
            }
            uint16_t* d = reinterpret_cast<uint16_t*>(c.y) + to;
            asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(d), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]), "r"(o[4]), "r"(o[5]),
                         "r"(o[6]), "r"(o[7]) : "memory");
          }
        }
        __syncwarp();
      }
      // ---- the state
      {
        uint32_t next[16], rest[16];
        tmem_ld16(lanes + TM_NEXT + quarter * 16, next);
        if (!WIDE) tmem_ld16(lanes + TM_NEXT + 64 + quarter * 16, rest);
        const float total = s.total;
        tmem_wait_ld16(next);
        if (!WIDE) tmem_wait_ld16(rest);
#pragma unroll
        for (int i = 0; i < 16; ++i) S[i] = fmaf(total, S[i], WIDE ? __uint_as_float(next[i]) : __uint_as_float(next[i]) + __uint_as_float(rest[i]));
        if (any_odd) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (first_odd[i] < len) S[i] = NAN;
        }
        if (Y && ci + 1 < chunks) put_state();
        if (keeps) {
#pragma unroll
          for (int p = 0; p < 16; ++p) __stcs(mem + p * NS, S[p]);
        }
      }
      tc_fence_before();
    }
    // ---- the carried rows of this head's channels, and of its group's B and C for the group's first head, once everyone has read them
    __syncthreads();
    if (*stop) break;
    const int K1 = c.d_conv - 1;
    if (r.stores() && K1 > 0) {
      const int width = NH + (h % (c.H / c.G) == 0 ? 2 * NS : 0);
      TI* carried = reinterpret_cast<TI*>(c.conv_state) + size_t(r.slot) * K1 * c.d_xBC;
      const TI* rows = reinterpret_cast<const TI*>(c.x) + size_t(r.q0) * c.ld_x + c.Di;
      if (tid < width) {
        const int ch = tid < NH ? h * NH + tid : tid < NH + NS ? c.Di + g * NS + tid - NH : c.Di + (c.G + g) * NS + tid - NH - NS;
        TI old[3];
#pragma unroll
        for (int j = 0; j < 3; ++j) {
          const int from = r.keep + j - K1;
          old[j] = TI(0.f);
          if (j < K1 && (from >= 0 || !r.fresh)) old[j] = from >= 0 ? rows[size_t(from) * c.ld_x + ch] : carried[size_t(from + K1) * c.d_xBC + ch];
        }
#pragma unroll
        for (int j = 0; j < 3; ++j)
          if (j < K1) carried[size_t(j) * c.d_xBC + ch] = old[j];
      }
    }
  }
  // (a copy that was asked for has landed before the block ends)
  tc_fence_before();
  __syncthreads();
  if (*stop && tid == 0) {
    mbar_wait(smem_u32(&bars->b_full), k & 1, 100000000ull);
    if (Y && !WIDE) mbar_wait(smem_u32(&bars->scores_full), k & 1, 100000000ull);
  }
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, 512);
}

template <typename TI, bool VEC, bool WIDE>
cudaError_t launch_vec(const LongArgs& a, cudaStream_t stream) {
  const ChunkScanCall& c = a.c;
  constexpr int PREP = prep_smem(WIDE), LONG = LONG_SMEM<WIDE>;
  static std::atomic<uint32_t> ready{0};                     // devices on which the kernels have been told their shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  // (states alone: nothing is wide)
  auto with = scan_long_kernel<TI, true, VEC, WIDE>, without = scan_long_kernel<TI, WIDE, VEC, WIDE>;
  if (dev >= 32 || !(ready.load() >> dev & 1u)) {
    e = cudaFuncSetAttribute(scan_prep_kernel<TI, VEC, WIDE>, cudaFuncAttributeMaxDynamicSharedMemorySize, PREP);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(with, cudaFuncAttributeMaxDynamicSharedMemorySize, LONG);
    if (e == cudaSuccess && !WIDE) e = cudaFuncSetAttribute(without, cudaFuncAttributeMaxDynamicSharedMemorySize, LONG);
    if (e != cudaSuccess) return e;
    if (dev < 32) ready.fetch_or(1u << dev);
  }
  const long long chunks = (long long)(scan_max_chunks(c.T, c.B)) * c.G, heads = (long long)(scan_max_long(c.T, c.B)) * c.H;
  // (not to start early: its blocks would take the room of those of the kernel in front, which has most of the work where no request has many rows)
  e = launch_behind(scan_prep_kernel<TI, VEC, WIDE>, dim3(unsigned(chunks < 148 ? chunks : 148)), dim3(256), PREP, stream, a);
  if (e != cudaSuccess) return e;
  return launch_pdl(c.y ? with : without, dim3(unsigned(heads < 148 ? heads : 148)), dim3(LONG_THREADS), LONG, stream, a);
}

template <typename TI, bool WIDE>
cudaError_t launch_for(LongArgs a, cudaStream_t stream) {
  const ChunkScanCall& c = a.c;
  auto on = [](const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; };
  const int item = c.y_dtype == CHUNK_F32 ? 4 : 2;
  a.y_vec = c.y && on(c.y, 32) && c.ld_y % (32 / item) == 0 ? 1 : 0;
  a.z_vec = sizeof(TI) == 2 && on(c.x, 32) && c.ld_x % 16 == 0 ? 1 : 0;
  const bool vec = c.d_conv == 4 && c.Di % 4 == 0 && c.ld_x % 4 == 0 && on(c.x, 4 * sizeof(TI)) && on(c.conv_state, 4 * sizeof(TI));
  return vec ? launch_vec<TI, true, WIDE>(a, stream) : launch_vec<TI, false, WIDE>(a, stream);
}

template <bool WIDE>
cudaError_t launch_long(const LongArgs& a, cudaStream_t stream) {
  if (a.c.in_dtype == CHUNK_F32) return launch_for<float, WIDE>(a, stream);
  return a.c.in_dtype == CHUNK_F16 ? launch_for<__half, WIDE>(a, stream) : launch_for<__nv_bfloat16, WIDE>(a, stream);
}

}  // namespace

}  // namespace hspec
