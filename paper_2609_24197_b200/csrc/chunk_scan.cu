// Short causal convolution, selective scan and gate of a ragged chunk of new tokens, from a carried state and back into it.
//
//   u_t = SiLU(b + sum_j w_j raw_{t - K + 1 + j}),  u = x | B | C      raw rows in front of the chunk come from the request's carried ones
//   dt_t = softplus(dt_raw_t + bias),  S_t = exp(-dt_t e^A_log) S_{t-1} + dt_t x_t B_t^T,  y_t = (S_t C_t + D x_t) SiLU(z_t)
//
// Row after row, any shape, two kernels.  scan_rows_kernel convolves the rows into a scratch of 32-bit rows, with their steps and decays; a thread takes four
// channels of some rows, the thread of a request's first rows also moves the carried rows on, which nobody else reads.  scan_state_kernel (scan_few_kernel in
// calls with hardly more rows than requests) carries the states through the rows: a block has some rows of a head's state in registers, from the first token
// to the last, and reads the convolved rows from shared memory, a few tokens ahead of their use.  Single tokens are bound by the state, which is read and
// written once (64 of 160 heads of 64 x 128: 121 us, 5.7 TB/s), long requests with small states by the chain of their rows (100 ns a row; 29 requests of up to
// 700 rows, 8 heads of 64 x 16: 85 us).
// By products, heads of 64 channels with 128 state elements: scan_groups_kernel convolves, sums up the steps and multiplies C with B for requests of up to 32
// rows, which scan_block_kernel finishes; scan_prep_kernel and scan_long_kernel take those with more.  Where these are chosen stands at chunk_scan_launch.
#include "chunk_scan.cuh"

#include <climits>
#include <type_traits>

namespace hspec {

namespace {

constexpr int CONV_THREADS = 256;
constexpr int CONV_TILE = 8;         // rows of a block

struct ConvArgs {
  ChunkScanCall c;
  ScanScratch s;
  int ch_blocks, dt_blocks;          // blocks of an item: channels, then steps
  int32_t *plan, *list, *chunks;     // of the requests with many rows (LongArgs); null: there are none
  int max_long, max_chunks;
};

// The requests that say what cannot be.  One block.
__device__ void count_bad(const ChunkScanCall& c) {
  for (int b = threadIdx.x; b < c.B; b += CONV_THREADS) {
    const ScanRequest r = scan_request(c, b);
    if (chunk_request_bad(c.cu_q[b], c.cu_q[b + 1], INT_MAX, c.T, INT_MAX) || (r.n > 0 && r.slot < 0))
      atomicAdd(c.status + STATUS_WORD_BAD_INPUT, 1u);
  }
}

// The requests with many rows: a list, longest first, and their chunks in the order of the requests.  One block.
constexpr int PLAN_SORT = 1024;
__device__ void plan_long(const ConvArgs& a, int* room) {     // room for 3 PLAN_SORT numbers
  const ChunkScanCall& c = a.c;
  int *key = room, *who = room + PLAN_SORT, *front = room + 2 * PLAN_SORT;
  __shared__ int sums[2][CONV_THREADS / 32], totals[2];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int n_long = 0, n_chunks = 0;
  bool full = false;
  for (int base = 0; base < c.B; base += CONV_THREADS) {
    const int b = base + tid;
    int upto = 0, count = 0;
    if (b < c.B) {
      const ScanRequest r = scan_request(c, b);
      upto = scan_upto(c, r);
      if (upto > a.s.few) count = chunk_count(r.keep, upto);
    }
    const int one = count > 0 ? 1 : 0;
    int i1 = one, i2 = count;                                // sums up to and with this request
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int u1 = __shfl_up_sync(0xffffffffu, i1, off), u2 = __shfl_up_sync(0xffffffffu, i2, off);
      if (lane >= off) { i1 += u1; i2 += u2; }
    }
    if (lane == 31) { sums[0][warp] = i1; sums[1][warp] = i2; }
    __syncthreads();
    for (int w = 0; w < warp; ++w) { i1 += sums[0][w]; i2 += sums[1][w]; }
    i1 += n_long;
    i2 += n_chunks;
    // (offsets that do not ascend could ask for more than there is room for: these requests are left out, and counted)
    const bool fits = i1 <= a.max_long && i2 <= a.max_chunks && !full;
    if (one && !fits) atomicAdd(c.status + STATUS_WORD_BAD_INPUT, 1u);
    if (one && fits) {
      const int at = i1 - 1, first = i2 - count;
      if (at < PLAN_SORT) { key[at] = upto; who[at] = b; front[at] = first; }
      a.list[2 * at] = b;
      a.list[2 * at + 1] = first;
      for (int j = 0; j < count; ++j) {
        a.chunks[2 * (first + j)] = b;
        a.chunks[2 * (first + j) + 1] = j;
      }
    }
    // the last one that fits ends the sums
    if (tid == 0) { totals[0] = n_long; totals[1] = n_chunks; }
    __syncthreads();
    if (fits) { atomicMax(&totals[0], i1); atomicMax(&totals[1], i2); }
    full = __syncthreads_or(one && !fits) || full;
    n_long = totals[0];
    n_chunks = totals[1];
    __syncthreads();
  }
  if (n_long <= PLAN_SORT)
    for (int i = tid; i < n_long; i += CONV_THREADS) {
      int rank = 0;
      for (int j = 0; j < n_long; ++j) rank += key[j] > key[i] || (key[j] == key[i] && j < i);
      a.list[2 * rank] = who[i];
      a.list[2 * rank + 1] = front[i];
    }
  if (tid == 0) {
    a.plan[0] = n_long;
    a.plan[1] = n_chunks;
  }
}

// A word of W row values, widened.
template <typename T, int W>
__device__ __forceinline__ void load_wide(const T* p, float (&x)[W]) {
  const Word<T, W> w = *reinterpret_cast<const Word<T, W>*>(p);
#pragma unroll
  for (int e = 0; e < W; ++e) x[e] = to_f32(w.v[e]);
}

template <typename TI, int W, int K>
__global__ void __launch_bounds__(CONV_THREADS) scan_rows_kernel(ConvArgs a) {
  const ChunkScanCall& c = a.c;
  pdl_wait();
  // (the next kernel does not start early: its blocks would take the room of this one's, 29 requests of up to 700 rows 104 us instead of 84)
  const int tid = threadIdx.x, blocks = a.ch_blocks + a.dt_blocks, part = (blockIdx.x - 1) % blocks;
  if (blockIdx.x == 0) {
    extern __shared__ __align__(16) int plan_room[];
    count_bad(c);
    if (a.plan) plan_long(a, plan_room);
    return;
  }
  // (a request without rows has an item too, for its carried ones; one with many rows goes another way altogether)
  const ChunkItem item = chunk_item(c.B, CONV_TILE, 1, (blockIdx.x - 1) / blocks, tid & 31, [&](int b) {
    const ScanRequest r = scan_request(c, b);
    const int n = scan_upto(c, r);
    return ChunkRows{r.q0, n > a.s.few ? -1 : n};
  });
  if (item.b < 0) return;
  const int rows = min(CONV_TILE, item.n - item.first), t0 = item.q0 + item.first;
  const size_t out0 = a.s.row(item.b, item.q0, item.first);
  if (part >= a.ch_blocks) {
    // ---- steps and decays
    const int i = (part - a.ch_blocks) * CONV_THREADS + tid, h = i % c.H, r = i / c.H;
    if (r < rows) {
      const size_t t = t0 + r;
      const float raw = c.dt_raw ? c.dt_raw[t * c.H + h] : to_f32(reinterpret_cast<const TI*>(c.x)[t * c.ld_x + c.Di + c.d_xBC + h]);
      const float dt = softplus_f32(raw + c.dt_bias[h]);
      const float fall = -dt * expf(c.A_log[h]), less = expm1f(fall);
      const float decay = less > -0.5f ? 1.f + less : expf(fall);            // (what falls by half in a row does not add up errors)
      a.s.step[(out0 + r) * c.H + h] = make_float4(dt, decay, less > -0.5f ? less - (decay - 1.f) : 0.f, 0.f);
    }
    return;
  }
  const ScanRequest r = scan_request(c, item.b);
  const int ch = (part * CONV_THREADS + tid) * W;
  if (ch >= c.d_xBC) return;
  float w[K][W], bias[W], raw[K - 1 + CONV_TILE][W];
  // (a thread's weights are W rows of K)
#pragma unroll
  for (int e = 0; e < W; ++e) {
    bias[e] = c.conv_b[ch + e];
#pragma unroll
    for (int j = 0; j < K; ++j) w[j][e] = c.conv_w[size_t(ch + e) * K + j];
  }
  TI* carried = reinterpret_cast<TI*>(c.conv_state) + (r.slot < 0 ? 0 : size_t(r.slot) * (K - 1) * c.d_xBC) + ch;
  const TI* src = reinterpret_cast<const TI*>(c.x) + size_t(t0) * c.ld_x + c.Di + ch;
  if (item.first == 0) {
    using V = Word<TI, W>;
    V old[K - 1 > 0 ? K - 1 : 1];
#pragma unroll
    for (int j = 0; j < K - 1; ++j) {
      if (r.fresh) old[j] = V{};
      else old[j] = *reinterpret_cast<const V*>(carried + size_t(j) * c.d_xBC);
#pragma unroll
      for (int e = 0; e < W; ++e) raw[j][e] = to_f32(old[j].v[e]);
    }
    if (r.stores()) {
#pragma unroll
      for (int j = 0; j < K - 1; ++j) {
        const int from = r.keep + j - (K - 1);             // the chunk's row that comes to place j; below zero: a carried one
        V v{};
        if (from >= 0) {
          v = *reinterpret_cast<const V*>(src + size_t(from) * c.ld_x);
        } else {
#pragma unroll
          for (int o = 0; o < K - 1; ++o)
            if (o == r.keep + j) v = old[o];
        }
        *reinterpret_cast<V*>(carried + size_t(j) * c.d_xBC) = v;
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < K - 1; ++j) load_wide<TI, W>(src + (j - (K - 1)) * (long long)(c.ld_x), raw[j]);
  }
#pragma unroll
  for (int i = 0; i < CONV_TILE; ++i)
    if (i < rows) load_wide<TI, W>(src + size_t(i) * c.ld_x, raw[K - 1 + i]);
#pragma unroll
  for (int i = 0; i < CONV_TILE; ++i) {
    if (i >= rows) break;
    Word<float, W> out;
#pragma unroll
    for (int e = 0; e < W; ++e) {
      float v = bias[e];
#pragma unroll
      for (int j = 0; j < K; ++j) v = fmaf(w[j][e], raw[i + j][e], v);
      out.v[e] = silu_f32(v);
    }
    *reinterpret_cast<Word<float, W>*>(a.s.xbc + (out0 + i) * a.s.pitch + ch) = out;
  }
}

// B and C of a group, for a request with up to SCAN_FEW rows (N = 128): a thread a channel.  B goes into the scratch as it is, C in its bf16 parts; their
// products by pairs of rows.
constexpr int CB_PITCH = 128 + 4;
// x of a request with few rows: a thread two channels.
template <typename TI, int K, bool VEC>
__device__ void x_of_request(const ConvArgs& a, int b, int ch) {
  const ChunkScanCall& c = a.c;
  const ScanRequest r = scan_request(c, b);
  const int n = scan_upto(c, r);
  constexpr int K1 = K - 1;
  if (n > a.s.few || ch >= c.Di || (n == 0 && !r.stores())) return;
  const RawRows<VEC, 2, TI> raw(c, r, ch);
  Taps<1, K> taps;
  taps.load(c, ch);
  Word<TI, 2> front[3] = {};
  uint64_t before[3][1];
  if (n > 0) {
    raw.front(front, 0, n - 1);
    raw.front_value(front, 0, before);
  }
  if (r.stores()) {
    TI* carried = reinterpret_cast<TI*>(c.conv_state) + size_t(r.slot) * K1 * c.d_xBC + ch;
    for (int j = 0; j < K1; ++j) {
      const int from = r.keep + j - K1;                      // the row that comes to place j; below zero: a carried one (front: rows -3 .. -1)
      Word<TI, 2> v = from == -3 ? front[0] : from == -2 ? front[1] : front[2];
      if (from >= 0) v = raw.row(from, n - 1);
      else if (r.fresh) v = Word<TI, 2>{};
      carried[size_t(j) * c.d_xBC] = v.v[0];
      carried[size_t(j) * c.d_xBC + 1] = v.v[1];
    }
  }
  for (int i0 = 0; i0 < n; i0 += 8) {
    Word<TI, 2> rows[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rows[i] = raw.row(i0 + i, n - 1);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i0 + i >= n) break;
      uint64_t now[1], v[1];
      widen(rows[i], now);
      taps.next(before, now, v);
      *reinterpret_cast<uint64_t*>(a.s.xbc + a.s.row(b, r.q0, i0 + i) * a.s.pitch + ch) = v[0];
    }
  }
}

// The steps of a request with few rows: a thread a head.  The log-decays' sums are 64-bit and stored in two parts.
template <typename TI>
__device__ void steps_of_request(const ConvArgs& a, int b) {
  const ChunkScanCall& c = a.c;
  const ScanRequest r = scan_request(c, b);
  const int n = scan_upto(c, r);
  if (n > a.s.few) return;
  for (int h = threadIdx.x; h < c.H; h += CONV_THREADS) {
    const float bias = c.dt_bias[h];
    const double rate = double(-expf(c.A_log[h]));
    double sum = 0.0;
    for (int i0 = 0; i0 < n; i0 += 8) {
      float in[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const size_t t = size_t(r.q0) + min(i0 + i, n - 1);
        in[i] = c.dt_raw ? c.dt_raw[t * c.H + h] : to_f32(reinterpret_cast<const TI*>(c.x)[t * c.ld_x + c.Di + c.d_xBC + h]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (i0 + i >= n) break;
        const float dt = softplus_f32(in[i] + bias);
        sum += double(dt) * rate;
        const float hi = float(sum);
        a.s.sums[a.s.row(b, r.q0, i0 + i) * c.H + h] = make_float4(dt, expf(hi), hi, float(sum - double(hi)));
      }
    }
  }
}

template <typename TI, int K, bool VEC>
__global__ void __launch_bounds__(CONV_THREADS) scan_groups_kernel(ConvArgs a) {
  const ChunkScanCall& c = a.c;
  pdl_wait();
  // (nor does the next one here: 17 rows of 32 requests 94 us with an early start, 82 without)
  extern __shared__ __align__(16) float rows_sm[];           // B, then C: [SCAN_FEW][CB_PITCH] each
  if (blockIdx.x == 0) {
    count_bad(c);
    if (a.plan) plan_long(a, reinterpret_cast<int*>(rows_sm));
    return;
  }
  // (a request's blocks: its groups, its steps, 512 channels of x each)
  const int x_blocks = (c.Di + 2 * CONV_THREADS - 1) / (2 * CONV_THREADS), each = c.G + 1 + x_blocks;
  const int b = (blockIdx.x - 1) / each, g = (blockIdx.x - 1) % each;
  if (g > c.G) { x_of_request<TI, K, VEC>(a, b, (g - c.G - 1) * 2 * CONV_THREADS + 2 * threadIdx.x); return; }
  if (g == c.G) { steps_of_request<TI>(a, b); return; }
  const ScanRequest r = scan_request(c, b);
  const int n = scan_upto(c, r), tid = threadIdx.x, e = tid & 127;
  const bool isC = tid >= 128, wide = scan_wide(c);
  if (n > a.s.few || (n == 0 && !r.stores())) return;
  const int ch = c.Di + ((isC ? c.G : 0) + g) * 128 + e;
  float w[K], raw[K];
  const float bias = c.conv_b[ch];
#pragma unroll
  for (int j = 0; j < K; ++j) w[j] = c.conv_w[size_t(ch) * K + j];
  TI* carried = reinterpret_cast<TI*>(c.conv_state) + (r.slot < 0 ? 0 : size_t(r.slot) * (K - 1) * c.d_xBC) + ch;
  const TI* src = reinterpret_cast<const TI*>(c.x) + size_t(r.q0) * c.ld_x + c.Di + ch;
  TI old[K];
#pragma unroll
  for (int j = 0; j < K - 1; ++j) {
    old[j] = r.fresh ? TI(0.f) : carried[size_t(j) * c.d_xBC];
    raw[j] = to_f32(old[j]);
  }
  if (r.stores()) {
#pragma unroll
    for (int j = 0; j < K - 1; ++j) {
      const int from = r.keep + j - (K - 1);
      TI v = TI(0.f);
      if (from >= 0) v = src[size_t(from) * c.ld_x];
#pragma unroll
      for (int o = 0; o < K - 1; ++o)
        if (from < 0 && o == r.keep + j) v = old[o];
      carried[size_t(j) * c.d_xBC] = v;
    }
  }
  for (int i0 = 0; i0 < n; i0 += 8) {
    TI next[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) next[i] = src[size_t(min(i0 + i, n - 1)) * c.ld_x];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i0 + i >= n) break;
      raw[K - 1] = to_f32(next[i]);
      float v = bias;
#pragma unroll
      for (int j = 0; j < K; ++j) v = fmaf(w[j], raw[j], v);
#pragma unroll
      for (int j = 0; j < K - 1; ++j) raw[j] = raw[j + 1];
      v = silu_f32(v);
      rows_sm[((isC ? SCAN_FEW : 0) + i0 + i) * CB_PITCH + e] = v;
      const size_t row = a.s.row(b, r.q0, i0 + i);
      if (isC) {
        __nv_bfloat16* parts = reinterpret_cast<__nv_bfloat16*>(a.s.c_parts) + (row * c.G + g) * (SCAN_C_PARTS * 128) + e;
#pragma unroll
        for (int p = 0; p < SCAN_C_PARTS; ++p) {
          if (p == 2 && !wide) break;
          const __nv_bfloat16 part = parts[p * 128] = __float2bfloat16_rn(v);
          v -= __bfloat162float(part);
        }
      } else {
        a.s.xbc[row * a.s.pitch + ch] = v;
      }
    }
  }
  if (!c.y) return;
  __syncthreads();
  for (int pair = tid; pair < n * n; pair += CONV_THREADS) {
    const int t = pair / n, s = pair % n;
    if (s > t) continue;
    const float4* ct = reinterpret_cast<const float4*>(rows_sm + (SCAN_FEW + t) * CB_PITCH);
    const float4* bs = reinterpret_cast<const float4*>(rows_sm + s * CB_PITCH);
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int i = 0; i < 32; ++i) {
      const float4 x = ct[i], y = bs[i];
      sum.x = fmaf(x.x, y.x, sum.x); sum.y = fmaf(x.y, y.y, sum.y); sum.z = fmaf(x.z, y.z, sum.z); sum.w = fmaf(x.w, y.w, sum.w);
    }
    a.s.cb[((size_t(b) * c.G + g) * SCAN_FEW + t) * SCAN_FEW + s] = (sum.x + sum.y) + (sum.z + sum.w);
  }
}

// ---------------------------------------------------------------------------------------------------
// The states through the rows.  A group of L lanes has PR rows of a head's state [P, N]: lane l of the group the elements n = 4 (l + L k) .. + 3.
// Decays are next to one, and there may be thousands of rows.  So a decay comes in two parts, and (CARRY) what a row's rounding leaves out of the state is
// carried to the next: otherwise both add up, in one direction where rows are alike (8000 equal rows: 4e-4 of the sum of all that entered, so 1e-6).  It
// costs 1 % where the chain of rows bounds (29 requests of up to 700 rows 84 -> 85 us), and 13 % for blocks (17 rows of 32 requests, 24 heads of 40 x 24: 31 ->
// 35).  Requests of up to STATE_FEW rows go without in calls with hardly more rows than requests: the registers are those of their loads (64 tokens of 160
// heads of 64 x 128 121 us; 145 with the rest carried).
constexpr int STATE_THREADS = 128, STATE_FEW = 8;

__host__ __device__ constexpr int state_tile(int pr, int npt) { return pr * npt <= 8 ? 32 : 8; }
template <typename TI, int L, int PR, int NPT, bool VECN, bool Y, bool CARRY>
__device__ __forceinline__ void scan_state(const StateArgs& a, const ScanRequest& r, const int upto, const int h, const int b, const int p0, const int p_block) {
  constexpr bool SMALL = PR * NPT <= 8;                      // few elements a thread: the rows' operands and gates are fetched far ahead
  constexpr int TILE = state_tile(PR, NPT);                  // tokens that are fetched together
  constexpr int NP = L * NPT;                                // N is not above it
  constexpr int B_AT = 4, C_AT = B_AT + NP, X_AT = C_AT + NP;          // of a row in shared memory: dt, decay, its rest | B | C | x
  constexpr int DUP = L / PR;                                // lanes that end up with the same row's sum
  constexpr int ROWS = (TILE + DUP - 1) / DUP;               // tokens of a tile whose outputs a lane finishes
  const ChunkScanCall& c = a.c;
  const int tid = threadIdx.x, l = tid % L, g = h / (c.H / c.G);
  const int pt = p0 + tid / L * PR;                          // the thread's first row (p0: the block's, p_block: as many)
  uint64_t S[PR][NPT / 2], rest[CARRY ? PR : 1][CARRY ? NPT / 2 : 1] = {};         // the state, and what its rounding has left out so far
  float* state = c.ssm_state + ((size_t(r.slot < 0 ? 0 : r.slot) * c.H + h) * c.P + pt) * c.N;
#pragma unroll
  for (int i = 0; i < PR; ++i) {
#pragma unroll
    for (int k = 0; k < NPT / 4; ++k) {
      const int n = 4 * (l + L * k);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (!r.fresh && (upto > 0) && pt + i < c.P && n < c.N) {
        const float* p = state + size_t(i) * c.N + n;
        if (VECN) v = __ldcs(reinterpret_cast<const float4*>(p));
        else {
          v.x = p[0];
          if (n + 1 < c.N) v.y = p[1];
          if (n + 2 < c.N) v.z = p[2];
          if (n + 3 < c.N) v.w = p[3];
        }
      }
      S[i][2 * k] = pack_f32x2(v.x, v.y);
      S[i][2 * k + 1] = pack_f32x2(v.z, v.w);
    }
  }
  pdl_wait();
  pdl_trigger();
  if (upto == 0 && !r.stores()) return;
  auto store = [&] {
#pragma unroll
    for (int i = 0; i < PR; ++i) {
#pragma unroll
      for (int k = 0; k < NPT / 4; ++k) {
        const int n = 4 * (l + L * k);
        if (pt + i >= c.P || n >= c.N) continue;
        float4 v;
        uint64_t lo = S[i][2 * k], hi = S[i][2 * k + 1];
        if constexpr (CARRY) { lo = add_f32x2(lo, rest[i][2 * k]); hi = add_f32x2(hi, rest[i][2 * k + 1]); }
        unpack_f32x2(lo, v.x, v.y);
        unpack_f32x2(hi, v.z, v.w);
        float* p = state + size_t(i) * c.N + n;
        if (VECN) __stcs(reinterpret_cast<float4*>(p), v);
        else {
          p[0] = v.x;
          if (n + 1 < c.N) p[1] = v.y;
          if (n + 2 < c.N) p[2] = v.z;
          if (n + 3 < c.N) p[3] = v.w;
        }
      }
    }
  };
  if (r.keep == 0 && r.stores()) store();                    // a fresh request of which nothing is kept: zeros
  if (upto == 0) return;

  const size_t at0 = a.s.row(b, r.q0, 0);
  extern __shared__ __align__(16) float sm[];
  const int per = X_AT + (p_block + 3) / 4 * 4, stage = per * TILE;
  if (c.N < NP || c.P - p0 < p_block) {                      // what lies behind N and P stays zero
    for (int i = tid; i < 2 * stage; i += blockDim.x) sm[i] = 0.f;
    __syncthreads();
  }
  // fetches tokens first .. first + TILE - 1 of the request into a stage
  auto fetch = [&](int first, int buf) {
    const int count = min(TILE, upto - first);
    float* dst = sm + buf * stage;
    const float* rows = a.s.xbc + (at0 + first) * a.s.pitch;
    const int xn = min(p_block, c.P - p0);
    // (a thread's elements lie blockDim apart: a step forward in the rows and in the row)
    if (VECN && c.P % 4 == 0) {
      const int nv = c.N / 4, all = 2 * nv + xn / 4, step = blockDim.x % all, down = blockDim.x / all;
      for (int row = tid / all, e = tid % all; row < count; row += down, e += step) {
        if (e >= all) {
          e -= all;
          if (++row >= count) break;
        }
        const int from = e < nv ? c.Di + g * c.N + 4 * e : e < 2 * nv ? c.Di + (c.G + g) * c.N + 4 * (e - nv) : h * c.P + p0 + 4 * (e - 2 * nv);
        const int to = e < nv ? B_AT + 4 * e : e < 2 * nv ? C_AT + 4 * (e - nv) : X_AT + 4 * (e - 2 * nv);
        cp_async16(smem_u32(dst + row * per + to), rows + size_t(row) * a.s.pitch + from, true);
      }
    } else {
      const int all = 2 * c.N + xn, step = blockDim.x % all, down = blockDim.x / all;
      for (int row = tid / all, e = tid % all; row < count; row += down, e += step) {
        if (e >= all) {
          e -= all;
          if (++row >= count) break;
        }
        const int from = e < c.N ? c.Di + g * c.N + e : e < 2 * c.N ? c.Di + (c.G + g) * c.N + e - c.N : h * c.P + p0 + e - 2 * c.N;
        const int to = e < c.N ? B_AT + e : e < 2 * c.N ? C_AT + e - c.N : X_AT + e - 2 * c.N;
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(dst + row * per + to)), "l"(rows + size_t(row) * a.s.pitch + from) : "memory");
      }
    }
    if (tid < count)
      cp_async16(smem_u32(dst + tid * per), a.s.step + (at0 + first + tid) * c.H + h, true);
    cp_async_commit();
  };
  // the row of the state whose output the lane finishes, and its place among the lanes that do
  const int mine = l / DUP, dup = l % DUP, pm = pt + mine;
  const TI* z = reinterpret_cast<const TI*>(c.x) + size_t(r.q0) * c.ld_x + h * c.P + pm;
  const float D = Y && pm < c.P ? c.Dskip[h] : 0.f;
  // small states: the tile's gates, row by row, through registers into shared memory a tile ahead
  constexpr int GATES = SMALL ? TILE * PR / L : 1;
  float* gates = sm + 2 * stage;                             // [2][TILE][p_block]
  float ahead[GATES];
  const int gate_row = tid / p_block, gate_p = p0 + tid % p_block, gate_rows = L / PR;       // (blockDim / p_block of them a step)
  auto fetch_gates = [&](int first) {
    const int count = gate_p < c.P ? min(TILE, upto - first) : 0;
    const TI* from = reinterpret_cast<const TI*>(c.x) + size_t(r.q0 + first + gate_row) * c.ld_x + h * c.P + gate_p;
#pragma unroll
    for (int i = 0; i < GATES; ++i) ahead[i] = gate_row + i * gate_rows < count ? to_f32(from[size_t(i * gate_rows) * c.ld_x]) : 0.f;
  };
  auto put_gates = [&](int buf) {
#pragma unroll
    for (int i = 0; i < GATES; ++i) gates[buf * TILE * p_block + tid + i * blockDim.x] = silu_f32(ahead[i]);
  };
  fetch(0, 0);
  if (SMALL && Y) {
    fetch_gates(0);
    put_gates(0);
  }
  for (int first = 0, buf = 0; first < upto; first += TILE, buf ^= 1) {
    const int count = min(TILE, upto - first);
    float gate[ROWS];                                        // (of a tile's rows that this lane finishes)
    if (Y && !SMALL) {
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const int row = i * DUP + dup;
        gate[i] = row < count && pm < c.P ? to_f32(z[size_t(first + row) * c.ld_x]) : 0.f;
      }
    }
    if (SMALL && Y && first + TILE < upto) fetch_gates(first + TILE);
    if (first + TILE < upto) fetch(first + TILE, buf ^ 1);
    else cp_async_commit();
    cp_async_wait<1>();
    __syncthreads();
    const float* rows = sm + buf * stage;
    // a row's addition to the state; the sum of this lane's row of the state with C
    auto add = [&](int row) {
      const float* now = rows + row * per;
      const float4 step = *reinterpret_cast<const float4*>(now);
      const uint64_t decay = dup2(step.y), decay_rest = dup2(step.z), minus = dup2(-step.y);
      uint64_t xd[PR], y2[PR];
#pragma unroll
      for (int i = 0; i < PR; ++i) {
        const float x = now[X_AT + (pt - p0) + i];
        xd[i] = pack_f32x2(step.x * x, step.x * x);
        y2[i] = 0ull;
      }
#pragma unroll
      for (int k = 0; k < NPT / 4; ++k) {
        const ulonglong2 Bv = *reinterpret_cast<const ulonglong2*>(now + B_AT + 4 * (l + L * k));
        ulonglong2 Cv;
        if (Y) Cv = *reinterpret_cast<const ulonglong2*>(now + C_AT + 4 * (l + L * k));
#pragma unroll
        for (int i = 0; i < PR; ++i) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint64_t s = S[i][2 * k + e], more = fma_f32x2(decay_rest, s, mul_f32x2(xd[i], e ? Bv.y : Bv.x));
            if constexpr (CARRY) {
              const uint64_t all = fma_f32x2(decay, rest[i][2 * k + e], more), next = fma_f32x2(decay, s, all);
              rest[i][2 * k + e] = fma_f32x2(fma_f32x2(minus, s, next), dup2(-1.f), all);
              S[i][2 * k + e] = next;
            } else {
              S[i][2 * k + e] = fma_f32x2(decay, s, more);
            }
          }
          if (Y) {
            y2[i] = fma_f32x2(S[i][2 * k], Cv.x, y2[i]);
            y2[i] = fma_f32x2(S[i][2 * k + 1], Cv.y, y2[i]);
          }
        }
      }
      float sum = 0.f;
      if (Y) {
        // the group's sums: every step hands half of the rows to the partner, until a lane has one
        float v[PR];
#pragma unroll
        for (int i = 0; i < PR; ++i) {
          float lo, hi;
          unpack_f32x2(y2[i], lo, hi);
          v[i] = lo + hi;
        }
#pragma unroll
        for (int half = PR / 2, off = L / 2; off >= 1; off /= 2, half /= 2) {
          if (half >= 1) {
            const bool up = (l & off) != 0;
#pragma unroll
            for (int i = 0; i < PR / 2; ++i) {
              if (i >= half) break;
              const float got = __shfl_xor_sync(0xffffffffu, up ? v[i] : v[i + half], off);
              v[i] = (up ? v[i + half] : v[i]) + got;
            }
          } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], off);
          }
        }
        sum = v[0];
      }
      return sum;
    };
    auto finish = [&](int row, float sum) {
      if (pm >= c.P) return;
      float g;
      if constexpr (SMALL) g = gates[(buf * TILE + row) * p_block + pm - p0];
      else g = silu_f32(gate[row / DUP]);
      store_row(c.y, c.y_dtype, size_t(r.q0 + first + row) * c.ld_y + h * c.P + pm, fmaf(D, rows[row * per + X_AT + pm - p0], sum) * g, c.status);
    };
    auto one = [&](int row) {
      const float sum = add(row);
      if (Y && row % DUP == dup) finish(row, sum);
    };
    if constexpr (SMALL) {
      // Eight rows in a row, so that the next ones' operands and the last ones' sums are under way beside the one thing that has to wait, an addition to
      // the state a row.
#pragma unroll 1
      for (int r0 = 0; r0 < count; r0 += 8) {
        const bool inside = r.stores() && r.keep > first + r0 && r.keep < first + r0 + 8;        // the state is stored among them
        if (r0 + 8 <= count && !inside) {
          constexpr int MINE = (8 + DUP - 1) / DUP;          // of the eight that this lane finishes
          float sums[MINE];
#pragma unroll
          for (int row = 0; row < 8; ++row) {
            const float sum = add(r0 + row);
            if (row % DUP == 0) sums[row / DUP] = sum;
            else sums[row / DUP] = row % DUP == dup ? sum : sums[row / DUP];
          }
          if (Y) {
#pragma unroll
            for (int i = 0; i < MINE; ++i)
              if (DUP <= 8 || dup < 8) finish(r0 + i * DUP + dup, sums[i]);
          }
          if (first + r0 + 8 == r.keep && r.stores()) store();
        } else {
#pragma unroll 1
          for (int row = r0; row < min(r0 + 8, count); ++row) {
            one(row);
            if (first + row + 1 == r.keep && r.stores()) store();
          }
        }
      }
      if (Y && first + TILE < upto) put_gates(buf ^ 1);
    } else {
      auto step = [&](int row) {
        one(row);
        if (first + row + 1 == r.keep && r.stores()) store();
      };
      if constexpr (CARRY) {                                 // (all eight mixed take more registers than there are)
#pragma unroll 4
        for (int row = 0; row < TILE; ++row) {
          if (row >= count) break;
          step(row);
        }
      } else {
#pragma unroll
        for (int row = 0; row < TILE; ++row) {
          if (row >= count) break;
          step(row);
        }
      }
    }
    __syncthreads();
  }
}

template <typename TI, int L, int PR, int NPT, bool VECN, bool Y>
__global__ void __launch_bounds__(STATE_THREADS, NPT == 16 ? 3 : 5) scan_state_kernel(StateArgs a) {
  const int h = blockIdx.x / a.p_blocks, b = blockIdx.y, p0 = blockIdx.x % a.p_blocks * a.p_block;
  // (before the wait only what is at least two kernels back is read: the arrays that describe the chunk, and the states)
  const ScanRequest r = scan_request(a.c, b);
  scan_state<TI, L, PR, NPT, VECN, Y, true>(a, r, scan_upto(a.c, r), h, b, p0, a.p_block);
}
// The same for calls with hardly more rows than requests.  (A request that has many of them all the same goes through half of the block's part at a time,
// where a thread has many elements.)
template <typename TI, int L, int PR, int NPT, bool VECN, bool Y>
__global__ void __launch_bounds__(STATE_THREADS) scan_few_kernel(StateArgs a) {
  const int h = blockIdx.x / a.p_blocks, b = blockIdx.y, p0 = blockIdx.x % a.p_blocks * a.p_block;
  const ScanRequest r = scan_request(a.c, b);
  const int upto = scan_upto(a.c, r);
  if (upto > a.s.few) {
    pdl_wait();
  } else if (upto <= STATE_FEW) {
    scan_state<TI, L, PR, NPT, VECN, Y, false>(a, r, upto, h, b, p0, a.p_block);
  } else if constexpr (PR == 1) {
    scan_state<TI, L, PR, NPT, VECN, Y, true>(a, r, upto, h, b, p0, a.p_block);
  } else {
#pragma unroll 1
    for (int half = 0; half < a.p_block && p0 + half < a.c.P; half += a.p_block / 2)
      scan_state<TI, L, PR / 2, NPT, VECN, Y, true>(a, r, upto, h, b, p0 + half, a.p_block / 2);
  }
}

template <typename TI, int L, int PR, int NPT, bool CARRY>
cudaError_t launch_state(StateArgs a, cudaStream_t stream) {
  const ChunkScanCall& c = a.c;
  // (at most 64 rows of the state where a lane has one of them: x and the gates of more, 32 tokens twice, would not fit)
  constexpr int MOST = L == 1 ? 64 : STATE_THREADS / L;
  constexpr auto smem_of = [](int p_block) {
    return size_t(2) * state_tile(PR, NPT) * (4 + 2 * L * NPT + (p_block + 3) / 4 * 4 + (PR * NPT <= 8 ? p_block : 0)) * 4;
  };
  static_assert(smem_of(MOST * PR) <= 48 * 1024, "more shared memory than a kernel has without asking: the launch would fail behind the rows' kernel");
  int groups = MOST;
  while (groups * L > 32 && (groups / 2) * PR >= c.P) groups /= 2;
  a.p_block = groups * PR;
  a.p_blocks = (c.P + a.p_block - 1) / a.p_block;
  const size_t smem = smem_of(a.p_block);
  const bool vec = c.N % 4 == 0 && c.Di % 4 == 0;
  const dim3 grid(unsigned(c.H * a.p_blocks), unsigned(c.B));
  auto go = [&](auto kernel) { return launch_pdl(kernel, grid, dim3(unsigned(groups * L)), smem, stream, a); };
  auto pick = [&](auto with, auto without) { return c.y ? go(with) : go(without); };
  if constexpr (CARRY)
    return vec ? pick(scan_state_kernel<TI, L, PR, NPT, true, true>, scan_state_kernel<TI, L, PR, NPT, true, false>)
               : pick(scan_state_kernel<TI, L, PR, NPT, false, true>, scan_state_kernel<TI, L, PR, NPT, false, false>);
  else
    return vec ? pick(scan_few_kernel<TI, L, PR, NPT, true, true>, scan_few_kernel<TI, L, PR, NPT, true, false>)
               : pick(scan_few_kernel<TI, L, PR, NPT, false, true>, scan_few_kernel<TI, L, PR, NPT, false, false>);
}

template <typename TI, bool CARRY>
cudaError_t launch_states(const StateArgs& a, cudaStream_t stream) {
  const int N = a.c.N;
  constexpr int PR = CARRY ? 2 : 4;                          // (64 elements a thread, or 32 and what their roundings left out)
  if (N <= 4) return launch_state<TI, 1, 1, 4, CARRY>(a, stream);
  if (N <= 16) return launch_state<TI, 4, 1, 4, CARRY>(a, stream);
  if (N <= 32) return launch_state<TI, 8, 1, 4, CARRY>(a, stream);
  if (N <= 64) return launch_state<TI, 8, 1, 8, CARRY>(a, stream);
  if (N <= 128) return launch_state<TI, 8, PR, 16, CARRY>(a, stream);
  return launch_state<TI, 16, PR, 16, CARRY>(a, stream);
}

template <typename TI, int W, int K>
cudaError_t launch_rows_k(const ConvArgs& a, unsigned blocks, cudaStream_t stream) {
  return launch_pdl(scan_rows_kernel<TI, W, K>, dim3(blocks), dim3(CONV_THREADS), a.plan ? 3 * PLAN_SORT * sizeof(int) : 0, stream, a);
}
template <typename TI, int W>
cudaError_t launch_rows_w(const ConvArgs& a, unsigned blocks, cudaStream_t stream) {
  switch (a.c.d_conv) {
    case 1: return launch_rows_k<TI, W, 1>(a, blocks, stream);
    case 2: return launch_rows_k<TI, W, 2>(a, blocks, stream);
    case 3: return launch_rows_k<TI, W, 3>(a, blocks, stream);
    default: return launch_rows_k<TI, W, 4>(a, blocks, stream);
  }
}

template <typename TI, int K>
cudaError_t launch_groups_k(const ConvArgs& a, cudaStream_t stream) {
  const ChunkScanCall& c = a.c;
  const long long blocks = 1 + (long long)(c.B) * (c.G + 1 + (c.Di + 2 * CONV_THREADS - 1) / (2 * CONV_THREADS));
  if (blocks > INT_MAX) return cudaErrorInvalidConfiguration;
  auto on = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % (2 * sizeof(TI)) == 0; };
  const bool vec = c.ld_x % 2 == 0 && on(c.x) && on(c.conv_state);
  return launch_pdl(vec ? scan_groups_kernel<TI, K, true> : scan_groups_kernel<TI, K, false>, dim3(unsigned(blocks)), dim3(CONV_THREADS),
                    size_t(2) * SCAN_FEW * CB_PITCH * 4, stream, a);
}
template <typename TI>
cudaError_t launch_groups(const ConvArgs& a, cudaStream_t stream) {
  switch (a.c.d_conv) {
    case 1: return launch_groups_k<TI, 1>(a, stream);
    case 2: return launch_groups_k<TI, 2>(a, stream);
    case 3: return launch_groups_k<TI, 3>(a, stream);
    default: return launch_groups_k<TI, 4>(a, stream);
  }
}

template <typename TI>
cudaError_t launch_all(ConvArgs a, cudaStream_t stream) {
  const ChunkScanCall& c = a.c;
  if (a.s.c_parts) {
    const cudaError_t e = launch_groups<TI>(a, stream);
    StateArgs s{};
    s.c = c;
    s.s = a.s;
    return e != cudaSuccess ? e : scan_block_launch(s, stream);
  }
  // words of four row values, where all rows and both parts of a row start on their boundaries
  auto aligned = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % (4 * sizeof(TI)) == 0; };
  const bool wide = c.Di % 4 == 0 && c.d_xBC % 4 == 0 && c.ld_x % 4 == 0 && aligned(c.x) && aligned(c.conv_state);
  a.ch_blocks = (c.d_xBC + CONV_THREADS * (wide ? 4 : 1) - 1) / (CONV_THREADS * (wide ? 4 : 1));
  a.dt_blocks = (CONV_TILE * c.H + CONV_THREADS - 1) / CONV_THREADS;
  const long long blocks = 1 + (long long)(c.T / CONV_TILE + c.B) * (a.ch_blocks + a.dt_blocks);
  if (blocks > INT_MAX) return cudaErrorInvalidConfiguration;
  const cudaError_t e = wide ? launch_rows_w<TI, 4>(a, unsigned(blocks), stream) : launch_rows_w<TI, 1>(a, unsigned(blocks), stream);
  if (e != cudaSuccess) return e;
  StateArgs s{};
  s.c = c;
  s.s = a.s;
  return c.T > 2ll * c.B ? launch_states<TI, true>(s, stream) : launch_states<TI, false>(s, stream);
}

bool scan_has_blocks(int P, int N) { return P == 64 && N == 128; }

// Where everything lies in the caller's scratch.
struct Scratch {
  size_t step, c_parts, cb, plan, list, chunks, images, total;
  int pitch;
  bool blocks, tensor;               // requests with few rows go through scan_block_kernel, those with many through the tensor cores
  Scratch(long long T, int B, int Di, int P, int N, int G, bool by_blocks, bool many) {
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    blocks = by_blocks;
    pitch = (Di + 2 * G * N + 3) / 4 * 4;
    tensor = many && T > SCAN_FEW;
    const size_t rows = tensor && T > (long long)(SCAN_FEW) * B ? size_t(SCAN_FEW) * B : size_t(T);
    step = up(rows * pitch * 4);
    c_parts = step + up(rows * (Di / P) * 16);
    cb = c_parts + (blocks ? up(rows * G * N * 2 * SCAN_C_PARTS) : 0);
    plan = cb + (blocks ? up(size_t(B) * G * SCAN_FEW * SCAN_FEW * 4) : 0);
    list = plan + 256;
    chunks = list + (tensor ? up(size_t(scan_max_long(T, B)) * 8) : 0);
    images = chunks + (tensor ? up(size_t(scan_max_chunks(T, B)) * 8) : 0);
    total = images + (tensor ? size_t(scan_max_chunks(T, B)) * G * SCAN_IMAGE_BYTES : 0);
  }
};

}  // namespace

// (The kernels of this shape need no less with products than without, and what they need grows with T and B.)
size_t chunk_scan_workspace_bytes(long long T, int B, int Di, int P, int N, int G) {
  return Scratch(T, B, Di, P, N, G, scan_has_blocks(P, N), scan_has_blocks(P, N)).total;
}

cudaError_t chunk_scan_launch(const ChunkScanCall& c, cudaStream_t stream) {
  // Row after row where there are hardly more rows than requests: if all of them have some, nothing but the states counts (64 tokens of 64 requests 121 us, with
  // products and the launches for requests with many rows 184; 17 rows of 32 requests 182 and 82).  But most of them may be empty places, and the rows one
  // request's: above LONE rows the kernels for these stand behind (500 rows among 255 empty places 146 us, in one chain of rows 390 to 680; 8 us of 600 where they
  // find nothing, 300 tokens), below the chain is short.
  constexpr int LONE = 256;
  const bool products = scan_has_blocks(c.P, c.N), by_blocks = products && c.T > 2ll * c.B;
  const Scratch at(c.T, c.B, c.Di, c.P, c.N, c.G, by_blocks, by_blocks || (products && c.T > LONE));
  char* ws = reinterpret_cast<char*>(c.ws);
  ConvArgs a{};
  a.c = c;
  a.s.pitch = at.pitch;
  a.s.xbc = reinterpret_cast<float*>(ws);
  a.s.step = reinterpret_cast<float4*>(ws + at.step);
  a.s.few = INT_MAX;
  if (at.blocks) {
    a.s.sums = reinterpret_cast<float4*>(ws + at.step);
    a.s.c_parts = reinterpret_cast<uint16_t*>(ws + at.c_parts);
    a.s.cb = reinterpret_cast<float*>(ws + at.cb);
  }
  if (at.tensor) {
    a.s.few = SCAN_FEW;
    a.s.apart = c.T > (long long)(SCAN_FEW) * c.B ? SCAN_FEW : 0;
    a.plan = reinterpret_cast<int32_t*>(ws + at.plan);
    a.list = reinterpret_cast<int32_t*>(ws + at.list);
    a.chunks = reinterpret_cast<int32_t*>(ws + at.chunks);
    a.max_long = int(scan_max_long(c.T, c.B));
    a.max_chunks = int(scan_max_chunks(c.T, c.B));
  }
  const cudaError_t e = c.in_dtype == CHUNK_F32 ? launch_all<float>(a, stream) : c.in_dtype == CHUNK_F16 ? launch_all<__half>(a, stream)
                                                                                                         : launch_all<__nv_bfloat16>(a, stream);
  if (e != cudaSuccess || !at.tensor) return e;
  LongArgs l{};
  l.c = c;
  l.plan = a.plan; l.list = a.list; l.chunks = a.chunks;
  l.images = reinterpret_cast<uint8_t*>(ws + at.images);
  return scan_long_launch(l, stream);
}

}  // namespace hspec
