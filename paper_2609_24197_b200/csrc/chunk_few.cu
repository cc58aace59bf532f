// Attention of a chunk's requests that have few rows, single tokens above all, over the paged cache: at most 8 rows of a KV head.
//   o[t, h] = sum_j p_j v[j, g] / sum_j p_j,  p_j = exp(scale q[t, h] . k[j, g]),  the keys as in chunk_attention.cu
//
// With 4 or 8 rows there is next to nothing to compute, and what counts is how many bytes are under way and how long the way from an item's first byte to
// its result is.  The tcgen05 kernel has one item at a time on an SM, and that way takes 13 000 clocks.  Here every warp has an item of its own, twelve to
// an SM, and needs no shared memory and no barrier for it.  32 query heads on 8 of 128, bf16: 2000 single tokens over 300 others 412 us (6.0 TB/s; the
// other kernel 1324), 8192 over 100 others 677 us (5.5 TB/s; 3080), one over 2047 others 14.0 us (20.5; latency alone).
//
// A warp takes 16 keys a step, on mma.sync with the keys in the rows of the product: S^T = K Q^T and O^T += V^T P^T, so that 8 columns hold all rows of
// the head and nothing is padded.  Loads go straight to registers, 16 bytes of a key (value) for a thread, and are under way a step ahead.
//   K: the sum over the head's elements may run in any order, so that thread (g, c) = (lane / 4, lane % 4) takes the 16-byte pieces c, c + 4, .. of
//      keys g and g + 8, and of Q's row g: each piece is the operand of two products.
//   V: thread (g, c) loads columns 8 g .. 8 g + 7 of keys 2 c, 2 c + 1, 2 c + 8, 2 c + 9; neighbouring keys are paired by byte permutes, and its columns
//      take rows g and g + 8 of four products.  The result then lies as 8 neighbouring columns of rows 2 c and 2 c + 1.
//   P: weights come out transposed, and movmatrix turns them.  They are rounded to the pools' type for the product (see weights_of in chunk_attention.cu); their
//      sums are of 32-bit ones.
// The reference maximum moves when a score exceeds it by 2^8 (fp16 weights hold 2^15); sums are a thread's own until the item's end.
#include "chunk_plan.cuh"

namespace hspec {

namespace {

// Keys that are not shared between warps: one token over 2047 others takes 14.0 us, 15.4 with 64 and 15.1 with 16 (more parts to join), and long lines
// do not care.
constexpr int TILE = 32;
constexpr int WARPS = 12;            // of an SM: as many as 168 registers leave room for (10 are 3 to 6 % slower on long lines)
constexpr int UNITS = 148 * WARPS;
constexpr int COST_ITEM = 1, COST_TILE = 1;
constexpr float LAZY = 8.0f;

__device__ __forceinline__ uint4 load_once(const uint16_t* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
template <bool F16>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  const uint32_t a[4] = {a0, a1, a2, a3};
  if (F16) mma_f16_16816(c, a, b0, b1);
  else mma_bf16_16816(c, a, b0, b1);
}
template <bool F16>
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
  if (F16) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  return pack_bf16(lo, hi);
}
template <bool F16> __device__ __forceinline__ bool not_finite16(uint32_t x) {
  constexpr uint32_t m = F16 ? 0x7c00u : 0x7f80u;
  return (x & m) == m;
}
template <bool F16> __device__ __forceinline__ float widen16(uint16_t x) { return F16 ? __half2float(__ushort_as_half(x)) : bf16_bits_to_float(x); }

__device__ __forceinline__ long long quotient(long long a, int b) {      // (a >= 0, b > 0; a 64-bit division is some hundred instructions)
  return (a >> 32) == 0 ? (long long)(uint32_t(a) / uint32_t(b)) : a / b;
}
// place_of, for items of one row tile and costs of one a tile: every lane may ask for another part.
__device__ __forceinline__ int4 place_of_few(const Args& a, const Line& line, int i) {
  const long long* sums = line.sums;
  const int B = a.c.B, groups = a.c.Hkv / a.group;
  const long long u = quotient(sums[B] * i, line.parts);
  auto request_at = [&](long long v) {                        // the request with sums[r] <= v < sums[r + 1], or B
    int lo = 0, hi = B;
    while (lo < hi) { const int mid = (lo + hi) >> 1; if (sums[mid + 1] <= v) lo = mid + 1; else hi = mid; }
    return lo;
  };
  const int r = request_at(u);
  if (r >= B) return make_int4(B, 0, 0, 0);
  const long long each = quotient(sums[r + 1] - sums[r], groups);
  const int item = int(each), rest0 = int(u - sums[r] - quotient(u - sums[r], item) * item), g = int(quotient(u - sums[r], item));
  const int off = rest0 > 0 ? max(1, rest0 - line.k.item) : 0;
  if (off < item - line.k.item) return make_int4(r, g, 0, off);
  if (g + 1 < groups) return make_int4(r, g + 1, 0, 0);
  return make_int4(request_at(sums[r + 1]), 0, 0, 0);
}

template <int DH, bool F16>
__global__ void __launch_bounds__(WARPS * 32, 1) chunk_few_kernel(const __grid_constant__ Args a) {
  constexpr int KP = DH / 32, VB = DH / 64;                   // 16-byte pieces of a key for a thread, blocks of 64 columns
  extern __shared__ long long sums[];
  pdl_wait();
  pdl_trigger();
  const ChunkAttnCall& c = a.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c4 = lane & 3;
  const int unit = blockIdx.x * WARPS + warp, part = unit / a.group, groups = c.Hkv / a.group;
  const Line line = make_line<TILE>(a, sums, Costs{COST_ITEM, COST_TILE, COST_TILE}, int(gridDim.x) * WARPS / a.group);
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.ws_count = line.parts;
  if (part >= line.parts) return;
  int4 start = place_of_few(a, line, part + (lane & 1)), stop;
  stop.x = __shfl_sync(0xffffffffu, start.x, 1); stop.y = __shfl_sync(0xffffffffu, start.y, 1); stop.w = __shfl_sync(0xffffffffu, start.w, 1);
  start.x = __shfl_sync(0xffffffffu, start.x, 0); start.y = __shfl_sync(0xffffffffu, start.y, 0); start.w = __shfl_sync(0xffffffffu, start.w, 0);
  int b = start.x, group = start.y, tile = start.w, slot = 2 * unit;
  ChunkRequest q = load_request(a, b), q_next = load_request(a, b + 1);
  if (lane == 0) put_start(a, unit, start, q);
  const uint16_t *pool_k = reinterpret_cast<const uint16_t*>(c.k_pool), *pool_v = reinterpret_cast<const uint16_t*>(c.v_pool);
  for (;;) {
    const ItemGeo geo = item_geo<TILE>(q, a.rep, c.window, 0);
    const int kvh = group * a.group + unit % a.group;
    const int t0 = geo.t0 + tile, t1 = b == stop.x && group == stop.y ? geo.t0 + stop.w : geo.t1;
    const bool whole = tile == 0 && t1 == geo.t1;
    const int s0 = max(t0 * (TILE / 16), geo.key_lo / 16), s1 = min(t1 * (TILE / 16), (geo.key_hi + 15) / 16);      // steps with keys that any row sees
    const int32_t* table = c.page_table + size_t(b) * c.page_table_stride;
    // this lane's key of a step (two lanes each): its page, and a step later its place in the pools
    auto page_of = [&](int s) {
      const int key = s * 16 + (lane & 15);
      return s < s1 && key >= geo.key_lo && key < geo.key_hi ? table[key / c.page_size] : -1;
    };
    auto place = [&](int s, int page) {
      const int key = s * 16 + (lane & 15), in = key % c.page_size;
      const bool on = s < s1 && key >= geo.key_lo && key < geo.key_hi;
      if (unsigned(page) < unsigned(c.num_pages)) return ((long long)page * c.page_size + in) * c.Hkv + kvh;
      if (on && lane < 16 && (in == 0 || key == geo.key_lo)) atomicAdd(c.status + STATUS_WORD_BAD_INPUT, 1u);
      return -1ll;
    };
    uint4 kr[2][KP], vr[VB][4];
    auto load_k = [&](long long row) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const long long r = __shfl_sync(0xffffffffu, row, g + 8 * i);
#pragma unroll
        for (int p = 0; p < KP; ++p) kr[i][p] = r >= 0 ? load_once(pool_k + r * DH + (c4 + 4 * p) * 8) : make_uint4(0u, 0u, 0u, 0u);
      }
    };
    auto load_v = [&](long long row) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const long long r = __shfl_sync(0xffffffffu, row, 2 * c4 + (i & 1) + 8 * (i >> 1));
#pragma unroll
        for (int v = 0; v < VB; ++v) vr[v][i] = r >= 0 ? load_once(pool_v + r * DH + v * 64 + g * 8) : make_uint4(0u, 0u, 0u, 0u);
      }
    };
    long long row = place(s0, page_of(s0));
    load_k(row);
    load_v(row);
    int page = page_of(s0 + 1);
    // Q's row g; this thread's rows of the scores, 2 c4 and 2 c4 + 1: keys lo .. hi are seen
    const int rows = q.n * a.rep;
    uint32_t qr[KP][4];
    {
      const int token = g / a.rep, head = g - token * a.rep;
      const uint16_t* src = reinterpret_cast<const uint16_t*>(c.q) + size_t(q.q0 + token) * c.ldq + size_t(kvh * a.rep + head) * DH;
#pragma unroll
      for (int p = 0; p < KP; ++p) {
        const uint4 x = g < rows ? *reinterpret_cast<const uint4*>(src + (c4 + 4 * p) * 8) : make_uint4(0u, 0u, 0u, 0u);
        qr[p][0] = x.x; qr[p][1] = x.y; qr[p][2] = x.z; qr[p][3] = x.w;
      }
    }
    int hi[2], lo[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      hi[i] = 2 * c4 + i < rows ? max(-1, q.len - q.n + (2 * c4 + i) / a.rep) : -1;
      lo[i] = c.window > 0 ? max(0, hi[i] - c.window + 1) : 0;
    }
    auto all_see = [&](int key) { return key <= geo.pos0 && (c.window <= 0 || key > geo.pos1 - c.window); };
    float o[2 * KP][4];                                       // [block of 64 columns * 4 + pair of columns][column of the pair, row]
#pragma unroll
    for (int i = 0; i < 2 * KP; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    float ref[2] = {NEG, NEG}, sum[2] = {0.f, 0.f};
    bool bad = false;
    for (int s = s0; s < s1; ++s) {
      const long long row_next = place(s + 1, page);
      page = page_of(s + 2);
      const int key0 = s * 16;
      const bool mixed = !all_see(key0) || !all_see(key0 + 15);                   // (what rows that are not there see goes nowhere)
      float x[4] = {0.f, 0.f, 0.f, 0.f};                      // (key g, row 2 c4), (g, 2 c4 + 1), (g + 8, 2 c4), (g + 8, 2 c4 + 1)
#pragma unroll
      for (int p = 0; p < KP; ++p) {
        mma<F16>(x, kr[0][p].x, kr[1][p].x, kr[0][p].y, kr[1][p].y, qr[p][0], qr[p][1]);
        mma<F16>(x, kr[0][p].z, kr[1][p].z, kr[0][p].w, kr[1][p].w, qr[p][2], qr[p][3]);
      }
      load_k(row_next);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = key0 + g + 8 * (i >> 1);
        x[i] = !mixed || (key <= hi[i & 1] && key >= lo[i & 1]) ? x[i] * a.scale_log2 : -INFINITY;
      }
      const float m0 = fmaxf(x[0], x[2]), m1 = fmaxf(x[1], x[3]);
      if (__any_sync(0xffffffffu, m0 > ref[0] + LAZY || m1 > ref[1] + LAZY)) {
        float m[2] = {fmaxf(m0, ref[0]), fmaxf(m1, ref[1])};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          for (int off = 4; off < 32; off <<= 1) m[i] = fmaxf(m[i], __shfl_xor_sync(0xffffffffu, m[i], off));
          if (!(m[i] > ref[i] + LAZY)) m[i] = ref[i];         // (another row's: this one's result does not hang on it)
          const float f = ex2_ftz(ref[i] - m[i]);
          ref[i] = m[i];
          sum[i] *= f;
#pragma unroll
          for (int e = 0; e < 2 * KP; ++e) { o[e][i] *= f; o[e][2 + i] *= f; }
        }
        if (lane == 0 && s > s0) atomicAdd(c.status + STATUS_WORD_RESCALES, 1u);
      }
      float w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = ex2_ftz(x[i] - ref[i & 1]);
      sum[0] += w[0] + w[2];
      sum[1] += w[1] + w[3];
      const uint32_t p0 = transposed(pack_pair<F16>(w[0], w[1])), p1 = transposed(pack_pair<F16>(w[2], w[3]));
      if (mixed) {
        // Values that are not finite and that some rows do not see: zero here, added to the rows that see them at the end.
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (all_see(key0 + 2 * c4 + (i & 1) + 8 * (i >> 1))) continue;
#pragma unroll
          for (int v = 0; v < VB; ++v) {
            uint32_t y[4] = {vr[v][i].x, vr[v][i].y, vr[v][i].z, vr[v][i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if (not_finite16<F16>(y[e])) { y[e] &= 0xffff0000u; bad = true; }
              if (not_finite16<F16>(y[e] >> 16)) { y[e] &= 0x0000ffffu; bad = true; }
            }
            vr[v][i] = make_uint4(y[0], y[1], y[2], y[3]);
          }
        }
      }
#pragma unroll
      for (int v = 0; v < VB; ++v) {
        const uint32_t y[4][4] = {{vr[v][0].x, vr[v][0].y, vr[v][0].z, vr[v][0].w}, {vr[v][1].x, vr[v][1].y, vr[v][1].z, vr[v][1].w},
                                  {vr[v][2].x, vr[v][2].y, vr[v][2].z, vr[v][2].w}, {vr[v][3].x, vr[v][3].y, vr[v][3].z, vr[v][3].w}};
#pragma unroll
        for (int e = 0; e < 4; ++e)                           // columns 2 e and 2 e + 1 of this thread's 8, keys 2 c4, 2 c4 + 1 and 8 further
          mma<F16>(o[v * 4 + e], __byte_perm(y[0][e], y[1][e], 0x5410), __byte_perm(y[0][e], y[1][e], 0x7632), __byte_perm(y[2][e], y[3][e], 0x5410),
                   __byte_perm(y[2][e], y[3][e], 0x7632), p0, p1);
      }
      load_v(row_next);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      for (int off = 4; off < 32; off <<= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], off);
    if (__any_sync(0xffffffffu, bad)) {                       // (a path that nothing else takes)
#pragma unroll 1
      for (int key = s0 * 16; key < min(s1 * 16, geo.key_hi); ++key) {
        if (key < geo.key_lo || all_see(key)) continue;
        const int id = table[key / c.page_size];
        if (unsigned(id) >= unsigned(c.num_pages)) continue;
        const uint16_t* src = pool_v + (((long long)id * c.page_size + key % c.page_size) * c.Hkv + kvh) * DH + g * 8;
#pragma unroll
        for (int v = 0; v < VB; ++v)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint16_t y = src[v * 64 + e];
#pragma unroll
            for (int i = 0; i < 2; ++i)
              if (not_finite16<F16>(y) && key <= hi[i] && key >= lo[i]) o[v * 4 + e / 2][(e & 1) * 2 + i] += widen16<F16>(y);
          }
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = 2 * c4 + i;
      if (r >= rows) continue;
      if (whole) {
        const int token = r / a.rep, head = r - token * a.rep;
        const float inv = sum[i] > 0.f ? 1.f / sum[i] : (sum[i] == 0.f ? 0.f : sum[i]);      // (nothing seen: zero; NaN stays)
        uint16_t* dst = reinterpret_cast<uint16_t*>(c.o) + size_t(q.q0 + token) * c.ldo + size_t(kvh * a.rep + head) * DH + g * 8;
#pragma unroll
        for (int v = 0; v < VB; ++v) {
          uint32_t y[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            y[e] = F16 ? pack_f16_sat(o[v * 4 + e][i] * inv, o[v * 4 + e][2 + i] * inv, c.status) : pack_bf16(o[v * 4 + e][i] * inv, o[v * 4 + e][2 + i] * inv);
          *reinterpret_cast<uint4*>(dst + v * 64) = make_uint4(y[0], y[1], y[2], y[3]);
        }
      } else {
        float* dst = a.ws_o + (size_t(slot) * FEW_ROWS + r) * DH + g * 8;
#pragma unroll
        for (int v = 0; v < VB; ++v)
#pragma unroll
          for (int e = 0; e < 4; e += 2)
            *reinterpret_cast<float4*>(dst + v * 64 + e * 2) = make_float4(o[v * 4 + e][i], o[v * 4 + e][2 + i], o[v * 4 + e + 1][i], o[v * 4 + e + 1][2 + i]);
        if (g == 0) a.ws_ml[size_t(slot) * FEW_ROWS + r] = make_float2(ref[i], sum[i]);
      }
    }
    // ---- on to the next item of this warp's part
    slot = 2 * unit + 1;
    tile = 0;
    if (t1 < geo.t1) break;
    if (++group == groups) {
      group = 0;
      ++b;
      q = q_next;
      if (q.n == 0) q = request_from(a, b);
      q_next = load_request(a, b + 1);
    }
    if (b >= c.B || (stop.w == 0 && b == stop.x && group == stop.y)) break;
  }
}

// Joins the items that a cut went through; the part that an item begins in speaks for it.  A block looks at a part for every SM (a warp each), then
// joins what there is to join, 16 warps to an item: a warp per row and share of the parts.  What it waits for in turn is the places, the rows' maxima
// and sums, and the partial results.
constexpr int JOIN_WARPS = 16, JOIN_AHEAD = 16;             // partial results under way at a time
template <int DH, bool F16>
__global__ void __launch_bounds__(JOIN_WARPS * 32) chunk_few_join_kernel(const __grid_constant__ Args a) {
  pdl_wait();
  pdl_trigger();
  constexpr int COLS = DH / 32;                               // of a lane
  static_assert(WARPS <= JOIN_WARPS, "a warp for every part");
  struct Job { int4 at, item; int unit, first, n; };
  __shared__ Job jobs[WARPS];
  __shared__ float part[JOIN_WARPS][DH];
  __shared__ float2 part_ml[JOIN_WARPS];
  const ChunkAttnCall& c = a.c;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (warp < WARPS) {
    const int me = blockIdx.x + gridDim.x * warp, next = me + a.group, behind = next + lane * a.group;
    int n = 0;
    if (next < a.units) {
      const int count = *a.ws_count * a.group;
      const int4 mine = a.ws_start[me], x = a.ws_start[next], item = a.ws_start[a.units + next];
      const int4 y = behind < a.units ? a.ws_start[behind] : make_int4(-1, 0, 0, 0);  // (of parts without work: anything)
      auto same = [&](const int4& p) { return p.x == x.x && p.y == x.y && p.z == x.z; };
      // a cut through an item here, and no earlier part that speaks for it
      if (next < count && x.w > 0 && !(same(mine) && mine.w > 0)) {
        unsigned run = __ballot_sync(0xffffffffu, behind < count && same(y));
        n = 1 + (run == 0xffffffffu ? 32 : __ffs(~run) - 1);
        for (int base = next + 32 * a.group; run == 0xffffffffu; base += 32 * a.group) {
          const int at = base + lane * a.group;
          run = __ballot_sync(0xffffffffu, at < count && same(a.ws_start[at < count ? at : me]));
          n += run == 0xffffffffu ? 32 : __ffs(~run) - 1;
        }
        if (lane == 0) jobs[warp] = Job{x, item, me, 2 * me + (same(mine) ? 0 : 1), n};
      }
    }
    if (n == 0 && lane == 0) jobs[warp].n = 0;
  }
  __syncthreads();
  for (int j = 0; j < WARPS; ++j) {
    const int n = jobs[j].n;
    if (n == 0) continue;
    const int rows = jobs[j].item.w, me = jobs[j].unit, first = jobs[j].first;
    const int wide = rows > 4 ? 8 : rows > 2 ? 4 : rows, shares = JOIN_WARPS / wide, r = warp % wide, share = warp / wide;
    auto row_of = [&](int i) { return unsigned(i == 0 ? first : 2 * (me + i * a.group)) * FEW_ROWS + r; };
    float m = NEG, sum = 0.f, acc[COLS];
#pragma unroll
    for (int e = 0; e < COLS; ++e) acc[e] = 0.f;
    // this warp's parts: share, share + shares, ..
    for (int base = share; base < n && r < rows; base += 32 * shares) {
      const int mine = base + lane * shares, count = min(32, (n - base + shares - 1) / shares);
      const float2 ml = mine < n ? a.ws_ml[row_of(mine)] : make_float2(NEG, 0.f);
      float v[JOIN_AHEAD][COLS];
      auto load = [&](int i) {
#pragma unroll
        for (int u = 0; u < JOIN_AHEAD; ++u)
#pragma unroll
          for (int e = 0; e < COLS; e += 2) {
            const float2 x = i + u < count ? *reinterpret_cast<const float2*>(a.ws_o + row_of(base + (i + u) * shares) * DH + lane * COLS + e) : make_float2(0.f, 0.f);
            v[u][e] = x.x; v[u][e + 1] = x.y;
          }
      };
      load(0);                                                // (under way with the maxima)
      float mm = fmaxf(ml.x, m);
      for (int off = 16; off > 0; off >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, off));
      const float f = ex2_ftz(m - mm), w = ml.x == NEG && ml.y == 0.f ? 0.f : ex2_ftz(ml.x - mm);
      float s = ml.y * w;
      for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
      m = mm;
      sum = sum * f + s;
#pragma unroll
      for (int e = 0; e < COLS; ++e) acc[e] *= f;
      for (int i = 0; i < count; i += JOIN_AHEAD) {
        if (i > 0) load(i);
#pragma unroll
        for (int u = 0; u < JOIN_AHEAD; ++u) {
          const float wi = __shfl_sync(0xffffffffu, w, (i + u) & 31);
#pragma unroll
          for (int e = 0; e < COLS; ++e) acc[e] = i + u < count ? fmaf(wi, v[u][e], acc[e]) : acc[e];
        }
      }
    }
#pragma unroll
    for (int e = 0; e < COLS; ++e) part[warp][lane * COLS + e] = acc[e];
    if (lane == 0) part_ml[warp] = make_float2(m, sum);
    __syncthreads();
    if (share == 0 && r < rows) {
      for (int i = 1; i < shares; ++i) m = fmaxf(m, part_ml[i * wide + r].x);
      sum = 0.f;
#pragma unroll
      for (int e = 0; e < COLS; ++e) acc[e] = 0.f;
      for (int i = 0; i < shares; ++i) {
        const float2 ml = part_ml[i * wide + r];
        const float f = ml.x == NEG && ml.y == 0.f ? 0.f : ex2_ftz(ml.x - m);
        sum += ml.y * f;
#pragma unroll
        for (int e = 0; e < COLS; ++e) acc[e] = fmaf(part[i * wide + r][lane * COLS + e], f, acc[e]);
      }
      const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);
      const int4 item = jobs[j].item;
      const int at = item.z + r, token = item.y + at / a.rep, kvh = jobs[j].at.y * a.group + me % a.group;
      uint16_t* dst = reinterpret_cast<uint16_t*>(c.o) + size_t(item.x + token) * c.ldo + size_t(kvh * a.rep + at % a.rep) * DH + lane * COLS;
#pragma unroll
      for (int e = 0; e < COLS; e += 2)
        *reinterpret_cast<uint32_t*>(dst + e) = F16 ? pack_f16_sat(acc[e] * inv, acc[e + 1] * inv, c.status) : pack_bf16(acc[e] * inv, acc[e + 1] * inv);
    }
    __syncthreads();                                          // (the arrays are free again)
  }
}

template <int DH, bool F16>
cudaError_t launch_for(const Args& a, cudaStream_t stream) {
  static bool done[MAX_DEVICES] = {};
  static int sms[MAX_DEVICES] = {};
  cudaError_t e = once_per_device(done, [&](int dev) {
    cudaError_t e1 = cudaDeviceGetAttribute(&sms[dev], cudaDevAttrMultiProcessorCount, dev);
    if (e1 == cudaSuccess) e1 = cudaFuncSetAttribute(chunk_few_kernel<DH, F16>, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * 8193 * 8);
    return e1;
  });
  if (e != cudaSuccess) return e;
  const int n = min(sms[current_device()], UNITS / WARPS);
  e = launch_pdl(chunk_few_kernel<DH, F16>, dim3(n), dim3(WARPS * 32), 2 * (size_t(a.c.B) + 1) * 8, stream, a);
  if (e != cudaSuccess) return e;
  return launch_pdl(chunk_few_join_kernel<DH, F16>, dim3(UNITS / WARPS), dim3(JOIN_WARPS * 32), 0, stream, a);
}

}  // namespace

size_t chunk_few_workspace_bytes(int dh) { return size_t(2 * UNITS) * FEW_ROWS * (size_t(dh) * 4 + 8) + 2 * UNITS * sizeof(int4) + 256; }

// Where most requests are short.  With long rows about, one kernel for all is mostly better: 63 single tokens over 2000 and 512 rows over 2000 take 155 us in
// one and 191 in two, 256 over 1000 and 2048 rows over none 380 and 360.  What the host cannot see costs batches without long rows 6 to 8 us, the other
// kernel's launches.
bool chunk_few_takes(const ChunkAttnCall& c) {
  const int rep = c.Hq / c.Hkv;
  return rep <= FEW_ROWS && (long long)c.T * rep <= 2ll * FEW_ROWS * c.B;
}
bool chunk_few_takes_all(const ChunkAttnCall& c) { return (long long)c.T * (c.Hq / c.Hkv) <= FEW_ROWS; }

cudaError_t chunk_few_launch(const ChunkAttnCall& c, void* ws, cudaStream_t stream) {
  Args a{};
  a.c = c;
  a.rep = c.Hq / c.Hkv;
  a.scale_log2 = c.scale * 1.4426950408889634f;
  a.kind = KIND_FEW;
  a.units = UNITS;
  // neighbouring warps take neighbouring heads of the same keys, as many as divide the heads
  for (a.group = min(c.Hkv, 16); c.Hkv % a.group; --a.group) {}
  a.ws_o = reinterpret_cast<float*>(ws);
  a.ws_ml = reinterpret_cast<float2*>(a.ws_o + size_t(2 * UNITS) * FEW_ROWS * c.dh);
  a.ws_start = reinterpret_cast<int4*>(a.ws_ml + size_t(2 * UNITS) * FEW_ROWS);
  a.ws_count = reinterpret_cast<int*>(a.ws_start + 2 * UNITS);
  if (c.dh == 64) return c.f16 ? launch_for<64, true>(a, stream) : launch_for<64, false>(a, stream);
  return c.f16 ? launch_for<128, true>(a, stream) : launch_for<128, false>(a, stream);
}

}  // namespace hspec
