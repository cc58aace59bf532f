// Attention of a ragged chunk: how the work is described and cut into parts, for both of its kernels (chunk_attention.cu, chunk_few.cu).
#pragma once
#include "chunk.cuh"

namespace hspec {

namespace {

constexpr int ITEM_ROWS = 256;
constexpr int FEW_ROWS = 8;          // requests with this many rows of a KV head or fewer have a kernel of their own
constexpr float NEG = -3.402823466e38f;   // the maximum of scores that are not there: the lowest number, so that no score lies below it
enum { KIND_ALL, KIND_FEW, KIND_MANY };

struct Args {
  ChunkAttnCall c;
  int rep, box_rows;                 // rows of a TMA box; 0: pages are copied by 16-byte loads
  uint32_t inv_rep;                  // 2^20 / rep, rounded up
  int group;                         // KV heads that are worked on side by side
  float scale_log2;
  float* ws_o;                       // [slot][DH / 4][256 rows][4]
  float2* ws_ml;                     // [slot][256 rows]
  int4* ws_start;                    // [unit]: where its part begins; [units + unit]: of the item there, first row, token and query head of the first
                                     // row, rows.  How many units (per head of a group) have work lies in ws_count
  int* ws_count;
  int units;                         // most of them: CTAs, or warps
  int kind;                          // whose requests are meant
};

// ------------------------------------------------------------------ geometry, the same for every role
struct ItemGeo {
  int r0, r1;                        // rows of the head
  int pos0, pos1;                    // positions of the first and the last row's token
  int key_lo, key_hi;                // keys that any row sees
  int t0, t1;                        // tiles
};
__device__ __forceinline__ bool takes_turns(int rows) { return rows <= 128; }
__device__ __forceinline__ int row_tiles(int rows) { return takes_turns(rows) ? (rows > 0 ? 1 : 0) : (rows + ITEM_ROWS - 1) / ITEM_ROWS; }
template <int TILE>
__device__ __forceinline__ ItemGeo item_geo(const ChunkRequest& q, int rep, int window, int rt) {
  ItemGeo g;
  const int rows = q.n * rep;
  g.r0 = rt * ITEM_ROWS;
  g.r1 = min(rows, g.r0 + ITEM_ROWS);
  g.pos0 = max(-1, q.len - q.n + g.r0 / rep);                 // (a place in front of the cache sees nothing, whichever it is: no window wraps round)
  g.pos1 = max(-1, q.len - q.n + (g.r1 - 1) / rep);
  g.key_lo = window > 0 ? max(0, g.pos0 - window + 1) : 0;
  g.key_hi = max(0, g.pos1 + 1);
  g.t0 = g.key_lo / TILE;
  g.t1 = max(g.t0 + 1, (g.key_hi + TILE - 1) / TILE);
  return g;
}

// A request without rows where it is not of the kind that is meant.
__device__ __forceinline__ ChunkRequest load_request(const Args& a, int b) {
  const ChunkAttnCall& c = a.c;
  if (b >= c.B) return ChunkRequest{0, 0, 0};
  ChunkRequest q = chunk_request(c.cu_q[b], c.cu_q[b + 1], c.kv_lens[b], c.T, c.max_len);
  if (a.kind != KIND_ALL && (a.kind == KIND_FEW) != (q.n * a.rep <= FEW_ROWS)) q.n = 0;
  return q;
}
// The first request with rows from b on, 32 at a time (one warp); moves b there, to B where there is none.
__device__ __forceinline__ ChunkRequest request_from(const Args& a, int& b) {
  const int lane = threadIdx.x & 31;
  for (; b < a.c.B; b += 32) {
    const ChunkRequest q = load_request(a, b + lane);
    const unsigned m = __ballot_sync(0xffffffffu, q.n > 0);
    if (m) {
      const int l = __ffs(m) - 1;
      b += l;
      return ChunkRequest{__shfl_sync(0xffffffffu, q.q0, l), __shfl_sync(0xffffffffu, q.n, l), __shfl_sync(0xffffffffu, q.len, l)};
    }
  }
  b = a.c.B;
  return ChunkRequest{0, 0, 0};
}

// ------------------------------------------------------------------ the plan
// The line is measured in costs: an item has `item` in front of its first tile and `turns` or `both` for every tile.  A tile belongs to the part in
// which its beginning lies.  Where the parts would be so short that one might hold no beginning, every tile counts one and nothing else does.
struct Costs { int item, turns, both; };
struct Line {
  Costs k;
  const long long* sums;             // costs up to every request
  int parts;
};
template <int TILE>
__device__ __forceinline__ int item_cost(const Costs& k, const ChunkRequest& q, const Args& a, int rt, int* tiles) {
  const ItemGeo g = item_geo<TILE>(q, a.rep, a.c.window, rt);
  *tiles = g.t1 - g.t0;
  return k.item + (takes_turns(q.n * a.rep) ? k.turns : k.both) * (g.t1 - g.t0);
}
// Costs and tiles of every request and their running sums, by the whole block.  `sums` is shared memory for twice B + 1 numbers.
template <int TILE>
__device__ __forceinline__ Line make_line(const Args& a, long long* sums, Costs k, int most) {
  const ChunkAttnCall& c = a.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5, groups = c.Hkv / a.group;
  long long* tile_sums = sums + c.B + 1;
  // a request per lane; those with more than one row tile by the whole warp
  for (int base = warp * 32; base < c.B; base += warps * 32) {
    const int b = base + lane;
    const bool on = b < c.B;
    if (a.kind != KIND_MANY && blockIdx.x == 0 && on && chunk_request_bad(c.cu_q[b], c.cu_q[b + 1], c.kv_lens[b], c.T, c.max_len))
      atomicAdd(c.status + STATUS_WORD_BAD_INPUT, 1u);
    const ChunkRequest mine = load_request(a, b);
    const int count = row_tiles(mine.n * a.rep);
    long long n = 0, m = 0;
    if (count == 1) {
      int tiles;
      n = item_cost<TILE>(k, mine, a, 0, &tiles);
      m = tiles;
    }
    for (unsigned many = __ballot_sync(0xffffffffu, count > 1); many; many &= many - 1) {
      const int l = __ffs(many) - 1;
      const ChunkRequest q{0, __shfl_sync(0xffffffffu, mine.n, l), __shfl_sync(0xffffffffu, mine.len, l)};
      long long ni = 0, mi = 0;
      for (int rt = lane; rt < row_tiles(q.n * a.rep); rt += 32) {
        int tiles;
        ni += item_cost<TILE>(k, q, a, rt, &tiles);
        mi += tiles;
      }
      for (int off = 16; off > 0; off >>= 1) { ni += __shfl_xor_sync(0xffffffffu, ni, off); mi += __shfl_xor_sync(0xffffffffu, mi, off); }
      if (lane == l) { n = ni; m = mi; }
    }
    if (on) { sums[b + 1] = n * groups; tile_sums[b + 1] = m * groups; }
  }
  if (threadIdx.x == 0) sums[0] = tile_sums[0] = 0;
  __syncthreads();
  if (warp < 2) {
    long long* s = warp == 0 ? sums : tile_sums;
    long long before = 0;
    for (int base = 0; base < c.B; base += 32) {
      long long n = base + lane < c.B ? s[base + lane + 1] : 0;
      for (int off = 1; off < 32; off <<= 1) { const long long o = __shfl_up_sync(0xffffffffu, n, off); if (lane >= off) n += o; }
      if (base + lane < c.B) s[base + lane + 1] = before + n;
      before += __shfl_sync(0xffffffffu, n, 31);
    }
  }
  __syncthreads();
  if (sums[c.B] < (long long)most * (k.item + (k.both > k.turns ? k.both : k.turns))) {
    k = Costs{0, 1, 1};
    sums = tile_sums;
  }
  return Line{k, sums, int(min((long long)most, sums[c.B]))};
}
// Where part i begins: the first tile that begins at its share of the line or behind (one warp): request, group of heads, row tile, tile of the item;
// request B at the end of the line.
template <int TILE>
__device__ __forceinline__ int4 place_of(const Args& a, const Line& line, int i, int lane) {
  const ChunkAttnCall& c = a.c;
  const Costs& k = line.k;
  const long long* sums = line.sums;
  const long long u = sums[c.B] * i / line.parts;
  const int groups = c.Hkv / a.group;
  if (u >= sums[c.B]) return make_int4(c.B, 0, 0, 0);
  int lo = 0, hi = c.B;                                       // the request with sums[lo] <= u < sums[lo + 1]
  while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (sums[mid] <= u) lo = mid; else hi = mid; }
  const ChunkRequest q = load_request(a, lo);
  const long long per_group = (sums[lo + 1] - sums[lo]) / groups;
  int g = int((u - sums[lo]) / per_group), rt = 0;
  long long rest = (u - sums[lo]) - g * per_group;
  const int count = row_tiles(q.n * a.rep);
  for (int base = 0; base < count; base += 32) {
    int tiles;
    long long upto = base + lane < count ? item_cost<TILE>(k, q, a, base + lane, &tiles) : 0;
    for (int off = 1; off < 32; off <<= 1) { const long long o = __shfl_up_sync(0xffffffffu, upto, off); if (lane >= off) upto += o; }
    const unsigned in = __ballot_sync(0xffffffffu, upto > rest);
    if (in) {
      const int l = __ffs(in) - 1;
      const long long before = __shfl_sync(0xffffffffu, upto, l > 0 ? l - 1 : 0);
      rt = base + l;
      rest -= l > 0 ? before : 0;
      break;
    }
    rest -= __shfl_sync(0xffffffffu, upto, 31);
  }
  int tiles, off = 0;
  item_cost<TILE>(k, q, a, rt, &tiles);
  const int each = takes_turns(q.n * a.rep) ? k.turns : k.both;
  if (rest > 0) off = max(1, int((rest - k.item + each - 1) / each));
  if (off < tiles) return make_int4(lo, g, rt, off);
  if (rt + 1 < count) return make_int4(lo, g, rt + 1, 0);
  if (g + 1 < groups) return make_int4(lo, g + 1, 0, 0);
  for (++lo; lo < c.B; lo += 32) {                            // the next request with work
    const unsigned m = __ballot_sync(0xffffffffu, lo + lane < c.B && sums[lo + lane + 1] != sums[lo + lane]);
    if (m) return make_int4(lo + __ffs(m) - 1, 0, 0, 0);
  }
  return make_int4(c.B, 0, 0, 0);
}
// For the kernel that joins the parts (one thread).
__device__ __forceinline__ void put_start(const Args& a, int unit, const int4& at, const ChunkRequest& q) {
  const int r0 = at.z * ITEM_ROWS, tok0 = r0 / a.rep;
  a.ws_start[unit] = at;
  a.ws_start[a.units + unit] = make_int4(q.q0, tok0, r0 - tok0 * a.rep, min(q.n * a.rep - r0, ITEM_ROWS));
}

}  // namespace

}  // namespace hspec
