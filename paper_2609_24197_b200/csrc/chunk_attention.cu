// Attention of a ragged chunk of new tokens over the paged cache that holds their keys and values already.
//   o[t, h] = sum_j p_j v[j, g] / sum_j p_j,  p_j = exp(scale q[t, h] . k[j, g]),  j <= pos(t), j > pos(t) - window,  g = h / (Hq / Hkv)
// A row that sees no key is zero.
//
// Rows of a request that share a KV head are packed: row r of the head is token r / rep, query head r % rep.  A work item is up to 256 rows
// of one (request, KV head) and all the 128-key tiles that any of them sees; tiles lie at multiples of 128 keys.  The items' tiles, request by
// request, are one long line that is cut into equal parts: however ragged the batch, every SM gets the same number of tiles, and an item that a
// cut goes through leaves partial results (at most two per CTA) which a second kernel joins.  A part is worked on by as many CTAs as a group
// has KV heads, one for each: they read neighbouring bytes of the same pages at the same time.
//
//   warps 0..7, 8..15  softmax of the two halves, two threads per row with half of a tile's keys each: scores from tensor memory, one pass with a
//                      reference maximum that moves only when the row's outgrows it by 2^8, weights back into tensor memory over the scores they
//                      came from.  With more than 128 rows a half is 128 rows and both see every tile; with fewer both have the same rows and take
//                      turns at the tiles (two tiles are then in the softmax at once), and their accumulators meet at the end.
//   warps 16, 18       producers of the K and of the V tiles, a ring each, by TMA boxes of a page's rows (by 16-byte copies where pages are not
//                      whole groups of 8 rows).  One warp for both could not issue the boxes of 16-token pages fast enough.
//   warp 17            issues S = Q K^T and O += P V (P from tensor memory), one half behind the other: while a half's scores are in the
//                      softmax the tensor core works for the other
//   warp 19            finds the CTA's share of the items, one after the other, and hands it to the others through shared memory (a place in the
//                      walk that every thread kept for itself went to local memory, and cost 20 000 clocks an item); and goes over the V tiles
//                      that not every row sees in full: values that no row sees, whatever was in the cache or in shared memory,
//                      become zero (a zero weight times NaN would not), and so do single values that are not finite and that some rows do not see.
//                      They are added to these rows' results at the end, from the cache, on a path that nothing else takes.
//
// Every wait is bounded; a role whose wait runs out sets a status word, and the CTA unwinds.
#include "chunk_plan.cuh"

#include <cstddef>
#include <type_traits>

namespace hspec {

namespace {

constexpr int KT = 128;              // keys per tile
constexpr int MAX_CTAS = 148;
// What an item costs where every CTA has many tiles, in units of 900 clocks: a tile whose halves take turns 2650 (its 64 KB at a CTA's share of
// the memory's rate), a tile that both halves see 3550, the way from an item's last tile to the next one's first 12 600 (with 5 in
// place of 14 a prompt of 8192 tokens takes 638 us, not 548).
constexpr int COST_TURNS = 3, COST_BOTH = 4, COST_ITEM = 14;
constexpr float LAZY = 8.0f;         // the reference maximum moves, for the next tile, when the row's exceeds it by 2^8
// And at once when it exceeds it by more than the weights' type can hold, or 32 bits a tile's products with values up to 2^60.
constexpr float LIMIT_BF16 = 60.0f, LIMIT_F16 = 15.0f;
constexpr int THREADS = 640;

template <int DH> struct Shape {
  static constexpr int HALF = KT * 128;                      // [128 rows x 64 values]: 16 KiB, rows of 128 swizzled bytes
  static constexpr int TILE = KT * DH * 2;                   // Q, K or V tile
  static constexpr int NK = DH == 128 ? 2 : 4, NV = DH == 128 ? 3 : 6;      // slots of the rings: 160 KiB of K and V tiles
};



// A CTA's share of an item, as every role needs it.
struct Segment {
  ItemGeo g;
  int b, kvh, q0, pos;               // request, KV head, the request's first row and its position
  int tok0, rem0;                    // the item's first row is query head rem0 (of the KV head's) of the request's token tok0
  int ta, tb;                        // tiles
  int nt[2];                         // tiles of each half
  int turns, whole, end;             // end: there is none any more
};
constexpr int SEGS = 4;

struct __align__(16) Bars {
  // a slot's tile has arrived, has been read, and for V tiles that not every row sees in full: has arrived and is to be gone over, after which
  // the warp that does so gives the arrival of `full`
  uint64_t k_full[4], k_empty[4], v_full[6], v_empty[6], v_raw[6];
  uint64_t q_ready[2], s_ready[2], p_half[2], p_ready[2], pv_done[2], o_free[2];
  uint64_t x_write, x_read, drain;
  uint64_t seg_full[SEGS], seg_empty[SEGS];
  Segment seg[SEGS];                 // what the roles work on, in order
  uint32_t tmem_base, abort_flag;
  uint32_t bad[16];                  // n + 1 where segment n (modulo 16; at most 6 fit into the ring) met a value that is not finite in a tile
                                     // that not every row sees in full
  int4 start, stop;                  // where this CTA's part begins and where the next one's does: request, group of KV heads, row tile, tile of the item
  ChunkRequest req[2];               // the request that it begins in and the one behind it
  float xch[2][2][128];              // [half][half of the columns][row]: what the threads of a row tell each other
};
constexpr size_t smem_bytes(int tile, int slots) { return size_t(tile) * (2 + slots) + sizeof(Bars); }

struct Walk {                        // this CTA's part of the line, item by item; `next` is request b + 1
  int b, g, kvh, rt, off;
  int4 stop;
  ChunkRequest q, next;
};
__device__ __forceinline__ Walk walk_begin(const Args& a, const Bars* bars) {
  Walk w;
  w.b = bars->start.x; w.g = bars->start.y; w.rt = bars->start.z; w.off = bars->start.w;
  w.kvh = w.g * a.group + blockIdx.x % a.group;
  w.stop = bars->stop;
  w.q = bars->req[0];
  w.next = bars->req[1];
  return w;
}
__device__ __forceinline__ Segment segment_of(const Walk& w, const Args& a) {
  Segment s;
  s.g = item_geo<KT>(w.q, a.rep, a.c.window, w.rt);
  s.b = w.b; s.kvh = w.kvh; s.q0 = w.q.q0; s.pos = w.q.len - w.q.n;
  s.tok0 = s.g.r0 / a.rep; s.rem0 = s.g.r0 - s.tok0 * a.rep;
  s.ta = s.g.t0 + w.off;
  s.tb = w.b == w.stop.x && w.g == w.stop.y && w.rt == w.stop.z ? s.g.t0 + w.stop.w : s.g.t1;
  s.whole = w.off == 0 && s.tb == s.g.t1;
  s.turns = takes_turns(w.q.n * a.rep);
  s.end = 0;
  const int T = s.tb - s.ta;
  if (s.turns) {
    s.nt[0] = (T + 1) / 2; s.nt[1] = T / 2;
  } else if (s.g.r1 - s.g.r0 > 128) {
    // the first half's rows end earlier, and with them the tiles that they see
    const int end = max(s.g.t0 + 1, (s.pos + (s.g.r0 + 127) / a.rep + KT) / KT);
    s.nt[0] = max(0, min(end - s.ta, T)); s.nt[1] = T;
  } else {
    s.nt[0] = T; s.nt[1] = 0;
  }
  return s;
}
// On to the next item; false at the end of this CTA's part.  (The whole warp.)
__device__ __forceinline__ bool walk_on(Walk& w, const Segment& s, const Args& a) {
  w.off = 0;
  if (s.tb < s.g.t1) return false;
  if (++w.rt == row_tiles(w.q.n * a.rep)) {
    w.rt = 0;
    w.kvh += a.group;
    if (++w.g == a.c.Hkv / a.group) {
      w.kvh -= w.g * a.group;
      w.g = 0;
      ++w.b;
      w.q = w.next;
      if (w.q.n == 0) w.q = request_from(a, w.b);
      w.next = load_request(a, w.b + 1);
    }
  }
  return w.b < a.c.B && !(w.stop.w == 0 && w.b == w.stop.x && w.g == w.stop.y && w.rt == w.stop.z);
}
// Row r of the item (below 256): its token, and its query head among the KV head's.  (x inv_rep >> 20 is x / rep for x (inv_rep rep - 2^20) < 2^20, which
// x < 256 + rep and rep <= 512 hold to; a division took 100 clocks several times an item.)
__device__ __forceinline__ void token_of(const Segment& s, const Args& a, int r, int& token, int& head) {
  const uint32_t x = uint32_t(s.rem0 + r), t = (x * a.inv_rep) >> 20;
  token = s.tok0 + int(t);
  head = int(x - t * uint32_t(a.rep));
}
// Segment n is there (bounded), and has been read.
__device__ __forceinline__ bool segment_wait(Bars* bars, uint32_t n) { return mbar_wait(smem_u32(&bars->seg_full[n % SEGS]), (n / SEGS) & 1); }
__device__ __forceinline__ void segment_read(Bars* bars, uint32_t n) { mbar_arrive(smem_u32(&bars->seg_empty[n % SEGS])); }
// Not every row of the item sees all of the tile's keys.
__device__ __forceinline__ bool partial_tile(const ItemGeo& g, int window, int t) {
  return t * KT + KT - 1 > g.pos0 || (window > 0 && t * KT < g.pos1 - window + 1);
}
// byte offset of (row, 16-byte chunk) in an operand tile: halves of 64 values, 128-byte swizzle
__device__ __forceinline__ uint32_t tile_off(int row, int chunk) {
  return uint32_t((chunk >> 3) * Shape<128>::HALF + (row >> 3) * 1024 + (row & 7) * 128 + (((chunk & 7) ^ (row & 7)) << 4));
}
__device__ __forceinline__ uint32_t idesc(bool f16, int n, bool b_mn_major) {
  const uint32_t fmt = f16 ? 0u : 1u;
  return (1u << 4) | (fmt << 7) | (fmt << 10) | ((b_mn_major ? 1u : 0u) << 16) | (uint32_t(n >> 3) << 17) | ((128u >> 4) << 24);
}
__device__ __forceinline__ void mbar_arrive_n(uint32_t bar, uint32_t n) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(n) : "memory");
}
template <bool F16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  if (F16) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  return pack_bf16(lo, hi);
}
template <bool F16>
__device__ __forceinline__ bool not_finite16(uint32_t x) {
  constexpr uint32_t m = F16 ? 0x7c00u : 0x7f80u;
  return (x & m) == m;
}

// ------------------------------------------------------------------ the plan
// Cuts the line: `sums` is shared memory for twice B + 1 numbers.  Returns false for a CTA without work.
__device__ __forceinline__ bool make_plan(const Args& a, Bars* bars, long long* sums) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, most = gridDim.x / a.group, me = blockIdx.x / a.group;
  const Line l = make_line<KT>(a, sums, Costs{COST_ITEM, COST_TURNS, COST_BOTH}, most);
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.ws_count = l.parts;
  if (me >= l.parts) return false;
  if (warp < 2) {
    const int4 at = place_of<KT>(a, l, me + warp, lane);
    if (warp == 0 && lane == 0) {
      bars->start = at;
      bars->req[0] = load_request(a, at.x);
      bars->req[1] = load_request(a, at.x + 1);
      put_start(a, blockIdx.x, at, bars->req[0]);
    }
    if (warp == 1 && lane == 0) bars->stop = at;
  }
  return true;                                                // (read behind the next barrier)
}

// ------------------------------------------------------------------ producers (one warp each)
template <int DH, bool IS_V>
__device__ __forceinline__ void produce(const Args& a, const CUtensorMap* tm, uint8_t* ring, Bars* bars, int lane) {
  constexpr int NS = IS_V ? Shape<DH>::NV : Shape<DH>::NK, TILE = Shape<DH>::TILE;
  const ChunkAttnCall& c = a.c;
  uint64_t* full = IS_V ? bars->v_full : bars->k_full;
  uint64_t* empty = IS_V ? bars->v_empty : bars->k_empty;
  volatile uint32_t* abort_flag = &bars->abort_flag;
  uint32_t at = 0;                                            // tiles issued
  uint32_t raw_phase = 0, is_raw = 0;                         // a bit per slot: phase of `v_raw`, and whether the slot's last tile went there
  bool ok = true;
  const int boxes = a.box_rows ? KT / a.box_rows : 0;
  for (uint32_t n = 0; ok; ++n) {
    if (!segment_wait(bars, n)) { ok = false; break; }
    const Segment s = bars->seg[n % SEGS];
    __syncwarp();
    if (lane == 0) segment_read(bars, n);
    if (s.end) break;
    const int32_t* table = c.page_table + size_t(s.b) * c.page_table_stride;
    // page of this lane's box (up to 16 of them), fetched a tile ahead
    auto page_of = [&](int t) {
      if (lane >= boxes || t >= s.tb) return -1;
      const int key = t * KT + lane * a.box_rows;
      return key < s.g.key_hi && key + a.box_rows > s.g.key_lo ? table[key / c.page_size] : -1;
    };
    int page_next = page_of(s.ta);
    for (int t = s.ta; t < s.tb; ++t, ++at) {
      const int page = page_next;
      page_next = page_of(t + 1);
      const uint32_t slot = at % NS;
      if (at >= NS && !mbar_wait(smem_u32(&empty[slot]), ((at / NS) - 1) & 1)) ok = false;
      if (!ok || *abort_flag) { ok = false; break; }
      const bool raw = IS_V && partial_tile(s.g, c.window, t);
      const uint32_t dst = smem_u32(ring) + slot * TILE, bar = smem_u32(raw ? &bars->v_raw[slot] : &full[slot]);
      const int key0 = t * KT;
      is_raw = raw ? is_raw | (1u << slot) : is_raw & ~(1u << slot);
      if (raw) raw_phase ^= 1u << slot;
      if (a.box_rows) {
        const int key = key0 + lane * a.box_rows;
        const bool on = lane < boxes && key < s.g.key_hi && key + a.box_rows > s.g.key_lo;
        const unsigned count = __popc(__ballot_sync(0xffffffffu, on));
        if (lane == 0) {
          if (count) mbar_expect_tx(bar, count * a.box_rows * DH * 2);
          else mbar_arrive(bar);
        }
        __syncwarp();
        if (on) {
          // (a page id outside the pool is outside the tensor map: the copy delivers zeros and touches no memory)
          if (!IS_V && unsigned(page) >= unsigned(c.num_pages)) atomicAdd(c.status + STATUS_WORD_BAD_INPUT, 1u);
#pragma unroll
          for (int h = 0; h < DH / 64; ++h)
            tma_load_4d(dst + h * Shape<DH>::HALF + lane * a.box_rows * 128, tm, h * 64, s.kvh, key % c.page_size, page, bar);
        }
      } else {
        const uint16_t* pool = reinterpret_cast<const uint16_t*>(IS_V ? c.v_pool : c.k_pool);
        for (int i = lane; i < KT * (DH / 8); i += 32) {
          const int r = i / (DH / 8), chunk = i % (DH / 8), key = key0 + r;
          bool on = key >= s.g.key_lo && key < s.g.key_hi;
          size_t from = 0;
          if (on) {
            const int id = table[key / c.page_size];
            if (unsigned(id) >= unsigned(c.num_pages)) {
              on = false;
              if (!IS_V && chunk == 0 && (key % c.page_size == 0 || key == s.g.key_lo)) atomicAdd(c.status + STATUS_WORD_BAD_INPUT, 1u);
            } else {
              from = ((size_t(id) * c.page_size + key % c.page_size) * c.Hkv + s.kvh) * DH + chunk * 8;
            }
          }
          cp_async16(dst + tile_off(r, chunk), pool + from, on);
        }
        cp_async_commit();
        cp_async_wait<0>();
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
      }
    }
  }
  if (!ok) {
    if (lane == 0) {
      if (!*abort_flag) atomicExch(c.status, STATUS_TIMEOUT_PRODUCER);
      *abort_flag = 1;
    }
    // what has been asked for still arrives in shared memory: it must not outlive the CTA
    for (uint32_t p = at > NS ? at - NS : 0; p < at; ++p) {
      const uint32_t slot = p % NS;
      if ((is_raw >> slot) & 1) mbar_wait(smem_u32(&bars->v_raw[slot]), ((raw_phase >> slot) & 1) ^ 1);
      else mbar_wait(smem_u32(&full[slot]), (p / NS) & 1);
    }
  }
}

// ------------------------------------------------------------------ the segments, and values that not every row sees
// This warp also tells the others what they work on, two segments ahead of its own.
template <int DH, bool F16>
__device__ __forceinline__ void lead_and_clean(const Args& a, uint8_t* ring, Bars* bars, int lane) {
  constexpr int NS = Shape<DH>::NV, TILE = Shape<DH>::TILE;
  volatile uint32_t* abort_flag = &bars->abort_flag;
  Walk w = walk_begin(a, bars);
  Segment ahead = segment_of(w, a);
  uint32_t told = 0;                                          // segments that the others know of
  bool more = true;
  auto tell = [&]() {
    if (told >= SEGS && !mbar_wait(smem_u32(&bars->seg_empty[told % SEGS]), ((told / SEGS) - 1) & 1)) return false;
    if (!more) ahead.end = 1;
    if (lane == 0) {
      bars->seg[told % SEGS] = ahead;
      mbar_arrive(smem_u32(&bars->seg_full[told % SEGS]));
    }
    __syncwarp();
    ++told;
    if (more) {
      more = walk_on(w, ahead, a);
      if (more) ahead = segment_of(w, a);
    }
    return true;
  };
  uint32_t base = 0, phase = 0;                               // phase of `v_raw`, a bit per slot
  for (uint32_t seg = 0;; ++seg) {
    while (told <= seg + 2 && !ahead.end) {
      if (!tell()) {
        if (lane == 0 && !*abort_flag) { atomicExch(a.c.status, STATUS_TIMEOUT_EPILOGUE); *abort_flag = 1; }
        return;
      }
    }
    const Segment s = bars->seg[seg % SEGS];
    if (s.end) return;
    for (int t = s.ta; t < s.tb; ++t) {
      if (!partial_tile(s.g, a.c.window, t)) continue;
      const uint32_t slot = (base + (t - s.ta)) % NS;
      if (!mbar_wait(smem_u32(&bars->v_raw[slot]), (phase >> slot) & 1) || *abort_flag) {
        if (lane == 0 && !*abort_flag) { atomicExch(a.c.status, STATUS_TIMEOUT_EPILOGUE); *abort_flag = 1; }
        return;
      }
      phase ^= 1u << slot;
      // rows [seen0, seen1) of the tile are seen by some rows of the item, [all0, all1) of them by every one
      const int key = t * KT, seen0 = max(0, s.g.key_lo - key), seen1 = min(KT, s.g.key_hi - key);
      const int all0 = a.c.window > 0 ? max(seen0, s.g.pos1 - a.c.window + 1 - key) : seen0, all1 = min(seen1, s.g.pos0 + 1 - key);
      uint8_t* tile = ring + slot * TILE;
      constexpr uint32_t EXP = F16 ? 0x7c007c00u : 0x7f807f80u, ONE = F16 ? 0x04000400u : 0x00800080u;
      bool bad = false;
      // a row is 128 bytes in each half of the tile; 4 rows a step of the warp, from the first step that has rows to look at
      auto go_over = [&](int from, int to) {
#pragma unroll 4
        for (int i = from; i < to; ++i) {
          const int r = i * 4 + (lane >> 3);
#pragma unroll
          for (int half = 0; half < DH / 64; ++half) {
            uint4* p = reinterpret_cast<uint4*>(tile + half * Shape<DH>::HALF) + i * 32 + lane;
            if (r >= all0 && r < all1) continue;
            if (r < seen0 || r >= seen1) { *p = make_uint4(0u, 0u, 0u, 0u); continue; }
            const uint4 v = *p;
            // (an exponent of ones is the only one that carries into its sign's place)
            if (((((v.x & EXP) + ONE) | ((v.y & EXP) + ONE) | ((v.z & EXP) + ONE) | ((v.w & EXP) + ONE)) & 0x80008000u) != 0u) {
              uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if (not_finite16<F16>(x[e])) x[e] &= 0xffff0000u;
                if (not_finite16<F16>(x[e] >> 16)) x[e] &= 0x0000ffffu;
              }
              *p = make_uint4(x[0], x[1], x[2], x[3]);
              bad = true;
            }
          }
        }
      };
      if (all0 < all1) {
        go_over(0, min((all0 + 3) / 4, all1 / 4));
        go_over(all1 / 4, KT / 4);
      } else {
        go_over(0, KT / 4);
      }
      if (bad) *reinterpret_cast<volatile uint32_t*>(&bars->bad[seg & 15]) = seg + 1;
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars->v_full[slot]));
    }
    base += s.tb - s.ta;
  }
}

// ------------------------------------------------------------------ MMA issuer (one thread)
// Everything this thread does between two products is time in which the tensor core may run dry: descriptors are a constant upper word and a lower
// word that is added to, places in the rings are counted along and not divided out, tiles are asked for before the weights that they wait for.
constexpr uint32_t DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);          // groups of 8 rows 1024 bytes apart, 128-byte swizzle
__device__ __forceinline__ uint32_t desc_lo_kmajor(uint32_t addr) { return (addr >> 4) | (1u << 16); }
__device__ __forceinline__ uint32_t desc_lo_mnmajor(uint32_t addr) { return (addr >> 4) | (uint32_t(Shape<128>::HALF >> 4) << 16); }
template <bool ACC>
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t id) {
  asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tmov.b64 a, {%1, %4};\n\tmov.b64 b, {%2, %4};\n\tsetp.ne.b32 p, %5, 0;\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(id), "r"(DESC_HI), "r"(ACC ? 1u : 0u)
               : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t id, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tmov.b64 b, {%2, %4};\n\tsetp.ne.b32 p, %5, 0;\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b_lo), "r"(id), "r"(DESC_HI), "r"(acc)
               : "memory");
}
template <int N> struct RingPos {    // a place in a ring of N slots, and the parity of its use
  uint32_t slot = 0, phase = 0;
  __device__ __forceinline__ void step(uint32_t n) {          // n <= N
    slot += n;
    if (slot >= N) { slot -= N; phase ^= 1u; }
  }
};

template <int DH, bool F16>
__device__ __forceinline__ void issue_mmas(const Args& a, uint8_t* sQ, uint8_t* ring_k, uint8_t* ring_v, Bars* bars, uint32_t tmem) {
  constexpr int NK = Shape<DH>::NK, NV = Shape<DH>::NV, TILE = Shape<DH>::TILE, HALF = Shape<DH>::HALF;
  const uint32_t id_s = idesc(F16, KT, false), id_o = idesc(F16, DH, true);
  const uint32_t q_lo = desc_lo_kmajor(smem_u32(sQ)), k_lo = desc_lo_kmajor(smem_u32(ring_k)), v_lo = desc_lo_mnmajor(smem_u32(ring_v));
  const uint32_t bar0 = smem_u32(bars);
#define BAR(field, i) (bar0 + uint32_t(offsetof(Bars, field)) + uint32_t(i) * 8u)
  volatile uint32_t* abort_flag = &bars->abort_flag;
  RingPos<NK> k_at[2];                                        // next K and V tile of each half
  RingPos<NV> v_at[2];
  uint32_t q_phase[2] = {0, 0}, p_phase[2] = {0, 0}, o_phase[2] = {1, 1};
  bool ok = true;
  for (uint32_t n = 0; ok; ++n) {
    if (!segment_wait(bars, n)) { ok = false; break; }
    const Segment* s = &bars->seg[n % SEGS];
    const bool turns = s->turns, end = s->end;
    const int T = s->tb - s->ta, nt0 = s->nt[0], nt1 = s->nt[1];
    segment_read(bars, n);
    if (end) break;
    const uint32_t step = turns ? 2 : 1;
    if (turns) { k_at[1].step(1); v_at[1].step(1); }
    auto scores = [&](auto H, bool there, bool last_reader) {
      constexpr int h = decltype(H)::value;
      if (!there && !mbar_wait_spin(BAR(k_full, k_at[h].slot), k_at[h].phase)) { ok = false; return; }
      const uint32_t kb = k_lo + k_at[h].slot * (TILE >> 4), qb = q_lo + h * (TILE >> 4);
#pragma unroll
      for (int ks = 0; ks < DH / 16; ++ks) {
        constexpr uint32_t H4 = HALF >> 4;
        const uint32_t off = (ks >> 2) * H4 + (ks & 3) * 2;
        if (ks == 0) mma_ss<false>(tmem + h * 128, qb + off, kb + off, id_s);
        else mma_ss<true>(tmem + h * 128, qb + off, kb + off, id_s);
      }
      umma_commit(BAR(s_ready, h));
      if (last_reader) umma_commit(BAR(k_empty, k_at[h].slot));
      k_at[h].step(step);
    };
    auto first = [&](auto H, int nt, bool last_reader) {
      constexpr int h = decltype(H)::value;
      if (nt == 0 || !ok) return;
      if (!mbar_wait_spin(BAR(q_ready, h), q_phase[h])) { ok = false; return; }
      q_phase[h] ^= 1u;
      tc_fence_after();
      scores(H, false, last_reader);
    };
    // tile j of one half: the product of its weights, and the scores of the half's next tile behind it.  A tile's last reader frees its slot.
    auto step_of = [&](auto H, int j, int nt, bool last_reader, bool last_reader_next) {
      constexpr int h = decltype(H)::value;
      if (j >= nt || !ok) return;
      if (j == 0) {                                           // the accumulator is written over: the item before must have been read out
        if (!mbar_wait_spin(BAR(o_free, h), o_phase[h])) { ok = false; return; }
        o_phase[h] ^= 1u;
      }
      const bool more = j + 1 < nt;
      if (!mbar_wait_spin(BAR(v_full, v_at[h].slot), v_at[h].phase)) { ok = false; return; }
      const bool there = more && mbar_test(BAR(k_full, k_at[h].slot), k_at[h].phase);
      const uint32_t vb = v_lo + v_at[h].slot * (TILE >> 4), o = tmem + 256 + h * 128, p = tmem + h * 128;
      if (!mbar_wait_spin(BAR(p_half, h), p_phase[h])) { ok = false; return; }
      tc_fence_after();
      // the first half of every thread's weights: keys 0 .. 31 and 64 .. 95 (16 keys: 8 columns of weights, 2048 bytes of values)
      mma_ts(o, p, vb, id_o, j > 0);
      mma_ts(o, p + 8, vb + 128, id_o, 1);
      mma_ts(o, p + 64, vb + 512, id_o, 1);
      mma_ts(o, p + 72, vb + 640, id_o, 1);
      if (!mbar_wait_spin(BAR(p_ready, h), p_phase[h])) { ok = false; return; }
      p_phase[h] ^= 1u;
      tc_fence_after();
      mma_ts(o, p + 16, vb + 256, id_o, 1);
      mma_ts(o, p + 24, vb + 384, id_o, 1);
      mma_ts(o, p + 80, vb + 768, id_o, 1);
      mma_ts(o, p + 88, vb + 896, id_o, 1);
      if (last_reader) umma_commit(BAR(v_empty, v_at[h].slot));
      v_at[h].step(step);
      if (more) scores(H, there, last_reader_next);
      umma_commit(BAR(pv_done, h));
    };
    using H0 = std::integral_constant<int, 0>;
    using H1 = std::integral_constant<int, 1>;
    first(H0{}, nt0, turns || nt1 == 0);
    first(H1{}, nt1, true);
    const int most = nt0 > nt1 ? nt0 : nt1;
    for (int j = 0; j < most && ok; ++j) {
      step_of(H0{}, j, nt0, turns || j >= nt1, turns || j + 1 >= nt1);
      step_of(H1{}, j, nt1, true, true);
    }
    if (!ok) break;
    // both halves' places go on behind the segment's last tile
    if (turns) {
      const int ahead = T & 1 ? 0 : 1;                        // the half that stands one tile further on than the segment's end
      if (ahead) { k_at[1] = k_at[0]; v_at[1] = v_at[0]; }
      else { k_at[0] = k_at[1]; v_at[0] = v_at[1]; }
    } else if (nt0 >= nt1) {
      k_at[1] = k_at[0]; v_at[1] = v_at[0];
    } else {
      k_at[0] = k_at[1]; v_at[0] = v_at[1];
    }
  }
  if (!ok) {
    if (!*abort_flag) atomicExch(a.c.status, STATUS_TIMEOUT_MMA);
    *abort_flag = 1;
    umma_commit(BAR(drain, 0));                               // products under way end before the CTA does
    mbar_wait(BAR(drain, 0), 0);
  }
#undef BAR
}

// ------------------------------------------------------------------ softmax of one half
// Adds to 16 columns of a row's accumulator the values that are not finite and that the row sees, from the tiles that were cleaned of them.
template <int DH, bool F16>
__device__ __noinline__ void add_not_finite(const Args& a, const Segment& s, int lo, int hi, int col, float* acc) {
  const ChunkAttnCall& c = a.c;
  for (int t = s.ta; t < s.tb; ++t) {
    if (!partial_tile(s.g, c.window, t)) continue;
    for (int key = max(lo, t * KT); key <= min(hi, t * KT + KT - 1); ++key) {
      if (key <= s.g.pos0 && (c.window <= 0 || key > s.g.pos1 - c.window)) continue;         // (seen by every row: left as it was)
      const int id = c.page_table[size_t(s.b) * c.page_table_stride + key / c.page_size];
      if (unsigned(id) >= unsigned(c.num_pages)) continue;
      const uint16_t* v = reinterpret_cast<const uint16_t*>(c.v_pool) + ((size_t(id) * c.page_size + key % c.page_size) * c.Hkv + s.kvh) * DH + col;
      for (int e = 0; e < 16; ++e) {
        const uint16_t x = v[e];
        if (not_finite16<F16>(x)) acc[e] += F16 ? __half2float(__ushort_as_half(x)) : bf16_bits_to_float(x);
      }
    }
  }
}

// The weights' reference is a rounded product with the scale, the scores' own products are exact (one fma with the difference): all weights of a row have the
// same error, which the division by their sum takes away.  From 2^23 on that error could be more than a weight's type holds, and the scores' products have to be
// rounded as the reference's was.  (Infinities and the maximum of nothing are not meant.)
__device__ __forceinline__ bool far_score(float x) { return (__float_as_uint(x) & 0x7fffffffu) - 0x4b000000u < 0x7f7fffffu - 0x4b000000u; }
// The 32 weights of a row in this way: 16 words of them over the first of the scores; returns their sum.  (A function of its own, because the inner loop has no
// registers to spare: the look at the references costs a piece of 1024 tokens over 30777 others 1140 -> 1165 us and a prompt of 8192 nothing; with the
// choice in the loop they take 7 % more.)
template <bool F16>
__device__ __noinline__ float far_weights(float* x, float scale, float ref) {
  const bool far = far_score(ref);
  float sum = 0.f;
  for (int i = 0; i < 32; i += 2) {
    const float p0 = ex2_ftz(far ? __fmul_rn(x[i], scale) - ref : fmaf(x[i], scale, -ref));
    const float p1 = ex2_ftz(far ? __fmul_rn(x[i + 1], scale) - ref : fmaf(x[i + 1], scale, -ref));
    sum += p0 + p1;
    x[i / 2] = __uint_as_float(pack16<F16>(p0, p1));
  }
  return sum;
}

// The largest of three; NaN where one of them is.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// Half of a row of Q: 16-byte asynchronous copies into the operand layout, zeros for rows that are not there.
template <int DH>
__device__ __forceinline__ void copy_q(const Args& a, const Segment& s, uint32_t q_tile, int h, int row, int ch) {
  const int r = (s.turns ? 0 : h * 128) + row;
  const bool on = s.g.r0 + r < s.g.r1;
  int token, head;
  token_of(s, a, r, token, head);
  const uint16_t* src = reinterpret_cast<const uint16_t*>(a.c.q);
  if (on) src += size_t(s.q0 + token) * a.c.ldq + size_t(s.kvh * a.rep + head) * DH + ch * (DH / 2);
#pragma unroll
  for (int i = 0; i < DH / 16; ++i) cp_async16(q_tile + tile_off(row, ch * (DH / 16) + i), src + (on ? i * 8 : 0), on);
  cp_async_commit();
}
// Warp w of the half's eight: rows 32 (w % 4) .. + 31, key columns 64 (w / 4) .. + 63 of every tile.
template <int DH, bool F16>
__device__ __forceinline__ void softmax_half(const Args& a, uint8_t* sQ, Bars* bars, uint32_t tmem, int h, int tid) {
  constexpr int TILE = Shape<DH>::TILE;
  const ChunkAttnCall& c = a.c;
  volatile uint32_t* abort_flag = &bars->abort_flag;
  const int row = tid & 127, ch = (tid >> 7) & 1, quarter = row >> 5, lane = tid & 31;
  const uint32_t lane_base = uint32_t(quarter * 32) << 16;
  const uint32_t t_s = tmem + h * 128 + lane_base, t_o = tmem + 256 + h * 128 + lane_base;
  float* mine = &bars->xch[h][ch][row];
  const float* theirs = &bars->xch[h][ch ^ 1][row];
  const uint32_t my_q = smem_u32(sQ) + h * TILE;
  auto q_finish = [&]() {
    cp_async_wait<0>();
    fence_proxy_async();
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&bars->q_ready[h]));
  };
  // Both warps of a row have come here, and see what the other has written before.  This wait has no limit of its own: the two warps come here
  // equally often, also after one of the bounded waits has run out, because nothing below leaves a loop early.
  auto pair_sync = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(1 + h * 4 + quarter) : "memory"); };
  bool ok = true;
  auto wait = [&](uint64_t* bar, uint32_t parity) { if (ok) ok = mbar_wait(smem_u32(bar), parity); };
  // True in both warps of a row, or in neither.
  auto pair_and = [&](bool x) {
    int r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, %2, 64, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"(int(x)), "r"(1 + h * 4 + quarter) : "memory");
    return r != 0;
  };
  uint32_t done0 = 0, done1 = 0, shared_segs = 0;             // tiles of the halves so far, segments whose rows the halves share
  bool x_pending = false;
  int slot = 2 * blockIdx.x;                                  // where this CTA's partial results go: its first segment's, then its last one's
  // Q of segment n, if this half has tiles there
  auto q_of = [&](uint32_t n) {
    if (ok) ok = segment_wait(bars, n);
    const Segment& s = bars->seg[n % SEGS];
    if (!ok || s.end || s.nt[h] == 0) return false;
    copy_q<DH>(a, s, my_q, h, row, ch);
    return true;
  };
  if (q_of(0)) q_finish();
  for (uint32_t seg = 0;; ++seg) {
    if (ok) ok = segment_wait(bars, seg);
    if (!pair_and(ok)) { ok = false; break; }                 // (without a segment there is nothing to go through)
    const Segment& s = bars->seg[seg % SEGS];
    if (s.end) break;
    const bool turns = s.turns;
    const int nt = s.nt[h], nt_other = s.nt[h ^ 1];
    const int r = (turns ? 0 : h * 128) + row, rows = s.g.r1 - s.g.r0;              // row of the item
    const bool row_ok = r < rows;
    int token, head;
    token_of(s, a, r, token, head);
    const int hi = row_ok ? max(-1, s.pos + token) : -1;      // keys lo .. hi are seen
    const int lo = c.window > 0 ? max(0, hi - c.window + 1) : 0;
    const bool live = r - row + quarter * 32 < rows;          // (the same for both warps of a row)
    int key0 = (s.ta + (turns ? h : 0)) * KT + ch * 64;       // first of this thread's keys
    const int key_step = turns ? 2 * KT : KT;
    float m_ref = NEG, m_next = NEG, l_sum = 0.f;
    bool far = false;                                         // a row of this warp has a reference of 2^23 or more
    if (nt == 0 && q_of(seg + 1)) q_finish();
    const uint32_t done = h == 0 ? done0 : done1;
    for (int j = 0; j < nt; ++j, key0 += key_step) {
      const uint32_t n = done + j;
      wait(&bars->s_ready[h], n & 1);
      // with the last tile's scores all products that read this Q have finished: the next item's goes in
      const bool q_now = j == nt - 1 && q_of(seg + 1);
      if (live) {
        tc_fence_after();
        const bool masked = __any_sync(0xffffffffu, hi < key0 + 63 || lo > key0);
        // 32 scores of the row at a time: more would not fit into the registers, and local memory is out of reach here (its lines miss an L1 that
        // shared memory has taken nearly all of)
        float x[32];
        auto fetch = [&](int part) {
          tmem_ld32(t_s + ch * 64 + part * 32, reinterpret_cast<uint32_t*>(x));
          tmem_wait_ld32(reinterpret_cast<uint32_t*>(x));
          if (masked) {
            const int jh = hi - key0 - part * 32, jl = lo - key0 - part * 32;
#pragma unroll
            for (int i = 0; i < 32; ++i) x[i] = (i <= jh && i >= jl) ? x[i] : -INFINITY;
          }
        };
        auto largest = [&]() {
          float m0 = x[0], m1 = x[1];
#pragma unroll
          for (int i = 2; i < 30; i += 4) { m0 = max3(m0, x[i], x[i + 1]); m1 = max3(m1, x[i + 2], x[i + 3]); }
          return max3(max3(m0, m1, x[30]), x[31], x[31]);
        };
        // The threads of a row tell each other their maxima.  (What was written here a tile ago has been read: the scores of this tile were issued
        // behind the weights of all eight warps.)
        auto exchange = [&](float own) {
          *mine = own;
          pair_sync();
          return max3(own, *theirs, *theirs) * a.scale_log2;
        };
        // The accumulated values and the sum follow the reference maximum.
        auto rescale = [&](float factor) {
          l_sum *= factor;
          if (j == 0) return;
          wait(&bars->pv_done[h], (n - 1) & 1);
          tc_fence_after();
          if (lane == 0 && ch == 0) atomicAdd(c.status + STATUS_WORD_RESCALES, 1u);
#pragma unroll 1
          for (int col = ch * (DH / 2); col < (ch + 1) * (DH / 2); col += 16) {
            uint32_t o[16];
            tmem_ld16(t_o + col, o);
            tmem_wait_ld16(o);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
            tmem_st16(t_o + col, o);
          }
          tmem_st_wait();
        };
        uint64_t ls[2] = {0ull, 0ull};
        // Weights of the 32 keys, over scores of this thread that have been fetched.  They are rounded to the pools' type, which the product with the values needs:
        // half a step each, at most half a step of sum p |v| together.  In fp16 those under 2^-14 of the reference lose bits and those under 2^-25 all of them,
        // while the sum, which is of 32-bit weights, has them: 2^-25 of the reference's weight for a key at most.
        auto weights_of = [&](int part, float ref, bool any_far) {
          if (any_far) {
            float copy[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) copy[e] = x[e];
            ls[0] = add_f32x2(ls[0], pack_f32x2(far_weights<F16>(copy, a.scale_log2, ref), 0.f));
            uint32_t p[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) p[e] = __float_as_uint(copy[e]);
            tmem_st16(t_s + ch * 64 + part * 16, p);
            return;
          }
          const uint64_t scale2 = pack_f32x2(a.scale_log2, a.scale_log2), neg_m2 = pack_f32x2(-ref, -ref);
          uint32_t p[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            float x0, x1;
            unpack_f32x2(fma_f32x2(pack_f32x2(x[2 * e], x[2 * e + 1]), scale2, neg_m2), x0, x1);
            const float p0 = ex2_ftz(x0), p1 = ex2_ftz(x1);
            ls[e & 1] = add_f32x2(ls[e & 1], pack_f32x2(p0, p1));
            p[e] = pack16<F16>(p0, p1);
          }
          tmem_st16(t_s + ch * 64 + part * 16, p);
        };
        constexpr float LIMIT = F16 ? LIMIT_F16 : LIMIT_BF16;
        float mx;
        if (j == 0) {
          fetch(1);
          mx = largest();
          fetch(0);
          mx = max3(mx, largest(), largest());
          if (x_pending) wait(&bars->x_read, (shared_segs - 1) & 1);                // (an item ago the halves talked here)
          x_pending = false;
          mx = exchange(mx);
          m_ref = max3(mx, NEG, NEG);
          far = __any_sync(0xffffffffu, far_score(m_ref));
          weights_of(0, m_ref, far);
          fetch(1);
        } else {
          // The weights do not wait for the row's maximum: the reference is that of the tiles before.  Only where this tile is above it by more than
          // the weights' type can hold do they follow at once: the first 32 from their own maximum, then, when the row's is known, scaled to it (and
          // rounded a second time).
          if (__any_sync(0xffffffffu, m_next != m_ref)) {
            const float factor = m_next != m_ref ? ex2_ftz(m_ref - m_next) : 1.f;
            m_ref = m_next;
            far = __any_sync(0xffffffffu, far_score(m_ref));
            rescale(factor);
          }
          fetch(0);
          mx = largest();
          const float own = mx * a.scale_log2;
          const float ref0 = !(own <= m_ref + LIMIT) ? own : m_ref;                 // (NaN: it becomes the reference, and all of the row)
          weights_of(0, ref0, __any_sync(0xffffffffu, far_score(ref0)));
          fetch(1);
          mx = exchange(max3(mx, largest(), largest()));
          const bool over = !(mx <= m_ref + LIMIT);
          if (__any_sync(0xffffffffu, over)) {
            const float m_new = over ? mx : m_ref;
            const float factor = over ? ex2_ftz(m_ref - m_new) : 1.f, f0 = over ? ex2_ftz(ref0 - m_new) : 1.f;
            m_ref = m_new;
            far = __any_sync(0xffffffffu, far_score(m_ref));
            rescale(factor);
            tmem_st_wait();
            uint32_t p[16];
            tmem_ld16(t_s + ch * 64, p);
            tmem_wait_ld16(p);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float p0 = F16 ? __half2float(__ushort_as_half(uint16_t(p[e] & 0xffffu))) : bf16_bits_to_float(uint16_t(p[e] & 0xffffu));
              const float p1 = F16 ? __half2float(__ushort_as_half(uint16_t(p[e] >> 16))) : bf16_bits_to_float(uint16_t(p[e] >> 16));
              p[e] = pack16<F16>(p0 * f0, p1 * f0);
            }
            tmem_st16(t_s + ch * 64, p);
            const uint64_t f2 = pack_f32x2(f0, f0);
            ls[0] = fma_f32x2(ls[0], f2, 0ull); ls[1] = fma_f32x2(ls[1], f2, 0ull);
          }
        }
        m_next = mx > m_ref + LAZY ? mx : m_ref;
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars->p_half[h]));
        weights_of(1, m_ref, far);
        tmem_st_wait();
        tc_fence_before();
        float s0, s1, s2, s3;
        unpack_f32x2(ls[0], s0, s1);
        unpack_f32x2(ls[1], s2, s3);
        l_sum += (s0 + s1) + (s2 + s3);
      } else if (lane == 0) {
        mbar_arrive(smem_u32(&bars->p_half[h]));
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars->p_ready[h]));
      if (q_now) q_finish();
    }
    done0 += s.nt[0]; done1 += s.nt[1];
    // ---- read-out
    if (nt > 0) wait(&bars->pv_done[h], ((h == 0 ? done0 : done1) - 1) & 1);
    if (x_pending) wait(&bars->x_read, (shared_segs - 1) & 1);
    x_pending = false;
    if (live) {                                               // the row's sum from its two threads
      *mine = l_sum;
      pair_sync();
      l_sum = ch == 0 ? l_sum + *theirs : *theirs + l_sum;    // (in one order: the same bits in both)
      pair_sync();
    }
    float weight0 = 1.f, weight1 = 0.f;
    if (s.turns) {
      // the halves' rows are the same: maxima and sums are exchanged, and each of a row's four threads finishes a quarter of the columns
      if (ch == 0) {
        bars->xch[h][0][row] = m_ref;
        bars->xch[h][1][row] = l_sum;
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars->x_write));
      }
      wait(&bars->x_write, shared_segs & 1);
      const float m0 = bars->xch[0][0][row], l0 = bars->xch[0][1][row], m1 = bars->xch[1][0][row], l1 = bars->xch[1][1][row];
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars->x_read));
      ++shared_segs;
      x_pending = true;
      if (nt_other > 0) wait(&bars->pv_done[h ^ 1], ((h == 0 ? done1 : done0) - 1) & 1);
      m_ref = fmaxf(m0, m1);
      weight0 = ex2_ftz(m0 - m_ref); weight1 = ex2_ftz(m1 - m_ref);
      l_sum = l0 * weight0 + l1 * weight1;
    }
    tc_fence_after();
    const bool fix = *reinterpret_cast<volatile uint32_t*>(&bars->bad[seg & 15]) == seg + 1;
    const int cols = s.turns ? DH / 4 : DH / 2, col0 = (s.turns ? h * 2 + ch : ch) * cols;
    const float inv = l_sum > 0.f ? 1.f / l_sum : (l_sum == 0.f ? 0.f : l_sum);      // (nothing seen: zero; NaN stays)
    if (*abort_flag) ok = false;
    if (!s.whole && row_ok && ch == 0 && (!s.turns || h == 0)) a.ws_ml[size_t(slot) * ITEM_ROWS + r] = make_float2(m_ref, l_sum);
    if (live && (s.turns || nt > 0)) {
      token_of(s, a, r, token, head);
      const long long dst = row_ok && ok ? (long long)(s.q0 + token) * c.ldo + (s.kvh * a.rep + head) * DH : -1;
      float* part = a.ws_o + size_t(slot) * DH * ITEM_ROWS + size_t(r) * 4;
      // 16 columns of the row, of both halves where they share it
      auto read16 = [&](int col, float (&v)[16]) {
        uint32_t o[16];
        if (turns) {
          tmem_ld16(tmem + 256 + lane_base + col, o);         // (the first half always has a tile)
          tmem_wait_ld16(o);
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e] = __uint_as_float(o[e]) * weight0;
          if (s.nt[1] > 0) {
            tmem_ld16(tmem + 384 + lane_base + col, o);
            tmem_wait_ld16(o);
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = fmaf(__uint_as_float(o[e]), weight1, v[e]);
          }
        } else {
          tmem_ld16(t_o + col, o);
          tmem_wait_ld16(o);
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e] = __uint_as_float(o[e]);
        }
        if (fix && row_ok) {
          float copy[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) copy[e] = v[e];
          add_not_finite<DH, F16>(a, s, lo, hi, col, copy);
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e] = copy[e];
        }
        __syncwarp();
      };
      if (s.whole) {
        // Four lanes exchange 16-byte pieces until each holds the same piece of four rows: a store of the warp then touches 16 half lines and not 32
        // pieces of as many lines (which took the load/store unit 4000 clocks an item).  32 columns at a time, or 16 of a quarter of heads of 64.
        const int q = lane & 3;
        long long to[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i] = __shfl_sync(0xffffffffu, dst, (lane & ~3) + i);
#pragma unroll 1
        for (int col = col0; col < col0 + cols; col += 32) {
          const bool wide = col + 32 <= col0 + cols;
          uint32_t p[4][4];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float v[16];
            if (k == 0 || wide) read16(col + k * 16, v);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              p[2 * k + e / 4][e % 4] = F16 ? pack_f16_sat(v[2 * e] * inv, v[2 * e + 1] * inv, row_ok && (k == 0 || wide) ? c.status : nullptr)
                                            : pack_bf16(v[2 * e] * inv, v[2 * e + 1] * inv);
          }
#pragma unroll
          for (int m = 1; m < 4; m <<= 1) {
            const bool up = (q & m) != 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              if (k & m) continue;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? p[k][e] : p[k + m][e], m);
                if (up) p[k][e] = got;
                else p[k + m][e] = got;
              }
            }
          }
          if (wide || q < 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (to[i] >= 0)
                *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(c.o) + to[i] + col + q * 8) = make_uint4(p[i][0], p[i][1], p[i][2], p[i][3]);
          }
          __syncwarp();
        }
      } else {
#pragma unroll 1
        for (int col = col0; col < col0 + cols; col += 16) {
          float v[16];
          read16(col, v);
          // [column group][row][4]: the lanes of a warp write neighbouring 16 bytes
          if (row_ok && ok) {
#pragma unroll
            for (int e = 0; e < 16; e += 4) *reinterpret_cast<float4*>(part + size_t((col + e) / 4) * ITEM_ROWS * 4) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
          }
          __syncwarp();
        }
      }
    }
    tc_fence_before();
    __syncwarp();
    if (lane == 0) {
      if (turns) {
        if (s.nt[0] > 0) mbar_arrive(smem_u32(&bars->o_free[0]));
        if (s.nt[1] > 0) mbar_arrive(smem_u32(&bars->o_free[1]));
      } else if (nt > 0) {
        mbar_arrive_n(smem_u32(&bars->o_free[h]), 2);
      }
    }
    if (lane == 0) segment_read(bars, seg);
    slot = 2 * blockIdx.x + 1;
  }
  if (!ok) { if (!*abort_flag) atomicExch(c.status, STATUS_TIMEOUT_EPILOGUE); *abort_flag = 1; }
  tc_fence_before();
}

template <int DH, bool F16>
__global__ void __launch_bounds__(THREADS, 1)
chunk_attn_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ Args a) {
  constexpr int NK = Shape<DH>::NK, NV = Shape<DH>::NV, TILE = Shape<DH>::TILE;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* sQ = smem;
  uint8_t* ring_k = smem + 2 * TILE;
  uint8_t* ring_v = ring_k + NK * TILE;
  Bars* bars = reinterpret_cast<Bars*>(ring_v + NV * TILE);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (smem_u32(smem) & 1023) {                                // the swizzled tiles need a 1 KiB-aligned base
    pdl_wait();
    if (tid == 0) atomicExch(a.c.status, STATUS_BAD_SMEM_BASE);
    return;
  }
  if (tid == 0) {
    if (a.box_rows) { tma_prefetch_desc(&tmK); tma_prefetch_desc(&tmV); }
    for (int i = 0; i < NK; ++i) {
      mbar_init(smem_u32(&bars->k_full[i]), 1);
      mbar_init(smem_u32(&bars->k_empty[i]), 1);
    }
    for (int i = 0; i < NV; ++i) {
      mbar_init(smem_u32(&bars->v_full[i]), 1);
      mbar_init(smem_u32(&bars->v_empty[i]), 1);
      mbar_init(smem_u32(&bars->v_raw[i]), 1);
    }
    for (int h = 0; h < 2; ++h) {
      mbar_init(smem_u32(&bars->q_ready[h]), 8);
      mbar_init(smem_u32(&bars->s_ready[h]), 1);
      mbar_init(smem_u32(&bars->p_half[h]), 8);
      mbar_init(smem_u32(&bars->p_ready[h]), 8);
      mbar_init(smem_u32(&bars->pv_done[h]), 1);
      mbar_init(smem_u32(&bars->o_free[h]), 16);
    }
    mbar_init(smem_u32(&bars->x_write), 8);
    mbar_init(smem_u32(&bars->x_read), 16);
    mbar_init(smem_u32(&bars->drain), 1);
    for (int i = 0; i < SEGS; ++i) {
      mbar_init(smem_u32(&bars->seg_full[i]), 1);
      mbar_init(smem_u32(&bars->seg_empty[i]), 19);           // sixteen softmax warps, two producers, the MMA thread
    }
    bars->abort_flag = 0;
    for (int i = 0; i < 16; ++i) bars->bad[i] = 0;
    fence_mbar_init();
  }
  if (warp == 17) {
    tmem_alloc(smem_u32(&bars->tmem_base), 512);
    tmem_relinquish();
  }
  pdl_wait();
  pdl_trigger();
  const bool work = make_plan(a, bars, reinterpret_cast<long long*>(ring_k));
  fence_proxy_async();                                        // (the plan's sums lay where the copies now go)
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars->tmem_base;      // scores (and the weights over them) of the halves in columns 0 and 128, accumulators in 256 and 384
  if (!work) {
    // nothing to do here (uniform for the CTA)
  } else if (warp < 16) {
    softmax_half<DH, F16>(a, sQ, bars, tmem, warp >> 3, tid);
  } else {
    if (warp == 16) {
      produce<DH, false>(a, &tmK, ring_k, bars, lane);
    } else if (warp == 18) {
      produce<DH, true>(a, &tmV, ring_v, bars, lane);
    } else if (warp == 17) {
      if (elect_one()) issue_mmas<DH, F16>(a, sQ, ring_k, ring_v, bars, tmem);
      __syncwarp();
    } else {
      lead_and_clean<DH, F16>(a, ring_v, bars, lane);
    }
  }
  __syncthreads();
  if (warp == 17) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// ------------------------------------------------------------------ joining items that a cut went through
// One block per (CTA, 32 rows).  The CTA whose part an item begins in speaks for it: its partial result and those of the parts behind, in order.
// Lane = row, warp = 16 (or 8) columns, so that the loads follow the partials' layout.  All that the kernel waits for in turn is the places, then the
// rows' maxima and sums, then the partials, four under way per thread (with the places one after the other and the request's lengths behind them a
// single token's call took 1.4 us more).
template <int DH, bool F16>
__global__ void __launch_bounds__(256) chunk_attn_join_kernel(const __grid_constant__ Args a) {
  pdl_wait();
  pdl_trigger();
  constexpr int COLS = DH / 8, ROW = DH * 2 + 16;
  __shared__ __align__(16) uint8_t tile[32 * ROW];
  __shared__ float2 ml[MAX_CTAS][32];
  const ChunkAttnCall& c = a.c;
  const int me = blockIdx.x, next = me + a.group, lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  if (next >= MAX_CTAS) return;
  const int count = *a.ws_count * a.group, behind = next + lane * a.group;
  const int4 mine = a.ws_start[me], x = a.ws_start[next], item = a.ws_start[a.units + next];
  const int4 y = behind < MAX_CTAS ? a.ws_start[behind] : make_int4(-1, 0, 0, 0);     // (of parts without work: anything)
  if (next >= count) return;
  auto same = [&](const int4& p) { return p.x == x.x && p.y == x.y && p.z == x.z; };
  if (x.w == 0 || (same(mine) && mine.w > 0)) return;         // no cut through an item here, or an earlier CTA speaks for it
  const int first = 2 * me + (same(mine) ? 0 : 1);
  // (a part that begins further on in the same item has its place behind the item's begin)
  unsigned run = __ballot_sync(0xffffffffu, behind < count && same(y));
  int n = 1 + (run == 0xffffffffu ? 32 : __ffs(~run) - 1);
  for (int base = next + 32 * a.group; run == 0xffffffffu; base += 32 * a.group) {
    const int at = base + lane * a.group;
    run = __ballot_sync(0xffffffffu, at < count && same(a.ws_start[at < count ? at : me]));
    n += run == 0xffffffffu ? 32 : __ffs(~run) - 1;
  }
  const int kvh = x.y * a.group + me % a.group, r = blockIdx.y * 32 + lane, rows = item.w;
  if (int(blockIdx.y) * 32 >= rows) return;
  auto slot = [&](int i) { return size_t(i == 0 ? first : 2 * (me + i * a.group)); };
  for (int i = w; i < n; i += 8) ml[i][lane] = r < rows ? a.ws_ml[slot(i) * ITEM_ROWS + r] : make_float2(NEG, 0.f);
  __syncthreads();
  if (r < rows) {
    float m = NEG;
    for (int i = 0; i < n; ++i) m = fmaxf(m, ml[i][lane].x);
    float acc[COLS], sum = 0.f;
#pragma unroll
    for (int e = 0; e < COLS; ++e) acc[e] = 0.f;
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      const float2 part = ml[i][lane];
      // a half whose rows saw nothing in that part may not even have written its accumulator
      const bool none = part.x == NEG && part.y == 0.f;
      const float f = none ? 0.f : ex2_ftz(part.x - m);
      sum += part.y * f;
      const float* src = a.ws_o + slot(i) * DH * ITEM_ROWS + (size_t(w * COLS) / 4 * ITEM_ROWS + r) * 4;
#pragma unroll
      for (int e = 0; e < COLS; e += 4) {
        const float4 v = none ? make_float4(0.f, 0.f, 0.f, 0.f) : *reinterpret_cast<const float4*>(src + size_t(e) * ITEM_ROWS);
        acc[e] += v.x * f; acc[e + 1] += v.y * f; acc[e + 2] += v.z * f; acc[e + 3] += v.w * f;
      }
    }
    const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);
#pragma unroll
    for (int e = 0; e < COLS; e += 8) {
      uint32_t p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        p[i] = F16 ? pack_f16_sat(acc[e + 2 * i] * inv, acc[e + 2 * i + 1] * inv, c.status) : pack_bf16(acc[e + 2 * i] * inv, acc[e + 2 * i + 1] * inv);
      *reinterpret_cast<uint4*>(tile + lane * ROW + (w * COLS + e) * 2) = make_uint4(p[0], p[1], p[2], p[3]);
    }
  }
  __syncthreads();
  constexpr int LANES = DH / 8;                               // lanes that write a row
  for (int i = threadIdx.x; i < 32 * LANES; i += 256) {
    const int rl = i / LANES, row = int(blockIdx.y) * 32 + rl;
    const uint32_t at = uint32_t(item.z + row), t = (at * a.inv_rep) >> 20;          // (token_of)
    if (row < rows)
      *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(c.o) + size_t(item.x + item.y + int(t)) * c.ldo + size_t(kvh * a.rep + int(at - t * a.rep)) * DH + (i % LANES) * 8) =
          *reinterpret_cast<const uint4*>(tile + rl * ROW + (i % LANES) * 16);
  }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// 4-D view of a pool [num_pages, page_size, Hkv, dh]; a box is box_rows rows of one page, one KV head, 64 values.
bool pool_tmap(CUtensorMap* tm, const void* pool, const ChunkAttnCall& c, int box_rows, std::string* err) {
  static const EncodeTiledFn enc = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) p = nullptr;
    return reinterpret_cast<EncodeTiledFn>(p);
  }();
  if (!enc) { *err = "cuTensorMapEncodeTiled is not available"; return false; }
  cuuint64_t dims[4] = {cuuint64_t(c.dh), cuuint64_t(c.Hkv), cuuint64_t(c.page_size), cuuint64_t(c.num_pages)};
  cuuint64_t strides[3] = {cuuint64_t(c.dh) * 2, cuuint64_t(c.Hkv) * c.dh * 2, cuuint64_t(c.page_size) * c.Hkv * c.dh * 2};
  cuuint32_t box[4] = {64, 1, cuuint32_t(box_rows), 1}, estr[4] = {1, 1, 1, 1};
  const CUresult r = enc(tm, c.f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(pool), dims, strides, box, estr,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) { *err = "cuTensorMapEncodeTiled (KV pool) failed with CUresult " + std::to_string(int(r)); return false; }
  return true;
}

template <int DH, bool F16>
cudaError_t launch_for(const Args& a, cudaStream_t stream, const CUtensorMap& tmK, const CUtensorMap& tmV) {
  constexpr size_t smem = smem_bytes(Shape<DH>::TILE, Shape<DH>::NK + Shape<DH>::NV);
  static_assert(smem <= 232448, "shared memory of an SM");
  static bool done[MAX_DEVICES] = {};
  static int ctas[MAX_DEVICES] = {};
  cudaError_t e = once_per_device(done, [&](int dev) {
    int sms = 0;
    cudaError_t e1 = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    ctas[dev] = sms < MAX_CTAS ? sms : MAX_CTAS;
    if (e1 == cudaSuccess) e1 = cudaFuncSetAttribute(chunk_attn_kernel<DH, F16>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem));
    return e1;
  });
  if (e != cudaSuccess) return e;
  const int n = ctas[current_device()];
  e = launch_pdl(chunk_attn_kernel<DH, F16>, dim3(n), dim3(THREADS), smem, stream, tmK, tmV, a);
  if (e != cudaSuccess) return e;
  const long long rows = (long long)a.c.T * a.rep;            // no item has more rows than this
  return launch_pdl(chunk_attn_join_kernel<DH, F16>, dim3(n, unsigned((rows < ITEM_ROWS ? rows + 31 : ITEM_ROWS) / 32)), dim3(256), 0, stream, a);
}

}  // namespace

static size_t own_workspace_bytes(int dh) { return size_t(2 * MAX_CTAS) * ITEM_ROWS * (size_t(dh) * 4 + 8) + 2 * MAX_CTAS * sizeof(int4) + 256; }
size_t chunk_attn_workspace_bytes(int, int, int dh) { return own_workspace_bytes(dh) + chunk_few_workspace_bytes(dh); }

cudaError_t chunk_attn_launch(const ChunkAttnCall& c, cudaStream_t stream, std::string* err) {
  Args a{};
  a.c = c;
  if (chunk_few_takes(c)) {
    const cudaError_t e = chunk_few_launch(c, reinterpret_cast<uint8_t*>(c.ws) + own_workspace_bytes(c.dh), stream);
    if (e != cudaSuccess || chunk_few_takes_all(c)) return e;
    a.kind = KIND_MANY;
  }
  a.rep = c.Hq / c.Hkv;
  a.inv_rep = ((1u << 20) + a.rep - 1) / a.rep;
  a.scale_log2 = c.scale * 1.4426950408889634f;
  // the largest group of heads that leaves at most four SMs without work
  for (a.group = c.Hkv < 16 ? c.Hkv : 16; a.group > 1 && (c.Hkv % a.group || MAX_CTAS % a.group > 4); --a.group) {}
  a.box_rows = 0;
  if (c.page_size % 8 == 0)
    for (a.box_rows = 8; a.box_rows < KT && c.page_size % (2 * a.box_rows) == 0;) a.box_rows *= 2;
  a.ws_o = reinterpret_cast<float*>(c.ws);
  a.ws_ml = reinterpret_cast<float2*>(a.ws_o + size_t(2 * MAX_CTAS) * ITEM_ROWS * c.dh);
  a.ws_start = reinterpret_cast<int4*>(a.ws_ml + size_t(2 * MAX_CTAS) * ITEM_ROWS);
  a.ws_count = reinterpret_cast<int*>(a.ws_start + 2 * MAX_CTAS);
  a.units = MAX_CTAS;
  CUtensorMap tmK{}, tmV{};
  if (a.box_rows && (!pool_tmap(&tmK, c.k_pool, c, a.box_rows, err) || !pool_tmap(&tmV, c.v_pool, c, a.box_rows, err))) return cudaErrorInvalidValue;
  if (c.dh == 64) return c.f16 ? launch_for<64, true>(a, stream, tmK, tmV) : launch_for<64, false>(a, stream, tmK, tmV);
  return c.f16 ? launch_for<128, true>(a, stream, tmK, tmV) : launch_for<128, false>(a, stream, tmK, tmV);
}

}  // namespace hspec
