// Verification of drafted tokens against the target's probabilities from given uniform numbers (App. A).
//
//   p = softmax(z_T / temperature), q = softmax(z_D / temperature) (or all of it on the drafted token where the drafter takes the arg-max)
//   draft i stands if every earlier one does, p_i(x_i) > 0 and min(1, p_i(x_i) / q_i(x_i)) >= alpha_i
//   behind the n drafts that stand one token more: from max(0, p_n - q_n) where draft n was refused, from p_n where none was; the lowest v whose
//   cumulative sum exceeds u times the whole
//
// Both answers are integers that hang on a comparison of real numbers, and they are decided as if in 64 bits: each comparison is made with 32-bit
// exponentials first and made again with 64-bit ones where the numbers come so near to one another that the first could be wrong.
//
// Three steps, a launch each, or the last two in one.  The first takes one (request, position) per cluster of blocks, reads the target's and the
// drafter's row once and decides whether the position would be refused; items are started position by position, and one whose request is known to have
// been refused before is not read.  The second takes one request per cluster and samples with 32-bit weights.  The third does so with 64-bit weights for
// the requests whose uniform number came within some 2^-16 of a border between two tokens: what falls among the many tokens of next to no weight.  The
// first two are bound by memory, the third by the latency of its 64-bit operations (their pipe is busy for a fifth of the time; 128 requests of 152 064
// tokens: 238 us in 64 bits alone, 70 and 64 in two steps).
#include "common.cuh"
#include "kernels.h"

#include <cfloat>
#include <cmath>
#include <type_traits>

namespace hspec {

namespace {

constexpr int VT = 512;              // threads of a block
constexpr int VW = VT / 32;
constexpr int MAX_S = 16;            // most blocks of a cluster
constexpr float LOG2E = 1.4426950408889634f;

// A logit as it counts: NaN as -infinity (as in every arg-max of this library), +infinity as the largest finite number.
__device__ __forceinline__ float logit(float v) { return fminf(fmaxf(v, -INFINITY), FLT_MAX); }
__device__ __forceinline__ float value_of(float v) { return v; }
__device__ __forceinline__ float value_of(__half v) { return __half2float(v); }
__device__ __forceinline__ float value_of(__nv_bfloat16 v) { return __bfloat162float(v); }

struct Row { const void* z; int dtype; };
__device__ __forceinline__ Row row_at(const void* base, int dtype, long long ld, long long row) {
  return Row{reinterpret_cast<const uint8_t*>(base) + size_t(row) * size_t(ld) * (dtype == CHUNK_F32 ? 4 : 2), dtype};
}
__device__ __forceinline__ float load_logit(const Row& r, int i) {
  if (r.dtype == CHUNK_F32) return logit(reinterpret_cast<const float*>(r.z)[i]);
  if (r.dtype == CHUNK_F16) return logit(value_of(reinterpret_cast<const __half*>(r.z)[i]));
  return logit(value_of(reinterpret_cast<const __nv_bfloat16*>(r.z)[i]));
}

// 16 bytes of a row as logits, or as they are.
template <bool LOGITS = true>
__device__ __forceinline__ void unpack16(const uint4& w, float (&v)[4], float) {
  v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
#pragma unroll
  for (int j = 0; j < 4; ++j) if (LOGITS) v[j] = logit(v[j]);
}
template <bool LOGITS = true>
__device__ __forceinline__ void unpack16(const uint4& w, float (&v)[8], __half) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x[j]));
    v[2 * j] = LOGITS ? logit(f.x) : f.x;
    v[2 * j + 1] = LOGITS ? logit(f.y) : f.y;
  }
}
template <bool LOGITS = true>
__device__ __forceinline__ void unpack16(const uint4& w, float (&v)[8], __nv_bfloat16) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float a = __uint_as_float(x[j] << 16), b = __uint_as_float(x[j] & 0xffff0000u);
    v[2 * j] = LOGITS ? logit(a) : a;
    v[2 * j + 1] = LOGITS ? logit(b) : b;
  }
}
// A word of logits that are all -infinity.
__device__ __forceinline__ uint32_t nothing(float) { return 0xff800000u; }
__device__ __forceinline__ uint32_t nothing(__half) { return 0xfc00fc00u; }
__device__ __forceinline__ uint32_t nothing(__nv_bfloat16) { return 0xff80ff80u; }
// Calls f(first index, values of N neighbours) for this thread's share of [begin, end): 16-byte loads, U of them in flight (behind the last: values
// of -infinity), scalar loads in front of the first 16-byte boundary and behind the last.  LOGITS: values as they count, else words as they are.
template <int U, bool LOGITS = true, typename T, typename F>
__device__ __forceinline__ void walk(const T* z, int begin, int end, F f) {
  constexpr int N = 16 / sizeof(T);
  const int off = int((reinterpret_cast<uintptr_t>(z + begin) & 15) / sizeof(T));
  const int head = min(end, begin + (off ? N - off : 0)), n16 = (end - head) / N;
  for (int i = begin + int(threadIdx.x); i < head; i += VT) { float v[1] = {logit(value_of(z[i]))}; f(i, v); }
  const uint4* p = reinterpret_cast<const uint4*>(z + head);
  const uint32_t none = nothing(T());
  uint4 next[U];
  auto fetch = [&](int i0) {
#pragma unroll
    for (int u = 0; u < U; ++u) next[u] = i0 + u * VT < n16 ? __ldg(p + i0 + u * VT) : make_uint4(none, none, none, none);
  };
  fetch(threadIdx.x);
  for (int i0 = threadIdx.x; i0 < n16; i0 += U * VT) {
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = next[u];
    fetch(i0 + U * VT);                           // (under way while these are dealt with)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[N];
      unpack16<LOGITS>(w[u], v, T());
      f(head + (i0 + u * VT) * N, v);
    }
  }
  for (int i = head + n16 * N + int(threadIdx.x); i < end; i += VT) { float v[1] = {logit(value_of(z[i]))}; f(i, v); }
}
template <int U, bool LOGITS = true, typename F>
__device__ __forceinline__ void walk(const Row& r, int begin, int end, F f) {
  if (r.dtype == CHUNK_F32) walk<U, LOGITS>(reinterpret_cast<const float*>(r.z), begin, end, f);
  else if (r.dtype == CHUNK_F16) walk<U, LOGITS>(reinterpret_cast<const __half*>(r.z), begin, end, f);
  else walk<U, LOGITS>(reinterpret_cast<const __nv_bfloat16*>(r.z), begin, end, f);
}

struct MaxSum { float mx, sum; };
__device__ __forceinline__ MaxSum merged(MaxSum a, MaxSum b, float c) {
  const float m = fmaxf(a.mx, b.mx);
  if (m == -INFINITY) return a;
  return MaxSum{m, (a.mx > -INFINITY ? a.sum * ex2_ftz((a.mx - m) * c) : 0.f) + (b.mx > -INFINITY ? b.sum * ex2_ftz((b.mx - m) * c) : 0.f)};
}
// One pass: the running maximum and the sum of 2^((z - max) c) over this thread's share.  16 values at a time with one maximum and one rescaling, two
// values to an instruction where there is one (14 instructions a value were more than the memory leaves time for; these are 5).  Without LOGITS values
// are taken as they are: NaN and +infinity make the sum NaN, and such a share is gone through once more with every value looked at.
template <bool LOGITS, typename T>
__device__ __forceinline__ MaxSum sum_share(const T* z, int begin, int end, float c) {
  constexpr int N = 16 / sizeof(T), U = 4, G = 16 / N;          // values of a word, words under way, words of 16 values
  float mx = -FLT_MAX, sum = 0.f;
  auto one = [&](float v) {
    const float m = fmaxf(mx, v);
    sum = sum * ex2_ftz((mx - m) * c) + ex2_ftz((v - m) * c);
    mx = m;
  };
  const int off = int((reinterpret_cast<uintptr_t>(z + begin) & 15) / sizeof(T));
  const int head = min(end, begin + (off ? N - off : 0)), n16 = (end - head) / N;
  for (int i = begin + int(threadIdx.x); i < head; i += VT) one(LOGITS ? logit(value_of(z[i])) : value_of(z[i]));
  for (int i = head + n16 * N + int(threadIdx.x); i < end; i += VT) one(LOGITS ? logit(value_of(z[i])) : value_of(z[i]));
  const uint4* p = reinterpret_cast<const uint4*>(z + head);
  const uint32_t none = nothing(T());
  uint4 next[U];
  auto fetch = [&](int i0) {
#pragma unroll
    for (int u = 0; u < U; ++u) next[u] = i0 + u * VT < n16 ? __ldg(p + i0 + u * VT) : make_uint4(none, none, none, none);
  };
  const uint64_t c2 = pack_f32x2(c, c);
  fetch(threadIdx.x);
  for (int i0 = threadIdx.x; i0 < n16; i0 += U * VT) {
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = next[u];
    fetch(i0 + U * VT);                           // (under way while these are dealt with)
#pragma unroll
    for (int g = 0; g < U / G; ++g) {
      float v[16];
#pragma unroll
      for (int u = 0; u < G; ++u) {
        float x[N];
        unpack16<LOGITS>(w[g * G + u], x, T());
#pragma unroll
        for (int j = 0; j < N; ++j) v[u * N + j] = x[j];
      }
      float m = mx;
#pragma unroll
      for (int j = 0; j < 16; j += 2) m = fmaxf(fmaxf(m, v[j]), v[j + 1]);
      const uint64_t neg = pack_f32x2(-m, -m);
      uint64_t part[2] = {0ull, 0ull};
#pragma unroll
      for (int j = 0; j < 16; j += 2) {
        float e0, e1;
        unpack_f32x2(fma_f32x2(add_f32x2(pack_f32x2(v[j], v[j + 1]), neg), c2, 0ull), e0, e1);
        part[(j >> 1) & 1] = add_f32x2(part[(j >> 1) & 1], pack_f32x2(ex2_ftz(e0), ex2_ftz(e1)));
      }
      float s0, s1;
      unpack_f32x2(add_f32x2(part[0], part[1]), s0, s1);
      sum = sum * ex2_ftz((mx - m) * c) + (s0 + s1);
      mx = m;
    }
  }
  return MaxSum{mx, sum};
}
// (Functions of their own, so that the three types' loops do not share the registers of the kernel around them; the first with the second inside it keeps its
// arguments past the loop, and 128 requests of 152 064 tokens take 292 us, not 288.)
__device__ __noinline__ MaxSum sum_row_careful(Row r, int begin, int end, float c) {
  if (r.dtype == CHUNK_F32) return sum_share<true>(reinterpret_cast<const float*>(r.z), begin, end, c);
  if (r.dtype == CHUNK_F16) return sum_share<true>(reinterpret_cast<const __half*>(r.z), begin, end, c);
  return sum_share<true>(reinterpret_cast<const __nv_bfloat16*>(r.z), begin, end, c);
}
__device__ __noinline__ MaxSum sum_row_quick(Row r, int begin, int end, float c) {
  MaxSum x = r.dtype == CHUNK_F32   ? sum_share<false>(reinterpret_cast<const float*>(r.z), begin, end, c)
             : r.dtype == CHUNK_F16 ? sum_share<false>(reinterpret_cast<const __half*>(r.z), begin, end, c)
                                    : sum_share<false>(reinterpret_cast<const __nv_bfloat16*>(r.z), begin, end, c);
  return x;
}
__device__ __forceinline__ MaxSum sum_row(Row r, int begin, int end, float c) {
  MaxSum x = sum_row_quick(r, begin, end, c);
  if (x.sum != x.sum) x = sum_row_careful(r, begin, end, c);
  if (x.sum == 0.f) x.mx = -INFINITY;             // (nothing but -infinity)
  return x;
}
// The largest value and its lowest index over this thread's share, as one number (argmax_key).  A word's maximum first, and its place where it is a new one.
__device__ __noinline__ unsigned long long key_row(Row r, int begin, int end) {
  float mx = -INFINITY;
  int at = begin;
  walk<4, false>(r, begin, end, [&](int i, auto& v) {
    constexpr int N = sizeof(v) / sizeof(float);
    float m = v[0];
#pragma unroll
    for (int j = 1; j < N; ++j) m = fmaxf(m, v[j]);           // (NaN gives way to a number)
    m = logit(m);                                             // (a word of nothing but NaN)
    if (m > mx) {
      mx = m;
#pragma unroll
      for (int j = N - 1; j >= 0; --j) if (logit(v[j]) == m) at = i + j;
    }
  });
  return begin < end ? argmax_key(mx, at) : 0;
}

// e^((z - m) / t) in 64 bits; nothing where z is -infinity.  (As the square of e^(x / 2) where 64 bits end: the function itself may be off by 2^-1074 there,
// which is all or nothing.)
__device__ __forceinline__ double weight64(float z, float m, double inv_t) {
  if (!(z > -INFINITY)) return 0.0;
  const double x = (double(z) - double(m)) * inv_t, e = exp(x > -700.0 ? x : 0.5 * x);
  return x > -700.0 ? e : e * e;
}
// Calls f(4 U values) for this thread's share of [begin, end), begin a multiple of 4, by index and not by address as walk does: sums over equal rows are then equal
// to the bit wherever the rows lie and whatever type holds them, so that p / q of them is 1 and p - q nothing.  Four neighbours at a time, one load where the row
// begins on a boundary of four; behind the last: -infinity.
template <int U, typename T, typename F>
__device__ __forceinline__ void walk_by_index(const T* z, int begin, int end, F f) {
  struct __align__(4 * sizeof(T)) Four { T v[4]; };
  const bool whole = reinterpret_cast<uintptr_t>(z) % sizeof(Four) == 0;
  Four next[U];
  auto fetch = [&](int i0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * 4 * VT;
      if (whole && i + 4 <= end) {
        next[u] = *reinterpret_cast<const Four*>(z + i);
      } else if (i < end) {
#pragma unroll
        for (int j = 0; j < 4; ++j) next[u].v[j] = z[min(i + j, end - 1)];
      }
    }
  };
  fetch(begin + int(threadIdx.x) * 4);
  for (int i0 = begin + int(threadIdx.x) * 4; i0 < end; i0 += U * 4 * VT) {
    float v[4 * U];
#pragma unroll
    for (int j = 0; j < 4 * U; ++j) v[j] = i0 + (j / 4) * 4 * VT + j % 4 < end ? logit(value_of(next[j / 4].v[j % 4])) : -INFINITY;
    fetch(i0 + U * 4 * VT);                       // (under way while these are dealt with)
    f(v);
  }
}
template <int U, typename F>
__device__ __forceinline__ void walk_by_index(const Row& r, int begin, int end, F f) {
  if (r.dtype == CHUNK_F32) walk_by_index<U>(reinterpret_cast<const float*>(r.z), begin, end, f);
  else if (r.dtype == CHUNK_F16) walk_by_index<U>(reinterpret_cast<const __half*>(r.z), begin, end, f);
  else walk_by_index<U>(reinterpret_cast<const __nv_bfloat16*>(r.z), begin, end, f);
}
template <typename W>
__device__ __forceinline__ double sum_row64(const Row& r, int begin, int end, float m, W weigh) {
  double s0 = 0.0, s1 = 0.0;
  if (m > -INFINITY)
    walk_by_index<1>(r, begin, end, [&](auto& v) {
#pragma unroll
      for (int j = 0; j < 4; ++j) (j & 1 ? s1 : s0) += weigh(v[j]);
    });
  return s0 + s1;
}

__device__ __forceinline__ double shfl_xor64(double v, int off) { return __shfl_xor_sync(0xffffffffu, v, off); }
__device__ __forceinline__ double shfl_up64(double v, int off) { return __shfl_up_sync(0xffffffffu, v, off); }

__device__ __forceinline__ void st_cluster_f64(const void* p, int rank, double v) {
  asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(mapa_rank(smem_u32(p), uint32_t(rank))), "d"(v) : "memory");
}
__device__ __forceinline__ void st_cluster_u64(const void* p, int rank, unsigned long long v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(mapa_rank(smem_u32(p), uint32_t(rank))), "l"(v) : "memory");
}
__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_or_block_sync(int S) {
  if (S > 1) cluster_sync_all();
  else __syncthreads();
}

// Sum over the cluster's threads, the same bits in every one of them: lanes, warps and blocks are added in a fixed order.
struct Reduce64 {
  double warp[2][VW];
  double block[2][MAX_S];
};
__device__ __forceinline__ void cluster_sum2(Reduce64& sh, int S, int rank, double& a, double& b) {
  for (int off = 16; off > 0; off >>= 1) { a += shfl_xor64(a, off); b += shfl_xor64(b, off); }
  if ((threadIdx.x & 31) == 0) { sh.warp[0][threadIdx.x >> 5] = a; sh.warp[1][threadIdx.x >> 5] = b; }
  __syncthreads();
  if (threadIdx.x < unsigned(S)) {
    double x = 0.0, y = 0.0;
    for (int w = 0; w < VW; ++w) { x += sh.warp[0][w]; y += sh.warp[1][w]; }
    st_cluster_f64(&sh.block[0][rank], threadIdx.x, x);
    st_cluster_f64(&sh.block[1][rank], threadIdx.x, y);
  }
  cluster_or_block_sync(S);
  a = b = 0.0;
  for (int i = 0; i < S; ++i) { a += sh.block[0][i]; b += sh.block[1][i]; }
  cluster_or_block_sync(S);              // (the arrays are free again)
}

struct ReduceKey {
  unsigned long long warp[VW], block[MAX_S];
};
__device__ __forceinline__ unsigned long long cluster_max_key(ReduceKey& sh, int S, int rank, unsigned long long k) {
  for (int off = 16; off > 0; off >>= 1) { const unsigned long long o = __shfl_xor_sync(0xffffffffu, k, off); k = o > k ? o : k; }
  if ((threadIdx.x & 31) == 0) sh.warp[threadIdx.x >> 5] = k;
  __syncthreads();
  if (threadIdx.x < unsigned(S)) {
    unsigned long long x = 0;
    for (int w = 0; w < VW; ++w) x = sh.warp[w] > x ? sh.warp[w] : x;
    st_cluster_u64(&sh.block[rank], threadIdx.x, x);
  }
  cluster_or_block_sync(S);
  k = 0;
  for (int i = 0; i < S; ++i) k = sh.block[i] > k ? sh.block[i] : k;
  cluster_or_block_sync(S);
  return k;
}

// Rows and drafts of a request, and its temperature (not above zero, or NaN: greedy).  That is held where it and its inverse are numbers of full 32 bits.
struct Request { int row0, drafts; float t; bool greedy; };
__device__ __forceinline__ Request request(const VerifyCall& c, int b) {
  Request r;
  int lo = b * (c.k + 1), hi = lo + c.k + 1;
  if (c.cu_q) { lo = c.cu_q[b]; hi = c.cu_q[b + 1]; }
  r.row0 = min(max(lo, 0), c.T);
  r.drafts = min(min(max(hi, r.row0), c.T) - r.row0 - 1, c.k);     // -1: no row at all, nothing to sample from (held first: a far offset's difference wraps)
  const float t = c.temperature ? c.temperature[b] : 1.f;
  r.t = fminf(fmaxf(t, 1e-36f), 1e36f);
  r.greedy = !(t > 0.f);
  return r;
}
// Place of a token in the drafter's vocabulary, or -1.
__device__ __forceinline__ int draft_index(const VerifyCall& c, int id) {
  if (!c.vocab_map) return id < c.Vd ? id : -1;
  int lo = 0, hi = c.Vd;
  while (lo < hi) { const int mid = (lo + hi) >> 1; if (c.vocab_map[mid] < id) lo = mid + 1; else hi = mid; }
  return lo < c.Vd && c.vocab_map[lo] == id ? lo : -1;
}
__device__ __forceinline__ void share_of(int n, int S, int rank, int& begin, int& end) {
  const int per = ((n + S - 1) / S + 7) & ~7;
  begin = min(n, rank * per);
  end = min(n, begin + per);
}

__global__ void verify_init_kernel(int* first, int B) {
  pdl_wait();
  pdl_trigger();
  for (int i = threadIdx.x; i < B; i += blockDim.x) first[i] = 0x7fffffff;
}

// One item whose ratio is so near to alpha that the 32-bit sums do not decide: the same in 64 bits.  (Rare, and kept out of the registers of the rest.)
__device__ __noinline__ void verify_row64(const VerifyCall& c, const VerifyScratch& s, int S, int rank, int skip, int i, int b, Reduce64& sh_sum, float mt,
                                          float md) {
  const Request r = request(c, b);
  const int at = b * c.k + i, id = c.ids[at];
  const bool both = c.draft != nullptr;
  const Row zt = row_at(c.target, c.t_dtype, c.ld_t, r.row0 + i), zd = both ? row_at(c.draft, c.d_dtype, c.ld_d, at) : zt;
  int begin, end, dbegin, dend;
  share_of(c.V, S, rank, begin, end);
  share_of(c.Vd, S, rank, dbegin, dend);
  const double inv_t = 1.0 / double(r.t);
  double st = sum_row64(zt, begin, end, mt, [&](float z) { return weight64(z, mt, inv_t); });
  double sd = both ? sum_row64(zd, dbegin, dend, md, [&](float z) { return weight64(z, md, inv_t); }) : 0.0;
  cluster_sum2(sh_sum, S, rank, st, sd);
  if (rank == 0 && threadIdx.x == 0) {
    const double p = weight64(load_logit(zt, id), mt, inv_t) / st;
    const int di = both ? draft_index(c, id) : -1;
    const double q = !both ? 1.0 : di >= 0 ? weight64(load_logit(zd, di), md, inv_t) / sd : 0.0;
    const int verdict = p > 0.0 && (q > 0.0 ? p / q : INFINITY) >= double(c.alpha[at]);
    s.verdict[at] = verdict;
    if (skip && !verdict) atomicMin(s.first + b, i);
  }
}

__device__ __forceinline__ void verify_row(const VerifyCall& c, const VerifyScratch& s, int S, int rank, int skip, int i, int b, MaxSum (&sh_warp)[2][VW],
                                           unsigned long long (&sh_block)[2][8], Reduce64& sh_sum, ReduceKey& sh_key, float (&sh_max)[2], int& sh_near, float err) {
  const Request r = request(c, b);
  const int at = b * c.k + i, id = c.ids[at];
  const Row zt = row_at(c.target, c.t_dtype, c.ld_t, r.row0 + i);
  int begin, end;
  share_of(c.V, S, rank, begin, end);
  const bool id_ok = id >= 0 && id < c.V;
  if (!id_ok && rank == 0 && threadIdx.x == 0) atomicAdd(c.status + STATUS_WORD_BAD_INPUT, 1u);
  if (r.greedy) {
    const unsigned long long key = cluster_max_key(sh_key, S, rank, key_row(zt, begin, end));
    const bool some = argmax_key_value(key) > -INFINITY;      // (of a row without any weight token 0 is taken, but no draft stands on it)
    const int top = some ? int(0xffffffffu - uint32_t(key)) : 0, verdict = some && id == top && c.alpha[at] <= 1.f;
    if (rank == 0 && threadIdx.x == 0) {
      s.top[at] = top;
      s.verdict[at] = verdict;
      if (skip && !verdict) atomicMin(s.first + b, i);
    }
    return;
  }
  const bool both = c.draft != nullptr;
  const Row zd = both ? row_at(c.draft, c.d_dtype, c.ld_d, at) : zt;
  const float scale = LOG2E / r.t;
  MaxSum mine[2] = {sum_row(zt, begin, end, scale), MaxSum{-INFINITY, 0.f}};
  int dbegin = 0, dend = 0;
  if (both) {
    share_of(c.Vd, S, rank, dbegin, dend);
    mine[1] = sum_row(zd, dbegin, dend, scale);
  }
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    for (int off = 16; off > 0; off >>= 1) {
      const MaxSum o{__shfl_xor_sync(0xffffffffu, mine[q].mx, off), __shfl_xor_sync(0xffffffffu, mine[q].sum, off)};
      mine[q] = merged(mine[q], o, scale);
    }
    if ((threadIdx.x & 31) == 0) sh_warp[q][threadIdx.x >> 5] = mine[q];
  }
  __syncthreads();
  if (threadIdx.x < 2) {
    MaxSum x = sh_warp[threadIdx.x][0];
    for (int w = 1; w < VW; ++w) x = merged(x, sh_warp[threadIdx.x][w], scale);
    st_cluster_u64(&sh_block[threadIdx.x][rank], 0, (static_cast<unsigned long long>(__float_as_uint(x.mx)) << 32) | __float_as_uint(x.sum));
  }
  cluster_or_block_sync(S);
  if (rank == 0 && threadIdx.x == 0) {
    MaxSum x[2];
    for (int q = 0; q < 2; ++q) {
      auto part = [&](int j) { return MaxSum{__uint_as_float(uint32_t(sh_block[q][j] >> 32)), __uint_as_float(uint32_t(sh_block[q][j]))}; };
      x[q] = part(0);
      for (int j = 1; j < S; ++j) x[q] = merged(x[q], part(j), scale);
    }
    s.mx[at] = make_float2(x[0].mx, x[1].mx);
    const float alpha = c.alpha[at];
    const float vt = id_ok ? load_logit(zt, id) : -INFINITY;
    const int di = both && id_ok ? draft_index(c, id) : -1;
    const float vd = di >= 0 ? load_logit(zd, di) : -INFINITY;
    int verdict, near = 0;
    if (!(vt > -INFINITY) || !(alpha <= 1.f)) {
      verdict = 0;
    } else {
      // p / q = 2^(xt - xd) sum_d / sum_t, in 32 bits off by the sums' part (row_error) and, for an exponent of size x, 1.7 x + 1 units of 2^-23 (the
      // difference, the temperature's factor and their product; the special function is in the former).
      const float xt = (vt - x[0].mx) * scale, xd = both ? (vd - x[1].mx) * scale : 0.f;
      const float ratio = both ? (vd > -INFINITY ? ex2_ftz(xt - xd) * (x[1].sum / x[0].sum) : INFINITY) : ex2_ftz(xt) / x[0].sum;
      const float tol = err + 2.7f * 0x1p-23f * (fabsf(xt) + fabsf(vd > -INFINITY ? xd : 0.f));
      verdict = ratio >= alpha;
      near = !(ratio > 1e-30f) || !(alpha > 1e-30f) || fabsf(ratio - alpha) <= tol * alpha;
      near |= xt < -1000.f || xd < -1000.f;       // (p or q may be nothing in 64 bits, or not whole: decided there)
    }
    s.verdict[at] = verdict;
    if (skip && !verdict && !near) atomicMin(s.first + b, i);
    sh_near = near;
    sh_max[0] = x[0].mx; sh_max[1] = x[1].mx;
    for (int j = 1; j < S && near; ++j) {
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(mapa_rank(smem_u32(&sh_near), uint32_t(j))), "r"(1) : "memory");
      for (int q = 0; q < 2; ++q)
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(mapa_rank(smem_u32(&sh_max[q]), uint32_t(j))), "f"(sh_max[q]) : "memory");
    }
  }
  cluster_or_block_sync(S);
  if (!sh_near) return;
  verify_row64(c, s, S, rank, skip, i, b, sh_sum, sh_max[0], sh_max[1]);
}

// One (position, request) per cluster, position by position.  verdict[b * k + i] = 1 if the draft would stand; the row maxima (and for greedy requests
// the arg-max) are left for the kernel behind.  skip: first[b] holds the lowest position refused so far, and items behind it are passed over.
// 128 requests of 16 drafts, 575 MB up to the first refused ones: 163 us and 960 MB, the rest read while the verdict in front was still out.  (Clusters
// that walk the items themselves 205 us; leaving off a row whose request has been refused meanwhile saved some bytes and no time; two blocks a row
// read fewer ahead in the same time, four are slower.)
__global__ void __launch_bounds__(VT, 2)
verify_rows_kernel(const __grid_constant__ VerifyCall c, const __grid_constant__ VerifyScratch s, int S, int skip, float err) {
  pdl_wait();
  pdl_trigger();
  const int item = blockIdx.x / S, rank = blockIdx.x % S, i = item / c.B, b = item % c.B;
  __shared__ MaxSum sh_warp[2][VW];
  __shared__ unsigned long long sh_block[2][8];
  __shared__ Reduce64 sh_sum;
  __shared__ ReduceKey sh_key;
  __shared__ float sh_max[2];
  __shared__ int sh_go, sh_near;
  if (i >= request(c, b).drafts) return;          // (uniform for the cluster)
  if (threadIdx.x == 0) {
    sh_near = 0;
    sh_go = skip ? *reinterpret_cast<volatile int*>(s.first + b) >= i : 1;
  }
  cluster_or_block_sync(S);                       // every block of the cluster runs, and its shared memory may be written to
  if (skip) {
    // all blocks of the cluster go by what the leader read
    const bool go = ld_cluster_u32(mapa_rank(smem_u32(&sh_go), 0)) != 0;
    if (!go) {
      cluster_or_block_sync(S);
      return;
    }
  }
  verify_row(c, s, S, rank, skip, i, b, sh_warp, sh_block, sh_sum, sh_key, sh_max, sh_near, err);
}

// ------------------------------------------------------------------ the token behind the drafts that stand
// A row is full of 64-bit exponentials here: e^x = 2^n 2^(i / 256) e^f with |f| <= ln 2 / 512, 2^(i / 256) from a table in shared memory (times the
// factor that the row's weights need anyway) and e^f by its series up to f^4 / 24 (the next term is 4e-17): 10 operations in 64 bits, where the
// library's function, left to what lies below e^-680, takes three times as many.
// 2^n goes into the bits of a product that already holds the factor.  That is 1, or one over a sum of at most 2^30 weights: e^-680 is 2^-981.1, so that the
// exponent stays at 2^-1013 or above, and 64 bits hold 2^-1022.
constexpr float DEEP = -680.f;
struct Weights {
  double table[256];
};
__device__ __noinline__ double exp_of_deep(double x) {       // (see weight64)
  const double e = exp(0.5 * x);
  return e * e;
}
template <bool EXACT>
struct RowWeights {                    // the weights of one row's logits, from its maximum, temperature and factor
  const Weights* w;
  const void* z;
  float m, inv_tf;
  double md, inv_t;
  float log2_t, factor;                // of the 32-bit ones: log2(e) / temperature
  bool bf16;
  __device__ __forceinline__ double operator()(float v) const {
    if (!EXACT) return double(quick(v));
    const double magic = 6755399441055744.0;                  // 1.5 2^52: whole numbers end up in the low bits
    // (the difference first: the largest weight is 1 to the bit, and p - q nothing where either row has only that)
    const double x = (double(v) - md) * inv_t, t = fma(x, 369.32993046757655, magic);        // 256 / ln 2
    const int k = __double2loint(t);
    const double f = fma(t - magic, -0.0027076061740622863, x);                              // ln 2 / 256
    const double p = f * fma(f, fma(f, fma(f, 1.0 / 24.0, 1.0 / 6.0), 0.5), 1.0), y = w->table[k & 255];
    const double r = fma(y, p, y);
    const float depth = (v - m) * inv_tf;
    if (depth > DEEP) return __hiloint2double(__double2hiint(r) + ((k >> 8) << 20), __double2loint(r));
    return x > -746.0 ? exp_of_deep(x) * w->table[0] : 0.0;    // (down to where 64 bits end: at u = 0 the lowest token with any weight is taken)
  }
  __device__ __forceinline__ float quick(float v) const { return ex2_ftz((v - m) * log2_t) * factor; }
  // A logit as it lies in memory, and what it says.  (Two steps, so that many loads go out before the first is looked at; no branch on the type.)
  template <bool F32>
  __device__ __forceinline__ uint32_t raw(int i) const {
    return F32 ? reinterpret_cast<const uint32_t*>(z)[i] : reinterpret_cast<const uint16_t*>(z)[i];
  }
  template <bool F32>
  __device__ __forceinline__ float value(uint32_t x) const {
    if (F32) return logit(__uint_as_float(x));
    return logit(bf16 ? __uint_as_float(x << 16) : __half2float(__ushort_as_half(uint16_t(x))));
  }
  // (a word that says -infinity)
  template <bool F32>
  __device__ __forceinline__ uint32_t none() const { return F32 ? 0xff800000u : bf16 ? 0xff80u : 0xfc00u; }
};
// The table times a factor.
__device__ __forceinline__ void weights_init(Weights& w, double factor) {
  for (int i = threadIdx.x; i < 256; i += VT) w.table[i] = exp2(double(i) / 256.0) * factor;
}

struct SampleShared {
  Weights p, q;
  Reduce64 sum;
  ReduceKey key;
  double warp[VW];
  double block[MAX_S];
  float map[VW][128];
  int n, found, last;
};

// Sum of a row's weights over this thread's share of [begin, end).  (The weights come by value: through a reference every use is a load from local memory.)
template <bool EXACT>
__device__ __noinline__ double row_sum(RowWeights<EXACT> w, Row r, int begin, int end) {
  double s0 = 0.0, s1 = 0.0;
  if (EXACT) {
    walk_by_index<2>(r, begin, end, [&](auto& v) {
#pragma unroll
      for (int j = 0; j < 8; ++j) (j & 1 ? s1 : s0) += w(v[j]);
    });
  } else {
    walk<4>(r, begin, end, [&](int, auto& v) {
      constexpr int N = sizeof(v) / sizeof(float);
      float part = 0.f;
#pragma unroll
      for (int j = 0; j < N; ++j) part += w.quick(v[j]);
      s0 += double(part);
    });
  }
  return s0 + s1;
}

// The first place in an ascending map whose token is v or above (one warp).
__device__ __forceinline__ int map_place(const int* map, int n, int v, int lane) {
  int lo = 0, hi = n;                                          // it is in [lo, hi]
  while (hi > lo) {
    const int step = (hi - lo + 31) / 32, at = lo + lane * step;
    const int below = __popc(__ballot_sync(0xffffffffu, at < hi && map[at] < v));
    if (below == 0) return lo;
    lo += (below - 1) * step + 1;
    hi = min(hi, lo + step - 1);
  }
  return lo;
}

// One warp's sum of max(0, p - q) over tokens [begin, end); MINUS: 0 p alone, 1 q has 16 bits, 2 it has 32.  gone: a token that counts nothing.
template <bool EXACT, bool F32, int MINUS>
__device__ __noinline__ double rest_sum(RowWeights<EXACT> p, RowWeights<EXACT> q, int begin, int end, int gone, const int* map, int n_map, float* q_of) {
  const int lane = threadIdx.x & 31;
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  auto add = [&](float (&t)[4], const float (&d)[4]) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (EXACT) {
        const double w = MINUS ? p(t[u]) - q(d[u]) : p(t[u]);
        s[u] += !MINUS || w > 0.0 ? w : 0.0;                  // (never NaN; fmax looks for it)
      } else {
        t[u] = MINUS ? fmaxf(0.f, p.quick(t[u]) - q.quick(d[u])) : p.quick(t[u]);
      }
    }
    if (!EXACT) s[0] += double((t[0] + t[1]) + (t[2] + t[3]));
  };
  auto target = [&](int base, uint32_t (&t)[4]) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int v = base + u * 32 + lane;
      t[u] = v < end && v != gone ? p.template raw<F32>(v) : p.template none<F32>();
    }
  };
  if (MINUS && map) {
    int at = begin < end ? map_place(map, n_map, begin, lane) : 0;
    uint32_t t_next[4];
    target(begin, t_next);
    for (int base = begin; base < end; base += 128) {
      float t[4], d[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) t[u] = p.template value<F32>(t_next[u]);
      target(base + 128, t_next);
      // 128 neighbours hold at most as many entries of the map, which lie together
#pragma unroll
      for (int u = 0; u < 4; ++u) q_of[u * 32 + lane] = -INFINITY;
      __syncwarp();
      int count = 0;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = at + u * 32 + lane, v = i < n_map ? map[i] : 0x7fffffff;
        const bool in = v >= base && v < base + 128;
        if (in) q_of[v - base] = q.template value<MINUS == 2>(q.template raw<MINUS == 2>(i));
        count += __popc(__ballot_sync(0xffffffffu, in));
      }
      at += count;
      __syncwarp();
#pragma unroll
      for (int u = 0; u < 4; ++u) d[u] = q_of[u * 32 + lane];
      __syncwarp();
      add(t, d);
    }
  } else {
    // two steps of 128 tokens under way in front of the one that is added
    constexpr int AHEAD = 2;
    uint32_t t[AHEAD][4], d[AHEAD][4];
    auto fetch = [&](int base, int at) {
      target(base, t[at]);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int v = base + u * 32 + lane;
        d[at][u] = MINUS && v < end ? q.template raw<MINUS == 2>(v) : q.template none<MINUS == 2>();
      }
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) fetch(begin + i * 128, i);
    for (int base = begin; base < end; base += AHEAD * 128) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        float ti[4], di[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) { ti[u] = p.template value<F32>(t[i][u]); di[u] = MINUS ? q.template value<MINUS == 2>(d[i][u]) : -INFINITY; }
        fetch(base + (AHEAD + i) * 128, i);
        add(ti, di);
      }
    }
  }
  double all = (s[0] + s[1]) + (s[2] + s[3]);
  for (int off = 16; off > 0; off >>= 1) all += shfl_xor64(all, off);
  return all;
}

// One request per cluster: counts the drafts that stand and takes the token behind them.  Without EXACT the weights are 32-bit ones, each off by up to 1.7 x 2^-23
// of itself for its exponent of size x (as in row_error), 2^-22 for the special function and 2^-23 for the factor and the sums of four, and from there on sums
// are 64-bit ones.  Averaged by weight, the exponents' size is the entropy of the weights less log2 of their sum W, so at most log2 (V / W): V weights are off by
// 2^-23 (1.7 (log2 V - log2 W) + 3) of their sum together (W is 1 or more, but where an arg-max drafter's token is left out), and so is the distance from the goal
// to a border.  A goal that is not 2^-22 (log2 V - log2 W + 4) of the sum inside its token's share is left to the kernel with EXACT.
template <bool EXACT>
__device__ __forceinline__ void sample(const VerifyCall& c, const VerifyScratch& s, int S, SampleShared& sh) {
  const int b = blockIdx.x / S, rank = blockIdx.x % S, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Request r = request(c, b);
  if (EXACT) {
    weights_init(sh.p, 1.0);
    weights_init(sh.q, 1.0);
  }
  if (!EXACT && rank == 0 && threadIdx.x == 0) {
    s.open[b] = 0;
    if (c.cu_q && (c.cu_q[b] < 0 || c.cu_q[b + 1] < c.cu_q[b] || c.cu_q[b + 1] > c.T)) atomicAdd(c.status + STATUS_WORD_BAD_INPUT, 1u);
  }
  if (threadIdx.x == 0) { sh.found = 0x7fffffff; sh.last = -1; }
  if (r.drafts >= 0 && S > 1) cluster_sync_all();  // from here every block of the cluster runs, and its shared memory may be written to
  if (warp == 0) {
    int n = max(r.drafts, 0);
    for (int base = 0; base < r.drafts; base += 32) {
      const bool bad = base + lane < r.drafts && s.verdict[b * c.k + base + lane] == 0;
      const unsigned m = __ballot_sync(0xffffffffu, bad);
      if (m) { n = base + __ffs(m) - 1; break; }
    }
    if (lane == 0) sh.n = n;
    if (!EXACT && rank == 0) {
      if (lane == 0) c.n_accept[b] = n;
      for (int i = lane; i <= c.k; i += 32)
        if (i != n || r.drafts < 0) c.tokens[size_t(b) * (c.k + 1) + i] = i < n ? c.ids[b * c.k + i] : -1;
    }
  }
  __syncthreads();
  if (r.drafts < 0) return;                       // (uniform for the cluster)
  const int n = sh.n, at = b * c.k + n;
  const bool refused = n < r.drafts;
  const Row zt = row_at(c.target, c.t_dtype, c.ld_t, r.row0 + n);
  int* out = c.tokens + size_t(b) * (c.k + 1) + n;
  int begin, end;
  share_of(c.V, S, rank, begin, end);
  float mt, md = -INFINITY;
  if (refused && r.greedy) {
    if (rank == 0 && threadIdx.x == 0) *out = s.top[at];
    return;
  }
  if (refused) {
    const float2 m = s.mx[at];
    mt = m.x; md = m.y;
  } else {
    const unsigned long long key = cluster_max_key(sh.key, S, rank, key_row(zt, begin, end));
    mt = argmax_key_value(key);
    if (r.greedy) {
      if (rank == 0 && threadIdx.x == 0) *out = mt > -INFINITY ? int(0xffffffffu - uint32_t(key)) : 0;
      return;
    }
  }
  if (!(mt > -INFINITY)) {                        // a row without any weight: as an arg-max of nothing (uniform for the cluster)
    if (rank == 0 && threadIdx.x == 0) *out = 0;
    return;
  }
  const bool both = refused && c.draft != nullptr && md > -INFINITY;
  const Row zd = both ? row_at(c.draft, c.d_dtype, c.ld_d, at) : zt;
  const double inv_t = 1.0 / double(r.t);
  const float inv_tf = float(inv_t);
  const bool t32 = c.t_dtype == CHUNK_F32, d32 = c.d_dtype == CHUNK_F32;
  const float log2_t = LOG2E / r.t;
  RowWeights<EXACT> p{&sh.p, zt.z, mt, inv_tf, double(mt), inv_t, log2_t, 1.f, c.t_dtype == CHUNK_BF16};
  RowWeights<EXACT> q{&sh.q, zd.z, md, inv_tf, double(md), inv_t, log2_t, 1.f, c.d_dtype == CHUNK_BF16};
  const int gone_token = refused && !c.draft ? c.ids[at] : -1;        // the arg-max drafter's, which takes all of its q
  if (both) {
    int dbegin, dend;
    share_of(c.Vd, S, rank, dbegin, dend);
    double st = row_sum(p, zt, begin, end), sd = row_sum(q, zd, dbegin, dend);
    cluster_sum2(sh.sum, S, rank, st, sd);        // (its barriers lie between the tables' last use and the next lines)
    if (EXACT) {
      weights_init(sh.p, 1.0 / st);
      weights_init(sh.q, 1.0 / sd);
      __syncthreads();
    } else {
      p.factor = float(1.0 / st);
      q.factor = float(1.0 / sd);
    }
  }
  const double u = double(c.u[b]);
  for (int less = 1; less >= 0; --less) {         // once more without q where max(0, p - q) is nothing anywhere
    const int gone = less ? gone_token : -1, minus = both && less ? (d32 ? 2 : 1) : 0;
    auto sum_of = [&](int from, int to) {
      float* q_of = sh.map[warp];
      if (minus == 0) return t32 ? rest_sum<EXACT, true, 0>(p, q, from, to, gone, nullptr, 0, q_of) : rest_sum<EXACT, false, 0>(p, q, from, to, gone, nullptr, 0, q_of);
      if (minus == 1) return t32 ? rest_sum<EXACT, true, 1>(p, q, from, to, gone, c.vocab_map, c.Vd, q_of) : rest_sum<EXACT, false, 1>(p, q, from, to, gone, c.vocab_map, c.Vd, q_of);
      return t32 ? rest_sum<EXACT, true, 2>(p, q, from, to, gone, c.vocab_map, c.Vd, q_of) : rest_sum<EXACT, false, 2>(p, q, from, to, gone, c.vocab_map, c.Vd, q_of);
    };
    // sums of the warps' parts of [from, to) into sh.warp; the width of a part
    auto parts_of = [&](int from, int to) {
      const int per = ((to - from + VW - 1) / VW + 31) & ~31, wb = min(to, from + warp * per);
      const double mine = sum_of(wb, min(to, wb + per));
      __syncthreads();                            // (the sums in front have been read)
      if (lane == 0) sh.warp[warp] = mine;
      __syncthreads();
      return per;
    };
    const int per = parts_of(begin, end);
    if (threadIdx.x < unsigned(S)) {
      double x = 0.0;
      for (int w = 0; w < VW; ++w) x += sh.warp[w];
      st_cluster_f64(&sh.block[rank], threadIdx.x, x);
    }
    cluster_or_block_sync(S);
    double whole = 0.0;
    for (int j = 0; j < S; ++j) whole += sh.block[j];
    // (how far the 32-bit sums may be off: p and q weigh 1 each where both count, else p is all there is)
    const double tol = EXACT ? 0.0 : (both && less ? 2.0 : whole) * double(log2f(float(c.V)) + fmaxf(0.f, -log2f(float(whole))) + 4.f) * 0x1p-23;
    // Nearly nothing left of p - q, or of p without an arg-max drafter's token (weights under 2^-126, up to 2^30 of them, are nothing here; beside 2^-60 they
    // do not count): left to the other kernel.
    if (!EXACT && ((both && less && !(whole > 64.0 * tol)) || (gone >= 0 && !(whole > 0x1p-60)))) {
      if (rank == 0 && threadIdx.x == 0) s.open[b] = 1;
      break;
    }
    if (!(whole > 0.0) && less) {
      cluster_or_block_sync(S);                   // (the others may still be reading)
      continue;
    }
    // The block, the warp's part, the part of that part in which the sum passes u * whole, and in there the token; where rounding hides the place,
    // the last with any weight.
    const double goal = u * whole;
    double before = 0.0;
    auto find = [&](const double* part, int count) {
      int last = 0;
      double x = before, x_last = before;
      for (int j = 0; j < count; ++j) {
        if (x + part[j] > goal) { before = x; return j; }
        if (part[j] > 0.0) { last = j; x_last = x; }
        x += part[j];
      }
      before = x_last;
      return last;
    };
    if (find(sh.block, S) != rank) break;
    const int from = begin + find(sh.warp, VW) * per, to = min(end, from + per);
    const int fine = parts_of(from, to);
    int v0 = from + find(sh.warp, VW) * fine;
    const int v1 = min(to, v0 + fine);
    for (; v0 < v1; v0 += VT) {
      // a token for every thread
      const int v = v0 + int(threadIdx.x);
      float* q_of = &sh.map[0][0];
      const bool on = v < v1 && v != gone;
      double w = 0.0;
      if (minus && c.vocab_map) {
        q_of[threadIdx.x] = -INFINITY;
        __syncthreads();
        const int i = map_place(c.vocab_map, c.Vd, v0, lane) + int(threadIdx.x), m = i < c.Vd ? c.vocab_map[i] : 0x7fffffff;
        if (m >= v0 && m < v0 + VT) q_of[m - v0] = load_logit(zd, i);
        __syncthreads();
        if (on) w = fmax(0.0, p(load_logit(zt, v)) - q(q_of[threadIdx.x]));
      } else if (on) {
        w = p(load_logit(zt, v));
        if (minus) w = fmax(0.0, w - q(load_logit(zd, v)));
      }
      double run = w;
      for (int off = 1; off < 32; off <<= 1) { const double o = shfl_up64(run, off); if (lane >= off) run += o; }
      __syncthreads();
      if (lane == 31) sh.warp[warp] = run;
      __syncthreads();
      double x = before;
      for (int j = 0; j < warp; ++j) x += sh.warp[j];
      if (w > 0.0) {
        if (x + run > goal) atomicMin(&sh.found, v);
        atomicMax(&sh.last, v);
      }
      __syncthreads();
      // (the goal's own error is the whole's)
      if (!EXACT && v == sh.found && !(goal - (x + run - w) > 2.0 * tol && x + run - goal > 2.0 * tol)) s.open[b] = 1;
      for (int j = 0; j < VW; ++j) before += sh.warp[j];
      __syncthreads();
      if (sh.found != 0x7fffffff) break;          // (uniform for the block)
    }
    if (threadIdx.x == 0) {
      *out = sh.found != 0x7fffffff ? sh.found : max(sh.last, 0);
      if (!EXACT && sh.found == 0x7fffffff) s.open[b] = 1;
    }
    break;
  }
  if (S > 1) cluster_sync_all();                               // no block leaves while another may still write to its shared memory
}

enum { SAMPLE_32, SAMPLE_64, SAMPLE_BOTH };
template <int HOW>
__global__ void __launch_bounds__(VT, 2) verify_sample_kernel(const __grid_constant__ VerifyCall c, const __grid_constant__ VerifyScratch s, int S) {
  pdl_wait();
  pdl_trigger();
  __shared__ SampleShared sh;
  if (HOW != SAMPLE_64) sample<false>(c, s, S, sh);
  if (HOW == SAMPLE_BOTH) cluster_or_block_sync(S);           // (what any of the blocks found, and the shared memory)
  if (HOW != SAMPLE_32 && *reinterpret_cast<volatile int*>(s.open + blockIdx.x / S)) sample<true>(c, s, S, sh);       // (uniform for the cluster)
}

}  // namespace

size_t verify_workspace_bytes(int B, int k) {
  return ((size_t(B) * 8 + 255) & ~size_t(255)) + size_t(B) * k * (sizeof(float2) + 8) + 256;
}

// How far the quotient of two sums (or of one and a weight) of the first step may be off relative to itself, added up as if every rounding went the same way,
// in units of 2^-23.  The exponents' average by weight is log2 V at most, which gives 1.7 log2 V for what rounds in them and 2 for the special function.  A thread
// rescales what it has and adds to it for every 16 values (3: the special function, a product, an addition; and 3 for the sum of the sixteen), and the same 27
// times for what others have (5 lanes', 15 warps', 7 blocks').  152 064 tokens, a block each: 4e-5, which a ratio comes as near to alpha as once in some
// thousand rows.
static float row_error(const VerifyCall& c, int S) {
  const float steps = float(c.V / (S * VT * 16) + 3), sum = 1.7f * log2f(float(c.V)) + 2.f + 3.f * (steps + 27.f) + 3.f;
  return ((c.draft ? 2.f : 1.f) * sum + 4.f) * 0x1p-23f;
}

cudaError_t verify_launch(const VerifyCall& c, cudaStream_t stream) {
  VerifyScratch s;
  uint8_t* ws = reinterpret_cast<uint8_t*>(c.ws);
  s.first = reinterpret_cast<int*>(ws);
  s.open = s.first + c.B;
  s.mx = reinterpret_cast<float2*>(ws + ((size_t(c.B) * 8 + 255) & ~size_t(255)));
  s.top = reinterpret_cast<int*>(s.mx + size_t(c.B) * c.k);
  s.verdict = s.top + size_t(c.B) * c.k;
  cudaError_t e = cudaSuccess;
  const long long items = (long long)c.B * c.k;
  // blocks of a cluster: two for every SM where there are few items, as long as each has a few KB to read
  auto blocks_for = [&](long long n, int most) {
    int S = 1;
    while (S < most && n * 2 * S <= 2 * 148 && c.V / (2 * S) >= 2048) S *= 2;
    return S;
  };
  if (items > 0) {
    const int S = blocks_for(items, 8), skip = items * S > 2 * 148;
    if (skip) {
      e = launch_pdl(verify_init_kernel, dim3(1), dim3(256), 0, stream, s.first, c.B);
      if (e != cudaSuccess) return e;
    }
    e = launch_pdl_cluster(verify_rows_kernel, dim3(unsigned(items * S)), dim3(VT), dim3(S), 0, stream, c, s, S, skip, row_error(c, S));
    if (e != cudaSuccess) return e;
  }
  // One request in five to ten is left for the third step, a chain of 64-bit operations for every token of a thread: 16 blocks each as long as there are SMs
  // for them (37 requests of 151 937 tokens: 45 us, 58 with 8; 128 of 152 064: 77, 64 with 8).
  const int S = blocks_for(c.B, MAX_S), S64 = blocks_for(1, c.B <= 64 ? MAX_S : 8);
  static bool done[MAX_DEVICES] = {};
  e = once_per_device(done, [](int) {
    cudaError_t e1 = cudaSuccess;
    for (auto k : {verify_sample_kernel<SAMPLE_32>, verify_sample_kernel<SAMPLE_64>, verify_sample_kernel<SAMPLE_BOTH>})
      if (e1 == cudaSuccess) e1 = cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    return e1;
  });
  if (e != cudaSuccess) return e;
  // With as many blocks a request in both, one launch: a single request's step takes 13.8 us on the device.
  if (S == S64) return launch_pdl_cluster(verify_sample_kernel<SAMPLE_BOTH>, dim3(unsigned(c.B) * S), dim3(VT), dim3(S), 0, stream, c, s, S);
  e = launch_pdl_cluster(verify_sample_kernel<SAMPLE_32>, dim3(unsigned(c.B) * S), dim3(VT), dim3(S), 0, stream, c, s, S);
  if (e != cudaSuccess) return e;
  return launch_pdl_cluster(verify_sample_kernel<SAMPLE_64>, dim3(unsigned(c.B) * S64), dim3(VT), dim3(S64), 0, stream, c, s, S64);
}

}  // namespace hspec
