// Verification of drafted tokens against the target's probabilities from given uniform numbers (App. A).
//
//   p = softmax(z_T / temperature), q = softmax(z_D / temperature) (or all of it on the drafted token where the drafter takes the arg-max)
//   draft i stands if every earlier one does, p_i(x_i) > 0 and min(1, p_i(x_i) / q_i(x_i)) >= alpha_i
//   behind the n drafts that stand one token more: from max(0, p_n - q_n) where draft n was refused, from p_n where none was; the lowest v whose
//   cumulative sum exceeds u times the whole
//
// Both answers are integers that hang on a comparison of real numbers, so they are decided as if in 64 bits: the ratio is taken from 32-bit sums,
// and once more from 64-bit sums where it comes so near to alpha that the 32-bit ones could be on the wrong side; the cumulative sum is 64-bit
// throughout (a vocabulary has 10^5 steps, and a 32-bit sum would land on the wrong one in one of a hundred draws).
//
// Two launches.  The first takes one (request, position) per cluster of blocks, reads the target's and the drafter's row once and decides whether
// the position would be refused.  Items go out position by position, and one whose request is known to have been refused before is not read.
// The second takes one request per cluster and samples.  The first is bound by memory, the second by the 64-bit exponentials of its row.
#include "common.cuh"
#include "kernels.h"

#include <cfloat>
#include <type_traits>

namespace hspec {

namespace {

constexpr int VT = 512;              // threads of a block
constexpr int VW = VT / 32;
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

// Calls f(first index, values of N neighbours) for this thread's share of [begin, end): 16-byte loads, four of them in flight, scalar loads in
// front of the first 16-byte boundary and behind the last.
template <typename T, typename F>
__device__ __forceinline__ void walk(const T* z, int begin, int end, F f) {
  constexpr int N = 16 / sizeof(T), U = 4;
  const int off = int((reinterpret_cast<uintptr_t>(z + begin) & 15) / sizeof(T));
  const int head = min(end, begin + (off ? N - off : 0)), n16 = (end - head) / N;
  for (int i = begin + int(threadIdx.x); i < head; i += VT) { float v[1] = {logit(value_of(z[i]))}; f(i, v); }
  const uint4* p = reinterpret_cast<const uint4*>(z + head);
  for (int i0 = threadIdx.x; i0 < n16; i0 += U * VT) {
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) if (i0 + u * VT < n16) w[u] = __ldg(p + i0 + u * VT);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u * VT >= n16) break;
      float v[N];
      const T* e = reinterpret_cast<const T*>(&w[u]);
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = logit(value_of(e[j]));
      f(head + (i0 + u * VT) * N, v);
    }
  }
  for (int i = head + n16 * N + int(threadIdx.x); i < end; i += VT) { float v[1] = {logit(value_of(z[i]))}; f(i, v); }
}
template <typename F>
__device__ __forceinline__ void walk(const Row& r, int begin, int end, F f) {
  if (r.dtype == CHUNK_F32) walk(reinterpret_cast<const float*>(r.z), begin, end, f);
  else if (r.dtype == CHUNK_F16) walk(reinterpret_cast<const __half*>(r.z), begin, end, f);
  else walk(reinterpret_cast<const __nv_bfloat16*>(r.z), begin, end, f);
}

struct MaxSum { float mx, sum; };
__device__ __forceinline__ MaxSum merged(MaxSum a, MaxSum b, float c) {
  const float m = fmaxf(a.mx, b.mx);
  if (m == -INFINITY) return a;
  return MaxSum{m, (a.mx > -INFINITY ? a.sum * ex2_ftz((a.mx - m) * c) : 0.f) + (b.mx > -INFINITY ? b.sum * ex2_ftz((b.mx - m) * c) : 0.f)};
}
// One pass: the running maximum and the sum of 2^((z - max) c) over this thread's share.
__device__ __forceinline__ MaxSum sum_row(const Row& r, int begin, int end, float c) {
  float mx = -INFINITY, sum = 0.f;
  walk(r, begin, end, [&](int, auto& v) {
    constexpr int N = sizeof(v) / sizeof(float);
    float mu = v[0];
#pragma unroll
    for (int j = 1; j < N; ++j) mu = fmaxf(mu, v[j]);
    if (mu > mx) { sum *= ex2_ftz((mx - mu) * c); mx = mu; }
    if (mx > -INFINITY) {
#pragma unroll
      for (int j = 0; j < N; ++j) sum += ex2_ftz((v[j] - mx) * c);
    }
  });
  return MaxSum{mx, sum};
}
// The largest value and its lowest index over this thread's share, as one number (argmax_key).
__device__ __forceinline__ unsigned long long key_row(const Row& r, int begin, int end) {
  unsigned long long best = 0;
  float mx = -INFINITY;
  walk(r, begin, end, [&](int i, auto& v) {
    constexpr int N = sizeof(v) / sizeof(float);
#pragma unroll
    for (int j = 0; j < N; ++j) if (v[j] > mx || best == 0) { mx = v[j]; best = argmax_key(v[j], i + j); }
  });
  return best;
}

// e^((z - m) / t) in 64 bits; nothing where z is -infinity
__device__ __forceinline__ double weight64(float z, float m, double inv_t) {
  return z > -INFINITY ? exp((double(z) - double(m)) * inv_t) : 0.0;
}
__device__ __forceinline__ double sum_row64(const Row& r, int begin, int end, float m, double inv_t) {
  double s = 0.0;
  if (m > -INFINITY)
    walk(r, begin, end, [&](int, auto& v) {
      constexpr int N = sizeof(v) / sizeof(float);
#pragma unroll
      for (int j = 0; j < N; ++j) s += weight64(v[j], m, inv_t);
    });
  return s;
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
  double block[2][8];
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
  unsigned long long warp[VW], block[8];
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

// Rows and drafts of a request, and its temperature (not above zero, or NaN: greedy).
struct Request { int row0, drafts; float t; bool greedy; };
__device__ __forceinline__ Request request(const VerifyCall& c, int b) {
  Request r;
  int lo = b * (c.k + 1), hi = lo + c.k + 1;
  if (c.cu_q) { lo = c.cu_q[b]; hi = c.cu_q[b + 1]; }
  r.row0 = min(max(lo, 0), c.T);
  r.drafts = min(max(min(hi, c.T) - r.row0 - 1, -1), c.k);         // -1: no row at all, nothing to sample from
  r.t = c.temperature ? c.temperature[b] : 1.f;
  r.greedy = !(r.t > 0.f);
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

// One (position, request) per cluster.  verdict[b * k + i] = 1 if the draft would stand; the row maxima (and for greedy requests the arg-max) are
// left for the kernel behind.  skip: first[b] holds the lowest position refused so far.
__global__ void __launch_bounds__(VT)
verify_rows_kernel(VerifyCall c, VerifyScratch s, int S, int skip) {
  pdl_wait();
  pdl_trigger();
  const int item = blockIdx.x / S, rank = blockIdx.x % S, i = item / c.B, b = item % c.B;
  const Request r = request(c, b);
  __shared__ MaxSum sh_warp[2][VW];
  __shared__ unsigned long long sh_block[2][8];
  __shared__ Reduce64 sh_sum;
  __shared__ ReduceKey sh_key;
  __shared__ float sh_max[2];
  __shared__ int sh_go, sh_near;
  if (i >= r.drafts) return;                      // (uniform for the cluster)
  if (threadIdx.x == 0) {
    sh_near = 0;
    sh_go = skip ? *reinterpret_cast<volatile int*>(s.first + b) >= i : 1;
  }
  cluster_or_block_sync(S);                       // from here every block of the cluster runs, and its shared memory may be written to
  if (skip) {
    // all blocks of the cluster go by what the leader read
    const bool go = ld_cluster_u32(mapa_rank(smem_u32(&sh_go), 0)) != 0;
    if (!go) {
      cluster_or_block_sync(S);
      return;
    }
  }
  const int at = b * c.k + i, id = c.ids[at];
  const Row zt = row_at(c.target, c.t_dtype, c.ld_t, r.row0 + i);
  int begin, end;
  share_of(c.V, S, rank, begin, end);
  const bool id_ok = id >= 0 && id < c.V;
  if (!id_ok && rank == 0 && threadIdx.x == 0) atomicAdd(c.status + STATUS_WORD_BAD_INPUT, 1u);
  if (r.greedy) {
    const unsigned long long key = cluster_max_key(sh_key, S, rank, key_row(zt, begin, end));
    const int top = argmax_key_value(key) > -INFINITY ? int(0xffffffffu - uint32_t(key)) : 0;
    if (rank == 0 && threadIdx.x == 0) {
      s.top[at] = top;
      s.verdict[at] = id == top;
      if (skip && id != top) atomicMin(s.first + b, i);
    }
    return;
  }
  const bool both = c.draft != nullptr;
  const Row zd = both ? row_at(c.draft, c.d_dtype, c.ld_d, at) : zt;
  const float scale = fminf(fmaxf(LOG2E / r.t, 1e-30f), 1e30f);
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
      // p / q = 2^(xt - xd) sum_d / sum_t.  Each exponent is off by 2^-23 of its size (a subtraction and a product rounded, then the special
      // function's 2^-22), so are the sums' terms, and a sum of n terms by a few roundings more: 2^-17 of the whole covers sizes up to 24.
      const float xt = (vt - x[0].mx) * scale, xd = both ? (vd - x[1].mx) * scale : 0.f;
      const float ratio = both ? (vd > -INFINITY ? ex2_ftz(xt - xd) * (x[1].sum / x[0].sum) : INFINITY) : ex2_ftz(xt) / x[0].sum;
      const float tol = (24.f + fabsf(xt) + fabsf(vd > -INFINITY ? xd : 0.f)) * 3.2e-7f;
      verdict = ratio >= alpha;
      near = !(ratio > 1e-30f) || !(alpha > 1e-30f) || fabsf(ratio - alpha) <= tol * alpha;
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
  // so near to alpha that the 32-bit sums do not decide: the same in 64 bits
  const double inv_t = 1.0 / double(r.t);
  double st = sum_row64(zt, begin, end, sh_max[0], inv_t), sd = both ? sum_row64(zd, dbegin, dend, sh_max[1], inv_t) : 0.0;
  cluster_sum2(sh_sum, S, rank, st, sd);
  if (rank == 0 && threadIdx.x == 0) {
    const double p = weight64(load_logit(zt, id), sh_max[0], inv_t) / st;
    const int di = both ? draft_index(c, id) : -1;
    const double q = !both ? 1.0 : di >= 0 ? weight64(load_logit(zd, di), sh_max[1], inv_t) / sd : 0.0;
    const int verdict = p > 0.0 && (q > 0.0 ? p / q : INFINITY) >= double(c.alpha[at]);
    s.verdict[at] = verdict;
    if (skip && !verdict) atomicMin(s.first + b, i);
  }
}

struct SampleShared {
  Reduce64 sum;
  ReduceKey key;
  double warp[VW];
  double block[8];
  float q[VW][32];
  int n;
};

// One request per cluster: counts the drafts that stand and takes the token behind them.
__global__ void __launch_bounds__(VT)
verify_sample_kernel(VerifyCall c, VerifyScratch s, int S) {
  pdl_wait();
  pdl_trigger();
  __shared__ SampleShared sh;
  const int b = blockIdx.x / S, rank = blockIdx.x % S, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Request r = request(c, b);
  if (r.drafts >= 0 && S > 1) cluster_sync_all();  // from here every block of the cluster runs, and its shared memory may be written to
  if (warp == 0) {
    int n = max(r.drafts, 0);
    for (int base = 0; base < r.drafts; base += 32) {
      const bool bad = base + lane < r.drafts && s.verdict[b * c.k + base + lane] == 0;
      const unsigned m = __ballot_sync(0xffffffffu, bad);
      if (m) { n = base + __ffs(m) - 1; break; }
    }
    if (lane == 0) sh.n = n;
    if (rank == 0) {
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
  float mt, md = 0.f;
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
  const double inv_t = 1.0 / double(r.t), u = double(c.u[b]);
  const bool both = refused && c.draft != nullptr;
  const int gone = refused && !both ? c.ids[at] : -1;       // the arg-max drafter's token, which takes all of its q
  const Row zd = both ? row_at(c.draft, c.d_dtype, c.ld_d, at) : zt;
  double wt = 1.0, wd = 0.0;                                  // weights are p * wt and q * wd, up to a common factor
  if (both) {
    int dbegin, dend;
    share_of(c.Vd, S, rank, dbegin, dend);
    double st = sum_row64(zt, begin, end, mt, inv_t), sd = sum_row64(zd, dbegin, dend, md, inv_t);
    cluster_sum2(sh.sum, S, rank, st, sd);
    wt = 1.0 / st;
    wd = sd > 0.0 ? 1.0 / sd : 0.0;
  }
  // a warp's part of the block's share, walked 32 neighbours at a time
  const int per = ((end - begin + VW - 1) / VW + 31) & ~31;
  const int wb = min(end, begin + warp * per), we = min(end, wb + per);
  for (int less = 1; less >= 0; --less) {                     // once more without q where max(0, p - q) is nothing anywhere
    auto each = [&](auto take) {
      int mapped = 0;
      if (both && less && c.vocab_map) {                      // map entries below the part's first token
        int hi = c.Vd;
        while (mapped < hi) { const int mid = (mapped + hi) >> 1; if (c.vocab_map[mid] < wb) mapped = mid + 1; else hi = mid; }
      }
      for (int base = wb; base < we; base += 32) {
        const int v = base + lane;
        const bool on = v < we;
        float d = -INFINITY;
        if (both && less) {
          if (!c.vocab_map) {
            if (on && v < c.Vd) d = load_logit(zd, v);
          } else {
            // (32 neighbours hold at most 32 entries of an ascending map)
            sh.q[warp][lane] = -INFINITY;
            __syncwarp();
            const int m = mapped + lane < c.Vd ? c.vocab_map[mapped + lane] : 0x7fffffff;
            const bool in = m >= base && m < base + 32;
            if (in) sh.q[warp][m - base] = load_logit(zd, mapped + lane);
            mapped += __popc(__ballot_sync(0xffffffffu, in));
            __syncwarp();
            d = sh.q[warp][lane];
            __syncwarp();
          }
        }
        double w = 0.0;
        if (on && mt > -INFINITY && !(less && v == gone)) {
          w = weight64(load_logit(zt, v), mt, inv_t) * wt;
          if (both && less && d > -INFINITY) w = fmax(0.0, w - weight64(d, md, inv_t) * wd);
        }
        if (take(v, w)) return;
      }
    };
    double mine = 0.0;
    each([&](int, double w) { mine += w; return false; });
    for (int off = 16; off > 0; off >>= 1) mine += shfl_xor64(mine, off);
    __syncthreads();
    if (lane == 0) sh.warp[warp] = mine;
    __syncthreads();
    if (threadIdx.x < unsigned(S)) {
      double x = 0.0;
      for (int w = 0; w < VW; ++w) x += sh.warp[w];
      st_cluster_f64(&sh.block[rank], threadIdx.x, x);
    }
    cluster_or_block_sync(S);
    double whole = 0.0;
    for (int j = 0; j < S; ++j) whole += sh.block[j];
    if (!(whole > 0.0)) {
      if (less) { cluster_or_block_sync(S); continue; }       // (the others may still be reading)
      if (rank == 0 && threadIdx.x == 0) *out = 0;            // a row without any weight: as an arg-max of nothing
      break;
    }
    // the block, then the warp, in which the sum passes u * whole; where rounding hides the place, the last with any weight
    const double goal = u * whole;
    auto find = [&](const double* part, int count, double& before) {
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
    double before = 0.0;
    if (find(sh.block, S, before) == rank && find(sh.warp, VW, before) == warp) {
      int found = -1, last = wb;
      double x = before;
      each([&](int v, double w) {
        double run = w;
        for (int off = 1; off < 32; off <<= 1) { const double o = shfl_up64(run, off); if (lane >= off) run += o; }
        const unsigned hit = __ballot_sync(0xffffffffu, w > 0.0 && x + run > goal), any = __ballot_sync(0xffffffffu, w > 0.0);
        if (any) last = v - lane + 31 - __clz(any);
        if (hit) { found = v - lane + __ffs(hit) - 1; return true; }
        x += __shfl_sync(0xffffffffu, run, 31);
        return false;
      });
      if (lane == 0) *out = found >= 0 ? found : last;
    }
    break;
  }
  if (S > 1) cluster_sync_all();                               // no block leaves while another may still write to its shared memory
}

}  // namespace

size_t verify_workspace_bytes(int B, int k) {
  return ((size_t(B) * 4 + 255) & ~size_t(255)) + size_t(B) * k * (sizeof(float2) + 8) + 256;
}

cudaError_t verify_launch(const VerifyCall& c, cudaStream_t stream) {
  VerifyScratch s;
  uint8_t* ws = reinterpret_cast<uint8_t*>(c.ws);
  s.first = reinterpret_cast<int*>(ws);
  s.mx = reinterpret_cast<float2*>(ws + ((size_t(c.B) * 4 + 255) & ~size_t(255)));
  s.top = reinterpret_cast<int*>(s.mx + size_t(c.B) * c.k);
  s.verdict = s.top + size_t(c.B) * c.k;
  cudaError_t e = cudaSuccess;
  const long long items = (long long)c.B * c.k;
  auto blocks_for = [&](long long n, int least) {              // blocks of a cluster: two for every SM, as long as each has a few KB to read
    int S = least;
    while (S < 8 && n * S < 2 * 148 && c.V / (2 * S) >= 2048) S *= 2;
    return S;
  };
  if (items > 0) {
    const int S = blocks_for(items, 1), skip = items * S > 4 * 148;
    if (skip) {
      e = launch_pdl(verify_init_kernel, dim3(1), dim3(256), 0, stream, s.first, c.B);
      if (e != cudaSuccess) return e;
    }
    e = launch_pdl_cluster(verify_rows_kernel, dim3(unsigned(items * S)), dim3(VT), dim3(S), 0, stream, c, s, S, skip);
    if (e != cudaSuccess) return e;
  }
  const int S = blocks_for(c.B, 1);
  return launch_pdl_cluster(verify_sample_kernel, dim3(unsigned(c.B) * S), dim3(VT), dim3(S), 0, stream, c, s, S);
}

}  // namespace hspec
