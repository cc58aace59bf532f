// Attention of a ragged chunk of new tokens over the paged cache that holds their keys and values already.
//   o[t, h] = sum_j p_j v[j, g] / sum_j p_j,  p_j = exp(scale q[t, h] . k[j, g]),  j <= pos(t), j > pos(t) - window,  g = h / (Hq / Hkv)
// A row that sees no key is zero.  One warp per (row, head), one pass with the running maximum and sum.
#include "chunk.cuh"

namespace hspec {

namespace {

template <bool F16>
__device__ __forceinline__ float load16(const void* p, size_t i) {
  return F16 ? __half2float(reinterpret_cast<const __half*>(p)[i]) : bf16_bits_to_float(reinterpret_cast<const uint16_t*>(p)[i]);
}

template <int DH, bool F16>
__global__ void __launch_bounds__(256) chunk_attn_kernel(ChunkAttnCall c) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int t = int(w / c.Hq), h = int(w % c.Hq), g = h / (c.Hq / c.Hkv);
  if (t >= c.T) return;
  const int b = chunk_request_of(c.cu_q, c.B, t, lane);
  if (b >= c.B || t < c.cu_q[b]) return;
  const int cu0 = c.cu_q[b], cu1 = c.cu_q[b + 1], len = c.kv_lens[b];
  const ChunkRequest r = chunk_request(cu0, cu1, len, c.T, c.max_len);
  const bool counts = lane == 0 && h == 0 && t == r.q0;       // one row of the request speaks for it
  if (counts && chunk_request_bad(cu0, cu1, len, c.T, c.max_len)) atomicAdd(c.status + STATUS_WORD_BAD_INPUT, 1u);
  const int pos = r.len - r.n + (t - r.q0);
  constexpr int E = DH / 32;
  float q[E], acc[E], mx = -INFINITY, sum = 0.f;
  for (int e = 0; e < E; ++e) { q[e] = load16<F16>(c.q, size_t(t) * c.ldq + h * DH + e * 32 + lane) * c.scale; acc[e] = 0.f; }
  for (int j = c.window > 0 ? max(0, pos - c.window + 1) : 0; j <= pos; ++j) {
    const int page = c.page_table[size_t(b) * c.page_table_stride + j / c.page_size];
    const bool ok = page >= 0 && page < c.num_pages;
    if (!ok && counts) atomicAdd(c.status + STATUS_WORD_BAD_INPUT, 1u);
    const size_t at = ((size_t(ok ? page : 0) * c.page_size + j % c.page_size) * c.Hkv + g) * DH + lane;
    float s = 0.f;
    for (int e = 0; e < E; ++e) s += ok ? q[e] * load16<F16>(c.k_pool, at + e * 32) : 0.f;
    for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    const float nm = fmaxf(mx, s), f = expf(mx - nm), p = expf(s - nm);
    mx = nm;
    sum = sum * f + p;
    for (int e = 0; e < E; ++e) acc[e] = acc[e] * f + (ok ? p * load16<F16>(c.v_pool, at + e * 32) : 0.f);
  }
  for (int e = 0; e < E; ++e) {
    const float v = pos < 0 ? 0.f : acc[e] / sum;
    const size_t at = size_t(t) * c.ldo + h * DH + e * 32 + lane;
    if (F16) reinterpret_cast<__half*>(c.o)[at] = f16_sat(v, c.status);
    else reinterpret_cast<__nv_bfloat16*>(c.o)[at] = __float2bfloat16_rn(v);
  }
}

}  // namespace

size_t chunk_attn_workspace_bytes(int, int, int) { return 256; }

cudaError_t chunk_attn_launch(const ChunkAttnCall& c, cudaStream_t stream, std::string*) {
  const unsigned blocks = unsigned(((long long)c.T * c.Hq + 7) / 8);
  auto kernel = c.dh == 64 ? (c.f16 ? chunk_attn_kernel<64, true> : chunk_attn_kernel<64, false>)
                           : (c.f16 ? chunk_attn_kernel<128, true> : chunk_attn_kernel<128, false>);
  return launch_pdl(kernel, dim3(blocks), dim3(256), 0, stream, c);
}

}  // namespace hspec
