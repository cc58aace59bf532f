// What a request's rules do to the target's logits between the LM head and the verification: penalties for repeated tokens, biases, allowed tokens.
//
// For row i of request b, whose text is history[b, :len] and then its drafts 0 .. i - 1:
//   z <- z / r if z > 0, else z r          for every token of the text (prompt, answer or drafts)
//   z <- z - f count - p                   for every token of the answer or the drafts, `count` times there
//   z <- z + bias;   z <- -infinity where the row's bits forbid the token
// Bound by memory: every logit is read and written once (in place: only what changes).  A block takes a slice of the vocabulary and some rows of one
// request.  It counts the request's tokens that fall into the slice in shared memory (whole numbers, so that the order of the additions does not
// matter), marks the tokens that any rule but the bits touches in a bitmap, and then streams the rows: a 16-byte word of logits costs one look at the
// bitmap and one at the allowed bits, and the counts are read where a bit is set.  Between two rows the draft in front of the second is counted.
#include "chunk_scan.cuh"

#include <climits>
#include <type_traits>

namespace hspec {

namespace {

constexpr int RULE_THREADS = 256;
constexpr int MOST_ROWS = 32;                     // of a block
constexpr int RULE_AHEAD = 4;                      // 16-byte words of a thread under way
constexpr uint32_t IN_PROMPT = 0x80000000u;       // a token's word: said in the prompt, bias entry + 1, times said since
constexpr int BIAS_SHIFT = 20;
constexpr uint32_t BIAS_BITS = 0x7ff, COUNT_BITS = (1u << BIAS_SHIFT) - 1;

struct RuleArgs {
  LogitsCall c;
  int slice, slices, rows;                        // tokens of a slice, slices, rows of a block
  int tables;                                     // penalties or biases are asked for: counts are needed
};

template <typename T> __device__ __forceinline__ T from_f32(float v, uint32_t* status);
template <> __device__ __forceinline__ float from_f32(float v, uint32_t*) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float v, uint32_t*) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32(float v, uint32_t* status) { return f16_sat(v, status); }

// 32 bits from bit position `at` of a bit string (the word behind the last is not read: `words` of them)
__device__ __forceinline__ uint32_t bits_from(const uint32_t* w, int at, int words) {
  const int i = at >> 5;
  const uint32_t lo = w[i], hi = (at & 31) && i + 1 < words ? w[i + 1] : 0u;
  return __funnelshift_r(lo, hi, at & 31);
}

struct Rules {
  float r, f, p;
  bool penalise_repeat, subtract;
};

// One logit whose token is marked.
__device__ __forceinline__ float ruled(float z, uint32_t word, const Rules& u, const float* bias) {
  const uint32_t n = word & COUNT_BITS;
  if (u.penalise_repeat && (n || (word & IN_PROMPT))) z = z > 0.f ? z / u.r : z * u.r;
  if (u.subtract && n) z = z - u.f * float(n) - u.p;
  const uint32_t e = (word >> BIAS_SHIFT) & BIAS_BITS;
  return e ? z + bias[e - 1] : z;
}

template <typename TI, typename TO>
__global__ void __launch_bounds__(RULE_THREADS) adjust_logits_kernel(RuleArgs a) {
  constexpr int VEC = 16 / sizeof(TI);
  const LogitsCall& c = a.c;
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) uint32_t table[];          // [slice] words of the tokens
  uint32_t* marked = table + a.slice;                        // [slice / 32] bits
  float* bias = reinterpret_cast<float*>(marked + a.slice / 32);
  __shared__ int s_draft[MOST_ROWS], s_mask[MOST_ROWS];
  const int tid = threadIdx.x, lane = tid & 31;
  const int lo = (blockIdx.x % a.slices) * a.slice, hi = min(lo + a.slice, c.V);

  // ---- the block's request and rows (every warp looks for itself)
  ChunkItem item{int(blockIdx.x) / a.slices, int(blockIdx.x) / a.slices, 1, 0};
  if (c.cu_q) item = chunk_item(c.cu_q, c.B, c.T, a.rows, 0, item.b, lane);
  if (blockIdx.x == 0 && c.cu_q)
    for (int r = tid; r < c.B; r += RULE_THREADS)
      if (chunk_request_bad(c.cu_q[r], c.cu_q[r + 1], INT_MAX, c.T, INT_MAX)) atomicAdd(c.status + STATUS_WORD_BAD_INPUT, 1u);
  if (item.b < 0) return;
  const int b = item.b, first = item.first, t0 = item.q0 + first, rows = min(a.rows, item.n - first);
  Rules u{};
  if (a.tables) {
    for (int i = tid; i < a.slice; i += RULE_THREADS) table[i] = 0;
    for (int i = tid; i < a.slice / 32; i += RULE_THREADS) marked[i] = 0;
  }
  // row i's rule, and the draft in front of it (-1: none that counts)
  if (tid < rows) {
    int draft = -1, m = -1;
    if (c.drafts && first + tid > 0 && first + tid <= c.k) {
      draft = c.drafts[size_t(b) * c.k + first + tid - 1];
      if (draft < 0 || draft >= c.V) {
        if (lo == 0) atomicAdd(c.status + STATUS_WORD_BAD_INPUT, 1u);
        draft = -1;
      }
    }
    if (c.mask) {
      m = c.mask_rows ? c.mask_rows[t0 + tid] : t0 + tid;
      if (m < -1 || m >= c.n_masks) {
        if (lo == 0) atomicAdd(c.status + STATUS_WORD_BAD_INPUT, 1u);
        m = -1;
      }
    }
    s_draft[tid] = draft;
    s_mask[tid] = m;
  }
  __syncthreads();

  // ---- the request's tokens and biases of this slice
  const bool report = lo == 0 && first == 0;                 // one block of a request counts what is bad about it
  if (a.tables) {
    if (c.repetition) { u.r = c.repetition[b]; u.penalise_repeat = true; }
    if (c.frequency) { u.f = c.frequency[b]; u.subtract = true; }
    if (c.presence) { u.p = c.presence[b]; u.subtract = true; }
    const int32_t* text = c.history + size_t(b) * c.history_stride;
    int len = 0, prompt = 0, bad = 0;
    if (c.history) {
      const int l = c.history_lens ? c.history_lens[b] : c.history_stride, p = c.prompt_lens ? c.prompt_lens[b] : 0;
      len = min(max(l, 0), c.history_stride);
      prompt = min(max(p, 0), len);
      if (report && tid == 0 && (l < 0 || l > c.history_stride || p < 0 || p > len)) ++bad;
    }
    auto count = [&](int id, int j) {
      if (id >= lo && id < hi) {
        if (j < prompt) atomicOr(&table[id - lo], IN_PROMPT);
        else atomicAdd(&table[id - lo], 1u);
        atomicOr(&marked[(id - lo) >> 5], 1u << ((id - lo) & 31));
      } else if (report && (id < 0 || id >= c.V)) ++bad;
    };
    // 16-byte loads from the first boundary on
    const int head = min(len, int((16 - (reinterpret_cast<uintptr_t>(text) & 15)) & 15) / 4);
    if (tid < head) count(text[tid], tid);
    const int4* wide = reinterpret_cast<const int4*>(text + head);
    const int words = (len - head) / 4;
    int w = tid;
    for (; w + 3 * RULE_THREADS < words; w += 4 * RULE_THREADS) {
      int4 v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = wide[w + e * RULE_THREADS];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = head + 4 * (w + e * RULE_THREADS);
        count(v[e].x, j); count(v[e].y, j + 1); count(v[e].z, j + 2); count(v[e].w, j + 3);
      }
    }
    for (; w < words; w += RULE_THREADS) {
      const int4 v = wide[w];
      const int j = head + 4 * w;
      count(v.x, j); count(v.y, j + 1); count(v.z, j + 2); count(v.w, j + 3);
    }
    if (head + 4 * words + tid < len) count(text[head + 4 * words + tid], head + 4 * words + tid);
    if (c.drafts)
      for (int j = tid; j < min(first, c.k); j += RULE_THREADS) {
        const int id = c.drafts[size_t(b) * c.k + j];
        if (id >= lo && id < hi) count(id, INT_MAX);
      }
    __syncthreads();
    // Biases: one warp, entries in order.  Entries of one token add up in the order of the list (the first of them owns the place).
    if (c.bias_ids && tid < 32) {
      const int given = c.bias_counts ? c.bias_counts[b] : c.n_bias, m = min(max(given, 0), c.n_bias);
      if (report && lane == 0 && given != m) ++bad;
      int used = 0;
      for (int base = 0; base < m; base += 32) {
        const bool on = base + lane < m;
        const int id = on ? c.bias_ids[size_t(b) * c.n_bias + base + lane] : -1;
        const float v = on ? c.bias_values[size_t(b) * c.n_bias + base + lane] : 0.f;
        if (report && on && (id < 0 || id >= c.V)) ++bad;
        const bool in = on && id >= lo && id < hi;
        const uint32_t same = __match_any_sync(0xffffffffu, in ? id : -1 - lane);
        const bool owner = in && __ffs(same) - 1 == lane;
        const uint32_t had = in ? (table[id - lo] >> BIAS_SHIFT) & BIAS_BITS : 0u;
        const uint32_t fresh = __ballot_sync(0xffffffffu, owner && !had);
        const int at = had ? int(had) - 1 : used + __popc(fresh & ((1u << lane) - 1u));
        float sum = owner && had ? bias[at] : 0.f;
        for (int l = 0; l < 32; ++l) {
          const float x = __shfl_sync(0xffffffffu, v, l);
          if (owner && ((same >> l) & 1u)) sum += x;
        }
        if (owner) {
          bias[at] = sum;
          if (!had) {
            table[id - lo] |= uint32_t(at + 1) << BIAS_SHIFT;
            atomicOr(&marked[(id - lo) >> 5], 1u << ((id - lo) & 31));
          }
        }
        used += __popc(fresh);
        __syncwarp();
      }
    }
    if (bad) atomicAdd(c.status + STATUS_WORD_BAD_INPUT, uint32_t(bad));
    __syncthreads();
  }

  // ---- the rows
  const int mask_words = (c.V + 31) / 32;
  const bool in_place = c.in == c.out;
  for (int i = 0; i < rows; ++i) {
    const int t = t0 + i;
    const int draft = i && a.tables ? s_draft[i] : -1;
    if (draft >= lo && draft < hi) {                         // (the same for the whole block)
      __syncthreads();
      if (tid == 0) {
        table[draft - lo] += 1;
        marked[(draft - lo) >> 5] |= 1u << ((draft - lo) & 31);
      }
      __syncthreads();
    }
    const uint32_t* allowed = s_mask[i] < 0 ? nullptr : c.mask + size_t(s_mask[i]) * c.mask_stride;
    if (in_place && !a.tables && !allowed) continue;
    const TI* src = reinterpret_cast<const TI*>(c.in) + size_t(t) * c.ld_in;
    TO* dst = reinterpret_cast<TO*>(c.out) + size_t(t) * c.ld_out;
    auto one = [&](int v) {
      const bool touched = a.tables && ((marked[(v - lo) >> 5] >> ((v - lo) & 31)) & 1u);
      const bool out = allowed && !((allowed[v >> 5] >> (v & 31)) & 1u);
      if (in_place && !touched && !out) return;
      if (out) { dst[v] = from_f32<TO>(-INFINITY, c.status); return; }
      const TI x = src[v];
      if (touched) dst[v] = from_f32<TO>(ruled(to_f32(x), table[v - lo], u, bias), c.status);
      else if constexpr (std::is_same<TI, TO>::value) dst[v] = x;
      else dst[v] = from_f32<TO>(to_f32(x), c.status);
    };
    // single logits up to the row's first 16-byte boundary in the slice and behind its last, 16-byte words between
    const int from = min(hi, lo + int((16 - (reinterpret_cast<uintptr_t>(src + lo) & 15)) & 15) / int(sizeof(TI)));
    const int words = (hi - from) / VEC, rest = from + words * VEC;
    const bool out_words = (reinterpret_cast<uintptr_t>(dst + from) & 15) == 0;
    if (lo + tid < from) one(lo + tid);
    if (rest + tid < hi) one(rest + tid);
    for (int w = tid; w < words; w += RULE_AHEAD * RULE_THREADS) {
      Word<TI, VEC> x[RULE_AHEAD];
      uint32_t touched[RULE_AHEAD], out[RULE_AHEAD];
      constexpr uint32_t ALL = (1u << VEC) - 1u;
#pragma unroll
      for (int e = 0; e < RULE_AHEAD; ++e) {
        const int we = w + e * RULE_THREADS;
        touched[e] = out[e] = 0;
        x[e] = Word<TI, VEC>{};
        if (we >= words) continue;
        const int v = from + we * VEC;
        if (a.tables) touched[e] = bits_from(marked, v - lo, a.slice / 32) & ALL;
        if (allowed) out[e] = ~bits_from(allowed, v, mask_words) & ALL;
        touched[e] &= ~out[e];                               // (what is forbidden is nothing else)
        if (in_place ? ((touched[e] | out[e]) && out[e] != ALL) : out[e] != ALL) x[e] = *reinterpret_cast<const Word<TI, VEC>*>(src + v);
      }
#pragma unroll
      for (int e = 0; e < RULE_AHEAD; ++e) {
        const int we = w + e * RULE_THREADS;
        if (we >= words) continue;
        if (in_place && !(touched[e] | out[e])) continue;
        const int v = from + we * VEC;
        Word<TO, VEC> y;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          if constexpr (std::is_same<TI, TO>::value) y.v[j] = x[e].v[j];
          else y.v[j] = from_f32<TO>(to_f32(x[e].v[j]), c.status);
          if ((touched[e] >> j) & 1u) y.v[j] = from_f32<TO>(ruled(to_f32(x[e].v[j]), table[v + j - lo], u, bias), c.status);
          if ((out[e] >> j) & 1u) y.v[j] = from_f32<TO>(-INFINITY, c.status);
        }
        if (out_words) {
#pragma unroll
          for (int k = 0; k < int(sizeof(TO)) * VEC / 16; ++k) reinterpret_cast<uint4*>(dst + v)[k] = reinterpret_cast<const uint4*>(&y)[k];
        } else {
#pragma unroll
          for (int j = 0; j < VEC; ++j) dst[v + j] = y.v[j];
        }
      }
    }
  }
}

template <typename TI, typename TO>
cudaError_t launch_for(const RuleArgs& a, unsigned blocks, size_t smem, cudaStream_t stream) {
  return launch_pdl(adjust_logits_kernel<TI, TO>, dim3(blocks), dim3(RULE_THREADS), smem, stream, a);
}

}  // namespace

cudaError_t adjust_logits_launch(const LogitsCall& c, cudaStream_t stream) {
  RuleArgs a{};
  a.c = c;
  a.tables = (c.repetition || c.frequency || c.presence) && (c.history || c.drafts) ? 1 : 0;
  if (!a.tables) a.c.history = a.c.drafts = nullptr;
  if (c.bias_ids) a.tables = 1;
  // A block reads its request's whole text, so its slice is wide and its rows are many while there are four blocks for every SM.
  a.slice = 8192;
  a.rows = MOST_ROWS;
  auto blocks = [&] {
    a.slices = (c.V + a.slice - 1) / a.slice;
    return (long long)(a.slices) * (c.cu_q ? c.T / a.rows + (c.B < c.T ? c.B : c.T) : c.T);
  };
  while (a.rows > 4 && blocks() < 4 * 148) a.rows /= 2;
  while (a.slice > 1024 && blocks() < 4 * 148) a.slice /= 2;
  while (a.rows > 1 && blocks() < 4 * 148) a.rows /= 2;
  const long long n = blocks();
  if (n > INT_MAX) return cudaErrorInvalidConfiguration;
  const size_t smem = a.tables ? size_t(a.slice) * 4 + a.slice / 8 + (c.bias_ids ? size_t(c.n_bias) * 4 : 0) : 0;
  if (c.in_dtype == CHUNK_F32) return launch_for<float, float>(a, unsigned(n), smem, stream);
  if (c.in_dtype == CHUNK_F16)
    return c.out_dtype == CHUNK_F32 ? launch_for<__half, float>(a, unsigned(n), smem, stream) : launch_for<__half, __half>(a, unsigned(n), smem, stream);
  return c.out_dtype == CHUNK_F32 ? launch_for<__nv_bfloat16, float>(a, unsigned(n), smem, stream)
                                  : launch_for<__nv_bfloat16, __nv_bfloat16>(a, unsigned(n), smem, stream);
}

}  // namespace hspec
