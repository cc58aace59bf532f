// What a request's rules do to the target's logits between the LM head and the verification: penalties for repeated tokens, biases, allowed tokens.
//
// For row i of request b, whose text is history[b, :len] and then its drafts 0 .. i - 1:
//   z <- z / r if z > 0, else z r          for every token of the text (prompt, answer or drafts)
//   z <- z - f count - p                   for every token of the answer or the drafts, `count` times there
//   z <- z + bias;   z <- -infinity where the row's bits forbid the token
// Bound by memory: every logit is read and written once (in place: only what changes).  A block takes a slice of the vocabulary and some rows of one
// request.  It counts the request's tokens that fall into the slice in shared memory (whole numbers, so that the order of the additions does not
// matter) and lists those that any rule but the bits touches.  A row is then streamed in 16-byte words, which knows of the allowed bits alone, and the
// listed tokens are put right behind it: every warp has some of them, and with the rules inside the stream it is bound by its instructions (32 requests,
// 17 rows of 128 256, texts of 512 to 8192 tokens: 246 us; so 115, 3.7 TB/s of the
// 422 MB that have to move.  128 of them with fp32 rows: 505 to 540 us, 5 TB/s).  Between two rows the draft in front of the second is counted.
#include "chunk_scan.cuh"

#include <atomic>
#include <climits>
#include <type_traits>

namespace hspec {

namespace {

constexpr int RULE_THREADS = 256;
constexpr int MOST_ROWS = 32;                     // of a block
constexpr int RULE_AHEAD = 4;                     // 16-byte words of a row that a thread has
constexpr uint32_t IN_PROMPT = 0x80000000u;       // a token's word: said in the prompt, bias entry + 1, times said since
constexpr int BIAS_SHIFT = 20;
constexpr uint32_t BIAS_BITS = 0x7ff, COUNT_BITS = (1u << BIAS_SHIFT) - 1;

struct RuleArgs {
  LogitsCall c;
  int slice, slices, rows;                        // tokens of a slice (at most 2^16), slices, rows of a block
  int biases;                                     // room for biases, in multiples of four
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

// STAGED: with tables and out of place, the rows come through shared memory, the next one under way, so that the listed tokens find theirs there.
template <typename TI, typename TO, bool STAGED>
__global__ void __launch_bounds__(RULE_THREADS, 4) adjust_logits_kernel(RuleArgs a) {
  constexpr int VEC = 16 / sizeof(TI);
  const LogitsCall& c = a.c;
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) uint32_t table[];          // [slice] words of the tokens
  uint16_t* list = reinterpret_cast<uint16_t*>(table + a.slice);       // [slice] those that are not zero
  float* bias = reinterpret_cast<float*>(list + a.slice);
  uint8_t* stage = reinterpret_cast<uint8_t*>(bias + a.biases);                  // two rows of the slice, then two of its allowed bits
  __shared__ int s_draft[MOST_ROWS], s_mask[MOST_ROWS], listed;
  const int tid = threadIdx.x, lane = tid & 31;
  const int lo = (blockIdx.x % a.slices) * a.slice, hi = min(lo + a.slice, c.V);

  // ---- the block's request and rows (every warp looks for itself)
  ChunkItem item{int(blockIdx.x) / a.slices, int(blockIdx.x) / a.slices, 1, 0};
  if (c.cu_q)
    item = chunk_item(c.B, a.rows, 0, item.b, lane, [&](int b) {
      const ChunkRequest r = chunk_request(c.cu_q[b], c.cu_q[b + 1], 0, c.T, 0);
      return ChunkRows{r.q0, r.n};
    });
  if (blockIdx.x == 0 && c.cu_q)
    for (int r = tid; r < c.B; r += RULE_THREADS)
      if (chunk_request_bad(c.cu_q[r], c.cu_q[r + 1], INT_MAX, c.T, INT_MAX)) atomicAdd(c.status + STATUS_WORD_BAD_INPUT, 1u);
  if (item.b < 0) return;
  const int b = item.b, first = item.first, t0 = item.q0 + first, rows = min(a.rows, item.n - first);
  Rules u{};
  if (a.tables) {
    for (int i = tid; i < a.slice / 4; i += RULE_THREADS) reinterpret_cast<uint4*>(table)[i] = make_uint4(0, 0, 0, 0);
    if (tid == 0) listed = 0;
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
      if (uint32_t(id - lo) < uint32_t(hi - lo)) {
        // (the first one to find a token lists it: in any order, no result depends on it)
        const uint32_t had = j < prompt ? atomicOr(&table[id - lo], IN_PROMPT) : atomicAdd(&table[id - lo], 1u);
        if (!had) list[atomicAdd(&listed, 1)] = uint16_t(id - lo);
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
            if (!table[id - lo]) list[atomicAdd(&listed, 1)] = uint16_t(id - lo);
            table[id - lo] |= uint32_t(at + 1) << BIAS_SHIFT;
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
  // a row as the block sees it: 16-byte words from its first boundary in the slice on, single logits in front of them and behind
  struct Row {
    const uint32_t* allowed;
    const TI* src;
    TO* dst;
    int from, words;
  };
  const TI* src = reinterpret_cast<const TI*>(c.in) + size_t(t0) * c.ld_in;
  TO* dst = reinterpret_cast<TO*>(c.out) + size_t(t0) * c.ld_out;
  auto row_of = [&](int i) {                                 // (rows come one after another)
    Row r;
    r.allowed = s_mask[i] < 0 ? nullptr : c.mask + size_t(s_mask[i]) * c.mask_stride;
    r.src = src;
    r.dst = dst;
    src += c.ld_in;
    dst += c.ld_out;
    r.from = min(hi, lo + int((16 - (reinterpret_cast<uintptr_t>(r.src + lo) & 15)) & 15) / int(sizeof(TI)));
    r.words = in_place && !r.allowed ? 0 : (hi - r.from) / VEC;
    return r;
  };
  constexpr uint32_t ALL = (1u << VEC) - 1u;
  Word<TI, VEC> x[RULE_AHEAD];
  uint32_t out[RULE_AHEAD];                                  // tokens of the word that are not allowed
  auto load = [&](const Row& r) {
#pragma unroll
    for (int e = 0; e < RULE_AHEAD; ++e) {
      const int w = tid + e * RULE_THREADS, v = r.from + w * VEC;
      out[e] = 0;
      if (w >= r.words) continue;
      if (r.allowed) out[e] = ~bits_from(r.allowed, v, mask_words) & ALL;
      x[e] = *reinterpret_cast<const Word<TI, VEC>*>(r.src + v);          // (without waiting for the bits)
    }
  };
  auto store = [&](const Row& r) {
    const bool out_words = (reinterpret_cast<uintptr_t>(r.dst + r.from) & (sizeof(Word<TO, VEC>) - 1)) == 0;
#pragma unroll
    for (int e = 0; e < RULE_AHEAD; ++e) {
      const int w = tid + e * RULE_THREADS, v = r.from + w * VEC;
      if (e * RULE_THREADS >= r.words) break;
      if (w >= r.words || (in_place && !out[e])) continue;
      Word<TO, VEC> y;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        if constexpr (std::is_same<TI, TO>::value) y.v[j] = x[e].v[j];
        else y.v[j] = from_f32<TO>(to_f32(x[e].v[j]), c.status);
      }
      if (r.allowed) {                                       // (of the whole row: no branch for each word)
#pragma unroll
        for (int j = 0; j < VEC; ++j)
          if ((out[e] >> j) & 1u) y.v[j] = from_f32<TO>(-INFINITY, c.status);
      }
      if (out_words) {
        // (eight 32-bit logits in one store: two of 16 bytes would each leave every other half of a sector to the other one)
        if constexpr (sizeof(y) == 32)
          asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(r.dst + v), "f"(float(y.v[0])), "f"(float(y.v[1])), "f"(float(y.v[2])),
                       "f"(float(y.v[3])), "f"(float(y.v[4 % VEC])), "f"(float(y.v[5 % VEC])), "f"(float(y.v[6 % VEC])), "f"(float(y.v[7 % VEC])) : "memory");
        else
          *reinterpret_cast<uint4*>(r.dst + v) = *reinterpret_cast<const uint4*>(&y);
      } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) r.dst[v + j] = y.v[j];
      }
    }
    // (at most 7 logits on either side)
    const int rest = r.from + (hi - r.from) / VEC * VEC;
    if ((r.from > lo || rest < hi) && (!in_place || r.allowed)) {
      const int single = tid < 8 ? lo + tid : rest + tid - 8;
      if (tid < 16 && (tid < 8 ? single < r.from : single < hi)) {
        if (r.allowed && !((r.allowed[single >> 5] >> (single & 31)) & 1u)) r.dst[single] = from_f32<TO>(-INFINITY, c.status);
        else if (!in_place) r.dst[single] = from_f32<TO>(to_f32(r.src[single]), c.status);
      }
    }
  };
  auto listed_tokens = [&](int i, const Row& r, const TI* staged) {
    const int draft = i ? s_draft[i] : -1;                   // with the draft in front of this row among them
    if (draft >= lo && draft < hi) {                         // (the same for the whole block)
      if (tid == 0) {
        if (table[draft - lo] == 0) list[listed++] = uint16_t(draft - lo);
        table[draft - lo] += 1;
      }
      __syncthreads();
    }
    const int many = listed;
    for (int l = tid; l < many; l += RULE_THREADS) {
      const int at = list[l], v = lo + at, w = v - r.from;
      if (r.allowed && !((r.allowed[v >> 5] >> (v & 31)) & 1u)) continue;
      const TI z = STAGED && w >= 0 && w < r.words * VEC ? staged[w] : r.src[v];
      r.dst[v] = from_f32<TO>(ruled(to_f32(z), table[at], u, bias), c.status);
    }
  };
  Row row = row_of(0);
  if constexpr (STAGED) {
    constexpr int BYTES = RULE_AHEAD * RULE_THREADS * 16;
    uint32_t* bits = reinterpret_cast<uint32_t*>(stage + 2 * BYTES);
    const int bit_words = (hi - lo + 31) / 32;
    auto fetch = [&](const Row& r, int buf) {
      for (int w = tid; w < r.words; w += RULE_THREADS) cp_async16(smem_u32(stage + buf * BYTES + w * 16), r.src + r.from + w * VEC, true);
      if (r.allowed && tid < bit_words)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(bits + buf * (a.slice / 32) + tid)), "l"(r.allowed + lo / 32 + tid) : "memory");
      cp_async_commit();
    };
    fetch(row, 0);
    for (int i = 0; i < rows; ++i) {
      Row now = row;
      const bool ruled_out = now.allowed != nullptr;
      now.allowed = bits + (i & 1) * (a.slice / 32) - lo / 32;
      if (!ruled_out) now.allowed = nullptr;
      if (i + 1 < rows) {
        row = row_of(i + 1);
        fetch(row, (i + 1) & 1);                             // (its place was read before the barrier at the row's end)
      } else {
        cp_async_commit();
      }
      cp_async_wait<1>();                                    // (a thread streams the words that it has fetched itself; the bits are others')
      if (ruled_out) __syncthreads();
      const uint8_t* mine = stage + (i & 1) * BYTES;
#pragma unroll
      for (int e = 0; e < RULE_AHEAD; ++e) {
        const int w = tid + e * RULE_THREADS;
        out[e] = 0;
        if (e * RULE_THREADS >= now.words) break;
        if (w >= now.words) continue;
        if (now.allowed) out[e] = ~bits_from(now.allowed, now.from + w * VEC, lo / 32 + bit_words) & ALL;
        x[e] = *reinterpret_cast<const Word<TI, VEC>*>(mine + w * 16);
      }
      store(now);
      __syncthreads();                                       // (the row is streamed, and all of it is in shared memory for everyone)
      listed_tokens(i, now, reinterpret_cast<const TI*>(mine));
      __syncthreads();
    }
  } else {
    load(row);
    for (int i = 0; i < rows; ++i) {
      store(row);
      const Row now = row;
      if (i + 1 < rows) {                                    // the next row is under way while the listed tokens of this one are dealt with
        row = row_of(i + 1);
        load(row);
      }
      if (!a.tables) continue;
      __syncthreads();                                       // (the row is streamed, the listed tokens of the one before are done)
      listed_tokens(i, now, nullptr);
    }
  }
}

template <typename TI, typename TO, bool STAGED>
cudaError_t launch_as(const RuleArgs& a, unsigned blocks, size_t smem, cudaStream_t stream) {
  if (smem > 40 * 1024) {                                    // (with what the kernel has besides, up to 48 KB go without asking)
    static std::atomic<uint32_t> ready{0};                   // devices on which the kernel has been told how much it may take
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && (dev >= 32 || !(ready.load() >> dev & 1u)))
      e = cudaFuncSetAttribute(adjust_logits_kernel<TI, TO, STAGED>, cudaFuncAttributeMaxDynamicSharedMemorySize, 96 * 1024);
    if (e != cudaSuccess) return e;
    if (dev < 32) ready.fetch_or(1u << dev);
  }
  return launch_pdl(adjust_logits_kernel<TI, TO, STAGED>, dim3(blocks), dim3(RULE_THREADS), smem, stream, a);
}
template <typename TI, typename TO>
cudaError_t launch_for(const RuleArgs& a, unsigned blocks, cudaStream_t stream) {
  const size_t smem = a.tables ? size_t(a.slice) * 6 + size_t(a.biases) * 4 : 0;
  return a.tables && a.c.in != a.c.out ? launch_as<TI, TO, true>(a, blocks, smem + 2 * (RULE_AHEAD * RULE_THREADS * 16 + a.slice / 8), stream)
                                       : launch_as<TI, TO, false>(a, blocks, smem, stream);
}

}  // namespace

cudaError_t adjust_logits_launch(const LogitsCall& c, cudaStream_t stream) {
  RuleArgs a{};
  a.c = c;
  a.tables = (c.repetition || c.frequency || c.presence) && (c.history || c.drafts) ? 1 : 0;
  if (!a.tables) a.c.history = a.c.drafts = nullptr;
  if (c.bias_ids) a.tables = 1;
  a.biases = c.bias_ids ? (c.n_bias + 3) / 4 * 4 : 0;
  // With tables a block reads its request's whole text, so its slice is wide and its rows are many while there are several waves of blocks.  Without,
  // nothing is shared between its rows.
  a.slice = RULE_AHEAD * RULE_THREADS * 4;                   // (a row of 32-bit logits; 16-bit ones take half the words)
  if (!a.tables && c.in_dtype != CHUNK_F32) a.slice *= 2;
  a.rows = a.tables ? MOST_ROWS : 1;
  auto blocks = [&] {
    a.slices = (c.V + a.slice - 1) / a.slice;
    return (long long)(a.slices) * (c.cu_q ? c.T / a.rows + (c.B < c.T ? c.B : c.T) : c.T);
  };
  while (a.rows > 8 && blocks() < 8 * 148) a.rows /= 2;
  while (a.rows > 4 && blocks() < 4 * 148) a.rows /= 2;
  while (a.slice > 1024 && blocks() < 4 * 148) a.slice /= 2;
  while (a.rows > 1 && blocks() < 4 * 148) a.rows /= 2;
  const long long n = blocks();
  if (n > INT_MAX) return cudaErrorInvalidConfiguration;
  if (c.in_dtype == CHUNK_F32) return launch_for<float, float>(a, unsigned(n), stream);
  if (c.in_dtype == CHUNK_F16)
    return c.out_dtype == CHUNK_F32 ? launch_for<__half, float>(a, unsigned(n), stream) : launch_for<__half, __half>(a, unsigned(n), stream);
  return c.out_dtype == CHUNK_F32 ? launch_for<__nv_bfloat16, float>(a, unsigned(n), stream)
                                  : launch_for<__nv_bfloat16, __nv_bfloat16>(a, unsigned(n), stream);
}

}  // namespace hspec
