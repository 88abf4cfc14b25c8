// Logit adjustment per tree node: penalties for repeated tokens, biases and
// token masks (definition: d2sd_logits_args in d2sd.h).
//
// The adjustment of token j is the same for all nodes of a request but for the
// few draft tokens on their root paths, so it is y = x * (x > 0 ? mp : mn) + a
// with mp, mn and a per (request, token). A workgroup takes a chunk of the
// vocabulary of one request, builds these from the request's token history and
// bias list (counted in LDS, kept in registers, 8 tokens a thread), and then
// streams the chunk of up to kMaxPer of its nodes' rows past them: one read and
// one write of the logits, plus a bit per token where the node has a mask. Draft
// tokens in the chunk are listed per owning thread, with a bit for each of the
// workgroup's nodes that they are an ancestor of; a thread writes the tokens
// with a node's bit once more, corrected, so the loop over the rows has no
// barrier and seldom leaves its straight path. Counts are integers and bias
// lists are summed in order, so results do not depend on timing.
//
// Bound by memory: 2 bytes in and 2 out per bf16 logit. Occupancy hides its
// latency, so the registers of a thread decide: with 8 tokens (64 registers,
// eight workgroups per CU) 2560 rows of 32000 bf16 logits with 4000 tokens of
// history, 100 biases and 16 masks take 80 us, 4.1 TB/s, where 328 MB at a copy's
// rate would take 70. Measured at 83: 16 tokens (116 registers) 96, the next
// row's loads before this one's stores (70 registers) 89, 128 or 512 threads 99
// and 88, at most 4 or 12 nodes per workgroup 98 and 83. With 384 rows of 150001
// logits, which start at any even address, 55 us, 4.2 TB/s. Every workgroup goes
// through its request's whole history, so that the time grows with it: the 2560
// rows take 76 us with a token of history, 81 with 4000, 91 with 16000 and 110 with 32000.
#include "launchers.h"

namespace d2sd {

namespace {

constexpr int kThr = 256;
constexpr int kElems = 8;                           // tokens per thread
constexpr int kChunk = kThr * kElems;
constexpr int kListMax = D2SD_MAX_B + D2SD_MAX_B * (D2SD_MAX_B - 1) / 2;   // nodes of a request
constexpr int kMaskWords = (kListMax + 31) / 32;
constexpr int kMaxPer = 8;                          // nodes per workgroup, at most
static_assert(kMaxPer <= 12, "bits of a list entry");
constexpr int kBurst = 8;                           // loads of the history that a thread has in flight
constexpr uint32_t kNoEntry = 0xfffu;
constexpr uint32_t kPromptBit = 1u << 31;
static_assert(kListMax < (int)kNoEntry, "list entries are linked by 12 bits");

template <typename T>
struct Vec;
template <>
struct Vec<__bf16> {
  static constexpr int N = 8;
};
template <>
struct Vec<float> {
  static constexpr int N = 4;
};

// 16 bytes at an address aligned to the element only: rows of an odd
// vocabulary start anywhere, and gfx9 global accesses take any alignment.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
struct __attribute__((packed)) Loose16 {
  u32x4 v;
};

template <typename T>
__device__ __forceinline__ u32x4 load_vec(const T* row, int j, int V) {
  constexpr int N = Vec<T>::N;
  if (j + N <= V) return reinterpret_cast<const Loose16*>(row + j)->v;
  union {
    T e[N];
    u32x4 v;
  } u;
#pragma unroll
  for (int i = 0; i < N; ++i) u.e[i] = row[min(j + i, V - 1)];
  return u.v;
}
template <typename T>
__device__ __forceinline__ void store_vec(T* row, int j, int V, const u32x4& x) {
  constexpr int N = Vec<T>::N;
  if (j + N <= V) {
    reinterpret_cast<Loose16*>(row + j)->v = x;
    return;
  }
  union {
    u32x4 v;
    T e[N];
  } u;
  u.v = x;
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (j + i < V) row[j + i] = u.e[i];
}

__device__ __forceinline__ void unpack(const u32x4& x, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(x[i] << 16);
    v[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack(const u32x4& x, float (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(x[i]);
}
__device__ __forceinline__ u32x4 pack(const float (&v)[8]) {
  union {
    __bf16 e[8];
    u32x4 v;
  } u;
#pragma unroll
  for (int i = 0; i < 8; ++i) u.e[i] = (__bf16)v[i];
  return u.v;
}
__device__ __forceinline__ u32x4 pack(const float (&v)[4]) {
  return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
}

template <typename T>
__global__ __launch_bounds__(kThr) void adjust_logits_kernel(d2sd_logits_args a, int chunks, int groups, int nodes_per_group) {
  constexpr int N = Vec<T>::N;                      // tokens of a 16-byte vector
  constexpr int kVecs = kElems / N;                 // vectors per thread: tokens v kThr N + t N .. + N of the chunk
  __shared__ uint32_t s_tok[kChunk];                // counts, then bias values
  __shared__ uint32_t s_list[kListMax];             // next entry << 16 | token of the thread << 12 | the nodes that it is an ancestor of
  __shared__ uint32_t s_head[kThr];
  __shared__ uint32_t s_anc[kMaxPer][kMaskWords];   // ancestor masks of the workgroup's nodes
  __shared__ int s_row[kMaxPer];                    // their token masks
  __shared__ int s_n;

  int rest = blockIdx.x;
  const int ck = rest % chunks; rest /= chunks;
  const int grp = rest % groups;
  const int b = rest / groups;
  const int base = clampi(a.node_indptr[b], 0, a.total_nodes);
  const int nodes = clampi(a.node_indptr[b + 1], base, min(a.total_nodes, base + a.max_nodes)) - base;
  const int n0 = grp * nodes_per_group, n1 = min(nodes, n0 + nodes_per_group);
  if (n0 >= n1) return;
  const int c0 = ck * kChunk;                       // tokens c0 .. c0 + here - 1
  const int here = min(kChunk, a.vocab - c0);
  const int t = threadIdx.x;

  // ---- what the request's history and biases make of the chunk ----
#pragma unroll
  for (int i = 0; i < kElems; ++i) s_tok[i * kThr + t] = 0;
  const int node_words = (nodes + 31) >> 5;
  for (int i = t; i < (n1 - n0) * node_words; i += kThr)
    s_anc[i / node_words][i % node_words] = a.anc_mask[(size_t)(base + n0 + i / node_words) * a.mask_words + i % node_words];
  if (t < n1 - n0) s_row[t] = a.num_masks > 0 ? min(a.mask_row[base + n0 + t], a.num_masks - 1) : -1;
  s_head[t] = kNoEntry;
  if (t == 0) s_n = 0;
  __syncthreads();
  if (a.max_history > 0) {
    const int* hist = a.history + (size_t)b * a.max_history;
    const int len = clampi(a.history_len[b], 0, a.max_history);
    const int prompt = a.prompt_len ? clampi(a.prompt_len[b], 0, len) : 0;
    for (int i0 = t; i0 < len; i0 += kBurst * kThr) {
      int tok[kBurst];
#pragma unroll
      for (int k = 0; k < kBurst; ++k) tok[k] = hist[min(i0 + k * kThr, len - 1)];
#pragma unroll
      for (int k = 0; k < kBurst; ++k) {
        const int i = i0 + k * kThr;
        const uint32_t off = (uint32_t)tok[k] - (uint32_t)c0;
        if (i >= len || off >= (uint32_t)here) continue;
        if (i < prompt)
          atomicOr(&s_tok[off], kPromptBit);
        else
          atomicAdd(&s_tok[off], 1u);
      }
    }
  }
  __syncthreads();
  const float rep = a.repetition ? a.repetition[b] : 1.0f;
  const float inv_rep = 1.0f / rep;
  const float pres = a.presence ? a.presence[b] : 0.0f;
  const float freq = a.frequency ? a.frequency[b] : 0.0f;
  uint32_t seen = 0, counted = 0;                   // a bit per token of the thread
  float add[kElems];
#pragma unroll
  for (int i = 0; i < kElems; ++i) {
    const uint32_t c = s_tok[i / N * (kThr * N) + t * N + i % N];
    const float n = (float)(c & ~kPromptBit);
    add[i] = c & ~kPromptBit ? -(n * freq) - pres : 0.0f;
    seen |= (c ? 1u : 0u) << i;
    counted |= (c & ~kPromptBit ? 1u : 0u) << i;
  }
  if (a.max_bias > 0) {
    uint32_t* s_owner = s_list;                     // free until the list is made
    static_assert(kListMax >= kChunk);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kElems; ++i) {
      s_tok[i * kThr + t] = 0;
      s_owner[i * kThr + t] = ~0u;
    }
    __syncthreads();
    const int* tok = a.bias_token + (size_t)b * a.max_bias;
    const float* val = a.bias_value + (size_t)b * a.max_bias;
    const int len = a.bias_len ? clampi(a.bias_len[b], 0, a.max_bias) : a.max_bias;
    // kThr entries at a time; in a round every token's first entry that is left
    // adds its value, so that they are summed in order: one round without
    // repeats, and a list that is padded with zeros has none
    for (int i0 = 0; i0 < len; i0 += kThr) {
      const int i = i0 + t;
      const uint32_t off = i < len ? (uint32_t)tok[i] - (uint32_t)c0 : ~0u;
      const float value = i < len ? val[i] : 0.0f;
      bool left = off < (uint32_t)here && value != 0.0f;
      while (__syncthreads_or(left)) {
        if (left) atomicMin(&s_owner[off], (uint32_t)t);
        __syncthreads();
        if (left && s_owner[off] == (uint32_t)t) {
          s_tok[off] = __float_as_uint(__uint_as_float(s_tok[off]) + value);
          s_owner[off] = ~0u;
          left = false;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kElems; ++i) add[i] += __uint_as_float(s_tok[i / N * (kThr * N) + t * N + i % N]);
  }
  // draft tokens of the chunk, linked by the thread that owns them
  for (int n = t; n < nodes; n += kThr) {
    const uint32_t off = (uint32_t)a.draft_tokens[base + n] - (uint32_t)c0;
    if (off >= (uint32_t)here || a.depth[base + n] <= 0) continue;
    const int owner = (int)off % (kThr * N) / N;
    const uint32_t e = (uint32_t)off / (kThr * N) * N + off % N;
    const uint32_t at = (uint32_t)atomicAdd(&s_n, 1);
    uint32_t below = 0;                             // a bit per node of the workgroup: n is its ancestor or itself
    for (int k = 0; k < n1 - n0; ++k) below |= ((s_anc[k][n >> 5] >> (n & 31)) & 1u) << k;
    s_list[at] = atomicExch(&s_head[owner], at) << 16 | e << 12 | below;
  }
  __syncthreads();
  const uint32_t head = s_head[t];
  uint32_t below = 0;                               // the nodes that the thread has something more for
  for (uint32_t at = head; at != kNoEntry; at = s_list[at] >> 16) below |= s_list[at] & ((1u << kMaxPer) - 1u);

  // ---- the rows ----
  const T* in = static_cast<const T*>(a.logits);
  T* out = static_cast<T*>(a.out);
  const int words = (a.vocab + 31) >> 5;
  struct Row {
    u32x4 raw[kVecs];
    uint32_t allowed[kVecs];
  };
  auto fetch = [&](int n, Row& r) {
    const size_t row = (size_t)(base + n) * a.vocab;
    const int mr = s_row[n - n0];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      const int j = c0 + v * (kThr * N) + t * N;
      r.allowed[v] = ~0u;
      if (j >= a.vocab) continue;
      r.raw[v] = load_vec(in + row, j, a.vocab);
      if (mr >= 0) r.allowed[v] = a.token_mask[(size_t)mr * words + (j >> 5)] >> (j & 31);
    }
  };
  auto finish = [&](int n, const Row& r) {
    const size_t row = (size_t)(base + n) * a.vocab;
    // where x counts as a repeated token's, and what is added to it: y
    auto adjust = [&](float x, bool repeated, float more) { return x * (repeated ? (x > 0.0f ? inv_rep : rep) : 1.0f) + more; };
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      const int j = c0 + v * (kThr * N) + t * N;
      if (j >= a.vocab) continue;
      float x[N];
      unpack(r.raw[v], x);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        x[i] = adjust(x[i], (seen >> (v * N + i)) & 1u, add[v * N + i]);
        if (!((r.allowed[v] >> i) & 1u)) x[i] = -INFINITY;
      }
      store_vec(out + row, j, a.vocab, pack(x));
    }
    if (!((below >> (n - n0)) & 1u)) return;
    // tokens that the node or its ancestors draft, over what was written
    for (uint32_t at = head; at != kNoEntry; at = s_list[at] >> 16) {
      if (!((s_list[at] >> (n - n0)) & 1u)) continue;
      const uint32_t e = (s_list[at] >> 12) & 15u;
      int hits = 0;                                 // how many of them draft it
      for (uint32_t k = head; k != kNoEntry; k = s_list[k] >> 16)
        if (((s_list[k] >> 12) & 15u) == e) hits += (s_list[k] >> (n - n0)) & 1u;
      float x = 0.0f, more = 0.0f;
      bool allowed = true;
#pragma unroll
      for (int v = 0; v < kVecs; ++v) {
        float u[N];
        unpack(r.raw[v], u);
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (e == (uint32_t)(v * N + i)) {
            x = u[i];
            more = add[v * N + i];
            allowed = (r.allowed[v] >> i) & 1u;
          }
      }
      more += -((float)hits * freq) - ((counted >> e) & 1u ? 0.0f : pres);
      out[row + c0 + e / N * (kThr * N) + t * N + e % N] = allowed ? (T)adjust(x, true, more) : (T)-INFINITY;
    }
  };
  for (int n = n0; n < n1; ++n) {
    Row r;
    fetch(n, r);
    finish(n, r);
  }
}

}  // namespace

hipError_t launch_adjust_logits(const d2sd_logits_args& a, hipStream_t stream) {
  const int chunks = ceil_div(a.vocab, kChunk);
  // Nodes per workgroup: the history is counted once for all of them, but
  // there should be some eight workgroups for each of the 256 CUs.
  const long long rows = (long long)a.total_nodes * chunks;
  const int per = (int)max(1ll, min((long long)kMaxPer, rows / 2048));
  const int groups = ceil_div(a.max_nodes, per);
  const dim3 grid((unsigned)((long long)a.batch * groups * chunks));
  if (a.dtype == D2SD_BF16)
    hipLaunchKernelGGL(adjust_logits_kernel<__bf16>, grid, dim3(kThr), 0, stream, a, chunks, groups, per);
  else
    hipLaunchKernelGGL(adjust_logits_kernel<float>, grid, dim3(kThr), 0, stream, a, chunks, groups, per);
  return hipGetLastError();
}

}  // namespace d2sd
