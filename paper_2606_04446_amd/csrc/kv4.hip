// The 4-bit paged cache: new tokens quantised as they are written (prompts,
// accepted paths), and positions read back as values.
//
// A row (one token of one KV head) is 128 values in four blocks of 32, each
// with its own power of two. Sixteen lanes take a row, eight values each, so
// that four lanes (a DPP quad) hold a block: its largest magnitude is two quad
// exchanges away, 2^e follows from that magnitude's bits without a logarithm,
// and x / 2^e is rounded to E2M1 by the conversion instruction. Every step is
// exact but that rounding. All three are copies with a little arithmetic:
// bound by memory, and for small calls by the launch.
//
// A prompt's tiles are (page, KV head): 256 threads hold the page's 16 rows,
// so the codes leave as 1 KB in a row and the values arrive 256 (bf16) or 512
// bytes at a time. Workgroups take a page of a request and a few of its heads.
// Four prompts of 1000 to 8191 tokens, 8 heads, bf16: appended in 20 us and read
// back in 17 (95 MB each: 4.8 and 5.6 TB/s, part of it from the Infinity
// Cache); two contexts of 32768 tokens (340 MB) are read in 71 us, 4.8 TB/s.
#include "kv4_device.h"
#include "launchers.h"

namespace d2sd {

namespace {

constexpr int kKv4Threads = 256;
constexpr int kRowLanes = 16;                       // lanes per row, 8 values each
constexpr int kHeadsPerGroup = 2;                   // KV heads per workgroup of the paged kernels

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p);
  const float4 b = *reinterpret_cast<const float4*>(p + 4);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load8(const __bf16* p, float (&v)[8]) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void store8(float* p, uint32_t code, float scale) {
  float v[8];
  kv4_decode8(code, scale, v);
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(__bf16* p, uint32_t code, float scale) {
  *reinterpret_cast<uint4*>(p) = kv4_decode8_bf16(code, scale);
}

// Quantises eight values of lane `sub` (0..15) of a row and stores them; all
// four lanes of a quad have to be active.
__device__ __forceinline__ void write_row8(const float (&v)[8], uint8_t* codes, uint8_t* scales, size_t row, int sub) {
  uint32_t top = 0;   // magnitudes compare as integers, NaN above all
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, false));   // quad_perm [1,0,3,2]
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xf, 0xf, false));   // quad_perm [2,3,0,1]
  const int byte = kv4_scale_byte(top);
  // the codes of a block that reads as NaN do not matter, but are the same every time
  const uint32_t code = byte == kScaleNan ? 0u : kv4_encode8(v, kv4_scale((uint32_t)byte));
  *reinterpret_cast<uint32_t*>(codes + row * kKv4RowBytes + sub * 4) = code;
  if ((sub & 3) == 0) scales[row * kKv4Blocks + (sub >> 2)] = (uint8_t)byte;
}

// Row of the cache that holds position pos of a request, for KV head h.
__device__ __forceinline__ size_t cache_row(const int* table, int pos, int num_pages, int hkv, int h) {
  const int page = clampi(table[pos / D2SD_PAGE_SIZE], 0, num_pages - 1);
  return ((size_t)page * hkv + h) * D2SD_PAGE_SIZE + pos % D2SD_PAGE_SIZE;
}

// The tokens of request b among the rows of a ragged batch.
struct Span {
  int base, len;
};
__device__ __forceinline__ Span span_of(const int* indptr, int b, int total, int most) {
  const int base = clampi(indptr[b], 0, total);
  const int end = clampi(indptr[b + 1], base, total);
  return {base, min(end - base, most)};
}

template <typename T>
__global__ __launch_bounds__(kKv4Threads) void append_kv4_kernel(
    int hkv, int pages, int num_pages, int max_pages, int max_ctx, const int* __restrict__ token_indptr, int total,
    int max_tokens, const T* __restrict__ k, const T* __restrict__ v, const int* __restrict__ page_table,
    const int* __restrict__ ctx_len, d2sd_kv4_cache cache) {
  const int b = blockIdx.x / pages;
  const int C = clampi(ctx_len[b], 0, max_ctx);
  const Span s = span_of(token_indptr, b, total, min(max_tokens, max_pages * D2SD_PAGE_SIZE - C));
  // page number blockIdx.x % pages of those the new tokens touch
  const int pos = (C / D2SD_PAGE_SIZE + blockIdx.x % pages) * D2SD_PAGE_SIZE + threadIdx.x / kRowLanes;
  if (pos < C || pos - C >= s.len) return;           // whole rows of lanes
  const int sub = threadIdx.x % kRowLanes;
  const int h0 = blockIdx.y * kHeadsPerGroup;
  const int* table = page_table + (size_t)b * max_pages;
#pragma unroll
  for (int i = 0; i < kHeadsPerGroup; ++i) {
    const int h = h0 + i;
    if (h >= hkv) break;
    const size_t src = ((size_t)(s.base + pos - C) * hkv + h) * kKv4Dim + sub * 8;
    const size_t row = cache_row(table, pos, num_pages, hkv, h);
    float x[8], y[8];
    load8(k + src, x);
    load8(v + src, y);
    write_row8(x, cache.k, cache.k_scale, row, sub);
    write_row8(y, cache.v, cache.v_scale, row, sub);
  }
}

// Behind the append, which reads ctx_len in many workgroups.
__global__ __launch_bounds__(kKv4Threads) void advance_kernel(int batch, int max_pages, int max_ctx,
                                                              const int* __restrict__ token_indptr, int total,
                                                              int max_tokens, int* __restrict__ ctx_len) {
  const int b = blockIdx.x * kKv4Threads + threadIdx.x;
  if (b >= batch) return;
  const int C = clampi(ctx_len[b], 0, max_ctx);
  ctx_len[b] = C + span_of(token_indptr, b, total, min(max_tokens, max_pages * D2SD_PAGE_SIZE - C)).len;
}

// Few new rows: one workgroup per request, which then advances ctx_len itself.
// One launch: a token of 8 heads takes 2.5 us in a graph and 6.5 outside of one,
// where the two launches with a workgroup per page take 4.4 and 8.8; 128 rows
// 4.1 and 6.6 against 4.4 and 9.3, 256 rows 5.9 and 6.6 against 4.6 and 9.3, 512
// rows 9.7 both against 4.7 and 9.3.
constexpr int kFewThreads = 1024;
constexpr int kFewRows = 192;

template <typename T>
__global__ __launch_bounds__(kFewThreads) void append_few_kv4_kernel(
    int hkv, int num_pages, int max_pages, int max_ctx, const int* __restrict__ token_indptr, int total, int max_tokens,
    const T* __restrict__ k, const T* __restrict__ v, const int* __restrict__ page_table, int* __restrict__ ctx_len,
    d2sd_kv4_cache cache) {
  const int b = blockIdx.x;
  const int C = clampi(ctx_len[b], 0, max_ctx);
  const Span s = span_of(token_indptr, b, total, min(max_tokens, max_pages * D2SD_PAGE_SIZE - C));
  const int sub = threadIdx.x % kRowLanes;
  for (int r = threadIdx.x / kRowLanes; r < s.len * hkv; r += kFewThreads / kRowLanes) {   // whole rows of lanes
    const size_t src = ((size_t)s.base * hkv + r) * kKv4Dim + sub * 8;
    const size_t row = cache_row(page_table + (size_t)b * max_pages, C + r / hkv, num_pages, hkv, r % hkv);
    float x[8], y[8];
    load8(k + src, x);
    load8(v + src, y);
    write_row8(x, cache.k, cache.k_scale, row, sub);
    write_row8(y, cache.v, cache.v_scale, row, sub);
  }
  __syncthreads();                                  // every thread has read ctx_len[b]
  if (threadIdx.x == 0) ctx_len[b] = C + s.len;
}

// One workgroup per request, as a path is at most 64 tokens: ctx_len[b] can
// then be advanced by the kernel that reads it. A chain of loads (path, page,
// row) bounds it, not bytes: 32 fp32 paths of up to 16 tokens and 8 heads take
// 5.0 us with 64 rows at a time and 7.0 with 16.
constexpr int kCommitThreads = 1024;

template <typename T>
__global__ __launch_bounds__(kCommitThreads) void commit_kv4_kernel(
    int B, int hkv, int num_pages, int max_pages, int max_ctx, const int* __restrict__ node_indptr, int total_nodes,
    const int* __restrict__ path_nodes, const int* __restrict__ accept_len, const T* __restrict__ k_tree,
    const T* __restrict__ v_tree, const int* __restrict__ page_table, int* __restrict__ ctx_len, d2sd_kv4_cache cache) {
  const int b = blockIdx.x;
  const int C = clampi(ctx_len[b], 0, max_ctx);
  const int L = clampi(accept_len[b], 0, B - 1);
  const int base = clampi(node_indptr[b], 0, total_nodes);
  const int sub = threadIdx.x % kRowLanes;
  const long long rows = (long long)(L + 1) * hkv;
  for (long long r = threadIdx.x / kRowLanes; r < rows; r += kCommitThreads / kRowLanes) {
    const int d = (int)(r / hkv), h = (int)(r % hkv);
    const int local = path_nodes[(size_t)b * B + d];
    if (local < 0 || local >= total_nodes - base) continue;   // the same for the lanes of a row
    const size_t src = ((size_t)(base + local) * hkv + h) * kKv4Dim + sub * 8;
    const size_t row = cache_row(page_table + (size_t)b * max_pages, C + d, num_pages, hkv, h);
    float x[8], y[8];
    load8(k_tree + src, x);
    load8(v_tree + src, y);
    write_row8(x, cache.k, cache.k_scale, row, sub);
    write_row8(y, cache.v, cache.v_scale, row, sub);
  }
  __syncthreads();                                  // every thread has read ctx_len[b]
  if (threadIdx.x == 0) ctx_len[b] = C + L + 1;
}

template <typename T>
__global__ __launch_bounds__(kKv4Threads) void read_kv4_kernel(
    int hkv, int pages, int num_pages, int max_pages, const int* __restrict__ token_indptr, int total, int max_tokens,
    const int* __restrict__ start, const int* __restrict__ page_table, d2sd_kv4_cache cache, T* __restrict__ k_out,
    T* __restrict__ v_out) {
  const int b = blockIdx.x / pages;
  const Span s = span_of(token_indptr, b, total, max_tokens);
  const int last = max_pages * D2SD_PAGE_SIZE - 1;          // host: below 2^31
  const int S = start ? clampi(start[b], 0, last) : 0;
  const int pos = (S / D2SD_PAGE_SIZE + blockIdx.x % pages) * D2SD_PAGE_SIZE + threadIdx.x / kRowLanes;
  if (pos < S || pos - S >= s.len) return;
  const int sub = threadIdx.x % kRowLanes;
  const int h0 = blockIdx.y * kHeadsPerGroup;
#pragma unroll
  for (int i = 0; i < kHeadsPerGroup; ++i) {
    const int h = h0 + i;
    if (h >= hkv) break;
    const size_t dst = ((size_t)(s.base + pos - S) * hkv + h) * kKv4Dim + sub * 8;
    const size_t row = cache_row(page_table + (size_t)b * max_pages, min(pos, last), num_pages, hkv, h);
    const uint32_t ck = *reinterpret_cast<const uint32_t*>(cache.k + row * kKv4RowBytes + sub * 4);
    const uint32_t cv = *reinterpret_cast<const uint32_t*>(cache.v + row * kKv4RowBytes + sub * 4);
    const uint32_t sk = cache.k_scale[row * kKv4Blocks + (sub >> 2)];
    const uint32_t sv = cache.v_scale[row * kKv4Blocks + (sub >> 2)];
    store8(k_out + dst, ck, kv4_scale(sk));
    store8(v_out + dst, cv, kv4_scale(sv));
  }
}

// Pages that max_tokens tokens touch from any start.
int touched_pages(int max_tokens) { return ceil_div(max_tokens + D2SD_PAGE_SIZE - 1, D2SD_PAGE_SIZE); }

}  // namespace

long long kv4_page_groups(int batch, int max_tokens) { return (long long)batch * touched_pages(max_tokens); }

hipError_t launch_append_kv4(int batch, int hkv, int dtype, int num_pages, int max_pages, int max_ctx,
                             const int* token_indptr, int total, int max_tokens, const void* k, const void* v,
                             const int* page_table, int* ctx_len, const d2sd_kv4_cache& cache, hipStream_t stream) {
  if ((long long)max_tokens * hkv <= kFewRows) {
    auto launch = [&](auto kernel, auto* kk, auto* vv) {
      hipLaunchKernelGGL(kernel, dim3(batch), dim3(kFewThreads), 0, stream, hkv, num_pages, max_pages, max_ctx, token_indptr,
                         total, max_tokens, kk, vv, page_table, ctx_len, cache);
    };
    if (dtype == D2SD_BF16)
      launch(append_few_kv4_kernel<__bf16>, static_cast<const __bf16*>(k), static_cast<const __bf16*>(v));
    else
      launch(append_few_kv4_kernel<float>, static_cast<const float*>(k), static_cast<const float*>(v));
    return hipGetLastError();
  }
  const int pages = touched_pages(max_tokens);
  const dim3 grid((unsigned)(batch * (long long)pages), ceil_div(hkv, kHeadsPerGroup));
  auto launch = [&](auto kernel, auto* kk, auto* vv) {
    hipLaunchKernelGGL(kernel, grid, dim3(kKv4Threads), 0, stream, hkv, pages, num_pages, max_pages, max_ctx, token_indptr,
                       total, max_tokens, kk, vv, page_table, ctx_len, cache);
  };
  if (dtype == D2SD_BF16)
    launch(append_kv4_kernel<__bf16>, static_cast<const __bf16*>(k), static_cast<const __bf16*>(v));
  else
    launch(append_kv4_kernel<float>, static_cast<const float*>(k), static_cast<const float*>(v));
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(advance_kernel, dim3(ceil_div(batch, kKv4Threads)), dim3(kKv4Threads), 0, stream, batch, max_pages,
                     max_ctx, token_indptr, total, max_tokens, ctx_len);
  return hipGetLastError();
}

hipError_t launch_commit_kv4(int batch, int B, int hkv, int dtype, int num_pages, int max_pages, int max_ctx,
                             const int* node_indptr, int total_nodes, const int* path_nodes, const int* accept_len,
                             const void* k_tree, const void* v_tree, const int* page_table, int* ctx_len,
                             const d2sd_kv4_cache& cache, hipStream_t stream) {
  auto launch = [&](auto kernel, auto* kk, auto* vv) {
    hipLaunchKernelGGL(kernel, dim3(batch), dim3(kCommitThreads), 0, stream, B, hkv, num_pages, max_pages, max_ctx, node_indptr,
                       total_nodes, path_nodes, accept_len, kk, vv, page_table, ctx_len, cache);
  };
  if (dtype == D2SD_BF16)
    launch(commit_kv4_kernel<__bf16>, static_cast<const __bf16*>(k_tree), static_cast<const __bf16*>(v_tree));
  else
    launch(commit_kv4_kernel<float>, static_cast<const float*>(k_tree), static_cast<const float*>(v_tree));
  return hipGetLastError();
}

hipError_t launch_read_kv4(int batch, int hkv, int dtype, int num_pages, int max_pages, const int* token_indptr, int total,
                           int max_tokens, const int* start, const int* page_table, const d2sd_kv4_cache& cache,
                           void* k_out, void* v_out, hipStream_t stream) {
  const int pages = touched_pages(max_tokens);
  const dim3 grid((unsigned)(batch * (long long)pages), ceil_div(hkv, kHeadsPerGroup));
  auto launch = [&](auto kernel, auto* kk, auto* vv) {
    hipLaunchKernelGGL(kernel, grid, dim3(kKv4Threads), 0, stream, hkv, pages, num_pages, max_pages, token_indptr, total,
                       max_tokens, start, page_table, cache, kk, vv);
  };
  if (dtype == D2SD_BF16)
    launch(read_kv4_kernel<__bf16>, static_cast<__bf16*>(k_out), static_cast<__bf16*>(v_out));
  else
    launch(read_kv4_kernel<float>, static_cast<float*>(k_out), static_cast<float*>(v_out));
  return hipGetLastError();
}

}  // namespace d2sd
