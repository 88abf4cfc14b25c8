// Cascade verify attention with the context held in 4 bits (d2sd_kv4_cache).
//
// Work decomposition as for the other element types: the M = N_b G query rows
// of a (request, KV head) are cut into groups of 32 rows per wave, the context
// into splits; the tree keys go with split 0, and partial states are merged by
// log-sum-exp. A wave keeps one query per lane pair: S^T = K Q^T and
// O^T += V^T P^T with 32x32 MFMA tiles, keys (dims) on the row axis, queries
// on the column axis.
//
// What 4 bits change:
//  - Keys go into the matrix cores as they are stored. The block-scaled MFMA
//    takes an E2M1 operand with a power of two per 32 elements of its
//    contraction axis, which is how a key row is stored (blocks of 32 dims),
//    so a lane's operand is 16 bytes of the row and one byte of its scales,
//    with no conversion and a quarter of the LDS or cache traffic of bf16.
//    The queries are the other operand, as a sum of E2M3 terms: with u a power
//    of two, u >= max |x| / 16 over the lane's 32 dims, x / u is rounded to an
//    integer digit in [-16, 16], and the rest times 32 gives the next digit.
//    E2M3 holds these digits exactly (code = digit), and each term costs half
//    a bf16 product of the same shape by count of instructions. n terms leave
//    at most 2^-5n of the block's largest (its next power of two): five for
//    fp32 queries; three for bf16 ones, which are 8 bits long, so only
//    elements below 2^-7 of their block's largest are cut at all.
//  - Values are contracted over keys, along which their scales change, so they
//    are expanded to bf16, which holds them exactly, once per workgroup on
//    their way into LDS; P is rounded to bf16 (bf16) or to the sum of three
//    bf16 numbers, 24 bits (fp32).
//  - The tree's own keys and values arrive in the call's type: they are taken
//    as one (bf16) or three (fp32) bf16 planes through the bf16 MFMA.
// Sums, maxima and outputs are fp32 throughout, partial states as well.
#include <math.h>

#include "attention_device.h"
#include "kv4_device.h"
#include "kv4_plan.h"

namespace d2sd {

namespace {

constexpr int KT = 64;                              // keys per tile
constexpr int kRowBytes = kD * 2;                   // a bf16 row of V in LDS
constexpr int kTileBytes = KT * kRowBytes;
constexpr int kPages = KT / D2SD_PAGE_SIZE;         // pages per tile
constexpr float kGrowLog2 = 8.0f;                   // the running max moves when it grows by more than 2^8

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct Kv4Params {
  Params p;
  d2sd_kv4_cache cache;
};

template <typename T>
struct Terms;
template <>
struct Terms<__bf16> {
  static constexpr int Q = 3;   // E2M3 terms of a query
  static constexpr int P = 1;   // bf16 terms of P, and of tree queries, keys and values
};
template <>
struct Terms<float> {
  static constexpr int Q = 5;
  static constexpr int P = 3;
};

// E2M1 keys (32 x 64 dims) by E2M3 query terms; OA, OB: bytes of the scale words.
template <int OA, int OB>
__device__ __forceinline__ f32x16 mfma_kq(const uint4& k, const uint32_t (&q)[6], const f32x16& c, uint32_t sk, uint32_t sq) {
  const i32x8 a = {(int)k.x, (int)k.y, (int)k.z, (int)k.w, 0, 0, 0, 0};
  const i32x8 b = {(int)q[0], (int)q[1], (int)q[2], (int)q[3], (int)q[4], (int)q[5], 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 2, OA, (int)sk, OB, (int)sq);
}

__device__ __forceinline__ void unpack8(const float* p, float (&v)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p);
  const float4 b = *reinterpret_cast<const float4*>(p + 4);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void unpack8(const __bf16* p, float (&v)[8]) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// v as a sum of bf16 terms, the largest first: each is the rest rounded to bf16.
template <int N>
__device__ __forceinline__ void split_bf16(const float (&v)[8], bf16x8 (&t)[N]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float rest = v[i];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const __bf16 x = (__bf16)rest;
      t[n][i] = x;
      rest -= (float)x;
    }
  }
}

// The wave's queries as E2M3 digits: lane half hf holds dims 64 kk + 32 hf ..
// + 32 of its query for k-step kk, and the scale of step kk in byte kk of s.
template <int N>
struct Query {
  uint32_t d[N][2][6];
  uint32_t s[N];
};

template <typename T, int N>
__device__ __forceinline__ void load_query(Query<N>& q, const T* row, int hf) {
#pragma unroll
  for (int n = 0; n < N; ++n) q.s[n] = 0;
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    float x[32];
    uint32_t top = 0;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (row) unpack8(row + 64 * kk + 32 * hf + 8 * g, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[8 * g + i] = v[i];
        top = max(top, __float_as_uint(x[8 * g + i]) & 0x7fffffffu);
      }
    }
    // top < 2^e; below 2^-100 the digits are those of zero in all but name
    const int e = max((int)(top >> 23) - 126, -100);
    const bool bad = top >= 0x7f800000u;
    const float inv = __uint_as_float((uint32_t)(127 - (e - 4)) << 23);   // 1 / u, u = 2^(e - 4)
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] *= inv;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      uint32_t w[6] = {0, 0, 0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const float d = rintf(x[i]);
        x[i] = (x[i] - d) * 32.0f;
        const uint32_t code = (uint32_t)(int)fabsf(d) | (__float_as_uint(d) >> 31 << 5);
        constexpr int kBits = 6;
        const int at = kBits * i;
        w[at / 32] |= code << (at % 32);
        if (at % 32 > 32 - kBits) w[at / 32 + 1] |= code >> (32 - at % 32);
      }
#pragma unroll
      for (int j = 0; j < 6; ++j) q.d[n][kk][j] = w[j];
      // digit d of term n stands for d u 32^-n, its E2M3 code for d / 8
      const uint32_t s = bad ? 255u : (uint32_t)(e - 4 + 3 - 5 * n + 127);
      q.s[n] |= s << (8 * kk);
    }
  }
}

// LDS place of 16-byte chunk c of row r of a bf16 tile: the transposing reads
// take 32 bytes from each of four consecutive rows, the writes one chunk from
// each of eight, and both then fall on different banks.
__device__ __forceinline__ int chunk_at(int r, int c) {
  return r * kRowBytes + ((c ^ (((r & 3) << 2) | ((r >> 1) & 2))) << 4);
}

// Offsets of the transposing reads of V^T (first keys of the tile): lane i of
// a group of 16 points at V[k0 + i/4][d0 + 4 (i%4)] and gets keys k0 .. k0 + 3
// of dim d0 + i. Rows 8 keys on have the same swizzle.
struct ReadV {
  int at[4];
};
__device__ __forceinline__ ReadV read_v(int lane) {
  ReadV rv;
  const int grp = lane >> 4, i = lane & 15;
  const int row = 4 * (grp >> 1) + (i >> 2);
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) rv.at[dt] = chunk_at(row, dt * 4 + (grp & 1) * 2 + ((i & 3) >> 1)) + ((i & 1) << 3);
  return rv;
}

// O^T += V^T P^T over a tile of 64 keys, P as N bf16 terms.
template <int N>
__device__ __forceinline__ void pv_tile(const char* sV, const ReadV& rv, const bf16x8 (&pf)[N][4], f32x16 (&o)[4]) {
  typedef short s16x8 __attribute__((ext_vector_type(8)));
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) {
      const s16x4 lo = lds_tr16(sV, rv.at[dt] + (ks * 16) * kRowBytes);
      const s16x4 hi = lds_tr16(sV, rv.at[dt] + (ks * 16 + 8) * kRowBytes);
      const s16x8 a8 = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
      for (int n = N - 1; n >= 0; --n) o[dt] = mfma(__builtin_bit_cast(bf16x8, a8), pf[n][ks], o[dt]);
    }
  }
}

// Masks the scores of a tile: slot i of block kb is key 32 kb + (i/4)*8 + hf*4
// + i%4; bit k of vis: key k counts.
__device__ __forceinline__ void mask_scores(f32x16 (&s)[2], uint64_t vis, int hf) {
  const uint64_t m = vis >> (hf * 4);
  const uint32_t w[2] = {(uint32_t)m, (uint32_t)(m >> 32)};
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int bit = (i >> 2) * 8 + (i & 3);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) s[kb][i] = ((w[kb] >> bit) & 1u) ? s[kb][i] : -INFINITY;
  }
}

// One step of the running softmax over a tile of scores (c2: their scale to
// log2 units): moves the reference and rescales when it grows by more than 2^8
// (P is then at most 2^8 and its rounding relative to itself), adds the
// unrounded weights to the row sum, and leaves P as N bf16 terms in operand
// order.
template <int N>
__device__ __forceinline__ void softmax_tile(f32x16 (&s)[2], float& m_run, float& l_run, f32x16 (&o)[4], bf16x8 (&pf)[N][4],
                                             float c2) {
  float mx = -INFINITY;
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kb][i]);
  mx = xhalf_max(mx);
  const float m_new = fmaxf(m_run, mx);
  const bool grow = (m_new - m_run) * c2 > kGrowLog2;      // false when both are -inf
  if (__ballot(grow)) {
    const float alpha = m_run == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m_run - m_new) * c2);
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) o[dt] *= alpha;
    l_run *= alpha;
    m_run = m_new;
  }
  const float moff = m_run == -INFINITY ? 0.0f : m_run * c2;
  float l[2] = {0.0f, 0.0f};
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] = __builtin_amdgcn_exp2f(fmaf(s[kb][8 * t + j], c2, -moff));
        l[j & 1] += v[j];
      }
      bf16x8 x[N];
      split_bf16<N>(v, x);
#pragma unroll
      for (int n = 0; n < N; ++n) pf[n][2 * kb + t] = x[n];
    }
  l_run += l[0] + l[1];
}

// All waves' LDS writes are done and seen; loads in flight stay so.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// NW waves of 32 query rows share the tiles of V.
template <typename T, int NW>
__global__ __launch_bounds__(NW* kWave) void kv4_attention_kernel(Kv4Params kp) {
  constexpr int NQ = Terms<T>::Q, NP = Terms<T>::P;
  constexpr int kThr = NW * kWave;
  constexpr int kUnits = KT * kKv4Blocks * 2 / kThr;   // 8-byte pieces (16 codes) of a V tile per thread
  static_assert(kUnits >= 1, "a V tile has 512 pieces");
  const Params& p = kp.p;
  __shared__ __attribute__((aligned(1024))) char sv[2][kTileBytes];
  __shared__ int s_pid[kKv4MaxSplit / D2SD_PAGE_SIZE];
  __shared__ int s_flag;

  // consecutive items on one XCD: the row groups of a split share its L2
  const int per_xcd = gridDim.x / 8;
  const int item = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
  if (item >= p.items) return;
  int rest = item;
  const int rg = rest % p.n_rg_max; rest /= p.n_rg_max;
  const int ch = rest % p.n_ch_max; rest /= p.n_ch_max;
  const int h = rest % p.hkv;
  const int b = rest / p.hkv;
  const int node_base = clampi(p.node_indptr[b], 0, p.total_nodes);
  const int Nb = clampi(p.node_indptr[b + 1], node_base, min(p.total_nodes, node_base + p.max_nodes)) - node_base;
  const int Mb = Nb * p.G;
  const int r_lo = rg * (NW * kRowsPerTile);
  if (r_lo >= Mb) return;
  const int r_hi = min(Mb, r_lo + NW * kRowsPerTile);
  const int Cb = p.stage != D2SD_STAGE_TREE ? clampi(p.ctx_len[b], 0, p.max_ctx) : 0;
  const int n_ch_b = max(1, ceil_div(Cb, p.split));
  if (ch >= n_ch_b) return;
  const int c0 = ch * p.split;
  const int c1 = min(Cb, c0 + p.split);
  const int n_tiles = ceil_div(c1 - c0, KT);

  const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5;
  const int r = r_lo + (tid >> 6) * kRowsPerTile + (lane & 31);
  const bool active = r - (lane & 31) < r_hi;       // the wave holds a row
  const bool valid = r < r_hi;
  const int node = valid ? r / p.G : 0;
  const int qrow = valid ? (node_base + node) * p.hq + h * p.G + r % p.G : -1;
  const T* q_ptr = valid ? static_cast<const T*>(p.q) + (size_t)qrow * kD : nullptr;

  for (int i = tid; i < ceil_div(c1 - c0, D2SD_PAGE_SIZE); i += kThr)
    s_pid[i] = clampi(p.page_table[(size_t)b * p.max_pages + (c0 >> 4) + i], 0, p.num_pages - 1) * p.hkv + h;

  f32x16 o[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) o[dt] = f32x16{};
  float m_run = -INFINITY, l_run = 0.0f;
  const ReadV rv = read_v(lane);

  // ---- the tree's keys ----
  if (ch == 0 && p.stage != D2SD_STAGE_PREFIX) {
    const T* kt = static_cast<const T*>(p.k_tree);
    const T* vt = static_cast<const T*>(p.v_tree);
    for (int key0 = 0; key0 < Nb; key0 += KT) {
      const int nvalid = min(KT, Nb - key0);
      const size_t row0 = (size_t)(node_base + key0) * p.hkv + h;
      f32x16 s[2];
      uint64_t vis = 0;
      bf16x8 pf[NP][4];
      if (active) {
        s[0] = f32x16{};
        s[1] = f32x16{};
#pragma unroll
        for (int st = 0; st < 8; ++st) {              // dims 64 hf + 8 st .. + 8
          float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
          if (q_ptr) unpack8(q_ptr + 64 * hf + 8 * st, v);
          bf16x8 tq[NP];
          split_bf16<NP>(v, tq);
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) {
            const int key = min(32 * kb + (lane & 31), nvalid - 1);
            unpack8(kt + (row0 + (size_t)key * p.hkv) * kD + 64 * hf + 8 * st, v);
            bf16x8 tk[NP];
            split_bf16<NP>(v, tk);
#pragma unroll
            for (int i = NP - 1; i >= 0; --i)         // products below the last term are left out
#pragma unroll
              for (int j = NP - 1 - i; j >= 0; --j) s[kb] = mfma(tk[i], tq[j], s[kb]);
          }
        }
        const uint32_t* mrow = p.anc_mask + (size_t)(node_base + node) * p.mask_words;
        const int w0 = key0 >> 5;
        vis = (uint64_t)mrow[w0] | (w0 + 1 < p.mask_words ? (uint64_t)mrow[w0 + 1] << 32 : 0ull);
        if (!valid) vis = 0;
        if (nvalid < KT) vis &= (1ull << nvalid) - 1ull;
        mask_scores(s, vis, hf);
        softmax_tile<NP>(s, m_run, l_run, o, pf, p.c2);
      }
      if (tid == 0) s_flag = 0;
      lds_barrier();
#pragma unroll
      for (int n = 0; n < NP; ++n) {                  // planes of V
        for (int i = tid; i < KT * (kD / 8); i += kThr) {
          const int row = i / (kD / 8), c = i % (kD / 8);
          float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
          if (row < nvalid) unpack8(vt + (row0 + (size_t)row * p.hkv) * kD + 8 * c, v);
          bool wild = false;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if ((__float_as_uint(v[j]) & 0x7f800000u) == 0x7f800000u) {
              wild = true;
              v[j] = 0.0f;
            }
          if (wild) s_flag = 1;
          bf16x8 t[NP];
          split_bf16<NP>(v, t);
          *reinterpret_cast<bf16x8*>(sv[0] + chunk_at(row, c)) = t[n];
        }
        lds_barrier();
        if (active) {
          // plane n by the terms of P that are not below the last one
          typedef bf16x8 Terms1[1][4];
#pragma unroll
          for (int j = NP - 1 - n; j >= 0; --j) pv_tile<1>(sv[0], rv, reinterpret_cast<const Terms1&>(pf[j]), o);
        }
        if (n == NP - 1 && s_flag && active) {
          // an infinite or NaN value: added where its node is seen (a weight of 0 would spread it to all)
          for (int k = 0; k < nvalid; ++k) {
            if (!((vis >> k) & 1ull)) continue;
            const T* vr = vt + (row0 + (size_t)k * p.hkv) * kD;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const float x = (float)vr[dt * 32 + (i >> 2) * 8 + hf * 4 + (i & 3)];
                if ((__float_as_uint(x) & 0x7f800000u) == 0x7f800000u) o[dt][i] += x;
              }
          }
        }
        lds_barrier();
      }
    }
  }

  // ---- the context ----
  if (n_tiles > 0) {
    Query<NQ> q;
    if (active) load_query<T, NQ>(q, q_ptr, hf);
    lds_barrier();                                    // page ids
    const int pages_here = ceil_div(c1 - c0, D2SD_PAGE_SIZE);

    // this thread's pieces of a V tile: 8 bytes, 16 codes of half a block
    uint2 vraw[kUnits];
    int vscale[kUnits];
    auto load_v = [&](int j) {
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        const int unit = u * kThr + tid;              // lane = key in the page and block, then block half, page
        const int pg = min(j * kPages + (unit >> 7), pages_here - 1);
        const size_t row = (size_t)(uint32_t)s_pid[pg] * D2SD_PAGE_SIZE + (unit & 15);
        const int blk = (unit >> 4) & 3;
        vraw[u] = *reinterpret_cast<const uint2*>(kp.cache.v + row * kKv4RowBytes + blk * 16 + ((unit >> 6) & 1) * 8);
        vscale[u] = kp.cache.v_scale[row * kKv4Blocks + blk];
      }
    };
    auto store_v = [&](int j, char* dst) {
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        const int unit = u * kThr + tid;
        const int row = (unit >> 7) * D2SD_PAGE_SIZE + (unit & 15);
        const int c = ((unit >> 4) & 3) * 4 + ((unit >> 6) & 1) * 2;
        const bool in = c0 + j * KT + row < c1;       // rows past the context are zeros
        const float sc = kv4_scale(vscale[u]);
        const uint4 z = make_uint4(0u, 0u, 0u, 0u);
        *reinterpret_cast<uint4*>(dst + chunk_at(row, c)) = in ? kv4_decode8_bf16(vraw[u].x, sc) : z;
        *reinterpret_cast<uint4*>(dst + chunk_at(row, c + 1)) = in ? kv4_decode8_bf16(vraw[u].y, sc) : z;
      }
    };
    uint4 kraw[2][2];
    uint32_t kscale[2];
    auto load_k = [&](int j) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const int pg = min(j * kPages + 2 * kb + ((lane & 31) >> 4), pages_here - 1);
        const size_t row = (size_t)(uint32_t)s_pid[pg] * D2SD_PAGE_SIZE + (lane & 15);
        const uint8_t* src = kp.cache.k + row * kKv4RowBytes + hf * 16;
        kraw[kb][0] = *reinterpret_cast<const uint4*>(src);
        kraw[kb][1] = *reinterpret_cast<const uint4*>(src + 32);
        kscale[kb] = *reinterpret_cast<const uint32_t*>(kp.cache.k_scale + row * kKv4Blocks) >> (8 * hf);
      }
    };

    load_v(0);
    if (active) load_k(0);
    store_v(0, sv[0]);
    lds_barrier();
    for (int j = 0; j < n_tiles; ++j) {
      const bool more = j + 1 < n_tiles;
      if (more) load_v(j + 1);
      if (active) {
        f32x16 s[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          s[kb] = f32x16{};
#pragma unroll
          for (int n = NQ - 1; n >= 0; --n) {          // the small terms first
            s[kb] = mfma_kq<0, 0>(kraw[kb][0], q.d[n][0], s[kb], kscale[kb], q.s[n]);
            s[kb] = mfma_kq<2, 1>(kraw[kb][1], q.d[n][1], s[kb], kscale[kb], q.s[n]);
          }
        }
        if (more) load_k(j + 1);
        const int nvalid = c1 - (c0 + j * KT);
        if (nvalid < KT) mask_scores(s, (1ull << nvalid) - 1ull, hf);
        bf16x8 pf[NP][4];
        softmax_tile<NP>(s, m_run, l_run, o, pf, p.c2);
        pv_tile<NP>(sv[j & 1], rv, pf, o);
      }
      if (more) store_v(j + 1, sv[(j + 1) & 1]);
      lds_barrier();
    }
  }

  // ---- the row's state ----
  if (!active) return;
  const float l_all = l_run + __shfl_xor(l_run, 32);
  if (!valid) return;
  if (n_ch_b == 1) {
    const float inv = l_all == 0.0f ? 0.0f : 1.0f / l_all;
    T* dst = static_cast<T*>(p.out) + (size_t)qrow * kD;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = o[dt][q4 * 4 + i] * inv;
        store_out<T>(dst + dt * 32 + q4 * 8 + hf * 4, v);
      }
    if (p.lse && hf == 0) p.lse[qrow] = l_all == 0.0f ? -INFINITY : (m_run * p.c2 + __log2f(l_all)) * kLn2;
  } else {
    const size_t at = (size_t)ch * ((size_t)p.total_nodes * p.hq) + qrow;
    float* dst = static_cast<float*>(p.ws_o) + at * kD;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<float4*>(dst + dt * 32 + q4 * 8 + hf * 4) =
            make_float4(o[dt][q4 * 4], o[dt][q4 * 4 + 1], o[dt][q4 * 4 + 2], o[dt][q4 * 4 + 3]);
    if (hf == 0) {
      p.ws_m[at] = m_run * p.c2;
      p.ws_l[at] = l_all;
    }
  }
}

// Joins the splits of a row: 32 lanes per row, four dims each, two rows per
// wave; the splits are taken in order, four loads at a time.
constexpr int kMergeRows = kThreads / 32;

template <typename T>
__global__ __launch_bounds__(kThreads) void kv4_merge_kernel(Params p, int chunks) {
  const int b = blockIdx.x / chunks;
  const int node_base = clampi(p.node_indptr[b], 0, p.total_nodes);
  const int Nb = clampi(p.node_indptr[b + 1], node_base, min(p.total_nodes, node_base + p.max_nodes)) - node_base;
  const int rr = (blockIdx.x % chunks) * kMergeRows + threadIdx.x / 32;
  const int n = ceil_div(clampi(p.ctx_len[b], 0, p.max_ctx), p.split);
  if (n <= 1 || rr >= Nb * p.hq) return;              // one split: the row is finished
  const int d0 = (threadIdx.x & 31) * 4;
  const size_t row = (size_t)node_base * p.hq + rr, stride = (size_t)p.total_nodes * p.hq;
  float M = -INFINITY;
  for (int s = threadIdx.x & 31; s < n; s += 32) M = fmaxf(M, p.ws_m[s * stride + row]);
#pragma unroll
  for (int k = 16; k; k >>= 1) M = fmaxf(M, __shfl_xor(M, k));
  if (M == -INFINITY) M = 0.0f;
  float L = 0.0f, acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < n; ++s) {
    const size_t at = s * stride + row;
    const float w = __builtin_amdgcn_exp2f(p.ws_m[at] - M);
    const float4 v = *reinterpret_cast<const float4*>(static_cast<const float*>(p.ws_o) + at * kD + d0);
    L += w * p.ws_l[at];
    acc[0] += w * v.x;
    acc[1] += w * v.y;
    acc[2] += w * v.z;
    acc[3] += w * v.w;
  }
  const float inv = L == 0.0f ? 0.0f : 1.0f / L;
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i] *= inv;
  store_out<T>(static_cast<T*>(p.out) + row * kD + d0, acc);
  if (p.lse && d0 == 0) p.lse[row] = L == 0.0f ? -INFINITY : (M + __log2f(L)) * kLn2;
}

}  // namespace

hipError_t launch_kv4_attention(const d2sd_attn_args& a, const d2sd_kv4_cache& cache, const Kv4Plan& plan, void* ws,
                                hipStream_t stream) {
  Params p{};
  p.q = a.q; p.page_table = a.page_table; p.ctx_len = a.ctx_len; p.k_tree = a.k_tree; p.v_tree = a.v_tree;
  p.node_indptr = a.node_indptr; p.anc_mask = a.anc_mask; p.out = a.out; p.lse = a.lse;
  const size_t states = (size_t)plan.n_ch_max * a.total_nodes * a.num_qo_heads;
  p.ws_o = ws;
  p.ws_m = ws ? static_cast<float*>(ws) + states * kD : nullptr;
  p.ws_l = ws ? p.ws_m + states : nullptr;
  p.batch = a.batch; p.hq = a.num_qo_heads; p.hkv = a.num_kv_heads; p.G = a.num_qo_heads / a.num_kv_heads;
  p.stage = a.stage; p.total_nodes = a.total_nodes; p.max_nodes = a.max_nodes; p.max_ctx = a.max_ctx_len;
  p.num_pages = a.num_pages; p.max_pages = a.max_pages; p.mask_words = a.mask_words;
  p.split = plan.split; p.n_ch_max = plan.n_ch_max; p.n_rg_max = plan.n_rg_max; p.items = (int)plan.items;
  p.c2 = plan.scale * kLog2e;
  const Kv4Params kp{p, cache};
  const dim3 grid((unsigned)((plan.items + 7) / 8 * 8));
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(plan.waves * kWave), 0, stream, kp); };
  const bool bf16 = a.dtype == D2SD_BF16;
  if (plan.waves == 1)
    bf16 ? launch(kv4_attention_kernel<__bf16, 1>) : launch(kv4_attention_kernel<float, 1>);
  else if (plan.waves == 2)
    bf16 ? launch(kv4_attention_kernel<__bf16, 2>) : launch(kv4_attention_kernel<float, 2>);
  else if (plan.waves == 4)
    bf16 ? launch(kv4_attention_kernel<__bf16, 4>) : launch(kv4_attention_kernel<float, 4>);
  else
    bf16 ? launch(kv4_attention_kernel<__bf16, 8>) : launch(kv4_attention_kernel<float, 8>);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && plan.n_ch_max > 1) {
    const int chunks = ceil_div(a.max_nodes * a.num_qo_heads, kMergeRows);
    const dim3 mgrid((unsigned)(a.batch * chunks));
    if (bf16)
      hipLaunchKernelGGL(kv4_merge_kernel<__bf16>, mgrid, dim3(kThreads), 0, stream, p, chunks);
    else
      hipLaunchKernelGGL(kv4_merge_kernel<float>, mgrid, dim3(kThreads), 0, stream, p, chunks);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace d2sd
