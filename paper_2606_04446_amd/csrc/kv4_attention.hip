// Cascade verify attention with the context held in 4 bits (d2sd_kv4_cache).
//
// S^T = K Q^T and O^T += V^T P^T with 32x32 MFMA tiles: keys (dims) on the row
// axis, queries on the column axis, so a wave keeps one query per lane pair and
// the weights leave the first product in the order in which the second takes
// them. What 4 bits change:
//  - Keys go into the matrix cores as they are stored. The block-scaled MFMA
//    takes an E2M1 operand with a power of two per 32 elements of its
//    contraction axis, which is how a key row is stored (blocks of 32 dims),
//    so a lane's operand is 16 bytes of the row and one byte of its scales,
//    with no conversion and a quarter of the LDS traffic of bf16. The queries
//    are the other operand, as a sum of E2M3 terms: with u a power of two,
//    u >= max |x| / 16 over the lane's 32 dims, x / u is rounded to an integer
//    digit in [-16, 16], and the rest times 32 gives the next digit. E2M3 holds
//    these digits exactly (code = digit), and each term costs half a bf16
//    product of the same shape by time in the matrix cores. n terms leave at
//    most 2^-5n of the block's largest (its next power of two). bf16 queries are
//    held in four: they are 8 bits long, so nothing is lost of elements down to
//    2^-12 of that power of two, and 2^-20 of it of smaller ones. Three would cut
//    at 2^-15, which an lse shows wherever the mean key is not 0 (normal queries
//    with one dim of 32 that is 32 times the others: 3e-5 of it, however long
//    the context is), and take 554 us where four take 590: 32 requests of eight
//    row tiles over 16384 keys. With the softmax scale multiplied in, all
//    elements would be cut at 2^-20, so the scores are scaled instead. (Two E4M3
//    terms would hold a bf16 query, in 58 ns of matrix instructions per 32 keys
//    against 64, but an instruction adds its 8-bit products with 13 bits below
//    the largest.) fp32 queries take the scale and are held in five terms, 25
//    bits; their scores' accumulator starts at -m, so that they leave the
//    product ready for exp2.
//  - Values are contracted over keys, along which their scales change, so they
//    are expanded to bf16, which holds them exactly. The expansion is a product
//    with the identity in the block-scaled MFMA: its output has a lane's dim
//    and the keys in the order of the weights, so V^T needs no LDS. P is rounded
//    to bf16 (bf16) or to the sum of three bf16 numbers, 24 bits (fp32).
//  - The tree's own keys and values arrive in the call's type: they are taken
//    as one (bf16) or three (fp32) bf16 planes through the bf16 MFMA.
// Sums, maxima and outputs are fp32 throughout, partial states as well.
//
// What bounds it. Few rows: the cache's bytes; 64 requests of one token over 500
// to 16000 keys (576 MB) take 130 us, 4.4 TB/s, where a plain sum over memory
// reaches 4.0 and a copy 4.7. Many rows: 32 requests of eight row tiles over
// 16384 keys take 590 us, 934 TFLOP/s of the products asked for; 20 matrix
// instructions per 32 keys and row tile, 15 ns each at the clock that they leave,
// are 300 of it, and the 16 exponentials and 74 other vector operations beside
// them overlap only in part (one wave per SIMD takes 670 us with three query
// terms, two 538). Tried and slower: V expanded once per workgroup and read back
// transposed from LDS (545 against 571 of that version, but 246 against 233 with
// one row tile), the next scores' products ahead of a tile's exponentials (549,
// spilled), 64-key steps (same), three or four shares per CU (589, 598), eight
// waves and row tiles on one ring (546 against 548).
#include <math.h>

#include <type_traits>

#include "attention_device.h"
#include "kv4_device.h"
#include "kv4_plan.h"

namespace d2sd {

namespace {

constexpr int kThr = 4 * kWave;
constexpr int kRowBytes = kD * 2;                   // a bf16 row of V in LDS

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x6 __attribute__((ext_vector_type(6)));

// bf16 terms of P, and of tree queries, keys and values.
template <typename T>
constexpr int kTerms = sizeof(T) == 4 ? 3 : 1;

// E2M3 terms of a query.
template <typename T>
constexpr int kQueryTerms = sizeof(T) == 4 ? 5 : 4;

// E2M1 keys (32 x 64 dims) by E2M3 query terms; OA, OB: bytes of the scale words.
template <int OA, int OB>
__device__ __forceinline__ f32x16 mfma_kq(const uint4& k, const uint32_t (&q)[6], const f32x16& c, uint32_t sk, uint32_t sq) {
  const i32x8 a = {(int)k.x, (int)k.y, (int)k.z, (int)k.w, 0, 0, 0, 0};
  const i32x8 b = {(int)q[0], (int)q[1], (int)q[2], (int)q[3], (int)q[4], (int)q[5], 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 2, OA, (int)sk, OB, (int)sq);
}

// The transpose of E2M1 values as a product with one half of the identity: keys
// (32 x 64 dims, a lane holds 32 dims of a key) to fp32, key on the row axis,
// dim on the column axis.
template <int OA>
__device__ __forceinline__ f32x16 mfma_vt(const uint4& v, const uint4& half, uint32_t sv) {
  const i32x8 a = {(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0};
  const i32x8 b = {(int)half.x, (int)half.y, (int)half.z, (int)half.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, f32x16{}, 4, 4, OA, (int)sv, 0, 127);
}

// Eight elements as loaded.
template <typename T>
struct Raw8 {
  uint4 x[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* p) {
  Raw8<T> r;
#pragma unroll
  for (unsigned i = 0; i < sizeof(T) / 2; ++i) r.x[i] = reinterpret_cast<const uint4*>(p)[i];
  return r;
}
__device__ __forceinline__ void unpack8(const Raw8<float>& r, float (&v)[8]) {
  const uint32_t w[8] = {r.x[0].x, r.x[0].y, r.x[0].z, r.x[0].w, r.x[1].x, r.x[1].y, r.x[1].z, r.x[1].w};
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
}
__device__ __forceinline__ void unpack8(const Raw8<__bf16>& r, float (&v)[8]) {
  const uint32_t w[4] = {r.x[0].x, r.x[0].y, r.x[0].z, r.x[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// v as a sum of bf16 terms, the largest first: each is the rest rounded to bf16.
// WIDE: v may be any finite number. Rounding would make one above the largest
// bf16 infinite, so the first term stops there and the others hold what is left.
template <int N, bool WIDE = false>
__device__ __forceinline__ void split_bf16(const float (&v)[8], bf16x8 (&t)[N]) {
  const float most = __uint_as_float(0x7f7f0000u);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float rest = v[i];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const __bf16 x = (__bf16)(WIDE && N > 1 && n == 0 ? __builtin_amdgcn_fmed3f(rest, -most, most) : rest);
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
__device__ __forceinline__ void load_query(Query<N>& q, const T* row, int hf, float c2) {
#pragma unroll
  for (int n = 0; n < N; ++n) q.s[n] = 0;
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    asm volatile("" ::: "memory");                      // one half's registers at a time
    float x[32];
    uint32_t top = 0;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (row) unpack8(load8(row + 64 * kk + 32 * hf + 8 * g), v);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[8 * g + i] = v[i] * c2;
        top = max(top, __float_as_uint(x[8 * g + i]) & 0x7fffffffu);
      }
    }
    // top < 2^e; below 2^-100 the digits are those of zero in all but name
    const int e = max((int)(top >> 23) - 126, -100);
    const bool bad = top >= 0x7f800000u;
    const float inv = __uint_as_float((uint32_t)(127 - (e - 4)) << 23);   // 1 / u, u = 2^(e - 4)
    // the conversion takes its elements from two registers' worth in turn
    f32x16 even, odd;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      even[i] = x[2 * i] * inv;
      odd[i] = x[2 * i + 1] * inv;
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      // the nearest multiple of 32^-n, by the addition and in the conversion alike; a code is eighths
      const float unit = __uint_as_float((uint32_t)(127 - 5 * n) << 23), magic = 12582912.0f * unit;
      const i32x6 w = __builtin_bit_cast(i32x6, __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, 8.0f * unit));
#pragma unroll
      for (int j = 0; j < 6; ++j) {
        q.d[n][kk][j] = (uint32_t)w[j];
        asm volatile("" : "+v"(q.d[n][kk][j]));
      }
      if (n + 1 < N) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          even[i] -= (even[i] + magic) - magic;
          odd[i] -= (odd[i] + magic) - magic;
        }
      }
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

// V^T operand of dims 32 dt .. + 32 for step ks of 16 keys.
__device__ __forceinline__ bf16x8 read_va(const char* sV, const ReadV& rv, int ks, int dt) {
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  const s16x4 lo = lds_tr16(sV, rv.at[dt] + (ks * 16) * kRowBytes);
  const s16x4 hi = lds_tr16(sV, rv.at[dt] + (ks * 16 + 8) * kRowBytes);
  const s16x8 a8 = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(bf16x8, a8);
}

// O^T += V^T P^T over KS steps of 16 keys, P as N bf16 terms.
template <int N, int KS>
__device__ __forceinline__ void pv_tile(const char* sV, const ReadV& rv, const bf16x8 (&pf)[N][KS], f32x16 (&o)[4]) {
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) {
      const bf16x8 a = read_va(sV, rv, ks, dt);
#pragma unroll
      for (int n = N - 1; n >= 0; --n) o[dt] = mfma(a, pf[n][ks], o[dt]);
    }
  }
}

// Masks the scores of a tile: slot i of block kb is key 32 kb + (i/4)*8 + hf*4
// + i%4; bit k of vis: key k counts.
template <int KB>
__device__ __forceinline__ void mask_scores(f32x16 (&s)[KB], uint64_t vis, int hf) {
  const uint64_t m = vis >> (hf * 4);
  const uint32_t w[2] = {(uint32_t)m, (uint32_t)(m >> 32)};
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int bit = (i >> 2) * 8 + (i & 3);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) s[kb][i] = ((w[kb] >> bit) & 1u) ? s[kb][i] : -INFINITY;
  }
}

// The running softmax. A row's reference m (log2 units) is the largest score of
// its first keys; it moves, with a rescaling of what is summed up, only when the
// weights 2^(s - m) of a block of 16 pass kMostWeight in sum. Until then no
// maximum is needed: P may be well over 1, its rounding is relative to itself.
constexpr float kMostWeight = 8192.0f;

template <int KB>
__device__ __forceinline__ float max_score(const f32x16 (&s)[KB]) {
  float mx = -INFINITY;
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kb][i]);
  return xhalf_max(mx);
}
// Moves the reference up to mx, the row's largest new score.
__device__ __forceinline__ void move_reference(float mx, float& m_run, float& l_run, f32x16 (&o)[4]) {
  const float m_new = fmaxf(m_run, mx);
  const float alpha = m_run == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run - m_new);
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) o[dt] *= alpha;
  l_run *= alpha;
  m_run = m_new;
}
// Scores times c2 and less the reference.
__device__ __forceinline__ f32x16 ahead(const f32x16& x, float c2, float minus_m) {
  f32x16 s;
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = fmaf(x[i], c2, minus_m);
  return s;
}
// Scores less the reference to weights, in place; returns their sum.
__device__ __forceinline__ float weigh(f32x16& s) {
  float l[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    s[i] = __builtin_amdgcn_exp2f(s[i]);
    l[i & 1] += s[i];
  }
  return l[0] + l[1];
}
// The weights of a block as N bf16 terms in operand order.
template <int N>
__device__ __forceinline__ void split_weights(const f32x16& w, bf16x8 (&pf)[N][2]) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const float v[8] = {w[8 * t], w[8 * t + 1], w[8 * t + 2], w[8 * t + 3], w[8 * t + 4], w[8 * t + 5], w[8 * t + 6], w[8 * t + 7]};
    bf16x8 x[N];
    split_bf16<N>(v, x);
#pragma unroll
    for (int n = 0; n < N; ++n) pf[n][t] = x[n];
  }
}

// All waves' LDS writes are done and seen; loads in flight stay so.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// ---- division of the work ----
//
// The row tiles of a (request, KV head), 32 rows each, are taken four at a time
// and what is left as two and one: the four waves of a workgroup hold a row tile
// each, or share the keys of two or of one, so that none is idle. A stream is
// such a group of R tiles with all keys that they see. It has one step per tile
// of kKeys context keys and, before them, charge_of(R) steps for its start, its
// end and the tree, and one per 64 nodes beyond the first. A step of R tiles
// costs kv4_cost(R). All
// streams form one line, request by request and head by head, and workgroup i
// of G takes the steps that begin in [i W / G, (i + 1) W / G) of its W units of
// cost, so every workgroup has the same share whatever the lengths are, and at
// most two of its pieces are parts of a stream. These leave their state in a
// slot, and the merge joins the slots of every stream that was cut.
struct CutStream {
  int4 rows;           // first node of its request, KV head, first row of the group, rows
  int pieces;          // 0: none
  int unused[3];
};
static_assert(sizeof(CutStream) == kKv4CutBytes);

struct Kv4Params {
  Params p;
  d2sd_kv4_cache cache;
  int grid;            // G
  int whole;           // streams are not cut: each is one unit
  int most;            // cost of the largest group's step
  int charge[3];       // steps that a stream of 1, 2 or 4 tiles counts beside those of its keys
  int span, per;       // of the merge
  CutStream* cut;      // [G]: the stream whose second piece a workgroup holds
};

constexpr int kKeys = 128;   // context keys per step

struct RequestPlan {
  int base, nodes, tiles, ctx;   // first node, nodes, row tiles, context keys
  int pre, steps;                // of a stream: steps of the tree past its first 64 nodes; these and the steps of the context
  int head;                      // cost of a KV head
};

// Steps that a stream's start, its end and the first 64 nodes stand for.
__device__ __forceinline__ int charge_of(const Kv4Params& kp, int R) { return kp.whole ? 0 : R == 4 ? kp.charge[2] : R == 2 ? kp.charge[1] : kp.charge[0]; }

__device__ __forceinline__ int groups_of(int tiles) { return (tiles >> 2) + (tiles >> 1 & 1) + (tiles & 1); }

// What a plan is made of: first node, nodes, context keys.
struct Lengths {
  int base, nodes, ctx;
};
__device__ __forceinline__ Lengths lengths_of(const Kv4Params& kp, int b) {
  const Params& p = kp.p;
  Lengths n;
  n.base = clampi(p.node_indptr[b], 0, p.total_nodes);
  n.nodes = clampi(p.node_indptr[b + 1], n.base, min(p.total_nodes, n.base + p.max_nodes)) - n.base;
  n.ctx = p.stage != D2SD_STAGE_TREE ? clampi(p.ctx_len[b], 0, p.max_ctx) : 0;
  return n;
}
__device__ __forceinline__ RequestPlan plan_of(const Kv4Params& kp, const Lengths& n) {
  const Params& p = kp.p;
  RequestPlan q;
  q.base = n.base;
  q.nodes = n.nodes;
  q.ctx = n.ctx;
  q.tiles = ceil_div(q.nodes * p.G, kRowsPerTile);
  if (kp.whole) {
    q.pre = 0;
    q.steps = 1;
    q.head = groups_of(q.tiles);
  } else {
    q.pre = p.stage != D2SD_STAGE_PREFIX ? ceil_div(max(0, q.nodes - 64), 64) : 0;
    q.steps = q.pre + ceil_div(q.ctx, kKeys);
    q.head = (q.tiles >> 2) * kv4_cost(4) * (q.steps + kp.charge[2]);
    if (q.tiles & 2) q.head += kv4_cost(2) * (q.steps + kp.charge[1]);
    if (q.tiles & 1) q.head += kv4_cost(1) * (q.steps + kp.charge[0]);
  }
  return q;
}

// Group g of a head's row tiles: its first tile and its number of them.
struct Group {
  int first, R;
};
__device__ __forceinline__ Group group_of(int tiles, int g) {
  const int fours = tiles >> 2;
  if (g < fours) return {4 * g, 4};
  if (g == fours && (tiles & 2)) return {4 * fours, 2};
  return {tiles & ~1, 1};
}

// Values and arguments as if they were new: what a section derives from them
// is computed (loaded) there and holds no registers in the others.
__device__ __forceinline__ int afresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
typedef const __attribute__((address_space(4))) Kv4Params* ArgPtr;
__device__ __forceinline__ ArgPtr args_afresh() {
  ArgPtr a = (ArgPtr)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(a));
  return a;
}

// The shares of a line of W units for `grid` workgroups, each at least one unit:
// that of i starts at i W / grid, which takes one division in 64 bits for all.
struct Shares {
  long long each;
  int rest, grid;
  __device__ __forceinline__ Shares(long long W, int g) : grid(g) {
    each = (unsigned long long)W >> 32 ? W / g : (long long)((uint32_t)W / (uint32_t)g);
    rest = (int)(W - each * g);
  }
  __device__ __forceinline__ long long start(int i) const { return each * i + (uint32_t)rest * (uint32_t)i / (uint32_t)grid; }   // grid < 2^16
  // of unit x, which is in the share of `from` or a later one's
  __device__ __forceinline__ int holder(long long x, int from) const {
    int i = from + (int)((uint32_t)(x - start(from)) / ((uint32_t)min(each, 1ll << 30) + 1u));   // a stream's length: < 2^25
    while (start(i + 1) <= x) ++i;
    return i;
  }
};

// ---- tiles of the context ----
//
// Codes and scales travel global -> LDS by DMA into a ring of kStages tiles, so
// that a tile has some iterations to arrive and holds no registers.
constexpr int kStages = 4;
struct Tile {
  static constexpr int PAGES = kKeys / D2SD_PAGE_SIZE;    // 8: wave w copies pages w and w + 4
  static constexpr int OPS = 5;                           // its copies: K and V of two pages, and their scales together
  static constexpr int V = PAGES * kKv4PageBytes, S = 2 * V;   // offsets in a stage; K at 0
  static constexpr int BYTES = S + PAGES * 128;           // scales: 64 bytes of K and 64 of V per page, in the order of the copies
};
static_assert(Tile::PAGES == 8, "two pages per wave");

// Rows of 64 bytes in a stage: 16-byte chunk c of row r sits at c ^ (r/4 % 4),
// so that reads of one chunk from eight (16) consecutive rows are free of bank
// conflicts. The DMA writes in lane order, so its lanes fetch accordingly.
__device__ __forceinline__ int code_at(int r, int c) { return r * kKv4RowBytes + ((c ^ ((r >> 2) & 3)) << 4); }
// Scales of K of key r; those of V are 64 bytes on.
__device__ __forceinline__ int scale_at(int r) {
  const int page = r >> 4;
  return Tile::S + (page & 3) * 256 + (page >> 2) * 128 + (r & 15) * kKv4Blocks;
}

// A wave's copies: pages w and w + 4 of every tile of a piece.
struct Copies {
  const char *k, *v;
  const uint8_t* scales;       // K's in the lanes with bit 4 clear, V's in the others
  const int* table;
  uint32_t from;
  int wave, first_page, last_page, num_pages, hkv, h;
  __device__ __forceinline__ Copies(ArgPtr a, int b, int h_, int c0, int c1) {
    const int tid = afresh(threadIdx.x), lane = tid & 63;
    wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    k = reinterpret_cast<const char*>(a->cache.k);
    v = reinterpret_cast<const char*>(a->cache.v);
    scales = (lane & 16 ? a->cache.v_scale : a->cache.k_scale) + (lane & 15) * kKv4Blocks;
    table = a->p.page_table + (size_t)b * a->p.max_pages;
    from = code_at(lane >> 2, lane & 3);
    first_page = c0 / D2SD_PAGE_SIZE + wave;
    last_page = (c1 - 1) / D2SD_PAGE_SIZE;
    num_pages = a->p.num_pages;
    hkv = a->p.hkv;
    h = h_;
  }
  // ids: lane t % 64 holds the wave's pages of tile t (past the end: the last one)
  __device__ __forceinline__ void start(int t, char* ring, int (&ids)[2]) const {
    const int lane = threadIdx.x & 63;
    if ((t & (kWave - 1)) == 0) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int id = table[min(first_page + Tile::PAGES * (t + lane) + 4 * i, last_page)];
        ids[i] = clampi(id, 0, num_pages - 1) * hkv + h;
      }
    }
    const uint32_t stage = __builtin_amdgcn_readfirstlane(lds_addr(ring) + (uint32_t)t % kStages * Tile::BYTES);
    const size_t page[2] = {(uint32_t)lane_of(ids[0], t & (kWave - 1)), (uint32_t)lane_of(ids[1], t & (kWave - 1))};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t to = stage + (wave + 4 * i) * kKv4PageBytes;
      dma16s(k + page[i] * kKv4PageBytes, from, to);
      dma16s(v + page[i] * kKv4PageBytes, from, to + Tile::V);
    }
    dma4(scales + (lane & 32 ? page[1] : page[0]) * (D2SD_PAGE_SIZE * kKv4Blocks), stage + Tile::S + wave * 256);
  }
};

template <typename T>
__global__ __launch_bounds__(4 * kWave) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 4 ? 1 : 2))) void kv4_attention_kernel(Kv4Params kp) {
  constexpr int NP = kTerms<T>, NQ = kQueryTerms<T>;
  const Params& p = kp.p;
  __shared__ __attribute__((aligned(1024))) char ring[kStages * Tile::BYTES];
  __shared__ float s_m[4][kWave], s_l[4][kWave];
  __shared__ int s_len[4][3][kWave];
  __shared__ int s_flag;

  // consecutive shares on one XCD: the row groups of a KV head meet in its L2
  const int wg = (blockIdx.x % 8) * (kp.grid / 8) + blockIdx.x / 8;
  const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // ---- this workgroup's share: every wave finds it by itself ----
  // The lengths of 64 requests at a time: in the lanes, and in LDS for the walk.
  auto units_of = [&](int b0) {
    int u = 0;
    if (b0 + lane < p.batch) {
      const Lengths n = lengths_of(kp, b0 + lane);
      u = plan_of(kp, n).head * p.hkv;
      s_len[wave][0][lane] = n.base;
      s_len[wave][1][lane] = n.nodes;
      s_len[wave][2][lane] = n.ctx;
    }
    __builtin_amdgcn_wave_barrier();                  // other lanes read them
    return u;
  };
  auto plan_in_lds = [&](int i) {
    const Lengths n = {__builtin_amdgcn_readfirstlane(s_len[wave][0][i]), __builtin_amdgcn_readfirstlane(s_len[wave][1][i]),
                       __builtin_amdgcn_readfirstlane(s_len[wave][2][i])};
    return plan_of(kp, n);
  };
  long long W = 0;
  int units = 0;
  for (int b0 = (p.batch - 1) / kWave * kWave; b0 >= 0; b0 -= kWave) {
    units = units_of(b0);
    W += lane_of(wave_scan<false>(units), kWave - 1);
  }
  if (kp.cut && tid == 0) kp.cut[wg].pieces = 0;
  // no share is smaller than a step: none is empty, and a stream's pieces are consecutive workgroups
  const int grid = (int)min((long long)kp.grid, max(W / kp.most, min(W, 1ll)));
  if (wg >= grid) return;
  const Shares shares(W, grid);
  long long pos = shares.start(wg);
  const long long end = shares.start(wg + 1);
  int b = 0;
  long long at = 0;                                   // units before request b
  for (;;) {
    const int incl = wave_scan<false>(units);
    const uint64_t after = __ballot(b + lane < p.batch && at + incl > pos);
    if (after) {
      const int first = __ffsll((long long)after) - 1;
      b += first;
      at += lane_of(incl, first) - lane_of(units, first);
      break;
    }
    at += lane_of(incl, kWave - 1);
    b += kWave;
    units = units_of(b);
  }
  RequestPlan rq = plan_in_lds(b % kWave);

  while (pos < end) {
    while (rq.head * (long long)p.hkv <= pos - at) {  // on to the request that holds pos
      at += rq.head * (long long)p.hkv;
      if (++b % kWave == 0) units_of(b);
      rq = plan_in_lds(b % kWave);
    }
    // the KV head and the group of pos, the group's first unit and the cost of its steps
    const int h = (int)(pos - at) / rq.head, in_head = (int)(pos - at) % rq.head;
    const int fours = rq.tiles >> 2, four = kp.whole ? 1 : (rq.steps + kp.charge[2]) * kv4_cost(4);
    int rg, before;
    if (in_head < fours * four) {
      rg = in_head / four;
      before = rg * four;
    } else {
      const int two = rq.tiles & 2 ? kp.whole ? 1 : (rq.steps + kp.charge[1]) * kv4_cost(2) : 0;
      const bool past = in_head >= fours * four + two;
      rg = fours + (past && two ? 1 : 0);
      before = fours * four + (past ? two : 0);
    }
    const Group group = group_of(rq.tiles, rg);
    const int R = group.R, cost = kp.whole ? 1 : kv4_cost(R), pre = rq.pre + charge_of(kp, R), steps = rq.steps + charge_of(kp, R);
    const long long begin = at + (long long)h * rq.head + before, beyond = begin + (long long)steps * cost;
    const int u0 = ((int)(pos - begin) + cost - 1) / cost;
    const int u1 = end >= beyond ? steps : ((int)(end - begin) + cost - 1) / cost;
    const bool cut = u1 - u0 < steps;
    pos = min(end, beyond);
    if (u0 >= u1) continue;                           // the rest of a step that another workgroup does
    if (u0 > 0 && tid == 0 && kp.cut) {              // a second piece: the merge starts from here
      if (begin >= shares.start(wg - 1)) {
        const int r0 = group.first * kRowsPerTile;
        kp.cut[wg].rows = make_int4(rq.base, h, r0, min(rq.nodes * p.G - r0, R * kRowsPerTile));
        kp.cut[wg].pieces = shares.holder(beyond - cost, wg) - wg + 2;
      }
    }

    // R waves hold a row tile each, PH waves share the keys of a step
    const int rt = wave & (R - 1), ph = wave / R, PH = 4 / R;
    const int Nb = rq.nodes, node_base = rq.base;
    const int r_lo = group.first * kRowsPerTile;
    const int r_hi = min(Nb * p.G, r_lo + R * kRowsPerTile);
    const int r = r_lo + rt * kRowsPerTile + (lane & 31);
    const bool valid = r < r_hi;
    const int node = valid ? r / p.G : 0;
    const int qrow = valid ? (node_base + node) * p.hq + h * p.G + r % p.G : -1;
    const int t0 = kp.whole ? 0 : max(0, u0 - pre), t1 = kp.whole ? ceil_div(rq.ctx, kKeys) : max(0, u1 - pre);   // context tiles
    const int c0 = t0 * kKeys, c1 = min(rq.ctx, t1 * kKeys);

    // the first tiles start on their way
    const int n_tiles = ceil_div(c1 - c0, kKeys);
    int ids[2] = {0, 0};
    if (n_tiles > 0) {
      Copies copies(args_afresh(), b, h, c0, c1);
      for (int t = 0; t < min(n_tiles, kStages - 1); ++t) copies.start(t, ring, ids);
    }

    f32x16 o[4];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) o[dt] = f32x16{};
    float m_run = -INFINITY, l_run = 0.0f;

    // ---- the tree's keys: the waves of the first phase. Their values go through the ring's last stage ----
    char* const tree_v = ring + (kStages - 1) * Tile::BYTES;
    static_assert(64 * kRowBytes <= Tile::BYTES, "64 values of the tree");
    if (u0 == 0 && p.stage != D2SD_STAGE_PREFIX) {
      const ArgPtr a = args_afresh();
      const int tid = afresh(threadIdx.x), lane = tid & 63, hf = lane >> 5;
      const T* kt = static_cast<const T*>(a->p.k_tree);
      const T* vt = static_cast<const T*>(a->p.v_tree);
      const T* q_ptr = valid ? static_cast<const T*>(a->p.q) + (size_t)qrow * kD : nullptr;
      const ReadV rv = read_v(lane);
      const int hkv = a->p.hkv, mask_words = a->p.mask_words;
      const float c2 = a->p.c2;
      const bool mine = ph == 0;
      constexpr int kSteps = 4;    // of 16 dims at a time
      for (int key0 = 0; key0 < Nb; key0 += 64) {
        const int nvalid = min(64, Nb - key0);
        const size_t row0 = (size_t)(node_base + key0) * hkv + h;
        // all loads first: one trip to memory for the whole step
        constexpr int kVRows = 4;                     // of V per thread, eight dims each
        Raw8<T> rv8[kVRows];
#pragma unroll
        for (int u = 0; u < kVRows; ++u) {
          const int i = u * kThr + tid, row = i / (kD / 8);
          rv8[u] = Raw8<T>{};
          if (row < nvalid) rv8[u] = load8(vt + (row0 + (size_t)row * hkv) * kD + 8 * (i % (kD / 8)));
        }
        f32x16 s[2];
        uint64_t vis = 0;
        bf16x8 pf[2][NP][2];
        if (mine) {
          const uint32_t* mrow = a->p.anc_mask + (size_t)(node_base + node) * mask_words;
          const int w0 = key0 >> 5;
          vis = (uint64_t)mrow[w0] | (w0 + 1 < mask_words ? (uint64_t)mrow[w0 + 1] << 32 : 0ull);
          s[0] = f32x16{};
          s[1] = f32x16{};
#pragma unroll
          for (int half = 0; half < 8; half += kSteps) {
            Raw8<T> rq8[kSteps], rk8[2][kSteps];
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {        // dims 64 hf + 8 (half + i) .. + 8
              const int d = 64 * hf + 8 * (half + i);
              rq8[i] = Raw8<T>{};
              if (q_ptr) rq8[i] = load8(q_ptr + d);
#pragma unroll
              for (int kb = 0; kb < 2; ++kb)
                rk8[kb][i] = load8(kt + (row0 + (size_t)min(32 * kb + (lane & 31), nvalid - 1) * hkv) * kD + d);
            }
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
              float v[8];
              unpack8(rq8[i], v);
              bf16x8 tq[NP];
              split_bf16<NP, true>(v, tq);
#pragma unroll
              for (int kb = 0; kb < 2; ++kb) {
                unpack8(rk8[kb][i], v);
                bf16x8 tk[NP];
                split_bf16<NP, true>(v, tk);
#pragma unroll
                for (int x = NP - 1; x >= 0; --x)     // products below the last term are left out
#pragma unroll
                  for (int y = NP - 1 - x; y >= 0; --y) s[kb] = mfma(tk[x], tq[y], s[kb]);
              }
            }
          }
          if (!valid) vis = 0;
          if (nvalid < 64) vis &= (1ull << nvalid) - 1ull;
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) s[kb] *= c2;
          mask_scores<2>(s, vis, hf);
          move_reference(max_score<2>(s), m_run, l_run, o);
          const float m0 = m_run == -INFINITY ? 0.0f : m_run;
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) {
            s[kb] -= m0;
            l_run += weigh(s[kb]);
            split_weights<NP>(s[kb], pf[kb]);
          }
        }
        if (tid == 0) s_flag = 0;
        lds_barrier();
#pragma unroll
        for (int n = 0; n < NP; ++n) {                // planes of V
#pragma unroll
          for (int u = 0; u < kVRows; ++u) {
            const int i = u * kThr + tid, row = i / (kD / 8), c = i % (kD / 8);
            float v[8];
            unpack8(rv8[u], v);
            bool wild = false;
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if ((__float_as_uint(v[j]) & 0x7f800000u) == 0x7f800000u) {
                wild = true;
                v[j] = 0.0f;
              }
            if (wild) s_flag = 1;
            bf16x8 t[NP];
            split_bf16<NP, true>(v, t);
            *reinterpret_cast<bf16x8*>(tree_v + chunk_at(row, c)) = t[n];
          }
          lds_barrier();
          if (mine) {
            // plane n by the terms of P that are not below the last one
            typedef bf16x8 Term[1][2];
#pragma unroll
            for (int j = NP - 1 - n; j >= 0; --j)
#pragma unroll
              for (int kb = 0; kb < 2; ++kb) pv_tile<1, 2>(tree_v + kb * 32 * kRowBytes, rv, reinterpret_cast<const Term&>(pf[kb][j]), o);
          }
          if (n == NP - 1 && s_flag && mine) {
            // an infinite or NaN value: added where its node is seen (a weight of 0 would spread it to all)
            for (int k = 0; k < nvalid; ++k) {
              if (!((vis >> k) & 1ull)) continue;
              const T* vr = vt + (row0 + (size_t)k * hkv) * kD;
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
      const ArgPtr a = args_afresh();
      const int tid = afresh(threadIdx.x), lane = tid & 63, hf = lane >> 5;
      const T* q_ptr = valid ? static_cast<const T*>(a->p.q) + (size_t)qrow * kD : nullptr;
      const float c2 = a->p.c2;
      Copies copies(a, b, h, c0, c1);
      Query<NQ> q;
      // bf16 queries stay as they are, so that four terms hold them, and their scores are scaled
      constexpr bool kScaled = sizeof(T) == 4;
      load_query<T, NQ>(q, q_ptr, hf, kScaled ? c2 : 1.0f);
      sync_keep<0>();
      const int k_at0 = code_at(lane & 31, hf), k_at1 = code_at(lane & 31, 2 + hf);
      // halves of the identity: 1.0 (code 2) at dim lane % 32 of the first or of the second 32 dims
      uint4 unit[2];
      {
        const int n = lane & 31;
        const uint32_t one = 2u << (4 * (n & 7));
        const uint4 e = make_uint4(n < 8 ? one : 0u, n >> 3 == 1 ? one : 0u, n >> 3 == 2 ? one : 0u, n >> 3 == 3 ? one : 0u);
        unit[0] = hf ? zero4() : e;
        unit[1] = hf ? e : zero4();
      }
      f32x16 less = {};                                // -m in all slots: the initial value of scaled scores
      if (m_run != -INFINITY) less -= m_run;
      // One tile; `steady`: the next one is whole and there is one to copy.
      auto step = [&](int j, auto steady) {
        if (steady.value || j + kStages - 1 < n_tiles) copies.start(j + kStages - 1, ring, ids);
        {
          const char* stage = ring + (uint32_t)j % kStages * Tile::BYTES;
#pragma unroll 1
          for (int kb = ph; kb < kKeys / 32; kb += PH) {   // its blocks of 32 keys
            const int nvalid = steady.value ? 32 : c1 - (c0 + j * kKeys) - 32 * kb;
            if (!steady.value && nvalid <= 0) break;
            const char* blk = stage + kb * 32 * kKv4RowBytes;
            const char* scales = stage + scale_at(32 * kb + (lane & 31));
            const uint4 k0 = *reinterpret_cast<const uint4*>(blk + k_at0);
            const uint4 k1 = *reinterpret_cast<const uint4*>(blk + k_at1);
            const uint32_t sk = *reinterpret_cast<const uint32_t*>(scales) >> (8 * hf);
            uint4 v[2] = {*reinterpret_cast<const uint4*>(blk + Tile::V + k_at0), *reinterpret_cast<const uint4*>(blk + Tile::V + k_at1)};
            uint32_t vw = *reinterpret_cast<const uint32_t*>(scales + 64) >> (8 * hf);
            if (!steady.value && (lane & 31) >= nvalid) {   // a key past the context: its values are zeros
              v[0] = v[1] = zero4();
              vw = 0x007f007fu;
            }
            // the half that a product leaves out must not be NaN
            const uint32_t vs[2] = {hf ? 0x007f007fu : vw, hf ? vw : 0x007f007fu};
            auto scores = [&](const f32x16& from) {
              f32x16 x = from;
#pragma unroll
              for (int n = NQ - 1; n >= 0; --n) {      // the small terms first
                x = mfma_kq<0, 0>(k0, q.d[n][0], x, sk, q.s[n]);
                x = mfma_kq<2, 1>(k1, q.d[n][1], x, sk, q.s[n]);
              }
              if constexpr (!steady.value) {
                f32x16 y[1] = {x};
                if (nvalid < 32) mask_scores<1>(y, (1ull << nvalid) - 1ull, hf);
                x = y[0];
              }
              return x;
            };
            f32x16 x = scores(kScaled ? less : f32x16{}), s = x;
            if constexpr (!kScaled) s = ahead(x, c2, less[0]);
            float l = weigh(s);
            if (__ballot(!(l <= kMostWeight)) || (!steady.value && j == 0 && kb == ph)) {
              f32x16 y[1] = {kScaled ? scores(f32x16{}) : x * c2};
              move_reference(max_score<1>(y), m_run, l_run, o);
              const float m0 = m_run == -INFINITY ? 0.0f : m_run;
              less = f32x16{} - m0;
              s = kScaled ? y[0] - m0 : ahead(x, c2, -m0);
              l = weigh(s);
            }
            l_run += l;
            bf16x8 pf[NP][2];
            split_weights<NP>(s, pf);
            // O^T += V^T P^T: a transposed tile has its keys in the order of the weights
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) {
              const f32x16 x = dt < 2 ? mfma_vt<0>(v[0], unit[dt & 1], vs[dt & 1]) : mfma_vt<2>(v[1], unit[dt & 1], vs[dt & 1]);
#pragma unroll
              for (int t = 0; t < 2; ++t) {
                bf16x8 va;
#pragma unroll
                for (int i = 0; i < 8; ++i) va[i] = (__bf16)x[8 * t + i];
#pragma unroll
                for (int n = NP - 1; n >= 0; --n) o[dt] = mfma(va, pf[n][t], o[dt]);
              }
            }
          }
        }
        // tile j + 1 has to be there: all copies but those of the last kStages - 2 steps
        if constexpr (steady.value) sync_keep<Tile::OPS*(kStages - 2)>();
        else sync_keep<0>();
      };
      // the first tile sets the references; a steady one copies tile j + kStages - 1
      step(0, std::false_type{});
      int j = 1;
      for (; j + kStages - 1 < n_tiles; ++j) step(j, std::true_type{});
      for (; j < n_tiles; ++j) step(j, std::false_type{});
    }

    // ---- the rows' state: to the output, or to a slot ----
    const ArgPtr a = args_afresh();
    l_run += __shfl_xor(l_run, 32);
    float weight = 1.0f, m_all = m_run, l_all = l_run;   // of this wave's part, and all parts' reference and sum
    // part: dims 32 dt .. + 32 of the rows' joined sums
    auto put = [&](int dt, f32x16 part) {
      if (!valid) return;
      if (!cut) {
        part *= l_all == 0.0f ? 0.0f : 1.0f / l_all;
        T* dst = static_cast<T*>(a->p.out) + (size_t)qrow * kD + dt * 32 + hf * 4;
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const float v[4] = {part[q4 * 4], part[q4 * 4 + 1], part[q4 * 4 + 2], part[q4 * 4 + 3]};
          store_out<T>(dst + q4 * 8, v);
        }
        if (a->p.lse && dt == 0 && hf == 0) a->p.lse[qrow] = l_all == 0.0f ? -INFINITY : (m_all + __log2f(l_all)) * kLn2;
      } else {
        const size_t slot = (size_t)(2 * wg + (u0 == 0)) * a->p.slot_rows + (r - r_lo);
        float* dst = static_cast<float*>(a->p.ws_o) + slot * kD + dt * 32 + hf * 4;
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          *reinterpret_cast<float4*>(dst + q4 * 8) = make_float4(part[q4 * 4], part[q4 * 4 + 1], part[q4 * 4 + 2], part[q4 * 4 + 3]);
        if (dt == 0 && hf == 0) {
          a->p.ws_m[slot] = m_all;
          a->p.ws_l[slot] = l_all;
        }
      }
    };
    if (PH == 1) {
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) put(dt, o[dt]);
    } else {
      // join the phases: every wave leaves its sums, scaled to the largest
      // reference, and takes 4 / PH quarters of the dims from all of them
      s_m[wave][lane] = m_run;
      s_l[wave][lane] = l_run;
      lds_barrier();
      for (int w = rt; w < 4; w += R) m_all = fmaxf(m_all, s_m[w][lane]);
      l_all = 0.0f;
      for (int w = rt; w < 4; w += R) l_all += s_l[w][lane] == 0.0f ? 0.0f : s_l[w][lane] * __builtin_amdgcn_exp2f(s_m[w][lane] - m_all);
      weight = m_run == -INFINITY && l_run == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(m_run - m_all);
      float* state = reinterpret_cast<float*>(ring);  // [4 waves][4 dt][4][64 lanes][4]
      static_assert(4 * 64 * kWave * sizeof(float) <= sizeof ring, "states of the four waves");
      auto place = [&](int w, int dt, int q4) { return reinterpret_cast<float4*>(state + (((w * 4 + dt) * 4 + q4) * kWave + lane) * 4); };
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          *place(wave, dt, q4) = make_float4(o[dt][4 * q4] * weight, o[dt][4 * q4 + 1] * weight, o[dt][4 * q4 + 2] * weight, o[dt][4 * q4 + 3] * weight);
      lds_barrier();
      for (int dt = ph * R; dt < ph * R + R; ++dt) {
        f32x16 part = {};
        for (int w = rt; w < 4; w += R)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const float4 v = *place(w, dt, q4);
            part[4 * q4] += v.x;
            part[4 * q4 + 1] += v.y;
            part[4 * q4 + 2] += v.z;
            part[4 * q4 + 3] += v.w;
          }
        put(dt, part);
      }
      lds_barrier();                                   // the ring is free for the next piece
    }
  }
}

// Joins the pieces of the streams that were cut. A workgroup looks through the
// entries of kp.span workgroups of the attention for second pieces, and takes
// kMergeRows / kp.per rows of each stream that it finds: 32 lanes fold four
// dims each of every kp.per-th piece of a row in order, and such sums are then
// joined in order through LDS. The host has span and per from the mean number
// of pieces, so that about one stream falls to a workgroup and a lane has
// few pieces in turn.
constexpr int kMergeRows = kThreads / 32;

template <typename T>
__global__ __launch_bounds__(kThreads) void kv4_merge_kernel(Kv4Params kp) {
  const Params& p = kp.p;
  __shared__ float s_o[kMergeRows][kD], s_ml[kMergeRows][2];
  const int per = kp.per, rows_here = kMergeRows / per, chunks = p.slot_rows / rows_here;
  const int i0 = (int)(blockIdx.x / chunks) * kp.span, lane = threadIdx.x & (kWave - 1);
  const int grp = threadIdx.x / 32, d0 = (threadIdx.x & 31) * 4;
  const int rr = (int)(blockIdx.x % chunks) * rows_here + grp / per;
  int pieces = 0;
  int4 of = make_int4(0, 0, 0, 0);
  if (lane < kp.span && i0 + lane < kp.grid) {
    pieces = kp.cut[i0 + lane].pieces;
    of = kp.cut[i0 + lane].rows;
  }
  for (uint64_t found = __ballot(pieces >= 2); found; found &= found - 1) {
    const int at = __ffsll((long long)found) - 1, i = i0 + at, n = lane_of(pieces, at);
    const int base = lane_of(of.x, at), h = lane_of(of.y, at), r_lo = lane_of(of.z, at), rows = lane_of(of.w, at);
    const bool there = rr < rows;
    float M = -INFINITY, L = 0.0f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    auto fold = [&](float m, float l, const float4& v) {
      const float Mn = fmaxf(M, m);
      const float a = M == -INFINITY && L == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(M - Mn);
      const float w = m == -INFINITY && l == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(m - Mn);
      L = L * a + w * l;
      acc[0] = acc[0] * a + w * v.x;
      acc[1] = acc[1] * a + w * v.y;
      acc[2] = acc[2] * a + w * v.z;
      acc[3] = acc[3] * a + w * v.w;
      M = Mn;
    };
    if (there) {
#pragma unroll 4
      for (int k = grp % per; k < n; k += per) {
        const size_t slot = (size_t)(k == 0 ? 2 * (i - 1) + 1 : 2 * (i - 1 + k)) * p.slot_rows + rr;
        fold(p.ws_m[slot], p.ws_l[slot], *reinterpret_cast<const float4*>(static_cast<const float*>(p.ws_o) + slot * kD + d0));
      }
    }
    if (per > 1) {
      __syncthreads();
      *reinterpret_cast<float4*>(&s_o[grp][d0]) = make_float4(acc[0], acc[1], acc[2], acc[3]);
      if (d0 == 0) {
        s_ml[grp][0] = M;
        s_ml[grp][1] = L;
      }
      __syncthreads();
      if (grp % per == 0)
        for (int g = grp + 1; g < grp + per; ++g) fold(s_ml[g][0], s_ml[g][1], *reinterpret_cast<const float4*>(&s_o[g][d0]));
    }
    if (!there || grp % per) continue;
    const int r = r_lo + rr;
    const size_t row = (size_t)(base + r / p.G) * p.hq + h * p.G + r % p.G;
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] *= inv;
    store_out<T>(static_cast<T*>(p.out) + row * kD + d0, acc);
    if (p.lse && d0 == 0) p.lse[row] = L == 0.0f ? -INFINITY : (M + __log2f(L)) * kLn2;
  }
}

}  // namespace

hipError_t launch_kv4_attention(const d2sd_attn_args& a, const d2sd_kv4_cache& cache, const Kv4Plan& plan, void* ws,
                                hipStream_t stream, hipEvent_t (&ev)[3]) {
  Params p{};
  p.q = a.q; p.page_table = a.page_table; p.ctx_len = a.ctx_len; p.k_tree = a.k_tree; p.v_tree = a.v_tree;
  p.node_indptr = a.node_indptr; p.anc_mask = a.anc_mask; p.out = a.out; p.lse = a.lse;
  // slots: outputs, m, l; then the list of cut streams
  const size_t states = (size_t)2 * plan.grid * plan.slot_rows;
  p.ws_o = ws;
  p.ws_m = ws ? static_cast<float*>(ws) + states * kD : nullptr;
  p.ws_l = ws ? p.ws_m + states : nullptr;
  p.slot_rows = plan.slot_rows;
  p.batch = a.batch; p.hq = a.num_qo_heads; p.hkv = a.num_kv_heads; p.G = a.num_qo_heads / a.num_kv_heads;
  p.stage = a.stage; p.total_nodes = a.total_nodes; p.max_nodes = a.max_nodes; p.max_ctx = a.max_ctx_len;
  p.num_pages = a.num_pages; p.max_pages = a.max_pages; p.mask_words = a.mask_words;
  p.c2 = plan.scale * kLog2e;
  const Kv4Params kp{p, cache, plan.grid, plan.whole, plan.most, {plan.charge[0], plan.charge[1], plan.charge[2]}, plan.span, plan.per, ws && !plan.whole ? reinterpret_cast<CutStream*>(p.ws_l + states) : nullptr};
  const dim3 grid((unsigned)plan.grid), mgrid((unsigned)((plan.grid + plan.span - 1) / plan.span * (plan.slot_rows * plan.per / kMergeRows)));
  hipError_t e = hipSuccess;
  auto launch = [&](auto kernel, auto merge) {
    if (ev[0]) (void)hipEventRecord(ev[0], stream);
    hipLaunchKernelGGL(kernel, grid, dim3(4 * kWave), 0, stream, kp);
    e = hipGetLastError();
    if (e != hipSuccess) return;
    if (ev[1]) (void)hipEventRecord(ev[1], stream);
    if (plan.whole) return;
    hipLaunchKernelGGL(merge, mgrid, dim3(kThreads), 0, stream, kp);
    e = hipGetLastError();
    if (ev[2]) (void)hipEventRecord(ev[2], stream);
  };
  if (a.dtype == D2SD_BF16) launch(kv4_attention_kernel<__bf16>, kv4_merge_kernel<__bf16>);
  else launch(kv4_attention_kernel<float>, kv4_merge_kernel<float>);
  return e;
}

}  // namespace d2sd
