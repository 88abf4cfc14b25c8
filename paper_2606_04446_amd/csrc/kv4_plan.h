// Plan of a verify attention over a 4-bit cache (host side) and its launcher.
#pragma once

#include "common.h"

namespace d2sd {

constexpr size_t kKv4CutBytes = 32;   // of an entry of the list of cut streams

struct Kv4Plan {
  int grid;          // workgroups, a multiple of 8
  int whole;         // no stream is cut: no partial states, no merge
  int most;          // cost of the largest group's step (1 when whole)
  int charge[3];     // steps that a stream of 1, 2 or 4 row tiles counts beside those of its keys
  int span, per;     // the merge: entries per workgroup (up to 64), lanes' groups per row (1, 4 or 8)
  int slot_rows;     // rows of a partial state's slot
  size_t ws_bytes;   // slots and the list of cut streams (0 when whole)
  float scale;       // softmax scale
};

// Cost of a step (128 keys) for a workgroup that holds 1, 2 or 4 row tiles, and
// of a step for all `tiles` row tiles of a KV head (four at a time, then two,
// then one). The matrix cores' part is proportional to the tiles, that of copies
// and barriers is not; 32 requests of 16384 keys and up to 14 tiles take 863 us
// with 8 : 5 : 3, 872 with 8 : 4 : 2 and 874 with 18 : 9 : 5.
__host__ __device__ inline int kv4_cost(int tiles) { return 8 * (tiles >> 2) + (tiles & 2 ? 5 : 0) + (tiles & 1 ? 3 : 0); }

hipError_t launch_kv4_attention(const d2sd_attn_args& a, const d2sd_kv4_cache& cache, const Kv4Plan& plan, void* ws,
                                hipStream_t stream, hipEvent_t (&ev)[3]);

}  // namespace d2sd
