// Plan of a verify attention over a 4-bit cache (host side) and its launcher.
#pragma once

#include "common.h"

namespace d2sd {

constexpr int kKv4MaxSplit = 32768;   // context tokens per split: its page ids are staged in LDS

struct Kv4Plan {
  int waves;         // waves of 32 query rows per workgroup: 1, 2, 4 or 8
  int split;         // context tokens per split (multiple of 64)
  int n_ch_max;      // splits of the longest context (>= 1)
  int n_rg_max;      // row groups of the largest request (>= 1)
  long long items;   // batch * hkv * n_ch_max * n_rg_max
  size_t ws_bytes;   // partial states (0 for one split)
  float scale;       // softmax scale
};

hipError_t launch_kv4_attention(const d2sd_attn_args& a, const d2sd_kv4_cache& cache, const Kv4Plan& plan, void* ws,
                                hipStream_t stream);

}  // namespace d2sd
