// Host-side helpers shared by the files that implement the C ABI.
#pragma once

#include "common.h"

namespace d2sd {

// Records the calling thread's error message and returns s.
d2sd_status fail(d2sd_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
// Clears the message.
d2sd_status ok();
d2sd_status hip_status(hipError_t e, const char* what);

// Sizes, head counts, stage and node_indptr_host of an attention call; with
// pointers, also that the device pointers are there and 16-byte aligned.
d2sd_status validate_attn(const d2sd_attn_args* a, bool pointers);

// Events around an attention call's main kernel and its merge when kernel
// timing is on (else null): to be recorded before, between and after.
void timing_begin(hipEvent_t (&ev)[3]);
void timing_end(hipEvent_t (&ev)[3], bool launched, bool merged);

// Largest tree any entry point accepts: the canonical tree of B = D2SD_MAX_B
// with every re-anchor position (the accept kernel stages one tree in LDS).
constexpr int kMaxTreeNodes = D2SD_MAX_B + D2SD_MAX_B * (D2SD_MAX_B - 1) / 2;

}  // namespace d2sd
