// What the files of the C-ABI layer share: argument checks and error reports (host only).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/kvev.h"

namespace kvev {

int hip_fail(hipError_t e);                                   // keeps the error's text for kvev_last_hip_error
int check_shape(const kvev_shape *sh, bool chunked = true);   // 0 when the shape itself is usable, else a status
int device_compute_units();                                   // of the current device
size_t attn_stream_bytes();                                   // launches that read more take their rows with the non-temporal hint

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
// key-value heads: the caches, summaries, gate state and kept sets exist per (layer, batch row, KV head)
inline int kv_heads(const kvev_shape *sh) { return sh->H_kv > 0 ? sh->H_kv : sh->H; }

}  // namespace kvev
